"""What stands around the linear layer on 8-bit rows, as cases that can be timed and checked.

Six operators: the root-mean-square norm with the residual's addition, whose
output is the 8-bit rows that the layer's products read, and its gradient; the
projection by 4-bit weights with a scale for each group of channels, and its
gradient with respect to the input; the products of rows sorted by expert with
each expert's weights, and both of their gradients.

A case is a dict of plain values.  `prepare` makes what a program holds before
the call, `run` makes one pass: with `own` false in elementary torch operations
in 32 bits (64 for the norm's values, which are rounded to codes), with `own`
true through the package's entry points.  `exact` computes the same outputs in
64 bits from the definitions.

Values: activations are normal with a few channels twenty times as wide, and
some rows are zero (padding tokens); gradients are normal with a spread of row
sizes and zero rows (tokens without a loss); weights are normal; experts get
very different numbers of rows, some none.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-5


# ------------------------------------------------------------------ the cases

def _norm(name, m, c, dtype, residual, stride=0):
    """Norm of m rows of c channels; stride: elements from row to row of x (0: c)."""
    return dict(name=name, op="norm", m=m, c=c, dtype=dtype, residual=residual, stride=stride or c)


def _norm_grad(name, m, c, dtype, residual, stride=0):
    """Its gradient; residual: a gradient arrives at the sum as well; stride: between dy's rows."""
    return dict(name=name, op="norm_grad", m=m, c=c, dtype=dtype, residual=residual, stride=stride or c)


def _groups(name, op, m, c, k, group, scales, dtype):
    """m rows through k x c 4-bit weights with scales (of type `scales`) for each `group` channels."""
    return dict(name=name, op=op, m=m, c=c, k=k, group=group, scales=scales, dtype=dtype)


def _experts(name, op, m, experts, c, k, bits, dtype, group=0, scales="f32"):
    """m rows in all for some of the experts, of k x c weights each; group: 0 for one scale a row."""
    return dict(name=name, op=op, m=m, experts=experts, c=c, k=k, bits=bits, group=group, scales=scales, dtype=dtype)


def listed():
    return [
        # between two layers of one decoding step, a few requests: latency
        _norm("norm_m16_c4096_bf16", 16, 4096, "bf16", True),
        # the same of a training batch: memory
        _norm("norm_m8192_c4096_bf16", 8192, 4096, "bf16", True),
        # the training batch's backward pass, the residual's gradient added
        _norm_grad("norm_grad_m8192_c4096_bf16", 8192, 4096, "bf16", True),
        # a last norm without a residual, of an odd width, the gradient a slice of a wider matrix
        _norm_grad("norm_grad_m1021_c5003_f16_strided", 1021, 5003, "f16", False, stride=5050),
        # one token of one request: latency, the weights' bytes
        _groups("groups_m1_c4096_k8192_g128", "groups", 1, 4096, 8192, 128, "f16", "bf16"),
        # a prompt through weights of odd sizes, the last group short
        _groups("groups_m1543_c2824_k5003_g32", "groups", 1543, 2824, 5003, 32, "bf16", "f16"),
        # adapters trained through frozen weights: the gradient of a batch
        _groups("groups_grad_m4096_c4096_k4096_g128", "groups_grad", 4096, 4096, 4096, 128, "f16", "bf16"),
        # a short batch, odd output channels
        _groups("groups_grad_m333_c2824_k1001_g64", "groups_grad", 333, 2824, 1001, 64, "f32", "f16"),
        # one decoding step of 16 requests on two experts each, many experts
        _experts("experts_m32_e64_c2048_k4096_w4_g128", "experts", 32, 64, 2048, 4096, 4, "bf16", 128, "f16"),
        # the forward pass of a training batch, two experts a token
        _experts("experts_m16384_e8_c4096_k4096_w8", "experts", 16384, 8, 4096, 4096, 8, "bf16"),
        # both gradients of that batch
        _experts("experts_grad_m16384_e8_c4096_k4096_w8", "experts_grad", 16384, 8, 4096, 4096, 8, "bf16"),
        # both of a short batch on many small experts of odd sizes
        _experts("experts_grad_m1999_e24_c1411_k1003_w8", "experts_grad", 1999, 24, 1411, 1003, 8, "f16"),
    ]


LARGEST_FLOPS = 1.1e12       # both gradients of the training batch
LARGEST_BYTES = 8e8


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A width between lo and hi: one usual for layers, a multiple of 8, or any."""
    kind = rng.choice(("usual", "usual", "eights", "any"))
    if kind == "usual":
        return rng.choice([w for w in (256, 384, 512, 768, 1024, 1280, 1536, 2048, 2560, 4096, 5120, 6144, 8192)
                           if lo <= w <= hi])
    n = _log(rng, lo, hi)
    return n if kind == "any" else max(lo, n // 8 * 8)


def draw(rng):
    """One more case of these ranges: any operator, sizes over their whole range."""
    while True:
        op = rng.choice(("norm", "norm_grad", "groups", "groups", "groups_grad", "experts", "experts", "experts_grad"))
        dtype = rng.choice(("bf16", "bf16", "f16"))
        c, k = _size(rng, 256, 8192), _size(rng, 256, 8192)
        eights = max(256, c // 8 * 8)
        if op in ("norm", "norm_grad"):
            dtype = rng.choice(("bf16", "f16", "f32"))
            case = dict(op=op, m=_log(rng, 1, 16384), c=c, dtype=dtype, residual=rng.random() < 0.6,
                        stride=c + rng.choice((0, 0, 8, 47)))
        elif op in ("groups", "groups_grad"):
            case = dict(op=op, m=_log(rng, 1, 8192), c=eights, k=k, group=rng.choice((32, 64, 128, 128)),
                        scales=rng.choice(("f16", "bf16", "f32")), dtype=dtype)
        else:
            bits = rng.choice((4, 8))
            case = dict(op=op, m=_log(rng, 1, 16384), experts=_log(rng, 2, 96), c=eights if bits == 4 else c, k=k,
                        bits=bits, group=rng.choice((0, 32, 64, 128)) if bits == 4 else 0,
                        scales=rng.choice(("f16", "bf16", "f32")), dtype=dtype)
        w = work(case)
        weights = case.get("experts", 1) * case.get("k", 0) * c
        if w["flops"] <= LARGEST_FLOPS and w["bytes"] <= LARGEST_BYTES and weights <= 3e8 and (w["bytes"] > 1e5 or op == "norm"):
            return case


# ------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _padding(g, m):
    """About one row in fifty is zero where there are many."""
    return (torch.rand(m, 1, generator=g, device="cuda") > (0.02 if m > 16 else 0.0)).float()


def _activations(g, m, c):
    wide = (torch.rand(c, generator=g, device="cuda") < 0.004).float() * 19.0 + 1.0
    return _normal(g, m, c) * wide * _padding(g, m)


def _gradients(g, m, k):
    return _normal(g, m, k) * torch.exp(_normal(g, m, 1)) * 0.01 * _padding(g, m)


def _wide_buffer(x, stride):
    """x as the first columns of a wider matrix, whose other columns hold something else."""
    buf = torch.full((x.shape[0], stride), 3.0, dtype=x.dtype, device=x.device)
    buf[:, :x.shape[1]] = x
    return buf[:, :x.shape[1]]


def _rows8(x):
    """int8 codes (rows of whole 16-byte vectors) and power-of-two row scales of a float32 matrix."""
    m, c = x.shape
    amax = x.abs().amax(1)
    e = torch.ceil(torch.log2(amax.double() / 127.0)).float()
    scale = torch.where(amax > 0, torch.exp2(e), torch.zeros_like(e))
    codes = torch.zeros((m, -(-c // 16) * 16), dtype=torch.int8, device=x.device)
    codes[:, :c] = torch.round(x / torch.exp2(e)[:, None]).nan_to_num(0.0).clamp(-127.0, 127.0).to(torch.int8)
    return codes, scale


def _words4(q):
    """Signed 4-bit values, eight to a 32-bit word (channel 8j+i in bits 4i..4i+3), zero-filled to 16-byte vectors."""
    m, c = q.shape
    words = torch.zeros((m, -(-c // 32) * 4), dtype=torch.int32, device=q.device)
    nibbles = torch.nn.functional.pad(q.to(torch.int32) & 15, (0, words.shape[1] * 8 - c)).reshape(m, -1, 8)
    for i in range(8):
        words |= nibbles[:, :, i] << (4 * i)
    return words


def _rows4(w, group, scales):
    """4-bit words and scales: one a row (group 0, 32 bits), or one for each group of channels."""
    k, c = w.shape
    if not group:
        scale = w.abs().amax(1) / 7.5
        return _words4(torch.round(w / scale[:, None]).clamp(-8, 7)), scale
    groups = -(-c // group)
    v = torch.nn.functional.pad(w, (0, groups * group - c)).reshape(k, groups, group)
    scale = (v.abs().amax(2) / 7.5).to(DTYPES[scales])
    q = torch.round(v / scale.float()[:, :, None]).nan_to_num(0.0).clamp(-8, 7).reshape(k, -1)[:, :c]
    return _words4(q), scale


def _weights(g, case):
    """Codes and scales of the weights, of every expert one below the other."""
    k, c = case["k"], case["c"]
    parts = []
    for _ in range(case.get("experts", 1)):
        w = _normal(g, k, c) * c ** -0.5
        parts.append(_rows8(w) if case.get("bits", 4) == 8 else _rows4(w, case["group"], case["scales"]))
    return torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])


def _counts(case):
    """Rows of each expert, in falling order: shares spread by a factor of about ten, and chance."""
    rng = random.Random(case["m"] * 131 + case["experts"])
    shares = [math.exp(rng.gauss(0.0, 0.7)) for _ in range(case["experts"])]
    chosen = rng.choices(range(case["experts"]), weights=shares, k=case["m"])
    counts = [0] * case["experts"]
    for e in chosen:
        counts[e] += 1
    return sorted(counts, reverse=True)


def _offsets(g, case):
    """int32 first row of each expert, and the last one's end: which expert has which count is chance."""
    counts = torch.tensor(_counts(case), device="cuda")
    counts = counts[torch.randperm(case["experts"], generator=g, device="cuda")]
    return torch.nn.functional.pad(torch.cumsum(counts, 0), (1, 0)).to(torch.int32)


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    m, c, dtype = case["m"], case["c"], DTYPES[case["dtype"]]
    if op in ("norm", "norm_grad"):
        gain = (1.0 + 0.2 * _normal(g, c)).to(dtype)
        if op == "norm":
            x = _wide_buffer(_activations(g, m, c).to(dtype), case["stride"])
            return {"op": op, "x": x, "gain": gain, "residual": _activations(g, m, c).to(dtype) if case["residual"] else None}
        h = _activations(g, m, c).to(dtype)
        rstd = torch.rsqrt(h.double().square().mean(1) + EPS).float()
        return {"op": op, "dy": _wide_buffer(_gradients(g, m, c).to(dtype), case["stride"]), "h": h, "gain": gain,
                "rstd": rstd, "dsum": _gradients(g, m, c).to(dtype) if case["residual"] else None}
    w, w_scale = _weights(g, case)
    s = {"op": op, "c": c, "k": case["k"], "dtype": dtype, "w": w, "w_scale": w_scale, "bits": case.get("bits", 4),
         "group": case["group"], "offsets": _offsets(g, case) if "experts" in case else None}
    if op in ("groups", "experts", "experts_grad"):
        s["x"], s["x_scale"] = _rows8(_activations(g, m, c))
    if op in ("groups_grad", "experts_grad"):
        s["dy"] = _gradients(g, m, case["k"]).to(dtype)
    return s


# ------------------------------------------------------------------ a pass

def _values(codes, scale, c, bits=8, group=0):
    """The float32 values that codes and scales stand for."""
    if bits == 4:
        nibbles = (codes[..., None] >> (4 * torch.arange(8, device=codes.device, dtype=torch.int32))) & 15
        codes = (((nibbles + 8) & 15) - 8).reshape(codes.shape[0], -1)
    scale = scale.float()
    if group:
        return codes[:, :c].float() * scale[:, torch.arange(c, device=codes.device) // group]
    return codes[:, :c].float() * scale[:, None]


def _plain_norm(s):
    x = s["x"]
    h = x if s["residual"] is None else (x.float() + s["residual"].float()).to(x.dtype)
    wide = h.double()
    r = 1.0 / torch.sqrt((wide * wide).mean(1) + EPS)
    y = wide * r[:, None] * s["gain"].double()
    amax = y.abs().amax(1)
    mantissa, e = torch.frexp(amax)                           # amax = mantissa 2^e, 1/2 <= mantissa < 1
    e = torch.clamp(e - 7 + (mantissa > 127 / 128).to(e.dtype), min=-126)
    scale = torch.ldexp(torch.ones_like(amax), e)
    codes = torch.round(y / scale[:, None]).to(torch.int8)
    return codes, torch.where(amax > 0, scale, torch.zeros_like(scale)).float(), h, r.float()


def _plain_norm_grad(s):
    dy, h, r = s["dy"].float(), s["h"].float(), s["rstd"][:, None]
    t = dy * s["gain"].float()
    dx = r * t - h * (r * r * r * (t * h).mean(1, keepdim=True))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    return dx.to(s["h"].dtype), (dy * h * r).sum(0)


def _plain(s):
    op, c, k = s["op"], s.get("c"), s.get("k")
    if op == "norm":
        return _plain_norm(s)
    if op == "norm_grad":
        return _plain_norm_grad(s)
    if op == "groups":
        y = _values(s["x"], s["x_scale"], c) @ _values(s["w"], s["w_scale"], c, 4, s["group"]).t()
        return y.to(s["dtype"])
    if op == "groups_grad":
        return (s["dy"].float() @ _values(s["w"], s["w_scale"], c, 4, s["group"])).to(s["dtype"])
    ends = s["offsets"].tolist()
    outs = []
    for e in range(len(ends) - 1):
        rows, mine = slice(ends[e], ends[e + 1]), slice(e * k, e * k + k)
        if op == "experts":
            if ends[e] == ends[e + 1]:
                continue
            w = _values(s["w"][mine], s["w_scale"][mine], c, s["bits"], s["group"])
            outs.append((_values(s["x"][rows], s["x_scale"][rows], c) @ w.t()).to(s["dtype"]))
        else:
            dy = s["dy"][rows].float()
            dw = dy.t() @ _values(s["x"][rows], s["x_scale"][rows], c)
            if ends[e] == ends[e + 1]:
                outs.append((s["dy"].new_zeros((0, c)), dw))
                continue
            w = _values(s["w"][mine], s["w_scale"][mine], c, s["bits"], s["group"])
            outs.append(((dy @ w).to(s["dtype"]), dw))
    if op == "experts":
        return torch.cat(outs)
    return torch.cat([o[0] for o in outs]), torch.stack([o[1] for o in outs])


def _own(s):
    from paper_2202_06819_amd import linear as L
    op = s["op"]
    if op == "norm":
        y = L.norm_rows(s["x"], s["gain"], residual=s["residual"], eps=EPS)
        return y.rows.codes[:, :y.rows.channels], y.rows.scale, y.sum, y.rstd
    if op == "norm_grad":
        return L.norm_rows_grad(s["dy"], s["h"], s["gain"], s["rstd"], dsum=s["dsum"])
    w = L.GroupRows(s["w"], s["w_scale"], s["c"], s["group"]) if s["group"] else L.Rows(s["w"], s["w_scale"], s["c"], s["bits"])
    x = L.Rows(s["x"], s["x_scale"], s["c"]) if "x" in s else None
    if op == "groups":
        return L.linear(x, w, dtype=s["dtype"])
    if op == "groups_grad":
        return L.linear_grad_input(s["dy"], w)
    if op == "experts":
        return L.linear_experts(x, w, s["offsets"], dtype=s["dtype"])
    return L.linear_experts_grad_input(s["dy"], w, s["offsets"]), L.linear_experts_grad_weight(s["dy"], x, s["offsets"])


def run(state):
    return _own(state) if own else _plain(state)


# -------------------------------------------------------------- what it needs

def work(case):
    op, m, c = case["op"], case["m"], case["c"]
    size = 4 if case["dtype"] == "f32" else 2
    if op == "norm":
        return {"bytes": m * c * (size * (3 if case["residual"] else 1) + 1) + 8 * m + size * c, "flops": 0}
    if op == "norm_grad":
        return {"bytes": m * c * size * (4 if case["residual"] else 3) + 4 * m + (size + 4) * c, "flops": 0}
    k, experts = case["k"], case.get("experts", 1)
    used = sum(n > 0 for n in _counts(case)) if "experts" in case else 1
    one = 4 if case["scales"] == "f32" else 2
    scales = 4 * k if not case["group"] else one * k * -(-c // case["group"])
    weights = used * (k * c * case.get("bits", 4) // 8 + scales)
    rows = m * c + 4 * m
    if op in ("groups", "experts"):
        return {"bytes": rows + weights + 2 * m * k, "flops": 2 * m * k * c}
    if op == "groups_grad":
        return {"bytes": 2 * m * k + weights + 2 * m * c, "flops": 2 * m * k * c}
    return {"bytes": 2 * m * k + weights + 2 * m * c + rows + 4 * experts * k * c, "flops": 4 * m * k * c}


# ------------------------------------------------------- the same, 64 bits wide

def _wide_values(codes, scale, c, bits, group):
    if bits == 4:
        parts = [((codes.to(torch.int64) >> (4 * i)) & 15) for i in range(8)]
        v = torch.stack(parts, dim=-1).reshape(codes.shape[0], -1)
        codes = v - 16 * (v >= 8).to(torch.int64)
    v = codes[:, :c].double()
    if not group:
        return v * scale.double()[:, None]
    for n in range(scale.shape[1]):
        v[:, n * group:(n + 1) * group] *= scale[:, n:n + 1].double()
    return v


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    c = case["c"]
    if op == "norm":
        x = s["x"].double()
        h = x if s["residual"] is None else (x + s["residual"].double()).to(s["x"].dtype).double()
        power = (h ** 2).sum(dim=1) / c
        y = h * s["gain"].double() / (power + EPS).sqrt()[:, None]
        amax = y.abs().max(dim=1).values
        e = torch.floor(torch.log2(amax / 127))
        e = torch.where(amax > 127 * torch.exp2(e), e + 1, e)
        scale = torch.where(amax > 0, torch.exp2(e), torch.ones_like(amax))
        return torch.round(y / scale[:, None]).to(torch.int8), torch.where(amax > 0, scale, 0 * scale), h, (power + EPS) ** -0.5
    if op == "norm_grad":
        dy, h, gain, r = s["dy"].double(), s["h"].double(), s["gain"].double(), s["rstd"].double()
        along = (dy * gain * h).sum(dim=1) / c
        dx = (dy * gain - h * (r ** 2 * along)[:, None]) * r[:, None]
        if s["dsum"] is not None:
            dx = dx + s["dsum"].double()
        return dx, torch.mv((dy * h).t().contiguous(), r)
    k = case["k"]
    ends = s["offsets"].tolist() if "experts" in case else [0, case["m"]]
    y = torch.zeros((case["m"], k), dtype=torch.float64, device="cuda")
    dx = torch.zeros((case["m"], c), dtype=torch.float64, device="cuda")
    dw = torch.zeros((len(ends) - 1, k, c), dtype=torch.float64, device="cuda")
    for e, (begin, end) in enumerate(zip(ends[:-1], ends[1:])):
        if begin == end:
            continue
        w = _wide_values(s["w"][e * k:(e + 1) * k], s["w_scale"][e * k:(e + 1) * k], c, s["bits"], s["group"])
        if "x" in s:
            x = _wide_values(s["x"][begin:end], s["x_scale"][begin:end], c, 8, 0)
        if op in ("groups", "experts"):
            y[begin:end] = x.matmul(w.t().contiguous())
        else:
            dy = s["dy"][begin:end].double()
            dx[begin:end] = dy.matmul(w)
            if op == "experts_grad":
                dw[e] = dy.t().contiguous().matmul(x)
    return y if op in ("groups", "experts") else dx if op == "groups_grad" else (dx, dw)

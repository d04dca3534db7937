"""The operators around the linear layer together, as a block uses them: trained through
the differentiable layers, served captured; on other streams, and their refusals."""
import pytest
import torch

pytestmark = pytest.mark.gpu

HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
DTYPES = (torch.bfloat16, torch.float16)


@pytest.fixture(scope="module")
def L():
    from paper_2202_06819_amd import build, linear
    build.ensure_built()
    return linear


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _values(rows):
    return rows.codes[:, :rows.channels].double() * rows.scale.double()[:, None]


def _close(got, want, size, halves):
    """In norm: ``halves`` times a half ulp of ``size`` (a tenth more for what 32-bit sums
    and the roundings' products add)."""
    error = float((got.double() - want).norm())
    limit = 1.1 * halves * float(size.norm())
    assert error <= limit, f"{error:.3g} > {limit:.3g}"


# ------------------------------------------------------------------- layers

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("residual", [False, True])
def test_norm_linear_layer(L, dtype, residual):
    g = _gen(1)
    x, more = (_randn(g, 3, 50, 136).to(dtype).requires_grad_() for _ in range(2))
    gain = (1 + 0.2 * _randn(g, 136)).requires_grad_()
    w = (_randn(g, 72, 136) * 0.1).requires_grad_()
    y, total = L.norm_linear_layer(x, gain, w, residual=more if residual else None, eps=1e-5)
    assert y.shape == (3, 50, 72) and y.dtype == dtype and total.shape == x.shape
    dy, dsum = _randn(g, 3, 50, 72).to(dtype), _randn(g, 3, 50, 136).to(dtype)
    ((y * dy).sum() + (total * dsum).sum() if residual else (y * dy).sum()).backward()
    # from the layer's own 8-bit rows, in 64 bits
    h = (x.float() + more.float()).to(dtype) if residual else x.detach()
    n8 = L.norm_rows(h.detach().reshape(-1, 136), gain.detach(), eps=1e-5)
    w8 = L.quantize_rows(w.detach())
    assert torch.equal(total.detach(), h.detach())
    assert torch.equal(y.detach().reshape(-1, 72), L.linear(n8.rows, w8, dtype=dtype))
    d = dy.reshape(-1, 72).double()
    dn = d @ _values(w8)
    r, hh = n8.rstd.double()[:, None], h.detach().reshape(-1, 136).double()
    t, n = dn * gain.detach().double(), hh * r
    dx = r * (t - n * (t * n).mean(1, keepdim=True))
    size = r * t.abs()
    if residual:
        dx, size = dx + dsum.reshape(-1, 136).double(), size + dsum.reshape(-1, 136).double().abs()
    u = HALF_ULP[dtype]
    # dn is rounded once on its way, dx at its end (the norm's gradient shortens t's error)
    _close(x.grad.reshape(-1, 136), dx, size, 2 * u)
    if residual:
        assert torch.equal(more.grad, x.grad) and more.grad.data_ptr() != x.grad.data_ptr()
    _close(gain.grad, (dn * n).sum(0), (dn * n).norm(dim=0), u + 2.0 ** -20)
    assert torch.equal(w.grad, L.linear_grad_weight(dy.reshape(-1, 72), n8.rows))


def test_norm_linear_layer_with_unused_outputs_and_views(L):
    g = _gen(2)
    x, more = _randn(g, 96, 40).bfloat16().t(), _randn(g, 1, 96).bfloat16().expand(40, 96)
    gain, w = torch.ones(192, device="cuda")[::2].requires_grad_(), (_randn(g, 24, 96) * 0.1).requires_grad_()
    x, more = x.requires_grad_(), more.requires_grad_()
    plain = [t.detach().clone(memory_format=torch.contiguous_format).requires_grad_() for t in (x, more, gain, w)]
    for use in ("both", "y", "sum"):
        grads = []
        for args in ((x, more, gain, w), plain):
            y, total = L.norm_linear_layer(args[0], args[2], args[3], residual=args[1])
            value = (y.float().sum() if use != "sum" else 0.0) + (total.float().square().sum() if use != "y" else 0.0)
            grads.append(torch.autograd.grad(value, args, allow_unused=True))
        for a, b in zip(*grads):
            assert (a is None and b is None) or torch.equal(a, b)
        assert (grads[0][3] is None) == (use == "sum")
    with pytest.raises(L.QConvError):
        L.norm_linear_layer(x, gain, w, residual=more[:1])
    # one tensor as both summands
    v = plain[0].detach().requires_grad_()
    y, total = L.norm_linear_layer(v, plain[2].detach(), plain[3].detach(), residual=v)
    y.float().sum().backward()
    a, b = (plain[0].detach().clone().requires_grad_() for _ in range(2))
    y, total = L.norm_linear_layer(a, plain[2].detach(), plain[3].detach(), residual=b)
    y.float().sum().backward()
    assert torch.equal(v.grad, a.grad + b.grad)


@pytest.mark.parametrize("dtype", DTYPES)
def test_experts_layer(L, dtype):
    g = _gen(3)
    counts, c, k, before, after = [0, 5, 70, 1, 0, 33], 136, 72, 2, 3
    m = before + sum(counts) + after
    offsets = torch.tensor([before] + counts, device="cuda").cumsum(0).to(torch.int32)
    x = _randn(g, m, c).to(dtype).requires_grad_()
    w = (_randn(g, len(counts), k, c) * 0.1).requires_grad_()
    y = L.experts_layer(x, w, offsets)
    dy = _randn(g, m, k).to(dtype)
    y.backward(dy)
    x8 = L.quantize_rows(x.detach())
    u = HALF_ULP[dtype]
    assert not y[:before].any() and not y[m - after:].any() and not x.grad[:before].any() and not x.grad[m - after:].any()
    at = before
    for e, n in enumerate(counts):
        if not n:
            assert not w.grad[e].any()
            continue
        rows, w8 = slice(at, at + n), L.quantize_rows(w[e].detach())
        xv, wv, d = _values(x8)[rows], _values(w8), dy[rows].double()
        _close(y[rows].detach(), xv @ wv.t().contiguous(), xv @ wv.t().contiguous(), u)
        _close(x.grad[rows], d @ wv, d @ wv, u)
        want = d.t().contiguous() @ xv
        _close(w.grad[e], want, want, 2.0 ** -18)
        at += n
    with pytest.raises(L.QConvError):
        L.experts_layer(x, w, offsets[:-1])


def test_a_block_trains(L):
    """Norm, projection, experts and their gradients in one step: every leaf gets the
    gradient that the parts give one by one."""
    g = _gen(4)
    tokens, c, k, experts = 60, 128, 96, 4
    h0, x0 = _randn(g, tokens, c).bfloat16(), _randn(g, tokens, c).bfloat16()
    leaves = [h0, x0, 1 + 0.1 * _randn(g, c), _randn(g, c, c) * 0.1, _randn(g, experts, k, c) * 0.1]
    order = torch.randperm(tokens, generator=g, device="cuda")
    offsets = torch.tensor([0, 20, 20, 45, 60], dtype=torch.int32, device="cuda")

    def step(h, x, gain, w, we):
        y, total = L.norm_linear_layer(x, gain, w, residual=h)
        return L.experts_layer(torch.nn.functional.silu(y)[order], we, offsets), total
    leaves = [t.requires_grad_() for t in leaves]
    z, total = step(*leaves)
    (z.float().square().mean() + total.float().mean()).backward()
    assert all(t.grad is not None and torch.isfinite(t.grad).all() and t.grad.any() for t in leaves)
    # the same from the parts
    h, x, gain, w, we = (t.detach() for t in leaves)
    n = L.norm_rows(x, gain, residual=h)
    w8, we8 = L.quantize_rows(w), L.quantize_rows(we.reshape(-1, c))
    y = L.linear(n.rows, w8).requires_grad_()
    a = torch.nn.functional.silu(y)[order]
    a8 = L.quantize_rows(a.detach())
    z2 = L.linear_experts(a8, we8, offsets)
    assert torch.equal(z, z2)
    zz = z2.clone().requires_grad_()
    dz, = torch.autograd.grad(zz.float().square().mean(), zz)
    da = L.linear_experts_grad_input(dz, we8, offsets)
    dy, = torch.autograd.grad(a, y, da)
    assert torch.equal(leaves[4].grad.reshape(-1, c), L.linear_experts_grad_weight(dz, a8, offsets).reshape(-1, c))
    assert torch.equal(leaves[3].grad, L.linear_grad_weight(dy, n.rows))
    t = n.sum.clone().requires_grad_()
    dsum, = torch.autograd.grad(t.float().mean(), t)
    dx, dgain = L.norm_rows_grad(L.linear_grad_input(dy, w8), n.sum, gain, n.rstd, dsum=dsum)
    assert torch.equal(leaves[1].grad, dx) and torch.equal(leaves[0].grad, dx) and torch.equal(leaves[2].grad, dgain)


# --------------------------------------------------------- streams and graphs

def _weights4(L, g, k, c, group):
    q = torch.randint(-8, 8, (k, c), generator=g, device="cuda").to(torch.int8)
    return L.pack_groups4(q, (torch.rand(k, -(-c // group), generator=g, device="cuda") * 0.02 + 0.01).half(), group)


def _serving(L, g, m, c, k, experts, group):
    """One decoding step, and what it reads."""
    s = {"h": _randn(g, m, c).bfloat16(), "x": _randn(g, m, c).bfloat16(), "gain": 1 + 0.1 * _randn(g, c),
         "offsets": torch.linspace(0, m, experts + 1, device="cuda").to(torch.int32), "dy": _randn(g, m, k).bfloat16()}
    w, we, w8 = _weights4(L, g, c, c, group), _weights4(L, g, experts * k, c, group), L.quantize_rows(_randn(g, experts * k, c))

    def step(**on):
        n = L.norm_rows(s["x"], s["gain"], residual=s["h"], **on)
        y = L.linear(n.rows, w, **on)
        x8 = L.quantize_rows(y, **on)
        z = L.linear_experts(x8, we, s["offsets"], **on)
        dx = L.linear_experts_grad_input(s["dy"], w8, s["offsets"], **on)
        dw = L.linear_experts_grad_weight(s["dy"], x8, s["offsets"], **on)
        dh, dgain = L.norm_rows_grad(L.linear_grad_input(dx, w, **on), n.sum, s["gain"], n.rstd, dsum=s["x"], **on)
        return n.rows.codes, n.sum, y, z, dx, dw, dh, dgain
    return s, step


@pytest.mark.parametrize("m", [3, 150])
def test_streams_and_graphs(L, m):
    """On the current stream, on another current one, on a given one: the same; captured,
    with the inputs and the experts' shares changed between replays, what an eager call
    gives."""
    g = _gen(m)
    s, step = _serving(L, g, m, 256, 96, 5, 64)
    eager = [t.clone() for t in step()]
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        there = step()
    torch.cuda.current_stream().wait_stream(other)
    assert all(torch.equal(a, b) for a, b in zip(eager, there))
    given = step(stream=other)
    other.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, given))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for turn in range(4):
        if turn:
            s["x"].copy_(_randn(g, *s["x"].shape))
            s["dy"].copy_(_randn(g, *s["dy"].shape))
            s["offsets"][1:-1] = torch.randint(0, m + 1, (4,), generator=g, device="cuda").sort().values
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        assert all(torch.equal(a, b) for a, b in zip(got, step()))


def test_two_calls_at_once(L):
    """Two steps on two streams, their work queued together, share nothing."""
    g = _gen(7)
    (_, one), (_, two) = _serving(L, g, 700, 512, 256, 4, 32), _serving(L, g, 900, 512, 256, 4, 32)
    want = [[t.clone() for t in step()] for step in (one, two)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, step in enumerate((one, two)):
            got[i].append(step(stream=streams[i]))
    torch.cuda.synchronize()
    for outs, expected in zip(got, want):
        for out in outs:
            assert all(torch.equal(a, b) for a, b in zip(out, expected))


OPS = ["norm_rows", "norm_rows_grad", "groups", "groups_grad", "experts", "experts_groups", "experts_grad_input",
       "experts_grad_weight", "pack_groups4"]


def _operation(L, g, op):
    """(operands, the call on them)"""
    m, c, k = 2048, 512, 512
    v, dy = _randn(g, m, c).bfloat16(), _randn(g, m, k).bfloat16()
    x8, w8, w4 = L.quantize_rows(v), L.quantize_rows(_randn(g, 4 * k, c)), _weights4(L, g, k, c, 64)
    e4 = _weights4(L, g, 4 * k, c, 64)
    gain, offsets = _randn(g, c), torch.tensor([0, 100, 1000, 1500, m], dtype=torch.int32, device="cuda")
    rows = lambda t: L.Rows(t[0], t[1], c)
    four = lambda t: L.GroupRows(t[0], t[1], c, 64)
    return {
        "norm_rows": ([v, gain, dy], lambda t, **on: L.norm_rows(t[0], t[1], residual=t[2], **on).rows.codes),
        "norm_rows_grad": ([dy, v, gain, torch.rand(m, generator=g, device="cuda"), v.clone()],
                           lambda t, **on: L.norm_rows_grad(*t[:4], dsum=t[4], **on)[0]),
        "groups": ([*x8[:2], *w4[:2]], lambda t, **on: L.linear(rows(t), four(t[2:]), **on)),
        "groups_grad": ([dy, *w4[:2]], lambda t, **on: L.linear_grad_input(t[0], four(t[1:]), **on)),
        "experts": ([*x8[:2], *w8[:2], offsets], lambda t, **on: L.linear_experts(rows(t), rows(t[2:]), t[4], **on)),
        "experts_groups": ([*x8[:2], *e4[:2], offsets], lambda t, **on: L.linear_experts(rows(t), four(t[2:]), t[4], **on)),
        "experts_grad_input": ([dy, *w8[:2], offsets], lambda t, **on: L.linear_experts_grad_input(t[0], rows(t[1:]), t[3], **on)),
        "experts_grad_weight": ([dy, *x8[:2], offsets], lambda t, **on: L.linear_experts_grad_weight(t[0], rows(t[1:]), t[3], **on)),
        "pack_groups4": ([x8.codes, w4.scale], lambda t, **on: L.pack_groups4(t[0], t[1], 64, **on).codes),
    }[op]


@pytest.mark.parametrize("op", OPS)
def test_operands_are_kept_until_a_given_stream_has_read_them(L, op):
    g = _gen(8)
    operands, call = _operation(L, g, op)
    want = call(operands)
    s = torch.cuda.Stream()
    call(operands, stream=s)
    mine = [t.clone() for t in operands]
    sizes_of = [t.numel() * t.element_size() for t in mine]
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(200_000_000)
    got = call(mine, stream=s)
    del mine
    new = [torch.full((n,), 99, dtype=torch.uint8, device="cuda") for n in sizes_of * 2]
    torch.cuda.synchronize()
    assert torch.equal(got, want) and all((t == 99).all() for t in new)


@pytest.mark.parametrize("op", OPS)
def test_a_given_streams_results_do_not_meet_the_current_streams_memory(L, op):
    g = _gen(9)
    operands, call = _operation(L, g, op)
    want = call(operands)
    held = want.numel() * want.element_size()
    s, current = torch.cuda.Stream(), torch.cuda.current_stream()
    call(operands, stream=s)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    old = torch.full((held,), 77, dtype=torch.uint8, device="cuda")
    read = torch.empty_like(old)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    read.copy_(old)
    del old
    got = call(operands, stream=s)
    s.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and (read == 77).all()
    again = call(operands, stream=s)
    current.wait_stream(s)
    torch.cuda._sleep(200_000_000)
    copy = again.clone()
    del again, got
    with torch.cuda.stream(s):
        other = torch.full((held,), 99, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    assert torch.equal(copy, want) and (other == 99).all()


# ------------------------------------------------------------------ refusals

def test_refusals_of_tensors(L):
    g = _gen(10)
    x, gain = _randn(g, 6, 64).bfloat16(), torch.ones(64, device="cuda")
    x8, w8 = L.quantize_rows(x), L.quantize_rows(_randn(g, 48, 64))
    w4, dy = _weights4(L, g, 48, 64, 32), _randn(g, 6, 24).bfloat16()
    rstd, offsets = torch.ones(6, device="cuda"), torch.tensor([0, 3, 6], dtype=torch.int32, device="cuda")
    ad = L.Adapters(torch.zeros(1, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 48, 8, dtype=torch.bfloat16, device="cuda"),
                    torch.ones(1, device="cuda"))
    bad = [
        lambda: L.norm_rows(x.double(), gain),
        lambda: L.norm_rows(x, gain[:32]),
        lambda: L.norm_rows(x, gain.double()),
        lambda: L.norm_rows(x, gain.cpu()),
        lambda: L.norm_rows(x, torch.ones(128, device="cuda")[::2]),
        lambda: L.norm_rows(x, gain, residual=x.half()),
        lambda: L.norm_rows(x, gain, residual=x[:3]),
        lambda: L.norm_rows(x, gain, residual=x[:1].expand(6, 64)),
        lambda: L.norm_rows(x, gain, sum_out=x),
        lambda: L.norm_rows(x, gain, residual=x, sum_out=x.half()),
        lambda: L.norm_rows(x, gain, eps=-1.0),
        lambda: L.norm_rows(x, gain, out=x8._replace(channels=48)),
        lambda: L.norm_rows_grad(x, x.half(), gain, rstd),
        lambda: L.norm_rows_grad(x, x, gain, rstd[:3]),
        lambda: L.norm_rows_grad(x, x, gain, rstd.double()),
        lambda: L.norm_rows_grad(x, x, gain, rstd, dsum=x[:, :32]),
        lambda: L.norm_rows_grad(x, x, gain, rstd, out=x),
        lambda: L.norm_rows_grad(x, x, gain, rstd, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")),
        lambda: L.linear(x8, w4._replace(group=48)),
        lambda: L.linear(x8, w4._replace(group=16)),
        lambda: L.linear(x8, w4._replace(group=64)),
        lambda: L.linear(x8, w4._replace(scale=w4.scale.double())),
        lambda: L.linear(x8, w4._replace(scale=w4.scale[:5])),
        lambda: L.linear(x8, w4._replace(scale=w4.scale.t().contiguous().t())),
        lambda: L.linear(x8, w4._replace(codes=w4.codes.to(torch.int8))),
        lambda: L.linear(x8, w4, adapters=ad, row_adapter=torch.zeros(6, dtype=torch.int32, device="cuda")),
        lambda: L.linear_grad_input(dy, w4),
        lambda: L.linear_experts(x8, w8, offsets.long()),
        lambda: L.linear_experts(x8, w8, offsets.cpu()),
        lambda: L.linear_experts(x8, w8, offsets[:1]),
        lambda: L.linear_experts(x8, L.quantize_rows(_randn(g, 47, 64)), offsets),
        lambda: L.linear_experts(x8, w8, offsets, dtype=torch.float32),
        lambda: L.linear_experts(x8, w8, offsets, out=torch.empty(6, 48, dtype=torch.bfloat16, device="cuda")),
        lambda: L.linear_experts_grad_input(dy[:, :20], w8, offsets),
        lambda: L.linear_experts_grad_input(dy.float(), w8, offsets),
        lambda: L.linear_experts_grad_weight(dy[:4], x8, offsets),
        lambda: L.linear_experts_grad_weight(dy, x8, offsets, out=torch.empty(2, 24, 64, dtype=torch.bfloat16, device="cuda")),
        lambda: L.pack_groups4(torch.zeros(4, 12, dtype=torch.int8, device="cuda"), torch.zeros(4, 1, device="cuda"), 32),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(L.QConvError):
            call()
            pytest.fail(f"case {i} was accepted")

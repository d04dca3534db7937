"""Products by weights with scales of groups of channels and by the weights of experts,
and their gradients, against plain 64-bit computations.

Tolerances follow from the roundings alone.  A group's sum of codes is exact; the kernels
add scaled sums of 32 channels or more in 32 bits, with an error of at most (their
number) * 2^-24 of the sum of their absolute values; the two scales add a few roundings.
A 16-bit result is rounded once, half an ulp.  In the gradients a code times its scale
is rounded to the 16-bit type, another half ulp of each product (none for scales that are
powers of two), and sums are 32-bit."""
import math

import pytest
import torch

import around_sizes as sizes

pytestmark = pytest.mark.gpu

HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
DTYPES = (torch.bfloat16, torch.float16)
SCALES = (torch.float16, torch.bfloat16, torch.float32)


@pytest.fixture(scope="module")
def L():
    from paper_2202_06819_amd import build, linear
    build.ensure_built()
    return linear


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _rows8(L, g, m, c):
    codes = torch.zeros((m, L.rows_pitch(c)), dtype=torch.int8, device="cuda")
    codes[:, :c] = torch.randint(-127, 128, (m, c), generator=g, device="cuda").to(torch.int8)
    return L.Rows(codes, torch.rand(m, generator=g, device="cuda") * 0.02 + 0.001, c)


def _weights(L, g, k, c, bits=4, group=0, scales=torch.float32):
    """Rows and the whole numbers that they hold."""
    if bits == 8:
        rows = _rows8(L, g, k, c)
        return rows, rows.codes[:, :c]
    q = torch.randint(-8, 8, (k, c), generator=g, device="cuda").to(torch.int8)
    shape = (k, -(-c // group)) if group else (k,)
    scale = (torch.rand(*shape, generator=g, device="cuda") * 0.02 + 0.005).to(scales if group else torch.float32)
    return (L.pack_groups4(q, scale, group) if group else L.pack_rows4(q, scale)), q


def _scale(w, c):
    """The scale of every weight, in 64 bits."""
    s = w.scale.double()
    if s.dim() == 1:
        return s[:, None].expand(-1, c)
    return s[:, torch.arange(c, device="cuda") // w.group]


def _product(x, w, q):
    """The result, and the sum of the absolute values of its parts of 32 channels."""
    c = x.channels
    xv, wv = x.codes[:, :c].double(), q.double() * _scale(w, c)
    want = torch.zeros((xv.shape[0], wv.shape[0]), dtype=torch.float64, device="cuda")
    size = want.clone()
    for at in range(0, c, 32):
        part = xv[:, at:at + 32].contiguous() @ wv[:, at:at + 32].t().contiguous()
        want += part
        size += part.abs()
    s = x.scale.double()[:, None]
    return want * s, size * s.abs()


def _near(got, want, size, terms, dtype):
    tol = size * (terms + 4) * 2.0 ** -24
    if dtype in HALF_ULP:
        tol = tol * (1 + HALF_ULP[dtype]) + want.abs() * HALF_ULP[dtype] + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    bad = (got.double() - want).abs() > tol + 1e-300
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, worst {float(((got.double() - want).abs() / tol).max()):.3g}"


# ------------------------------------------------------------------- groups

GROUPS = [(1, 32, 1, 32), (1, 8, 3, 32), (1, 4096, 33, 128), (2, 520, 40, 64), (4, 264, 17, 32), (5, 1000, 130, 32), (7, 96, 50, 96),
          (8, 2048, 64, 64), (9, 392, 100, 32), (13, 640, 33, 160), (16, 1032, 20, 128), (17, 136, 64, 32), (33, 384, 200, 64),
          (64, 520, 130, 128), (65, 64, 129, 32), (100, 1000, 300, 256), (129, 2048, 257, 32), (250, 8200, 400, 128),
          (515, 136, 700, 64), (3, 256, 40, 4096), (40, 256, 40, 4096), (700, 392, 1100, 32), (6, 131064, 4, 32)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,c,k,group", GROUPS)
def test_groups(L, m, c, k, group, dtype):
    g = _gen(m + c + k + group)
    x = _rows8(L, g, m, c)
    w, q = _weights(L, g, k, c, group=group, scales=SCALES[(m + c // 8 + k) % 3])
    want, size = _product(x, w, q)
    y = L.linear(x, w, dtype=dtype)
    _near(y, want, size, c // 32 + 8, dtype)
    assert torch.equal(y, L.linear(x, w, dtype=dtype))


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("scales", SCALES)
def test_groups_large_tiles(L, group, scales):
    g = _gen(group)
    m, c, k = 3500, 328, 4100
    x = _rows8(L, g, m, c)
    w, q = _weights(L, g, k, c, group=group, scales=scales)
    want, size = _product(x, w, q)
    _near(L.linear(x, w), want, size, c // 32 + 8, torch.bfloat16)


@pytest.mark.parametrize("m", [1, 3, 20, 300])
@pytest.mark.parametrize("group", [32, 64, 96, 128])
def test_groups_of_views(L, m, group):
    """Scales and codes as parts of wider matrices, y as another's columns; what lies
    beside them is neither read nor written."""
    g = _gen(m + group)
    c, k = 328, 70
    x = _rows8(L, g, m, c)
    w, q = _weights(L, g, k, c, group=group, scales=torch.float16)
    n = w.scale.shape[1]
    wide = torch.full((k, n + 5), math.nan, dtype=torch.float16, device="cuda")
    wide[:, 2:2 + n] = w.scale
    words = torch.full((k, w.codes.shape[1] + 8), -1, dtype=torch.int32, device="cuda")
    words[:, 4:4 + w.codes.shape[1]] = w.codes
    view = L.GroupRows(words[:, 4:4 + w.codes.shape[1]], wide[:, 2:2 + n], c, group)
    out = torch.full((m, k + 9), 7.0, dtype=torch.bfloat16, device="cuda")
    y = L.linear(x, view, out=out[:, 3:3 + k])
    assert torch.equal(y, L.linear(x, w)) and (out[:, :3] == 7).all() and (out[:, 3 + k:] == 7).all()
    dy = _randn(g, m, k).bfloat16()
    assert torch.equal(L.linear_grad_input(dy, view), L.linear_grad_input(dy, w))


@pytest.mark.parametrize("m", [1, 5, 30, 200])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_one_scales_fault_stays_in_its_channel(L, m, group):
    """A scale that is not finite reaches its own output channel, and of the gradient
    its own group of input channels; a row's scale its own row."""
    g = _gen(m)
    c, k = 392, 90
    x = _rows8(L, g, m, c)
    w, q = _weights(L, g, k, c, group=group)
    clean = L.linear(x, w)
    dy = _randn(g, m, k).bfloat16()
    dx_clean = L.linear_grad_input(dy, w)
    w.scale[7, 1] = math.nan
    x.scale[m - 1] = math.inf
    y = L.linear(x, w)
    hit = (torch.arange(k, device="cuda") == 7)[None] | (torch.arange(m, device="cuda") == m - 1)[:, None]
    assert torch.equal(y[~hit], clean[~hit]) and y[:, 7].isnan().all() and not torch.isfinite(y[m - 1]).any()
    dx = L.linear_grad_input(dy, w)
    group_of = torch.arange(c, device="cuda") // group == 1
    assert torch.equal(dx[:, ~group_of], dx_clean[:, ~group_of]) and dx[:, group_of].isnan().all()


def _dy(g, m, k, dtype, stride=0):
    buf = torch.full((m, stride or k), 3.0, dtype=dtype, device="cuda")
    buf[:, :k] = _randn(g, m, k).to(dtype)
    return buf[:, :k]


def _grad(dy, w, q, c):
    wv = q.double() * _scale(w, c)
    d = dy.double().contiguous()
    return d @ wv, d.abs() @ wv.abs()


def _grad_near(got, want, size, depth, dtype):
    """(any scales: the product of code and scale is rounded to the type.)"""
    tol = size * (HALF_ULP[dtype] * 1.01 + (depth + 4) * 2.0 ** -24)
    tol = tol * (1 + HALF_ULP[dtype]) + want.abs() * HALF_ULP[dtype] + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    bad = (got.double() - want).abs() > tol + 1e-300
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, worst {float(((got.double() - want).abs() / tol).max()):.3g}"


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,c,k,group,stride", [
    (1, 8, 1, 32, 0), (3, 40, 33, 32, 0), (65, 136, 70, 64, 80), (130, 1000, 256, 128, 256), (300, 264, 1001, 32, 1011),
    (1000, 1024, 2640, 96, 0), (20, 520, 5000, 64, 0), (333, 2824, 1001, 64, 0), (5, 4096, 64, 4096, 64), (2, 64, 200, 32, 0)])
def test_groups_grad_input(L, m, c, k, group, stride, dtype):
    g = _gen(m + c + k)
    dy = _dy(g, m, k, dtype, stride)
    w, q = _weights(L, g, k, c, group=group, scales=SCALES[(m + k) % 3])
    want, size = _grad(dy, w, q, c)
    dx = L.linear_grad_input(dy, w)
    _grad_near(dx, want, size, k, dtype)
    assert torch.equal(dx, L.linear_grad_input(dy, w))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("k", [520, 1001])
def test_groups_grad_input_large_tiles(L, k, group, dtype):
    g = _gen(group + k)
    m, c = 3000, 4104
    dy = _dy(g, m, k, dtype)
    for scales in SCALES:
        w, q = _weights(L, g, k, c, group=group, scales=scales)
        want, size = _grad(dy, w, q, c)
        _grad_near(L.linear_grad_input(dy, w), want, size, k, dtype)


# ------------------------------------------------------------------ experts

def _offsets(counts, first=0):
    return torch.tensor([first] + counts, device="cuda").cumsum(0).to(torch.int32)


WEIGHTS = [(8, 0, torch.float32), (4, 0, torch.float32), (4, 32, torch.float16), (4, 64, torch.bfloat16), (4, 128, torch.float32)]
DEALT = [
    ([1], 64, 40), ([0, 0, 3], 256, 33), ([5, 0, 1, 0, 17, 2], 136, 70), ([0] * 30 + [1, 1, 2, 0, 1], 264, 130),
    ([64, 64, 64], 128, 64), ([63, 65, 0, 130], 520, 200), ([1] * 70, 96, 50), ([0] * 66 + [9] + [0] * 70, 200, 100),
    ([300, 1, 0, 5, 700], 328, 300), ([16, 16, 15, 17, 33], 1000, 96), ([0, 0], 64, 8), ([2000, 900, 0, 1300], 264, 1100),
]


@pytest.mark.parametrize("bits,group,scales", WEIGHTS)
@pytest.mark.parametrize("counts,c,k", DEALT)
def test_experts(L, counts, c, k, bits, group, scales):
    """Each expert's rows are what its weights alone give; rows of no expert are left."""
    dtype = DTYPES[len(counts) % 2]
    g = _gen(sum(counts) + c + k)
    experts, first, more = len(counts), 2, 3
    m = first + sum(counts) + more
    x = _rows8(L, g, m, c)
    w, q = _weights(L, g, experts * k, c, bits, group, scales)
    offsets = _offsets(counts, first)
    out = torch.full((m, k + 1), 7.0, dtype=dtype, device="cuda")[:, :k]
    y = L.linear_experts(x, w, offsets, dtype=dtype, out=out)
    assert (y[:first] == 7).all() and (y[m - more:] == 7).all()
    at = first
    for e, n in enumerate(counts):
        if n:
            rows = L.Rows(x.codes[at:at + n], x.scale[at:at + n], c)
            mine = slice(e * k, e * k + k)
            part = L.GroupRows(w.codes[mine], w.scale[mine], c, group) if group else L.Rows(w.codes[mine], w.scale[mine], c, bits)
            want, size = _product(rows, part, q[mine])
            _near(y[at:at + n], want, size, c // 32 + 8, dtype)
        at += n


@pytest.mark.parametrize("bits,group,scales", WEIGHTS)
@pytest.mark.parametrize("counts,c,k", DEALT)
def test_experts_grad_input(L, counts, c, k, bits, group, scales):
    dtype = DTYPES[(len(counts) + group) % 2]
    g = _gen(sum(counts) + c + k)
    experts, first, more = len(counts), 1, 4
    m = first + sum(counts) + more
    dy = _dy(g, m, k, dtype, k + (8 if c % 3 else 0))
    w, q = _weights(L, g, experts * k, c, bits, group, scales)
    out = torch.full((m, c + 1), 7.0, dtype=dtype, device="cuda")[:, :c]
    dx = L.linear_experts_grad_input(dy, w, _offsets(counts, first), out=out)
    assert (dx[:first] == 7).all() and (dx[m - more:] == 7).all()
    at = first
    for e, n in enumerate(counts):
        if n:
            mine = slice(e * k, e * k + k)
            part = L.GroupRows(w.codes[mine], w.scale[mine], c, group) if group else L.Rows(w.codes[mine], w.scale[mine], c, bits)
            want, size = _grad(dy[at:at + n], part, q[mine], c)
            _grad_near(dx[at:at + n], want, size, k, dtype)
        at += n


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("odd", [0, 3])
@pytest.mark.parametrize("counts,c,k", DEALT + [([5, 0, 4000], 300, 40), ([3000, 2900], 1300, 1100)])
def test_experts_grad_weight(L, counts, c, k, odd, dtype):
    g = _gen(sum(counts) + c + k)
    experts, first, more = len(counts), 3, 2
    m, c, k = first + sum(counts) + more, c + odd, k + odd
    dy, x = _dy(g, m, k, dtype, k + (k + odd) % 8), _rows8(L, g, m, c)
    out = torch.full((experts, k, c), math.nan, device="cuda")
    dw = L.linear_experts_grad_weight(dy, x, _offsets(counts, first), out=out)
    assert dw is out
    at = first
    for e, n in enumerate(counts):
        d, v = dy[at:at + n].double(), x.codes[at:at + n, :c].double() * x.scale.double()[at:at + n, None]
        want, size = d.t().contiguous() @ v, d.abs().t().contiguous() @ v.abs()
        tol = size * (HALF_ULP[dtype] * 1.01 + (n + 4) * 2.0 ** -24)
        assert bool(((dw[e].double() - want).abs() <= tol).all())
        at += n
    assert torch.equal(dw, L.linear_experts_grad_weight(dy, x, _offsets(counts, first)))


def test_offsets_out_of_range(L):
    """Offsets past the rows, and negative ones, are held to the rows: nothing else is
    read or written."""
    g = _gen(1)
    x, dy = _rows8(L, g, 40, 64), _dy(g, 40, 32, torch.bfloat16)
    w, q = _weights(L, g, 3 * 32, 64, 8)
    want = L.linear_experts(x, w, torch.tensor([0, 10, 20, 40], dtype=torch.int32, device="cuda"))
    bad = torch.tensor([-5, 10, 20, 1 << 30], dtype=torch.int32, device="cuda")
    assert torch.equal(L.linear_experts(x, w, bad), want)
    assert torch.equal(L.linear_experts_grad_input(dy, w, bad),
                       L.linear_experts_grad_input(dy, w, torch.tensor([0, 10, 20, 40], dtype=torch.int32, device="cuda")))
    out = torch.full((40, 32), 7.0, dtype=torch.bfloat16, device="cuda")
    L.linear_experts(x, w, torch.tensor([100, 200, 300, 400], dtype=torch.int32, device="cuda"), out=out)
    assert (out == 7).all()
    dw = L.linear_experts_grad_weight(dy, x, torch.tensor([30, 20, 10, 5], dtype=torch.int32, device="cuda"))
    assert not dw.any()


def test_no_rows(L):
    g = _gen(2)
    x = L.Rows(torch.empty((0, 64), dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda"), 64)
    w, _ = _weights(L, g, 64, 64, 8)
    w4, _ = _weights(L, g, 64, 64, 4, 32)
    offsets = torch.zeros(3, dtype=torch.int32, device="cuda")
    none = torch.empty((0, 32), dtype=torch.bfloat16, device="cuda")
    assert L.linear(x, w4).shape == (0, 64) and L.linear_experts(x, w, offsets).shape == (0, 32)
    assert L.linear_grad_input(torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"), w4).shape == (0, 64)
    assert L.linear_experts_grad_input(none, w, offsets).shape == (0, 64)
    dw = L.linear_experts_grad_weight(none, x, offsets)
    assert dw.shape == (2, 32, 64) and not dw.any()


# ------------------------------------------------------------- every kernel

def _dealt(m, experts):
    """Very different shares, none for some."""
    g = torch.Generator().manual_seed(m + experts)
    cuts = (torch.rand(experts - 1, generator=g) ** 2 * (m + 1)).long().sort().values.tolist() if experts > 1 else []
    return [b - a for a, b in zip([0] + cuts, cuts + [m])]


@pytest.mark.parametrize("op,m,c,k,bits,group,scales,experts,dtype", sizes.PRODUCTS)
def test_every_kernel(L, op, m, c, k, bits, group, scales, experts, dtype):
    """The sizes between them launch every kernel (which another test records)."""
    g = _gen(m + c + k + experts)
    dtype = DTYPES[dtype]
    counts = _dealt(m, experts) if experts else [m]
    offsets = _offsets(counts)
    if op != "grad_weight":
        w, q = _weights(L, g, max(experts, 1) * k, c, bits, group, (torch.bfloat16, torch.float16, torch.float32)[scales])
    if op != "grad_input":
        x = _rows8(L, g, m, c)
    if op != "forward":
        dy = _dy(g, m, k, dtype)
    if op == "forward":
        got = L.linear_experts(x, w, offsets, dtype=dtype) if experts else L.linear(x, w, dtype=dtype)
    elif op == "grad_input":
        got = L.linear_experts_grad_input(dy, w, offsets) if experts else L.linear_grad_input(dy, w)
    else:
        got = L.linear_experts_grad_weight(dy, x, offsets)
    at = 0
    for e, n in enumerate(counts):
        rows, mine = slice(at, at + n), slice(e * k, e * k + k)
        at += n
        if op == "grad_weight":
            d, v = dy[rows].double(), x.codes[rows, :c].double() * x.scale.double()[rows, None]
            want, size = d.t().contiguous() @ v, d.abs().t().contiguous() @ v.abs()
            assert bool(((got[e].double() - want).abs() <= size * (HALF_ULP[dtype] * 1.01 + (n + 4) * 2.0 ** -24)).all())
        elif n:
            part = L.GroupRows(w.codes[mine], w.scale[mine], c, group) if group else L.Rows(w.codes[mine], w.scale[mine], c, bits)
            if op == "forward":
                want, size = _product(L.Rows(x.codes[rows], x.scale[rows], c), part, q[mine])
                _near(got[rows], want, size, c // 32 + 8, dtype)
            else:
                want, size = _grad(dy[rows], part, q[mine], c)
                _grad_near(got[rows], want, size, k, dtype)

"""Input gradients through frozen 4-bit weights: scales of groups of channels, and the
weights of experts with one scale a row, of any values.

Tolerances follow from the roundings alone.  A scale enters the product as two parts, the
first of so few bits that a code times it is exact in the 16-bit type; the second is at most
1 + 2^-6 times 2^-4 (bf16) or 2^-7 (f16) of the scale, and a code times it is rounded once,
half an ulp: 2^-12 and 2^-18 of a product, and 2^-6 of that.  Twice as many products as the sum has terms are added in 32
bits, each with an error of at most 2^-24 of the sum of their absolute values, and the
result is rounded once, half an ulp."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
PARTS = {torch.bfloat16: 2.0 ** -12 * (1 + 2.0 ** -6), torch.float16: 2.0 ** -18 * (1 + 2.0 ** -6)}
DTYPES = (torch.bfloat16, torch.float16)
SCALES = (torch.float16, torch.bfloat16, torch.float32)

# rows, channels, outputs (of each expert), experts (0: none): tiles of 64 with one, two and
# four groups of waves, split or not, of 128 and of 256, copied to LDS and through registers
SIZES = [(1, 64, 33, 0), (20, 520, 5000, 0), (333, 2824, 1001, 0), (1000, 1024, 2640, 0), (130, 1000, 256, 0),
         (2000, 2048, 1001, 0), (3000, 4104, 520, 0), (3000, 4104, 1001, 0),
         (40, 264, 300, 3), (700, 1024, 264, 4), (4000, 1024, 264, 6), (6000, 2048, 264, 3), (6000, 2048, 261, 3)]


@pytest.fixture(scope="module")
def L():
    from paper_2202_06819_amd import build, linear
    build.ensure_built()
    return linear


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _weights(L, g, k, c, group, scales):
    """4-bit rows (group 0: one scale a row), and the whole numbers that they hold."""
    q = torch.randint(-8, 8, (k, c), generator=g, device="cuda").to(torch.int8)
    shape = (k, -(-c // group)) if group else (k,)
    scale = (torch.rand(*shape, generator=g, device="cuda") * 0.02 + 0.005).to(scales)
    return (L.pack_groups4(q, scale, group) if group else L.pack_rows4(q, scale)), q


def _values(w, q):
    s = w.scale.double()
    c = q.shape[1]
    return q.double() * (s[:, None] if s.dim() == 1 else s[:, torch.arange(c, device="cuda") // w.group])


def _split(m, experts):
    """The rows of each expert: unlike ones, none for the second."""
    if not experts:
        return [0, m]
    first = m // (experts + 1)
    return [0, first, first] + [first + (m - first) * (n + 1) // (experts - 2) for n in range(experts - 2)]


def _run(L, dy, w, ends, experts, c):
    """The gradient, into memory that holds NaN."""
    out = torch.full((dy.shape[0], c), math.nan, dtype=dy.dtype, device="cuda")
    if not experts:
        return L.linear_grad_input(dy, w, out=out)
    return L.linear_experts_grad_input(dy, w, torch.tensor(ends, dtype=torch.int32, device="cuda"), out=out)


def _expected(dy, values, ends, k):
    """The gradient in 64 bits, and the sums of the absolute values behind it."""
    d = dy.double().contiguous()
    parts = [(d[a:b], values[e * k:e * k + k]) for e, (a, b) in enumerate(zip(ends[:-1], ends[1:]))]
    return torch.cat([a @ b for a, b in parts]), torch.cat([a.abs() @ b.abs() for a, b in parts])


def _tolerance(want, size, k, dtype):
    tol = size * (PARTS[dtype] + (2 * k + 4) * 2.0 ** -24)
    return tol * (1 + HALF_ULP[dtype]) + want.abs() * HALF_ULP[dtype] + (2.0 ** -25 if dtype == torch.float16 else 1e-300)


def _near(got, want, tol):
    ok = (got.double() - want).abs() <= tol   # (false for a NaN)
    assert bool(ok.all()), f"{int((~ok).sum())} of {ok.numel()} off, worst {float(((got.double() - want).abs() / tol).max()):.3g}"


def _case(L, m, c, k, experts, group, scales, dtype, factors=None):
    g = _gen(m + c + k + group)
    dy = torch.randn(m, k, generator=g, device="cuda").to(dtype)
    w, q = _weights(L, g, max(experts, 1) * k, c, group, scales)
    if factors is not None:
        w = w._replace(scale=w.scale * factors)
    ends = _split(m, experts)
    return dy, w, q, ends


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,c,k,experts", SIZES)
def test_scales_keep_their_bits(L, m, c, k, experts, dtype):
    """Scales of any values, in all of their bits."""
    for n, (group, scales) in enumerate([(32, SCALES[(m + c) % 3]), (64, torch.float32), (128, torch.float16), (0, torch.float32)]):
        if not group and not experts or n and c < 2 * group:
            continue
        dy, w, q, ends = _case(L, m, c, k, experts, group, scales, dtype)
        got = _run(L, dy, w, ends, experts, c)
        want, size = _expected(dy, _values(w, q), ends, k)
        _near(got, want, _tolerance(want, size, k, dtype))
        assert torch.equal(got, _run(L, dy, w, ends, experts, c))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("experts", [0, 3])
def test_scales_at_the_edges(L, dtype, experts):
    """Negative, zero and infinite scales, NaN, the largest float, and some whose first part
    rounds up to the next power of two: what each reaches is what 32-bit products give it."""
    m, c, k = 40, 256, 96
    dy, w, q, ends = _case(L, m, c, k, experts, 32, torch.float32, dtype)
    top = torch.finfo(torch.float32).max
    w.scale[:, 0] = 0.0
    w.scale[:, 1] *= -1
    w.scale[3, 2], w.scale[4, 2] = 1.9999998, -1.99
    w.scale[5, 3], w.scale[6, 4], w.scale[7, 5] = math.inf, math.nan, -math.inf
    w.scale[8, 6] = top
    if experts:   # (the same of every expert)
        for e in range(1, experts):
            w.scale[e * k:(e + 1) * k] = w.scale[:k]
    got = _run(L, dy, w, ends, experts, c)
    want, size = _expected(dy, _values(w, q), ends, k)
    channels = torch.arange(c, device="cuda") // 32
    plain = (channels <= 2) | (channels == 7)
    _near(got[:, plain], want[:, plain], _tolerance(want, size, k, dtype)[:, plain])
    assert not got[:, channels == 0].any()
    # an infinite scale: infinities of one sign, NaN where the code (or dy) is zero; NaN everywhere
    for group in (3, 4, 5):
        a, b = got[:, channels == group], want[:, channels == group]
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.isinf(), b.isinf())
        assert bool((a[a.isinf()] > 0).eq(b[b.isinf()] > 0).all())
    # the largest float: no NaN (a code above one takes it past 32 bits)
    assert not got[:, channels == 6].isnan().any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scales", ["any", "five bits", "powers of two"])
@pytest.mark.parametrize("m,c,k,experts", SIZES)
def test_infinite_gradients(L, m, c, k, experts, scales, dtype):
    """An infinity in dy gives infinities of the weights' signs, NaN where the weight is zero
    or another infinity meets it, and nothing in other rows, whatever parts a scale has."""
    dy, w, q, ends = _case(L, m, c, k, experts, 32, torch.float32, dtype)
    if scales == "five bits":
        w = w._replace(scale=(w.scale * 1024).round().clamp(1, 31) / 1024)
    elif scales == "powers of two":
        w = w._replace(scale=torch.exp2(torch.log2(w.scale).round()))
    clean = _run(L, dy, w, ends, experts, c)
    hit = torch.zeros(m, dtype=torch.bool, device="cuda")
    for n, row in enumerate(range(0, m, max(m // 9, 1))):
        dy[row, (row * 7) % k] = math.inf if n % 2 else -math.inf
        if n % 4 == 3:
            dy[row, (row * 7 + k // 2) % k] = math.inf
        hit[row] = True
    got = _run(L, dy, w, ends, experts, c)
    want, _ = _expected(dy, _values(w, q), ends, k)
    assert torch.equal(got[~hit], clean[~hit])
    a, b = got[hit], want[hit]
    assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.isinf(), b.isinf())
    assert torch.equal(a[a.isinf()] > 0, b[b.isinf()] > 0) and not torch.isfinite(a).any()


@pytest.mark.parametrize("m,c,k,experts", SIZES)
@pytest.mark.parametrize("group", [32, 64])
def test_far_scales_leave_other_groups(L, m, c, k, experts, group):
    """f16: a group of channels keeps its bits whatever the scales of the groups beside it,
    as different columns of the result that they are."""
    if c < 2 * group:
        pytest.skip("one group")
    groups = -(-c // group)
    n = torch.arange(groups, device="cuda")
    for factors in (torch.where(n % 3 == 1, 2.0 ** 14, 2.0 ** -10),           # 2^24 apart, all of f16's normal range
                    torch.where(n % 3 == 1, 1e30, 1.0),                     # infinite results beside ordinary ones
                    torch.where(n % 4 == 2, 1.0, 2.0 ** (3 + n % 2 * -20.0))):
        dy, w, q, ends = _case(L, m, c, k, experts, group, torch.float32, torch.float16, factors)
        got = _run(L, dy, w, ends, experts, c)
        want, size = _expected(dy, _values(w, q), ends, k)
        inside = (factors < 1e9)[torch.arange(c, device="cuda") // group]
        fits = inside[None] & (want.abs() < 65000)
        tol = _tolerance(want, size, k, torch.float16)
        _near(got[fits], want[fits], tol[fits])
        assert not got.isnan().any()

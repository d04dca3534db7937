"""The norm to 8-bit rows and its gradient against plain 64-bit computations.

A code is the rounding of the 64-bit value, so codes and scales have to be equal; h is
one rounding of an exact sum, equal too.  r is one rounding to 32 bits (and a few 2^-53
before it).  The gradient: 32-bit sums of c (for dgain: m) products with an error of at
most (their number) * 2^-24 of the sum of absolute products, a few roundings of 2^-24
of each term, and dx rounded to its type (half an ulp)."""
import math

import pytest
import torch

import around_sizes as sizes

pytestmark = pytest.mark.gpu

DTYPES = (torch.bfloat16, torch.float16, torch.float32)
HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module")
def L():
    from paper_2202_06819_amd import build, linear
    build.ensure_built()
    return linear


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _view(t, stride):
    """t as the first columns of a wider matrix."""
    buf = torch.full((t.shape[0], stride), 5.0, dtype=t.dtype, device="cuda")
    buf[:, :t.shape[1]] = t
    return buf[:, :t.shape[1]]


def _expected(h, gain, eps):
    """Codes, scales and r of the definition, in 64 bits."""
    h = h.double()
    r = 1.0 / (h.square().mean(1) + eps).sqrt()
    y = h * r[:, None] * gain.double()
    amax = y.abs().amax(1)
    finite = torch.isfinite(y).all(1) & (amax <= torch.finfo(torch.float32).max)
    e = torch.where(finite & (amax > 0), torch.floor(torch.log2(amax / 127)) - 1, torch.zeros_like(amax))
    for _ in range(3):
        e = torch.where(finite & (amax > 127 * torch.exp2(e)), e + 1, e)
    e = e.clamp(min=-126)
    codes = torch.where(finite[:, None], torch.round(y / torch.exp2(e)[:, None]), torch.zeros_like(y)).nan_to_num(0.0)
    scale = torch.where(amax > 0, torch.exp2(e), torch.zeros_like(e))
    return codes.to(torch.int8), torch.where(finite, scale, torch.full_like(scale, math.nan)).float(), r


def _same(got, h, gain, eps):
    codes, scale, r = _expected(h, gain, eps)
    c = h.shape[1]
    assert torch.equal(got.rows.codes[:, :c], codes)
    assert not got.rows.codes[:, c:].any()
    assert torch.equal(got.rows.scale.nan_to_num(-1.0), scale.nan_to_num(-1.0))
    fine = torch.isfinite(scale) & (r < 1e38) & (r > 1e-37)
    assert ((got.rstd.double() - r).abs() <= r * 2.0 ** -23)[fine].all()


SHAPES = [(1, 1, 1), (3, 7, 7), (5, 16, 24), (2, 511, 515), (9, 2048, 2048), (4, 2049, 2056), (3, 8192, 8192), (2, 8200, 8203),
          (1, 20001, 20001), (1, 131071, 131071), (1030, 64, 64), (300, 4096, 4096)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("m,c,stride", SHAPES)
def test_codes_are_those_of_64_bits(L, m, c, stride, residual, dtype):
    g = _gen(m * 7 + c)
    x = _view((_randn(g, m, c) * torch.exp2(torch.randint(-9, 9, (m, 1), generator=g, device="cuda").float())).to(dtype), stride)
    more = _view(_randn(g, m, c).to(dtype), stride + 3) if residual else None
    gain = (1 + 0.3 * _randn(g, c)).to(DTYPES[(m + c) % 3])
    got = L.norm_rows(x, gain, residual=more, eps=1e-5)
    h = (x.float() + more.float()).to(dtype) if residual else x
    assert torch.equal(got.sum, h) and (residual or got.sum is x)
    _same(got, h, gain, 1e-5)


@pytest.mark.parametrize("c", [40, 2056])
@pytest.mark.parametrize("dtype", DTYPES)
def test_borders(L, dtype, c):
    """Rows whose values are ties or whose largest is 127 * 2^e, exact in 64 bits (a mean
    of squares of a power of four, eps 0, gains that are powers of two), and beside them."""
    # (values are laid out so that the row's sum of squares is c times a power of four)
    x = torch.ones((8, c), device="cuda")
    gain = torch.ones(c, device="cuda")
    x[1] *= 4
    x[2, :2] = torch.tensor([0.0, math.sqrt(2.0)], device="cuda")
    x[3] = -1
    x[4] *= 2.0 ** -14
    gain[3] = 1.0 / 128          # 64 + ties at a half after scaling
    gain[4] = 3.0 / 128
    gain[5] = 1.984375           # 127 / 64
    gain[6] = -5.0 / 128
    x[5, 5] = 1.0 + 2.0 ** -7
    x[6] *= -0.25
    x[7, 6] = 0.0
    x = x.to(dtype)
    for gg in (gain, gain.to(torch.bfloat16), torch.ones_like(gain)):
        _same(L.norm_rows(x, gg, eps=0.0), x, gg, 0.0)


@pytest.mark.parametrize("c", [40, 2056, 8200])
@pytest.mark.parametrize("dtype", DTYPES)
def test_edges(L, dtype, c):
    """Zero rows, the type's extremes, infinities and NaN, in h and in the gain; eps of 0,
    tiny and huge."""
    f = torch.finfo(dtype)
    g = _gen(c)
    x = _randn(g, 12, c).to(dtype)
    x[0] = 0
    x[1, c - 1] = math.inf
    x[2, 0] = -math.inf
    x[3, c // 2] = math.nan
    x[4] = f.max
    x[5] = f.smallest_normal
    x[6] = 0
    x[6, 3] = f.max
    x[7] = 0
    x[7, c - 1] = f.smallest_normal
    x[8] = x[8] * f.smallest_normal
    x[9] = (_randn(g, c).clamp(-2, 2) * (f.max / 2)).to(dtype)
    gain = 1 + 0.1 * _randn(g, c)
    for eps in (1e-5, 1e-30, 1e20):
        got = L.norm_rows(x, gain, eps=eps)
        _same(got, x, gain, eps)
        assert got.rows.scale[0] == 0 and got.rows.scale[1:4].isnan().all()
    _same(L.norm_rows(x[1:], gain, eps=0.0), x[1:], gain, 0.0)
    assert L.norm_rows(x[:1], gain, eps=0.0).rows.scale.isnan().all()      # 0 / 0
    gain[2] = math.nan
    assert L.norm_rows(x, gain).rows.scale.isnan().all()
    gain[2] = 3e38
    _same(L.norm_rows(x[4:], gain, eps=1e-5), x[4:], gain, 1e-5)
    gain[:] = 1e-38
    _same(L.norm_rows(x[4:], gain, eps=1e-5), x[4:], gain, 1e-5)
    gain[:] = 0
    assert not L.norm_rows(x[4:], gain).rows.scale.any()


@pytest.mark.parametrize("c", [100, 4096, 9000])
def test_the_sum_in_place_and_into_views(L, c):
    g = _gen(c)
    x, more, gain = _randn(g, 6, c).bfloat16(), _randn(g, 6, c).bfloat16(), _randn(g, c)
    want = L.norm_rows(x, gain, residual=more)
    for place in ("x", "residual"):
        a, b = x.clone(), more.clone()
        got = L.norm_rows(a, gain, residual=b, sum_out=a if place == "x" else b)
        assert torch.equal(got.rows.codes, want.rows.codes) and torch.equal(got.rows.scale, want.rows.scale)
        assert torch.equal(got.sum, want.sum) and got.sum is (a if place == "x" else b)
        assert torch.equal(b if place == "x" else a, more if place == "x" else x)
    pitch = L.rows_pitch(c)
    big = torch.full((6, pitch + 64), 99, dtype=torch.int8, device="cuda")
    wide = torch.full((6, c + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    out = L.Rows(big[:, 16:16 + pitch], torch.empty(6, device="cuda"), c)
    got = L.norm_rows(x, gain, residual=more, out=out, sum_out=wide[:, 2:2 + c])
    assert got.rows is out and torch.equal(out.codes, want.rows.codes) and torch.equal(wide[:, 2:2 + c], want.sum)
    assert (big[:, :16] == 99).all() and (big[:, 16 + pitch:] == 99).all()
    assert (wide[:, :2] == 7).all() and (wide[:, 2 + c:] == 7).all()
    empty = L.norm_rows(x[:0], gain, residual=more[:0])
    assert empty.rows.codes.shape == (0, pitch) and empty.rstd.shape == (0,)


def _grad_expected(dy, h, gain, r, dsum):
    """dx, dgain and the sums of absolute values behind each."""
    dy, h, gain, r = dy.double(), h.double(), gain.double(), r.double()[:, None]
    t, n = dy * gain, h * r
    z, z_size = (t * n).mean(1, keepdim=True), (t * n).abs().mean(1, keepdim=True)
    dx = r * (t - n * z)
    size = r * (t.abs() + n.abs() * z_size)
    if dsum is not None:
        dx, size = dx + dsum.double(), size + dsum.double().abs()
    return dx, size, r * n.abs() * z_size, (dy * n).sum(0), (dy * n).abs().sum(0)


def _grad_near(got, want, m, c, dtype):
    dx, dgain = got
    x, size, along, gsum, gsize = want
    # z: c products; the rest of dx: at most eight roundings of 2^-24 of its terms
    tol = along * (c + 4) * 2.0 ** -24 + size * 8 * 2.0 ** -24
    tol = tol * (1 + HALF_ULP[dtype]) + x.abs() * HALF_ULP[dtype] + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -149)
    assert ((dx.double() - x).abs() <= tol).all(), float(((dx.double() - x).abs() / tol).max())
    assert ((dgain.double() - gsum).abs() <= gsize * (m + 4) * 2.0 ** -24 + 2.0 ** -149).all()


GRADS = [(1, 1), (2, 7), (5, 40), (3, 2048), (700, 64), (513, 2049), (40, 4096), (1200, 300), (9, 8192), (5, 8200), (515, 8199),
         (2, 131071), (3000, 1024)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("m,c", GRADS)
def test_gradient(L, m, c, residual, dtype):
    g = _gen(m + c)
    dy, h = _view((_randn(g, m, c) * 0.1).to(dtype), c + 3), _view((_randn(g, m, c) * 2).to(dtype), c + (8 if m % 2 else 0))
    gain = (1 + 0.3 * _randn(g, c)).to(DTYPES[(m + c) % 3])
    r = torch.rsqrt(h.double().square().mean(1) + 1e-5).float()
    dsum = _randn(g, m, c).to(dtype) if residual else None
    want = _grad_expected(dy, h, gain, r, dsum)
    got = L.norm_rows_grad(dy, h, gain, r, dsum=dsum)
    _grad_near(got, want, m, c, dtype)
    again = L.norm_rows_grad(dy, h, gain, r, dsum=dsum)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    if residual:   # in dsum's place
        place = dsum.clone()
        inside = L.norm_rows_grad(dy, h, gain, r, dsum=place, out=place)
        assert inside[0] is place and torch.equal(place, got[0]) and torch.equal(inside[1], got[1])


def test_gradient_of_no_rows(L):
    none = torch.empty((0, 33), dtype=torch.bfloat16, device="cuda")
    dx, dgain = L.norm_rows_grad(none, none, torch.ones(33, device="cuda"), torch.empty(0, device="cuda"))
    assert dx.shape == (0, 33) and not dgain.any()


def test_gradient_at_far_scales(L):
    """h of any size: r h is near one, and neither r^3 nor a sum of h leaves 32 bits."""
    g = _gen(3)
    for size in (1e-18, 1e-12, 1e12, 1e18):
        h = _randn(g, 20, 300) * size
        dy, gain = _randn(g, 20, 300), torch.ones(300, device="cuda")
        r = torch.rsqrt(h.double().square().mean(1)).float()
        _grad_near(L.norm_rows_grad(dy, h, gain, r), _grad_expected(dy, h, gain, r, None), 20, 300, torch.float32)


def test_one_rows_fault_stays_in_its_row(L):
    g = _gen(4)
    x, gain = _randn(g, 9, 5000).bfloat16(), _randn(g, 5000)
    clean = L.norm_rows(x, gain)
    x[4, 77] = math.nan
    got = L.norm_rows(x, gain)
    others = torch.arange(9, device="cuda") != 4
    assert torch.equal(got.rows.codes[others], clean.rows.codes[others]) and got.rows.scale[4].isnan()
    assert torch.equal(got.rows.scale[others], clean.rows.scale[others])
    dy = _randn(g, 9, 5000).bfloat16()
    dx, _ = L.norm_rows_grad(dy, got.sum, gain, got.rstd)
    dx_clean, _ = L.norm_rows_grad(dy, torch.where(others[:, None], x, torch.zeros_like(x)), gain, clean.rstd)
    assert torch.equal(dx[others], dx_clean[others])


def test_gradient_is_that_of_differences(L):
    """Central differences of the plain norm's sum of products, in 64 bits."""
    g = _gen(6)
    h, gain, dy = _randn(g, 3, 50), 1 + 0.3 * _randn(g, 50), _randn(g, 3, 50)

    def value(h, gain):
        return (h * (h.square().mean(1, keepdim=True) + 1e-3).rsqrt() * gain * dy.double()).sum()
    r = (h.double().square().mean(1) + 1e-3).rsqrt().float()
    dx, dgain = L.norm_rows_grad(dy, h, gain, r)
    step = 1e-4
    for row, col in ((0, 0), (1, 17), (2, 49)):
        move = torch.zeros_like(h, dtype=torch.float64)
        move[row, col] = step
        slope = (value(h.double() + move, gain.double()) - value(h.double() - move, gain.double())) / (2 * step)
        assert abs(dx[row, col].item() - slope.item()) < 1e-4
        move = torch.zeros(50, dtype=torch.float64, device="cuda")
        move[col] = step
        slope = (value(h.double(), gain.double() + move) - value(h.double(), gain.double() - move)) / (2 * step)
        assert abs(dgain[col].item() - slope.item()) < 1e-4


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("c", sizes.NORMS)
def test_every_kernel(L, c, residual, dtype):
    """At and past each bound of the kernels' sizes."""
    g = _gen(c)
    m = 21
    x, more = _randn(g, m, c).to(dtype), _randn(g, m, c).to(dtype) if residual else None
    gain = 1 + 0.3 * _randn(g, c)
    got = L.norm_rows(x, gain, residual=more, eps=1e-5)
    h = (x.float() + more.float()).to(dtype) if residual else x
    assert torch.equal(got.sum, h)
    _same(got, h, gain, 1e-5)
    dy = _randn(g, m, c).to(dtype)
    _grad_near(L.norm_rows_grad(dy, h, gain, got.rstd, dsum=more), _grad_expected(dy, h, gain, got.rstd, more), m, c, dtype)

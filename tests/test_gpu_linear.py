"""The linear layer on 8-bit rows against plain 64-bit computations.

Tolerances follow from the roundings alone.  Codes and their scales are exact,
so the quantiser has to be equal.  A 16-bit result is rounded once (half an ulp,
2^-8 for bfloat16 and 2^-11 for float16 of its size at most); sums are 32-bit,
with an error of at most depth * 2^-24 of the sum of absolute products, and f16
results below 2^-14 are on a grid of 2^-24.  Scales that are not powers of two
are rounded with the code (another half ulp of each product), and an adapter's
first product once to 16 bits, relative to its row's largest.
"""
import math

import pytest
import torch

import linear_sizes as sizes

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


def _expected_rows(x):
    """Codes and scales of the definition, in 64 bits."""
    x = x.double()
    amax = x.abs().amax(1)
    finite = torch.isfinite(x).all(1)
    e = torch.where(finite & (amax > 0), torch.floor(torch.log2(amax / 127)) - 1, torch.zeros_like(amax))
    for _ in range(3):
        e = torch.where(finite & (amax > 127 * torch.exp2(e)), e + 1, e)
    e = e.clamp(min=-126)
    scale = torch.exp2(e)
    codes = torch.round(x / scale[:, None])
    codes = torch.where(finite[:, None], codes, torch.zeros_like(codes))
    scale = torch.where(amax > 0, scale, torch.zeros_like(scale))
    return codes.to(torch.int8), torch.where(finite, scale, torch.full_like(scale, math.nan)).float()


def _rows8(L, g, m, c, pow2=True):
    codes = torch.zeros((m, L.rows_pitch(c)), dtype=torch.int8, device="cuda")
    codes[:, :c] = torch.randint(-127, 128, (m, c), generator=g, device="cuda").to(torch.int8)
    scale = torch.exp2(torch.randint(-9, -5, (m,), generator=g, device="cuda").float())
    if not pow2:
        scale = scale * (1 + torch.rand(m, generator=g, device="cuda"))
    return L.Rows(codes, scale, c)


def _rows4(L, g, k, c):
    q = torch.randint(-8, 8, (k, c), generator=g, device="cuda").to(torch.int8)
    scale = torch.rand(k, generator=g, device="cuda") * 0.02 + 0.005
    return L.pack_rows4(q, scale), q


def _values(rows, q=None):
    codes = rows.codes[:, :rows.channels] if q is None else q
    return codes.double() * rows.scale.double()[:, None]


def _product(x, w, q=None):
    """x times w transposed: the codes' sums (whole numbers, exact in 64 bits), then the two scales."""
    wc = (w.codes[:, :w.channels] if q is None else q).double()
    sums = x.codes[:, :x.channels].double() @ wc.t().contiguous()
    return sums * (x.scale.double()[:, None] * w.scale.double()[None])


def _near(got, want, size, depth, dtype, extra=0.0):
    """`size`: the sum of absolute products behind each result."""
    tol = size * (depth * 2.0 ** -24 + extra)
    if dtype in HALF_ULP:
        tol = tol * (1 + HALF_ULP[dtype]) + want.abs() * HALF_ULP[dtype] + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    else:
        tol = tol + want.abs() * 2.0 ** -24
    bad = (got.double() - want).abs() > tol + 1e-300
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst {((got.double() - want).abs() / tol).max():.3g}"


# ----------------------------------------------------------------- quantiser

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("m,c,stride", [(1, 1, 1), (3, 7, 7), (5, 16, 24), (2, 511, 515), (9, 2048, 2048), (4, 2049, 2056),
                                        (3, 8192, 8192), (2, 8200, 8203), (1, 20001, 20001), (1030, 64, 64)])
def test_rows_are_exact(L, dtype, m, c, stride):
    g = _gen(m * 1000 + c)
    buf = torch.full((m, stride), 7.0, dtype=dtype, device="cuda")
    buf[:, :c] = (_randn(g, m, c) * torch.exp2(torch.randint(-9, 9, (m, 1), generator=g, device="cuda").float())).to(dtype)
    x = buf[:, :c]
    rows = L.quantize_rows(x)
    codes, scale = _expected_rows(x)
    assert torch.equal(rows.codes[:, :c], codes) and torch.equal(rows.scale, scale)
    assert not rows.codes[:, c:].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_rows_at_the_edges(L, dtype):
    """Largest values at and beside 127 * 2^e, ties, the type's extremes, zeros,
    infinities and NaN."""
    f = torch.finfo(dtype)
    x = torch.zeros((14, 40), dtype=dtype, device="cuda")
    x[0, 3] = 127.0
    x[1, 3] = -127.5                     # past 127: the next scale
    x[2, :4] = torch.tensor([127.0, 0.5, 1.5, -2.5], device="cuda")   # ties to even
    x[3, :3] = torch.tensor([f.max, -f.max, f.max / 2], device="cuda")
    x[4, 39] = f.tiny
    x[5, 0] = f.smallest_normal / 4 if dtype != torch.float16 else 2.0 ** -24   # a subnormal
    x[7, 5] = math.inf
    x[8, 5] = -math.inf
    x[9, 5] = math.nan
    x[10, :] = 1.0
    x[11, 0] = 63.5
    x[12, 39] = math.nan
    x[13, 0], x[13, 1] = 64.0, -63.5
    rows = L.quantize_rows(x)
    codes, scale = _expected_rows(x)
    assert torch.equal(rows.codes[:, :40], codes)
    assert torch.equal(torch.nan_to_num(rows.scale, nan=-1.0), torch.nan_to_num(scale, nan=-1.0))
    assert rows.scale[6] == 0 and rows.scale[[7, 8, 9, 12]].isnan().all() and not rows.scale[[0, 1, 5, 10]].isnan().any()


def test_rows_into_a_view_and_nothing_else(L):
    g = _gen(5)
    x = _randn(g, 6, 50).bfloat16()
    big = torch.full((6, 128), 99, dtype=torch.int8, device="cuda")
    out = L.Rows(big[:, 16:80], torch.empty(6, device="cuda"), 50)
    assert L.quantize_rows(x, out=out) is out
    codes, _ = _expected_rows(x)
    assert torch.equal(big[:, 16:66], codes) and not big[:, 66:80].any()
    assert (big[:, :16] == 99).all() and (big[:, 80:] == 99).all()
    empty = L.quantize_rows(x[:0])
    assert empty.codes.shape == (0, 64) and empty.scale.shape == (0,)


# ------------------------------------------------------------------- forward

SHAPES = [(1, 16, 1), (1, 256, 40), (3, 48, 17), (16, 129, 64), (17, 1000, 33), (31, 128, 16), (33, 384, 200), (64, 520, 130),
          (65, 64, 129), (100, 1000, 300), (129, 2048, 257), (515, 136, 700)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,c,k", SHAPES)
def test_linear_8bit(L, m, c, k, dtype):
    g = _gen(m + c + k)
    x, w = _rows8(L, g, m, c, pow2=False), _rows8(L, g, k, c, pow2=False)
    want = _product(x, w)
    # the sum is exact; two scales and their product: three roundings
    _near(L.linear(x, w, dtype=dtype), want, want.abs(), 4, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,c,k", [(1, 8, 1), (1, 256, 40), (3, 48, 17), (16, 136, 64), (20, 1000, 33), (64, 520, 130),
                                   (65, 64, 129), (129, 2048, 257), (515, 136, 700)])
def test_linear_4bit(L, m, c, k, dtype):
    g = _gen(m + c + k)
    x, (w, q) = _rows8(L, g, m, c), _rows4(L, g, k, c)
    want = _product(x, w, q)
    _near(L.linear(x, w, dtype=dtype), want, want.abs(), 4, dtype)


@pytest.mark.parametrize("bits", [4, 8])
def test_linear_large_tiles(L, bits):
    """Sizes of the largest workgroup tiles, ragged at both ends."""
    g = _gen(bits)
    m, c, k = 3500, 328, 4100
    x = _rows8(L, g, m, c)
    w, q = _rows4(L, g, k, c) if bits == 4 else (_rows8(L, g, k, c), None)
    want = _product(x, w, q)
    _near(L.linear(x, w), want, want.abs(), 4, torch.bfloat16)


def test_linear_extreme_codes(L):
    """Sums at the bound of 32 bits: 131,071 channels of -128 times -128."""
    c = 131071
    codes = torch.zeros((2, L.rows_pitch(c)), dtype=torch.int8, device="cuda")
    codes[:, :c] = -128
    x = L.Rows(codes, torch.ones(2, device="cuda"), c)
    w = L.Rows(codes.repeat(40, 1), torch.ones(80, device="cuda"), c)
    assert (L.linear(x, w).double() == torch.tensor(128.0 * 128 * c).bfloat16().double().item()).all()
    x70 = L.Rows(codes[:1].repeat(70, 1), torch.ones(70, device="cuda"), c)
    assert (L.linear(x70, w).double() == torch.tensor(128.0 * 128 * c).bfloat16().double().item()).all()


def _adapters(L, g, n, rank, c, k, dtype):
    return L.Adapters((_randn(g, n, rank, c) * c ** -0.5).to(dtype), (_randn(g, n, k, rank) * 0.2).to(dtype),
                      torch.rand(n, generator=g, device="cuda") * 3 - 1)


def _adapter_part(x, ad, ids):
    """The adapters' part, the sum of absolute values behind it, and the bound
    of u's rounding (relative to a row's largest u) carried through B."""
    xv = _values(x)
    part = torch.zeros((xv.shape[0], ad.b.shape[1]), dtype=torch.float64, device="cuda")
    size, coarse = part.clone(), part.clone()
    for i in range(ad.a.shape[0]):
        mine = (ids == i).nonzero()[:, 0]
        if len(mine):
            a, b, f = ad.a[i].double(), ad.b[i].double(), ad.alpha[i].double()
            u = xv[mine] @ a.t().contiguous()
            part[mine] = f * (u @ b.t().contiguous())
            size[mine] = f.abs() * ((xv[mine].abs() @ a.abs().t().contiguous()) @ b.abs().t().contiguous())
            coarse[mine] = f.abs() * u.abs().amax(1, keepdim=True) * b.abs().sum(1)[None]
    return part, size, coarse


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,c,k,n,rank,bits", [
    (1, 64, 40, 3, 8, 8), (5, 256, 33, 2, 16, 4), (16, 4096, 64, 16, 16, 8), (30, 136, 50, 7, 24, 8),
    (64, 1000, 130, 40, 64, 4), (48, 512, 96, 1, 128, 8), (70, 264, 140, 5, 40, 8), (200, 512, 300, 9, 16, 4),
    (333, 136, 200, 3, 120, 8)])
def test_linear_with_adapters(L, m, c, k, n, rank, bits, dtype):
    g = _gen(m + c + k + n)
    x = _rows8(L, g, m, c)
    w, q = _rows4(L, g, k, c) if bits == 4 else (_rows8(L, g, k, c), None)
    ad = _adapters(L, g, n, rank, c, k, dtype)
    ids = torch.randint(-1, n, (m,), generator=g, device="cuda", dtype=torch.int32)
    base = _product(x, w, q)
    part, size, coarse = _adapter_part(x, ad, ids)
    y = L.linear(x, w, dtype=dtype, adapters=ad, row_adapter=ids)
    want = base + part
    tol = (HALF_ULP[dtype] * (coarse + want.abs()) * 1.01 + size * (c + rank + 8) * 2.0 ** -24 + base.abs() * 2.0 ** -22
           + (2.0 ** -25 if dtype == torch.float16 else 0.0))
    assert ((y.double() - want).abs() <= tol).all()
    none = torch.full_like(ids, -1)
    none[::2] = n                         # past the last adapter: none as well
    assert torch.equal(L.linear(x, w, dtype=dtype, adapters=ad, row_adapter=none), L.linear(x, w, dtype=dtype))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,c,k,n,rank,bits", [
    (1, 256, 40, 2, 16, 4), (5, 512, 33, 2, 24, 8), (40, 1000, 130, 7, 64, 8), (48, 512, 96, 1, 128, 8), (70, 264, 140, 5, 40, 4),
    (200, 512, 300, 9, 16, 4), (250, 8200, 4000, 6, 72, 4), (250, 2056, 4000, 3, 128, 8), (385, 264, 8200, 12, 40, 4),
    (1500, 264, 4100, 6, 128, 8), (3329, 200, 4100, 4, 72, 8)])
def test_an_adapters_first_product_keeps_more_than_16_bits(L, m, c, k, n, rank, bits, dtype):
    """u goes to the second product as two 16-bit parts: each rounding leaves half an
    ulp of its part, so what both leave is the square of it, relative to the row's
    largest u (f16: or half of its smallest subnormal, where that is more)."""
    g = _gen(m + c + k + n + 1)
    x = _rows8(L, g, m, c)
    w, q = _rows4(L, g, k, c) if bits == 4 else (_rows8(L, g, k, c), None)
    w.scale.mul_(2.0 ** -8)   # the adapters' part is the larger one
    ad = _adapters(L, g, n, rank, c, k, dtype)
    ids = torch.randint(0, n, (m,), generator=g, device="cuda", dtype=torch.int32)
    base = _product(x, w, q)
    part, size, coarse = _adapter_part(x, ad, ids)
    want = base + part
    y = L.linear(x, w, dtype=dtype, adapters=ad, row_adapter=ids)
    tol = (coarse * (HALF_ULP[dtype] ** 2 + 2.0 ** -24) + size * (c + 2 * rank + 8) * 2.0 ** -24 + base.abs() * 2.0 ** -22) * 1.01
    tol = tol + HALF_ULP[dtype] * want.abs() + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    assert ((y.double() - want).abs() <= tol).all()


def test_linear_large_tiles_with_adapters(L):
    g = _gen(77)
    m, c, k, n, rank = 3329, 200, 4100, 4, 16
    x, w = _rows8(L, g, m, c), _rows8(L, g, k, c)
    ad = _adapters(L, g, n, rank, c, k, torch.bfloat16)
    ids = (torch.arange(m, device="cuda") // 700 - 1).to(torch.int32)
    base = _product(x, w)
    part, size, coarse = _adapter_part(x, ad, ids)
    y = L.linear(x, w, adapters=ad, row_adapter=ids)
    tol = 2.0 ** -8 * (coarse + (base + part).abs()) * 1.01 + size * (c + rank + 8) * 2.0 ** -24 + base.abs() * 2.0 ** -22
    assert ((y.double() - base - part).abs() <= tol).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,c,k,n,rank,bits", [
    (250, 8200, 4000, 6, 72, 4), (129, 8200, 4100, 40, 16, 8), (250, 2056, 4000, 3, 128, 8), (161, 2056, 4001, 30, 24, 4),
    (385, 264, 8200, 12, 40, 4), (700, 264, 8200, 300, 8, 8), (100, 1160, 8000, 64, 64, 8)])
def test_linear_with_long_rows_and_middling_many(L, m, c, k, n, rank, bits, dtype):
    """Too few tiles to fill the chip: steps and adapters are dealt to groups of waves."""
    g = _gen(m + c + k + n)
    x = _rows8(L, g, m, c)
    w, q = _rows4(L, g, k, c) if bits == 4 else (_rows8(L, g, k, c), None)
    base = _product(x, w, q)
    _near(L.linear(x, w, dtype=dtype), base, base.abs(), 4, dtype)
    ad = _adapters(L, g, n, rank, c, k, dtype)
    ids = torch.randint(-1, n, (m,), generator=g, device="cuda", dtype=torch.int32)
    part, size, coarse = _adapter_part(x, ad, ids)
    want = base + part
    tol = (HALF_ULP[dtype] * (coarse + want.abs()) * 1.01 + size * (c + rank + 8) * 2.0 ** -24 + base.abs() * 2.0 ** -22
           + (2.0 ** -25 if dtype == torch.float16 else 0.0))
    y = L.linear(x, w, dtype=dtype, adapters=ad, row_adapter=ids)
    assert ((y.double() - want).abs() <= tol).all()
    # a row's scale and an adapter that are not finite reach only the rows that use them
    x.scale[3] = math.nan
    ad.a[1].fill_(math.inf)
    ad.b[1].fill_(math.inf)
    hit = (ids == 1) | (torch.arange(m, device="cuda") == 3)
    z = L.linear(x, w, dtype=dtype, adapters=ad, row_adapter=ids)
    assert torch.equal(z[~hit], y[~hit]) and not torch.isfinite(z[hit]).any()


@pytest.mark.parametrize("m", [8, 80])
def test_one_rows_fault_stays_in_its_row(L, m):
    """A row with a NaN scale, and an adapter with infinite weights, reach only
    the rows that use them."""
    g = _gen(m)
    c, k = 128, 48
    x, w = _rows8(L, g, m, c), _rows8(L, g, k, c)
    ad = _adapters(L, g, 3, 8, c, k, torch.bfloat16)
    ids = (torch.arange(m, device="cuda") % 3).to(torch.int32)
    clean = L.linear(x, w, adapters=ad, row_adapter=ids)
    x.scale[3] = math.nan
    ad.a[1].fill_(math.inf)
    ad.b[1].fill_(math.inf)
    y = L.linear(x, w, adapters=ad, row_adapter=ids)
    hit = (ids == 1) | (torch.arange(m, device="cuda") == 3)
    assert torch.equal(y[~hit], clean[~hit]) and not torch.isfinite(y[hit]).any()


def test_no_rows_with_adapters(L):
    g = _gen(3)
    x, w = _rows8(L, g, 4, 64), _rows8(L, g, 24, 64)
    ad = _adapters(L, g, 2, 8, 64, 24, torch.bfloat16)
    none = L.Rows(x.codes[:0], x.scale[:0], 64)
    y = L.linear(none, w, adapters=ad, row_adapter=torch.empty(0, dtype=torch.int32, device="cuda"))
    assert y.shape == (0, 24)


def test_linear_into_a_strided_view(L):
    g = _gen(3)
    for m, k in ((5, 20), (90, 150)):
        x, w = _rows8(L, g, m, 96), _rows8(L, g, k, 96)
        big = torch.full((m, k + 31), 5.0, dtype=torch.bfloat16, device="cuda")
        L.linear(x, w, out=big[:, 3:3 + k])
        assert torch.equal(big[:, 3:3 + k], L.linear(x, w))
        assert (big[:, :3] == 5).all() and (big[:, 3 + k:] == 5).all()
    none = L.Rows(x.codes[:0], x.scale[:0], 96)
    assert L.linear(none, w).shape == (0, 150)


# ------------------------------------------------------------------ backward

GRADS = [(1, 16, 1), (1, 200, 33), (7, 48, 64), (64, 64, 64), (65, 131, 70), (130, 1000, 257), (300, 129, 1001), (1000, 72, 40)]


def _dy(g, m, k, dtype, stride=0, at=0):
    buf = torch.full((m, (stride or k) + at), math.nan, dtype=dtype, device="cuda")
    dy = buf[:, at:at + k]
    dy.copy_(_randn(g, m, k) * torch.exp2(torch.randint(-4, 3, (m, 1), generator=g, device="cuda").float()))
    dy[m // 2] = 0
    return dy


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["tight", "aligned", "odd"])
@pytest.mark.parametrize("m,c,k", GRADS)
def test_grad_input_8bit(L, m, c, k, layout, dtype):
    g = _gen(m + c + k)
    stride, at = {"tight": (k, 0), "aligned": ((k + 15) // 8 * 8, 8), "odd": (k + 3, 1)}[layout]
    dy, w = _dy(g, m, k, dtype, stride, at), _rows8(L, g, k, c)
    want = dy.double().contiguous() @ _values(w)
    size = dy.double().abs().contiguous() @ _values(w).abs()
    _near(L.linear_grad_input(dy, w), want, size, k, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,c,k", [(1, 8, 1), (3, 40, 33), (65, 136, 70), (130, 1000, 256), (300, 264, 1001)])
def test_grad_input_4bit_any_scale(L, m, c, k, dtype):
    g = _gen(m + c + k)
    dy, (w, q) = _dy(g, m, k, dtype), _rows4(L, g, k, c)
    want = dy.double().contiguous() @ _values(w, q)
    size = dy.double().abs().contiguous() @ _values(w, q).abs()
    _near(L.linear_grad_input(dy, w), want, size, k, dtype, extra=HALF_ULP[dtype] * 1.01)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["tight", "aligned", "odd"])
@pytest.mark.parametrize("m,c,k", GRADS + [(5000, 96, 72)])
def test_grad_weight(L, m, c, k, layout, dtype):
    g = _gen(m + c + k)
    stride, at = {"tight": (k, 0), "aligned": ((k + 15) // 8 * 8, 8), "odd": (k + 3, 1)}[layout]
    dy, x = _dy(g, m, k, dtype, stride, at), _rows8(L, g, m, c)
    want = dy.double().t().contiguous() @ _values(x)
    size = dy.double().abs().t().contiguous() @ _values(x).abs()
    _near(L.linear_grad_weight(dy, x), want, size, m, torch.float32)


@pytest.mark.parametrize("dtype", DTYPES)
def test_grads_large_tiles(L, dtype):
    """Sizes of the largest workgroup tiles, ragged at both ends."""
    g = _gen(11)
    m, c, k = 3600, 4000, 392
    dy, w = _dy(g, m, k, dtype), _rows8(L, g, k, c)
    want, size = dy.double() @ _values(w), dy.double().abs() @ _values(w).abs()
    _near(L.linear_grad_input(dy, w), want, size, k, dtype)
    m, c, k = 333, 4005, 3602
    dy, x = _dy(g, m, k, dtype), _rows8(L, g, m, c)
    want, size = dy.double().t().contiguous() @ _values(x), dy.double().abs().t().contiguous() @ _values(x).abs()
    _near(L.linear_grad_weight(dy, x), want, size, m, torch.float32)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bits", [4, 8])
def test_grads_large_tiles_of_any_alignment(L, bits, dtype):
    g = _gen(12 + bits)
    m, c, k = 1541, 2712 if bits == 4 else 2710, 5113   # (4-bit rows have multiples of 8 channels)
    dy = _dy(g, m, k, dtype, k + 4, 3)
    if bits == 4:
        w, q = _rows4(L, g, k, c)
        values, extra = _values(w, q), HALF_ULP[dtype] * 1.01
    else:
        w = _rows8(L, g, k, c)
        values, extra = _values(w), 0.0
    want, size = dy.double().contiguous() @ values, dy.double().abs().contiguous() @ values.abs()
    _near(L.linear_grad_input(dy, w), want, size, k, dtype, extra=extra)
    m, c, k = 4111, 2690, 3001
    dy, x = _dy(g, m, k, dtype, k + 2, 1), _rows8(L, g, m, c)
    want, size = dy.double().t().contiguous() @ _values(x), dy.double().abs().t().contiguous() @ _values(x).abs()
    _near(L.linear_grad_weight(dy, x), want, size, m, torch.float32)


@pytest.mark.parametrize("m,c,k", [(128, 1024, 700), (1000, 1010, 2630), (70, 4000, 1001), (500, 640, 90)])
@pytest.mark.parametrize("odd", [0, 3])
def test_an_infinity_in_the_gradient_stays_one(L, m, c, k, odd):
    """An infinite value of dy reaches its row (of dw: its column's row) as that
    infinity times the codes, wherever the summed axis was cut, and no other row."""
    g = _gen(m + k)
    dy, w, x = _dy(g, m, k, torch.bfloat16, k + odd), _rows8(L, g, k, c), _rows8(L, g, m, c)
    for rows in (w, x):
        rows.codes[:, :c][rows.codes[:, :c] == 0] = 1
    clean = L.linear_grad_input(dy, w), L.linear_grad_weight(dy, x)
    hits = ((5, 3), (m - 1, k - 1))
    for i, j in hits:
        dy[i, j] = math.inf
    dx, dw = L.linear_grad_input(dy, w), L.linear_grad_weight(dy, x)
    for i, j in hits:
        assert torch.equal(dx[i].float(), math.inf * w.codes[j, :c].float())
        assert torch.equal(dw[j], math.inf * x.codes[i, :c].float())
    rest_x = [i for i in range(m) if i not in (5, m - 1)]
    rest_w = [j for j in range(k) if j not in (3, k - 1)]
    assert torch.equal(dx[rest_x], clean[0][rest_x]) and torch.equal(dw[rest_w], clean[1][rest_w])


def test_f16_gradients_at_far_scales(L):
    """Row scales far from one, and far from each other: f16 products are formed
    about the largest scale."""
    g = _gen(2)
    m, c, k = 96, 64, 80
    dy = _dy(g, m, k, torch.float16)
    for shift in (-30, 0, 12):
        x = _rows8(L, g, m, c)
        x = L.Rows(x.codes, x.scale * 2.0 ** shift * torch.exp2(-torch.arange(m, device="cuda") % 8.0), c)
        want = dy.double().t().contiguous() @ _values(x)
        size = dy.double().abs().t().contiguous() @ _values(x).abs()
        _near(L.linear_grad_weight(dy, x), want, size, m, torch.float32)
    zero = L.Rows(x.codes, torch.zeros_like(x.scale), c)
    assert not L.linear_grad_weight(dy, zero).any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("top", [1.0, 1.998, 1.999, 1.9995, 1.9998, 2.0 - 2.0 ** -23])
@pytest.mark.parametrize("shift", [-100, -9, 110])
@pytest.mark.parametrize("m", [70, 300])
def test_gradients_of_the_largest_codes(L, m, shift, top, dtype):
    """Codes of -128 under scales up to the next power of two: finite operands give
    finite gradients.  The code times its scale is rounded once (half an ulp)."""
    g = _gen(m + shift)
    c, k = 48, 40
    dy = _dy(g, m, k, dtype)
    for rows in (_rows8(L, g, m, c), _rows8(L, g, k, c)):
        rows.codes[:, :c][torch.rand(rows.codes.shape[0], c, generator=g, device="cuda") < 0.2] = -128
        rows.scale.copy_(top * torch.exp2(shift - torch.randint(0, 3, (len(rows.scale),), generator=g, device="cuda").float()))
        values = _values(rows)
        if len(rows.scale) == m:
            want, size = dy.double().t().contiguous() @ values, dy.double().abs().t().contiguous() @ values.abs()
            _near(L.linear_grad_weight(dy, rows), want, size, m, torch.float32, extra=HALF_ULP[dtype] * 1.01 + 2.0 ** -23)
        elif shift == -9:   # (a 16-bit result)
            want, size = dy.double() @ values, dy.double().abs() @ values.abs()
            _near(L.linear_grad_input(dy, rows), want, size, k, dtype, extra=HALF_ULP[dtype] * 1.01 + 2.0 ** -23)


@pytest.mark.parametrize("scale", [2.0 ** 127, 1.9999 * 2.0 ** 127])
def test_f16_gradients_at_the_largest_scales(L, scale):
    """A code times such a scale passes 32 bits, its product with a small gradient does not."""
    g = _gen(8)
    m, c, k = 20, 32, 24
    x = _rows8(L, g, m, c)
    x.scale.fill_(scale)
    dy = (2.0 ** -14 * (1 + torch.rand(m, k, generator=g, device="cuda")) * torch.sign(_randn(g, m, k))).half()
    want = dy.double().t().contiguous() @ _values(x)
    size = dy.double().abs().t().contiguous() @ _values(x).abs()
    assert size.max() < 2.0 ** 127
    _near(L.linear_grad_weight(dy, x), want, size, m, torch.float32, extra=HALF_ULP[torch.float16] * 1.01)


@pytest.mark.parametrize("k", [24, 25])
def test_grad_weight_of_no_rows_is_zero(L, k):
    x = L.Rows(torch.empty((0, 48), dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda"), 40)
    dw = torch.full((k, 40), 3.0, device="cuda")
    L.linear_grad_weight(torch.empty((0, k), dtype=torch.bfloat16, device="cuda"), x, out=dw)
    assert not dw.any()


def test_grads_repeat_bit_for_bit(L):
    """Split sums are added in a fixed order."""
    g = _gen(9)
    dy, x = _dy(g, 9000, 64, torch.bfloat16), _rows8(L, g, 9000, 64)
    assert L.grad_workspace_bytes(64, 64, 9000) > 0
    first = L.linear_grad_weight(dy, x)
    for _ in range(4):
        assert torch.equal(L.linear_grad_weight(dy, x), first)


def test_grads_are_the_forward_products_differences(L):
    """The layer is linear in each operand's values, so a central difference of
    the forward product (in 64 bits, of the very codes) is its gradient."""
    g = _gen(21)
    m, c, k = 12, 40, 24
    x, w, dy = _rows8(L, g, m, c), _rows8(L, g, k, c), _dy(g, m, k, torch.bfloat16)
    loss = lambda xv, wv: float(((xv @ wv.t()) * dy.double()).sum())   # noqa: E731
    xv, wv = _values(x), _values(w)
    dx, dw = L.linear_grad_input(dy, w).double(), L.linear_grad_weight(dy, x).double()
    for grad, which in ((dx, 0), (dw, 1)):
        for i, j in ((0, 0), (3, 17), (11, 39), (5, 8)):
            h = torch.zeros_like((xv, wv)[which])
            h[i, j] = 0.5
            args = [(xv + h, wv), (xv - h, wv)] if which == 0 else [(xv, wv + h), (xv, wv - h)]
            diff = loss(*args[0]) - loss(*args[1])
            scale = float((dy.double().abs() @ wv.abs())[i, j] if which == 0 else (dy.double().abs().t() @ xv.abs())[i, j])
            assert abs(diff - float(grad[i, j])) <= scale * 2.0 ** -8


# --------------------------------------------------- every kernel, in every form

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,c,k,bits,n,rank", sizes.LINEAR)
def test_every_kernel_of_the_projection(L, m, c, k, bits, n, rank, dtype):
    g = _gen(m + c + k + rank)
    x = _rows8(L, g, m, c)
    w, q = _rows4(L, g, k, c) if bits == 4 else (_rows8(L, g, k, c), None)
    base = _product(x, w, q)
    if not n:
        _near(L.linear(x, w, dtype=dtype), base, base.abs(), 4, dtype)
        return
    ad = _adapters(L, g, n, rank, c, k, dtype)
    ids = torch.randint(-1, n, (m,), generator=g, device="cuda", dtype=torch.int32)
    part, size, coarse = _adapter_part(x, ad, ids)
    want = base + part
    y = L.linear(x, w, dtype=dtype, adapters=ad, row_adapter=ids)
    tol = (coarse * (HALF_ULP[dtype] ** 2 + 2.0 ** -24) + size * (c + 2 * rank + 8) * 2.0 ** -24 + base.abs() * 2.0 ** -22) * 1.01
    tol = tol + HALF_ULP[dtype] * want.abs() + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    assert ((y.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,c,k,bits", sizes.GRAD_INPUT)
def test_every_kernel_of_the_input_gradient(L, m, c, k, bits, dtype):
    g = _gen(m + c + k + bits)
    dy = _dy(g, m, k, dtype, k + 8)
    if bits == 4:
        w, q = _rows4(L, g, k, c)
        values, extra = _values(w, q), HALF_ULP[dtype] * 1.01
    else:
        w = _rows8(L, g, k, c)
        values, extra = _values(w), 0.0
    want, size = dy.double().contiguous() @ values, dy.double().abs().contiguous() @ values.abs()
    _near(L.linear_grad_input(dy, w), want, size, k, dtype, extra=extra)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,c,k", sizes.GRAD_WEIGHT)
def test_every_kernel_of_the_weight_gradient(L, m, c, k, dtype):
    g = _gen(m + c + k)
    dy, x = _dy(g, m, k, dtype, k + 8), _rows8(L, g, m, c)
    want, size = dy.double().t().contiguous() @ _values(x), dy.double().abs().t().contiguous() @ _values(x).abs()
    _near(L.linear_grad_weight(dy, x), want, size, m, torch.float32)


# ----------------------------------------------------- streams, graphs, layer

def test_other_streams_and_graphs(L):
    """Every operator on a stream of its own, and captured: replays with other
    work between them equal the eager results."""
    g = _gen(31)
    m, c, k = 40, 256, 96
    x = _randn(g, m, c).bfloat16()
    w = L.quantize_rows(_randn(g, k, c))
    ad = _adapters(L, g, 4, 16, c, k, torch.bfloat16)
    ids = torch.randint(-1, 4, (m,), generator=g, device="cuda", dtype=torch.int32)
    dy = _dy(g, m, k, torch.bfloat16)

    def step(stream=None):
        x8 = L.quantize_rows(x, stream=stream)
        y = L.linear(x8, w, adapters=ad, row_adapter=ids, stream=stream)
        return x8.codes, y, L.linear_grad_input(dy, w, stream=stream), L.linear_grad_weight(dy, x8, stream=stream)

    eager = [t.clone() for t in step()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = step()
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(eager, other))
    given = step(stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, given))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for _ in range(4):
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, outs))
        (x.float() @ x.float().t()).sum().item()


@pytest.mark.parametrize("op", ["quantize_rows", "linear", "linear_grad_input", "linear_grad_weight", "split"])
def test_a_given_streams_results_do_not_meet_the_current_streams_memory(L, op):
    """A call on another stream is not ordered after the current one: what it makes must
    not lie in memory that was freed there while work on it is still queued, nor the
    other way round, when a result that the current stream still reads is given back."""
    g = _gen(61)
    m, c, k = (4096, 1024, 1024) if op != "split" else (16384, 512, 512)
    x, w = _rows8(L, g, m, c), _rows8(L, g, k, c)
    v = _randn(g, m, c).bfloat16()
    dy = _dy(g, m, k, torch.bfloat16)
    call = {"quantize_rows": lambda **on: L.quantize_rows(v, **on).codes,
            "linear": lambda **on: L.linear(x, w, **on),
            "linear_grad_input": lambda **on: L.linear_grad_input(dy, w, **on),
            "linear_grad_weight": lambda **on: L.linear_grad_weight(dy, x, **on),
            "split": lambda **on: L.linear_grad_weight(dy, x, **on)}[op]
    assert op != "split" or L.grad_workspace_bytes(k, c, m) > 0
    want = call()
    held = L.grad_workspace_bytes(k, c, m) if op == "split" else want.numel() * want.element_size()
    s, current = torch.cuda.Stream(), torch.cuda.current_stream()
    call(stream=s)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    # freed on the current stream, read there later
    old = torch.full((held,), 77, dtype=torch.uint8, device="cuda")
    read = torch.empty_like(old)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    read.copy_(old)
    del old
    got = call(stream=s)
    s.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and (read == 77).all()
    # a result read on the current stream, and given back
    again = call(stream=s)
    current.wait_stream(s)
    torch.cuda._sleep(200_000_000)
    copy = again.clone()
    del again, got
    with torch.cuda.stream(s):
        other = torch.full((want.numel() * want.element_size(),), 99, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    assert torch.equal(copy, want) and (other == 99).all()


def test_a_stream_as_a_raw_handle(L):
    g = _gen(62)
    x, w = _rows8(L, g, 70, 256), _rows8(L, g, 40, 256)
    want = L.linear(x, w)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (s, s.cuda_stream, torch.cuda.default_stream().cuda_stream):
        got = L.linear(x, w, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


@pytest.mark.parametrize("c", [256, 264])
@pytest.mark.parametrize("contiguous", [True, False])
def test_pack_rows4_on_a_given_stream(L, c, contiguous):
    """All of the packing runs on the stream that was given, whatever the current one
    is busy with, and its result is not memory that is still in use there."""
    g = _gen(c)
    k = 3000
    codes = torch.randint(-8, 8, (k, c + 8), generator=g, device="cuda").to(torch.int8)[:, :c]
    codes = codes.contiguous() if contiguous else codes
    scale = torch.ones(k, device="cuda")
    want = L.pack_rows4(codes, scale)
    s = torch.cuda.Stream()
    L.pack_rows4(codes, scale, stream=s)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    old = torch.full((want.codes.numel() * 4,), 77, dtype=torch.uint8, device="cuda")
    read = torch.empty_like(old)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    read.copy_(old)
    del old
    got = L.pack_rows4(codes, scale, stream=s)
    with torch.cuda.stream(s):
        copy = got.codes.clone()
        torch.full((k * 288,), 99, dtype=torch.uint8, device="cuda")   # (the padded codes' size: theirs, if given back)
    s.synchronize()
    assert torch.equal(copy, want.codes)
    torch.cuda.synchronize()
    assert (read == 77).all()


@pytest.mark.parametrize("op", ["quantize_rows", "linear", "linear_grad_input", "linear_grad_weight", "pack_rows4"])
def test_operands_are_kept_until_a_given_stream_has_read_them(L, op):
    """What a call on another stream reads may be given back on the current one right
    after the call: its memory is not used again before the call has run."""
    g = _gen(63)
    m, c, k = 2048, 512, 512
    x, w, v, dy = _rows8(L, g, m, c), _rows8(L, g, k, c), _randn(g, m, c).bfloat16(), _dy(g, m, k, torch.bfloat16)
    ad = _adapters(L, g, 2, 16, c, k, torch.bfloat16)
    ids = torch.randint(-1, 2, (m,), generator=g, device="cuda", dtype=torch.int32)
    calls = {"quantize_rows": ([v], lambda t, **on: L.quantize_rows(*t, **on).codes),
             "linear": ([x.codes, x.scale, w.codes, w.scale, *ad, ids],
                        lambda t, **on: L.linear(L.Rows(t[0], t[1], c), L.Rows(t[2], t[3], c),
                                                 adapters=L.Adapters(*t[4:7]), row_adapter=t[7], **on)),
             "linear_grad_input": ([dy, w.codes, w.scale],
                                   lambda t, **on: L.linear_grad_input(t[0], L.Rows(*t[1:], c), **on)),
             "linear_grad_weight": ([dy, x.codes, x.scale],
                                    lambda t, **on: L.linear_grad_weight(t[0], L.Rows(*t[1:], c), **on)),
             "pack_rows4": ([x.codes, x.scale], lambda t, **on: L.pack_rows4(*t, **on).codes)}
    operands, call = calls[op]
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


def test_a_given_stream_within_a_capture(L):
    """A captured step whose calls are given a stream that forks from the capturing one
    and joins it again: replays, with other work between them, equal the eager results."""
    g = _gen(64)
    m, c, k = 70, 256, 96
    v, w, dy = _randn(g, m, c).bfloat16(), _rows8(L, g, k, c), _dy(g, m, k, torch.bfloat16)
    q = torch.randint(-8, 8, (k, 264), generator=g, device="cuda").to(torch.int8)
    ad = _adapters(L, g, 3, 16, c, k, torch.bfloat16)
    ids = torch.randint(-1, 3, (m,), generator=g, device="cuda", dtype=torch.int32)

    def step(**on):
        x = L.quantize_rows(v, **on)
        return (x.codes, L.linear(x, w, adapters=ad, row_adapter=ids, **on), L.linear_grad_input(dy, w, **on),
                L.linear_grad_weight(dy, x, **on), L.pack_rows4(q, w.scale, **on).codes)

    eager = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    step(stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        outs = step(stream=side)
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(4):
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, outs))
        (v.float() @ v.float().t()).sum().item()


@pytest.mark.parametrize("dtype", DTYPES)
def test_layer_trains(L, dtype):
    """The differentiable layer: gradients of the rounded product, and a few
    steps that lower a loss."""
    g = _gen(41)
    x = _randn(g, 3, 40, 96).to(dtype).requires_grad_()
    w = (_randn(g, 72, 96) * 0.1).requires_grad_()
    y = L.linear_layer(x, w)
    assert y.shape == (3, 40, 72) and y.dtype == dtype
    dy = _randn(g, 3, 40, 72).to(dtype)
    y.backward(dy)
    x8, w8 = L.quantize_rows(x.detach().reshape(-1, 96)), L.quantize_rows(w.detach())
    assert torch.equal(x.grad.reshape(-1, 96), L.linear_grad_input(dy.reshape(-1, 72), w8))
    assert torch.equal(w.grad, L.linear_grad_weight(dy.reshape(-1, 72), x8))
    target = _randn(g, 3, 40, 72)
    losses = []
    for _ in range(20):
        w.grad = None
        loss = (L.linear_layer(x.detach(), w).float() - target).square().mean()
        loss.backward()
        losses.append(loss.item())
        with torch.no_grad():
            w -= 20.0 * w.grad
    assert losses[-1] < losses[0] * 0.8


@pytest.mark.parametrize("form", ["broadcast", "columns", "far rows", "weights"])
def test_layer_takes_any_view(L, form):
    """Views whose rows the operators do not read in place are copied by the layer: the
    same results and gradients as of the tensors themselves."""
    g = _gen(43)
    w = (_randn(g, 72, 96) * 0.1).bfloat16()
    if form == "broadcast":
        x = _randn(g, 1, 96).bfloat16().expand(40, 96)
    elif form == "columns":
        x = _randn(g, 96, 40).bfloat16().t()
    elif form == "far rows":
        x = torch.as_strided(_randn(g, (1 << 22) + 96).bfloat16(), (2, 96), (1 << 22, 1))
    else:
        x, w = _randn(g, 40, 96).bfloat16(), w.t().contiguous().t()
    dy = _randn(g, x.shape[0], 72).bfloat16()
    x, w = x.detach().requires_grad_(), w.detach().requires_grad_()
    plain = [t.detach().clone(memory_format=torch.contiguous_format).requires_grad_() for t in (x, w)]
    y, want = L.linear_layer(x, w), L.linear_layer(*plain)
    assert torch.equal(y, want)
    y.backward(dy)
    want.backward(dy)
    assert torch.equal(x.grad, plain[0].grad) and torch.equal(w.grad, plain[1].grad)
    with pytest.raises(L.QConvError):
        L.linear_layer(plain[0], plain[1][0])


def test_layer_keeps_only_bytes(L):
    x = torch.randn(64, 128, device="cuda").bfloat16().requires_grad_()
    w = torch.randn(32, 128, device="cuda").requires_grad_()
    kept = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t) or t, lambda t: t):
        L.linear_layer(x, w)
    assert sum(t.numel() * t.element_size() for t in kept) == 64 * 128 + 64 * 4 + 32 * 128 + 32 * 4


# ------------------------------------------------------------------ refusals

def test_refusals_of_tensors(L):
    g = _gen(1)
    x, w = _rows8(L, g, 4, 64), _rows8(L, g, 24, 64)
    dy = _dy(g, 4, 24, torch.bfloat16)
    ad = _adapters(L, g, 2, 8, 64, 24, torch.bfloat16)
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    y = L.linear(x, w)
    bad = [
        lambda: L.quantize_rows(torch.zeros(4, 8, dtype=torch.float64, device="cuda")),
        lambda: L.quantize_rows(torch.zeros(4, 8)),
        lambda: L.quantize_rows(torch.zeros(8, 4, device="cuda").t()),
        lambda: L.quantize_rows(torch.zeros(8, device="cuda")),
        lambda: L.linear(x, w, dtype=torch.float32),
        lambda: L.linear(x, _rows8(L, g, 24, 48)),
        lambda: L.linear(w._replace(bits=4), w),
        lambda: L.linear(x._replace(scale=x.scale.double()), w),
        lambda: L.linear(x._replace(codes=x.codes[:, :60]), w),
        lambda: L.linear(x._replace(codes=x.codes.cpu()), w),
        lambda: L.linear(x, w, out=y[:, :20]),
        lambda: L.linear(x, w, out=y.float()),
        lambda: L.linear(x, w, row_adapter=ids),
        lambda: L.linear(x, w, adapters=ad),
        lambda: L.linear(x, w, adapters=ad, row_adapter=ids.long()),
        lambda: L.linear(x, w, adapters=ad, row_adapter=ids[:3]),
        lambda: L.linear(x, w, dtype=torch.float16, adapters=ad, row_adapter=ids),
        lambda: L.linear(x, w, adapters=ad._replace(a=ad.a[:, :4].contiguous(), b=ad.b[:, :, :4].contiguous()), row_adapter=ids),
        lambda: L.linear(x, w, adapters=ad, row_adapter=ids, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")),
        lambda: L.linear_grad_input(dy.float(), w),
        lambda: L.linear_grad_input(dy[:, :20], w),
        lambda: L.linear_grad_input(dy.expand(4, 24).t(), w),
        lambda: L.linear_grad_input(dy[:1].expand(4, 24), w),
        lambda: L.linear_grad_weight(dy[:3], x),
        lambda: L.linear_grad_weight(dy, x, out=torch.empty(24, 64, dtype=torch.bfloat16, device="cuda")),
        lambda: L.pack_rows4(torch.zeros(4, 12, dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(L.QConvError):
            call()
            pytest.fail(f"case {i} was accepted")


# ------------------------------------------------------------------- example

def test_demo_trains_and_serves():
    """The operators together: the loss falls, half the bytes are kept, and the
    served block is the 64-bit one but for the two 8-bit roundings of its
    activations (each at most half a step of 1/64 of a row's largest, so about 1 %
    of a normal row) and bfloat16."""
    from paper_2202_06819_amd import linear_demo
    got = linear_demo.main(width=128, hidden=256, rows=512, steps=30)
    assert got["last_loss"] < 0.8 * got["first_loss"]
    assert got["kept_bytes"] < 0.55 * got["bytes_in_16_bits"]
    assert got["serving_error"] < 0.05

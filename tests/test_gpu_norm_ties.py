"""The norm's codes where a value lies on a tie, or a row's largest on the border of a scale.

Rows of one magnitude n, with eps 0: the mean of squares is n^2, exact in 64 bits for every
length here, r is 1 / n and y = h r gain is the gain itself, with the value's sign, however
the row is long.  So codes and scales are known without any rounding."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = (torch.bfloat16, torch.float16, torch.float32)
LENGTHS = (1, 3, 7, 40, 48, 100, 777, 1000, 2040, 3000, 5003, 9001, 20001)
SIZES = (1.0, 3.0, 5.0, 7.0, 1.25, 11.0, 13.0, 49.0, 0.375, 103.0, 107.0, 161.0, 197.0)   # (few bits: exact in every type)


@pytest.fixture(scope="module")
def L():
    from paper_2202_06819_amd import build, linear
    build.ensure_built()
    return linear


@pytest.mark.parametrize("top", [127.0, 100.0])
@pytest.mark.parametrize("c", LENGTHS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_values_on_ties(L, dtype, c, top):
    """Gains n + 1/2 under a scale of one: halves go to the even neighbour.  The largest is
    the scale's border, 127 exactly, or well inside."""
    g = torch.Generator(device="cuda").manual_seed(c)
    x = torch.tensor(SIZES, device="cuda")[:, None].expand(len(SIZES), c).clone()
    x *= 1 - 2 * (torch.rand(x.shape, generator=g, device="cuda") < 0.5).float()
    assert torch.equal(x.to(dtype).float(), x)
    gain = torch.randint(-100, 100, (c,), generator=g, device="cuda").float() + 0.5
    gain[0] = top
    y = x.sign().double() * gain.double()
    want = torch.round(y).to(torch.int8)        # (half to even)
    more = torch.zeros_like(x).to(dtype)
    for residual in (None, more):
        got = L.norm_rows(x.to(dtype), gain, residual=residual, eps=0.0)
        assert torch.equal(got.rows.codes[:, :c], want)
        assert (got.rows.scale == 1).all()
        assert torch.equal(got.rstd, (1.0 / torch.tensor(SIZES, device="cuda").double()).float())


@pytest.mark.parametrize("c", LENGTHS)
def test_rows_on_a_scales_border(L, c):
    """Largest values of 127 * 2^e in 64 bits, and the floats beside it."""
    x = torch.tensor(SIZES, device="cuda")[:, None].expand(len(SIZES), c).clone()
    for e in (-20, 0, 3):
        for gain, scale in ((127.0, 1.0), (127.0 - 2.0 ** -17, 1.0), (127.0 * (1 + 2.0 ** -23), 2.0)):
            g = torch.full((c,), gain * 2.0 ** e, device="cuda")
            got = L.norm_rows(x, g, eps=0.0)
            assert (got.rows.scale == scale * 2.0 ** e).all(), (e, gain)
            assert (got.rows.codes[:, :c] == (127 if scale == 1 else 64)).all()

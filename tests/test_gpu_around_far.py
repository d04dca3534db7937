"""The operators around the linear layer where an operand passes 4 GiB, and where rows of
other experts, or of none, hold what is not finite.

Tolerances are those of the operators' own tests; codes, sums and rstd of the norm do
not depend on the rows beside a row, and are equal."""
import math

import pytest
import torch

from test_gpu_experts import DTYPES, HALF_ULP, L, _gen, _grad, _grad_near, _near, _product, _randn, _rows8, _weights

pytestmark = pytest.mark.gpu
TAIL = 70


@pytest.fixture(autouse=True)
def _memory():
    yield
    torch.cuda.empty_cache()


def _offsets(*at):
    return torch.tensor(at, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("bits,group", [(8, 0), (4, 0), (4, 64)])
def test_far_weights(L, bits, group):
    """Experts' weights of more than 4 GiB: the last expert's are found."""
    g = _gen(bits + group)
    experts, c = 9, 32768 if bits == 4 else 16384
    k = 32768
    w, q = _weights(L, g, k, c, bits, group, torch.float16)
    codes = torch.zeros((experts * k, w.codes.shape[1]), dtype=w.codes.dtype, device="cuda")
    assert codes.numel() * codes.element_size() > 1 << 32
    codes[(experts - 1) * k:] = w.codes
    scale = torch.full((experts * k, *w.scale.shape[1:]), 0.01, dtype=w.scale.dtype, device="cuda")
    scale[(experts - 1) * k:] = w.scale
    every = L.GroupRows(codes, scale, c, group) if group else L.Rows(codes, scale, c, bits)
    last = slice(k - TAIL, k)
    part = L.GroupRows(w.codes[last], w.scale[last], c, group) if group else L.Rows(w.codes[last], w.scale[last], c, bits)
    whole = q[last]
    for m in (3, 200):
        x = _rows8(L, g, m, c)
        y = L.linear_experts(x, every, _offsets(*[0] * experts, m))
        want, size = _product(x, part, whole)
        _near(y[:, last], want, size, c // 32 + 8, torch.bfloat16)
        dy = torch.zeros((m, k), dtype=torch.bfloat16, device="cuda")
        dy[:, last] = _randn(g, m, TAIL).bfloat16()
        dx = L.linear_experts_grad_input(dy, every, _offsets(*[0] * experts, m))
        want, size = _grad(dy[:, last], part, whole, c)
        _grad_near(dx, want, size, TAIL, torch.bfloat16)


def test_far_group_scales(L):
    """The same of one layer: 600,000 rows of 16384 channels in 4 bits."""
    g = _gen(5)
    c, k, group = 16384, 600000, 128
    w, q = _weights(L, g, TAIL, c, 4, group, torch.float16)
    codes = torch.zeros((k, w.codes.shape[1]), dtype=torch.int32, device="cuda")
    assert codes.numel() * 4 > 1 << 32
    codes[k - TAIL:] = w.codes
    scale = torch.full((k, c // group), 0.01, dtype=torch.float16, device="cuda")
    scale[k - TAIL:] = w.scale
    every = L.GroupRows(codes, scale, c, group)
    for m in (1, 40, 200):
        x = _rows8(L, g, m, c)
        want, size = _product(x, w, q)
        y = L.linear(x, every)
        _near(y[:, k - TAIL:], want, size, c // 32 + 8, torch.bfloat16)
        assert (y[:, :k - TAIL] == 0).all()
        dy = torch.zeros((m, k), dtype=torch.bfloat16, device="cuda")
        dy[:, k - TAIL:] = _randn(g, m, TAIL).bfloat16()
        want, size = _grad(dy[:, k - TAIL:], w, q, c)
        _grad_near(L.linear_grad_input(dy, every), want, size, TAIL, torch.bfloat16)


@pytest.mark.parametrize("bits,group", [(8, 0), (4, 32)])
def test_far_rows(L, bits, group):
    """Rows, results and their gradients of more than 4 GiB."""
    g = _gen(bits)
    m, c, k = 1050000, 4160, 2080
    codes = torch.zeros((m, c), dtype=torch.int8, device="cuda")
    codes[m - TAIL:] = _rows8(L, g, TAIL, c).codes
    x = L.Rows(codes, torch.rand(m, generator=g, device="cuda") * 0.02 + 0.001, c)
    tail = L.Rows(codes[m - TAIL:], x.scale[m - TAIL:], c)
    w, q = _weights(L, g, 2 * k, c, bits, group, torch.float16)
    mine = slice(k, 2 * k)
    part = L.GroupRows(w.codes[mine], w.scale[mine], c, group) if group else L.Rows(w.codes[mine], w.scale[mine], c, bits)
    offsets = _offsets(0, m // 2, m)
    y = L.linear_experts(x, w, offsets)
    assert codes.numel() > 1 << 32 and y.numel() * 2 > 1 << 32
    want, size = _product(tail, part, q[mine])
    _near(y[m - TAIL:], want, size, c // 32 + 8, torch.bfloat16)
    assert (y[:m - TAIL] == 0).all()
    if group:
        _near(L.linear(x, part)[m - TAIL:], want, size, c // 32 + 8, torch.bfloat16)
    dy = y.zero_()
    dy[m - TAIL:] = _randn(g, TAIL, k).bfloat16()
    dx = L.linear_experts_grad_input(dy, w, offsets)
    want, size = _grad(dy[m - TAIL:], part, q[mine], c)
    _grad_near(dx[m - TAIL:], want, size, k, torch.bfloat16)
    assert (dx[:m - TAIL] == 0).all()
    del dx
    dw = L.linear_experts_grad_weight(dy, x, offsets)
    d, v = dy[m - TAIL:].double(), tail.codes.double() * tail.scale.double()[:, None]
    want, size = d.t().contiguous() @ v, d.abs().t().contiguous() @ v.abs()
    assert bool(((dw[1].double() - want).abs() <= size * (HALF_ULP[torch.bfloat16] * 1.01 + (TAIL + 4) * 2.0 ** -24)).all())
    assert (dw[0] == 0).all()


def test_far_weight_gradient(L):
    g = _gen(9)
    experts, k, c = 6, 12000, 16000
    dy, x = _randn(g, TAIL, k).bfloat16(), _rows8(L, g, TAIL, c)
    dw = L.linear_experts_grad_weight(dy, x, _offsets(*[0] * experts, TAIL))
    assert dw.numel() * 4 > 1 << 32 and (dw[:experts - 1] == 0).all()
    d, v = dy.double(), x.codes[:, :c].double() * x.scale.double()[:, None]
    want, size = d.t().contiguous() @ v, d.abs().t().contiguous() @ v.abs()
    assert bool(((dw[experts - 1].double() - want).abs() <= size * (HALF_ULP[torch.bfloat16] * 1.01 + (TAIL + 4) * 2.0 ** -24)).all())


def test_far_norm(L):
    g = _gen(11)
    m, c = 1050000, 4100
    x, r = torch.zeros((m, c), dtype=torch.bfloat16, device="cuda"), torch.zeros((m, c), dtype=torch.bfloat16, device="cuda")
    x[m - TAIL:], r[m - TAIL:] = _randn(g, TAIL, c).bfloat16(), _randn(g, TAIL, c).bfloat16()
    gain = _randn(g, c)
    far = L.norm_rows(x, gain, residual=r)
    near = L.norm_rows(x[m - TAIL:], gain, residual=r[m - TAIL:])
    assert far.rows.codes.numel() > 1 << 32
    assert torch.equal(far.rows.codes[m - TAIL:], near.rows.codes) and torch.equal(far.rows.scale[m - TAIL:], near.rows.scale)
    assert torch.equal(far.sum[m - TAIL:], near.sum) and torch.equal(far.rstd[m - TAIL:], near.rstd)
    assert not far.rows.codes[:m - TAIL].any() and not far.rows.scale[:m - TAIL].any()
    del x, r
    dy = torch.zeros((m, c), dtype=torch.bfloat16, device="cuda")
    dy[m - TAIL:] = _randn(g, TAIL, c).bfloat16()
    dx, dgain = L.norm_rows_grad(dy, far.sum, gain, far.rstd)
    part, _ = L.norm_rows_grad(dy[m - TAIL:], near.sum, gain, near.rstd)
    assert torch.equal(dx[m - TAIL:], part) and not dx[:m - TAIL].any()
    n = dy[m - TAIL:].double() * near.sum.double() * near.rstd.double()[:, None]
    assert bool(((dgain.double() - n.sum(0)).abs() <= n.abs().sum(0) * (TAIL + 4) * 2.0 ** -24).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("counts,c,k", [((1, 3, 2), 64, 48), ((20, 33, 65), 328, 130), ((300, 70, 513), 520, 264)])
@pytest.mark.parametrize("bits,group", [(8, 0), (4, 0), (4, 32), (4, 128)])
def test_faults_stay_with_their_expert(L, bits, group, counts, c, k, dtype):
    """Rows of the second expert and of none that are not finite reach no other's results."""
    g = _gen(sum(counts) + bits + group)
    first, more = 2, 5
    m = first + sum(counts) + more
    at = [first + sum(counts[:e]) for e in range(4)]
    offsets = _offsets(*at)
    x, dy = _rows8(L, g, m, c), _randn(g, m, k).to(dtype)
    w, q = _weights(L, g, 3 * k, c, bits, group, torch.float32)
    others = [slice(at[0], at[1]), slice(at[2], at[3])]

    def run():
        return (L.linear_experts(x, w, offsets, dtype=dtype), L.linear_experts_grad_input(dy, w, offsets),
                L.linear_experts_grad_weight(dy, x, offsets))
    y, dx, dw = run()
    for rows, fault in ((slice(0, first), math.nan), (slice(at[1], at[2]), math.inf), (slice(at[3], m), -math.inf)):
        dy[rows] = fault
        x.scale[rows] = fault
    w.scale[k:2 * k] = math.nan
    y2, dx2, dw2 = run()
    for rows in others:
        assert torch.equal(y[rows], y2[rows]) and torch.equal(dx[rows], dx2[rows])
    assert torch.equal(dw[0], dw2[0]) and torch.equal(dw[2], dw2[2]) and not torch.isfinite(dw2[1]).any()
    assert not torch.isfinite(y2[at[1]:at[2]]).any() and not torch.isfinite(dx2[at[1]:at[2]]).any()

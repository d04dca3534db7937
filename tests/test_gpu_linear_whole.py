"""Every kernel of the linear layer and around it writes all of its result, whatever its
memory held: into results that hold NaN, after a call of the same sizes on operands full of
NaN (which leaves its traces in the kernels' shared memory), and with comparisons that a
NaN does not pass.  Sizes, inputs and tolerances are those of the other tests of these
kernels."""
import math

import pytest
import torch

import around_sizes
import linear_sizes
import test_gpu_experts as E
import test_gpu_frozen_grads as F
import test_gpu_linear as D

pytestmark = pytest.mark.gpu

DTYPES = (torch.bfloat16, torch.float16)
HALF_ULP = E.HALF_ULP


@pytest.fixture(scope="module")
def L():
    from paper_2202_06819_amd import build, linear
    build.ensure_built()
    return linear


def _nan(shape, dtype):
    return torch.full(shape, math.nan, dtype=dtype, device="cuda")


def _rounded(want, tol, dtype):
    """The tolerance of a result rounded to a 16-bit type from one within `tol`."""
    return tol * (1 + HALF_ULP[dtype]) + want.abs() * HALF_ULP[dtype] + (2.0 ** -25 if dtype == torch.float16 else 1e-300)


def _within(got, want, tol):
    ok = (got.double() - want).abs() <= tol   # (false for a NaN)
    assert bool(ok.all()), f"{int((~ok).sum())} of {ok.numel()} off, {int(got.isnan().sum())} NaN"


def _of_nan(rows):
    return rows._replace(scale=torch.full_like(rows.scale, math.nan))


@pytest.mark.parametrize("op,m,c,k,bits,group,scales,experts,dtype", around_sizes.PRODUCTS)
def test_around(L, op, m, c, k, bits, group, scales, experts, dtype):
    g = E._gen(m + c + k + experts + 1)
    dtype = DTYPES[dtype]
    counts = E._dealt(m, experts) if experts else [m]
    offsets = E._offsets(counts)
    n = max(experts, 1)
    w, q = E._weights(L, g, n * k, c, bits, group, (torch.bfloat16, torch.float16, torch.float32)[scales])
    x, dy = E._rows8(L, g, m, c), E._dy(g, m, k, dtype)

    def run(x, w, dy):
        if op == "forward":
            out = _nan((m, k), dtype)
            return L.linear_experts(x, w, offsets, dtype=dtype, out=out) if experts else L.linear(x, w, dtype=dtype, out=out)
        if op == "grad_input":
            out = _nan((m, c), dtype)
            return L.linear_experts_grad_input(dy, w, offsets, out=out) if experts else L.linear_grad_input(dy, w, out=out)
        return L.linear_experts_grad_weight(dy, x, offsets, out=_nan((experts, k, c), torch.float32))
    run(_of_nan(x), _of_nan(w), torch.full_like(dy, math.nan))
    got = run(x, w, dy)
    ends = [0]
    for count in counts:
        ends.append(ends[-1] + count)
    for e in range(len(counts)):
        rows, mine = slice(ends[e], ends[e + 1]), slice(e * k, e * k + k)
        if op == "grad_weight":
            d, v = dy[rows].double(), x.codes[rows, :c].double() * x.scale.double()[rows, None]
            want, size = d.t().contiguous() @ v, d.abs().t().contiguous() @ v.abs()
            _within(got[e], want, size * (HALF_ULP[dtype] * 1.01 + (counts[e] + 4) * 2.0 ** -24))
        elif counts[e]:
            part = L.GroupRows(w.codes[mine], w.scale[mine], c, group) if group else L.Rows(w.codes[mine], w.scale[mine], c, bits)
            if op == "forward":
                want, size = E._product(L.Rows(x.codes[rows], x.scale[rows], c), part, q[mine])
                _within(got[rows], want, _rounded(want, size * (c // 32 + 12) * 2.0 ** -24, dtype))
            else:
                want, size = E._grad(dy[rows], part, q[mine], c)
                products = F.PARTS[dtype] if bits == 4 else HALF_ULP[dtype] * 1.01
                _within(got[rows], want, _rounded(want, size * (products + (2 * k + 4) * 2.0 ** -24), dtype))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,c,k,bits,n,rank", linear_sizes.LINEAR)
def test_projection(L, m, c, k, bits, n, rank, dtype):
    g = D._gen(m + c + k + rank + 1)
    x = D._rows8(L, g, m, c)
    w, q = D._rows4(L, g, k, c) if bits == 4 else (D._rows8(L, g, k, c), None)
    base = D._product(x, w, q)
    tol = base.abs() * 4 * 2.0 ** -24
    more = {}
    if n:
        ad = D._adapters(L, g, n, rank, c, k, dtype)
        ids = torch.randint(-1, n, (m,), generator=g, device="cuda", dtype=torch.int32)
        more = {"adapters": ad, "row_adapter": ids}
        part, size, coarse = D._adapter_part(x, ad, ids)
        base, tol = base + part, (coarse * (HALF_ULP[dtype] ** 2 + 2.0 ** -24) + size * (c + 2 * rank + 8) * 2.0 ** -24
                                  + base.abs() * 2.0 ** -22)
    L.linear(_of_nan(x), _of_nan(w), dtype=dtype, **more)
    got = L.linear(x, w, dtype=dtype, out=_nan((m, k), dtype), **more)
    _within(got, base, _rounded(base, tol * 1.01, dtype))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,c,k,bits", linear_sizes.GRAD_INPUT)
def test_input_gradient(L, m, c, k, bits, dtype):
    g = D._gen(m + c + k + bits + 1)
    dy = D._dy(g, m, k, dtype, k + 8)
    w, q = D._rows4(L, g, k, c) if bits == 4 else (D._rows8(L, g, k, c), None)
    values, d = D._values(w, q), dy.double().contiguous()
    want, size = d @ values, d.abs() @ values.abs()
    L.linear_grad_input(torch.full_like(dy, math.nan), _of_nan(w))
    got = L.linear_grad_input(dy, w, out=_nan((m, c), dtype))
    _within(got, want, _rounded(want, size * (k * 2.0 ** -24 + (HALF_ULP[dtype] * 1.01 if bits == 4 else 0.0)), dtype))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,c,k", linear_sizes.GRAD_WEIGHT)
def test_weight_gradient(L, m, c, k, dtype):
    g = D._gen(m + c + k + 1)
    dy, x = D._dy(g, m, k, dtype, k + 8), D._rows8(L, g, m, c)
    v, d = D._values(x), dy.double().t().contiguous()
    want, size = d @ v, d.abs() @ v.abs()
    L.linear_grad_weight(torch.full_like(dy, math.nan), _of_nan(x))
    got = L.linear_grad_weight(dy, x, out=_nan((k, c), torch.float32))
    _within(got, want, size * m * 2.0 ** -24 + want.abs() * 2.0 ** -24 + 1e-300)

"""Host-side checks of the norm's entry points: every refusal comes before anything is
launched.  Pointers are plain integers that are never dereferenced."""
import ctypes

import pytest

A, B, C, D, E, F, G, H = (i << 36 for i in range(1, 9))   # far apart, 16-byte aligned
EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -3


@pytest.fixture(scope="module")
def L():
    from paper_2202_06819_amd import build, linear
    build.ensure_built()
    linear._lib()
    return linear


def _status(L, name, *args):
    rc = getattr(L._lib(), name)(*args)
    assert rc == 0 or L.qconv.lib().qconv_last_error()
    return rc


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), EINVAL), (dict(gain_dtype=-1), EINVAL), (dict(m=-1), EINVAL), (dict(c=0), EINVAL),
    (dict(m=(1 << 22) + 1), EUNSUPPORTED), (dict(c=131072, ldx=131072, ldr=131072, lds=131072, pitch=131072), EUNSUPPORTED),
    (dict(eps=-1e-9), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(eps=float("inf")), EINVAL),
    (dict(ldx=99), EINVAL), (dict(ldr=99), EINVAL), (dict(lds=99), EINVAL), (dict(ldx=(1 << 21) + 1), EUNSUPPORTED),
    (dict(pitch=96), EINVAL), (dict(pitch=120), EINVAL), (dict(pitch=(1 << 22) + 16), EUNSUPPORTED),
    (dict(x=None), EINVAL), (dict(gain=None), EINVAL), (dict(codes=None), EINVAL), (dict(scale=None), EINVAL),
    (dict(residual=None), EINVAL), (dict(sum=None), EINVAL),
    (dict(x=A + 1), EINVAL), (dict(residual=B + 1), EINVAL), (dict(sum=C + 1), EINVAL), (dict(gain=D + 2), EINVAL),
    (dict(codes=E + 8), EINVAL), (dict(scale=F + 2), EINVAL), (dict(rstd=G + 1), EINVAL),
    (dict(codes=A + 16), EINVAL), (dict(codes=B + 16), EINVAL), (dict(codes=C + 16), EINVAL), (dict(codes=D + 16), EINVAL),
    (dict(scale=E + 16), EINVAL), (dict(rstd=E + 16), EINVAL), (dict(rstd=F + 24), EINVAL), (dict(scale=D), EINVAL),
    (dict(sum=A + 2), EINVAL), (dict(sum=B + 200), EINVAL), (dict(sum=D), EINVAL), (dict(sum=A, lds=104), EINVAL),
])
def test_norm_refusals(L, kw, status):
    a = dict(x=A, ldx=100, residual=B, ldr=100, sum=C, lds=100, dtype=0, gain=D, gain_dtype=2, eps=1e-6, m=7, c=100, codes=E,
             pitch=112, scale=F, rstd=G)
    a.update(kw)
    assert _status(L, "qconv_norm_rows", *a.values(), None) == status


def test_nothing_to_do(L):
    assert _status(L, "qconv_norm_rows", None, 100, None, 0, None, 0, 2, D, 2, 1e-6, 0, 100, None, 112, None, None, None) == 0
    assert _status(L, "qconv_norm_rows", None, 100, None, 100, None, 100, 2, D, 2, 1e-6, 0, 100, None, 112, None, None, None) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), EINVAL), (dict(gain_dtype=9), EINVAL), (dict(m=-1), EINVAL), (dict(c=0), EINVAL),
    (dict(m=(1 << 22) + 1), EUNSUPPORTED), (dict(lddy=99), EINVAL), (dict(ldh=99), EINVAL), (dict(ldds=99), EINVAL),
    (dict(lddx=99), EINVAL), (dict(lddx=(1 << 21) + 1), EUNSUPPORTED),
    (dict(dy=None), EINVAL), (dict(h=None), EINVAL), (dict(gain=None), EINVAL), (dict(rstd=None), EINVAL),
    (dict(dx=None), EINVAL), (dict(dgain=None), EINVAL), (dict(dy=A + 1), EINVAL), (dict(rstd=E + 2), EINVAL),
    (dict(dgain=G + 2), EINVAL), (dict(ws=None), EWORKSPACE), (dict(less=1), EWORKSPACE), (dict(ws=H + 4), EINVAL),
    (dict(dx=A), EINVAL), (dict(dx=B), EINVAL), (dict(dx=C + 2), EINVAL), (dict(dx=C, lddx=104), EINVAL), (dict(dx=D), EINVAL),
    (dict(dx=E), EINVAL), (dict(dgain=A), EINVAL), (dict(dgain=F), EINVAL), (dict(ws=A), EINVAL), (dict(ws=F), EINVAL),
    (dict(ws=G), EINVAL), (dict(ws=C), EINVAL),
])
def test_norm_gradient_refusals(L, kw, status):
    a = dict(dy=A, lddy=100, h=B, ldh=100, dsum=C, ldds=100, dtype=0, gain=D, gain_dtype=2, rstd=E, m=7, c=100, dx=F, lddx=100,
             dgain=G, ws=H)
    need = L.norm_grad_workspace_bytes(7, 100)
    assert need > 0
    a.update({name: value for name, value in kw.items() if name != "less"})
    assert _status(L, "qconv_norm_rows_grad", *a.values(), need - kw.get("less", 0), None) == status


def test_workspace_query_refuses(L):
    n = ctypes.c_size_t(0)
    name = "qconv_norm_rows_grad_workspace_bytes"
    for m, c, to, status in ((4, 64, None, EINVAL), (-1, 64, ctypes.byref(n), EINVAL), (4, 0, ctypes.byref(n), EINVAL),
                             (4, 131072, ctypes.byref(n), EUNSUPPORTED)):
        assert _status(L, name, m, c, to) == status
    assert L.norm_grad_workspace_bytes(0, 64) == 0


def test_python_refuses(L):
    import torch
    x, gain = torch.zeros(4, 32), torch.ones(32)
    with pytest.raises(L.QConvError):
        L.norm_rows(x, gain)
    with pytest.raises(L.QConvError):
        L.norm_rows_grad(x, x, gain, torch.zeros(4))

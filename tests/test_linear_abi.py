"""Host-side checks of the linear layer's entry points: every refusal comes
before anything is launched, so no GPU is needed.  Pointers here are plain
integers that are never dereferenced."""
import ctypes

import pytest

A, B, C, D, E, F, G, H = (i << 36 for i in range(1, 9))   # far apart, 16-byte aligned


@pytest.fixture(scope="module")
def L():
    from paper_2202_06819_amd import build, linear
    build.ensure_built()
    linear._lib()
    return linear


def _rows(L, codes=A, scale=B, pitch=256, rows=32, channels=256, bits=8):
    return L.QConvRows(codes, scale, pitch, rows, channels, bits)


def _status(L, name, *args):
    args = [ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in args]
    rc = getattr(L._lib(), name)(*args)
    assert rc == 0 or L.qconv.lib().qconv_last_error()
    return rc


EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -3


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), EINVAL), (dict(dtype=-1), EINVAL), (dict(m=-1), EINVAL), (dict(c=0), EINVAL),
    (dict(c=131072, ldx=131072, pitch=131072), EUNSUPPORTED), (dict(ldx=99), EINVAL), (dict(ldx=(1 << 21) + 1), EUNSUPPORTED),
    (dict(pitch=96), EINVAL), (dict(pitch=120), EINVAL), (dict(pitch=(1 << 22) + 16), EUNSUPPORTED),
    (dict(x=None), EINVAL), (dict(codes=None), EINVAL), (dict(scale=None), EINVAL), (dict(x=A + 1), EINVAL),
    (dict(codes=B + 8), EINVAL), (dict(scale=C + 2), EINVAL), (dict(codes=A + 16), EINVAL), (dict(scale=B + 112), EINVAL),
])
def test_quantize_rows_refusals(L, kw, status):
    a = dict(x=A, dtype=0, ldx=100, m=7, c=100, codes=B, pitch=112, scale=C)
    a.update(kw)
    assert _status(L, "qconv_quantize_rows", a["x"], a["dtype"], a["ldx"], a["m"], a["c"], a["codes"], a["pitch"],
                   a["scale"], None) == status


def test_nothing_to_do(L):
    assert _status(L, "qconv_quantize_rows", None, 2, 100, 0, 100, None, 112, None, None) == 0
    none = _rows(L, None, None, rows=0)
    assert _status(L, "qconv_linear", none, _rows(L, C, D), None, None, 0, 32, None, 0, None) == 0
    assert _status(L, "qconv_linear_grad_input", None, 0, 32, 0, _rows(L), None, 256, None, 0, None) == 0


def test_nothing_to_do_with_adapters(L):
    """An empty tensor's pointer is NULL: of no rows none is asked for.  What is wrong
    with the adapters themselves is refused all the same."""
    none, w = _rows(L, None, None, rows=0), _rows(L, C, D)
    assert _status(L, "qconv_linear", none, w, _adapters(L, row=None), None, 0, 32, None, 0, None) == 0
    assert _status(L, "qconv_linear", none, w, _adapters(L, a=None), None, 0, 32, None, 0, None) == EINVAL
    assert _status(L, "qconv_linear", none, w, _adapters(L, rank=12), None, 0, 32, None, 0, None) == EUNSUPPORTED


BAD_ROWS = [
    (dict(rows=-1), EINVAL), (dict(channels=0), EINVAL), (dict(bits=16), EUNSUPPORTED), (dict(bits=0), EUNSUPPORTED),
    (dict(channels=131072, pitch=131072), EUNSUPPORTED), (dict(pitch=240), EINVAL), (dict(pitch=264), EINVAL),
    (dict(pitch=(1 << 22) + 16), EUNSUPPORTED), (dict(rows=(1 << 22) + 1), EUNSUPPORTED), (dict(codes=None), EINVAL),
    (dict(scale=None), EINVAL), (dict(codes=A + 8), EINVAL), (dict(scale=B + 1), EINVAL),
]


@pytest.mark.parametrize("kw,status", BAD_ROWS)
def test_rows_refusals(L, kw, status):
    bad, good = _rows(L, **kw), _rows(L, C, D)
    wide = max(kw.get("channels", 256), 256)
    good.channels = bad.channels if bad.channels > 0 else 256
    assert _status(L, "qconv_linear", bad, good, None, E, 0, 32, None, 0, None) == status
    assert _status(L, "qconv_linear_grad_input", C, 0, 1 << 21, 4, bad, E, wide, None, 0, None) == status
    assert _status(L, "qconv_linear_grad_weight", C, 0, 64, 64, bad, E, wide, None, 0, None) == status


def test_four_bits_are_for_weights(L):
    four = _rows(L, C, D, pitch=128, bits=4)
    assert _status(L, "qconv_linear", _rows(L, C, D, pitch=128, bits=4), four, None, E, 0, 32, None, 0, None) == EUNSUPPORTED
    assert _status(L, "qconv_linear_grad_weight", A, 0, 64, 64, four, E, 256, None, 0, None) == EUNSUPPORTED
    odd = _rows(L, C, D, pitch=128, channels=252, bits=4)
    assert _status(L, "qconv_linear", _rows(L, channels=252), odd, None, E, 0, 32, None, 0, None) == EUNSUPPORTED


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), EUNSUPPORTED), (dict(dtype=7), EINVAL), (dict(channels=240), EINVAL), (dict(k=0), EINVAL),
    (dict(y=None), EINVAL), (dict(y=E + 1), EINVAL), (dict(ldy=31), EINVAL), (dict(ldy=(1 << 21) + 1), EUNSUPPORTED),
    (dict(y=A + 64), EINVAL), (dict(y=B), EINVAL), (dict(y=C + 4096), EINVAL), (dict(y=D), EINVAL),
    (dict(rows=1 << 22, k=1 << 21, ldy=1 << 21), EUNSUPPORTED),
])
def test_linear_refusals(L, kw, status):
    a = dict(dtype=0, channels=256, k=32, y=E, ldy=32, rows=32)
    a.update(kw)
    x, w = _rows(L, rows=a["rows"]), _rows(L, C, D, channels=a["channels"], rows=a["k"])
    assert _status(L, "qconv_linear", x, w, None, a["y"], a["dtype"], a["ldy"], None, 0, None) == status


def _adapters(L, a=F, b=G, alpha=G + (1 << 30), row=G + (1 << 31), count=4, rank=16):
    return L.QConvAdapters(a, b, alpha, row, count, rank)


@pytest.mark.parametrize("kw,status", [
    (dict(count=-1), EINVAL), (dict(rank=0), EUNSUPPORTED), (dict(rank=12), EUNSUPPORTED), (dict(rank=136), EUNSUPPORTED),
    (dict(a=None), EINVAL), (dict(b=None), EINVAL), (dict(alpha=None), EINVAL), (dict(row=None), EINVAL),
    (dict(a=F + 8), EINVAL), (dict(b=G + 2), EINVAL), (dict(alpha=G + 2), EINVAL), (dict(row=G + 1), EINVAL),
    (dict(a=E), EINVAL), (dict(b=E + 16), EINVAL), (dict(alpha=E + 64), EINVAL), (dict(row=H + 64), EINVAL),
])
def test_adapter_refusals(L, kw, status):
    need = L.linear_workspace_bytes(32, 256, 16)
    assert need > 0 and L.linear_workspace_bytes(32, 256) == 0 and L.linear_workspace_bytes(0, 256, 16) == 0
    args = (E, 0, 32, H, need, None)
    assert _status(L, "qconv_linear", _rows(L), _rows(L, C, D), _adapters(L, **kw), *args) == status


def test_adapter_workspace_and_channels(L):
    need = L.linear_workspace_bytes(32, 256, 16)
    x, w, ad = _rows(L), _rows(L, C, D), _adapters(L)
    for ws, n, status in ((None, need, EWORKSPACE), (H, need - 1, EWORKSPACE), (H + 8, need, EINVAL), (A, need, EINVAL),
                          (E, need, EINVAL), (F, need, EINVAL)):
        assert _status(L, "qconv_linear", x, w, ad, E, 0, 32, ws, n, None) == status
    x9, w9 = _rows(L, channels=250), _rows(L, C, D, channels=250)
    assert _status(L, "qconv_linear", x9, w9, ad, E, 0, 32, H, need, None) == EUNSUPPORTED


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), EUNSUPPORTED), (dict(dtype=-2), EINVAL), (dict(n=-1), EINVAL), (dict(n=(1 << 22) + 1), EUNSUPPORTED),
    (dict(dy=None), EINVAL), (dict(dy=E + 1), EINVAL), (dict(out=None), EINVAL), (dict(out=F + 1), EINVAL),
    (dict(lddy=31), EINVAL), (dict(lddy=(1 << 21) + 1), EUNSUPPORTED), (dict(ldo=255), EINVAL),
    (dict(out=E), EINVAL), (dict(out=A), EINVAL), (dict(out=B), EINVAL),
])
def test_gradient_refusals(L, kw, status):
    a = dict(dy=E, dtype=0, lddy=64, n=32, out=F, ldo=256)
    a.update(kw)
    need = max(L.grad_workspace_bytes(32, 256, 32), 16)
    for name in ("qconv_linear_grad_input", "qconv_linear_grad_weight"):
        assert _status(L, name, a["dy"], a["dtype"], a["lddy"], a["n"], _rows(L), a["out"], a["ldo"], H, need, None) == status


def test_gradient_workspace(L):
    x = _rows(L, rows=100000)
    need = L.grad_workspace_bytes(32, 256, 100000)
    assert need > 0
    for ws, n, status in ((None, need, EWORKSPACE), (H, need - 1, EWORKSPACE), (H + 4, need, EINVAL), (A, need, EINVAL),
                          (E, need, EINVAL), (F, need, EINVAL)):
        assert _status(L, "qconv_linear_grad_weight", E, 0, 32, 32, x, F, 256, ws, n, None) == status
    assert _status(L, "qconv_linear_grad_weight", E, 0, 32, 0, x, F, 256, H, need, None) == EINVAL
    assert L.grad_workspace_bytes(0, 8, 100) == 0


def test_workspace_queries_refuse(L):
    n = ctypes.c_size_t(0)
    assert _status(L, "qconv_linear_workspace_bytes", 4, 64, None, None) == EINVAL
    assert _status(L, "qconv_linear_workspace_bytes", -1, 64, None, n) == EINVAL
    assert _status(L, "qconv_linear_workspace_bytes", 4, 64, _adapters(L, count=-1), n) == EINVAL
    assert _status(L, "qconv_linear_grad_workspace_bytes", 4, 0, 64, n) == EINVAL
    assert _status(L, "qconv_linear_grad_workspace_bytes", 4, 64, -1, n) == EINVAL
    assert _status(L, "qconv_linear_grad_workspace_bytes", 4, 64, 64, None) == EINVAL


def test_python_refuses_host_tensors(L):
    import torch
    x = torch.zeros(4, 32)
    with pytest.raises(L.QConvError):
        L.quantize_rows(x)
    with pytest.raises(L.QConvError):
        L.linear(L.Rows(x.to(torch.int8), x[:, 0].contiguous(), 32), L.Rows(x.to(torch.int8), x[:, 0].contiguous(), 32))
    with pytest.raises(L.QConvError):
        L.linear_grad_weight(x.bfloat16(), L.Rows(x.to(torch.int8), x[:, 0].contiguous(), 32))

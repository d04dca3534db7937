"""Host-side checks of the products with group scales and of experts: every refusal
comes before anything is launched.  Pointers are plain integers that are never
dereferenced."""
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


def _rows(L, codes=A, scale=B, pitch=256, rows=32, channels=256, bits=8):
    return L.QConvRows(codes, scale, pitch, rows, channels, bits)


def _groups(L, codes=C, scale=D, pitch=128, scale_pitch=8, rows=64, channels=256, group=32, scale_dtype=1):
    return L.QConvGroupRows(codes, scale, pitch, scale_pitch, rows, channels, group, scale_dtype)


def _status(L, name, *args):
    args = [ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in args]
    rc = getattr(L._lib(), name)(*args)
    assert rc == 0 or L.qconv.lib().qconv_last_error()
    return rc


BAD_WEIGHTS = [
    (dict(scale_dtype=3), EINVAL), (dict(scale_dtype=-1), EINVAL), (dict(group=16), EUNSUPPORTED), (dict(group=0), EUNSUPPORTED),
    (dict(group=48), EUNSUPPORTED), (dict(group=4128), EUNSUPPORTED), (dict(scale_pitch=7), EINVAL),
    (dict(scale_pitch=(1 << 17) + 1), EUNSUPPORTED), (dict(scale=None), EINVAL), (dict(scale=D + 1), EINVAL),
    (dict(scale_dtype=2, scale=D + 2), EINVAL), (dict(codes=None), EINVAL), (dict(codes=C + 8), EINVAL), (dict(pitch=112), EINVAL),
    (dict(pitch=136), EINVAL), (dict(channels=252), EUNSUPPORTED), (dict(rows=-1), EINVAL), (dict(rows=0), EINVAL),
    (dict(rows=(1 << 22) + 64), EUNSUPPORTED),
]


@pytest.mark.parametrize("kw,status", BAD_WEIGHTS)
def test_group_rows_refusals(L, kw, status):
    w = _groups(L, **kw)
    c = w.channels
    x = _rows(L, channels=c)
    assert _status(L, "qconv_linear_groups", x, w, E, 0, 1 << 21, None) == status
    assert _status(L, "qconv_linear_groups_grad_input", A, 0, 1 << 21, 4, w, E, 256, H, 1 << 30, None) == status
    assert _status(L, "qconv_linear_experts_groups", x, w, F, 2, E, 0, 1 << 21, None) == status
    assert _status(L, "qconv_linear_experts_groups_grad_input", A, 0, 1 << 21, 4, w, F, 2, E, 256, None) == status


def test_null_structures(L):
    x, w = _rows(L), _groups(L)
    assert _status(L, "qconv_linear_groups", None, w, E, 0, 64, None) == EINVAL
    assert _status(L, "qconv_linear_groups", x, None, E, 0, 64, None) == EINVAL
    assert _status(L, "qconv_linear_experts", x, None, F, 2, E, 0, 64, None) == EINVAL
    assert _status(L, "qconv_linear_experts_grad_weight", C, 0, 64, 64, None, F, 2, E, 256, None) == EINVAL


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), EUNSUPPORTED), (dict(dtype=7), EINVAL), (dict(channels=240), EINVAL), (dict(y=None), EINVAL),
    (dict(y=E + 1), EINVAL), (dict(ldy=31), EINVAL), (dict(ldy=(1 << 21) + 1), EUNSUPPORTED), (dict(y=A + 64), EINVAL),
    (dict(y=B), EINVAL), (dict(y=C + 4096), EINVAL), (dict(y=D), EINVAL), (dict(bits=4), EUNSUPPORTED),
])
def test_forward_refusals(L, kw, status):
    a = dict(dtype=0, channels=256, y=E, ldy=64, bits=8)
    a.update(kw)
    x = _rows(L, channels=a["channels"], bits=a["bits"])
    assert _status(L, "qconv_linear_groups", x, _groups(L), a["y"], a["dtype"], a["ldy"], None) == status
    assert _status(L, "qconv_linear_experts_groups", x, _groups(L), F, 2, a["y"], a["dtype"], a["ldy"], None) == status
    w = _rows(L, C, D, rows=64)
    assert _status(L, "qconv_linear_experts", x, w, F, 2, a["y"], a["dtype"], a["ldy"], None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(experts=0), EINVAL), (dict(experts=-1), EINVAL), (dict(experts=4097), EUNSUPPORTED), (dict(experts=3), EINVAL),
    (dict(offsets=None), EINVAL), (dict(offsets=F + 2), EINVAL), (dict(offsets=E + 64), EINVAL),
])
def test_expert_refusals(L, kw, status):
    a = dict(offsets=F, experts=2)
    a.update(kw)
    x, w, w4 = _rows(L), _rows(L, C, D, rows=64), _groups(L)
    dealt = (a["offsets"], a["experts"])
    assert _status(L, "qconv_linear_experts", x, w, *dealt, E, 0, 64, None) == status
    assert _status(L, "qconv_linear_experts_groups", x, w4, *dealt, E, 0, 64, None) == status
    assert _status(L, "qconv_linear_experts_grad_input", A, 0, 64, 32, w, *dealt, E, 256, None) == status
    assert _status(L, "qconv_linear_experts_groups_grad_input", A, 0, 64, 32, w4, *dealt, E, 256, None) == status
    if kw != dict(experts=3):   # (k is a number of its own there)
        assert _status(L, "qconv_linear_experts_grad_weight", C, 0, 64, 32, x, *dealt, E, 256, None) == status


def test_too_large_results(L):
    """One tile more is counted for each expert."""
    w = _rows(L, C, D, rows=1 << 16)
    x = _rows(L, rows=1 << 22)
    assert _status(L, "qconv_linear_experts", x, w, F, 1, E, 0, 1 << 16, None) == EUNSUPPORTED
    assert _status(L, "qconv_linear_experts_grad_weight", C, 0, 1 << 21, 1 << 21, _rows(L, channels=256), F, 4, E, 256, None) == EUNSUPPORTED
    assert _status(L, "qconv_linear_experts_grad_weight", C, 0, 64, 0, _rows(L), F, 4, E, 256, None) == EINVAL


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), EUNSUPPORTED), (dict(m=-1), EINVAL), (dict(m=(1 << 22) + 1), EUNSUPPORTED), (dict(dy=None), EINVAL),
    (dict(dy=A + 1), EINVAL), (dict(out=None), EINVAL), (dict(out=E + 1), EINVAL), (dict(lddy=31), EINVAL), (dict(ldo=255), EINVAL),
    (dict(out=A), EINVAL), (dict(out=C), EINVAL), (dict(out=D), EINVAL),
])
def test_grad_input_refusals(L, kw, status):
    a = dict(dy=A, dtype=0, lddy=64, m=32, out=E, ldo=256)
    a.update(kw)
    head, tail = (a["dy"], a["dtype"], a["lddy"], a["m"]), (a["out"], a["ldo"])
    assert _status(L, "qconv_linear_groups_grad_input", *head, _groups(L), *tail, H, 1 << 30, None) == status
    assert _status(L, "qconv_linear_experts_grad_input", *head, _rows(L, C, D, rows=64), F, 2, *tail, None) == status
    assert _status(L, "qconv_linear_experts_groups_grad_input", *head, _groups(L), F, 2, *tail, None) == status


def test_grad_input_workspace(L):
    w = _groups(L, rows=50000)
    need = L.grad_workspace_bytes(32, 256, 50000)
    assert need > 0
    for ws, n, status in ((None, need, EWORKSPACE), (H, need - 1, EWORKSPACE), (H + 4, need, EINVAL), (A, need, EINVAL),
                          (C, need, EINVAL), (D, need, EINVAL), (E, need, EINVAL)):
        assert _status(L, "qconv_linear_groups_grad_input", A, 0, 50000, 32, w, E, 256, ws, n, None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), EUNSUPPORTED), (dict(dy=None), EINVAL), (dict(dy=C + 1), EINVAL), (dict(out=None), EINVAL),
    (dict(out=E + 2), EINVAL), (dict(lddy=31), EINVAL), (dict(ldo=255), EINVAL), (dict(out=A), EINVAL), (dict(out=B), EINVAL),
    (dict(out=C), EINVAL), (dict(out=F), EINVAL),
])
def test_grad_weight_refusals(L, kw, status):
    a = dict(dy=C, dtype=0, lddy=64, out=E, ldo=256)
    a.update(kw)
    assert _status(L, "qconv_linear_experts_grad_weight", a["dy"], a["dtype"], a["lddy"], 32, _rows(L), F, 2, a["out"], a["ldo"],
                   None) == status


def test_nothing_to_do(L):
    none = _rows(L, None, None, rows=0)
    assert _status(L, "qconv_linear_groups", none, _groups(L), None, 0, 64, None) == 0
    assert _status(L, "qconv_linear_groups_grad_input", None, 0, 64, 0, _groups(L), None, 256, None, 0, None) == 0
    assert _status(L, "qconv_linear_experts", none, _rows(L, C, D, rows=64), F, 2, None, 0, 64, None) == 0
    assert _status(L, "qconv_linear_experts_grad_input", None, 0, 64, 0, _rows(L, C, D, rows=64), F, 2, None, 256, None) == 0


def test_python_refuses_host_tensors(L):
    import torch
    x = torch.zeros(4, 32)
    rows = L.Rows(x.to(torch.int8), x[:, 0].contiguous(), 32)
    four = L.GroupRows(torch.zeros(4, 4, dtype=torch.int32), torch.zeros(4, 1), 32, 32)
    offsets = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: L.linear(rows, four), lambda: L.linear_experts(rows, rows, offsets),
                 lambda: L.linear_grad_input(x.bfloat16(), four), lambda: L.linear_experts_grad_input(x.bfloat16(), rows, offsets),
                 lambda: L.linear_experts_grad_weight(x.bfloat16(), rows, offsets), lambda: L.experts_layer(x, x, offsets)):
        with pytest.raises(L.QConvError):
            call()

"""The linear layer on 8-bit rows: argument marshalling, and the layer for autograd.

Every step runs in the HIP kernels behind the C ABI (``qconv_quantize_rows``,
``qconv_linear``, ``qconv_linear_grad_input``, ``qconv_linear_grad_weight`` in
``include/qconv.h``); there is no fallback.

One storage form serves the whole layer: :class:`Rows`, low-bit codes with one
float scale for each row.  Activations quantised by :func:`quantize_rows` are
the integer product's operand in :func:`linear` and, kept in place of the
16-bit input, what :func:`linear_grad_weight` reads in the backward pass; the
weights are rows of the same form (8-bit, or 4-bit from :func:`pack_rows4`) in
:func:`linear` and :func:`linear_grad_input`.

    x8 = quantize_rows(x)                       # rows of activations, any float type
    w8 = quantize_rows(w)                       # k x c weights
    y = linear(x8, w8, dtype=torch.bfloat16)
    dx = linear_grad_input(dy, w8)
    dw = linear_grad_weight(dy, x8)             # float32

:func:`linear_layer` is those calls as one differentiable function; with
``adapters`` the forward product serves many requests, each with its own
low-rank adapter.

Around it: :func:`norm_rows` makes the 8-bit rows as the root-mean-square norm of
a sum with the residual, and :func:`norm_rows_grad` is its gradient (both layers
together: :func:`norm_linear_layer`); :class:`GroupRows` are 4-bit weights with a
scale for each group of channels, for :func:`linear` and :func:`linear_grad_input`;
:func:`linear_experts` and its gradients take rows sorted by expert, each through
its expert's weights (:func:`experts_layer`).

    x8, h, rstd = norm_rows(x, gain, residual=h)
    y = linear(x8, pack_groups4(codes, scales, 128))
    z = linear_experts(x8, experts8, offsets)   # rows offsets[e] .. offsets[e + 1] - 1: expert e's

Tensors may live on any GPU: a call runs on their device's
current stream, or on ``stream`` (a torch stream or a raw handle), after that
stream's earlier work and no other's; what it allocates is that stream's memory, and
what it reads is kept until it has run.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple

import torch

from . import qconv
from .qconv import EINVAL, EUNSUPPORTED, QConvError, _check

DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}

_i32, _i64, _vp, _size, _f64 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_double


class Rows(NamedTuple):
    """Rows of codes: value = code * scale of its row.

    ``codes``: 8 bits: int8, rows x pitch bytes; 4 bits: int32, rows x pitch / 4
    words of eight values.  The last axis is contiguous and 16-byte vectors are
    whole (``channels`` of it are in use, the rest zero)."""
    codes: torch.Tensor
    scale: torch.Tensor      # float32, one for each row
    channels: int
    bits: int = 8


class GroupRows(NamedTuple):
    """4-bit rows with a scale for each group of channels: value = code * scale of its
    row and group.

    ``codes``: int32, rows x pitch / 4 words as of 4-bit :class:`Rows`.  ``scale``: rows
    x ceil(channels / group) of bfloat16, float16 or float32, the last axis contiguous.
    ``group``: a multiple of 32."""
    codes: torch.Tensor
    scale: torch.Tensor
    channels: int
    group: int


class Adapters(NamedTuple):
    """Low-rank adapters over one projection (see qconv_adapters)."""
    a: torch.Tensor          # adapters x rank x c
    b: torch.Tensor          # adapters x k x rank
    alpha: torch.Tensor      # float32, one factor for each adapter


class Normed(NamedTuple):
    """What :func:`norm_rows` gives: the 8-bit rows, and what its gradient reads."""
    rows: Rows
    sum: torch.Tensor        # x plus the residual, or x itself
    rstd: torch.Tensor       # float32, one for each row


class QConvRows(ctypes.Structure):
    _fields_ = [("codes", _vp), ("scale", _vp), ("pitch", _i64), ("rows", _i32), ("channels", _i32), ("bits", _i32)]


class QConvGroupRows(ctypes.Structure):
    _fields_ = [("codes", _vp), ("scale", _vp), ("pitch", _i64), ("scale_pitch", _i64), ("rows", _i32), ("channels", _i32),
                ("group", _i32), ("scale_dtype", _i32)]


class QConvAdapters(ctypes.Structure):
    _fields_ = [("a", _vp), ("b", _vp), ("alpha", _vp), ("row", _vp), ("count", _i32), ("rank", _i32)]


_calls = None


def _lib():
    """The library with this module's entry points declared."""
    global _calls
    if _calls is None:
        L, P = qconv.lib(), ctypes.POINTER
        L.qconv_quantize_rows.argtypes = [_vp, _i32, _i64, _i32, _i32, _vp, _i64, _vp, _vp]
        L.qconv_linear_workspace_bytes.argtypes = [_i32, _i32, P(QConvAdapters), P(_size)]
        L.qconv_linear.argtypes = [P(QConvRows), P(QConvRows), P(QConvAdapters), _vp, _i32, _i64, _vp, _size, _vp]
        L.qconv_linear_grad_workspace_bytes.argtypes = [_i32, _i32, _i32, P(_size)]
        L.qconv_linear_grad_input.argtypes = [_vp, _i32, _i64, _i32, P(QConvRows), _vp, _i64, _vp, _size, _vp]
        L.qconv_linear_grad_weight.argtypes = [_vp, _i32, _i64, _i32, P(QConvRows), _vp, _i64, _vp, _size, _vp]
        L.qconv_norm_rows.argtypes = [_vp, _i64, _vp, _i64, _vp, _i64, _i32, _vp, _i32, _f64, _i32, _i32, _vp, _i64, _vp, _vp,
                                      _vp]
        L.qconv_norm_rows_grad_workspace_bytes.argtypes = [_i32, _i32, P(_size)]
        L.qconv_norm_rows_grad.argtypes = [_vp, _i64, _vp, _i64, _vp, _i64, _i32, _vp, _i32, _vp, _i32, _i32, _vp, _i64, _vp,
                                           _vp, _size, _vp]
        L.qconv_linear_groups.argtypes = [P(QConvRows), P(QConvGroupRows), _vp, _i32, _i64, _vp]
        L.qconv_linear_groups_grad_input.argtypes = [_vp, _i32, _i64, _i32, P(QConvGroupRows), _vp, _i64, _vp, _size, _vp]
        for f, w in (("", QConvRows), ("_groups", QConvGroupRows)):
            getattr(L, f"qconv_linear_experts{f}").argtypes = [P(QConvRows), P(w), _vp, _i32, _vp, _i32, _i64, _vp]
            getattr(L, f"qconv_linear_experts{f}_grad_input").argtypes = [_vp, _i32, _i64, _i32, P(w), _vp, _i32, _vp, _i64, _vp]
        L.qconv_linear_experts_grad_weight.argtypes = [_vp, _i32, _i64, _i32, P(QConvRows), _vp, _i32, _vp, _i64, _vp]
        for f in ("qconv_linear_groups", "qconv_linear_groups_grad_input", "qconv_linear_experts",
                  "qconv_linear_experts_groups", "qconv_linear_experts_grad_input", "qconv_linear_experts_groups_grad_input",
                  "qconv_linear_experts_grad_weight"):
            getattr(L, f).restype = ctypes.c_int
        for f in ("qconv_quantize_rows", "qconv_norm_rows", "qconv_norm_rows_grad_workspace_bytes", "qconv_norm_rows_grad", "qconv_linear_workspace_bytes", "qconv_linear",
                  "qconv_linear_grad_workspace_bytes", "qconv_linear_grad_input", "qconv_linear_grad_weight"):
            getattr(L, f).restype = ctypes.c_int
        _calls = L
    return _calls


def _matrix(t: torch.Tensor, name: str, dtypes=(torch.bfloat16, torch.float16)) -> None:
    if t.dtype not in dtypes or t.dim() != 2:
        raise QConvError(EINVAL, f"{name} must be a matrix of {' or '.join(str(d).split('.')[1] for d in dtypes)}")
    if not t.is_cuda:
        raise QConvError(EINVAL, f"{name} must be a device tensor")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise QConvError(EINVAL, f"{name}: the columns of a row must be contiguous")


def _ld(t: torch.Tensor) -> int:
    """Elements from row to row (of a single row: its length)."""
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)


def _codes_arg(codes: torch.Tensor, channels: int, bits: int, name: str, device: torch.device) -> QConvRows:
    """Rows of codes without their scales."""
    if codes.dim() != 2 or codes.dtype is not (torch.int32 if bits == 4 else torch.int8):
        raise QConvError(EINVAL, f"{name}.codes must be a matrix of {'int32 words' if bits == 4 else 'int8'}")
    m, width = codes.shape
    pitch, step = codes.stride()
    if width > 1 and step != 1:
        raise QConvError(EINVAL, f"{name}.codes: the codes of a row must be contiguous")
    if m < 2:
        pitch = width
    if bits == 4:
        width, pitch = width * 4, pitch * 4
    if width < (channels * bits // 8 + 15) // 16 * 16:
        raise QConvError(EINVAL, f"{name}.codes: rows of {width} bytes do not hold {channels} channels in whole "
                                 "16-byte vectors")
    if codes.get_device() != device.index:
        raise QConvError(EINVAL, f"{name} must be on {device}")
    return QConvRows(codes.data_ptr(), None, pitch, m, channels, bits)


def _rows_arg(r: Rows, name: str, device: torch.device) -> QConvRows:
    codes, scale, channels, bits = r
    a = _codes_arg(codes, channels, bits, name, device)
    if scale.dtype is not torch.float32 or scale.shape != (a.rows,) or not scale.is_contiguous():
        raise QConvError(EINVAL, f"{name}.scale must be one float32 for each row")
    if scale.get_device() != device.index:
        raise QConvError(EINVAL, f"{name} must be on {device}")
    a.scale = scale.data_ptr()
    return a


def _group_rows_arg(r: GroupRows, name: str, device: torch.device) -> QConvGroupRows:
    codes, scale, channels, group = r
    if scale.dtype not in DTYPES or scale.dim() != 2 or scale.shape[0] != codes.shape[0]:
        raise QConvError(EINVAL, f"{name}.scale must be one row of bfloat16, float16 or float32 for each row of codes")
    if group < 1 or scale.shape[1] != -(-channels // group):
        raise QConvError(EINVAL, f"{name}.scale must have one column for each {group} of {channels} channels")
    if scale.shape[1] > 1 and scale.stride(1) != 1:
        raise QConvError(EINVAL, f"{name}.scale: the scales of a row must be contiguous")
    if scale.get_device() != device.index:
        raise QConvError(EINVAL, f"{name} must be on {device}")
    # (the codes as those of 4-bit rows)
    a = _codes_arg(codes, channels, 4, name, device)
    return QConvGroupRows(a.codes, scale.data_ptr(), a.pitch, _ld(scale), a.rows, channels, group, DTYPES[scale.dtype])


def _weights_arg(w: Rows | GroupRows, device: torch.device):
    """The weights for a call, and the part of the entry points' names that says their form."""
    if isinstance(w, GroupRows):
        return _group_rows_arg(w, "w", device), "_groups"
    return _rows_arg(w, "w", device), ""


def _empty(shape, dtype: torch.dtype, device: torch.device, stream) -> torch.Tensor:
    """Memory that the call writes on ``stream``: that stream's own, since what was freed
    on another one may still be in use by work queued there.  It is kept for the current
    stream too, where the caller may read it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(_as_stream(stream, device)):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(torch.cuda.current_stream(device))
    return t


def _as_stream(stream, device: torch.device) -> torch.cuda.Stream:
    """``stream``, or torch's view of a raw handle."""
    if isinstance(stream, torch.cuda.Stream):
        return stream
    return torch.cuda.ExternalStream(_stream(stream, device), device=device)


def _hold(stream, *tensors) -> None:
    """Keeps the memory of what a call on ``stream`` reads or writes until it has run,
    should the caller give it back before."""
    if stream is not None:
        for t in tensors:
            if t is not None:
                t.record_stream(_as_stream(stream, t.device))


def _on(device: torch.device, out: torch.Tensor | None, shape: tuple, dtype: torch.dtype, name: str,
        stream) -> torch.Tensor:
    """The output: new, or the caller's after a check."""
    if out is None:
        return _empty(shape, dtype, device, stream)
    if out.shape != shape or out.dtype is not dtype or out.device != device:
        raise QConvError(EINVAL, f"{name} must be {shape} of {dtype} on {device}")
    if shape[1] > 1 and out.stride(1) != 1:
        raise QConvError(EINVAL, f"{name}: the columns of a row must be contiguous")
    return out


def _workspace(need: int, workspace: torch.Tensor | None, device: torch.device, stream):
    """(tensor to keep, pointer, bytes) of the call's scratch: the caller's, or
    from torch's allocator."""
    if workspace is not None:
        if workspace.device != device or not workspace.is_contiguous():
            raise QConvError(EINVAL, f"workspace must be contiguous and on {device}")
        return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()
    if not need:
        return None, None, 0
    t = _empty(need, torch.uint8, device, stream)
    return t, t.data_ptr(), need


def _stream(stream, device: torch.device) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device.index)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _call(device: torch.device, fn, *args) -> int:
    """fn on the tensors' device (a launch goes to the current one)."""
    if torch._C._cuda_getDevice() == device.index:
        return fn(*args)
    with torch.cuda.device(device):
        return fn(*args)


def rows_pitch(channels: int) -> int:
    """Bytes of an 8-bit row: its channels in whole 16-byte vectors."""
    return (channels + 15) // 16 * 16


def quantize_rows(x: torch.Tensor, out: Rows | None = None, stream=None) -> Rows:
    """Rows of bfloat16, float16 or float32 to 8 bits (qconv_quantize_rows)."""
    _matrix(x, "x", tuple(DTYPES))
    m, c = x.shape
    device = x.device
    out, to = _rows_out(out, m, c, device, stream)
    _check(_call(device, _lib().qconv_quantize_rows, x.data_ptr(), DTYPES[x.dtype], _ld(x), m, c, *to,
                 _stream(stream, device)), "qconv_quantize_rows")
    _hold(stream, x, out.codes, out.scale)
    return out


def _gain(t: torch.Tensor, c: int, device: torch.device) -> None:
    if t.dtype not in DTYPES or t.shape != (c,) or not t.is_contiguous() or t.device != device:
        raise QConvError(EINVAL, f"gain must be {c} contiguous bfloat16, float16 or float32 on {device}")


def _like(t: torch.Tensor, x: torch.Tensor, name: str) -> None:
    if t.dtype is not x.dtype or t.shape != x.shape or t.device != x.device:
        raise QConvError(EINVAL, f"{name} must be {tuple(x.shape)} of {x.dtype} on {x.device}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise QConvError(EINVAL, f"{name}: the columns of a row must be contiguous")


def _rows_out(out: Rows | None, m: int, c: int, device: torch.device, stream):
    """8-bit rows to write, new or the caller's after a check, and what a call takes of them."""
    if out is None:
        pitch = rows_pitch(c)
        codes, scale = _empty((m, pitch), torch.int8, device, stream), _empty(m, torch.float32, device, stream)
        return Rows(codes, scale, c), (codes.data_ptr(), pitch, scale.data_ptr())
    if out.bits != 8 or out.channels != c or out.codes.shape[0] != m:
        raise QConvError(EINVAL, f"out must be 8-bit rows, {m} of {c} channels")
    r = _rows_arg(out, "out", device)
    return out, (r.codes, r.pitch, r.scale)


def norm_rows(x: torch.Tensor, gain: torch.Tensor, *, residual: torch.Tensor | None = None, eps: float = 1e-6,
              out: Rows | None = None, sum_out: torch.Tensor | None = None, stream=None) -> Normed:
    """Root-mean-square norm of the rows of x plus the residual, as 8-bit rows
    (qconv_norm_rows).  ``sum_out``: where x + residual goes; the whole of x or of the
    residual may be given, new memory otherwise."""
    _matrix(x, "x", tuple(DTYPES))
    m, c = x.shape
    device = x.device
    _gain(gain, c, device)
    total = x
    if residual is not None:
        _like(residual, x, "residual")
        total = _on(device, sum_out, (m, c), x.dtype, "sum_out", stream)
    elif sum_out is not None:
        raise QConvError(EINVAL, "sum_out without a residual")
    rows, to = _rows_out(out, m, c, device, stream)
    rstd = _empty(m, torch.float32, device, stream)
    add = (None, 0, None, 0) if residual is None else (residual.data_ptr(), _ld(residual), total.data_ptr(), _ld(total))
    _check(_call(device, _lib().qconv_norm_rows, x.data_ptr(), _ld(x), *add, DTYPES[x.dtype], gain.data_ptr(),
                 DTYPES[gain.dtype], eps, m, c, *to, rstd.data_ptr(), _stream(stream, device)), "qconv_norm_rows")
    _hold(stream, x, gain, residual, rows.codes, rows.scale, sum_out)
    return Normed(rows, total, rstd)


def norm_grad_workspace_bytes(rows: int, channels: int) -> int:
    """Scratch of :func:`norm_rows_grad`."""
    n = _size(0)
    _check(_lib().qconv_norm_rows_grad_workspace_bytes(rows, channels, ctypes.byref(n)), "qconv_norm_rows_grad_workspace_bytes")
    return n.value


def norm_rows_grad(dy: torch.Tensor, h: torch.Tensor, gain: torch.Tensor, rstd: torch.Tensor, *,
                   dsum: torch.Tensor | None = None, out: torch.Tensor | None = None,
                   workspace: torch.Tensor | None = None, stream=None) -> tuple[torch.Tensor, torch.Tensor]:
    """Gradients (of x and the residual alike, of dy's type; of the gain, float32) from
    the gradient dy of the norm's values and dsum of h, the norm's ``sum``
    (qconv_norm_rows_grad).  ``out`` may be dsum itself."""
    _matrix(dy, "dy", tuple(DTYPES))
    _like(h, dy, "h")
    m, c = dy.shape
    device = dy.device
    _gain(gain, c, device)
    if rstd.dtype is not torch.float32 or rstd.shape != (m,) or not rstd.is_contiguous() or rstd.device != device:
        raise QConvError(EINVAL, f"rstd must be one float32 for each row, on {device}")
    if dsum is not None:
        _like(dsum, dy, "dsum")
    dx = _on(device, out, (m, c), dy.dtype, "out", stream)
    dgain = _empty(c, torch.float32, device, stream)
    keep, ws, ws_bytes = _workspace(norm_grad_workspace_bytes(m, c), workspace, device, stream)
    _check(_call(device, _lib().qconv_norm_rows_grad, dy.data_ptr(), _ld(dy), h.data_ptr(), _ld(h),
                 None if dsum is None else dsum.data_ptr(), 0 if dsum is None else _ld(dsum), DTYPES[dy.dtype],
                 gain.data_ptr(), DTYPES[gain.dtype], rstd.data_ptr(), m, c, dx.data_ptr(), _ld(dx), dgain.data_ptr(), ws,
                 ws_bytes, _stream(stream, device)), "qconv_norm_rows_grad")
    _hold(stream, dy, h, gain, rstd, dsum, out, workspace)
    return dx, dgain


def pack_rows4(codes: torch.Tensor, scale: torch.Tensor, stream=None) -> Rows:
    """int8 codes (rows x channels, saturated into [-8, 7]) and their float32
    scales as 4-bit rows: qconv_pack of rows of whole 16-byte vectors."""
    if codes.dim() != 2 or codes.dtype != torch.int8:
        raise QConvError(EINVAL, "codes must be an int8 matrix")
    if not codes.is_cuda:
        raise QConvError(EINVAL, "codes must be a device tensor")
    k, c = codes.shape
    if c % 8:
        raise QConvError(EINVAL, f"4-bit rows need channels % 8 == 0 (got {c})")
    device = codes.device
    current = torch.cuda.current_stream(device)
    # (the copies too: they are made and given back on the stream that reads them)
    with torch.cuda.stream(current if stream is None else _as_stream(stream, device)):
        _hold(stream, codes)
        if c % 32:
            codes = torch.nn.functional.pad(codes, (0, 32 - c % 32))
        words = qconv.pack(codes.contiguous().reshape(k, -1, 1, 1), 4, True)
    words.record_stream(current)
    return Rows(words.reshape(k, -1), scale, c, 4)


def pack_groups4(codes: torch.Tensor, scale: torch.Tensor, group: int, stream=None) -> GroupRows:
    """int8 codes (rows x channels, saturated into [-8, 7]) and the scales of their
    groups of channels as 4-bit rows (see :func:`pack_rows4`)."""
    words, _, channels, _ = pack_rows4(codes, scale, stream)
    return GroupRows(words, scale, channels, group)


def _adapters_arg(ad: Adapters, row_adapter, m: int, c: int, k: int, dtype, device) -> QConvAdapters:
    a, b, alpha = ad
    n, rank = a.shape[:2] if a.dim() == 3 else (0, 0)
    if a.shape != (n, rank, c) or b.shape != (n, k, rank):
        raise QConvError(EINVAL, f"adapters: a must be n x rank x {c} and b n x {k} x rank")
    if a.dtype is not dtype or b.dtype is not dtype:
        raise QConvError(EINVAL, f"adapters: a and b must be of y's type, {dtype}")
    if alpha.dtype is not torch.float32 or alpha.shape != (n,):
        raise QConvError(EINVAL, "adapters: alpha must be one float32 for each adapter")
    if row_adapter is None or row_adapter.dtype is not torch.int32 or row_adapter.shape != (m,):
        raise QConvError(EINVAL, "row_adapter must be one int32 for each row of x")
    on = device.index
    for t in (a, b, alpha, row_adapter):
        if t.get_device() != on or not t.is_contiguous():
            raise QConvError(EINVAL, f"adapters: a, b, alpha and row_adapter must be contiguous and on {device}")
    return QConvAdapters(a.data_ptr(), b.data_ptr(), alpha.data_ptr(), row_adapter.data_ptr(), n, rank)


def linear(x: Rows, w: Rows | GroupRows, *, dtype: torch.dtype = torch.bfloat16, adapters: Adapters | None = None,
           row_adapter: torch.Tensor | None = None, out: torch.Tensor | None = None,
           workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """rows x k products of 8-bit rows with k x c weights, plus each row's
    adapter's part (qconv_linear).  ``row_adapter``: int32 for each row, -1 for
    none.  ``workspace``: any contiguous device tensor of
    :func:`linear_workspace_bytes`; made by the call if not given.  Weights with scales
    of groups (qconv_linear_groups) need none, and take no adapters."""
    if dtype not in (torch.bfloat16, torch.float16):
        raise QConvError(EINVAL, "dtype must be torch.bfloat16 or torch.float16")
    device = x.codes.device
    if device.type != "cuda":
        raise QConvError(EINVAL, "x must be on a GPU")
    rx, (rw, form) = _rows_arg(x, "x", device), _weights_arg(w, device)
    L = _lib()
    if form:
        if adapters is not None or row_adapter is not None:
            raise QConvError(EUNSUPPORTED, "adapters need weights with one scale a row")
        y = _on(device, out, (rx.rows, rw.rows), dtype, "out", stream)
        _check(_call(device, L.qconv_linear_groups, ctypes.byref(rx), ctypes.byref(rw), y.data_ptr(), DTYPES[dtype], _ld(y),
                     _stream(stream, device)), "qconv_linear_groups")
        _hold(stream, *x[:2], *w[:2], out)
        return y
    ad, need = None, 0
    if adapters is not None:
        ad = _adapters_arg(adapters, row_adapter, rx.rows, rx.channels, rw.rows, dtype, device)
        need = _linear_workspace(L, rx.rows, rx.channels, ad)
        ad = ctypes.byref(ad)
    elif row_adapter is not None:
        raise QConvError(EINVAL, "row_adapter without adapters")
    y = _on(device, out, (rx.rows, rw.rows), dtype, "out", stream)
    keep, ws, ws_bytes = _workspace(need, workspace, device, stream)
    _check(_call(device, L.qconv_linear, ctypes.byref(rx), ctypes.byref(rw), ad, y.data_ptr(), DTYPES[dtype], _ld(y), ws,
                 ws_bytes, _stream(stream, device)), "qconv_linear")
    _hold(stream, *x[:2], *w[:2], *(adapters or ()), row_adapter, out, workspace)
    return y


def _linear_workspace(L, m: int, c: int, ad: QConvAdapters) -> int:
    n = _size(0)
    _check(L.qconv_linear_workspace_bytes(m, c, ctypes.byref(ad), ctypes.byref(n)), "qconv_linear_workspace_bytes")
    return n.value


def linear_workspace_bytes(rows: int, channels: int, rank: int = 0) -> int:
    """Scratch of :func:`linear` (0 without adapters, rank == 0)."""
    return _linear_workspace(_lib(), int(rows), int(channels), QConvAdapters(None, None, None, None, int(rank > 0), int(rank)))


def grad_workspace_bytes(rows: int, cols: int, depth: int) -> int:
    """Scratch of a backward product of rows x cols results summed over depth:
    (m, c, k) for :func:`linear_grad_input`, (k, c, m) for :func:`linear_grad_weight`."""
    n = _size(0)
    _check(_lib().qconv_linear_grad_workspace_bytes(int(rows), int(cols), int(depth), ctypes.byref(n)),
           "qconv_linear_grad_workspace_bytes")
    return n.value


def linear_grad_input(dy: torch.Tensor, w: Rows | GroupRows, *, out: torch.Tensor | None = None,
                      workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """dy (rows x k) times the weights (k x c), of dy's type (qconv_linear_grad_input, or
    qconv_linear_groups_grad_input by weights with scales of groups)."""
    _matrix(dy, "dy")
    device = dy.device
    rw, form = _weights_arg(w, device)
    name = f"qconv_linear{form}_grad_input"
    m = dy.shape[0]
    if dy.shape[1] != rw.rows:
        raise QConvError(EINVAL, f"dy has {dy.shape[1]} columns, w {rw.rows} rows")
    dx = _on(device, out, (m, rw.channels), dy.dtype, "out", stream)
    keep, ws, ws_bytes = _workspace(grad_workspace_bytes(m, rw.channels, rw.rows), workspace, device, stream)
    _check(_call(device, getattr(_lib(), name), dy.data_ptr(), DTYPES[dy.dtype], _ld(dy), m, ctypes.byref(rw),
                 dx.data_ptr(), _ld(dx), ws, ws_bytes, _stream(stream, device)), name)
    _hold(stream, dy, *w[:2], out, workspace)
    return dx


def linear_grad_weight(dy: torch.Tensor, x: Rows, *, out: torch.Tensor | None = None,
                       workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """dy transposed (k x rows) times the 8-bit rows (rows x c): float32 k x c
    (qconv_linear_grad_weight)."""
    _matrix(dy, "dy")
    device = dy.device
    rx = _rows_arg(x, "x", device)
    m, k = dy.shape
    if m != rx.rows:
        raise QConvError(EINVAL, f"dy has {m} rows, x {rx.rows}")
    dw = _on(device, out, (k, rx.channels), torch.float32, "out", stream)
    keep, ws, ws_bytes = _workspace(grad_workspace_bytes(k, rx.channels, m), workspace, device, stream)
    _check(_call(device, _lib().qconv_linear_grad_weight, dy.data_ptr(), DTYPES[dy.dtype], _ld(dy), k, ctypes.byref(rx),
                 dw.data_ptr(), _ld(dw), ws, ws_bytes, _stream(stream, device)), "qconv_linear_grad_weight")
    _hold(stream, dy, *x[:2], out, workspace)
    return dw


def _experts_arg(offsets: torch.Tensor, device: torch.device) -> tuple[int, int]:
    """(pointer, experts)."""
    if offsets.dtype is not torch.int32 or offsets.dim() != 1 or offsets.shape[0] < 2 or not offsets.is_contiguous():
        raise QConvError(EINVAL, "offsets must be int32: the first row of each expert, and the end of the last one's")
    if offsets.get_device() != device.index:
        raise QConvError(EINVAL, f"offsets must be on {device}")
    return offsets.data_ptr(), offsets.shape[0] - 1


def _of_experts(rows: int, experts: int) -> int:
    if rows % experts:
        raise QConvError(EINVAL, f"w has {rows} rows, not those of {experts} experts")
    return rows // experts


def linear_experts(x: Rows, w: Rows | GroupRows, offsets: torch.Tensor, *, dtype: torch.dtype = torch.bfloat16,
                   out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Rows sorted by expert, each times its expert's k x c weights (qconv_linear_experts):
    expert e has rows ``offsets[e]`` to ``offsets[e + 1] - 1`` of x, and rows e k to
    e k + k - 1 of w.  ``offsets`` is int32 on the device and read there.  Rows of no
    expert keep what ``out`` holds (memory made by the call: anything)."""
    if dtype not in (torch.bfloat16, torch.float16):
        raise QConvError(EINVAL, "dtype must be torch.bfloat16 or torch.float16")
    device = x.codes.device
    if device.type != "cuda":
        raise QConvError(EINVAL, "x must be on a GPU")
    rx, (rw, form) = _rows_arg(x, "x", device), _weights_arg(w, device)
    at, experts = _experts_arg(offsets, device)
    y = _on(device, out, (rx.rows, _of_experts(rw.rows, experts)), dtype, "out", stream)
    name = f"qconv_linear_experts{form}"
    _check(_call(device, getattr(_lib(), name), ctypes.byref(rx), ctypes.byref(rw), at, experts, y.data_ptr(), DTYPES[dtype],
                 _ld(y), _stream(stream, device)), name)
    _hold(stream, *x[:2], *w[:2], offsets, out)
    return y


def linear_experts_grad_input(dy: torch.Tensor, w: Rows | GroupRows, offsets: torch.Tensor, *,
                              out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Each row of dy (rows x k) times its expert's weights (k x c), of dy's type
    (qconv_linear_experts_grad_input).  Rows of no expert keep what ``out`` holds."""
    _matrix(dy, "dy")
    device = dy.device
    rw, form = _weights_arg(w, device)
    at, experts = _experts_arg(offsets, device)
    m, k = dy.shape
    if k != _of_experts(rw.rows, experts):
        raise QConvError(EINVAL, f"dy has {k} columns, an expert {rw.rows // experts} rows")
    dx = _on(device, out, (m, rw.channels), dy.dtype, "out", stream)
    name = f"qconv_linear_experts{form}_grad_input"
    _check(_call(device, getattr(_lib(), name), dy.data_ptr(), DTYPES[dy.dtype], _ld(dy), m, ctypes.byref(rw), at, experts,
                 dx.data_ptr(), _ld(dx), _stream(stream, device)), name)
    _hold(stream, dy, *w[:2], offsets, out)
    return dx


def linear_experts_grad_weight(dy: torch.Tensor, x: Rows, offsets: torch.Tensor, *, out: torch.Tensor | None = None,
                               stream=None) -> torch.Tensor:
    """For each expert, its rows of dy transposed (k x rows) times its rows of x: float32,
    experts x k x c, zeros for an expert without rows (qconv_linear_experts_grad_weight).
    ``out``: contiguous."""
    _matrix(dy, "dy")
    device = dy.device
    rx = _rows_arg(x, "x", device)
    at, experts = _experts_arg(offsets, device)
    m, k = dy.shape
    if m != rx.rows:
        raise QConvError(EINVAL, f"dy has {m} rows, x {rx.rows}")
    shape = (experts, k, rx.channels)
    if out is None:
        dw = _empty(shape, torch.float32, device, stream)
    elif out.shape != shape or out.dtype is not torch.float32 or out.device != device or not out.is_contiguous():
        raise QConvError(EINVAL, f"out must be {shape} of torch.float32, contiguous and on {device}")
    else:
        dw = out
    _check(_call(device, _lib().qconv_linear_experts_grad_weight, dy.data_ptr(), DTYPES[dy.dtype], _ld(dy), k,
                 ctypes.byref(rx), at, experts, dw.data_ptr(), rx.channels, _stream(stream, device)),
           "qconv_linear_experts_grad_weight")
    _hold(stream, dy, *x[:2], offsets, out)
    return dw


def _readable(t: torch.Tensor) -> torch.Tensor:
    """The matrix, or a copy where the operators do not read it in place: columns apart,
    rows that overlap (a broadcast one), rows more than 2^21 elements apart."""
    if t.dim() != 2:
        return t   # (refused by the operator)
    m, n = t.shape
    apart = n > 1 and t.stride(1) != 1
    return t.contiguous() if apart or (m > 1 and not n <= t.stride(0) <= 1 << 21) else t


class _LinearLayer(torch.autograd.Function):
    """Rounding to 8 bits is taken as the identity in the backward pass: the
    gradients are those of the product of the rounded values."""

    @staticmethod
    def forward(ctx, x, w):
        x8, w8 = quantize_rows(_readable(x)), quantize_rows(_readable(w))
        ctx.save_for_backward(x8.codes, x8.scale, w8.codes, w8.scale)
        ctx.channels, ctx.x_dtype, ctx.w_dtype = x8.channels, x.dtype, w.dtype
        return linear(x8, w8, dtype=x.dtype)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x_codes, x_scale, w_codes, w_scale = ctx.saved_tensors
        dy = _readable(dy)
        dx = dw = None
        if ctx.needs_input_grad[0]:
            dx = linear_grad_input(dy, Rows(w_codes, w_scale, ctx.channels))
        if ctx.needs_input_grad[1]:
            dw = linear_grad_weight(dy, Rows(x_codes, x_scale, ctx.channels)).to(ctx.w_dtype)
        return dx, dw


def linear_layer(x: torch.Tensor, w: torch.Tensor) -> torch.Tensor:
    """x (... x c, bfloat16 or float16) times the k x c weights' transpose, both
    rounded to 8-bit rows, differentiable in both.  Either may be any view.  Between
    the passes only the 8-bit rows are kept: 1 byte a value of x instead of 2."""
    y = _LinearLayer.apply(x.reshape(-1, x.shape[-1]), w)
    return y.reshape(*x.shape[:-1], w.shape[0])


class _NormLinearLayer(torch.autograd.Function):
    """The norm's rounding to 8 bits, and the weights', are taken as the identity in the
    backward pass, as in :class:`_LinearLayer`."""

    @staticmethod
    def forward(ctx, x, residual, gain, w, eps):
        ctx.set_materialize_grads(False)
        x8, h, rstd = norm_rows(_readable(x), gain.contiguous(), eps=eps,
                                residual=None if residual is None else _readable(residual))
        w8 = quantize_rows(_readable(w))
        ctx.save_for_backward(x8.codes, x8.scale, w8.codes, w8.scale, h, gain, rstd)
        ctx.channels, ctx.w_dtype = x8.channels, w.dtype
        y = linear(x8, w8, dtype=x.dtype)
        return y if residual is None else (y, h)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dsum=None):
        x_codes, x_scale, w_codes, w_scale, h, gain, rstd = ctx.saved_tensors
        needs_x, needs_residual, needs_gain, needs_w, _ = ctx.needs_input_grad
        dx = dgain = dw = None
        if dy is None:   # y was not used
            return *_NormLinearLayer._both(dsum, needs_x, needs_residual), None, None, None
        dy = _readable(dy)
        if needs_x or needs_residual or needs_gain:
            dn = linear_grad_input(dy, Rows(w_codes, w_scale, ctx.channels))
            dx, dgain = norm_rows_grad(dn, h, gain.contiguous(), rstd, dsum=None if dsum is None else _readable(dsum))
        if needs_w:
            dw = linear_grad_weight(dy, Rows(x_codes, x_scale, ctx.channels)).to(ctx.w_dtype)
        return *_NormLinearLayer._both(dx, needs_x, needs_residual), dgain.to(gain.dtype) if needs_gain else None, dw, None

    @staticmethod
    def _both(dx, needs_x, needs_residual):
        """The gradient of x and of the residual: tensors of their own, since either may
        become a leaf's and be changed in place."""
        if dx is None or not (needs_x and needs_residual):
            return dx if needs_x else None, dx if needs_residual else None
        return dx, dx.clone()


def norm_linear_layer(x: torch.Tensor, gain: torch.Tensor, w: torch.Tensor, *, residual: torch.Tensor | None = None,
                      eps: float = 1e-6) -> tuple[torch.Tensor, torch.Tensor]:
    """The root-mean-square norm of x plus the residual (... x c, bfloat16 or float16)
    times the k x c weights' transpose, through 8-bit rows, and that sum, the next
    residual: differentiable in x, the residual, the gain and the weights.  Between the
    passes the sum and the 8-bit rows are kept."""
    if residual is not None and (residual.shape != x.shape or residual.dtype is not x.dtype):
        raise QConvError(EINVAL, "residual must be of x's shape and type")
    c = x.shape[-1]
    flat = x.reshape(-1, c)
    if residual is None:
        y, total = _NormLinearLayer.apply(flat, None, gain, w, eps), flat
    else:
        y, total = _NormLinearLayer.apply(flat, residual.reshape(-1, c), gain, w, eps)
    return y.reshape(*x.shape[:-1], w.shape[0]), total.reshape(x.shape)


class _ExpertsLayer(torch.autograd.Function):
    """As :class:`_LinearLayer`; rows of no expert give zeros, and get a gradient of zero."""

    @staticmethod
    def forward(ctx, x, w, offsets):
        experts, k, c = w.shape
        x8, w8 = quantize_rows(_readable(x)), quantize_rows(_readable(w.reshape(experts * k, c)))
        ctx.save_for_backward(x8.codes, x8.scale, w8.codes, w8.scale, offsets)
        ctx.channels, ctx.w_dtype = c, w.dtype
        return linear_experts(x8, w8, offsets, dtype=x.dtype, out=x.new_zeros((x.shape[0], k)))

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x_codes, x_scale, w_codes, w_scale, offsets = ctx.saved_tensors
        dy = _readable(dy)
        dx = dw = None
        if ctx.needs_input_grad[0]:
            dx = linear_experts_grad_input(dy, Rows(w_codes, w_scale, ctx.channels), offsets,
                                           out=dy.new_zeros((dy.shape[0], ctx.channels)))
        if ctx.needs_input_grad[1]:
            dw = linear_experts_grad_weight(dy, Rows(x_codes, x_scale, ctx.channels), offsets).to(ctx.w_dtype)
        return dx, dw, None


def experts_layer(x: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor) -> torch.Tensor:
    """Rows sorted by expert (m x c, bfloat16 or float16), each times its expert's weights
    (w: experts x k x c) through 8-bit rows: differentiable in both.  ``offsets`` as of
    :func:`linear_experts`."""
    if w.dim() != 3 or offsets.dim() != 1 or offsets.shape[0] != w.shape[0] + 1:
        raise QConvError(EINVAL, "w must be experts x k x c, and offsets hold one number more than experts")
    return _ExpertsLayer.apply(x, w, offsets)

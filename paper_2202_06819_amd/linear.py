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
low-rank adapter.  Tensors may live on any GPU: a call runs on their device's
current stream, or on ``stream`` (a torch stream or a raw handle), after that
stream's earlier work and no other's; what it allocates is that stream's memory, and
what it reads is kept until it has run.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple

import torch

from . import qconv
from .qconv import EINVAL, QConvError, _check

DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}

_i32, _i64, _vp, _size = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t


class Rows(NamedTuple):
    """Rows of codes: value = code * scale of its row.

    ``codes``: 8 bits: int8, rows x pitch bytes; 4 bits: int32, rows x pitch / 4
    words of eight values.  The last axis is contiguous and 16-byte vectors are
    whole (``channels`` of it are in use, the rest zero)."""
    codes: torch.Tensor
    scale: torch.Tensor      # float32, one for each row
    channels: int
    bits: int = 8


class Adapters(NamedTuple):
    """Low-rank adapters over one projection (see qconv_adapters)."""
    a: torch.Tensor          # adapters x rank x c
    b: torch.Tensor          # adapters x k x rank
    alpha: torch.Tensor      # float32, one factor for each adapter


class QConvRows(ctypes.Structure):
    _fields_ = [("codes", _vp), ("scale", _vp), ("pitch", _i64), ("rows", _i32), ("channels", _i32), ("bits", _i32)]


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
        for f in ("qconv_quantize_rows", "qconv_linear_workspace_bytes", "qconv_linear",
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


def _rows_arg(r: Rows, name: str, device: torch.device) -> QConvRows:
    codes, scale, channels, bits = r
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
    if scale.dtype is not torch.float32 or scale.shape != (m,) or not scale.is_contiguous():
        raise QConvError(EINVAL, f"{name}.scale must be one float32 for each row")
    if codes.get_device() != device.index or scale.get_device() != device.index:
        raise QConvError(EINVAL, f"{name} must be on {device}")
    return QConvRows(codes.data_ptr(), scale.data_ptr(), pitch, m, channels, bits)


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
    if out is None:
        pitch = rows_pitch(c)
        codes = _empty((m, pitch), torch.int8, device, stream)
        scale = _empty(m, torch.float32, device, stream)
        out = Rows(codes, scale, c)
        to = (codes.data_ptr(), pitch, scale.data_ptr())
    else:
        if out.bits != 8 or out.channels != c or out.codes.shape[0] != m:
            raise QConvError(EINVAL, f"out must be 8-bit rows, {m} of {c} channels")
        r = _rows_arg(out, "out", device)
        to = (r.codes, r.pitch, r.scale)
    _check(_call(device, _lib().qconv_quantize_rows, x.data_ptr(), DTYPES[x.dtype], _ld(x), m, c, *to,
                 _stream(stream, device)), "qconv_quantize_rows")
    _hold(stream, x, out.codes, out.scale)
    return out


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


def linear(x: Rows, w: Rows, *, dtype: torch.dtype = torch.bfloat16, adapters: Adapters | None = None,
           row_adapter: torch.Tensor | None = None, out: torch.Tensor | None = None,
           workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """rows x k products of 8-bit rows with k x c weights, plus each row's
    adapter's part (qconv_linear).  ``row_adapter``: int32 for each row, -1 for
    none.  ``workspace``: any contiguous device tensor of
    :func:`linear_workspace_bytes`; made by the call if not given."""
    if dtype not in (torch.bfloat16, torch.float16):
        raise QConvError(EINVAL, "dtype must be torch.bfloat16 or torch.float16")
    device = x.codes.device
    if device.type != "cuda":
        raise QConvError(EINVAL, "x must be on a GPU")
    rx, rw = _rows_arg(x, "x", device), _rows_arg(w, "w", device)
    L = _lib()
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


def linear_grad_input(dy: torch.Tensor, w: Rows, *, out: torch.Tensor | None = None,
                      workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """dy (rows x k) times the weights (k x c), of dy's type (qconv_linear_grad_input)."""
    _matrix(dy, "dy")
    device = dy.device
    rw = _rows_arg(w, "w", device)
    m = dy.shape[0]
    if dy.shape[1] != rw.rows:
        raise QConvError(EINVAL, f"dy has {dy.shape[1]} columns, w {rw.rows} rows")
    dx = _on(device, out, (m, rw.channels), dy.dtype, "out", stream)
    keep, ws, ws_bytes = _workspace(grad_workspace_bytes(m, rw.channels, rw.rows), workspace, device, stream)
    _check(_call(device, _lib().qconv_linear_grad_input, dy.data_ptr(), DTYPES[dy.dtype], _ld(dy), m, ctypes.byref(rw),
                 dx.data_ptr(), _ld(dx), ws, ws_bytes, _stream(stream, device)), "qconv_linear_grad_input")
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

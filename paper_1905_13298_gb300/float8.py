"""Tensor-level helpers of the 8-bit floating-point operators (see the header's section on them).

Calls run on the current stream, or on ``stream`` (a torch stream or a handle), to which what they return then belongs.

An ``F8Matrix`` holds 8-bit values and their scales, one per block of 128.  The helpers check what the C ABI cannot
see (dtype, shape, strides, device), allocate outputs with torch, and make one call each.

A training step of a gated feed-forward block reads::

    # 8-bit rows of the norm, the new residual stream; powers of two, since the blocks of n change below
    n, h, rstd = rmsnorm_f8(x, norm_w, residual=stream, pow2=True)
    gu = linear_f8(n, w_gu)                                    # w_gu: quantize_f8(weight, "tiles", "tiles")[0]
    a, kept = gated_f8(gu, features)                           # only `kept` is needed again
    y = linear_f8(a, w_down)
    ...
    d, d_t = quantize_f8(dy, "rows", "rows")                   # the gradient by rows and by columns
    da = linear_f8(d, w_down_t)
    dgu, dgu_t, a_t = gated_f8_backward(kept, da)
    grad_down = linear_f8(d_t, a_t, add=grad_down, out=grad_down, dtype=torch.float32)
    n_t = quantize_f8(n, None, "tiles", pow2=True)[1]          # n's values, turned, not rounded again
    grad_gu = linear_f8(dgu_t, n_t, add=grad_gu, out=grad_gu, dtype=torch.float32)
    dx, grad_norm = rmsnorm_f8_backward(linear_f8(dgu, w_gu_t), h, rstd, norm_w, dh=dy)
"""
from __future__ import annotations

from operator import attrgetter

import torch

from . import (DS_F8_E4M3, DS_F8_E5M2, DS_F8_POW2, DS_F8_ROWS, DS_F8_TILES, DS_TYPE_BF16, DS_TYPE_F16, DS_TYPE_F32,
               _check, _stream, ds_expand_shift_weights_f8, ds_f8_matrix, lib)

_TYPES = {torch.float32: DS_TYPE_F32, torch.bfloat16: DS_TYPE_BF16, torch.float16: DS_TYPE_F16}
_FORMATS = {torch.float8_e4m3fn: DS_F8_E4M3, torch.float8_e5m2: DS_F8_E5M2}
_BLOCKS = {"rows": DS_F8_ROWS, "tiles": DS_F8_TILES}
BLOCK = 128


class F8Matrix:
    """8-bit values ``q`` [rows, cols] (``torch.float8_e4m3fn`` or ``float8_e5m2``, rows a multiple of 16 bytes apart)
    and float32 scales: ``scale`` [rows, ceil(cols / 128)], or with ``tiles`` [ceil(rows / 128), ceil(cols / 128)].  Both stay
    the tensors that it was made with: calls read and write their memory."""

    __slots__ = ("_q", "_scale", "desc")
    q, scale = property(attrgetter("_q")), property(attrgetter("_scale"))

    def __init__(self, q, scale, tiles: bool = False):
        fmt = _FORMATS.get(q.dtype)
        if fmt is None:
            raise ValueError(f"q must be torch.float8_e4m3fn or torch.float8_e5m2, got {q.dtype}")
        if scale.dtype != torch.float32:
            raise ValueError(f"scale must be torch.float32, got {scale.dtype}")
        if q.dim() != 2 or scale.dim() != 2:
            raise ValueError("q and scale must have two dimensions")
        rows, cols = q.shape
        ld, ld_scale = _row_stride(q, "q"), _row_stride(scale, "scale")
        if ld % 16:
            raise ValueError(f"rows of q must start a multiple of 16 bytes apart, got {ld} (pad the columns)")
        want = (-(-rows // BLOCK) if tiles else rows, -(-cols // BLOCK))
        if scale.shape != want:
            raise ValueError(f"scale has shape {tuple(scale.shape)}, expected {want}")
        if q.get_device() < 0 or q.get_device() != scale.get_device():
            raise ValueError("q and scale must be CUDA tensors of one device")
        self._q, self._scale = q, scale
        self.desc = ds_f8_matrix(q.data_ptr(), scale.data_ptr(), rows, cols, ld, ld_scale, fmt,
                                 DS_F8_TILES if tiles else DS_F8_ROWS)

    @classmethod
    def empty(cls, rows: int, cols: int, device, dtype=torch.float8_e4m3fn, tiles: bool = False) -> "F8Matrix":
        """Uninitialised memory for a matrix, rows padded to a multiple of 16 bytes."""
        fmt = _FORMATS.get(dtype)
        if fmt is None:
            raise ValueError(f"dtype must be torch.float8_e4m3fn or torch.float8_e5m2, got {dtype}")
        m = cls.__new__(cls)
        ld, nb = (cols + 15) // 16 * 16, (cols + BLOCK - 1) // BLOCK
        if ld == cols:
            m._q = torch.empty((rows, cols), dtype=dtype, device=device)
        else:
            m._q = torch.empty_strided((rows, cols), (ld, 1), dtype=dtype, device=device)
        m._scale = torch.empty(((rows + BLOCK - 1) // BLOCK if tiles else rows, nb), dtype=torch.float32, device=device)
        m.desc = ds_f8_matrix(m._q.data_ptr(), m._scale.data_ptr(), rows, cols, ld, nb, fmt,
                              DS_F8_TILES if tiles else DS_F8_ROWS)
        return m

    @property
    def rows(self) -> int:
        return self.desc.rows

    @property
    def cols(self) -> int:
        return self.desc.cols

    @property
    def tiles(self) -> bool:
        return self.desc.blocks == DS_F8_TILES

    def dequantize(self):
        """The float32 values [rows, cols]."""
        s = self.scale.repeat_interleave(BLOCK, 1)[:, : self.cols]
        if self.tiles:
            s = s.repeat_interleave(BLOCK, 0)[: self.rows]
        return self.q.float() * s


def _row_stride(t, name: str) -> int:
    """Elements between the rows of a matrix whose columns are next to each other (a row alone has any stride)."""
    rows, cols = t.shape
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{name} must have consecutive columns")
    if rows <= 1 or cols == 0:  # the stride is not used; torch may have set it to anything
        ld = max(ld, cols)
        if t.element_size() == 1:
            ld = (ld + 15) // 16 * 16
    elif ld < cols:
        raise ValueError(f"rows of {name} overlap")
    return ld


def _on_gpu(t, name: str, device: int = -1) -> int:
    """The tensor's device index: the current GPU, to which calls go, or `device` where an input has named it."""
    d = t.get_device()
    if d < 0:
        raise ValueError(f"{name} must be a CUDA tensor")
    if device < 0:
        device = torch.cuda.current_device()
        if d != device:
            raise ValueError(f"{name} is on cuda:{d}, the current device is cuda:{device} (torch.cuda.set_device)")
    elif d != device:
        raise ValueError(f"{name} is on cuda:{d}, the input on cuda:{device}")
    return d


def _matrix(t, name: str) -> int:
    """Checks a [rows, cols] tensor of a supported type; returns its row stride."""
    if t.dtype not in _TYPES:
        raise ValueError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    if t.dim() != 2:
        raise ValueError(f"{name} must have two dimensions")
    return _row_stride(t, name)


def _like(t, name: str, rows: int, cols: int, dtype, device: int) -> tuple:
    """Checks a [rows, cols] tensor of one type; returns (address, row stride), (None, 0) for None."""
    if t is None:
        return None, 0
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != (rows, cols):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {(rows, cols)}")
    _on_gpu(t, name, device)
    return t.data_ptr(), _row_stride(t, name)


def _vector(t, name: str, n: int, device: int):
    """Checks a contiguous float32 vector of n values; returns its address (None for None)."""
    if t is None:
        return None
    if t.dtype != torch.float32:
        raise ValueError(f"{name} must be torch.float32, got {t.dtype}")
    if t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous vector of {n} values, got shape {tuple(t.shape)}")
    _on_gpu(t, name, device)
    return t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _on_stream(device: int):
    """The current stream of the tensors' device (by torch's short way where it has one)."""
    return _raw_stream(device) if _raw_stream is not None else _stream(None)


def _given(stream):
    """Makes the caller's stream (a torch stream, a handle, or what has one as ``cuda_stream``) current: a call's outputs
    and its workspace then belong to it, so none of that memory is still in use, or used again, by the work of another
    stream.  As for anything made on a stream, the caller orders the inputs before the call and the use of the results on
    other streams behind it."""
    if not isinstance(stream, torch.cuda.Stream):
        handle = _stream(stream)
        # 1 is CUDA's other name of the default stream
        stream = torch.cuda.default_stream() if handle in (0, 1) else torch.cuda.ExternalStream(handle)
    return torch.cuda.stream(stream)


def _f8(m, name: str):
    if not isinstance(m, F8Matrix):
        raise ValueError(f"{name} must be an F8Matrix")
    return m.desc


def quantize_f8(x, blocks: str | None = "rows", transposed: str | None = None, pow2: bool = False,
                dtype=torch.float8_e4m3fn, stream=None):
    """Rounds x [rows, cols] (a tensor, or an F8Matrix whose blocks change) to 8 bits with a scale per block of 128.

    ``blocks`` is the kind of blocks of the result ("rows", "tiles", or None for no result) and ``transposed`` that of
    its transpose [cols, rows]; returns (result, transpose), made in one pass over x.  ``pow2`` rounds scales up to
    powers of two.
    """
    if stream is not None:
        with _given(stream):
            return quantize_f8(x, blocks, transposed, pow2, dtype)
    for b in (blocks, transposed):
        if b is not None and b not in _BLOCKS:
            raise ValueError(f"blocks are 'rows', 'tiles' or None, got {b!r}")
    if dtype not in _FORMATS:
        raise ValueError(f"dtype must be torch.float8_e4m3fn or torch.float8_e5m2, got {dtype}")
    if blocks is None and transposed is None:
        raise ValueError("neither the matrix nor its transpose is asked for")
    is_f8 = isinstance(x, F8Matrix)
    if is_f8:
        rows, cols, device = x.desc.rows, x.desc.cols, x._q.device
        _on_gpu(x._q, "x")
    else:
        ld = _matrix(x, "x")
        rows, cols = x.shape
        device = x.device
        _on_gpu(x, "x")
    out = F8Matrix.empty(rows, cols, device, dtype, blocks == "tiles") if blocks else None
    out_t = F8Matrix.empty(cols, rows, device, dtype, transposed == "tiles") if transposed else None
    d, d_t = out.desc if out else None, out_t.desc if out_t else None
    flags = DS_F8_POW2 if pow2 else 0
    stream = _on_stream(device.index)
    if is_f8:
        _check(lib().ds_requantize_f8(x.desc, d, d_t, flags, stream))
    else:
        _check(lib().ds_quantize_f8(x.data_ptr(), _TYPES[x.dtype], rows, cols, ld, d, d_t, flags, stream))
    return out, out_t


def expand_shift_weights_f8(w, stream=None) -> F8Matrix:
    """The weights s * 2^p of a PackedShiftWeights as an e4m3 matrix in tiles (exact: q = s * 2^(p + 8), scales 2^-8)."""
    if stream is not None:
        with _given(stream):
            return expand_shift_weights_f8(w)
    _on_gpu(w.blob, "w")
    m = F8Matrix.empty(w.n_out, w.k_red, w.blob.device, tiles=True)
    ds_expand_shift_weights_f8(w.desc, m.desc)
    return m


def linear_f8(x: F8Matrix, w: F8Matrix, bias=None, add=None, out=None, dtype=torch.bfloat16, stream=None):
    """y = x @ w^T + bias + add for 8-bit x [M, K] and w [N, K]: a tensor [M, N] of ``dtype`` (or ``out``'s).

    ``bias`` is float32 [N], ``add`` float32 [M, N]; ``out`` may be ``add`` itself, which then accumulates."""
    if stream is not None:
        with _given(stream):
            return linear_f8(x, w, bias, add, out, dtype)
    dx, dw = _f8(x, "x"), _f8(w, "w")
    M, N = dx.rows, dw.rows
    device = _on_gpu(x._q, "x")
    _on_gpu(w._q, "w", device)
    y = out
    if y is None:
        if dtype not in _TYPES:
            raise ValueError(f"dtype must be float32, bfloat16 or float16, got {dtype}")
        y = torch.empty((M, N), dtype=dtype, device=x._q.device)
        py, ldy = y.data_ptr(), N
    else:
        if y.dtype not in _TYPES:
            raise ValueError(f"out must be float32, bfloat16 or float16, got {y.dtype}")
        py, ldy = _like(y, "out", M, N, y.dtype, device)
    pa, ld_add = _like(add, "add", M, N, torch.float32, device)
    _check(lib().ds_linear_f8(dx, dw, _vector(bias, "bias", N, device), pa, ld_add, py, _TYPES[y.dtype], ldy,
                              _on_stream(device)))
    return y


def rmsnorm_f8(x, weight, residual=None, eps: float = 1e-5, pow2: bool = False, dtype=torch.float8_e4m3fn, h=None,
               stream=None):
    """Root-mean-square norm of h = x + residual, in 8 bits with a scale per row and 128 columns (weight: 16-byte aligned).

    Returns (n, h, rstd): the F8Matrix of h * rstd * weight, h in x's dtype (x itself without a residual, ``h`` where
    given; it may be x or residual), and the float32 reciprocal root mean squares that the backward pass reads."""
    if stream is not None:
        with _given(stream):
            return rmsnorm_f8(x, weight, residual, eps, pow2, dtype, h)
    ldx = _matrix(x, "x")
    rows, cols = x.shape
    device, kind = _on_gpu(x, "x"), x.dtype
    pw = _vector(weight, "weight", cols, device)
    pr, ldr = _like(residual, "residual", rows, cols, kind, device)
    ph, ldh = _like(h, "h", rows, cols, kind, device)
    if h is None:
        if residual is None:
            h = x
        else:
            h = torch.empty((rows, cols), dtype=kind, device=x.device)
            ph, ldh = h.data_ptr(), cols
    n = F8Matrix.empty(rows, cols, x.device, dtype)
    rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
    _check(lib().ds_rmsnorm_f8(x.data_ptr(), ldx, pr, ldr, pw, _TYPES[kind], rows, cols, eps, n.desc, ph, ldh,
                               rstd.data_ptr(), DS_F8_POW2 if pow2 else 0, _on_stream(device)))
    return n, h, rstd


def rmsnorm_f8_backward(dy, h, rstd, weight, dh=None, out=None, stream=None):
    """Backward pass of rmsnorm_f8: (dx, dweight) from the gradient dy of the norm (the rounding to 8 bits passes it
    unchanged), what the forward pass returned, and the gradient dh that the stream h brings (or None).  dx is the
    gradient of x and of residual alike; ``out`` may be dy, h or dh."""
    if stream is not None:
        with _given(stream):
            return rmsnorm_f8_backward(dy, h, rstd, weight, dh, out)
    lddy = _matrix(dy, "dy")
    rows, cols = dy.shape
    device, kind = _on_gpu(dy, "dy"), dy.dtype
    ph, ldh = _like(h, "h", rows, cols, kind, device)
    pdh, lddh = _like(dh, "dh", rows, cols, kind, device)
    pr, pw = _vector(rstd, "rstd", rows, device), _vector(weight, "weight", cols, device)
    pdx, lddx = _like(out, "out", rows, cols, kind, device)
    dx = out
    if dx is None:
        dx = torch.empty((rows, cols), dtype=kind, device=dy.device)
        pdx, lddx = dx.data_ptr(), cols
    dw = torch.empty(cols, dtype=torch.float32, device=dy.device)
    nbytes = lib().ds_rmsnorm_f8_backward_workspace_bytes(rows, cols)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dy.device)
    _check(lib().ds_rmsnorm_f8_backward(dy.data_ptr(), lddy, ph, ldh, pr, pw, pdh, lddh, _TYPES[kind], rows, cols, pdx,
                                        lddx, dw.data_ptr(), ws.data_ptr(), nbytes, _on_stream(device)))
    return dx, dw


def _gate_width(features: int) -> int:
    """Columns of a gate's input: the up half starts at the next multiple of 128."""
    return (features + BLOCK - 1) // BLOCK * BLOCK + features


def gated_f8(gu, features: int, checkpoint: bool = True, pow2: bool = False, dtype=torch.float8_e4m3fn, stream=None):
    """a = silu(g) * u in 8 bits, for gu [rows, up + features] with g in columns [0, features) and u from column
    up = features rounded up to a multiple of 128.  Returns (a, kept): kept is the 8-bit checkpoint of gu that
    gated_f8_backward reads (None without ``checkpoint``)."""
    if stream is not None:
        with _given(stream):
            return gated_f8(gu, features, checkpoint, pow2, dtype)
    ld = _matrix(gu, "gu")
    rows, width = gu.shape
    if features <= 0 or width != _gate_width(features):
        raise ValueError(f"gu has {width} columns, expected {_gate_width(features)} for {features} features")
    device = _on_gpu(gu, "gu")
    a = F8Matrix.empty(rows, features, gu.device, dtype)
    kept = F8Matrix.empty(rows, width, gu.device, dtype) if checkpoint else None
    _check(lib().ds_gated_f8(gu.data_ptr(), _TYPES[gu.dtype], ld, rows, features, a.desc,
                             kept.desc if kept else None, DS_F8_POW2 if pow2 else 0, _on_stream(device)))
    return a, kept


def gated_f8_backward(kept: F8Matrix, da, pow2: bool = False, dtype=torch.float8_e4m3fn, transposed: bool = True,
                      stream=None):
    """Backward pass of gated_f8 from its checkpoint and the gradient da [rows, features] of a.  Returns
    (dgu, dgu_t, a_t) in 8 bits: the gradient of gu, its transpose, and the transpose of a made again from the
    checkpoint (the operands of the two weight gradients; None without ``transposed``)."""
    if stream is not None:
        with _given(stream):
            return gated_f8_backward(kept, da, pow2, dtype, transposed)
    dk = _f8(kept, "kept")
    ld = _matrix(da, "da")
    rows, features = da.shape
    if features == 0 or dk.rows != rows or dk.cols != _gate_width(features):
        raise ValueError(f"kept is {dk.rows} x {dk.cols}, expected {rows} x {_gate_width(features)}")
    device = _on_gpu(da, "da", _on_gpu(kept._q, "kept"))
    dgu = F8Matrix.empty(rows, dk.cols, da.device, dtype)
    dgu_t = F8Matrix.empty(dk.cols, rows, da.device, dtype) if transposed else None
    a_t = F8Matrix.empty(features, rows, da.device, dtype) if transposed else None
    _check(lib().ds_gated_f8_backward(dk, da.data_ptr(), _TYPES[da.dtype], ld, features, dgu.desc,
                                      dgu_t.desc if dgu_t else None, a_t.desc if a_t else None,
                                      DS_F8_POW2 if pow2 else 0, _on_stream(device)))
    return dgu, dgu_t, a_t

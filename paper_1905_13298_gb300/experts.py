"""Tensor-level helpers of a feed-forward block with experts (see the header's section on them): tokens in order of
their expert and back, the experts' products with 8-bit operands, and their gradients.

Calls run on the current stream, or on ``stream`` (a torch stream or a handle), to which what they return then belongs.
Nothing waits for the host: sizes follow from the number of tokens alone, whatever experts they choose.

A training step of such a block reads::

    order = expert_order(ids, experts, align=128)              # ids, weights: [tokens, top_k] of the router
    xs = expert_gather(n, order)                               # n: 8-bit rows of the norm, scales powers of two
    gu = expert_linear_f8(xs, w_gu, order)                     # w_gu: [experts * rows, hidden] in tiles
    a, kept = gated_f8(gu, features)
    y = expert_linear_f8(a, w_down, order)
    out = expert_combine(y, order, weights, add=h)
    ...
    dy, dweights = expert_combine_backward(dout, y, order, weights)
    d, d_t = quantize_f8(dy, "rows", "rows")
    dgu, dgu_t, a_t = gated_f8_backward(kept, expert_linear_f8(d, w_down_t, order))
    grad_down = expert_weight_grad_f8(d_t, a_t, order, add=grad_down, out=grad_down)
    xs_t = quantize_f8(xs, None, "tiles", pow2=True)[1]        # xs's values, turned, not rounded again
    grad_gu = expert_weight_grad_f8(dgu_t, xs_t, order, add=grad_gu, out=grad_gu)
    dn = expert_combine(expert_linear_f8(dgu, w_gu_t, order), order)    # the gradient of expert_gather
"""
from __future__ import annotations

from operator import attrgetter

import torch

from . import DS_INDEX_I32, DS_INDEX_I64, DsError, DS_ERR_UNSUPPORTED, _check, ds_expert_slots, lib
from .float8 import _TYPES, F8Matrix, _f8, _given, _like, _matrix, _on_gpu, _on_stream

_INDEX = {torch.int32: DS_INDEX_I32, torch.int64: DS_INDEX_I64}


def _ints(t, name: str, shape: tuple, device: int) -> int:
    """Checks a contiguous int32 tensor; returns its address."""
    if t.dtype != torch.int32:
        raise ValueError(f"{name} must be torch.int32, got {t.dtype}")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous of shape {shape}, got {tuple(t.shape)}")
    if t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, the offsets on cuda:{device}")
    return t.data_ptr()


class ExpertOrder:
    """Which rows the slots (token, choice) of a block with experts have, as ``expert_order`` makes it: int32 tensors
    ``offsets`` [experts + 1] of the experts' segments, ``counts`` [experts], ``position`` [tokens, top_k], the row of
    a slot or -1, and ``slot`` [rows], the slot (token * top_k + choice) of a row or -1.  Segments start at multiples
    of ``align``.  The tensors stay those that it was made with: calls read their memory."""

    __slots__ = ("_offsets", "_counts", "_position", "_slot", "device", "desc")
    offsets, counts, position, slot = (property(attrgetter(name)) for name in __slots__[:4])

    def __init__(self, offsets, counts, position, slot, align: int = 1):
        if offsets.dim() != 1 or offsets.shape[0] < 2:
            raise ValueError("offsets must be a vector of at least 2 values")
        if position.dim() != 2 or slot.dim() != 1:
            raise ValueError("position must have two dimensions, slot one")
        device = offsets.get_device()
        if device < 0:
            raise ValueError("offsets must be a CUDA tensor")
        experts, (tokens, top_k), rows = offsets.shape[0] - 1, position.shape, slot.shape[0]
        self._offsets, self._counts, self._position, self._slot, self.device = offsets, counts, position, slot, device
        self.desc = ds_expert_slots(_ints(offsets, "offsets", (experts + 1,), device),
                                    _ints(counts, "counts", (experts,), device),
                                    _ints(position, "position", (tokens, top_k), device),
                                    _ints(slot, "slot", (rows,), device), tokens, rows, top_k, experts, align, 0)

    @property
    def tokens(self) -> int:
        return self.desc.tokens

    @property
    def top_k(self) -> int:
        return self.desc.top_k

    @property
    def experts(self) -> int:
        return self.desc.experts

    @property
    def align(self) -> int:
        return self.desc.align

    @property
    def rows(self) -> int:
        return self.desc.rows


def _order(order, device: int):
    """The order's descriptor; its tensors are on the input's device."""
    if not isinstance(order, ExpertOrder):
        raise ValueError("order must be an ExpertOrder")
    if order.device != device:
        raise ValueError(f"order is on cuda:{order.device}, the input on cuda:{device}")
    return order.desc


def _weights(w, desc, device: int, name: str = "weights"):
    """Checks contiguous float32 [tokens, top_k]; returns the address (None for None)."""
    if w is None:
        return None
    if w.dtype != torch.float32:
        raise ValueError(f"{name} must be torch.float32, got {w.dtype}")
    if w.shape != (desc.tokens, desc.top_k) or not w.is_contiguous():
        raise ValueError(f"{name} must be contiguous of shape {(desc.tokens, desc.top_k)}, got {tuple(w.shape)}")
    _on_gpu(w, name, device)
    return w.data_ptr()


def expert_order(ids, experts: int, align: int = 1, stream=None) -> ExpertOrder:
    """The order of the slots of ids [tokens, top_k] (int32 or int64) by expert; ids outside [0, experts) go nowhere.

    Segments of rows start at multiples of ``align``: 128 for training, so that the blocks of the 8-bit matrices' and of
    their transposes hold one expert's rows; 1 leaves no gaps."""
    if stream is not None:
        with _given(stream):
            return expert_order(ids, experts, align)
    if ids.dtype not in _INDEX:
        raise ValueError(f"ids must be torch.int32 or torch.int64, got {ids.dtype}")
    if ids.dim() != 2 or not ids.is_contiguous():
        raise ValueError(f"ids must be contiguous [tokens, top_k], got shape {tuple(ids.shape)}")
    device, (tokens, top_k) = _on_gpu(ids, "ids"), ids.shape
    if top_k < 1 or experts < 1 or align < 1:
        raise ValueError("top_k, experts and align must be at least 1")
    rows = lib().ds_expert_rows(tokens, top_k, experts, align)
    if rows < 0:
        raise DsError(DS_ERR_UNSUPPORTED, "too many experts, tokens or rows, or align too large")
    order, kind, where = ExpertOrder.__new__(ExpertOrder), torch.int32, ids.device
    # four allocations cost the host less than four views of one
    offsets = order._offsets = torch.empty(experts + 1, dtype=kind, device=where)
    counts = order._counts = torch.empty(experts, dtype=kind, device=where)
    position = order._position = torch.empty((tokens, top_k), dtype=kind, device=where)
    slot = order._slot = torch.empty(rows, dtype=kind, device=where)
    order.device = device
    order.desc = ds_expert_slots(offsets.data_ptr(), counts.data_ptr(), position.data_ptr(), slot.data_ptr(), tokens,
                                 rows, top_k, experts, align, 0)
    _check(lib().ds_expert_order(ids.data_ptr(), _INDEX[ids.dtype], order.desc, _on_stream(device)))
    return order


def expert_gather(x, order: ExpertOrder, out=None, stream=None):
    """The rows of x [tokens, cols] (a tensor, or an F8Matrix with blocks by rows) in the order of their slots:
    [order.rows, cols], zeros in rows without a slot."""
    if stream is not None:
        with _given(stream):
            return expert_gather(x, order, out)
    if isinstance(x, F8Matrix):
        device = _on_gpu(x._q, "x")
        desc, dx = _order(order, device), x.desc
        if x.tiles or (out is not None and _f8(out, "out").blocks != dx.blocks):
            raise ValueError("x and out must have blocks by rows: rows of tiles cannot be moved")
        if dx.rows != desc.tokens:
            raise ValueError(f"x has {dx.rows} rows, the order {desc.tokens} tokens")
        if out is None:
            out = F8Matrix.empty(desc.rows, dx.cols, x._q.device, x._q.dtype)
        else:
            _on_gpu(out._q, "out", device)
        _check(lib().ds_expert_gather_f8(dx, desc, out.desc, _on_stream(device)))
        return out
    ldx = _matrix(x, "x")
    device, cols = _on_gpu(x, "x"), x.shape[1]
    desc = _order(order, device)
    if x.shape[0] != desc.tokens:
        raise ValueError(f"x has {x.shape[0]} rows, the order {desc.tokens} tokens")
    if isinstance(out, F8Matrix):
        raise ValueError("out is an F8Matrix, x is not")
    if out is None:
        out = torch.empty((desc.rows, cols), dtype=x.dtype, device=x.device)
        po, ldo = out.data_ptr(), cols
    else:
        po, ldo = _like(out, "out", desc.rows, cols, x.dtype, device)
    _check(lib().ds_expert_gather(x.data_ptr(), _TYPES[x.dtype], ldx, cols, desc, po, ldo, _on_stream(device)))
    return out


def expert_combine(y, order: ExpertOrder, weights=None, add=None, out=None, stream=None):
    """[tokens, cols]: add + the sum over a token's slots of weight times row of y [order.rows, cols].

    ``weights`` is float32 [tokens, top_k]; without them the sum is the gradient of ``expert_gather``.  ``add`` has y's
    dtype, and ``out`` may be it."""
    if stream is not None:
        with _given(stream):
            return expert_combine(y, order, weights, add, out)
    ldy = _matrix(y, "y")
    device, cols, kind = _on_gpu(y, "y"), y.shape[1], y.dtype
    desc = _order(order, device)
    if y.shape[0] != desc.rows:
        raise ValueError(f"y has {y.shape[0]} rows, the order {desc.rows}")
    pw = _weights(weights, desc, device)
    pa, ld_add = _like(add, "add", desc.tokens, cols, kind, device)
    if out is None:
        out = torch.empty((desc.tokens, cols), dtype=kind, device=y.device)
        po, ldo = out.data_ptr(), cols
    else:
        po, ldo = _like(out, "out", desc.tokens, cols, kind, device)
    _check(lib().ds_expert_combine(y.data_ptr(), _TYPES[kind], ldy, cols, desc, pw, pa, ld_add, po, ldo,
                                   _on_stream(device)))
    return out


def expert_combine_backward(dout, y, order: ExpertOrder, weights=None, out=None, stream=None):
    """Backward pass of expert_combine from the gradient dout [tokens, cols] of its result: (dy, dweights).  dy is that
    of y, [order.rows, cols], zeros in rows without a slot; ``out`` may be y itself.  The gradient of ``add`` is dout.
    Without ``weights`` (all 1) dweights is None and y is not read."""
    if stream is not None:
        with _given(stream):
            return expert_combine_backward(dout, y, order, weights, out)
    ldd = _matrix(dout, "dout")
    device, cols, kind = _on_gpu(dout, "dout"), dout.shape[1], dout.dtype
    desc = _order(order, device)
    if dout.shape[0] != desc.tokens:
        raise ValueError(f"dout has {dout.shape[0]} rows, the order {desc.tokens} tokens")
    if cols == 0:
        raise ValueError("a gradient needs columns")
    pw = _weights(weights, desc, device)
    py, ldy = _like(y if weights is not None else None, "y", desc.rows, cols, kind, device)
    if weights is not None and y is None:
        raise ValueError("y is needed for the gradient of the weights")
    dy = out
    if dy is None:
        dy = torch.empty((desc.rows, cols), dtype=kind, device=dout.device)
        pdy, lddy = dy.data_ptr(), cols
    else:
        pdy, lddy = _like(dy, "out", desc.rows, cols, kind, device)
    dw = torch.empty((desc.tokens, desc.top_k), dtype=torch.float32, device=dout.device) if weights is not None else None
    _check(lib().ds_expert_combine_backward(dout.data_ptr(), ldd, py, ldy, _TYPES[kind], cols, desc, pw, pdy, lddy,
                                            dw.data_ptr() if dw is not None else None, _on_stream(device)))
    return dy, dw


def expert_linear_f8(x: F8Matrix, w: F8Matrix, order: ExpertOrder, bias=None, out=None, dtype=torch.bfloat16,
                     stream=None):
    """[order.rows, N]: row r of an expert e's segment is x[r] @ w_e^T + bias[e], for 8-bit x [order.rows, K] and w
    [experts * N, K], w_e being rows e N to (e + 1) N; zeros behind the last segment.  ``bias`` is float32 [experts, N].
    A w in tiles needs an N that is a multiple of 128."""
    if stream is not None:
        with _given(stream):
            return expert_linear_f8(x, w, order, bias, out, dtype)
    dx, dw = _f8(x, "x"), _f8(w, "w")
    device = _on_gpu(x._q, "x")
    _on_gpu(w._q, "w", device)
    desc = _order(order, device)
    n = dw.rows // desc.experts
    y = out
    if y is None:
        if dtype not in _TYPES:
            raise ValueError(f"dtype must be float32, bfloat16 or float16, got {dtype}")
        y = torch.empty((desc.rows, n), dtype=dtype, device=x._q.device)
        py, ldy = y.data_ptr(), n
    else:
        if y.dtype not in _TYPES:
            raise ValueError(f"out must be float32, bfloat16 or float16, got {y.dtype}")
        py, ldy = _like(y, "out", desc.rows, n, y.dtype, device)
    pb = None
    if bias is not None:
        if bias.dtype != torch.float32 or bias.shape != (desc.experts, n) or not bias.is_contiguous():
            raise ValueError(f"bias must be contiguous float32 of shape {(desc.experts, n)}")
        _on_gpu(bias, "bias", device)
        pb = bias.data_ptr()
    _check(lib().ds_expert_linear_f8(dx, dw, desc, pb, py, _TYPES[y.dtype], ldy, _on_stream(device)))
    return y


def expert_weight_grad_f8(dy_t: F8Matrix, x_t: F8Matrix, order: ExpertOrder, add=None, out=None, stream=None):
    """The experts' weight gradients, float32 [experts, N, K]: add[e] + dy_t[:, segment e] @ x_t[:, segment e]^T for
    8-bit dy_t [N, order.rows] and x_t [K, order.rows] (the products' gradient and input, transposed).  The order's
    align is a multiple of 128; ``out`` may be ``add`` itself, which then accumulates."""
    if stream is not None:
        with _given(stream):
            return expert_weight_grad_f8(dy_t, x_t, order, add, out)
    dd, dx = _f8(dy_t, "dy_t"), _f8(x_t, "x_t")
    device = _on_gpu(dy_t._q, "dy_t")
    _on_gpu(x_t._q, "x_t", device)
    desc = _order(order, device)
    shape = (desc.experts, dd.rows, dx.rows)

    def held(t, name):
        if t is None:
            return None
        if t.dtype != torch.float32 or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous float32 of shape {shape}, got {tuple(t.shape)}")
        _on_gpu(t, name, device)
        return t.data_ptr()

    pa = held(add, "add")
    dw = torch.empty(shape, dtype=torch.float32, device=dy_t._q.device) if out is None else out
    _check(lib().ds_expert_weight_grad_f8(dd, dx, desc, pa, dx.rows, held(dw, "out"), dx.rows, _on_stream(device)))
    return dw

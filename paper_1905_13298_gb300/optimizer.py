"""AdamW over many tensors at once, with states of 32 or 8 bits (see the header's section on the optimizer).

    optimizer = AdamW(params, grads, lr=1e-3, state_dtype=torch.float8_e4m3fn, copies=[p.bfloat16() for p in params])
    ...                     # a backward pass that writes or accumulates into grads
    optimizer.step()        # one launch for up to 400 tensors
"""
from __future__ import annotations

from numbers import Real

import torch

from . import DsError, _check, ds_adamw_options, ds_adamw_tensor, lib
from .float8 import _TYPES, BLOCK, _given, _on_gpu, _on_stream


def _flat(t, name: str, n: int | None, dtypes, device: int) -> int:
    """Checks contiguous memory of n values; returns its address."""
    if t.dtype not in dtypes:
        raise ValueError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if n is not None and t.numel() != n:
        raise ValueError(f"{name} has {t.numel()} values, expected {n}")
    if t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, the first parameter on cuda:{device}")
    return t.data_ptr()


def _scalar(t, name: str, dtype, device: int) -> int:
    if t.numel() != 1:
        raise ValueError(f"{name} must hold one value, got shape {tuple(t.shape)}")
    return _flat(t, name, 1, (dtype,), device)


def _memory(tensors) -> list:
    """The storages of tensors: while one is held, its memory goes to nobody else, whatever the tensor is given instead."""
    return [t.untyped_storage() for t in tensors if isinstance(t, torch.Tensor)]


class AdamW:
    """Adam with decoupled weight decay on ``params`` (float32, bfloat16 or float16), updated in place from ``grads``
    (tensors of the same sizes, any of these dtypes), which the optimizer keeps and reads at each step.

    ``m`` and ``v`` are the states: float32 tensors of the parameters' sizes, or for 8 bits pairs (values, scales) of
    ``torch.float8_e4m3fn`` values and a float32 scale per 128 of them; v's are those of the second moment's root.
    Without them zeros of ``state_dtype`` are made.  ``copies`` are 16-bit (or float32) tensors that each step writes
    the rounded parameters to.  ``weight_decay`` is one number or one per tensor.  ``steps`` is how many steps were
    done: a number, or a CUDA int64 tensor, which ``step`` then counts up on the device; with that, ``lr`` may be a
    CUDA float32 tensor too, and a step can be captured in a CUDA graph.  ``grad_scale``, a CUDA float32 tensor of one
    value, multiplies all gradients.  ``seed`` begins the random bits that 8-bit states are rounded by.

    A step works on the memory that parameters, states and copies had when the optimizer was made, and holds it.  Where a
    parameter, gradient or copy has been given other memory since, it is refused.  States are loaded by copying into them
    (``opt.m[k].copy_(...)``): entries of ``m`` and ``v`` that are replaced or given other memory are passed over."""

    def __init__(self, params, grads, m=None, v=None, copies=None, lr=1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay=0.01, grad_scale=None, steps=0, seed: int = 0, state_dtype=torch.float32):
        self.params, self.grads = list(params), list(grads)
        count = len(self.params)
        if count == 0:
            raise ValueError("no parameters")
        device = self._device = _on_gpu(self.params[0], "params[0]")
        where = self.params[0].device
        if state_dtype not in (torch.float32, torch.float8_e4m3fn):
            raise ValueError(f"state_dtype must be torch.float32 or torch.float8_e4m3fn, got {state_dtype}")

        def zeros(n):
            if state_dtype == torch.float32:
                return torch.zeros(n, device=where)
            return (torch.zeros(n, dtype=torch.uint8, device=where).view(state_dtype),
                    torch.zeros((n + BLOCK - 1) // BLOCK, device=where))

        self.m = [zeros(p.numel()) for p in self.params] if m is None else list(m)
        self.v = [zeros(p.numel()) for p in self.params] if v is None else list(v)
        self.copies = None if copies is None else list(copies)
        decay = [weight_decay] * count if isinstance(weight_decay, Real) else list(weight_decay)
        for name, x in (("grads", self.grads), ("m", self.m), ("v", self.v), ("weight_decay", decay),
                        ("copies", self.copies)):
            if x is not None and len(x) != count:
                raise ValueError(f"{name} has {len(x)} entries, expected {count}")
        self._tensors = (ds_adamw_tensor * count)()
        for k, p in enumerate(self.params):
            d, n = self._tensors[k], p.numel()
            d.p, d.p_type, d.n = _flat(p, f"params[{k}]", n, _TYPES, device), _TYPES[p.dtype], n
            d.weight_decay = decay[k]
            for name, state in (("m", self.m[k]), ("v", self.v[k])):
                if isinstance(state, (tuple, list)):
                    q, scale = state
                    setattr(d, name, _flat(q, f"{name}[{k}]", n, (torch.float8_e4m3fn,), device))
                    setattr(d, name + "_scale",
                            _flat(scale, f"{name}[{k}]'s scales", (n + BLOCK - 1) // BLOCK, (torch.float32,), device))
                else:
                    setattr(d, name, _flat(state, f"{name}[{k}]", n, (torch.float32,), device))
            if self.copies is not None and self.copies[k] is not None:
                c = self.copies[k]
                d.copy, d.copy_type = _flat(c, f"copies[{k}]", n, _TYPES, device), _TYPES[c.dtype]
        self._kept = self.params + [c for c in self.copies or [] if c is not None]
        self._kept_at = list(map(torch.Tensor.data_ptr, self._kept))
        states = [t for state in (*self.m, *self.v) for t in (state if isinstance(state, (tuple, list)) else (state,))]
        self._kept_memory = _memory(self._kept + states)
        self._take(self.grads)
        self.lr, self.betas, self.eps, self.grad_scale, self.steps, self.seed = lr, betas, eps, grad_scale, steps, seed

    def _take(self, grads) -> None:
        """Notes gradients, and where all lies that a step looks at: it refuses what was given other memory since."""
        got = [(_flat(g, f"grads[{k}]", self._tensors[k].n, _TYPES, self._device), _TYPES[g.dtype])
               for k, g in enumerate(grads)]
        for d, (at, kind) in zip(self._tensors, got):
            d.g, d.g_type = at, kind
        self._all, self._held = self._kept + grads, self._kept_at + [at for at, _ in got]
        self._grad_memory = _memory(grads)

    def step(self, grads=None, stream=None) -> None:
        """One step; ``grads`` replace those of the steps before."""
        if stream is not None:
            with _given(stream):
                return self.step(grads)
        device = _on_gpu(self.params[0], "params[0]")
        if grads is not None:
            grads = list(grads)
            if len(grads) != len(self.params):
                raise ValueError(f"grads has {len(grads)} entries, expected {len(self.params)}")
        look, held = (self._all, self._held) if grads is None else (self._kept, self._kept_at)
        if list(map(torch.Tensor.data_ptr, look)) != held:
            raise ValueError("a parameter, gradient or copy has other memory than when it was given")
        if grads is not None:
            self._take(grads)
            self.grads = grads
        o = ds_adamw_options(0.0, self.betas[0], self.betas[1], self.eps, 0, None, None, None, self.seed & 0xFFFFFFFF, 0)
        if isinstance(self.lr, torch.Tensor):
            o.lr_dev = _scalar(self.lr, "lr", torch.float32, device)
        else:
            o.lr = self.lr
        if self.grad_scale is not None:
            o.grad_scale = _scalar(self.grad_scale, "grad_scale", torch.float32, device)
        if isinstance(self.steps, torch.Tensor):
            o.step_dev = _scalar(self.steps, "steps", torch.int64, device)
        else:
            if torch.cuda.is_current_stream_capturing():
                raise ValueError("a captured step needs steps as a CUDA tensor: a replay would repeat this step's number")
            o.step = self.steps + 1
        self.steps += 1  # a tensor counts up on the device, before the step reads it
        try:
            _check(lib().ds_adamw(self._tensors, len(self.params), o, _on_stream(device)))
        except DsError:
            self.steps -= 1
            raise

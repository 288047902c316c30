"""A gated feed-forward block in 8 bits: the operators of ``float8`` as a training step and a serving step run them.

    h = stream + x                         n = rmsnorm(h) * w_norm              (n in 8 bits)
    g, u = n W_gu^T                        a = silu(g) u                        (a in 8 bits, g and u kept in 8 bits)
    y = a W_down^T                         the next block's x; h is its stream

Weights are held twice in 8-bit tiles, as they are and transposed, and made again from their float32 masters after a
step.  ``ExpertsFeedForward`` is the block with experts: of g, u and y each token takes the parts that a router chooses.
Run it (one GPU) to train a block on a synthetic target and to time a step and a token::

    python -m paper_1905_13298_gb300.feed_forward --tokens 4096 --hidden 2048 --features 4096 --steps 20
    python -m paper_1905_13298_gb300.feed_forward --shift      # serve with weights rounded to powers of two (exact in 8 bits)
    python -m paper_1905_13298_gb300.feed_forward --experts 16 --top-k 2 --features 1024 --adamw 8   # states in 8 bits
"""
from __future__ import annotations

import argparse
from numbers import Real

import torch

from . import pack_shift_weights, quantize_shift_weights
from .experts import (expert_combine, expert_combine_backward, expert_gather, expert_linear_f8, expert_order,
                      expert_weight_grad_f8)
from .optimizer import AdamW
from .float8 import (_gate_width, expand_shift_weights_f8, gated_f8, gated_f8_backward, linear_f8, quantize_f8, rmsnorm_f8,
                     rmsnorm_f8_backward)


class GatedFeedForward:
    """One block; ``forward`` and ``backward`` make a training step, ``token`` the serving form without a checkpoint."""

    def __init__(self, hidden: int, features: int, device="cuda", seed: int = 0):
        r = torch.Generator(device=device).manual_seed(seed)
        self.hidden, self.features = hidden, features
        self.norm = torch.ones(hidden, device=device)
        # gate rows, rows up to the next multiple of 128 that stay zero, up rows
        self.gate_up = torch.randn((_gate_width(features), hidden), generator=r, device=device) * hidden**-0.5
        self.gate_up[features : self.up_at] = 0
        self.down = torch.randn((hidden, features), generator=r, device=device) * features**-0.5
        self.refresh()

    @property
    def up_at(self) -> int:
        return _gate_width(self.features) - self.features

    def refresh(self) -> None:
        """The 8-bit weights, and their transposes for the input gradients, from the float32 masters."""
        self.w_gate_up, self.w_gate_up_t = quantize_f8(self.gate_up, "tiles", "tiles")
        self.w_down, self.w_down_t = quantize_f8(self.down, "tiles", "tiles")

    def use_shift_weights(self) -> None:
        """Takes the weights s * 2^p of the power-of-two quantizer (Eq. 4-6; magnitudes above 1 become 1), which are exact
        as 8-bit tiles, and so are their transposes: gradients are those of the shift weights (passed on to the masters,
        as the paper's straight-through estimate does).  ``refresh`` and ``step`` go back to rounded float weights."""
        self.w_gate_up = expand_shift_weights_f8(pack_shift_weights(*quantize_shift_weights(self.gate_up)))
        self.w_down = expand_shift_weights_f8(pack_shift_weights(*quantize_shift_weights(self.down)))
        self.w_gate_up_t = quantize_f8(self.w_gate_up, None, "tiles", pow2=True)[1]
        self.w_down_t = quantize_f8(self.w_down, None, "tiles", pow2=True)[1]

    def forward(self, x, stream):
        """(y, h, saved) for x and the residual stream, both [tokens, hidden]."""
        n, h, rstd = rmsnorm_f8(x, self.norm, residual=stream, pow2=True)
        a, kept = gated_f8(linear_f8(n, self.w_gate_up, dtype=x.dtype), self.features)
        return linear_f8(a, self.w_down, dtype=x.dtype), h, (n, h, rstd, kept)

    def backward(self, dy, dh, saved, grads=None):
        """(dx, grads) from the gradients of y and h; dx is that of x and of the stream alike.  ``grads`` holds the
        float32 sums of the weights' gradients so far and is added to in place."""
        n, h, rstd, kept = saved
        d, d_t = quantize_f8(dy, "rows", "rows")
        dgu, dgu_t, a_t = gated_f8_backward(kept, linear_f8(d, self.w_down_t, dtype=dy.dtype))
        # a right operand in tiles takes the faster product; with scales that are powers of two the values stay as they are
        _, n_t = quantize_f8(n, None, "tiles", pow2=True)
        g = grads or {}
        down = linear_f8(d_t, a_t, add=g.get("down"), out=g.get("down"), dtype=torch.float32)
        gate_up = linear_f8(dgu_t, n_t, add=g.get("gate_up"), out=g.get("gate_up"), dtype=torch.float32)
        dx, norm = rmsnorm_f8_backward(linear_f8(dgu, self.w_gate_up_t, dtype=dy.dtype), h, rstd, self.norm, dh=dh)
        if grads:
            norm = g["norm"].add_(norm)
        return dx, {"norm": norm, "gate_up": gate_up, "down": down}

    def token(self, x, stream):
        """(y, h) for a few tokens while serving."""
        n, h, _ = rmsnorm_f8(x, self.norm, residual=stream, pow2=True)
        a, _ = gated_f8(linear_f8(n, self.w_gate_up, dtype=x.dtype), self.features, checkpoint=False)
        return linear_f8(a, self.w_down, dtype=x.dtype), h

    def step(self, grads, rate: float) -> None:
        """Plain gradient descent on the masters."""
        self.norm.sub_(grads["norm"], alpha=rate)
        self.gate_up.sub_(grads["gate_up"], alpha=rate)
        self.gate_up[self.features : self.up_at] = 0
        self.down.sub_(grads["down"], alpha=rate)
        self.refresh()

    def masters(self) -> dict:
        """The float32 weights by the names of their gradients."""
        return {"norm": self.norm, "gate_up": self.gate_up, "down": self.down}

    def adamw(self, grads, **options) -> AdamW:
        """An optimizer of the masters, for ``step_by``; no decay of the norm's weight unless options say otherwise."""
        names, decay = list(self.masters()), options.pop("weight_decay", 0.01)
        each = [0.0 if k == "norm" else decay for k in names] if isinstance(decay, Real) else list(decay)
        return AdamW(list(self.masters().values()), [grads[k] for k in names], weight_decay=each, **options)

    def step_by(self, optimizer: AdamW, grads) -> None:
        """A step of the optimizer.  Rows of zeros between gate and up rows have no gradient and stay as they are."""
        optimizer.step([grads[k] for k in self.masters()])
        self.refresh()


class ExpertsFeedForward(GatedFeedForward):
    """A block with experts: each token takes ``top_k`` of them, weighted by the softmax of their logits n W_router^T.

        y[t] = sum_j weights[t, j] a_e W_down,e^T     with g, u = n[t] W_gu,e^T, a_e = silu(g) u, e = ids[t, j]

    Tokens are put in order of their expert, and the experts' products run over the segments; nothing waits for the host.
    hidden and features have to be multiples of 128: the experts' weights are held in tiles."""

    def __init__(self, hidden: int, features: int, experts: int, top_k: int, device="cuda", seed: int = 0):
        if hidden % 128 or features % 128:
            raise ValueError("hidden and features must be multiples of 128: the experts' weights are held in tiles")
        if not 1 <= top_k <= experts:
            raise ValueError("top_k must be between 1 and the number of experts")
        r = torch.Generator(device=device).manual_seed(seed)
        self.hidden, self.features, self.experts, self.top_k = hidden, features, experts, top_k
        self.norm = torch.ones(hidden, device=device)
        self.router = torch.randn((experts, hidden), generator=r, device=device) * hidden**-0.5
        self.gate_up = torch.randn((experts, 2 * features, hidden), generator=r, device=device) * hidden**-0.5
        self.down = torch.randn((experts, hidden, features), generator=r, device=device) * features**-0.5
        self.refresh()

    def refresh(self) -> None:
        def both(w):  # [experts, N, K] and [experts, K, N], a matrix in tiles each
            return (quantize_f8(w.flatten(0, 1), "tiles")[0],
                    quantize_f8(w.transpose(1, 2).reshape(-1, w.shape[1]), "tiles")[0])

        self.w_router, self.w_router_t = quantize_f8(self.router, "tiles", "tiles")
        self.w_gate_up, self.w_gate_up_t = both(self.gate_up)
        self.w_down, self.w_down_t = both(self.down)

    def use_shift_weights(self) -> None:
        """As for the block without experts: the experts' weights, and their transposes, are exact; the router keeps its own."""
        def both(w):
            m = expand_shift_weights_f8(pack_shift_weights(*quantize_shift_weights(w.flatten(0, 1))))
            turned = m.dequantize().view(w.shape).transpose(1, 2).reshape(-1, w.shape[1])
            return m, quantize_f8(turned, "tiles", pow2=True)[0]

        self.w_gate_up, self.w_gate_up_t = both(self.gate_up)
        self.w_down, self.w_down_t = both(self.down)

    def route(self, n, padding=None):
        """(ids, weights) [tokens, top_k] of the norm's 8-bit rows; tokens of ``padding`` (truth values) go nowhere.
        Their rows have to be finite all the same: the gradients of the norm's weight and of the router multiply them by 0."""
        best, ids = linear_f8(n, self.w_router, dtype=torch.float32).topk(self.top_k, 1)
        if padding is not None:
            ids.masked_fill_(padding[:, None], -1)
        return ids, torch.softmax(best, 1)

    def _experts(self, n, ids, weights, align: int, keep: bool, kind):
        order = expert_order(ids, self.experts, align=align)
        xs = expert_gather(n, order)
        a, kept = gated_f8(expert_linear_f8(xs, self.w_gate_up, order, dtype=kind), self.features, checkpoint=keep)
        ys = expert_linear_f8(a, self.w_down, order, dtype=kind)
        return expert_combine(ys, order, weights), (order, xs, kept, ys)

    def forward(self, x, stream, padding=None):
        n, h, rstd = rmsnorm_f8(x, self.norm, residual=stream, pow2=True)
        ids, weights = self.route(n, padding)
        y, saved = self._experts(n, ids, weights, 128, True, x.dtype)
        return y, h, (n, h, rstd, ids, weights, *saved)

    def backward(self, dy, dh, saved, grads=None):
        n, h, rstd, ids, weights, order, xs, kept, ys = saved
        g, kind = grads or {}, dy.dtype
        dys, dweights = expert_combine_backward(dy, ys, order, weights)
        d, d_t = quantize_f8(dys, "rows", "rows")
        dgu, dgu_t, a_t = gated_f8_backward(kept, expert_linear_f8(d, self.w_down_t, order, dtype=kind))
        down = expert_weight_grad_f8(d_t, a_t, order, add=g.get("down"), out=g.get("down"))
        _, xs_t = quantize_f8(xs, None, "tiles", pow2=True)  # the values of the forward pass, turned
        gate_up = expert_weight_grad_f8(dgu_t, xs_t, order, add=g.get("gate_up"), out=g.get("gate_up"))
        # of the softmax over a token's choices, at their logits (padding has no gradient)
        dbest = weights * (dweights - (weights * dweights).sum(1, keepdim=True))
        dlogits = torch.zeros((ids.shape[0], self.experts), device=ids.device)
        dlogits.scatter_add_(1, ids.clamp(min=0), dbest.masked_fill(ids < 0, 0.0))
        l, l_t = quantize_f8(dlogits, "rows", "rows")
        _, n_t = quantize_f8(n, None, "tiles", pow2=True)
        router = linear_f8(l_t, n_t, add=g.get("router"), out=g.get("router"), dtype=torch.float32)
        dn = expert_combine(expert_linear_f8(dgu, self.w_gate_up_t, order, dtype=kind), order,
                            add=linear_f8(l, self.w_router_t, dtype=kind))
        dx, norm = rmsnorm_f8_backward(dn, h, rstd, self.norm, dh=dh)
        if grads:
            norm = g["norm"].add_(norm)
        return dx, {"norm": norm, "router": router, "gate_up": gate_up, "down": down}

    def token(self, x, stream):
        n, h, _ = rmsnorm_f8(x, self.norm, residual=stream, pow2=True)
        return self._experts(n, *self.route(n), 1, False, x.dtype)[0], h

    def step(self, grads, rate: float) -> None:
        for k, w in self.masters().items():
            w.sub_(grads[k], alpha=rate)
        self.refresh()

    def masters(self) -> dict:
        return {"norm": self.norm, "router": self.router, "gate_up": self.gate_up, "down": self.down}


def _time(f, n: int = 20) -> float:
    """Microseconds of a call among others, by events on the current stream."""
    for _ in range(3):
        f()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(n):
        f()
    end.record()
    end.synchronize()
    return begin.elapsed_time(end) * 1e3 / n


def main(argv=None) -> list[float]:
    """Trains a block towards the outputs of another one; returns the losses."""
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--tokens", type=int, default=4096)
    p.add_argument("--hidden", type=int, default=2048)
    p.add_argument("--features", type=int, default=4096)
    p.add_argument("--steps", type=int, default=20)
    p.add_argument("--rate", type=float, default=0.3)
    p.add_argument("--shift", action="store_true", help="serve with power-of-two weights after training")
    p.add_argument("--experts", type=int, default=0, help="a block with so many experts")
    p.add_argument("--top-k", type=int, default=2, help="experts of a token")
    p.add_argument("--adamw", type=int, choices=(8, 32), help="train by AdamW with states of so many bits (rate: its lr)")
    a = p.parse_args(argv)
    if min(a.tokens, a.hidden, a.features, a.steps) < 1:
        p.error("--tokens, --hidden, --features and --steps must be at least 1")
    if a.experts and a.shift:
        p.error("--shift is of blocks without experts")
    if a.experts and (not 1 <= a.top_k <= a.experts or a.hidden % 128 or a.features % 128):
        p.error("--top-k must be between 1 and --experts, --hidden and --features multiples of 128")
    r = torch.Generator(device="cuda").manual_seed(1)
    shape = (a.tokens, a.hidden)

    def make(seed):
        if a.experts:
            return ExpertsFeedForward(a.hidden, a.features, a.experts, a.top_k, seed=seed)
        return GatedFeedForward(a.hidden, a.features, seed=seed)

    block, teacher, optimizer = make(2), make(3), None
    losses = []
    for _ in range(a.steps):
        x = torch.randn(shape, generator=r, device="cuda").to(torch.bfloat16)
        stream = torch.randn(shape, generator=r, device="cuda").to(torch.bfloat16)
        y, h, saved = block.forward(x, stream)
        off = y.float() - teacher.token(x, stream)[0].float()
        losses.append(float(off.square().mean()))
        dy = (off / off.numel() * 2 * a.hidden).to(torch.bfloat16)
        _, grads = block.backward(dy, torch.zeros_like(dy), saved)
        if a.adamw is None:
            block.step(grads, a.rate)
        else:
            if optimizer is None:
                kind = torch.float32 if a.adamw == 32 else torch.float8_e4m3fn
                optimizer = block.adamw(grads, lr=a.rate, state_dtype=kind)
            block.step_by(optimizer, grads)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} in {a.steps} steps")
    dh = torch.zeros_like(dy)
    print(f"{a.tokens} tokens: forward {_time(lambda: block.forward(x, stream)):.0f} us, "
          f"backward {_time(lambda: block.backward(dy, dh, saved)):.0f} us")
    if a.shift:
        block.use_shift_weights()
    print(f"one token: {_time(lambda: block.token(x[:1], stream[:1])):.0f} us")
    return losses


if __name__ == "__main__":
    main()

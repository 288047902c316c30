"""A gated feed-forward block in 8 bits: the operators of ``float8`` as a training step and a serving step run them.

    h = stream + x                         n = rmsnorm(h) * w_norm              (n in 8 bits)
    g, u = n W_gu^T                        a = silu(g) u                        (a in 8 bits, g and u kept in 8 bits)
    y = a W_down^T                         the next block's x; h is its stream

Weights are held twice in 8-bit tiles, as they are and transposed, and made again from their float32 masters after a
step.  Run it (one GPU) to train a block on a synthetic target and to time a step and a token::

    python -m paper_1905_13298_gb300.feed_forward --tokens 4096 --hidden 2048 --features 4096 --steps 20
    python -m paper_1905_13298_gb300.feed_forward --shift      # serve with weights rounded to powers of two (exact in 8 bits)
"""
from __future__ import annotations

import argparse

import torch

from . import pack_shift_weights, quantize_shift_weights
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
    a = p.parse_args(argv)
    if min(a.tokens, a.hidden, a.features, a.steps) < 1:
        p.error("--tokens, --hidden, --features and --steps must be at least 1")
    r = torch.Generator(device="cuda").manual_seed(1)
    shape = (a.tokens, a.hidden)
    block, teacher = GatedFeedForward(a.hidden, a.features, seed=2), GatedFeedForward(a.hidden, a.features, seed=3)
    losses = []
    for _ in range(a.steps):
        x = torch.randn(shape, generator=r, device="cuda").to(torch.bfloat16)
        stream = torch.randn(shape, generator=r, device="cuda").to(torch.bfloat16)
        y, h, saved = block.forward(x, stream)
        off = y.float() - teacher.token(x, stream)[0].float()
        losses.append(float(off.square().mean()))
        dy = (off / off.numel() * 2 * a.hidden).to(torch.bfloat16)
        _, grads = block.backward(dy, torch.zeros_like(dy), saved)
        block.step(grads, a.rate)
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

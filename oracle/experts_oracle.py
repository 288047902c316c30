"""Numpy oracle of the experts' operators and of the optimizer step, from their definitions."""
import numpy as np


def rows_needed(tokens, top_k, experts, align):
    """The largest number of rows that any choice of experts takes."""
    slots = tokens * top_k
    return (slots + min(experts, slots) * (align - 1)) // align * align


def order(ids, experts, align, rows):
    """(offsets, counts, position, slot) of ids [tokens, top_k], slot after slot."""
    flat = ids.reshape(-1)
    lists = [[] for _ in range(experts)]
    for s, e in enumerate(flat):
        if 0 <= e < experts:
            lists[e].append(s)
    offsets = [0]
    position, slot = np.full(flat.size, -1, np.int32), np.full(rows, -1, np.int32)
    for members in lists:
        for i, s in enumerate(members):
            position[s] = offsets[-1] + i
            slot[offsets[-1] + i] = s
        offsets.append(offsets[-1] + -(-len(members) // align) * align)
    return (np.array(offsets, np.int32), np.array([len(m) for m in lists], np.int32), position.reshape(ids.shape), slot)


def gather(x, slot, top_k):
    out = np.zeros((slot.size,) + x.shape[1:], x.dtype)
    for r, s in enumerate(slot):
        if s >= 0:
            out[r] = x[s // top_k]
    return out


def combine(y, position, weights=None, add=None):
    """(result, sum of its terms' magnitudes) in float64."""
    tokens, top_k = position.shape
    out = np.zeros((tokens, y.shape[1])) if add is None else add.astype(np.float64).copy()
    size = np.abs(out)
    for t in range(tokens):
        for j in range(top_k):
            if position[t, j] >= 0:
                w = 1.0 if weights is None else float(weights[t, j])
                out[t] += w * y[position[t, j]]
                size[t] += np.abs(w * y[position[t, j]])
    return out, size


def combine_backward(dout, y, position, rows, weights=None):
    """(dy, dweights, magnitudes of dweights' terms)"""
    tokens, top_k = position.shape
    dy, dw, size = np.zeros((rows, dout.shape[1])), np.zeros((tokens, top_k)), np.zeros((tokens, top_k))
    for t in range(tokens):
        for j in range(top_k):
            r = position[t, j]
            if r >= 0:
                dy[r] = dout[t] * (1.0 if weights is None else float(weights[t, j]))
                dw[t, j] = dout[t] @ y[r]
                size[t, j] = np.abs(dout[t]) @ np.abs(y[r])
    return dy, dw, size


def linear(x, w, offsets, bias=None):
    """(y, magnitudes) of float64 x [rows, K] and w [experts, N, K]; bias [experts, N]."""
    y = np.zeros((x.shape[0], w.shape[1]))
    size = np.zeros_like(y)
    for e in range(w.shape[0]):
        a, b = offsets[e], offsets[e + 1]
        y[a:b] = x[a:b] @ w[e].T
        size[a:b] = np.abs(x[a:b]) @ np.abs(w[e].T)
        if bias is not None:
            y[a:b] += bias[e]
            size[a:b] += np.abs(bias[e])
    return y, size


def weight_grad(dy_t, x_t, offsets, add=None):
    """(dw, magnitudes) of float64 dy_t [N, rows] and x_t [K, rows]."""
    experts = len(offsets) - 1
    dw = np.zeros((experts, dy_t.shape[0], x_t.shape[0])) if add is None else add.astype(np.float64).copy()
    size = np.abs(dw)
    for e in range(experts):
        a, b = offsets[e], offsets[e + 1]
        dw[e] += dy_t[:, a:b] @ x_t[:, a:b].T
        size[e] += np.abs(dy_t[:, a:b]) @ np.abs(x_t[:, a:b].T)
    return dw, size


# ------------------------------------------------------------------------------------------------- the optimizer


def adamw64(p, g, m, v, t, lr, betas, eps, decay, grad_scale=1.0):
    """(p, m, v) after step t, in float64."""
    g = g * grad_scale
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    new = p * (1 - lr * decay) - m * (lr / (1 - betas[0] ** t)) / (np.sqrt(v) / np.sqrt(1 - betas[1] ** t) + eps)
    return new, m, v


def adamw32(p, g, m, v, t, lr, betas, eps, decay, grad_scale=None):
    """(p, m, v, root of v) after step t in the defined order of float32 operations."""
    f = np.float32
    if grad_scale is not None:
        g = g * f(grad_scale)
    m = m * f(betas[0]) + g * f(1.0 - betas[0])
    v = v * f(betas[1]) + (g * g) * f(1.0 - betas[1])
    root = np.sqrt(v)
    rate, factor = f(lr / (1.0 - betas[0] ** t)), f(1.0 / np.sqrt(1.0 - betas[1] ** t))
    p = p * f(1.0 - lr * float(f(decay))) - (m * rate) / (root * factor + f(eps))
    assert all(a.dtype == np.float32 for a in (p, m, v, root))
    return p, m, v, root


def random_bits(n, t, number, seed):
    """The hash of n indices: (low halves, high halves)."""
    with np.errstate(over="ignore"):
        x = np.arange(n, dtype=np.uint32) * np.uint32(0x9E3779B1)
        x += np.uint32((t * 0xBB67AE85 + number * 0x6A09E667 + seed) & 0xFFFFFFFF)
        x = (x ^ (x >> np.uint32(16))) * np.uint32(0x243F6A89)
        x = (x ^ (x >> np.uint32(15))) * np.uint32(0xB7E15163)
    x ^= x >> np.uint32(16)
    return x & np.uint32(0xFFFF), x >> np.uint32(16)


def state_to_f8(v, bits, positive):
    """(e4m3 values as float32, scales) of a state, rounded by its random bits."""
    f, n = np.float32, v.size
    a = np.zeros(-(-n // 128) * 128, np.float32)
    a[:n] = np.where(np.isfinite(v), np.abs(v), 0)
    top = a.reshape(-1, 128).max(1)
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        scale = np.maximum(top / f(448), f(2.0**-126))
        u = np.abs(v) * np.repeat(np.minimum(f(448) / top, f(2.0**126)), 128)[:n]
    step = np.ldexp(1.0, np.maximum(np.frexp(u)[1] - 1, -6) - 3)
    # the addition that moves u where it is below 2^-6 rounds to float32
    moved = np.where(u < f(2.0**-6), (u + f(2.0**-6)).astype(np.float64) - 2.0**-6, u.astype(np.float64))
    q = np.floor(moved / step + (bits + 0.5) / 65536) * step
    if positive:
        q = np.where(v > 0, np.maximum(q, 2.0**-9), q)
    q = np.where(np.isfinite(v), np.copysign(np.minimum(q, 448.0), v), np.nan)
    return q.astype(np.float32), scale

"""Cases of the 8-bit floating-point operators: what each has to compute, in a plain form and through the library.

The operators are the parts of an 8-bit linear layer and of a gated feed-forward block built from it: the conversion
to 8 bits with a scale per block of 128 values, the product of two such matrices, the root-mean-square norm that
writes its output in 8 bits, and the gated activation that keeps its inputs as an 8-bit checkpoint for its backward
pass.  An 8-bit matrix is float8 values q [rows, cols] and float32 scales: one per row and 128 columns ("rows"), or
one per 128 x 128 block ("tiles").
"""
import math

import torch

own = False

BLOCK = 128
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
FLOAT8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5


def listed():
    return [
        # one token through a square layer while a text is generated: the weights are read once, latency counts
        dict(name="product_token", op="product", m=1, k=4096, n=4096, tiles=True, out="bf16", bias=False, add=False, fmt="e4m3"),
        # a short prompt with a ragged reduction and output width, and a bias
        dict(name="product_ragged", op="product", m=300, k=1000, n=2050, tiles=True, out="bf16", bias=True, add=False, fmt="e4m3"),
        # the forward product of a training step
        dict(name="product_forward", op="product", m=8192, k=4096, n=4096, tiles=True, out="bf16", bias=False, add=False, fmt="e4m3"),
        # a weight gradient over 8192 tokens added to the float32 sum of earlier micro-batches, gradients in e5m2
        dict(name="product_weight_grad", op="product", m=4096, k=8192, n=2048, tiles=False, out="f32", bias=False, add=True, fmt="e5m2"),
        # the gradient that enters a layer's backward pass: by rows for the input's product, by columns for the weight's
        dict(name="quantize_gradient", op="quantize", rows=8192, cols=4096, type="bf16", out="rows", out_t="rows", pow2=False, fmt="e4m3"),
        # an 8-bit activation kept from the forward pass, turned to column blocks for the weight gradient
        dict(name="quantize_reblock", op="quantize", rows=4096, cols=8192, type="f8", out="", out_t="rows", pow2=True, fmt="e4m3"),
        # one decoding step of a few sequences: norm of the residual stream
        dict(name="norm_token", op="norm", rows=4, cols=4096, type="bf16", residual=True),
        # the norm of a training step
        dict(name="norm_forward", op="norm", rows=8192, cols=4096, type="bf16", residual=True),
        # and its backward pass, with the gradient that the residual stream brings
        dict(name="norm_backward", op="norm_backward", rows=8192, cols=4096, type="bf16", residual=True),
        # the gate of a few tokens: no checkpoint is kept while serving
        dict(name="gated_token", op="gated", rows=8, cols=8192, type="bf16", keep=False),
        # the gate of a training step, odd widths, its inputs kept in 8 bits
        dict(name="gated_forward", op="gated", rows=4095, cols=8200, type="bf16", keep=True),
        # its backward pass from the checkpoint
        dict(name="gated_backward", op="gated_backward", rows=8192, cols=8192, type="bf16"),
    ]


def _size(rng, low, high):
    """A size spread over the logarithm of its range: mostly multiples of 64 or 8, every third one as it comes."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    step = rng.choice((1, 8, 64))
    return max(low, n // step * step) if n >= step else n


def draw(rng):
    op = rng.choice(("product", "product", "product", "quantize", "norm", "norm_backward", "gated", "gated_backward"))
    if op == "product":
        m, k, n = _size(rng, 1, 8192), _size(rng, 256, 8192), _size(rng, 256, 8192)
        while m * k * n > 8192 * 4096 * 4096:
            m, k, n = (m + 1) // 2, k, n
        grad = rng.random() < 0.3
        return dict(op=op, m=m, k=k, n=n, tiles=not grad, out="f32" if grad else rng.choice(("bf16", "bf16", "f16")),
                    bias=not grad and rng.random() < 0.3, add=grad, fmt="e5m2" if grad and rng.random() < 0.5 else "e4m3")
    rows, cols = _size(rng, 1, 8192), _size(rng, 256, 4096 if op.startswith("norm") else 8192)
    if op == "quantize":
        while rows * cols > 8192 * 4096:
            rows = (rows + 1) // 2
        out, out_t = rng.choice((("rows", ""), ("rows", "rows"), ("", "rows"), ("tiles", "tiles"), ("tiles", "")))
        return dict(op=op, rows=rows, cols=cols, type=rng.choice(("f32", "bf16", "f16", "f8")), out=out, out_t=out_t,
                    pow2=rng.random() < 0.5, fmt=rng.choice(("e4m3", "e4m3", "e5m2")))
    kind = rng.choice(("bf16", "bf16", "f16", "f32"))
    if kind == "f32":
        rows = (rows + 1) // 2
    if op == "gated":
        return dict(op=op, rows=(rows + 1) // 2, cols=cols, type=kind, keep=rng.random() < 0.7)
    if op == "gated_backward":
        return dict(op=op, rows=rows, cols=cols, type=kind)
    return dict(op=op, rows=rows, cols=cols, type=kind, residual=rng.random() < 0.7)


# ------------------------------------------------------------------------------------------------ the plain form


def _ceil(n, step):
    return -(-n // step) * step


def _pad(v, rows, cols):
    if v.shape == (rows, cols):
        return v
    out = v.new_zeros(rows, cols)
    out[: v.shape[0], : v.shape[1]] = v
    return out


def _scales(v, tiles, pow2, fmt):
    """The scale of each block: its largest finite magnitude over the format's largest value, at least 2^-126."""
    rows, cols = v.shape
    nb = _ceil(cols, BLOCK) // BLOCK
    a = torch.where(torch.isfinite(v), v.abs(), 0.0)
    if tiles:
        mb = _ceil(rows, BLOCK) // BLOCK
        a = _pad(a, mb * BLOCK, nb * BLOCK).view(mb, BLOCK, nb, BLOCK).amax((1, 3))
    else:
        a = _pad(a, rows, nb * BLOCK).view(rows, nb, BLOCK).amax(2)
    s = (a / LARGEST[fmt]).clamp(min=2.0**-126)
    if pow2:  # up to the next power of two
        s = ((s.view(torch.int32) + 0x7FFFFF) & -0x800000).view(torch.float32)
    return s


def _spread(s, rows, cols, tiles):
    s = s.repeat_interleave(BLOCK, 1)[:, :cols]
    return s.repeat_interleave(BLOCK, 0)[:rows] if tiles else s


def _to_f8(v, tiles=False, pow2=False, fmt="e4m3"):
    s = _scales(v, tiles, pow2, fmt)
    u = (v / _spread(s, *v.shape, tiles)).clamp(-LARGEST[fmt], LARGEST[fmt])
    return torch.where(torch.isfinite(v), u, math.nan).to(FLOAT8[fmt]), s


def _from_f8(q, s, tiles):
    return q.float() * _spread(s, *q.shape, tiles)


def _silu_parts(g):
    sig = 1.0 / (1.0 + torch.exp(-g))
    return g * sig, sig * (1.0 + g * (1.0 - sig))


def _halves(rows, cols, gate, up):
    """Gate and up side by side; the up half starts at the next multiple of 128."""
    start = _ceil(cols, BLOCK)
    both = gate.new_zeros(rows, start + cols)
    both[:, :cols] = gate
    both[:, start:] = up
    return both


def _plain(s):
    c = s["case"]
    if c["op"] == "product":
        y = _from_f8(s["qa"], s["sa"], False) @ _from_f8(s["qb"], s["sb"], c["tiles"]).t()
        if c["bias"]:
            y = y + s["bias"]
        if c["add"]:
            y = y + s["add"]
        return y.to(TYPES[c["out"]])
    if c["op"] == "quantize":
        v = _from_f8(s["q"], s["s"], False) if c["type"] == "f8" else s["x"].float()
        got = {}
        if c["out"]:
            got["q"], got["scale"] = _to_f8(v, c["out"] == "tiles", c["pow2"], c["fmt"])
        if c["out_t"]:
            got["q_t"], got["scale_t"] = _to_f8(v.t().contiguous(), c["out_t"] == "tiles", c["pow2"], c["fmt"])
        return got
    if c["op"] == "norm":
        h = s["x"].float()
        if c["residual"]:
            h = h + s["r"].float()
        rstd = torch.rsqrt(h.square().mean(1) + EPS)
        q, scale = _to_f8(h * rstd[:, None] * s["w"])
        return {"q": q, "scale": scale, "h": h.to(TYPES[c["type"]]), "rstd": rstd}
    if c["op"] == "norm_backward":
        dy, h, w, rstd = s["dy"].float(), s["h"].float(), s["w"], s["rstd"][:, None]
        xhat = h * rstd
        g = dy * w
        dx = rstd * (g - xhat * (g * xhat).mean(1, keepdim=True))
        if c["residual"]:
            dx = dx + s["dh"].float()
        return {"dx": dx.to(TYPES[c["type"]]), "dw": (dy * xhat).sum(0)}
    if c["op"] == "gated":
        n, start = c["cols"], _ceil(c["cols"], BLOCK)
        g, u = s["gu"][:, :n].float(), s["gu"][:, start:].float()
        got = {}
        got["q"], got["scale"] = _to_f8(_silu_parts(g)[0] * u)
        if c["keep"]:
            got["kept"], got["kept_scale"] = _to_f8(_halves(*g.shape, g, u))
        return got
    n, start = c["cols"], _ceil(c["cols"], BLOCK)
    both = _from_f8(s["q"], s["s"], False)
    g, u, da = both[:, :n], both[:, start:], s["da"].float()
    act, slope = _silu_parts(g)
    d = _halves(c["rows"], n, da * u * slope, da * act)
    got = {}
    got["q"], got["scale"] = _to_f8(d)
    got["q_t"], got["scale_t"] = _to_f8(d.t().contiguous())
    got["a_t"], got["a_scale_t"] = _to_f8((act * u).t().contiguous())
    return got


# ------------------------------------------------------------------------------------------------ the library's


def _library(s):
    import paper_1905_13298_gb300 as ds

    c = s["case"]
    if c["op"] == "product":
        a = ds.F8Matrix(s["qa"], s["sa"])
        b = ds.F8Matrix(s["qb"], s["sb"], tiles=c["tiles"])
        return ds.linear_f8(a, b, bias=s["bias"] if c["bias"] else None, add=s["add"] if c["add"] else None, dtype=TYPES[c["out"]])
    if c["op"] == "quantize":
        x = ds.F8Matrix(s["q"], s["s"]) if c["type"] == "f8" else s["x"]
        m, t = ds.quantize_f8(x, blocks=c["out"] or None, transposed=c["out_t"] or None, pow2=c["pow2"], dtype=FLOAT8[c["fmt"]])
        got = {}
        if m is not None:
            got["q"], got["scale"] = m.q, m.scale
        if t is not None:
            got["q_t"], got["scale_t"] = t.q, t.scale
        return got
    if c["op"] == "norm":
        n, h, rstd = ds.rmsnorm_f8(s["x"], s["w"], residual=s["r"] if c["residual"] else None, eps=EPS)
        return {"q": n.q, "scale": n.scale, "h": h, "rstd": rstd}
    if c["op"] == "norm_backward":
        dx, dw = ds.rmsnorm_f8_backward(s["dy"], s["h"], s["rstd"], s["w"], dh=s["dh"] if c["residual"] else None)
        return {"dx": dx, "dw": dw}
    if c["op"] == "gated":
        a, kept = ds.gated_f8(s["gu"], c["cols"], checkpoint=c["keep"])
        got = {"q": a.q, "scale": a.scale}
        if c["keep"]:
            got["kept"], got["kept_scale"] = kept.q, kept.scale
        return got
    d, d_t, a_t = ds.gated_f8_backward(ds.F8Matrix(s["q"], s["s"]), s["da"])
    return {"q": d.q, "scale": d.scale, "q_t": d_t.q, "scale_t": d_t.scale, "a_t": a_t.q, "a_scale_t": a_t.scale}


def run(state):
    return _library(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------ the inputs


def _rows16(q):
    """The same values in rows that start 16 bytes apart or a multiple of it, as 8-bit matrices are laid out."""
    held = torch.zeros(q.shape[0], _ceil(q.shape[1], 16), dtype=q.dtype, device=q.device)
    out = held[:, : q.shape[1]]
    out.copy_(q)
    return out


def prepare(case, seed):
    r = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=r, device="cuda")

    def activations(rows, cols):
        # columns of different strength, a few of them large
        strength = torch.exp(0.5 * normal(cols)) * torch.where(torch.rand(cols, generator=r, device="cuda") < 0.003, 20.0, 1.0)
        return normal(rows, cols) * strength

    def gradients(rows, cols):
        # rows of different strength: tokens that the loss weighs more or less
        return normal(rows, cols) * torch.exp(normal(rows, 1)) * 1e-3

    c, s = case, {"case": case}
    if c["op"] == "product":
        a = gradients(c["m"], c["k"]) if c["add"] else activations(c["m"], c["k"])
        b = activations(c["n"], c["k"]) if c["add"] else normal(c["n"], c["k"]) * 0.02
        s["qa"], s["sa"] = _to_f8(a, False, False, c["fmt"])
        s["qb"], s["sb"] = _to_f8(b, c["tiles"])
        s["qa"], s["qb"] = _rows16(s["qa"]), _rows16(s["qb"])
        if c["bias"]:
            s["bias"] = normal(c["n"])
        if c["add"]:
            s["add"] = normal(c["m"], c["n"]) * 0.1
        return s
    rows, cols = c["rows"], c["cols"]
    if c["op"] == "quantize":
        if c["type"] == "f8":
            q, s["s"] = _to_f8(activations(rows, cols), False, c["pow2"])
            s["q"] = _rows16(q)
        else:
            s["x"] = gradients(rows, cols).to(TYPES[c["type"]])
        return s
    kind = TYPES[c["type"]]
    if c["op"] in ("norm", "norm_backward"):
        s["w"] = 1.0 + 0.1 * normal(cols)
    if c["op"] == "norm":
        s["x"] = activations(rows, cols).to(kind)
        if c["residual"]:
            s["r"] = activations(rows, cols).to(kind)
    elif c["op"] == "norm_backward":
        s["h"] = activations(rows, cols).to(kind)
        s["rstd"] = torch.rsqrt(s["h"].float().square().mean(1) + EPS)
        s["dy"] = normal(rows, cols).to(kind)
        if c["residual"]:
            s["dh"] = normal(rows, cols).to(kind)
    elif c["op"] == "gated":
        s["gu"] = _halves(rows, cols, 2.0 * normal(rows, cols), normal(rows, cols)).to(kind)
    else:
        q, s["s"] = _to_f8(_halves(rows, cols, 2.0 * normal(rows, cols), normal(rows, cols)))
        s["q"] = _rows16(q)
        s["da"] = normal(rows, cols).to(kind)
    return s


def work(case):
    c = case
    if c["op"] == "product":
        m, k, n = c["m"], c["k"], c["n"]
        kb, nt = _ceil(k, BLOCK) // BLOCK, _ceil(n, BLOCK) // BLOCK if c["tiles"] else n
        moved = (m + n) * k + 4 * kb * (m + nt) + m * n * SIZE[c["out"]] + (4 * n if c["bias"] else 0) + (4 * m * n if c["add"] else 0)
        return {"bytes": moved, "flops": 2 * m * k * n}
    rows, cols = c["rows"], c["cols"]
    e, rb, cb = rows * cols, _ceil(rows, BLOCK) // BLOCK, _ceil(cols, BLOCK) // BLOCK
    if c["op"] == "quantize":
        moved = e + 4 * rows * cb if c["type"] == "f8" else e * SIZE[c["type"]]
        moved += (e + 4 * cb * (rb if c["out"] == "tiles" else rows)) if c["out"] else 0
        moved += (e + 4 * rb * (cb if c["out_t"] == "tiles" else cols)) if c["out_t"] else 0
        return {"bytes": moved, "flops": 4 * e}
    t = SIZE[c["type"]]
    if c["op"] == "norm":
        return {"bytes": e * (t * (3 if c["residual"] else 2) + 1) + 4 * rows * (cb + 1) + 4 * cols, "flops": 8 * e}
    if c["op"] == "norm_backward":
        return {"bytes": e * t * (4 if c["residual"] else 3) + 4 * rows + 8 * cols, "flops": 10 * e}
    if c["op"] == "gated":
        return {"bytes": e * (2 * t + 1 + (2 if c["keep"] else 0)) + 4 * rows * cb * (3 if c["keep"] else 1), "flops": 12 * e}
    return {"bytes": e * (t + 7) + 4 * (4 * rows * cb + 3 * cols * rb), "flops": 30 * e}


# ------------------------------------------------------------------------------------------------ in 64 bits


def _exact_f8(v, tiles=False, pow2=False, fmt="e4m3"):
    """Blocks, scales and rounding from their definition, in float64; values stand in a [rows, cols] matrix."""
    rows, cols = v.shape
    rb, cb = -(-rows // 128), -(-cols // 128)
    scale = torch.empty(rb if tiles else rows, cb, dtype=torch.float64, device=v.device)
    q = torch.empty_like(v)
    digits, lowest = {"e4m3": (3, -6), "e5m2": (2, -14)}[fmt]
    for j in range(cb):
        part = v[:, 128 * j : 128 * j + 128]
        size = part.abs().amax(1)
        if tiles:
            size = torch.stack([b.max() for b in size.split(128)])
        scale[:, j] = torch.maximum(size / LARGEST[fmt], torch.full_like(size, 2.0**-126))
        if pow2:
            m, e = torch.frexp(scale[:, j])
            scale[:, j] = torch.pow(torch.full_like(m, 2.0), torch.where(m == 0.5, e - 1, e).double())
        each = scale[:, j].repeat_interleave(128)[:rows] if tiles else scale[:, j]
        u = part / each[:, None]
        step = torch.pow(torch.full_like(u, 2.0), (torch.frexp(u)[1].double() - 1).clamp(min=lowest) - digits)
        q[:, 128 * j : 128 * j + 128] = torch.round(u / step) * step
    return q, scale


def _exact_value(q, s, tiles=False):
    v = q.double()
    for j in range(s.shape[1]):
        each = s[:, j].double()
        each = each.repeat_interleave(128)[: v.shape[0]] if tiles else each
        v[:, 128 * j : 128 * j + 128] *= each[:, None]
    return v


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "product":
        y = torch.mm(_exact_value(s["qa"], s["sa"]), _exact_value(s["qb"], s["sb"], c["tiles"]).T)
        if c["bias"]:
            y += s["bias"].double()
        if c["add"]:
            y += s["add"].double()
        return y
    if c["op"] == "quantize":
        v = _exact_value(s["q"], s["s"]) if c["type"] == "f8" else s["x"].double()
        got = {}
        if c["out"]:
            got["q"], got["scale"] = _exact_f8(v, c["out"] == "tiles", c["pow2"], c["fmt"])
        if c["out_t"]:
            got["q_t"], got["scale_t"] = _exact_f8(v.T.contiguous(), c["out_t"] == "tiles", c["pow2"], c["fmt"])
        return got
    if c["op"] == "norm":
        h = s["x"].double()
        if c["residual"]:
            h += s["r"].double()
        rstd = (torch.sum(h * h, 1) / c["cols"] + EPS) ** -0.5
        q, scale = _exact_f8(torch.einsum("rc,r,c->rc", h, rstd, s["w"].double()))
        return {"q": q, "scale": scale, "h": h, "rstd": rstd}
    if c["op"] == "norm_backward":
        dy, h, w, rstd = s["dy"].double(), s["h"].double(), s["w"].double(), s["rstd"].double()
        along = torch.sum(dy * w * h, 1) * rstd**3 / c["cols"]
        dx = dy * w * rstd[:, None] - h * along[:, None]
        if c["residual"]:
            dx += s["dh"].double()
        return {"dx": dx, "dw": torch.mv((dy * h).T, rstd)}
    n, start = c["cols"], _ceil(c["cols"], 128)
    both = s["gu"].double() if c["op"] == "gated" else _exact_value(s["q"], s["s"])
    g, u = both[:, :n], both[:, start:]
    sig = torch.sigmoid(g)
    if c["op"] == "gated":
        got = {}
        got["q"], got["scale"] = _exact_f8(g * sig * u)
        if c["keep"]:
            got["kept"], got["kept_scale"] = _exact_f8(both)
        return got
    da = s["da"].double()
    d = torch.zeros_like(both)
    d[:, :n] = da * u * (sig + g * sig * (1 - sig))
    d[:, start:] = da * g * sig
    got = {}
    got["q"], got["scale"] = _exact_f8(d)
    got["q_t"], got["scale_t"] = _exact_f8(d.T.contiguous())
    got["a_t"], got["a_scale_t"] = _exact_f8((g * sig * u).T.contiguous())
    return got

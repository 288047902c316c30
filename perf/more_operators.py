"""Cases of the experts' operators and of the optimizer step: what each has to compute, in a plain form and through the
library.

A feed-forward block with experts sends each token to `top_k` of `experts` blocks.  Its slots (token, choice) are put in
order of their expert, with a segment of rows for each that starts at a multiple of `align`; the tokens are copied to
these rows ("dispatch"), go through the experts' products with 8-bit operands ("product", "weight_grad"), and come back
weighted ("combine", "combine_backward").  Slots whose expert is -1 belong to padding and go nowhere; rows without a
slot are zeros.

The optimizer step ("adamw") updates many tensors at once.  Its two states are float32, or 8 bits: e4m3 values with a
float32 scale per 128 values of a tensor, the first moment and the root of the second.  A value between two 8-bit
neighbours becomes the upper one with a probability of its distance from the lower one; the random bits are a hash of
seed, step, the tensor's number and the value's index.
"""
import math

import torch

own = False

BLOCK = 128
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "": 0}
F8 = torch.float8_e4m3fn
LR, BETAS, EPS, DECAY, SEED, FIRST_STEP = 1e-3, (0.9, 0.999), 1e-8, 0.1, 17, 100


def listed():
    return [
        # norms, biases and small matrices of a few blocks, float32 throughout: one launch's latency counts
        dict(name="adamw_small", op="adamw", tensors=48, values=200_000, p="f32", g="f32", states="f32", copy=""),
        # the matrices of a block with float32 masters, 16-bit gradients, and the 16-bit copy that the products read
        dict(name="adamw_masters", op="adamw", tensors=9, values=50_000_000, p="f32", g="bf16", states="f32", copy="bf16"),
        # the same with both states in 8 bits
        dict(name="adamw_8bit", op="adamw", tensors=9, values=50_000_000, p="f32", g="bf16", states="f8", copy="bf16"),
        # a decoding step of 16 sequences: tokens in 8 bits to their experts, rows without gaps
        dict(name="dispatch_token", op="dispatch", tokens=16, top_k=4, experts=32, align=1, cols=4096, type="f8", padded=False),
        # a training batch whose last tokens are padding; segments start at whole blocks, for the weight gradients
        dict(name="dispatch_train", op="dispatch", tokens=8192, top_k=4, experts=32, align=128, cols=2048, type="bf16", padded=True),
        # the experts' outputs of the decoding step back to their tokens
        dict(name="combine_token", op="combine", tokens=16, top_k=4, experts=32, align=1, cols=4096, type="bf16", weighted=True, add=True, padded=False),
        # those of the training batch, added to the residual stream
        dict(name="combine_train", op="combine", tokens=8192, top_k=4, experts=32, align=128, cols=2048, type="bf16", weighted=True, add=True, padded=True),
        # the gradient of the tokens' copies, summed over their choices: odd sizes
        dict(name="dispatch_gradient", op="combine", tokens=4095, top_k=2, experts=8, align=128, cols=2050, type="bf16", weighted=False, add=False, padded=True),
        # the gradients of the experts' outputs and of the weights
        dict(name="combine_backward", op="combine_backward", tokens=8192, top_k=4, experts=32, align=128, cols=2048, type="bf16", padded=True),
        # the experts' products of the decoding step: the weights of the experts that are met are read once
        dict(name="product_token", op="product", tokens=16, top_k=4, experts=32, align=1, k=2048, n=4096, tiles=True, out="bf16", bias=False, padded=False),
        # and of the training batch
        dict(name="product_train", op="product", tokens=8192, top_k=4, experts=32, align=128, k=2048, n=4096, tiles=True, out="bf16", bias=False, padded=True),
        # the experts' weight gradients, added to those of earlier micro-batches
        dict(name="weight_grad_train", op="weight_grad", tokens=8192, top_k=4, experts=32, align=128, k=2048, n=2048, tiles=True, add=True, padded=True),
    ]


def _size(rng, low, high):
    """A size spread over the logarithm of its range: mostly multiples of 64 or 8, every third one as it comes."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    step = rng.choice((1, 8, 64))
    return max(low, n // step * step) if n >= step else n


def draw(rng):
    op = rng.choice(("adamw", "adamw", "dispatch", "combine", "combine_backward", "product", "product", "weight_grad"))
    if op == "adamw":
        p = rng.choice(("f32", "f32", "f32", "bf16"))
        return dict(op=op, tensors=_size(rng, 1, 64), values=_size(rng, 10_000, 40_000_000), p=p,
                    g=rng.choice(("f32", "bf16")) if p == "f32" else p, states=rng.choice(("f32", "f8", "f8")),
                    copy=rng.choice(("", "bf16", "f16")) if p == "f32" else "")
    tokens, experts = _size(rng, 1, 8192), rng.choice((4, 8, 16, 32, 60, 64))
    top_k = min(rng.choice((1, 2, 4, 6, 8)), experts)
    while tokens * top_k > 32768:
        tokens = (tokens + 1) // 2
    route = dict(op=op, tokens=tokens, top_k=top_k, experts=experts, align=rng.choice((1, 128)) if tokens > 256 else 1, padded=rng.random() < 0.5)
    if op == "dispatch":
        return dict(route, cols=_size(rng, 256, 2048), type=rng.choice(("f8", "bf16", "f16")))
    if op == "combine":
        weighted = rng.random() < 0.7
        return dict(route, cols=_size(rng, 256, 2048), type=rng.choice(("bf16", "bf16", "f16", "f32")), weighted=weighted, add=weighted and rng.random() < 0.5)
    if op == "combine_backward":
        return dict(route, cols=_size(rng, 256, 2048), type=rng.choice(("bf16", "bf16", "f16")))
    k, n = _size(rng, 256, 2048), _size(rng, 256, 4096 if op == "product" else 2048)
    if op == "product":
        while experts * n * k > 32 * 4096 * 2048:
            n = (n + 1) // 2
        return dict(route, k=k, n=n, tiles=n % BLOCK == 0, out=rng.choice(("bf16", "bf16", "f16", "f32")), bias=rng.random() < 0.3)
    while experts * n * k > 32 * 2048 * 2048:
        n = (n + 1) // 2
    route["align"] = 128
    return dict(route, k=k, n=n, tiles=rng.random() < 0.7, add=rng.random() < 0.5)


def _ceil(n, step):
    return -(-n // step) * step


def _rows(c):
    """Rows that the segments of any routing fit in."""
    slots = c["tokens"] * c["top_k"]
    return (slots + min(c["experts"], slots) * (c["align"] - 1)) // c["align"] * c["align"]


def _sizes(c):
    """The tensors of an optimizer's case: of several sizes, every third one odd."""
    share = [1 + 3 * (i % 4) for i in range(c["tensors"])]
    return [max(1, c["values"] * w // sum(share) - (5 * i + 3 if i % 3 == 1 else 0)) for i, w in enumerate(share)]


# ------------------------------------------------------------------------------------------------ the plain form


def _spread(s, rows, cols, tiles):
    s = s.repeat_interleave(BLOCK, 1)[:, :cols]
    return s.repeat_interleave(BLOCK, 0)[:rows] if tiles else s


def _from_f8(q, s, tiles=False):
    return q.float() * _spread(s, *q.shape, tiles)


def _to_f8(v, tiles=False):
    """Blocks of 128 values of a row, or of 128 x 128, rounded to the nearest e4m3 values."""
    rows, cols = v.shape
    rb, cb = _ceil(rows, BLOCK), _ceil(cols, BLOCK)
    a = torch.zeros(rb, cb, device=v.device)
    a[:rows, :cols] = v.abs()
    a = a.view(rb // BLOCK, BLOCK, cb // BLOCK, BLOCK).amax((1, 3)) if tiles else a[:rows].view(rows, cb // BLOCK, BLOCK).amax(2)
    s = (a / 448.0).clamp(min=2.0**-126)
    q = torch.zeros(rows, _ceil(cols, 16), dtype=F8, device=v.device)[:, :cols]  # rows 16 bytes apart or a multiple of it
    q.copy_((v / _spread(s, rows, cols, tiles)).clamp(-448.0, 448.0).to(F8))
    return q, s


def _order(ids, experts, align, rows):
    """Segments, counts, the row of each slot (-1: none) and the slot of each row (-1: none); slots stay in their order."""
    flat = ids.reshape(-1).long()
    here = (flat >= 0) & (flat < experts)
    each = torch.arange(experts, device=ids.device)[:, None] == flat
    before = each.cumsum(1, dtype=torch.int32)
    counts = before[:, -1].clone()
    offsets = torch.zeros(experts + 1, dtype=torch.int32, device=ids.device)
    offsets[1:] = ((counts + align - 1) // align * align).cumsum(0)
    key = torch.where(here, flat, 0)
    position = offsets[key] + before.gather(0, key[None])[0] - 1
    slot = torch.full((rows + 1,), -1, dtype=torch.int32, device=ids.device)
    slot[torch.where(here, position, rows).long()] = torch.arange(flat.numel(), dtype=torch.int32, device=ids.device)
    return {"offsets": offsets, "counts": counts, "position": torch.where(here, position, -1).view(ids.shape), "slot": slot[:rows].clone()}


def _gather(x, slot, top_k):
    return torch.where((slot >= 0)[:, None], x[(slot // top_k).clamp(min=0).long()], torch.zeros((), dtype=x.dtype, device=x.device))


def _uniform(n, key, device):
    """Two random numbers in (0, 1) for each of n values: the halves of a hash of the index."""
    low = 0xFFFFFFFF
    x = (torch.arange(n, device=device) * 0x9E3779B1 + key) & low
    x = ((x ^ (x >> 16)) * 0x243F6A89) & low
    x = ((x ^ (x >> 15)) * 0xB7E15163) & low
    x = x ^ (x >> 16)
    return x & 0xFFFF, x >> 16


def _state_to_f8(v, bits, positive):
    """A tensor's values in blocks of 128: to the neighbour above where the 16 random bits say so, else to that below."""
    n = v.numel()
    a = torch.zeros(_ceil(n, BLOCK), device=v.device)
    a[:n] = v.abs()
    top = a.view(-1, BLOCK).amax(1)
    most = torch.full_like(top, 448.0)
    scale = (top / most).clamp(min=2.0**-126)
    u = a[:n] * (most / top).clamp(max=2.0**126).repeat_interleave(BLOCK)[:n]
    # below the smallest normal value (2^-6) the neighbours are 2^-9 apart, as they are between 2^-6 and 2^-5
    low = u < 2.0**-6
    w = torch.where(low, u + 2.0**-6, u).view(torch.int32)
    w = ((w + bits.to(torch.int32) * 16 + 8) & ~0xFFFFF).view(torch.float32)
    w = torch.where(low, w - 2.0**-6, w).clamp(max=448.0)
    if positive:  # no root becomes zero, by which an update would be divided
        w = torch.where(v > 0, w.clamp(min=2.0**-9), w)
    return torch.copysign(w, v).to(F8), scale


def _state_value(q, scale):
    return q.float() * scale.repeat_interleave(BLOCK)[: q.numel()]


def _key(step, number):
    return (step * 0xBB67AE85 + number * 0x6A09E667 + SEED) & 0xFFFFFFFF


def _adamw_plain(s):
    c, (b1, b2) = s["case"], BETAS
    s["step"] += 1
    step = s["step"]
    rate, root_factor = LR / (1 - b1**step), 1 / math.sqrt(1 - b2**step)
    p = [x.float() for x in s["p"]]
    g = [x.float() * s["scale"] for x in s["g"]]
    if c["states"] == "f8":
        m = [_state_value(q, a) for q, a in s["m"]]
        root = [_state_value(q, a) for q, a in s["v"]]
        v = torch._foreach_mul(root, root)
    else:
        m, v = s["m"], s["v"]
    m = torch._foreach_add(torch._foreach_mul(m, b1), torch._foreach_mul(g, 1 - b1))
    v = torch._foreach_add(torch._foreach_mul(v, b2), torch._foreach_mul(torch._foreach_mul(g, g), 1 - b2))
    root = torch._foreach_sqrt(v)
    under = torch._foreach_add(torch._foreach_mul(root, root_factor), EPS)
    p = torch._foreach_sub(torch._foreach_mul(p, [1 - LR * d for d in s["decay"]]), torch._foreach_div(torch._foreach_mul(m, rate), under))
    torch._foreach_copy_(s["p"], p)
    if c["copy"]:
        torch._foreach_copy_(s["copy"], p)
    if c["states"] == "f8":
        bits = [_uniform(x.numel(), _key(step, i), x.device) for i, x in enumerate(p)]
        new_m = [_state_to_f8(x, b[0], False) for x, b in zip(m, bits)]
        new_v = [_state_to_f8(x, b[1], True) for x, b in zip(root, bits)]
        [(a[0].copy_(b[0]), a[1].copy_(b[1])) for a, b in zip(s["m"] + s["v"], new_m + new_v)]
    else:
        torch._foreach_copy_(s["m"], m)
        torch._foreach_copy_(s["v"], v)
    return s["all"]


def _plain(s):
    c = s["case"]
    if c["op"] == "adamw":
        return _adamw_plain(s)
    if c["op"] == "dispatch":
        got = _order(s["ids"], c["experts"], c["align"], _rows(c))
        if c["type"] == "f8":
            got["q"] = _gather(s["q"].view(torch.uint8), got["slot"], c["top_k"]).view(F8)
            got["scale"] = _gather(s["s"], got["slot"], c["top_k"])
        else:
            got["rows"] = _gather(s["x"], got["slot"], c["top_k"])
        return got
    o, kind = s["order"], TYPES[c.get("type", "f32")]
    if c["op"] == "combine":
        there = o["position"] >= 0
        y = torch.where(there[:, :, None], s["y"][o["position"].clamp(min=0).long()].float(), 0.0)
        if c["weighted"]:
            y = y * s["w"][:, :, None]
        y = y.sum(1)
        return (y + s["add"].float() if c["add"] else y).to(kind)
    if c["op"] == "combine_backward":
        there = o["position"] >= 0
        d = s["d"].float()
        w = s["w"].reshape(-1)[o["slot"].clamp(min=0).long()]
        dw = (d[:, None, :] * s["y"][o["position"].clamp(min=0).long()].float()).sum(2)
        return {"dy": (_gather(d, o["slot"], c["top_k"]) * w[:, None]).to(kind), "dw": torch.where(there, dw, 0.0)}
    b = s["bounds"]
    if c["op"] == "product":
        x, w = _from_f8(s["qx"], s["sx"]), _from_f8(s["qw"], s["sw"], c["tiles"]).view(c["experts"], c["n"], c["k"])
        y = [x[b[e] : b[e + 1]] @ w[e].t() + (s["bias"][e] if c["bias"] else 0.0) for e in range(c["experts"])]
        return torch.cat(y + [x.new_zeros(x.shape[0] - b[-1], c["n"])]).to(TYPES[c["out"]])
    d, x = _from_f8(s["qd"], s["sd"]), _from_f8(s["qx"], s["sx"], c["tiles"])
    dw = torch.stack([d[:, b[e] : b[e + 1]] @ x[:, b[e] : b[e + 1]].t() for e in range(c["experts"])])
    return dw + s["add"] if c["add"] else dw


# ------------------------------------------------------------------------------------------------ the library's


def _library(s):
    import paper_1905_13298_gb300 as ds

    c = s["case"]
    if c["op"] == "adamw":
        if "optimizer" not in s:  # made once by a program and kept
            s["optimizer"] = ds.AdamW(s["p"], s["g"], m=s["m"], v=s["v"], copies=s["copy"] if c["copy"] else None, lr=LR, betas=BETAS, eps=EPS,
                                      weight_decay=s["decay"], grad_scale=s["scale"], steps=s["step"], seed=SEED)
        s["optimizer"].step()
        return s["all"]
    if c["op"] == "dispatch":
        x = ds.F8Matrix(s["q"], s["s"]) if c["type"] == "f8" else s["x"]
        order = ds.expert_order(s["ids"], c["experts"], align=c["align"])
        rows = ds.expert_gather(x, order)
        got = {"offsets": order.offsets, "counts": order.counts, "position": order.position, "slot": order.slot}
        return dict(got, q=rows.q, scale=rows.scale) if c["type"] == "f8" else dict(got, rows=rows)
    if "kept" not in s:  # what expert_order returned in the forward pass
        o = s["order"]
        s["kept"] = ds.ExpertOrder(o["offsets"], o["counts"], o["position"], o["slot"], align=c["align"])
    order = s["kept"]
    if c["op"] == "combine":
        return ds.expert_combine(s["y"], order, weights=s["w"] if c["weighted"] else None, add=s["add"] if c["add"] else None)
    if c["op"] == "combine_backward":
        dy, dw = ds.expert_combine_backward(s["d"], s["y"], order, s["w"])
        return {"dy": dy, "dw": dw}
    if c["op"] == "product":
        x, w = ds.F8Matrix(s["qx"], s["sx"]), ds.F8Matrix(s["qw"], s["sw"], tiles=c["tiles"])
        return ds.expert_linear_f8(x, w, order, bias=s["bias"] if c["bias"] else None, dtype=TYPES[c["out"]])
    d, x = ds.F8Matrix(s["qd"], s["sd"]), ds.F8Matrix(s["qx"], s["sx"], tiles=c["tiles"])
    return ds.expert_weight_grad_f8(d, x, order, add=s["add"] if c["add"] else None)


def run(state):
    return _library(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------ the inputs


def prepare(case, seed):
    r = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=r, device="cuda")

    c, s = case, {"case": case}
    if c["op"] == "adamw":
        sizes = _sizes(c)
        # the tensors lie in one memory, as a program lays out its parameters
        at = [0]
        for n in sizes:
            at.append(at[-1] + _ceil(n, BLOCK))

        def views(flat, unit=1):
            return [flat[a // unit : a // unit + -(-n // unit)] for a, n in zip(at, sizes)]

        total = at[-1]
        p = (normal(total) * 0.02).to(TYPES[c["p"]])
        g = (normal(total) * 1e-3 * torch.exp(normal(total // BLOCK)).repeat_interleave(BLOCK)).to(TYPES[c["g"]])
        m, v = normal(total) * 3e-4, (normal(total) * 1e-3).square()
        s["all"] = {"p": p}
        s["p"], s["g"] = views(p), views(g)
        if c["states"] == "f8":
            qm, sm = _to_f8(m.view(-1, BLOCK))
            qv, sv = _to_f8(v.sqrt().view(-1, BLOCK))
            s["all"].update(m=qm.reshape(-1), m_scale=sm.reshape(-1), v=qv.reshape(-1), v_scale=sv.reshape(-1))
            s["m"] = list(zip(views(s["all"]["m"]), views(s["all"]["m_scale"], BLOCK)))
            s["v"] = list(zip(views(s["all"]["v"]), views(s["all"]["v_scale"], BLOCK)))
        else:
            s["all"].update(m=m, v=v)
            s["m"], s["v"] = views(m), views(v)
        if c["copy"]:
            s["all"]["copy"] = p.to(TYPES[c["copy"]])
            s["copy"] = views(s["all"]["copy"])
        s["decay"] = [DECAY if n > 4096 else 0.0 for n in sizes]  # none on norms and biases
        s["scale"] = torch.full((), 0.75, device="cuda")  # a norm of all gradients was above its bound
        s["step"] = FIRST_STEP
        return s

    # some experts are asked for more than others
    likes = normal(c["tokens"], c["experts"]) + 0.7 * normal(c["experts"])
    best, ids = likes.topk(c["top_k"], 1)
    if c["padded"]:
        ids[c["tokens"] - c["tokens"] // 32 :] = -1
    rows, weights = _rows(c), torch.softmax(best, 1)
    if c["op"] == "dispatch":
        x = normal(c["tokens"], c["cols"])
        s["ids"] = ids
        if c["type"] == "f8":
            s["q"], s["s"] = _to_f8(x)
        else:
            s["x"] = x.to(TYPES[c["type"]])
        return s
    o = s["order"] = _order(ids, c["experts"], c["align"], rows)
    if c["op"] in ("combine", "combine_backward"):
        kind = TYPES[c["type"]]
        s["y"] = normal(rows, c["cols"]).to(kind)
        s["w"] = weights
        if c["op"] == "combine_backward":
            s["d"] = normal(c["tokens"], c["cols"]).to(kind)
        elif c["add"]:
            s["add"] = normal(c["tokens"], c["cols"]).to(kind)
        return s
    s["bounds"] = o["offsets"].tolist()
    if c["op"] == "product":
        s["qx"], s["sx"] = _to_f8(_gather(normal(c["tokens"], c["k"]), o["slot"], c["top_k"]))
        s["qw"], s["sw"] = _to_f8(normal(c["experts"] * c["n"], c["k"]) * c["k"] ** -0.5, c["tiles"])
        if c["bias"]:
            s["bias"] = normal(c["experts"], c["n"])
        return s
    d = _gather(normal(c["tokens"], c["n"]) * torch.exp(normal(c["tokens"], 1)) * 1e-3, o["slot"], c["top_k"])
    s["qd"], s["sd"] = _to_f8(d.t().contiguous())
    s["qx"], s["sx"] = _to_f8(_gather(normal(c["tokens"], c["k"]), o["slot"], c["top_k"]).t().contiguous(), c["tiles"])
    if c["add"]:
        s["add"] = normal(c["experts"], c["n"], c["k"]) * 0.01
    return s


def work(case):
    c = case
    if c["op"] == "adamw":
        n = sum(_sizes(c))
        states = 16 if c["states"] == "f32" else 4 + 16 / BLOCK
        return {"bytes": n * (2 * SIZE[c["p"]] + SIZE[c["g"]] + states + SIZE[c["copy"]]), "flops": n * (16 if c["states"] == "f32" else 40)}
    slots, rows, t, e = c["tokens"] * c["top_k"], _rows(c), c["tokens"], c["experts"]
    index = 4 * (slots + rows + 2 * e + 1)
    if c["op"] == "dispatch":
        width = c["cols"] + 4 * (_ceil(c["cols"], BLOCK) // BLOCK) if c["type"] == "f8" else c["cols"] * SIZE[c["type"]]
        return {"bytes": 8 * slots + index + (t + rows) * width, "flops": slots * 4}
    if c["op"] == "combine":
        width = c["cols"] * SIZE[c["type"]]
        moved = (slots + t * (2 if c["add"] else 1)) * width + slots * (8 if c["weighted"] else 4)
        return {"bytes": moved, "flops": slots * c["cols"] * 2}
    if c["op"] == "combine_backward":
        return {"bytes": (t + slots + rows) * c["cols"] * SIZE[c["type"]] + 12 * slots + 4 * rows, "flops": slots * c["cols"] * 3}
    k, n, blocks = c["k"], c["n"], _ceil(c["k"], BLOCK) // BLOCK
    if c["op"] == "product":
        met = e * (1 - (1 - c["top_k"] / e) ** t)  # experts with rows, where all are asked for alike
        scales = 4 * blocks * (n / BLOCK if c["tiles"] else n)
        return {"bytes": slots * (k + 4 * blocks) + met * (n * k + scales) + rows * n * SIZE[c["out"]], "flops": 2 * slots * n * k}
    moved = rows * (n + k) + rows // BLOCK * 4 * (n + (k / BLOCK if c["tiles"] else k)) + e * n * k * (8 if c["add"] else 4)
    return {"bytes": moved, "flops": 2 * slots * n * k}


# ------------------------------------------------------------------------------------------------ in 64 bits


def _exact_value(q, s, tiles=False):
    v = q.double()
    for j in range(s.shape[1]):
        each = s[:, j].double()
        each = each.repeat_interleave(128)[: v.shape[0]] if tiles else each
        v[:, 128 * j : 128 * j + 128] *= each[:, None]
    return v


def _exact_state(v, bits, positive):
    """Blocks and neighbours from their definition, in float64; the values, and the scales."""
    n = v.numel()
    blocks = torch.nn.functional.pad(v, (0, -n % 128)).view(-1, 128)
    scale = (blocks.abs().max(1).values / 448.0).clamp(min=2.0**-126)
    u = (blocks / scale[:, None]).reshape(-1)[:n].abs()
    step = torch.exp2((torch.frexp(u)[1].double() - 1).clamp(min=-6) - 3)
    q = torch.floor(u / step + (bits.double() + 0.5) / 65536.0) * step
    if positive:
        q = torch.where(v > 0, q.clamp(min=2.0**-9), q)
    return torch.sign(v) * q.clamp(max=448.0), scale


def _exact_adamw(s):
    c, t = s["case"], FIRST_STEP + 1
    got = {k: v.double() for k, v in s["all"].items()}
    at = 0
    for i, g in enumerate(s["g"]):
        n = g.numel()
        part = slice(at, at + n)
        blocks = slice(at // BLOCK, (at + n + BLOCK - 1) // BLOCK)
        g = g.double() * 0.75
        if c["states"] == "f8":
            m = got["m"][part] * got["m_scale"][blocks].repeat_interleave(128)[:n]
            v = (got["v"][part] * got["v_scale"][blocks].repeat_interleave(128)[:n]) ** 2
        else:
            m, v = got["m"][part], got["v"][part]
        m = BETAS[0] * m + (1 - BETAS[0]) * g
        v = BETAS[1] * v + (1 - BETAS[1]) * g**2
        step = LR * (m / (1 - BETAS[0] ** t)) / (torch.sqrt(v / (1 - BETAS[1] ** t)) + EPS)
        p = got["p"][part] - LR * s["decay"][i] * got["p"][part] - step
        got["p"][part] = p
        if c["copy"]:
            got["copy"][part] = p
        if c["states"] == "f8":
            low, high = _uniform(n, _key(t, i), g.device)
            got["m"][part], got["m_scale"][blocks] = _exact_state(m, low, False)
            got["v"][part], got["v_scale"][blocks] = _exact_state(torch.sqrt(v), high, True)
        else:
            got["m"][part], got["v"][part] = m, v
        at += -(-n // BLOCK) * BLOCK
    return got


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "adamw":
        return _exact_adamw(s)
    if c["op"] == "dispatch":
        got = {"offsets": None, "counts": None, "position": None, "slot": None}  # whole numbers are compared with the plain form's
        o = _order(s["ids"], c["experts"], c["align"], _rows(c))
        used = torch.nonzero(o["slot"] >= 0)[:, 0]
        token = torch.div(o["slot"][used].long(), c["top_k"], rounding_mode="floor")
        for name, x in (("q", s["q"]), ("scale", s["s"])) if c["type"] == "f8" else (("rows", s["x"]),):
            got[name] = torch.zeros(_rows(c), x.shape[1], dtype=torch.float64, device=x.device)
            got[name][used] = x.double()[token]
        return got
    o = s["order"]
    if c["op"] in ("combine", "combine_backward"):
        slots = torch.nonzero(o["position"].reshape(-1) >= 0)[:, 0]
        row, token = o["position"].reshape(-1)[slots].long(), torch.div(slots, c["top_k"], rounding_mode="floor")
        w = s["w"].double().reshape(-1)[slots]
        if c["op"] == "combine":
            y = s["add"].double() if c["add"] else torch.zeros(c["tokens"], c["cols"], dtype=torch.float64, device=w.device)
            return y.index_add_(0, token, s["y"].double()[row] * (w[:, None] if c["weighted"] else 1.0))
        d = s["d"].double()[token]
        dy = torch.zeros(_rows(c), c["cols"], dtype=torch.float64, device=w.device)
        dy[row] = d * w[:, None]
        dw = torch.zeros(c["tokens"] * c["top_k"], dtype=torch.float64, device=w.device)
        dw[slots] = torch.einsum("sc,sc->s", d, s["y"].double()[row])
        return {"dy": dy, "dw": dw.view(c["tokens"], c["top_k"])}
    b = s["bounds"]
    if c["op"] == "product":
        x, w = _exact_value(s["qx"], s["sx"]), _exact_value(s["qw"], s["sw"], c["tiles"])
        y = torch.zeros(x.shape[0], c["n"], dtype=torch.float64, device=x.device)
        for e in range(c["experts"]):
            y[b[e] : b[e + 1]] = torch.einsum("rk,nk->rn", x[b[e] : b[e + 1]], w[e * c["n"] : (e + 1) * c["n"]])
            if c["bias"]:
                y[b[e] : b[e + 1]] += s["bias"][e].double()
        return y
    d, x = _exact_value(s["qd"], s["sd"]), _exact_value(s["qx"], s["sx"], c["tiles"])
    dw = s["add"].double() if c["add"] else torch.zeros(c["experts"], c["n"], c["k"], dtype=torch.float64, device=d.device)
    for e in range(c["experts"]):
        dw[e] += torch.einsum("nr,kr->nk", d[:, b[e] : b[e + 1]], x[:, b[e] : b[e + 1]])
    return dw

"""GPU parity of the experts' operators (order, gather, combine, products) with the numpy oracle.

Tolerances follow from the arithmetic and were fixed before the first run: whole numbers and copies are equal; a result
may be off by half a step of its type (`HALF`), a sum of n float32 terms by n * 2^-24 of the sum of their magnitudes,
and the 8-bit products by TOL of it, as those of the dense product (test_gpu_f8.py).
"""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as X
from oracle import float8_oracle as F

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {k: torch.finfo(t).eps / 2 for k, t in TYPES.items()}
TINY = {"f32": 1e-38, "bf16": 1e-38, "f16": 2.0**-25}
TOL = 1e-5


def _rng(*key):
    return np.random.default_rng(sum(ord(c) * (i + 1) for i, c in enumerate(str(key))))


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _ids(r, tokens, top_k, experts, kind="even"):
    if kind == "one":  # all to one expert, the same one several times
        return np.full((tokens, top_k), experts // 2, np.int64)
    ids = r.integers(0, experts, (tokens, top_k))
    if kind == "dropped":  # padding, and numbers that are no expert's
        ids = np.where(r.random(ids.shape) < 0.3, r.choice([-1, -7, experts, experts + 5, 2**31 - 1], ids.shape), ids)
    if kind == "none":
        ids = np.full_like(ids, -1)
    return ids.astype(np.int64)


def _order(ds, ids, experts, align, kind=torch.int64):
    tokens, top_k = ids.shape
    order = ds.expert_order(torch.from_numpy(ids).cuda().to(kind), experts, align=align)
    want = X.order(ids, experts, align, X.rows_needed(tokens, top_k, experts, align))
    return order, want


def _check_order(order, want):
    for name, w in zip(("offsets", "counts", "position", "slot"), want):
        assert np.array_equal(getattr(order, name).cpu().numpy(), w), name


def _strided(t, extra):
    """The same matrix with rows `extra` elements further apart, its neighbours NaN."""
    held = torch.full((t.shape[0], t.shape[1] + extra), float("nan"), dtype=t.dtype, device=t.device)
    held[:, : t.shape[1]] = t
    return held[:, : t.shape[1]]


def _near(got, want, bound):
    err = np.abs(got - want)
    assert np.all(err <= bound), float((err / np.maximum(bound, 1e-300)).max())


# ------------------------------------------------------------------------------------------------------------- order


@pytest.mark.parametrize("tokens,top_k,experts", [(1, 1, 1), (1, 4, 7), (3, 2, 1024), (16, 4, 32), (33, 1, 5), (257, 8, 60),
                                                  (1023, 1, 3), (1025, 2, 64), (4100, 4, 33), (9000, 8, 256)])
@pytest.mark.parametrize("align", [1, 16, 128])
@pytest.mark.parametrize("kind", ["even", "one", "dropped", "none"])
def test_order(dslib, tokens, top_k, experts, align, kind):
    r = _rng("order", tokens, top_k, experts, align, kind)
    ids = _ids(r, tokens, top_k, experts, kind)
    order, want = _order(dslib, ids, experts, align)
    _check_order(order, want)
    order, _ = _order(dslib, ids, experts, align, torch.int32)
    _check_order(order, want)
    assert (order.tokens, order.top_k, order.experts, order.align) == (tokens, top_k, experts, align)


def test_order_of_no_tokens(dslib):
    order = dslib.expert_order(torch.empty((0, 4), dtype=torch.int64, device="cuda"), 5, align=128)
    assert order.rows == 0 and order.offsets.tolist() == [0] * 6 and order.counts.tolist() == [0] * 5
    x = torch.empty((0, 256), device="cuda", dtype=torch.bfloat16)
    rows = dslib.expert_gather(x, order)
    assert rows.shape == (0, 256) and dslib.expert_combine(rows, order).shape == (0, 256)


def test_order_of_large_ids(dslib):
    """64-bit ids whose low 32 bits are an expert's number."""
    ids = np.array([[1, 2**32 + 1], [-(2**32) + 2, 2]], np.int64)
    order, want = _order(dslib, ids, 4, 1)
    _check_order(order, want)
    assert order.counts.tolist() == [0, 1, 1, 0]


def test_order_with_more_rows_than_needed(dslib):
    """A caller's own memory with room behind: the rows there hold no slot."""
    ids = _ids(_rng("room"), 20, 2, 6)
    n = X.rows_needed(20, 2, 6, 16) + 77
    t = lambda *s: torch.full(s, 99, dtype=torch.int32, device="cuda")  # noqa: E731
    order = dslib.ExpertOrder(t(7), t(6), t(20, 2), t(n), align=16)
    dslib.ds_expert_order(torch.from_numpy(ids).cuda(), dslib.DS_INDEX_I64, order.desc)
    _check_order(order, X.order(ids, 6, 16, n))


# ------------------------------------------------------------------------------------------------- gather and combine

COLS = [1, 8, 127, 256, 2050, 4096]


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tokens,top_k,experts,align,kind", [(5, 3, 4, 1, "dropped"), (40, 9, 6, 16, "even"), (70, 2, 5, 128, "dropped")])
def test_gather(dslib, cols, dtype, tokens, top_k, experts, align, kind):
    r = _rng("gather", cols, dtype, tokens)
    order, want = _order(dslib, _ids(r, tokens, top_k, experts, kind), experts, align)
    x = torch.from_numpy(r.standard_normal((tokens, cols)).astype(np.float32)).cuda().to(TYPES[dtype])
    rows = X.gather(_np(x), want[3], top_k)
    assert np.array_equal(_np(dslib.expert_gather(x, order)), rows)
    for extra in (1, 2, 4, 8):  # strides that allow accesses of every width; what lies between rows stays
        out = _strided(torch.full((order.rows, cols), 5.0, dtype=x.dtype, device="cuda"), extra)
        got = dslib.expert_gather(_strided(x, extra), order, out=out)
        assert got is out and np.array_equal(_np(got), rows)
        beyond = torch.as_strided(out, (order.rows - 1, extra), (cols + extra, 1), out.storage_offset() + cols)
        assert bool(torch.isnan(beyond).all())


@pytest.mark.parametrize("cols", [1, 16, 100, 128, 400, 4096])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_gather_f8(dslib, cols, fmt):
    r = _rng("gather8", cols, fmt)
    order, want = _order(dslib, _ids(r, 37, 3, 5, "dropped"), 5, 16)
    q, s = F.quantize(r.standard_normal((37, cols)), False, False, fmt)
    kind = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}[fmt]
    held = torch.full((37, -(-cols // 16) * 16 + 16), float("nan"), device="cuda").to(kind)
    held[:, :cols] = torch.from_numpy(q.astype(np.float32)).cuda().to(kind)
    x = dslib.F8Matrix(held[:, :cols], torch.from_numpy(s).cuda())
    m = dslib.expert_gather(x, order)
    assert np.array_equal(_np(m.q), X.gather(q.astype(np.float64), want[3], 3))
    assert np.array_equal(m.scale.cpu().numpy(), X.gather(s, want[3], 3))


@pytest.mark.parametrize("tokens", [0, 3])
def test_gather_f8_zeroes_rows_behind(dslib, tokens):
    """Rows above what the tokens need hold no slot: their values and scales are zeros, also without any token, where x has
    no memory."""
    t = lambda *s: torch.full(s, 99, dtype=torch.int32, device="cuda")  # noqa: E731
    order = dslib.ExpertOrder(t(4), t(3), t(tokens, 2), t(128 + tokens))
    ids = torch.arange(2 * tokens, device="cuda").view(tokens, 2) % 3
    dslib.ds_expert_order(ids, dslib.DS_INDEX_I64, order.desc)
    x = dslib.F8Matrix.empty(tokens, 400, torch.device("cuda"))
    x.q.view(torch.uint8).fill_(0x38)  # ones
    x.scale.fill_(2.0)
    out = dslib.F8Matrix.empty(order.rows, 400, torch.device("cuda"))
    out.q.view(torch.uint8).fill_(0x7F)  # NaN
    out.scale.fill_(float("nan"))
    assert dslib.expert_gather(x, order, out=out) is out
    held = order.slot >= 0
    assert int(held.sum()) == 2 * tokens
    assert torch.equal(out.scale, (2.0 * held[:, None]).expand(-1, 4))
    assert torch.equal(out.dequantize(), (2.0 * held[:, None]).expand(-1, 400))


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tokens,top_k,experts,align,kind", [(5, 3, 4, 1, "dropped"), (33, 17, 6, 16, "even"), (64, 2, 5, 128, "dropped"), (4, 2, 3, 1, "none")])
@pytest.mark.parametrize("weighted,added,extra", [(True, True, 0), (True, False, 1), (False, False, 8), (False, True, 2)])
def test_combine(dslib, cols, dtype, tokens, top_k, experts, align, kind, weighted, added, extra):
    r = _rng("combine", cols, dtype, tokens, weighted, added)
    order, want = _order(dslib, _ids(r, tokens, top_k, experts, kind), experts, align)
    dev = lambda *s: torch.from_numpy(r.standard_normal(s).astype(np.float32)).cuda()  # noqa: E731
    y = dev(order.rows, cols).to(TYPES[dtype])
    y[torch.from_numpy(want[3] < 0).cuda()] = float("nan")  # rows without a slot are not read
    w = dev(tokens, top_k) if weighted else None
    add = dev(tokens, cols).to(TYPES[dtype]) if added else None
    exact, size = X.combine(_np(y), want[2], None if w is None else _np(w), None if add is None else _np(add))
    bound = HALF[dtype] * np.abs(exact) + (top_k + 2) * 2.0**-24 * size + TINY[dtype]
    if extra:
        y = _strided(y, extra)
    got = dslib.expert_combine(y, order, w, add)
    _near(_np(got), exact, bound)
    if added:  # in place, the same bits
        assert dslib.expert_combine(y, order, w, add, out=add) is add and torch.equal(add, got)


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tokens,top_k,experts,align,kind", [(5, 3, 4, 1, "dropped"), (33, 17, 6, 16, "even"), (64, 2, 5, 128, "dropped"), (4, 2, 3, 128, "none")])
@pytest.mark.parametrize("weighted,extra", [(True, 0), (True, 1), (False, 2)])
def test_combine_backward(dslib, cols, dtype, tokens, top_k, experts, align, kind, weighted, extra):
    r = _rng("backward", cols, dtype, tokens, weighted)
    order, want = _order(dslib, _ids(r, tokens, top_k, experts, kind), experts, align)
    dev = lambda *s: torch.from_numpy(r.standard_normal(s).astype(np.float32)).cuda()  # noqa: E731
    d, y = dev(tokens, cols).to(TYPES[dtype]), dev(order.rows, cols).to(TYPES[dtype])
    y[torch.from_numpy(want[3] < 0).cuda()] = float("nan")
    w = dev(tokens, top_k) if weighted else None
    dy, dw, size = X.combine_backward(_np(d), np.nan_to_num(_np(y)), want[2], order.rows, None if w is None else _np(w))
    if extra:
        d, y = _strided(d, extra), _strided(y, extra)
    got, gw = dslib.expert_combine_backward(d, y, order, w)
    _near(_np(got), dy, (HALF[dtype] + 2.0**-24) * np.abs(dy) + TINY[dtype])
    if weighted:
        _near(_np(gw), dw, (cols / 32 + 16) * 2.0**-24 * size + 1e-38)
        again, gw2 = dslib.expert_combine_backward(d, y, order, w, out=y)  # over y itself, the same bits
        assert again is y and torch.equal(again, got) and torch.equal(gw, gw2)
    else:
        assert gw is None


def test_gradients_against_differences(dslib):
    """The gradients of sum(out * r) with out = combine(gather(x)) by central differences in float64: the operators are
    linear in x and in the weights, so differences are exact but for float32 roundings (sums of 24 terms of size 1)."""
    r = _rng("differences")
    tokens, top_k, experts, cols = 12, 2, 5, 24
    ids = _ids(r, tokens, top_k, experts, "dropped")
    order, want = _order(dslib, ids, experts, 16)
    x, w, c = (r.standard_normal(s) for s in ((tokens, cols), (tokens, top_k), (tokens, cols)))
    dev = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()  # noqa: E731
    x, w, c = (a.astype(np.float32).astype(np.float64) for a in (x, w, c))
    f = lambda x, w: float((X.combine(X.gather(x, want[3], top_k), want[2], w)[0] * c).sum())  # noqa: E731
    y = dslib.expert_gather(dev(x), order)
    dy, dw = dslib.expert_combine_backward(dev(c), y, order, dev(w))
    dx = dslib.expert_combine(dy, order)
    for t, j in ((0, 0), (3, 1), (7, 0), (11, 1)):
        h = np.zeros_like(w)
        h[t, j] = 0.5
        assert abs((f(x, w + h) - f(x, w - h)) - float(dw[t, j])) < 1e-4
    for t, i in ((0, 0), (4, 23), (9, 7)):
        h = np.zeros_like(x)
        h[t, i] = 0.5
        assert abs((f(x + h, w) - f(x - h, w)) - float(dx[t, i])) < 1e-4


# ---------------------------------------------------------------------------------------------------------- products


def _f8(ds, x, tiles=False, fmt="e4m3"):
    """An F8Matrix made by the oracle, the bytes between its rows NaN codes; and its float64 values."""
    q, s = F.quantize(x, tiles, False, fmt)
    rows, cols = q.shape
    kind = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}[fmt]
    held = torch.full((rows, (cols + 15) // 16 * 16), float("nan"), device="cuda").to(kind)
    held[:, :cols] = torch.from_numpy(q.astype(np.float32)).cuda().to(kind)
    return ds.F8Matrix(held[:, :cols], torch.from_numpy(s).cuda(), tiles), F.dequantize(q, s, tiles)


@pytest.mark.parametrize("tokens,top_k,experts,align,kind", [(1, 1, 1, 1, "even"), (1, 2, 6, 1, "even"), (16, 4, 9, 1, "dropped"),
                                                             (200, 2, 5, 1, "even"), (150, 3, 4, 128, "dropped"), (300, 1, 3, 16, "one"),
                                                             (7, 2, 4, 128, "none"), (40, 8, 64, 1, "even")])
@pytest.mark.parametrize("n,k,tiles,xtiles", [(128, 128, True, False), (256, 384, True, False), (640, 200, True, False), (77, 130, False, False),
                                              (300, 512, False, False), (128, 256, True, True)])
@pytest.mark.parametrize("out,bias", [("bf16", False), ("f32", True), ("f16", False)])
def test_linear(dslib, tokens, top_k, experts, align, kind, n, k, tiles, xtiles, out, bias):
    xtiles = xtiles and align % 128 == 0  # the rows of a tile belong to one expert
    r = _rng("linear", tokens, experts, n, k, out)
    order, want = _order(dslib, _ids(r, tokens, top_k, experts, kind), experts, align)
    rows = X.gather(r.standard_normal((tokens, k)), want[3], top_k)
    x, vx = _f8(dslib, rows, xtiles)
    w, vw = _f8(dslib, r.standard_normal((experts * n, k)) * k**-0.5, tiles, "e5m2" if out == "f16" else "e4m3")
    b = torch.from_numpy(r.standard_normal((experts, n)).astype(np.float32)).cuda() if bias else None
    y, size = X.linear(vx, vw.reshape(experts, n, k), want[0], None if b is None else _np(b))
    got = dslib.expert_linear_f8(x, w, order, bias=b, dtype=TYPES[out])
    _near(_np(got), y, HALF[out] * np.abs(y) + TOL * size + TINY[out])
    assert torch.equal(got, dslib.expert_linear_f8(x, w, order, bias=b, dtype=TYPES[out]))  # the same bits again
    for extra in (1, 2, 8):  # rows of every alignment, and nothing written between them
        held = _strided(torch.full_like(got, 3.0), extra)
        dslib.expert_linear_f8(x, w, order, bias=b, out=held)
        assert torch.equal(held, got)
        if held.shape[0] > 1:
            assert bool(torch.isnan(torch.as_strided(held, (held.shape[0] - 1, extra), (n + extra, 1), n)).all())
    assert dslib.lib().ds_f8_fault_flag() == 0


@pytest.mark.parametrize("tokens,top_k,experts,kind", [(1, 1, 1, "even"), (100, 2, 4, "dropped"), (500, 2, 3, "even"), (300, 1, 5, "one"),
                                                       (6, 2, 4, "none"), (700, 4, 2, "even")])
@pytest.mark.parametrize("n,k,tiles", [(128, 128, True), (64, 300, False), (200, 256, True), (257, 131, False), (384, 640, True)])
@pytest.mark.parametrize("added", [False, True])
@pytest.mark.parametrize("align", [128, 256])
def test_weight_grad(dslib, tokens, top_k, experts, kind, n, k, tiles, added, align):
    r = _rng("grad", tokens, experts, n, k)
    order, want = _order(dslib, _ids(r, tokens, top_k, experts, kind), experts, align)
    d = X.gather(r.standard_normal((tokens, n)) * 1e-3, want[3], top_k)
    x = X.gather(r.standard_normal((tokens, k)), want[3], top_k)
    dt, vd = _f8(dslib, np.ascontiguousarray(d.T), False, "e5m2")
    xt, vx = _f8(dslib, np.ascontiguousarray(x.T), tiles)
    add = torch.from_numpy(r.standard_normal((experts, n, k)).astype(np.float32)).cuda() if added else None
    dw, size = X.weight_grad(vd, vx, want[0], None if add is None else _np(add))
    got = dslib.expert_weight_grad_f8(dt, xt, order, add=add)
    _near(_np(got), dw, HALF["f32"] * np.abs(dw) + TOL * size + 1e-38)
    if added:
        assert dslib.expert_weight_grad_f8(dt, xt, order, add=add, out=add) is add and torch.equal(add, got)
    assert dslib.lib().ds_f8_fault_flag() == 0


@pytest.mark.parametrize("n,k,tiles", [(128, 256, True), (130, 256, False), (512, 1024, True)])
def test_one_expert_is_the_dense_product(dslib, n, k, tiles):
    """One expert with all rows: what linear_f8 gives, up to the order of its float32 sums."""
    r = _rng("dense", n, k)
    order, _ = _order(dslib, np.zeros((300, 1), np.int64), 1, 1)
    x, _ = _f8(dslib, r.standard_normal((300, k)))
    w, _ = _f8(dslib, r.standard_normal((n, k)), tiles)
    a = _np(dslib.expert_linear_f8(x, w, order, dtype=torch.float32))
    b = _np(dslib.linear_f8(x, w, dtype=torch.float32))
    terms = np.abs(x.dequantize().cpu().numpy()).astype(np.float64) @ np.abs(w.dequantize().cpu().numpy()).T
    _near(a, b, TOL * terms)


@pytest.mark.parametrize("k,tiles", [(130, False), (256, True), (512, False)])
@pytest.mark.parametrize("kind,align", [("even", 1), ("dropped", 128)])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_linear_of_many_rows(dslib, k, tiles, kind, align, out):
    """More rows than the device has SMs for tiles of half the width: by tiles of the whole width, aligned and not."""
    tokens, top_k, experts, n = 5000, 2, 6, 256
    r = _rng("many", k, kind, out)
    order, want = _order(dslib, _ids(r, tokens, top_k, experts, kind), experts, align)
    rows = r.standard_normal((order.rows, k))
    rows[want[3] < 0] = 0
    x, vx = _f8(dslib, rows)
    w, vw = _f8(dslib, r.standard_normal((experts * n, k)) * k**-0.5, tiles)
    y, size = X.linear(vx, vw.reshape(experts, n, k), want[0])
    got = dslib.expert_linear_f8(x, w, order, dtype=TYPES[out])
    _near(_np(got), y, HALF[out] * np.abs(y) + TOL * size + TINY[out])
    for extra in (1, 2):
        held = _strided(torch.full_like(got, 3.0), extra)
        dslib.expert_linear_f8(x, w, order, out=held)
        # tiles of another width sum in the same order: the same bits
        assert torch.equal(held, got)
    assert dslib.lib().ds_f8_fault_flag() == 0


def test_weight_grad_of_many_tiles(dslib):
    """More tiles than SMs, experts without rows among them, reductions of none to many blocks."""
    tokens, experts, n, k = 1500, 40, 256, 512
    r = _rng("tiles")
    ids = np.minimum(r.geometric(0.12, (tokens, 2)) - 1, experts + 3).astype(np.int64)
    order, want = _order(dslib, ids, experts, 128)
    assert int((order.counts == 0).sum()) > 0
    d = X.gather(r.standard_normal((tokens, n)) * 1e-3, want[3], 2)
    x = X.gather(r.standard_normal((tokens, k)), want[3], 2)
    for tiles in (True, False):
        dt, vd = _f8(dslib, np.ascontiguousarray(d.T))
        xt, vx = _f8(dslib, np.ascontiguousarray(x.T), tiles)
        dw, size = X.weight_grad(vd, vx, want[0])
        got = dslib.expert_weight_grad_f8(dt, xt, order)
        _near(_np(got), dw, HALF["f32"] * np.abs(dw) + TOL * size + 1e-38)
        add = torch.randn(got.shape, device="cuda")
        both = dslib.expert_weight_grad_f8(dt, xt, order, add=add)
        assert torch.equal(both, got + add)  # one rounding more, as the sum of the two

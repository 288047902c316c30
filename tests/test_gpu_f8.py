"""GPU parity of the 8-bit floating-point operators with the float64 oracle.

Tolerances follow from the arithmetic and were fixed before the first run.  Conversions are compared bit for bit (their
definition is a fixed sequence of float32 steps).  Elsewhere a result may be off by its own final rounding (`ulp` of
its type; half a step of an 8-bit value) and by TOL times the sum of the magnitudes of its terms: sums of up to a few
thousand float32 terms in trees or in blocks of 128 (at most 60 roundings of 2^-24 in sequence, 4e-6), exponentials
and quotients within 40 float32 steps (3e-6).
"""
import numpy as np
import pytest
import torch

from oracle import float8_oracle as F

pytestmark = pytest.mark.gpu
TOL = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ULP = {"f32": 2.0**-24, "bf16": 2.0**-8, "f16": 2.0**-10}  # with room for subnormal halves: see _near
FORMATS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


def _rng(*key):
    return np.random.default_rng(sum(ord(c) * (i + 1) for i, c in enumerate(str(key))))


def _dev(a, kind="f32"):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(TYPES[kind])


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _strided(t, extra):
    """The same matrix with rows `extra` elements further apart, its neighbours NaN."""
    held = torch.full((t.shape[0], t.shape[1] + extra), float("nan"), dtype=t.dtype, device=t.device)
    held[:, : t.shape[1]] = t
    return held[:, : t.shape[1]]


def _near(got, want, terms, kind):
    if kind == "f16":  # from half a step above 65504 on, the nearest half is infinite
        over = np.abs(want) >= 65520
        assert np.array_equal(got[over], np.copysign(np.inf, want[over]))
        got, want, terms = got[~over], want[~over], np.broadcast_to(terms, over.shape)[~over]
    err = np.abs(got - want)
    tiny = {"f32": 1e-38, "bf16": 1e-38, "f16": 2.0**-25}[kind]
    bound = ULP[kind] * np.abs(want) + TOL * terms + tiny
    assert np.all(err <= bound), float((err / bound).max())


def _near8(m, want, terms, fmt="e4m3"):
    """An 8-bit result: each scale to TOL of the block's largest term, each value within a rounding."""
    q, s = _np(m.q), _np(m.scale)
    s_want = np.maximum(F.amax(want, m.tiles) / F.MAX[fmt], 2.0**-126)
    s_terms = F.amax(terms, m.tiles) / F.MAX[fmt]
    assert np.all(np.abs(s - s_want) <= TOL * s_terms + 2.0**-126 * TOL)
    each = F.spread(s, *q.shape, m.tiles)
    bound = F.rounding_bound(want, each, fmt) * (1 + TOL) + 2 * TOL * terms
    assert np.all(np.abs(q * each - want) <= bound)


def _as_f8(ds, x, tiles=False, pow2=False, fmt="e4m3", pad_nan=True):
    """An F8Matrix made by the oracle, the bytes between its rows NaN codes; and its float64 values."""
    q, s = F.quantize(x, tiles, pow2, fmt)
    rows, cols = q.shape
    held = torch.full((rows, (cols + 15) // 16 * 16), float("nan"), device="cuda").to(FORMATS[fmt])
    held[:, :cols] = torch.from_numpy(q.astype(np.float32)).cuda().to(FORMATS[fmt])
    return ds.F8Matrix(held[:, :cols], torch.from_numpy(s).cuda(), tiles), F.dequantize(q, s, tiles)


# ------------------------------------------------------------------------------------------------------ conversion

SHAPES = [(1, 1), (1, 128), (3, 129), (127, 7), (128, 128), (130, 260), (257, 385), (1, 4096), (300, 1000)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("blocks,transposed", [("rows", None), ("rows", "rows"), (None, "rows"), ("tiles", "tiles"),
                                               ("tiles", None), ("rows", "tiles")])
def test_quantize_bit_for_bit(dslib, rows, cols, kind, blocks, transposed):
    x = _dev(_rng(rows, cols, kind).standard_normal((rows, cols)) * 3, kind)
    fmt = "e5m2" if (rows + cols) % 3 == 0 else "e4m3"
    pow2 = cols % 2 == 0
    m, t = dslib.quantize_f8(x, blocks, transposed, pow2=pow2, dtype=FORMATS[fmt])
    want = x.float().cpu().numpy()
    for got, v, b in ((m, want, blocks), (t, want.T, transposed)):
        assert (got is None) == (b is None)
        if got is not None:
            q, s = F.quantize(v, b == "tiles", pow2, fmt)
            assert np.array_equal(_np(got.q), q) and np.array_equal(_np(got.scale), s)
    if blocks == "tiles" and transposed == "tiles":
        assert torch.equal(m.q.float().t(), t.q.float()) and torch.equal(m.scale.t(), t.scale)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("extra", [1, 3, 8])
def test_quantize_reads_strided_rows(dslib, kind, extra):
    x = _dev(_rng(kind, extra).standard_normal((140, 270)), kind)
    for blocks, transposed in (("rows", None), ("rows", "rows")):
        a = dslib.quantize_f8(x, blocks, transposed)
        for view in (_strided(x, extra), _strided(torch.cat([x[:, :1], x], 1), 0)[:, 1:]):
            b = dslib.quantize_f8(view, blocks, transposed)
            for m, n in zip(a, b):
                if m is not None:
                    assert torch.equal(m.q.float(), n.q.float()) and torch.equal(m.scale, n.scale)


@pytest.mark.parametrize("blocks,transposed", [("rows", None), ("rows", "rows"), ("tiles", "tiles")])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_quantize_extremes(dslib, blocks, transposed, fmt):
    """Zeros, subnormals, the largest float32, infinities and NaN; a block of nothing finite."""
    x = _rng(fmt).standard_normal((256, 256)).astype(np.float32)
    x[0] = 0
    x[1, :128], x[1, 128:] = 1e-42, -1e-38
    x[2, 5] = 3.4e38
    x[3, 7], x[3, 200], x[4, 9] = np.inf, -np.inf, np.nan
    x[5, :128] = np.nan
    x[6, 128:] = np.inf
    x[140:, 130:] *= 1e-40
    m, t = dslib.quantize_f8(torch.from_numpy(x).cuda(), blocks, transposed, dtype=FORMATS[fmt])
    for got, v, b in ((m, x, blocks), (t, x.T, transposed)):
        if got is not None:
            q, s = F.quantize(v, b == "tiles", False, fmt)
            assert np.array_equal(_np(got.q), q, equal_nan=True) and np.array_equal(_np(got.scale), s)


@pytest.mark.parametrize("rows,cols", [(1, 1), (130, 260), (200, 129), (4, 4096)])
@pytest.mark.parametrize("tiles", [False, True])
@pytest.mark.parametrize("blocks,transposed", [("tiles", None), (None, "rows"), ("rows", "tiles"), ("rows", None)])
def test_requantize_bit_for_bit(dslib, rows, cols, tiles, blocks, transposed):
    x, _ = _as_f8(dslib, _rng(rows, cols).standard_normal((rows, cols)), tiles, fmt="e5m2" if tiles else "e4m3")
    m, t = dslib.quantize_f8(x, blocks, transposed)
    v = x.dequantize().cpu().numpy()  # one float32 product each, as the kernel's
    for got, src, b in ((m, v, blocks), (t, v.T, transposed)):
        if got is not None:
            q, s = F.quantize(src, b == "tiles")
            assert np.array_equal(_np(got.q), q) and np.array_equal(_np(got.scale), s)


def test_power_of_two_scales_change_blocks_without_rounding(dslib):
    """Rows to columns to rows: as long as no value falls below the format's range, nothing changes."""
    x = _dev(_rng("p2").uniform(0.5, 2, (256, 384)))
    m, _ = dslib.quantize_f8(x, "rows", None, pow2=True)
    _, t = dslib.quantize_f8(m, None, "rows", pow2=True)
    assert torch.equal(t.dequantize().t(), m.dequantize())


def test_quantize_past_32_bit_offsets(dslib):
    """More than 2^31 elements: the rows at both ends as if alone."""
    rows, cols = (1 << 18) + 5, 8192 + 128
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda").normal_()
    assert x.numel() > 1 << 31
    m, t = dslib.quantize_f8(x, "rows", "rows")
    alone, _ = dslib.quantize_f8(x[-133:].clone(), "rows")
    assert torch.equal(m.q[-133:].float(), alone.q.float()) and torch.equal(m.scale[-133:], alone.scale)
    last = rows // 128 * 128  # the last block of rows
    _, alone_t = dslib.quantize_f8(x[last:].clone(), None, "rows")
    assert torch.equal(t.q[:, last:].float(), alone_t.q.float()) and torch.equal(t.scale[:, -1:], alone_t.scale)
    del m, t
    m, _ = dslib.quantize_f8(x, "rows")
    assert torch.equal(m.q[-133:].float(), alone.q.float())


# --------------------------------------------------------------------------------------------------------- product

PRODUCTS = [(1, 16, 1), (1, 128, 128), (2, 129, 130), (16, 4096, 512), (17, 1000, 300), (33, 255, 127), (64, 640, 256),
            (65, 130, 384), (128, 512, 128), (129, 257, 129), (300, 1000, 520), (512, 1024, 640), (1000, 384, 1003)]


@pytest.mark.parametrize("M,K,N", PRODUCTS)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tiles_x,tiles_w", [(False, True), (False, False), (True, True)])
def test_product(dslib, M, K, N, kind, tiles_x, tiles_w):
    r = _rng(M, K, N, kind)
    fx, fw = ("e5m2", "e4m3") if kind == "f32" else ("e4m3", "e5m2" if tiles_x else "e4m3")
    x, xv = _as_f8(dslib, r.standard_normal((M, K)) * np.exp(r.standard_normal((M, 1))), tiles_x, fmt=fx)
    w, wv = _as_f8(dslib, r.standard_normal((N, K)) * np.exp(r.standard_normal((N, 1))), tiles_w, fmt=fw)
    bias = r.standard_normal(N).astype(np.float32) if M % 2 else None
    add = r.standard_normal((M, N)).astype(np.float32) if kind == "f32" else None
    y = dslib.linear_f8(x, w, None if bias is None else _dev(bias), None if add is None else _dev(add), dtype=TYPES[kind])
    want, terms = F.linear(xv, wv, bias, add)
    assert y.dtype == TYPES[kind]
    _near(_np(y), want, terms, kind)
    assert dslib.ds_f8_fault_flag() == 0


@pytest.mark.parametrize("M", [1, 40, 300])
def test_product_of_small_integers_is_exact(dslib, M):
    """Integers with scale 1 whose sums fit 24 bits: every step is exact, so is the result."""
    r = _rng("int", M)
    K, N = 700, 260
    x, w = r.integers(-8, 9, (M, K)), r.integers(-8, 9, (N, K))
    put = lambda v: dslib.F8Matrix(_pad16(v), torch.ones((v.shape[0], 6), device="cuda"))
    y = dslib.linear_f8(put(x), put(w), dtype=torch.float32)
    assert np.array_equal(_np(y), (x @ w.T).astype(np.float64))


def _pad16(v):
    held = torch.zeros((v.shape[0], (v.shape[1] + 15) // 16 * 16), device="cuda").to(torch.float8_e4m3fn)
    held[:, : v.shape[1]] = _dev(v).to(torch.float8_e4m3fn)
    return held[:, : v.shape[1]]


@pytest.mark.parametrize("M", [1, 24, 200])
def test_product_empty_reduction_and_empty_sides(dslib, M):
    q = torch.empty((M, 0), device="cuda").to(torch.float8_e4m3fn)
    w = torch.empty((70, 0), device="cuda").to(torch.float8_e4m3fn)
    s = lambda n: torch.empty((n, 0), device="cuda")
    bias, add = _dev(_rng(M).standard_normal(70)), _dev(_rng(M, 1).standard_normal((M, 70)))
    x, w = dslib.F8Matrix(q, s(M)), dslib.F8Matrix(w, s(70))
    assert not dslib.linear_f8(x, w, dtype=torch.float32).any()
    assert torch.equal(dslib.linear_f8(x, w, bias, add, dtype=torch.float32), bias + add)
    full, _ = _as_f8(dslib, _rng("f").standard_normal((5, 256)))
    none, _ = dslib.quantize_f8(torch.empty((0, 256), device="cuda"), "rows")
    assert dslib.linear_f8(none, full).shape == (0, 5) and dslib.linear_f8(full, none).shape == (5, 0)


@pytest.mark.parametrize("M,N", [(1, 300), (20, 129), (200, 515), (600, 700)])
def test_product_writes_strided_rows_in_place_and_nothing_else(dslib, M, N):
    r = _rng(M, N)
    x, xv = _as_f8(dslib, r.standard_normal((M, 300)))
    w, wv = _as_f8(dslib, r.standard_normal((N, 300)), True)
    for kind, extra in (("f32", 5), ("bf16", 1), ("f16", 4)):
        held = torch.full((M + 2, N + extra), 7.0, dtype=TYPES[kind], device="cuda")
        out = held[1:-1, :N]
        add = out if kind == "f32" else None
        dslib.linear_f8(x, w, add=add, out=out)
        want, terms = F.linear(xv, wv, None, np.full((M, N), 7.0) if kind == "f32" else None)
        _near(_np(out), want, terms, kind)
        assert (held[0] == 7).all() and (held[-1] == 7).all() and (held[:, N:] == 7).all()


def test_product_keeps_rows_apart(dslib):
    """NaN, and scales of zero, infinity or NaN in one row of either operand stay in that row of the result."""
    r = _rng("apart")
    for M in (5, 150):
        x, xv = _as_f8(dslib, r.standard_normal((M, 400)))
        w, _ = _as_f8(dslib, r.standard_normal((200, 400)))
        clean = dslib.linear_f8(x, w, dtype=torch.float32)
        x.q[1, 390] = float("nan")
        x.scale[2, 0] = float("nan")
        w.q[130, 0] = float("nan")
        w.scale[199, 3] = float("inf")
        y = dslib.linear_f8(x, w, dtype=torch.float32)
        rows = [i for i in range(M) if i not in (1, 2)]
        cols = [i for i in range(200) if i not in (130, 199)]
        assert torch.equal(y[rows][:, cols], clean[rows][:, cols])
        assert y[1].isnan().all() and y[2].isnan().all() and y[:, 130].isnan().all()
        assert not y[rows][:, 199].isfinite().any()
        x.scale[3] = 0.0
        assert not dslib.linear_f8(x, w, dtype=torch.float32)[3, cols].any()


@pytest.mark.parametrize("M,K,N", [(1, 4096, 4096), (64, 4096, 1024), (2048, 2048, 4096)])
def test_product_repeats_bit_for_bit_on_another_stream(dslib, M, K, N):
    r = torch.Generator(device="cuda").manual_seed(M)
    x, _ = dslib.quantize_f8(torch.randn((M, K), generator=r, device="cuda"))
    w, _ = dslib.quantize_f8(torch.randn((N, K), generator=r, device="cuda"), "tiles")
    first = dslib.linear_f8(x, w, dtype=torch.float32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = [dslib.linear_f8(x, w, dtype=torch.float32) for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(first, y) for y in again)


def test_product_captured_in_a_graph(dslib):
    x, _ = _as_f8(dslib, _rng("g").standard_normal((3, 512)))
    w, _ = _as_f8(dslib, _rng("h").standard_normal((256, 512)), True)
    want = dslib.linear_f8(x, w)
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dslib.linear_f8(x, w, out=out)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_product_large_sampled(dslib):
    """The large layer of the float variant's test, 8192 x 4096 x 4096, on sampled rows."""
    r = torch.Generator(device="cuda").manual_seed(1)
    M, K, N = 8192, 4096, 4096
    x, _ = dslib.quantize_f8(torch.randn((M, K), generator=r, device="cuda"))
    for tiles in ("tiles", "rows"):
        w, _ = dslib.quantize_f8(torch.randn((N, K), generator=r, device="cuda"), tiles)
        y = dslib.linear_f8(x, w, dtype=torch.float32)
        rows = torch.tensor([0, 1, 127, 128, 4095, 8191], device="cuda")
        xv, wv = x.dequantize()[rows].double(), w.dequantize().double()
        want, terms = xv @ wv.t(), xv.abs() @ wv.abs().t()
        assert ((y[rows] - want).abs() <= TOL * terms).all()


def test_product_output_past_32_bit_offsets(dslib):
    """An output of more than 2^31 elements."""
    M, N, K = (1 << 16) + 3, (1 << 15) + 8, 32
    r = torch.Generator(device="cuda").manual_seed(2)
    x, _ = dslib.quantize_f8(torch.randn((M, K), generator=r, device="cuda"))
    w, _ = dslib.quantize_f8(torch.randn((N, K), generator=r, device="cuda"), "tiles")
    y = dslib.linear_f8(x, w)
    assert y.numel() > 1 << 31
    want = x.dequantize()[-4:].double() @ w.dequantize().double().t()
    terms = x.dequantize()[-4:].double().abs() @ w.dequantize().double().abs().t()
    assert ((y[-4:].double() - want).abs() <= ULP["bf16"] * want.abs() + TOL * terms).all()


def test_product_with_shift_weights(dslib):
    """A shift layer's packed weights as 8-bit tiles: exact, and its product that of s * 2^p."""
    r = _rng("shift")
    for N, K in ((130, 300), (1, 1), (256, 1024), (70, 33)):
        s, p = r.integers(-1, 2, (N, K)).astype(np.int8), r.integers(-15, 1, (N, K)).astype(np.int8)
        packed = dslib.pack_shift_weights(torch.from_numpy(s).cuda(), torch.from_numpy(p).cuda())
        w = dslib.expand_shift_weights_f8(packed)
        assert np.array_equal(_np(w.dequantize()), s * np.ldexp(1.0, p.astype(int)))
        x, xv = _as_f8(dslib, r.standard_normal((9, K)))
        want, terms = F.linear(xv, s * np.ldexp(1.0, p.astype(int)))
        _near(_np(dslib.linear_f8(x, w, dtype=torch.float32)), want, terms, "f32")


@pytest.mark.parametrize("M,K,N", [(8, 4096, 512), (1024, 1024, 1024)])
def test_bounded_wait_expiry_is_reported_and_recovered(dslib, M, K, N):
    """With the wait limit cut to one cycle a launch gives up, finishes what it issued and sets the flag; the context
    stays usable and the next call is correct."""
    ds = dslib
    r = torch.Generator(device="cuda").manual_seed(3)
    x, _ = ds.quantize_f8(torch.randn((M, K), generator=r, device="cuda"))
    w, _ = ds.quantize_f8(torch.randn((N, K), generator=r, device="cuda"), "tiles")
    want = ds.linear_f8(x, w)
    assert ds.ds_f8_fault_flag() == 0
    try:
        ds.ds_f8_set_wait_limit(1)
        ds.linear_f8(x, w)
        torch.cuda.synchronize()
    finally:
        ds.ds_f8_set_wait_limit(0)
    assert ds.ds_f8_fault_flag() == 1 and ds.ds_f8_fault_flag() == 0
    assert torch.equal(ds.linear_f8(x, w), want) and ds.ds_f8_fault_flag() == 0


# ------------------------------------------------------------------------------------------------------------ norm

NORMS = [(1, 1), (1, 4096), (3, 7), (5, 129), (4, 2048), (3, 2056), (2, 4104), (7, 8192), (3, 8200), (2, 20001),
         (700, 264)]


@pytest.mark.parametrize("rows,cols", NORMS)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("residual", [False, True])
def test_norm(dslib, rows, cols, kind, residual):
    r = _rng(rows, cols, kind, residual)
    x, res = _dev(r.standard_normal((rows, cols)) * 2, kind), _dev(r.standard_normal((rows, cols)), kind)
    w = _dev(1 + 0.1 * r.standard_normal(cols))
    fmt = "e5m2" if cols % 5 == 0 else "e4m3"
    n, h, rstd = dslib.rmsnorm_f8(x, w, residual=res if residual else None, dtype=FORMATS[fmt])
    hv = _np(x) + (_np(res) if residual else 0)
    want, rs = F.rmsnorm(hv, _np(w), 1e-5)
    assert np.all(np.abs(_np(rstd) - rs) <= TOL * rs)
    _near8(n, want, np.abs(want), fmt)
    if residual:
        _near(_np(h), hv, np.abs(_np(x)) + np.abs(_np(res)), kind)
    else:
        assert h is x


@pytest.mark.parametrize("cols", [264, 4100, 8200])
def test_norm_in_place_strided_and_extremes(dslib, cols):
    """The residual updated in place, rows apart; a row of zeros, one that overflows the mean, one with NaN."""
    r = _rng("np", cols)
    x, res, w = _dev(r.standard_normal((6, cols)), "bf16"), _dev(r.standard_normal((6, cols)), "bf16"), _dev(np.ones(cols))
    n, h, rstd = dslib.rmsnorm_f8(x, w, residual=res)
    for extra in (1, 8):
        xs, rs = _strided(x, extra), _strided(res, extra)
        m, h2, rstd2 = dslib.rmsnorm_f8(xs, w, residual=rs, h=rs)
        assert h2 is rs and torch.equal(rs, h) and torch.equal(rstd, rstd2)
        assert torch.equal(m.q.float(), n.q.float()) and torch.equal(m.scale, n.scale)
        xs = _strided(x, extra)
        _, h3, _ = dslib.rmsnorm_f8(xs, w, residual=_strided(res, extra), h=xs)
        assert h3 is xs and torch.equal(xs, h)
    x[0], res[0] = 0, 0
    x[1] = 3e38
    x[2, 3] = float("nan")
    m, _, rstd2 = dslib.rmsnorm_f8(x, w, residual=res, eps=1e-6)
    assert not m.q[0].float().any() and abs(float(rstd2[0]) - 1e3) < 0.1
    assert float(rstd2[1]) == 0 and m.q[2].float().isnan().all()
    assert torch.equal(m.q[3:].float(), dslib.rmsnorm_f8(x[3:], w, residual=res[3:], eps=1e-6)[0].q.float())


@pytest.mark.parametrize("rows,cols", NORMS)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("with_dh", [False, True])
def test_norm_backward(dslib, rows, cols, kind, with_dh):
    r = _rng(rows, cols, kind, with_dh, "b")
    dy, h, dh = (_dev(r.standard_normal((rows, cols)) * c, kind) for c in (1, 2, 0.5))
    w = _dev(1 + 0.1 * r.standard_normal(cols))
    rstd = (h.float().square().mean(1) + 1e-5).rsqrt()
    dx, dw = dslib.rmsnorm_f8_backward(dy, h, rstd, w, dh=dh if with_dh else None)
    want, want_w, size, size_w = F.rmsnorm_backward(_np(dy), _np(h), _np(rstd), _np(w), _np(dh) if with_dh else None)
    _near(_np(dx), want, size, kind)
    _near(_np(dw), want_w, size_w, "f32")


@pytest.mark.parametrize("cols", [200, 4100, 8200])
def test_norm_backward_in_place_strided_and_repeatable(dslib, cols):
    r = _rng("nb", cols)
    dy, h, dh = (_dev(r.standard_normal((1300, cols)), "bf16") for _ in range(3))
    w, rstd = _dev(1 + 0.1 * r.standard_normal(cols)), (h.float().square().mean(1) + 1e-5).rsqrt()
    dx, dw = dslib.rmsnorm_f8_backward(dy, h, rstd, w, dh=dh)
    for which in range(3):
        a = [_strided(t, 3) for t in (dy, h, dh)]
        dx2, dw2 = dslib.rmsnorm_f8_backward(a[0], a[1], rstd, w, dh=a[2], out=a[which])
        assert dx2 is a[which] and torch.equal(dx2, dx) and torch.equal(dw2, dw)


def test_norm_backward_without_rows(dslib):
    e = torch.empty((0, 300), device="cuda")
    dx, dw = dslib.rmsnorm_f8_backward(e, e, torch.empty(0, device="cuda"), torch.ones(300, device="cuda"))
    assert dx.shape == (0, 300) and dw.shape == (300,) and not dw.any()


def test_norm_gradient_against_differences(dslib):
    """The kernel's gradient against central differences of the float64 norm, in a random direction."""
    r = _rng("diff")
    h, w, dy, d, dwd = (r.standard_normal(s) for s in ((5, 300), 300, (5, 300), (5, 300), 300))
    h, w, dy = (v.astype(np.float32).astype(np.float64) for v in (h, w, dy))
    rstd = F.rmsnorm(h, w, 1e-5)[1]
    dx, dw = dslib.rmsnorm_f8_backward(_dev(dy), _dev(h), _dev(rstd), _dev(w))
    f = lambda e: np.sum(F.rmsnorm(h + e * d, w + e * dwd, 1e-5)[0] * dy)
    slope = (f(1e-4) - f(-1e-4)) / 2e-4
    terms = np.sum(np.abs(_np(dx) * d)) + np.sum(np.abs(_np(dw) * dwd))
    # truncation of the difference is 1e-8 of the terms; the gradient's own tolerance is TOL
    assert abs(np.sum(_np(dx) * d) + np.sum(_np(dw) * dwd) - slope) <= 2 * TOL * terms


# ------------------------------------------------------------------------------------------------------------ gate

GATES = [(1, 1), (1, 8192), (3, 7), (5, 128), (130, 129), (127, 384), (128, 256), (257, 200)]


@pytest.mark.parametrize("rows,features", GATES)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("extra", [0, 3])
def test_gate(dslib, rows, features, kind, extra):
    r = _rng(rows, features, kind)
    gu = _dev(F.halves(3 * r.standard_normal((rows, features)), r.standard_normal((rows, features))), kind)
    up = F.blocks(features) * 128
    if up > features:
        gu[:, features:up] = float("nan")  # not read
    view = _strided(gu, extra)
    a, kept = dslib.gated_f8(view, features)
    g, u = _np(gu)[:, :features], _np(gu)[:, up:]
    want = F.gated(g, u)
    _near8(a, want, np.abs(want))
    q, s = F.quantize(F.halves(g, u))
    assert np.array_equal(_np(kept.q), q) and np.array_equal(_np(kept.scale), s)
    b, none = dslib.gated_f8(view, features, checkpoint=False)
    assert none is None and torch.equal(a.q.float(), b.q.float()) and torch.equal(a.scale, b.scale)


def test_gate_extremes(dslib):
    """Gates far out on both sides (sig = 0 or 1), infinities and NaN."""
    g = np.array([[-200.0, -90, -88, 88, 90, 200, 0, -0.0, 1e-30, -1e-30]], np.float32).repeat(4, 0)
    u = np.ones_like(g)
    u[1, 2], g[2, 4], u[3, 5] = np.inf, np.nan, np.nan
    gu = _dev(F.halves(g, u))
    a, kept = dslib.gated_f8(gu, 10)
    with np.errstate(invalid="ignore", over="ignore"):
        want = F.gated(g.astype(np.float64), u.astype(np.float64))
    got = _np(a.dequantize())
    assert np.array_equal(np.isnan(got), ~np.isfinite(want))
    fine = np.isfinite(want)
    assert np.all(np.abs(got - want)[fine] <= F.rounding_bound(want, _np(a.scale).repeat(10, 1))[fine] + TOL * np.abs(want[fine]))
    d, _, _ = dslib.gated_f8_backward(kept, _dev(np.ones((4, 10))))
    assert _np(d.q)[0].size and not np.isnan(_np(d.q)[0]).any()


@pytest.mark.parametrize("rows,features", GATES)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_gate_backward(dslib, rows, features, kind):
    r = _rng(rows, features, kind, "b")
    fmt = "e5m2" if features % 2 else "e4m3"
    kept, v = _as_f8(dslib, F.halves(3 * r.standard_normal((rows, features)), r.standard_normal((rows, features))))
    da = _dev(r.standard_normal((rows, features)), kind)
    up = F.blocks(features) * 128
    g, u = v[:, :features], v[:, up:]
    dg, du, tg, tu = F.gated_backward(g, u, _np(da))
    want, terms = F.halves(dg, du), F.halves(tg, tu)
    a = F.gated(g, u)
    for extra in (0, 5):
        d, d_t, a_t = dslib.gated_f8_backward(kept, _strided(da, extra), dtype=FORMATS[fmt])
        _near8(d, want, terms, fmt)
        _near8(d_t, want.T, terms.T, fmt)
        _near8(a_t, a.T, np.abs(a.T), fmt)
    only, none, none2 = dslib.gated_f8_backward(kept, da, dtype=FORMATS[fmt], transposed=False)
    assert none is None and none2 is None
    assert torch.equal(only.q.float(), d.q.float()) and torch.equal(only.scale, d.scale)


def test_gate_gradient_against_differences(dslib):
    """The kernel's gradient (a float32 value to half an 8-bit step) against central differences at the checkpoint."""
    r = _rng("gdiff")
    kept, v = _as_f8(dslib, F.halves(2 * r.standard_normal((20, 128)), r.standard_normal((20, 128))))
    da = r.standard_normal((20, 128)).astype(np.float32).astype(np.float64)
    d, _, _ = dslib.gated_f8_backward(kept, _dev(da))
    g, u, e = v[:, :128], v[:, 128:], 1e-5
    slope = np.concatenate([(F.gated(g + e, u) - F.gated(g - e, u)) * da, (F.gated(g, u + e) - F.gated(g, u - e)) * da], 1) / (2 * e)
    each = F.spread(_np(d.scale), 20, 256, False)
    assert np.all(np.abs(_np(d.q) * each - slope) <= F.rounding_bound(slope, each) * (1 + TOL) + 2 * TOL * np.abs(da).max() * 8)


def test_gate_backward_with_the_shortest_wait_limit(dslib):
    """With the wait limit cut to one cycle a launch whose copies are not there yet gives up and sets the flag (one whose
    copies are there need not wait, and is correct); the context stays usable and the next call is correct."""
    ds = dslib
    r = torch.Generator(device="cuda").manual_seed(4)
    kept, _ = ds.quantize_f8(torch.randn((4096, 4096), generator=r, device="cuda"))
    da = torch.randn((4096, 2048), generator=r, device="cuda")
    want = ds.gated_f8_backward(kept, da)
    equal = lambda got: all(torch.equal(m.q.float(), n.q.float()) and torch.equal(m.scale, n.scale) for m, n in zip(got, want))
    assert ds.ds_f8_fault_flag() == 0
    try:
        ds.ds_f8_set_wait_limit(1)
        got = ds.gated_f8_backward(kept, da)
        torch.cuda.synchronize()
    finally:
        ds.ds_f8_set_wait_limit(0)
    assert ds.ds_f8_fault_flag() == 1 or equal(got)
    assert ds.ds_f8_fault_flag() == 0
    assert equal(ds.gated_f8_backward(kept, da)) and ds.ds_f8_fault_flag() == 0


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_gate_backward_many_tiles_by_every_path(dslib, kind):
    """More tiles than SMs, ragged edges; rows of da that TMA can and cannot read, and a tile with an infinity."""
    r = torch.Generator(device="cuda").manual_seed(5)
    rows, features = 2100, 2000
    up = F.blocks(features) * 128
    kept, _ = dslib.quantize_f8(torch.randn((rows, up + features), generator=r, device="cuda"))
    da = torch.randn((rows, features), generator=r, device="cuda").to(TYPES[kind])
    first = dslib.gated_f8_backward(kept, da)
    for extra in (8, 1):
        again = dslib.gated_f8_backward(kept, _strided(da, extra))
        for m, n in zip(first, again):
            assert torch.equal(m.q.float(), n.q.float()) and torch.equal(m.scale, n.scale)
    for sample in (slice(0, 128), slice(1920, 2048), slice(2048, 2100)):  # rows of these blocks as if alone
        part = dslib.F8Matrix(kept.q[sample], kept.scale[sample])
        d, d_t, a_t = dslib.gated_f8_backward(part, da[sample])
        assert torch.equal(d.q.float(), first[0].q[sample].float()) and torch.equal(d.scale, first[0].scale[sample])
        for m, n in zip((d_t, a_t), first[1:]):
            assert torch.equal(m.q.float(), n.q[:, sample].float())
            assert torch.equal(m.scale[:, 0], n.scale[:, sample.start // 128])
    da[1500, 1000] = float("inf")
    d, d_t, _ = dslib.gated_f8_backward(kept, da)
    assert d.q[1500, 1000].isnan() and d_t.q[1000, 1500].isnan() and d.scale.isfinite().all()
    hit = torch.zeros((rows, up + features), dtype=torch.bool, device="cuda")
    hit[1500, 1000] = hit[1500, up + 1000] = True
    same = d.q.float() == first[0].q.float()
    assert (same | hit | (torch.arange(rows, device="cuda")[:, None] == 1500)).all()


def test_gate_without_rows(dslib):
    a, kept = dslib.gated_f8(torch.empty((0, 456), device="cuda"), 200)
    assert a.q.shape == (0, 200) and kept.q.shape == (0, 456)
    d, d_t, a_t = dslib.gated_f8_backward(kept, torch.empty((0, 200), device="cuda"))
    assert d.q.shape == (0, 456) and d_t.q.shape == (456, 0) and a_t.q.shape == (200, 0)
    g = dslib.linear_f8(d_t, dslib.quantize_f8(torch.empty((0, 64), device="cuda"), None, "rows")[1], dtype=torch.float32)
    assert g.shape == (456, 64) and not g.any()


# ----------------------------------------------------------------------------------------------------- guard bands

@pytest.mark.parametrize("rows,cols", [(5, 135), (130, 200)])
def test_outputs_stay_inside_their_rows(dslib, rows, cols):
    """Every 8-bit output inside a larger buffer: bytes between and around its rows keep their value."""
    ds = dslib
    up = F.blocks(cols) * 128 + cols
    held = []

    def out(r, c):
        ld, lds = (c + 15) // 16 * 16 + 16, F.blocks(c) + 3
        q = torch.full(((r + 2) * ld,), 0xA5, dtype=torch.uint8, device="cuda")
        s = torch.full(((r + 2) * lds,), -7.0, device="cuda")
        held.append((q, s, r, c, ld, lds))
        return ds.ds_f8_matrix(q.data_ptr() + ld, s.data_ptr() + 4 * lds, r, c, ld, lds, ds.DS_F8_E4M3, ds.DS_F8_ROWS)

    x, gu = _dev(_rng(1).standard_normal((rows, cols))), _dev(_rng(2).standard_normal((rows, up)))
    w = torch.ones(cols, device="cuda")
    ds.ds_quantize_f8(x, 0, rows, cols, cols, out(rows, cols), out(cols, rows))
    ds.ds_quantize_f8(x, 0, rows, cols, cols, out(rows, cols), None)
    ds.ds_rmsnorm_f8(x, cols, None, 0, w, 0, rows, cols, 1e-5, out(rows, cols), None, 0, None)
    ds.ds_gated_f8(gu, 0, up, rows, cols, out(rows, cols), out(rows, up))
    kept = ds.gated_f8(gu, cols)[1]
    ds.ds_gated_f8_backward(kept.desc, x, 0, cols, cols, out(rows, up), out(up, rows), out(cols, rows))
    torch.cuda.synchronize()
    for q, s, r, c, ld, lds in held:
        q, s = q.view(r + 2, ld), s.view(r + 2, lds)
        assert (q[0] == 0xA5).all() and (q[-1] == 0xA5).all() and (q[1:-1, c:] == 0xA5).all()
        assert (s[0] == -7).all() and (s[-1] == -7).all() and (s[1:-1, F.blocks(c):] == -7).all()
        assert (s[1:-1, :F.blocks(c)] != -7).all()


# ---------------------------------------------------------------------------------------------------- the block

def test_feed_forward_block_against_float64(dslib):
    """Outputs and gradients of the 8-bit block against the float64 block with the same weights.  A value rounded to
    e4m3 is off by at most 2^-4 of itself, 2^-4 / sqrt(3) = 3.6% in the mean; at most six such roundings stand between
    the inputs and a gradient, so its 2-norm is off by sqrt(6) 3.6% = 9%, and the bound is a little more."""
    from paper_1905_13298_gb300.feed_forward import GatedFeedForward
    r = torch.Generator(device="cuda").manual_seed(6)
    T, H, Fe = 384, 256, 200
    b = GatedFeedForward(H, Fe, seed=7)
    x, s, dy, dh = (torch.randn((T, H), generator=r, device="cuda").to(torch.bfloat16) for _ in range(4))
    y, h, saved = b.forward(x, s)
    dx, grads = b.backward(dy, dh, saved)
    xd, sd = (t.double().requires_grad_() for t in (x, s))
    norm = b.norm.double().requires_grad_()
    gate = b.gate_up[:Fe].double().requires_grad_()
    up = b.gate_up[b.up_at:].double().requires_grad_()
    down = b.down.double().requires_grad_()
    hd = xd + sd
    n = hd * (hd.square().mean(1, keepdim=True) + 1e-5).rsqrt() * norm
    yd = (torch.nn.functional.silu(n @ gate.t()) * (n @ up.t())) @ down.t()
    ((yd * dy.double()).sum() + (hd * dh.double()).sum()).backward()
    rel = lambda a, want: float((a.double() - want.detach()).norm() / want.detach().norm())
    assert rel(y, yd) < 0.12 and rel(h, hd) < 2.0**-8
    assert rel(dx, xd.grad) < 0.12
    assert rel(grads["norm"], norm.grad) < 0.12 and rel(grads["down"], down.grad) < 0.12
    assert rel(grads["gate_up"][:Fe], gate.grad) < 0.12 and rel(grads["gate_up"][b.up_at:], up.grad) < 0.12
    assert not grads["gate_up"][Fe : b.up_at].any()
    again = {k: v.clone() for k, v in grads.items()}
    b.backward(dy, dh, saved, again)  # a second micro-batch adds to the sums
    for k, v in again.items():
        assert rel(v, 2 * grads[k].double()) < 1e-6
    t, ht = b.token(x[:3], s[:3])
    assert torch.equal(ht, h[:3]) and rel(t, y[:3].double()) < 2.0**-7  # another kernel, another order of sums


def test_feed_forward_example_learns(dslib, capsys):
    from paper_1905_13298_gb300 import feed_forward
    losses = feed_forward.main(["--tokens", "512", "--hidden", "256", "--features", "384", "--steps", "12", "--shift"])
    assert losses[-1] < 0.9 * losses[0]
    assert "one token" in capsys.readouterr().out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("cols", [136, 1000, 1027, 2056, 4100, 8200])
@pytest.mark.parametrize("first,pad", [(1, 0), (0, 1), (2, 2), (4, 4), (3, 5)])
def test_rows_at_any_address_give_the_same_bits(dslib, dtype, cols, first, pad):
    """Rows that start at any element take other loads and stores, and the same sums and roundings."""
    rows, width = 9, (cols + 127) // 128 * 128 + cols
    g = torch.Generator(device="cuda").manual_seed(cols + first)

    def apart(t):  # the same values, the rows `pad` elements further apart, the first one `first` elements in
        r, c = t.shape
        flat = torch.full((first + r * (c + pad),), float("nan"), dtype=t.dtype, device="cuda")
        view = flat[first:].view(r, c + pad)[:, :c]
        view.copy_(t)
        return view

    x, res, dy, dh = (torch.randn(rows, cols, device="cuda", generator=g).to(dtype) for _ in range(4))
    gu = torch.randn(rows, width, device="cuda", generator=g).to(dtype)
    w = torch.rand(cols, device="cuda", generator=g) + 0.5

    def same(a, b):
        assert torch.equal(a.q.float(), b.q.float()) and torch.equal(a.scale, b.scale)

    for a, b in zip(dslib.quantize_f8(x, "rows", "rows"), dslib.quantize_f8(apart(x), "rows", "rows")):
        same(a, b)
    same(dslib.quantize_f8(x)[0], dslib.quantize_f8(apart(x))[0])
    n, h, rstd = dslib.rmsnorm_f8(x, w, residual=res)
    n2, h2, rstd2 = dslib.rmsnorm_f8(apart(x), w, residual=apart(res), h=apart(torch.zeros_like(x)))
    same(n, n2)
    assert torch.equal(h, h2) and torch.equal(rstd, rstd2)
    dx, dw = dslib.rmsnorm_f8_backward(dy, h, rstd, w, dh=dh)
    dx2, dw2 = dslib.rmsnorm_f8_backward(apart(dy), apart(h), rstd, w, dh=apart(dh), out=apart(torch.zeros_like(dy)))
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
    a, kept = dslib.gated_f8(gu, cols)
    a2, kept2 = dslib.gated_f8(apart(gu), cols)
    same(a, a2), same(kept, kept2)
    for one, two in zip(dslib.gated_f8_backward(kept, dy), dslib.gated_f8_backward(kept, apart(dy))):
        same(one, two)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("low,high", [(1, 1 << 23), (1 << 23, 0x7F7FFFFF), (0x3F000000, 0x40000000), (0x7E000000, 0x7F7FFFFF)])
def test_scales_over_the_range_of_float32(dslib, fmt, low, high):
    """Blocks whose largest magnitude has any bits: the scale and the factor to its units are correctly rounded."""
    rng = _rng(fmt, low)
    amax = rng.integers(low, high, size=(20000, 1)).astype(np.uint32).view(np.float32)
    x = (rng.uniform(-1, 1, (20000, 128)).astype(np.float32) * amax).astype(np.float32)
    x[np.arange(20000), rng.integers(0, 128, 20000)] = amax[:, 0] * rng.choice([-1, 1], 20000).astype(np.float32)
    m, _ = dslib.quantize_f8(torch.from_numpy(x).cuda(), dtype=FORMATS[fmt])
    q, s = F.quantize(x, False, False, fmt)
    assert np.array_equal(_np(m.scale), s) and np.array_equal(_np(m.q), q)


@pytest.mark.parametrize("M,N,K", [(1301, 517, 256), (1300, 518, 256), (2000, 1029, 130), (1100, 1152, 256), (130, 70, 300)])
@pytest.mark.parametrize("pad,first", [(0, 0), (1, 0), (2, 0), (3, 1), (6, 2), (8, 0)])
@pytest.mark.parametrize("tiles", [False, True])
def test_product_into_rows_of_any_alignment_is_exact(dslib, M, N, K, pad, first, tiles):
    """Small integers, whose sums are exact in any order, into rows that start at any element, with bias and add."""
    g = torch.Generator(device="cuda").manual_seed(M + N + pad)
    ints = lambda r, c, n: torch.randint(-n, n + 1, (r, c), device="cuda", generator=g).float()
    x, w, bias, add = ints(M, K, 2), ints(N, K, 2), ints(1, N, 9)[0].contiguous(), ints(M, N, 9)
    want = x.double() @ w.double().t()
    ld = (K + 15) // 16 * 16

    def matrix(v, tiled):
        q = torch.zeros(v.shape[0], ld, device="cuda").to(torch.float8_e4m3fn)
        q[:, :K] = v.to(torch.float8_e4m3fn)
        blocks = (-(-v.shape[0] // 128) if tiled else v.shape[0], -(-K // 128))
        return dslib.F8Matrix(q[:, :K], torch.ones(blocks, device="cuda"), tiles=tiled)

    a, b = matrix(x, False), matrix(w, tiles)
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        for with_bias, with_add in ((False, False), (True, False), (True, True)):
            room = torch.full((first + M * (N + pad),), 77.0, dtype=dtype, device="cuda")
            out = room[first:].view(M, N + pad)[:, :N]
            plus = torch.zeros(first + M * (N + pad), device="cuda")[first:].view(M, N + pad)[:, :N]
            plus.copy_(add)
            y = dslib.linear_f8(a, b, bias=bias if with_bias else None, add=plus if with_add else None, out=out)
            exact = want + (bias if with_bias else 0) + (add if with_add else 0)
            assert torch.equal(y, exact.to(dtype))
            assert bool((room[:first] == 77).all()) and bool((room[first:].view(M, N + pad)[:, N:] == 77).all())

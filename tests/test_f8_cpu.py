"""8-bit floating-point operators without a GPU: the oracle's own pins, and the refusals of the C ABI and the helpers."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import float8_oracle as F

FORMATS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_oracle_codes_are_torchs(fmt):
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    want = codes.view(FORMATS[fmt]).float().numpy().astype(np.float64)
    assert np.array_equal(F.decode_table(fmt), want, equal_nan=True)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_oracle_rounding_is_the_nearest_code(fmt):
    """Against a search over every code, at all codes, all midpoints and their float32 neighbours, and the ends."""
    table = F.decode_table(fmt)
    values = np.unique(table[np.isfinite(table)])
    mid = (values[1:] + values[:-1]) / 2
    near = np.concatenate([np.nextafter(mid.astype(np.float32), np.float32(d)).astype(np.float64) for d in (-1e9, 1e9)])
    u = np.concatenate([values, mid, near, [1e9, -1e9]])
    got = F.round8(u, fmt)
    d = np.abs(got[:, None] - u[:, None])
    best = np.abs(values[None, :] - u[:, None]).min(axis=1)
    assert np.array_equal(d[:, 0], best)
    ties = F.round8(mid, fmt)  # to the code with an even mantissa
    code = np.array([np.flatnonzero(table == v)[0] for v in ties])
    assert not (code & 1).any()
    assert np.isnan(F.round8(np.nan, fmt))


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_oracle_rounding_is_torchs(fmt):
    u = np.random.default_rng(3).standard_normal(20000).astype(np.float32) * np.float32(50)
    assert np.array_equal(F.round8(u, fmt), torch.from_numpy(u).to(FORMATS[fmt]).float().numpy())


@pytest.mark.parametrize("tiles", [False, True])
@pytest.mark.parametrize("pow2", [False, True])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_oracle_conversion_is_within_a_rounding(tiles, pow2, fmt):
    x = np.random.default_rng(4).standard_normal((150, 300)).astype(np.float32)
    q, s = F.quantize(x, tiles, pow2, fmt)
    each = F.spread(s.astype(np.float64), *x.shape, tiles)
    # the unit value carries two float32 roundings before the one to 8 bits
    assert np.all(np.abs(q * each - x) <= F.rounding_bound(x.astype(np.float64), each, fmt) * (1 + 2.0**-20) + 2.0**-22 * np.abs(x))
    if pow2:
        assert np.all(np.frexp(s)[0] == 0.5)


def _differences(f, v, eps=1e-5):
    grad = np.empty_like(v)
    for i in np.ndindex(*v.shape):
        old = v[i]
        v[i] = old + eps
        a = f()
        v[i] = old - eps
        b = f()
        v[i] = old
        grad[i] = (a - b) / (2 * eps)
    return grad


def test_oracle_norm_gradient_against_differences():
    rng = np.random.default_rng(5)
    h, w, dy, dh = (rng.standard_normal(s) for s in ((3, 7), 7, (3, 7), (3, 7)))

    def loss():  # the norm weighed by dy, and the stream by dh
        return np.sum(F.rmsnorm(h, w, 1e-3)[0] * dy) + np.sum(h * dh)

    rstd = F.rmsnorm(h, w, 1e-3)[1]
    dx, dw, _, _ = F.rmsnorm_backward(dy, h, rstd, w, dh)
    # central differences: O(eps^2) truncation and 1e-16 / eps rounding, both below 1e-9
    assert np.allclose(dx, _differences(loss, h), rtol=1e-7, atol=1e-8)
    assert np.allclose(dw, _differences(loss, w), rtol=1e-7, atol=1e-8)


def test_oracle_gate_gradient_against_differences():
    rng = np.random.default_rng(6)
    g, u, da = (3 * rng.standard_normal((4, 5)) for _ in range(3))
    dg, du, _, _ = F.gated_backward(g, u, da)
    assert np.allclose(dg, _differences(lambda: np.sum(F.gated(g, u) * da), g), rtol=1e-7, atol=1e-7)
    assert np.allclose(du, _differences(lambda: np.sum(F.gated(g, u) * da), u), rtol=1e-7, atol=1e-7)


def test_shift_weights_are_exact_e4m3():
    """s * 2^(p + 8) is a code of e4m3 for every shift and sign, so 2^-8 times it is the weight."""
    values = F.decode_table("e4m3")
    for p in range(-15, 1):
        for s in (-1, 0, 1):
            assert s * 2.0 ** (p + 8) in values


# ---------------------------------------------------------------------------------------------- refusals of the ABI

@pytest.fixture(scope="module")
def ds():
    from paper_1905_13298_gb300 import build
    build.build_library()
    import paper_1905_13298_gb300 as ds
    ds.lib()
    return ds


def _m(ds, rows, cols, at=1 << 20, **other):
    """A matrix of fake addresses (never read: every call here is refused)."""
    d = dict(q=at, scale=at + (1 << 30), rows=rows, cols=cols, ld=(cols + 15) // 16 * 16, ld_scale=(cols + 127) // 128,
             format=ds.DS_F8_E4M3, blocks=ds.DS_F8_ROWS)
    d.update(other)
    return ds.ds_f8_matrix(**d)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), "INVALID_ARG"), (dict(scale=None), "INVALID_ARG"), (dict(format=2), "INVALID_ARG"),
    (dict(blocks=-1), "INVALID_ARG"), (dict(q=(1 << 20) + 8), "ALIGNMENT"), (dict(scale=(1 << 30) + 2), "ALIGNMENT"),
    (dict(ld=200), "SHAPE"), (dict(ld=264), "ALIGNMENT"), (dict(ld_scale=1), "SHAPE"), (dict(rows=-1), "SHAPE"),
    (dict(cols=-1), "SHAPE"), (dict(rows=1 << 31), "UNSUPPORTED"), (dict(ld=1 << 40), "UNSUPPORTED"),
    (dict(rows=(1 << 31) - 256, ld=1 << 20), "UNSUPPORTED")])
def test_bad_matrices_are_refused(ds, change, status):
    L, ok, bad = ds.lib(), _m(ds, 4, 256, 1 << 40), _m(ds, **{"rows": 4, "cols": 256, **change})
    want = getattr(ds, "DS_ERR_" + status)
    assert L.ds_linear_f8(bad, ok, None, None, 0, 1 << 50, 0, 4, None) == want
    assert L.ds_linear_f8(ok, bad, None, None, 0, 1 << 50, 0, 1 << 32, None) == want
    assert L.ds_requantize_f8(bad, ok, None, 0, None) == want
    assert L.ds_quantize_f8(1 << 45, 0, 4, 256, 256, bad, None, 0, None) == want
    assert L.ds_rmsnorm_f8(1 << 45, 256, None, 0, 1 << 46, 0, 4, 256, 1e-5, bad, None, 0, None, 0, None) == want
    assert ds.ds_last_error()


def test_bad_products_are_refused(ds):
    L, x, w = ds.lib(), _m(ds, 4, 256, 1 << 40), _m(ds, 8, 256, 1 << 41)

    def call(x=x, w=w, bias=None, add=None, ld_add=8, y=1 << 50, type_=0, ldy=8):
        return L.ds_linear_f8(x, w, bias, add, ld_add, y, type_, ldy, None)

    assert call(x=None) == ds.DS_ERR_INVALID_ARG
    assert call(type_=3) == ds.DS_ERR_INVALID_ARG
    assert call(w=_m(ds, 8, 255, 1 << 41)) == ds.DS_ERR_SHAPE
    assert call(y=None) == ds.DS_ERR_INVALID_ARG
    assert call(ldy=7) == ds.DS_ERR_SHAPE
    assert call(add=1 << 45, ld_add=7) == ds.DS_ERR_SHAPE
    assert call(y=(1 << 50) + 2) == ds.DS_ERR_ALIGNMENT
    assert call(bias=(1 << 45) + 1) == ds.DS_ERR_ALIGNMENT
    assert call(y=1 << 40) == ds.DS_ERR_INVALID_ARG and "overlaps" in ds.ds_last_error()
    assert call(y=1 << 50, add=(1 << 50) + 4) == ds.DS_ERR_INVALID_ARG  # neither apart nor the same
    assert call(y=1 << 50, add=1 << 50, ldy=8, ld_add=9) == ds.DS_ERR_INVALID_ARG
    assert call(y=1 << 50, add=1 << 50, type_=1) == ds.DS_ERR_INVALID_ARG
    big = (1 << 31) - 256
    assert call(x=_m(ds, big, 16, 1 << 40), w=_m(ds, big, 16, 1 << 45), y=1 << 55, ldy=big) == ds.DS_ERR_UNSUPPORTED


def test_bad_conversions_are_refused(ds):
    L, out, out_t = ds.lib(), _m(ds, 4, 256, 1 << 40), _m(ds, 256, 4, 1 << 41)
    x = 1 << 45
    assert L.ds_quantize_f8(x, 0, 4, 256, 256, None, None, 0, None) == ds.DS_ERR_INVALID_ARG
    assert L.ds_quantize_f8(None, 0, 4, 256, 256, out, None, 0, None) == ds.DS_ERR_INVALID_ARG
    assert L.ds_quantize_f8(x, 9, 4, 256, 256, out, None, 0, None) == ds.DS_ERR_INVALID_ARG
    assert L.ds_quantize_f8(x, 0, 4, 256, 256, out, None, 2, None) == ds.DS_ERR_INVALID_ARG
    assert L.ds_quantize_f8(x, 0, 4, 256, 255, out, None, 0, None) == ds.DS_ERR_SHAPE
    assert L.ds_quantize_f8(x, 0, 5, 256, 256, out, None, 0, None) == ds.DS_ERR_SHAPE
    assert L.ds_quantize_f8(x, 0, 4, 256, 256, out, _m(ds, 4, 256, 1 << 41), 0, None) == ds.DS_ERR_SHAPE
    assert L.ds_quantize_f8(x + 2, 0, 4, 256, 256, out, None, 0, None) == ds.DS_ERR_ALIGNMENT
    assert L.ds_quantize_f8(1 << 40, 0, 4, 256, 256, out, None, 0, None) == ds.DS_ERR_INVALID_ARG  # x is out
    assert L.ds_quantize_f8(x, 0, 4, 256, 256, out, _m(ds, 256, 4, 1 << 40), 0, None) == ds.DS_ERR_INVALID_ARG
    assert L.ds_requantize_f8(None, out, out_t, 0, None) == ds.DS_ERR_INVALID_ARG
    assert L.ds_requantize_f8(out, out, None, 0, None) == ds.DS_ERR_INVALID_ARG
    w = ds.ds_weights()
    assert L.ds_expand_shift_weights_f8(w, out, None) == ds.DS_ERR_INVALID_ARG
    w = ds.ds_weights(magic=ds.DS_WEIGHTS_MAGIC, format=ds.DS_FORMAT_PLANES6, n_out=4, k_red=256, n_chunks=8, packed=256,
                      packed_bytes=ds.ds_packed_weight_bytes(4, 256))
    assert L.ds_expand_shift_weights_f8(w, out, None) == ds.DS_ERR_INVALID_ARG  # not tiles
    assert L.ds_expand_shift_weights_f8(w, _m(ds, 5, 256, blocks=1), None) == ds.DS_ERR_SHAPE


def test_bad_norms_are_refused(ds):
    L, out = ds.lib(), _m(ds, 4, 256, 1 << 40)

    def fwd(x=1 << 45, ldx=256, r=None, ldr=256, w=1 << 46, type_=0, rows=4, cols=256, eps=1e-5, out=out, h=None,
            ldh=256, rstd=None, flags=0):
        return L.ds_rmsnorm_f8(x, ldx, r, ldr, w, type_, rows, cols, eps, out, h, ldh, rstd, flags, None)

    assert fwd(x=None) == fwd(w=None) == fwd(out=None) == fwd(eps=-1.0) == fwd(eps=float("nan")) == ds.DS_ERR_INVALID_ARG
    assert fwd(cols=0, out=_m(ds, 4, 0)) == ds.DS_ERR_SHAPE
    assert fwd(ldx=255) == fwd(rows=5) == fwd(r=1 << 47, ldr=1) == fwd(h=1 << 47, ldh=1) == ds.DS_ERR_SHAPE
    assert fwd(w=(1 << 46) + 4) == fwd(rstd=(1 << 47) + 1) == ds.DS_ERR_ALIGNMENT
    assert fwd(out=_m(ds, 4, 256, blocks=ds.DS_F8_TILES)) == ds.DS_ERR_INVALID_ARG
    assert fwd(flags=4) == fwd(type_=-1) == ds.DS_ERR_INVALID_ARG
    assert fwd(h=(1 << 45) + 16) == fwd(h=1 << 45, ldh=257) == ds.DS_ERR_INVALID_ARG  # over x, but not x
    need = ds.ds_rmsnorm_f8_backward_workspace_bytes(4, 256)
    assert need == 4 * 256 * 4 and ds.ds_rmsnorm_f8_backward_workspace_bytes(4, 0) == 0
    assert ds.ds_rmsnorm_f8_backward_workspace_bytes(100000, 10) == (608 * 40 + 255) // 256 * 256

    def bwd(dy=1 << 40, h=1 << 41, rstd=1 << 42, w=1 << 43, dh=None, lddh=256, type_=0, rows=4, cols=256, dx=1 << 44,
            lddx=256, dw=1 << 45, ws=1 << 46, n=need):
        return L.ds_rmsnorm_f8_backward(dy, 256, h, 256, rstd, w, dh, lddh, type_, rows, cols, dx, lddx, dw, ws, n, None)

    for name in ("dy", "h", "rstd", "w", "dx", "dw", "ws"):
        assert bwd(**{name: None}) == ds.DS_ERR_INVALID_ARG, name
    assert bwd(n=need - 1) == ds.DS_ERR_BUFFER_TOO_SMALL
    assert bwd(ws=(1 << 46) + 4) == ds.DS_ERR_ALIGNMENT
    assert bwd(lddx=1) == bwd(dh=1 << 47, lddh=1) == ds.DS_ERR_SHAPE
    assert bwd(dx=1 << 40, lddx=257) == bwd(dx=(1 << 41) + 4) == bwd(dw=1 << 42) == ds.DS_ERR_INVALID_ARG


def test_bad_gates_are_refused(ds):
    L, out, kept = ds.lib(), _m(ds, 4, 200, 1 << 40), _m(ds, 4, 456, 1 << 41)

    def fwd(gu=1 << 45, type_=0, ld=456, rows=4, features=200, out=out, ckpt=kept, flags=0):
        return L.ds_gated_f8(gu, type_, ld, rows, features, out, ckpt, flags, None)

    assert fwd(gu=None) == fwd(out=None) == fwd(type_=5) == fwd(flags=8) == ds.DS_ERR_INVALID_ARG
    assert fwd(ld=455) == fwd(features=0) == fwd(features=199) == fwd(ckpt=_m(ds, 4, 400, 1 << 41)) == ds.DS_ERR_SHAPE
    assert fwd(gu=1 << 40) == fwd(ckpt=_m(ds, 4, 456, 1 << 40)) == ds.DS_ERR_INVALID_ARG

    def bwd(ckpt=kept, da=1 << 45, ld=200, features=200, dgu=_m(ds, 4, 456, 1 << 46), dgu_t=None, a_t=None, flags=0):
        return L.ds_gated_f8_backward(ckpt, da, 0, ld, features, dgu, dgu_t, a_t, flags, None)

    assert bwd(ckpt=None) == bwd(da=None) == bwd(dgu=None) == bwd(flags=2) == ds.DS_ERR_INVALID_ARG
    assert bwd(features=201) == bwd(ld=199) == bwd(dgu_t=_m(ds, 4, 456, 1 << 47)) == ds.DS_ERR_SHAPE
    assert bwd(a_t=_m(ds, 200, 5, 1 << 47)) == ds.DS_ERR_SHAPE
    assert bwd(dgu=_m(ds, 4, 456, 1 << 41)) == ds.DS_ERR_INVALID_ARG


def test_no_tokens_need_no_memory(ds):
    """Zero rows launch nothing (there is no GPU here) and succeed, with or without pointers."""
    L = ds.lib()
    none = dict(q=None, scale=None)
    assert L.ds_quantize_f8(None, 1, 0, 256, 256, _m(ds, 0, 256, **none), _m(ds, 256, 0, **none), 0, None) == ds.DS_OK
    assert L.ds_requantize_f8(_m(ds, 0, 256, **none), _m(ds, 0, 256, **none), None, 0, None) == ds.DS_OK
    assert L.ds_linear_f8(_m(ds, 0, 256, **none), _m(ds, 8, 256), None, None, 0, None, 1, 8, None) == ds.DS_OK
    assert L.ds_rmsnorm_f8(None, 256, None, 0, 256, 1, 0, 256, 1e-5, _m(ds, 0, 256, **none), None, 0, None, 0, None) == ds.DS_OK
    assert L.ds_gated_f8(None, 1, 456, 0, 200, _m(ds, 0, 200, **none), None, 0, None) == ds.DS_OK
    assert L.ds_gated_f8_backward(_m(ds, 0, 456, **none), None, 1, 200, 200, _m(ds, 0, 456, **none), None, None, 0, None) == ds.DS_OK


def test_struct_layout(ds):
    assert ds.lib().ds_abi_struct_size(2) == ctypes.sizeof(ds.ds_f8_matrix) == 56


def test_helpers_refuse_what_the_abi_cannot_see(ds):
    q, s = torch.zeros(4, 256).to(torch.float8_e4m3fn), torch.ones(4, 2)
    for bad in ((q.float(), s), (q, s.double()), (q, s[:, :1]), (q[0], s), (q.t(), s), (q[:, :200], s), (q, s)):
        with pytest.raises(ValueError):
            ds.F8Matrix(*bad)  # the last one is not on a GPU
    with pytest.raises(ValueError):
        ds.quantize_f8(torch.zeros(4, 256, dtype=torch.int32))
    with pytest.raises(ValueError):
        ds.quantize_f8(torch.zeros(4, 256), "columns")
    with pytest.raises(ValueError):
        ds.quantize_f8(torch.zeros(4, 256), None, None)
    with pytest.raises(ValueError):
        ds.quantize_f8(torch.zeros(4, 256))  # not on a GPU
    with pytest.raises(ValueError):
        ds.linear_f8(q, q)
    with pytest.raises(ValueError):
        ds.rmsnorm_f8(torch.zeros(4, 256), torch.zeros(255))
    with pytest.raises(ValueError):
        ds.rmsnorm_f8(torch.zeros(4, 256), torch.zeros(256), residual=torch.zeros(4, 256, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        ds.gated_f8(torch.zeros(4, 400), 200)
    with pytest.raises(ValueError):
        ds.rmsnorm_f8_backward(torch.zeros(4, 256), torch.zeros(4, 255), torch.zeros(4), torch.zeros(256))


def test_outputs_of_one_call_have_one_format(ds):
    L, x = ds.lib(), 1 << 45
    a, b = _m(ds, 4, 256, 1 << 40), _m(ds, 256, 4, 1 << 41, format=ds.DS_F8_E5M2)
    assert L.ds_quantize_f8(x, 0, 4, 256, 256, a, b, 0, None) == ds.DS_ERR_INVALID_ARG and "format" in ds.ds_last_error()
    assert L.ds_requantize_f8(_m(ds, 4, 256, 1 << 42), a, b, 0, None) == ds.DS_ERR_INVALID_ARG
    out, kept = _m(ds, 4, 200, 1 << 40), _m(ds, 4, 456, 1 << 41, format=ds.DS_F8_E5M2)
    assert L.ds_gated_f8(x, 0, 456, 4, 200, out, kept, 0, None) == ds.DS_ERR_INVALID_ARG
    d, d_t = _m(ds, 4, 456, 1 << 46), _m(ds, 456, 4, 1 << 47, format=ds.DS_F8_E5M2)
    assert L.ds_gated_f8_backward(kept, x, 0, 200, 200, d, d_t, None, 0, None) == ds.DS_ERR_INVALID_ARG


def test_refusals_of_alignment_name_the_bytes(ds):
    L, out = ds.lib(), _m(ds, 4, 256, 1 << 40)
    fwd = lambda x=1 << 45, w=1 << 46, type_=0: L.ds_rmsnorm_f8(x, 256, None, 0, w, type_, 4, 256, 1e-5, out, None, 0, None, 0, None)
    for call, what in ((lambda: fwd(w=(1 << 46) + 4), "weight must be 16-byte aligned"),
                       (lambda: fwd(x=(1 << 45) + 2), "x must be 4-byte aligned"),
                       (lambda: fwd(x=(1 << 45) + 1, type_=1), "x must be 2-byte aligned")):
        assert call() == ds.DS_ERR_ALIGNMENT and ds.ds_last_error() == what


def test_tile_of_refused_and_empty_products_is_zero(ds):
    L, x, w = ds.lib(), _m(ds, 4, 256, 1 << 40), _m(ds, 8, 256, 1 << 41)
    assert L.ds_linear_f8_tile(x, _m(ds, 8, 255, 1 << 41), None, 0, 1 << 50, 0, 8) == 0 and ds.ds_last_error()
    assert L.ds_linear_f8_tile(None, w, None, 0, 1 << 50, 0, 8) == 0
    assert L.ds_linear_f8_tile(_m(ds, 0, 256), w, None, 0, 1 << 50, 0, 8) == 0 and not ds.ds_last_error()


@pytest.mark.parametrize("what", ["--tokens", "--hidden", "--features", "--steps"])
def test_feed_forward_example_refuses_empty_sizes(what, capsys):
    from paper_1905_13298_gb300 import feed_forward
    with pytest.raises(SystemExit):
        feed_forward.main([what, "0"])
    assert "must be at least 1" in capsys.readouterr().err

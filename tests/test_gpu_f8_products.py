"""Products of 8-bit matrices: scales at the ends of float32, and every instance of the large kernel on exact integers."""
import numpy as np
import pytest
import torch

from oracle import float8_oracle as F
from test_gpu_f8 import FORMATS, TOL, _np, _rng

pytestmark = pytest.mark.gpu

# (scale of x, scale of w, exponent range of the 8-bit values): no block's sum leaves the normal numbers of float32 when
# it is multiplied by one of the scales, whichever that is, nor does the result
ENDS = [(2.0**-120 * 1.37, 2.0**-24 * 1.61, (-2, 8), "e4m3"),   # the scales' product has a few bits
        (2.0**-118 * 1.37, 2.0**-34 * 1.61, (13, 15), "e5m2"),  # ... none
        (2.0**100 * 1.37, 2.0**40 * 1.61, (-14, -12), "e5m2"),  # ... overflows
        (2.0**-63 * 1.37, 2.0**63 * 1.61, (-2, 8), "e4m3")]


@pytest.mark.parametrize("sx,sw,exponents,fmt", ENDS)
@pytest.mark.parametrize("M,K,N", [(5, 300, 260), (1100, 300, 1152), (1100, 300, 1151), (2500, 300, 3800)])
@pytest.mark.parametrize("tiles", [False, True])
def test_product_with_scales_at_the_ends_of_float32(dslib, sx, sw, exponents, fmt, M, K, N, tiles):
    """A block's sum times its two scales, one after the other: as near to float64 as with scales near one, in every
    kernel; zeros stay zeros."""
    r = _rng(sx, sw, M, N)

    def matrix(rows, scale, tiled):
        v = np.ldexp(r.choice([1, 1.25, 1.5, 1.75], (rows, K)), r.integers(*exponents, (rows, K))) * r.choice([-1, 1], (rows, K))
        v[rows // 2] = 0
        q = torch.zeros((rows, 304), device="cuda").to(FORMATS[fmt])
        q[:, :K] = torch.from_numpy(v.astype(np.float32)).cuda().to(FORMATS[fmt])
        s = torch.full((-(-rows // 128) if tiled else rows, 3), scale, device="cuda")
        s *= torch.from_numpy(r.uniform(0.9, 1.1, s.shape).astype(np.float32)).cuda()
        return dslib.F8Matrix(q[:, :K], s, tiles=tiled)

    def exact(m):
        s = m.scale.double().repeat_interleave(128, 1)[:, :K]
        return m.q.double() * (s.repeat_interleave(128, 0)[: m.rows] if m.tiles else s)

    x, w = matrix(M, sx, False), matrix(N, sw, tiles)
    y = dslib.linear_f8(x, w, dtype=torch.float32)
    want, terms = exact(x) @ exact(w).t(), exact(x).abs() @ exact(w).abs().t()
    assert float(terms.max()) > 2.0**-124 and float(terms.max()) < 2.0**127
    assert bool(((y.double() - want).abs() <= 2.0**-24 * want.abs() + TOL * terms + 2.0**-148).all())
    assert not y[M // 2].any() and not y[:, N // 2].any()


def _tile(ds, x, w, y, add=None):
    kinds = {torch.float32: ds.DS_TYPE_F32, torch.bfloat16: ds.DS_TYPE_BF16, torch.float16: ds.DS_TYPE_F16}
    return ds.ds_linear_f8_tile(x.desc, w.desc, add, 0 if add is None else add.stride(0), y, kinds[y.dtype], y.stride(0))


@pytest.mark.parametrize("M,N,tile", [(2500, 3800, 256), (2500, 3801, 256), (2100, 2104, 128), (2100, 2103, 128)])
@pytest.mark.parametrize("tiles_w", [False, True])
@pytest.mark.parametrize("fx", ["e4m3", "e5m2"])
@pytest.mark.parametrize("fw", ["e4m3", "e5m2"])
def test_large_products_of_small_integers_are_exact(dslib, M, N, tile, tiles_w, fx, fw):
    """Every instance of the large kernel (width of a tile, scales of w, rows that are aligned or not) and every pair of
    formats, over more tiles than SMs, 18 blocks of the reduction and ragged sides, with a bias, and accumulating in
    place: integers times scales that are powers of two, whose sums fit 24 bits, so that every step is exact."""
    K, r = 2200, torch.Generator(device="cuda").manual_seed(M + N)
    tiles_x = (fx == fw) != tiles_w

    def matrix(rows, fmt, tiled):
        q = torch.zeros((rows, 2208), device="cuda").to(FORMATS[fmt])
        q[:, :K] = torch.randint(-2, 3, (rows, K), generator=r, device="cuda").float().to(FORMATS[fmt])
        s = torch.randint(-2, 3, (-(-rows // 128) if tiled else rows, 18), generator=r, device="cuda")
        return dslib.F8Matrix(q[:, :K], torch.exp2(s.float()), tiles=tiled)

    x, w = matrix(M, fx, tiles_x), matrix(N, fw, tiles_w)
    assert -(-M // 128) * -(-N // tile) > torch.cuda.get_device_properties(0).multi_processor_count
    bias = torch.randint(-9, 10, (N,), generator=r, device="cuda").float()
    want = x.dequantize().double() @ w.dequantize().double().t()
    for dtype in (torch.bfloat16, torch.float16):
        y = torch.empty((M, N), dtype=dtype, device="cuda")
        assert _tile(dslib, x, w, y) == tile
        dslib.linear_f8(x, w, bias=bias if dtype == torch.bfloat16 else None, out=y)
        assert torch.equal(y, (want + bias if dtype == torch.bfloat16 else want).to(dtype))
    held = torch.randint(-9, 10, (M, N + 8), generator=r, device="cuda").float()
    before, sums = held.clone(), held[:, :N]
    assert _tile(dslib, x, w, sums, sums) == tile
    dslib.linear_f8(x, w, bias=bias, add=sums, out=sums)
    assert torch.equal(sums.double(), want + bias + before[:, :N]) and torch.equal(held[:, N:], before[:, N:])
    assert dslib.ds_f8_fault_flag() == 0


def test_sizes_at_the_ends_reach_every_kernel(dslib):
    """The sizes of the test with scales at the ends of float32: the small kernel, and both widths of the large one."""
    def tile(M, N, tiles):
        x, w = dslib.F8Matrix.empty(M, 300, "cuda"), dslib.F8Matrix.empty(N, 300, "cuda", tiles=tiles)
        return _tile(dslib, x, w, torch.empty((M, N), device="cuda"))

    for tiles in (False, True):
        assert tile(5, 260, tiles) == 16
        assert tile(1100, 1152, tiles) == 128 and tile(1100, 1151, tiles) == 128
        assert tile(2500, 3800, tiles) == 256

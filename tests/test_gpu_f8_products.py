"""Products of 8-bit matrices whose scales lie at the ends of float32."""
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

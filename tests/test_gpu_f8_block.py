"""The 8-bit gate against float32 arithmetic."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("low,high", [(-4.0, 4.0), (-80.0, 0.0)])
def test_gate_is_as_exact_as_the_formula_in_float32(dslib, low, high):
    """One value per block, so that the scale shows it in float32: the error of silu(g) in the mean square is that of
    g * (1 / (1 + exp(-g))) in float32 operations (3% for another order of roundings; 2^18 samples give 0.2%)."""
    rows, blocks = 4096, 64
    r = torch.Generator(device="cuda").manual_seed(8)
    g = torch.rand((rows, blocks), generator=r, device="cuda") * (high - low) + low
    gu = torch.zeros((rows, 2 * 128 * blocks), device="cuda")
    gu[:, 0 : 128 * blocks : 128] = g
    gu[:, 128 * blocks :: 128] = 1
    a, kept = dslib.gated_f8(gu, 128 * blocks)
    want = (g.double() * torch.sigmoid(g.double())).abs() / 448
    plain = (g * (1 / (1 + torch.exp(-g)))).abs() / 448
    big = want > 2.0**-100  # what the scale of a block can hold
    rms = lambda got: float(((got.double() - want) / want)[big].square().mean().sqrt())
    assert float(big.float().mean()) > 0.8
    assert rms(a.scale) <= 1.03 * rms(plain)

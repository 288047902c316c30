"""The 8-bit gate against float32 arithmetic, and what the feed-forward block built from the operators promises."""
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


def test_block_rounds_the_norm_once(dslib, monkeypatch):
    """The operand of the weight gradient holds the values of the forward pass, turned: changing the blocks of the norm's
    output rounds nothing but values below the format's range."""
    from paper_1905_13298_gb300 import feed_forward
    seen = []

    def watch(x, *args, **kw):
        got = quantize(x, *args, **kw)
        if isinstance(x, dslib.F8Matrix):
            seen.append((x, got[1]))
        return got

    quantize = feed_forward.quantize_f8
    r = torch.Generator(device="cuda").manual_seed(9)
    T, H, Fe = 300, 264, 200
    b = feed_forward.GatedFeedForward(H, Fe, seed=7)
    monkeypatch.setattr(feed_forward, "quantize_f8", watch)
    x, s, dy, dh = (torch.randn((T, H), generator=r, device="cuda").to(torch.bfloat16) for _ in range(4))
    y, h, saved = b.forward(x, s)
    b.backward(dy, dh, saved)
    (n, n_t), = seen
    v, v_t = n.dequantize(), n_t.dequantize().t()
    # the smallest normal number of e4m3 in a tile's units
    least = 2.0**-6 * n_t.scale.repeat_interleave(128, 0)[:H].repeat_interleave(128, 1)[:, :T].t()
    assert bool((v.abs() >= least).float().mean() > 0.9)
    assert bool(((v == v_t) | (v.abs() < least)).all())


def test_block_with_shift_weights_has_their_gradients(dslib):
    """After use_shift_weights the transposes are those of the shift weights, exactly, and so is the input's gradient."""
    from paper_1905_13298_gb300.feed_forward import GatedFeedForward
    T, H, Fe = 256, 256, 200
    b = GatedFeedForward(H, Fe, seed=7)
    b.use_shift_weights()
    for m, m_t in ((b.w_gate_up, b.w_gate_up_t), (b.w_down, b.w_down_t)):
        assert torch.equal(m.dequantize().t(), m_t.dequantize())
    r = torch.Generator(device="cuda").manual_seed(6)
    x, s, dy, dh = (torch.randn((T, H), generator=r, device="cuda").to(torch.bfloat16) for _ in range(4))
    y, h, saved = b.forward(x, s)
    dx, _ = b.backward(dy, dh, saved)
    xd, sd = (t.double().requires_grad_() for t in (x, s))
    w, down = b.w_gate_up.dequantize().double(), b.w_down.dequantize().double()
    hd = xd + sd
    n = hd * (hd.square().mean(1, keepdim=True) + 1e-5).rsqrt()
    yd = (torch.nn.functional.silu(n @ w[:Fe].t()) * (n @ w[b.up_at :].t())) @ down.t()
    ((yd * dy.double()).sum() + (hd * dh.double()).sum()).backward()
    # weights are exact: at most five roundings to e4m3 of 3.6% each, sqrt(5) 3.6% = 8%
    assert float((dx.double() - xd.grad).norm() / xd.grad.norm()) < 0.09

"""The feed-forward block with experts: its operators together, as a training step and a serving step run them, against
float64; the optimizer on its weights; its command."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _block(seed=3, hidden=256, features=128, experts=5, top_k=2):
    from paper_1905_13298_gb300.feed_forward import ExpertsFeedForward
    return ExpertsFeedForward(hidden, features, experts, top_k, seed=seed)


def _inputs(seed, tokens=300, hidden=256):
    r = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn((tokens, hidden), generator=r, device="cuda").to(torch.bfloat16) for _ in range(4)]


def _exact(b, x, s, dy, dh, ids, padding):
    """y and all gradients in float64 with the 8-bit weights' values and the choices of the run."""
    E, Fe, H = b.experts, b.features, b.hidden
    xd, sd = (t.double().requires_grad_() for t in (x, s))
    w_r = b.w_router.dequantize().double().requires_grad_()
    w_gu = b.w_gate_up.dequantize().double().view(E, 2 * Fe, H).requires_grad_()
    w_d = b.w_down.dequantize().double().view(E, H, Fe).requires_grad_()
    norm = b.norm.double().requires_grad_()
    h = xd + sd
    n = h * (h.square().mean(1, keepdim=True) + 1e-5).rsqrt() * norm
    weights = torch.softmax((n @ w_r.t()).gather(1, ids.clamp(min=0)), 1)
    gu = torch.einsum("th,enh->ten", n, w_gu)
    a = torch.nn.functional.silu(gu[..., :Fe]) * gu[..., Fe:]
    each = torch.einsum("tef,ehf->teh", a, w_d).gather(1, ids.clamp(min=0)[..., None].expand(-1, -1, H))
    y = torch.where((ids >= 0)[..., None], each * weights[..., None], 0.0).sum(1)
    ((y * dy.double()).sum() + (h * dh.double()).sum()).backward()
    return y.detach(), xd.grad, {"norm": norm.grad, "router": w_r.grad, "gate_up": w_gu.grad, "down": w_d.grad}


def _off(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("padded", [False, True])
def test_training_step_against_float64(dslib, padded):
    """With the run's own choices of experts.  A rounding to e4m3 is off by 3.6% in the mean square (half a step is 2^-4
    of a value at most, uniform over it): y has two (n, a), a gradient at most seven in a chain (n twice, the kept g and
    u, a, and its own three: dy's, dgu's, the logits'), sqrt(7) 3.6% = 9.6%, each within 1.25 for sums of 128 features."""
    b, (x, s, dy, dh) = _block(), _inputs(5)
    padding = torch.arange(300, device="cuda") >= 280 if padded else None
    y, h, saved = b.forward(x, s, padding)
    dx, grads = b.backward(dy, dh, saved)
    ids = saved[3]
    want_y, want_dx, want = _exact(b, x, s, dy, dh, ids, padding)
    assert _off(y, want_y) < 0.0636  # sqrt(2) 3.6% 1.25
    assert _off(dx, want_dx) < 0.12
    for k, g in grads.items():
        assert g.shape == want[k].shape and _off(g, want[k]) < 0.12, (k, _off(g, want[k]))
    if padded:
        assert bool((y[280:] == 0).all())
    again = {k: v.clone() for k, v in grads.items()}
    b.backward(dy, dh, saved, again)  # accumulates in place
    for k, g in again.items():
        assert torch.allclose(g, 2 * grads[k], rtol=1e-5, atol=1e-5 * float(grads[k].abs().max()))
    assert dslib.lib().ds_f8_fault_flag() == 0


def test_shift_weights_have_their_gradients(dslib):
    """The experts' weights are s * 2^p exactly, transposes too; y and gradients are theirs, within the roundings counted
    above without those of the weights (there are none)."""
    b, (x, s, dy, dh) = _block(), _inputs(7)
    b.use_shift_weights()
    for w, m, m_t in ((b.gate_up, b.w_gate_up, b.w_gate_up_t), (b.down, b.w_down, b.w_down_t)):
        sign, power = dslib.quantize_shift_weights(w)
        assert torch.equal(m.dequantize().view(w.shape), sign.float() * torch.exp2(power.float()))
        assert torch.equal(m_t.dequantize().view(w.shape[0], w.shape[2], w.shape[1]), m.dequantize().view(w.shape).transpose(1, 2))
    y, h, saved = b.forward(x, s)
    dx, grads = b.backward(dy, dh, saved)
    want_y, want_dx, want = _exact(b, x, s, dy, dh, saved[3], None)
    assert _off(y, want_y) < 0.0636 and _off(dx, want_dx) < 0.12
    for k, g in grads.items():
        assert _off(g, want[k]) < 0.12, (k, _off(g, want[k]))
    t, _ = b.token(x[:7], s[:7])
    assert _off(t, y[:7].double()) < 0.02
    b.refresh()  # back to the rounded float weights
    assert not torch.equal(b.w_down.dequantize(), dslib.expand_shift_weights_f8(
        dslib.pack_shift_weights(*dslib.quantize_shift_weights(b.down.flatten(0, 1)))).dequantize())


def test_token_is_the_forward_pass(dslib):
    """Without gaps between segments and without a checkpoint: y within a bf16 step and the products' order of sums."""
    b, (x, s, _, _) = _block(), _inputs(6)
    y, h, _ = b.forward(x, s)
    t, ht = b.token(x[:7], s[:7])
    assert torch.equal(ht, h[:7]) and _off(t, y[:7].double()) < 0.02
    one, _ = b.token(x[3:4], s[3:4])
    assert _off(one, y[3:4].double()) < 0.02


def test_captured_step_with_other_choices(dslib):
    """A training step with its optimizer step, captured, and replayed on inputs whose tokens choose other experts: the
    bits of the calls."""
    b, ref = _block(), _block()
    held = _inputs(1)

    def make(block):
        y, h, saved = block.forward(*held[:2])
        _, grads = block.backward(*held[2:], saved)
        steps = torch.zeros((), dtype=torch.int64, device="cuda")
        return block.adamw({k: v.clone() for k, v in grads.items()}, steps=steps, state_dtype=torch.float8_e4m3fn, lr=1e-2)

    opt, opt_ref = make(b), make(ref)

    def step(block, optimizer):
        y, _, saved = block.forward(*held[:2])
        dx, grads = block.backward(*held[2:], saved)
        for a, k in zip(optimizer.grads, block.masters()):
            a.copy_(grads[k])
        optimizer.step()
        return y, dx

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(b, opt)
    torch.cuda.current_stream().wait_stream(side)
    step(ref, opt_ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(b, opt)
    for seed in (2, 3):
        for a, new in zip(held, _inputs(seed)):
            a.copy_(new)
        graph.replay()
        want = step(ref, opt_ref)
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
        for p, q in zip(opt.params, opt_ref.params):
            assert torch.equal(p, q)
    assert int(opt.steps) == 3


@pytest.mark.parametrize("extra", [[], ["--adamw", "8", "--rate", "0.01"], ["--adamw", "32", "--rate", "0.01"]])
@pytest.mark.parametrize("experts", [[], ["--experts", "6", "--top-k", "2"]])
def test_command_trains(dslib, extra, experts):
    from paper_1905_13298_gb300.feed_forward import main
    losses = main(["--tokens", "512", "--hidden", "256", "--features", "256", "--steps", "4", *extra, *experts])
    assert len(losses) == 4 and all(l == l and l < float("inf") for l in losses)


def test_command_refuses(dslib):
    from paper_1905_13298_gb300.feed_forward import ExpertsFeedForward, main
    for bad in (["--experts", "4", "--top-k", "5"], ["--experts", "4", "--features", "200"], ["--experts", "4", "--shift"]):
        with pytest.raises(SystemExit):
            main(bad)
    with pytest.raises(ValueError):
        ExpertsFeedForward(256, 200, 4, 2)
    with pytest.raises(ValueError):
        ExpertsFeedForward(256, 128, 4, 5)

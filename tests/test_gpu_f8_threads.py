"""The 8-bit operators from several host threads at once, and captured in a CUDA graph (in which a call that allocated
device memory or synchronised would fail)."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


def _inputs(seed, T=300, H=264, Fe=200):
    r = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn((T, H), generator=r, device="cuda").to(torch.bfloat16) for _ in range(4)]


def _step(block, x, s, dy, dh):
    """Every operator but the conversion of shift weights: (y, h, dx, gradients)."""
    y, h, saved = block.forward(x, s)
    dx, grads = block.backward(dy, dh, saved)
    t, _ = block.token(x[:3], s[:3])
    return [y, h, dx, t] + [grads[k] for k in ("norm", "gate_up", "down")]


def test_four_host_threads(dslib):
    """Each on its own stream with its own inputs: the bits of a thread alone."""
    from paper_1905_13298_gb300.feed_forward import GatedFeedForward
    block = GatedFeedForward(264, 200, seed=3)
    alone = {seed: [t.clone() for t in _step(block, *_inputs(seed))] for seed in range(4)}
    torch.cuda.synchronize()
    got, errors = {}, []

    def work(seed):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(5):
                    got[seed] = _step(block, *_inputs(seed))
            stream.synchronize()
        except Exception as e:  # reported by the main thread
            errors.append(e)

    threads = [threading.Thread(target=work, args=(seed,)) for seed in alone]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for seed, want in alone.items():
        assert all(torch.equal(a, b) for a, b in zip(got[seed], want)), seed
    assert dslib.ds_f8_fault_flag() == 0


def test_calls_captured_in_a_graph(dslib):
    """A training step, a token and the conversion of shift weights: replayed on new inputs, the bits of the calls."""
    from paper_1905_13298_gb300.feed_forward import GatedFeedForward
    block = GatedFeedForward(264, 200, seed=3)
    packed = dslib.pack_shift_weights(*dslib.quantize_shift_weights(block.down))
    held = _inputs(1)
    side = torch.cuda.Stream()  # as torch asks for: once outside the capture, on another stream
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(block, *held), dslib.expand_shift_weights_f8(packed)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _step(block, *held)
        w = dslib.expand_shift_weights_f8(packed)
    for seed in (2, 3):
        new = _inputs(seed)
        for a, b in zip(held, new):
            a.copy_(b)
        w.q.view(torch.uint8).zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(out, _step(block, *new)))
        again = dslib.expand_shift_weights_f8(packed)
        assert torch.equal(w.q.float(), again.q.float()) and torch.equal(w.scale, again.scale)

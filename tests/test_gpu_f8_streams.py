"""Calls of the 8-bit helpers on a stream that the caller gives: their memory belongs to that stream."""
import pytest
import torch

pytestmark = pytest.mark.gpu
SLEEP = 100_000_000  # cycles: 50 ms, within which the host runs far ahead of the stream


def _side(as_handle):
    """A stream behind the current one with a pause in front of what follows, and the argument that names it."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(SLEEP)
    return side.cuda_stream if as_handle else side, side


@pytest.mark.parametrize("as_handle", [False, True])
def test_workspace_lives_until_the_given_stream_is_done(dslib, as_handle):
    """What the current stream allocates and writes right after the call is not the call's workspace."""
    rows, cols = 1300, 4096
    r = torch.Generator(device="cuda").manual_seed(1)
    dy, h = (torch.randn((rows, cols), generator=r, device="cuda").bfloat16() for _ in range(2))
    w, rstd = torch.rand(cols, generator=r, device="cuda") + 0.5, (h.float().square().mean(1) + 1e-5).rsqrt()
    want = dslib.rmsnorm_f8_backward(dy, h, rstd, w)
    nbytes = dslib.ds_rmsnorm_f8_backward_workspace_bytes(rows, cols)
    torch.cuda.synchronize()
    stream, side = _side(as_handle)
    got = dslib.rmsnorm_f8_backward(dy, h, rstd, w, stream=stream)
    over = [torch.full((nbytes,), 0xFF, dtype=torch.uint8, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert all(bool((t == 0xFF).all()) for t in over)


@pytest.mark.parametrize("as_handle", [False, True])
def test_outputs_are_not_memory_that_the_current_stream_still_reads(dslib, as_handle):
    """Freed on the current stream with a read of it pending: not taken for the outputs of a call on another one."""
    rows, cols = 1024, 2048
    r = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((rows, cols), generator=r, device="cuda").bfloat16()
    weight = torch.ones(cols, device="cuda")
    calls = {
        "quantize": lambda **kw: dslib.quantize_f8(x, "rows", "rows", **kw),
        "norm": lambda **kw: dslib.rmsnorm_f8(x, weight, residual=x, **kw),
        "gate": lambda **kw: dslib.gated_f8(x, cols // 2, **kw),
    }
    q = calls["quantize"]()[0]
    kept, da = calls["gate"]()[1], x[:, : cols // 2].contiguous()
    calls["product"] = lambda **kw: dslib.linear_f8(q, q, **kw)
    calls["gate_backward"] = lambda **kw: dslib.gated_f8_backward(kept, da, **kw)
    calls["norm_backward"] = lambda **kw: dslib.rmsnorm_f8_backward(x, x, weight[:rows], weight, **kw)
    packed = dslib.pack_shift_weights(torch.ones((rows, cols), dtype=torch.int8, device="cuda"),
                                      torch.zeros((rows, cols), dtype=torch.int8, device="cuda"))
    calls["shift weights"] = lambda **kw: dslib.expand_shift_weights_f8(packed, **kw)

    def tensors(got):
        for t in got if isinstance(got, tuple) else (got,):
            if isinstance(t, dslib.F8Matrix):
                yield from (t.q.view(torch.uint8), t.scale)
            elif t is not None and t is not x:
                yield t

    for name, call in calls.items():
        want = [t.clone() for t in tensors(call())]
        torch.cuda.synchronize()
        stream, side = _side(as_handle)
        side.synchronize()
        torch.cuda._sleep(SLEEP)  # the current stream is behind now
        held = [torch.full_like(t, 3) for t in want for _ in range(3)]
        copies = [t.clone() for t in held]
        del held
        got = call(stream=stream)
        torch.cuda.synchronize()
        assert all(bool((t == 3).all()) for t in copies), name
        assert all(torch.equal(a, b) for a, b in zip(tensors(got), want)), name


def test_every_name_of_a_stream_is_taken(dslib):
    """A torch stream, its handle, an object with the handle as `cuda_stream`, and both handles of the default stream."""
    x = torch.randn((5, 256), device="cuda")
    want, _ = dslib.quantize_f8(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    class Other:
        cuda_stream = side.cuda_stream

    before = torch.cuda.current_stream()
    for name in (side, side.cuda_stream, Other(), 0, 1, torch.cuda.default_stream()):
        m, _ = dslib.quantize_f8(x, stream=name)
        torch.cuda.synchronize()
        assert torch.equal(m.q.float(), want.q.float()) and torch.cuda.current_stream() == before

"""The experts' operators and the optimizer step on streams that the caller gives, from several host threads, with a wait
limit that runs out, over memory past 2^31 values, and with tokens, columns or reductions of none."""
import threading

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
SLEEP = 100_000_000  # cycles: 50 ms, within which the host runs far ahead of the stream


def _state(ds, seed=1, tokens=600, hidden=256, features=128, experts=6, top_k=2):
    r = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=r, device="cuda")  # noqa: E731
    ids = torch.randint(-1, experts, (tokens, top_k), generator=r, device="cuda")
    order = ds.expert_order(ids, experts, align=128)
    x, y = n(tokens, hidden).bfloat16(), n(order.rows, hidden).bfloat16()
    rows = ds.expert_gather(ds.quantize_f8(x, pow2=True)[0], order)
    w = ds.quantize_f8(n(experts * features, hidden), "tiles")[0]
    d_t = ds.quantize_f8(ds.expert_gather(n(tokens, features), order), None, "rows")[1]
    x_t = ds.quantize_f8(rows, None, "tiles", pow2=True)[1]
    weights = torch.rand((tokens, top_k), generator=r, device="cuda")
    return dict(ids=ids, order=order, x=x, y=y, rows=rows, w=w, d_t=d_t, x_t=x_t, weights=weights, d=n(tokens, hidden).bfloat16())


def _calls(ds, s, kw):
    e = s["order"].experts
    return {"order": lambda: ds.expert_order(s["ids"], e, align=128, **kw), "gather": lambda: ds.expert_gather(s["x"], s["order"], **kw),
            "gather8": lambda: ds.expert_gather(ds.F8Matrix(s["x8"].q, s["x8"].scale) if "x8" in s else ds.quantize_f8(s["x"])[0], s["order"], **kw),
            "combine": lambda: ds.expert_combine(s["y"], s["order"], s["weights"], **kw),
            "backward": lambda: ds.expert_combine_backward(s["d"], s["y"], s["order"], s["weights"], **kw),
            "linear": lambda: ds.expert_linear_f8(s["rows"], s["w"], s["order"], **kw),
            "grad": lambda: ds.expert_weight_grad_f8(s["d_t"], s["x_t"], s["order"], **kw)}


def _tensors(ds, got):
    for t in got if isinstance(got, tuple) else (got,):
        if isinstance(t, ds.F8Matrix):
            yield from (t.q.view(torch.uint8), t.scale)
        elif isinstance(t, ds.ExpertOrder):
            yield from (t.offsets, t.counts, t.position, t.slot)
        else:
            yield t


@pytest.mark.parametrize("as_handle", [False, True])
def test_outputs_belong_to_the_given_stream(dslib, as_handle):
    """Memory freed on the current stream with a read of it pending is not taken for the outputs of a call on another."""
    s = _state(dslib)
    s["x8"] = dslib.quantize_f8(s["x"])[0]
    for name, call in _calls(dslib, s, {}).items():
        want = [t.clone() for t in _tensors(dslib, call())]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        torch.cuda.synchronize()
        torch.cuda._sleep(SLEEP)  # the current stream is behind now
        held = [torch.full_like(t, 3) for t in want for _ in range(3)]
        copies = [t.clone() for t in held]
        del held
        got = _calls(dslib, s, {"stream": side.cuda_stream if as_handle else side})[name]()
        torch.cuda.synchronize()
        assert all(bool((t == 3).all()) for t in copies), name
        assert all(torch.equal(a, b) for a, b in zip(_tensors(dslib, got), want)), name


def test_four_host_threads(dslib):
    """Each on its own stream with its own inputs: the bits of a thread alone."""
    def work(seed):
        s = _state(dslib, seed)
        out = [t for call in _calls(dslib, s, {}).values() for t in _tensors(dslib, call())]
        p = [torch.ones(5000, device="cuda"), torch.ones(77, device="cuda")]
        opt = dslib.AdamW(p, [s["weights"].view(-1)[:100].repeat(50), s["weights"].view(-1)[:77].clone()], state_dtype=torch.float8_e4m3fn, seed=seed)
        for _ in range(3):
            opt.step()
        return out + p

    alone = {seed: [t.clone() for t in work(seed)] for seed in range(4)}
    torch.cuda.synchronize()
    got, errors = {}, []

    def run(seed):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(4):
                    got[seed] = work(seed)
            stream.synchronize()
        except Exception as e:  # reported by the main thread
            errors.append(e)

    threads = [threading.Thread(target=run, args=(seed,)) for seed in alone]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for seed, want in alone.items():
        assert all(torch.equal(a, b) for a, b in zip(got[seed], want)), seed
    assert dslib.ds_f8_fault_flag() == 0


@pytest.mark.parametrize("tokens", [5, 2000])
def test_products_with_the_shortest_wait_limit(dslib, tokens):
    """With the wait limit cut to one cycle a launch gives up and sets the flag (or never had to wait, and is correct); the
    context stays usable and the next call is correct.  5 tokens take the kernel of small products, 2000 the other."""
    s = _state(dslib, 2, tokens=tokens, hidden=1024, features=512)
    calls = _calls(dslib, s, {})
    for name in ("linear", "grad"):
        want = calls[name]()
        assert dslib.ds_f8_fault_flag() == 0
        try:
            dslib.ds_f8_set_wait_limit(1)
            got = calls[name]()
            torch.cuda.synchronize()
        finally:
            dslib.ds_f8_set_wait_limit(0)
        assert dslib.ds_f8_fault_flag() == 1 or torch.equal(got, want)
        assert dslib.ds_f8_fault_flag() == 0
        assert torch.equal(calls[name](), want) and dslib.ds_f8_fault_flag() == 0


def test_no_tokens(dslib):
    """An empty batch: empty rows, and weight gradients of zeros or what they are added to."""
    order = dslib.expert_order(torch.empty((0, 2), dtype=torch.int32, device="cuda"), 4, align=128)
    x = dslib.F8Matrix.empty(0, 256, "cuda")
    w = dslib.quantize_f8(torch.randn(4 * 128, 256, device="cuda"), "tiles")[0]
    rows = dslib.expert_gather(x, order)
    assert rows.q.shape == (0, 256) and dslib.expert_linear_f8(rows, w, order).shape == (0, 128)
    dy, dw = dslib.expert_combine_backward(torch.empty((0, 128), device="cuda"), torch.empty((0, 128), device="cuda"), order,
                                           torch.empty((0, 2), device="cuda"))
    assert dy.shape == (0, 128) and dw.shape == (0, 2)
    d_t, x_t = dslib.F8Matrix.empty(128, 0, "cuda"), dslib.F8Matrix.empty(256, 0, "cuda")
    assert bool((dslib.expert_weight_grad_f8(d_t, x_t, order) == 0).all())
    add = torch.randn(4, 128, 256, device="cuda")
    assert torch.equal(dslib.expert_weight_grad_f8(d_t, x_t, order, add=add), add)


def test_reduction_of_none(dslib):
    """K = 0: the bias in the experts' rows, zeros behind them."""
    order = dslib.expert_order(torch.tensor([[0], [2], [2]], device="cuda"), 3, align=128)
    x, w = dslib.F8Matrix.empty(order.rows, 0, "cuda"), dslib.F8Matrix.empty(3 * 128, 0, "cuda", tiles=True)
    bias = torch.randn(3, 128, device="cuda")
    y = dslib.expert_linear_f8(x, w, order, bias=bias, dtype=torch.float32)
    assert torch.equal(y[:128], bias[0].expand(128, -1)) and torch.equal(y[128:256], bias[2].expand(128, -1))
    assert bool((y[256:] == 0).all())


def test_every_row_of_a_large_matrix(dslib):
    """Rows whose offsets pass 2^31 values and 2^32 bytes: 1.1 million rows of 2049 bf16 (accesses of 2 bytes) and 2048."""
    tokens, top_k = 550_000, 2
    r = torch.Generator(device="cuda").manual_seed(3)
    ids = torch.randint(0, 7, (tokens, top_k), generator=r, device="cuda")
    order = dslib.expert_order(ids, 7, align=1)
    assert order.rows == tokens * top_k and bool((order.counts == ids.view(-1).bincount(minlength=7)).all())
    pos = order.position.long()
    for cols in (2048, 2049):
        x = torch.randn((tokens, cols), generator=r, device="cuda").bfloat16()
        rows = dslib.expert_gather(x, order)
        at = torch.randint(0, tokens, (2000,), generator=r, device="cuda")
        at[:3] = torch.tensor([0, 1, tokens - 1], device="cuda")
        for j in range(top_k):
            assert torch.equal(rows[pos[at, j]], x[at])
        twice = dslib.expert_combine(rows, order)  # x + x, exactly
        assert torch.equal(twice[at], 2 * x[at])
        dy, dw = dslib.expert_combine_backward(x, rows, order, torch.full((tokens, top_k), 0.5, device="cuda"), out=rows)
        assert torch.equal(dy[pos[at, 1]], 0.5 * x[at])
        exact = x[at].double().square().sum(1)
        assert bool(((dw[at, 0].double() - exact).abs() <= (cols / 32 + 16) * 2.0**-24 * exact).all())
        del x, rows, twice, dy


def test_optimizer_past_2_32_values(dslib):
    """One tensor of 2^32 + 4133 values with 8-bit states: its last values are those of a small one with their bits."""
    n, tail = 2**32 + 4133, 4133 + 128
    p, g = torch.zeros(n, device="cuda"), torch.full((n,), 1e-3, device="cuda", dtype=torch.bfloat16)
    p[-tail:] = torch.linspace(-1, 1, tail, device="cuda")
    g[-tail:] = torch.linspace(1e-3, 2e-3, tail, device="cuda").bfloat16()
    opt = dslib.AdamW([p], [g], state_dtype=torch.float8_e4m3fn, lr=1e-3)
    opt.step()
    # indices count modulo 2^32 in the hash: the values from 2^32 on have the bits of the first ones
    q, h = torch.linspace(-1, 1, tail, device="cuda")[128:].clone(), torch.linspace(1e-3, 2e-3, tail, device="cuda").bfloat16()[128:].clone()
    small = dslib.AdamW([q], [h], state_dtype=torch.float8_e4m3fn, lr=1e-3)
    small.step()
    assert torch.equal(p[2**32 :], q)
    for a, b in ((opt.m[0], small.m[0]), (opt.v[0], small.v[0])):
        assert torch.equal(a[0][2**32 :].view(torch.uint8), b[0].view(torch.uint8)) and torch.equal(a[1][2**25 :], b[1])
    assert bool((p[:1000] == p[0]).all()) and float(p[0]) < 0


@pytest.mark.parametrize("p,g", [("bfloat16", "bfloat16"), ("float16", "float32")])
def test_16_bit_parameters_with_8_bit_states(dslib, p, g):
    r = np.random.default_rng(6)
    a = torch.from_numpy(r.standard_normal(3001).astype(np.float32)).cuda()
    b = torch.from_numpy((r.standard_normal(3001) * 1e-3).astype(np.float32)).cuda().to(getattr(torch, g))
    low, full = a.to(getattr(torch, p)), a.to(getattr(torch, p)).float()
    x = dslib.AdamW([low], [b], state_dtype=torch.float8_e4m3fn, lr=1e-2, seed=4)
    y = dslib.AdamW([full], [b], state_dtype=torch.float8_e4m3fn, lr=1e-2, seed=4)
    x.step()
    y.step()
    assert torch.equal(low, full.to(low.dtype))  # rounded once; the states do not depend on the parameters' type
    assert torch.equal(x.m[0][0].view(torch.uint8), y.m[0][0].view(torch.uint8)) and torch.equal(x.v[0][1], y.v[0][1])

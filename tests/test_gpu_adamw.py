"""GPU parity of the optimizer step with the numpy oracle.

With the step's number and lr on the host the definition is a fixed sequence of float32 operations: parameters, states
and scales are equal bit for bit, 8-bit states too.  Against float64 a value may be off by the roundings of that
sequence (counted at the tests); with the number on the device, factors differ from those of the host by a few steps.
"""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as X

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
F8 = torch.float8_e4m3fn
LR, BETAS, EPS = 1e-3, (0.9, 0.999), 1e-8


def _rng(*key):
    return np.random.default_rng(sum(ord(c) * (i + 1) for i, c in enumerate(str(key))))


def _np(t):
    return t.detach().float().cpu().numpy()


def _at(values, kind, offset):
    """The values as a tensor that starts `offset` elements behind an aligned address."""
    held = torch.empty(values.size + offset, dtype=TYPES.get(kind, kind), device="cuda")
    out = held[offset:]
    out.copy_(torch.from_numpy(values.astype(np.float32)).cuda())
    return out


def _case(r, sizes, p="f32", g="f32", offset=0):
    """Parameters, gradients (some of them zero, some tiny, some large), first and second moments."""
    params = [_at(r.standard_normal(n) * 0.02, p, offset) for n in sizes]
    grads = []
    for n in sizes:
        a = r.standard_normal(n) * 1e-3 * 10.0 ** r.integers(-3, 2, n)
        a[r.random(n) < 0.1] = 0
        grads.append(_at(a, g, offset))
    m = [(r.standard_normal(n) * 1e-4).astype(np.float32) for n in sizes]
    v = [((r.standard_normal(n) * 1e-3) ** 2).astype(np.float32) for n in sizes]
    return params, grads, m, v


SIZES = [(1,), (7, 128, 129), (2048, 2049, 5000), (100_003,), tuple(range(1, 60))]


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("p,g,copy", [("f32", "f32", None), ("f32", "bf16", "bf16"), ("f32", "f16", "f16"), ("bf16", "bf16", None),
                                      ("f16", "f32", "f32")])
@pytest.mark.parametrize("offset", [0, 1, 4])
def test_float32_states_bit_for_bit(dslib, sizes, p, g, copy, offset):
    r = _rng("f32", sizes, p, g)
    params, grads, m, v = _case(r, sizes, p, g, offset)
    ms, vs = [_at(a, "f32", offset) for a in m], [_at(a, "f32", offset) for a in v]
    copies = [_at(np.zeros(n), copy, offset) for n in sizes] if copy else None
    decay = [0.1 if n > 100 else 0.0 for n in sizes]
    start = [_np(a) for a in params]
    opt = dslib.AdamW(params, grads, m=ms, v=vs, copies=copies, lr=LR, betas=BETAS, eps=EPS, weight_decay=decay, steps=41)
    for t in (42, 43):
        opt.step()
        assert opt.steps == t
        for k in range(len(sizes)):
            new, m[k], v[k], _ = X.adamw32(start[k], _np(grads[k]), m[k], v[k], t, LR, BETAS, EPS, decay[k])
            want = torch.from_numpy(new).to(TYPES[p])
            assert torch.equal(params[k].cpu(), want)
            assert np.array_equal(_np(ms[k]), m[k]) and np.array_equal(_np(vs[k]), v[k])
            if copy:
                assert torch.equal(copies[k].cpu(), torch.from_numpy(new).to(TYPES[copy]))
            start[k] = want.float().numpy()


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("g,copy", [("f32", None), ("bf16", "bf16")])
@pytest.mark.parametrize("offset", [0, 3])
def test_8bit_states_bit_for_bit(dslib, sizes, g, copy, offset):
    r = _rng("f8", sizes, g)
    params, grads, m, v = _case(r, sizes, "f32", g, offset)
    scale = torch.full((1,), 0.625, device="cuda")
    zero = lambda n: (_at(np.zeros(n), F8, offset), torch.zeros(-(-n // 128), device="cuda"))  # noqa: E731
    ms, vs = [zero(n) for n in sizes], [zero(n) for n in sizes]
    copies = [_at(np.zeros(n), copy, offset) for n in sizes] if copy else None
    now = [_np(a) for a in params]
    qm = [(np.zeros(n, np.float32), np.zeros(-(-n // 128), np.float32)) for n in sizes]
    qv = list(qm)
    opt = dslib.AdamW(params, grads, m=ms, v=vs, copies=copies, lr=LR, betas=BETAS, eps=EPS, weight_decay=0.1, grad_scale=scale, seed=5)
    value = lambda q: q[0] * np.repeat(q[1], 128)[: q[0].size]  # noqa: E731
    for t in (1, 2, 3):
        opt.step()
        for k, n in enumerate(sizes):
            root = value(qv[k])
            now[k], m1, _, root = X.adamw32(now[k], _np(grads[k]), value(qm[k]), root * root, t, LR, BETAS, EPS, 0.1, 0.625)
            low, high = X.random_bits(n, t, k, 5)
            qm[k], qv[k] = X.state_to_f8(m1, low, False), X.state_to_f8(root, high, True)
            assert np.array_equal(_np(params[k]), now[k])
            for got, want in ((ms[k], qm[k]), (vs[k], qv[k])):
                assert np.array_equal(_np(got[0]), want[0]) and np.array_equal(_np(got[1]), want[1])
            if copy:
                assert torch.equal(copies[k].cpu(), torch.from_numpy(now[k]).to(TYPES[copy]))


def test_against_float64(dslib):
    """Roundings of 2^-24 each: m three, of its two terms; v five; p four of itself, and the update's fourteen (m's three
    terms, the rate and the root's factor with their own, the root with half of v's, two sums and a quotient)."""
    r = _rng("f64")
    params, grads, m, v = _case(r, (50_000,))
    p0, g0, m0, v0 = (a.astype(np.float64) for a in (_np(params[0]), _np(grads[0]), m[0], v[0]))
    opt = dslib.AdamW(params, grads, m=[_at(m[0], "f32", 0)], v=[_at(v[0], "f32", 0)], lr=LR, betas=BETAS, eps=EPS, weight_decay=0.1, steps=9)
    opt.step()
    p1, m1, v1 = X.adamw64(p0, g0, m0, v0, 10, LR, BETAS, EPS, 0.1)
    ulp = 2.0**-24
    terms = np.abs(0.9 * m0) + np.abs(0.1 * g0)
    assert np.all(np.abs(_np(opt.m[0]) - m1) <= 4 * ulp * terms + 1e-44)
    assert np.all(np.abs(_np(opt.v[0]) - v1) <= 6 * ulp * v1 + 1e-44)
    update = terms * LR / (1 - 0.9**10) / (np.sqrt(v1 / (1 - 0.999**10)) + EPS)
    assert np.all(np.abs(_np(params[0]) - p1) <= 4 * ulp * np.abs(p0) + 20 * ulp * update)


def test_8bit_rounding_keeps_the_mean(dslib):
    """The mean of many roundings of one value is the value: 2^18 of them, each with a variance of at most a quarter
    step squared, so within 5 / 2^10 steps but once in a million; and 2^-17 for the finite number of random bits."""
    n = 128 * 2**11
    g = torch.full((n,), 0.3e-3, device="cuda")
    g[::128] = 1e-3  # the block's largest value, so that u = 0.3 * 448 lies between 128 and 144
    for k in range(3):
        p = torch.zeros(n, device="cuda")
        opt = dslib.AdamW([p], [g], betas=(0.0, 0.0), seed=k, state_dtype=F8)
        opt.step()
        u = 0.3 * 448
        for q, s in (opt.m[0], opt.v[0]):
            got = q.float().view(-1, 128)[:, 1:].cpu().numpy()
            assert set(np.unique(got)) == {128.0, 144.0}
            assert abs(got.mean(dtype=np.float64) - u) < 16 * (5 / 2**10 + 2.0**-17)
            assert bool((q.float().view(-1, 128)[:, 0] == 448).all()) and torch.allclose(s, torch.full_like(s, 1e-3 / 448), rtol=1e-6)


def test_8bit_root_is_never_lost(dslib):
    """A block with one large gradient: the others' roots are far below the smallest value and are held as it."""
    g = torch.full((256,), 1e-9, device="cuda")
    g[0] = 1.0
    p = torch.zeros(256, device="cuda")
    opt = dslib.AdamW([p], [g], state_dtype=F8, lr=LR)
    for _ in range(50):
        opt.step()
        assert bool((opt.v[0][0].float() >= 2.0**-9).all())
    assert bool(torch.isfinite(p).all()) and float(p.abs().max()) <= 50 * LR * 1.01 + 1e-6


def test_8bit_states_move(dslib):
    """With beta2 = 0.999 and a gradient that halves, the second moment follows (rounding to the nearest would keep it)."""
    n = 4096
    g = torch.ones(n, device="cuda")
    p = torch.zeros(n, device="cuda")
    opt = dslib.AdamW([p], [g], lr=0.0, state_dtype=F8)
    for _ in range(300):
        opt.step()
    g.fill_(0.5)
    g[::128] = 1.0  # the blocks' scales stay
    for _ in range(700):
        opt.step()
    q, s = opt.v[0]
    got = (q.float().view(-1, 128) * s[:, None])[:, 1:].square().mean()
    v = (1 - 0.999**300) * 0.999**700 + 0.25 * (1 - 0.999**700)
    # a rounding of the root by up to a step d adds d^2 / 4 to the mean square at most: 1/64 of it per step, which decays
    # as 0.999; so the mean stays within a fifth of v and clearly off where it was
    assert abs(float(got) / v - 1) < 0.2, (float(got), v)


def test_8bit_second_moment_is_above_the_recurrence_by_at_most_2_15(dslib):
    """As the oracle's (test_experts_cpu.py, where the bounds are derived), with 2^17 values: blocks whose scale stays."""
    n = 1 << 17
    r = torch.Generator(device="cuda").manual_seed(8)
    q, s = torch.zeros(n, device="cuda"), torch.full((n // 128,), 4 / 448, device="cuda")
    q[::128] = 448
    g, v = torch.empty(n, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
    state = (torch.zeros(n, device="cuda").to(F8), torch.zeros(n // 128, device="cuda"))
    opt = dslib.AdamW([torch.zeros(n, device="cuda")], [g], m=[state], v=[(q.to(F8), s)], lr=0.0, betas=(0.9, 0.999))
    for _ in range(2000):
        g.normal_(generator=r)
        g[::128] = 4
        v = 0.999 * v + 0.001 * g.double().square()
        opt.step()
    small = torch.arange(n, device="cuda") % 128 != 0
    held = (opt.v[0][0].float().view(-1, 128) * opt.v[0][1][:, None]).view(-1)
    off = float(held[small].double().square().mean() / v[small].mean()) - 1
    few = 5 * 0.5 / float(small.sum()) ** 0.5
    assert -few <= off <= 2 / 15 + few, off


@pytest.mark.parametrize("beta2", [0.501, 0.999])
@pytest.mark.parametrize("top,lost", [(1.0, False), (2.0**-57, False), (1e-18, True)])
def test_smallest_8bit_root_has_a_square(dslib, beta2, top, lost):
    """Without a gradient and with eps 0 a step divides 0 by the root: NaN shows a root whose square was 0 in float32."""
    n = 256
    q = torch.full((n,), 2.0**-9, device="cuda")
    q[::128] = 448
    zero = (torch.zeros(n, device="cuda").to(F8), torch.zeros(2, device="cuda"))
    p = torch.ones(n, device="cuda")
    state = (q.to(F8), torch.full((2,), top / 448, device="cuda"))
    dslib.AdamW([p], [torch.zeros(n, device="cuda")], m=[zero], v=[state], betas=(0.9, beta2), eps=0.0, weight_decay=0.0).step()
    if lost:
        assert bool(torch.isnan(p[1:128]).all()) and bool((p[::128] == 1).all())
    else:
        assert bool((p == 1).all())


@pytest.mark.parametrize("state", [torch.float32, F8])
def test_values_that_are_not_finite(dslib, state):
    """An infinite or NaN gradient spoils its own value and no other; its 8-bit states become NaN."""
    r = _rng("inf")
    g = torch.from_numpy((r.standard_normal(1000) * 1e-3).astype(np.float32)).cuda()
    clean = g.clone()
    g[5], g[300], g[999] = float("inf"), float("nan"), -float("inf")
    bad = torch.zeros(1000, dtype=torch.bool, device="cuda")
    bad[[5, 300, 999]] = True
    p, c = torch.ones(1000, device="cuda"), torch.ones(1000, device="cuda")
    a, b = dslib.AdamW([p], [g], state_dtype=state), dslib.AdamW([c], [clean], state_dtype=state)
    clean[bad] = 0
    a.step()
    b.step()
    assert torch.equal(p[~bad], c[~bad]) and not bool(torch.isfinite(p[bad]).any())
    if state == F8:
        for (q, s), (q0, s0) in ((a.m[0], b.m[0]), (a.v[0], b.v[0])):
            assert torch.equal(s, s0) and torch.equal(q.float()[~bad], q0.float()[~bad]) and bool(torch.isnan(q.float()[bad]).all())


def test_zero_gradients_and_eps_zero(dslib):
    """0 / 0 is NaN where eps is zero, as the formula says; with eps a value without gradient only decays."""
    p, q = torch.ones(130, device="cuda"), torch.ones(130, device="cuda")
    g = torch.zeros(130, device="cuda")
    dslib.AdamW([p], [g], lr=0.5, weight_decay=0.5, state_dtype=F8).step()
    assert bool((p == 0.75).all())
    opt = dslib.AdamW([q], [g], eps=0.0, state_dtype=F8)
    opt.step()
    assert bool(torch.isnan(q).all()) and bool((opt.v[0][0].float() == 0).all())


@pytest.mark.parametrize("state", [torch.float32, F8])
def test_step_on_the_device_and_in_a_graph(dslib, state):
    """A captured step replayed five times is five steps; its factors are within a few float32 steps of the host's."""
    r = _rng("graph")
    sizes = (1000, 4097)
    params, grads, _, _ = _case(r, sizes)
    others = [p.clone() for p in params]
    steps, lr = torch.zeros((), dtype=torch.int64, device="cuda"), torch.full((), LR, device="cuda")
    opt = dslib.AdamW(params, grads, lr=lr, steps=steps, state_dtype=state, seed=3)
    ref = dslib.AdamW(others, grads, lr=LR, state_dtype=state, seed=3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        opt.step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step()
    for _ in range(4):
        graph.replay()
    for _ in range(5):
        ref.step()
    assert int(steps) == 5 and ref.steps == 5
    for a, b in zip(params, others):
        # five updates of at most lr / sqrt(...) each: factors off by 2^-21; 8-bit states may round the other way rarely
        err = (a - b).abs()
        if state == F8:
            assert float((err > 1e-8).float().mean()) < 0.01
        else:
            assert float(err.max()) <= 5 * 10 * LR * 2.0**-20 + 2.0**-24 * 5


def test_many_tensors_take_several_launches(dslib):
    """900 tensors: three launches; each tensor as if alone (its number decides its random bits)."""
    r = _rng("many")
    sizes = tuple(int(n) for n in r.integers(1, 300, 900))
    params, grads, _, _ = _case(r, sizes)
    now = [_np(p) for p in params]
    opt = dslib.AdamW(params, grads, lr=LR, state_dtype=F8, seed=9, weight_decay=0.0)
    opt.step()
    for k in (0, 399, 400, 401, 799, 800, 899):
        new, m, _, root = X.adamw32(now[k], _np(grads[k]), np.zeros(sizes[k], np.float32), np.zeros(sizes[k], np.float32), 1, LR, BETAS, EPS, 0.0)
        assert np.array_equal(_np(params[k]), new)
        low, high = X.random_bits(sizes[k], 1, k, 9)
        assert np.array_equal(_np(opt.m[k][0]), X.state_to_f8(m, low, False)[0])
        assert np.array_equal(_np(opt.v[k][0]), X.state_to_f8(root, high, True)[0])


def test_another_stream_and_new_gradients(dslib):
    p, g = torch.ones(5000, device="cuda"), torch.full((5000,), 1e-3, device="cuda")
    c = p.clone()
    a, b = dslib.AdamW([p], [g]), dslib.AdamW([c], [g])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a.step(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    b.step()
    assert torch.equal(p, c)
    other = torch.full((5000,), -2e-3, device="cuda", dtype=torch.bfloat16)
    a.step([other])
    b.step([other.float()])
    assert torch.equal(p, c)


def test_refusals_on_a_gpu(dslib):
    p, g = torch.ones(100, device="cuda"), torch.ones(100, device="cuda")
    for bad in (lambda: dslib.AdamW([], []), lambda: dslib.AdamW([p], []), lambda: dslib.AdamW([p], [g[:50]]),
                lambda: dslib.AdamW([p], [g], m=[g.half()]), lambda: dslib.AdamW([p], [g.cpu()]),
                lambda: dslib.AdamW([p[::2]], [g[::2].contiguous()]), lambda: dslib.AdamW([p.int()], [g]),
                lambda: dslib.AdamW([p], [g], state_dtype=torch.float16), lambda: dslib.AdamW([p], [g], weight_decay=[0.1, 0.2])):
        with pytest.raises(ValueError):
            bad()
    before = p.clone()
    for bad in (dslib.AdamW([p, p], [g, g]), dslib.AdamW([p], [p]), dslib.AdamW([p[:60], p[50:]], [g[:60], g[50:]]),
                dslib.AdamW([p], [g], betas=(1.0, 0.9)), dslib.AdamW([p], [g], eps=-1.0), dslib.AdamW([p], [g], lr=-1.0),
                dslib.AdamW([p], [g], steps=-1), dslib.AdamW([p], [g], weight_decay=-0.1), dslib.AdamW([p], [g], copies=[g])):
        with pytest.raises(dslib.DsError):
            bad.step()
        assert bad.steps in (0, -1) and torch.equal(p, before)
    opt = dslib.AdamW([p], [g])
    with pytest.raises(ValueError):
        opt.step([g[:10]])
    opt.params[0].data = torch.zeros(100, device="cuda")
    with pytest.raises(ValueError, match="other memory"):
        opt.step()
    shared = dslib.AdamW([torch.ones(100, device="cuda"), torch.ones(100, device="cuda")], [g, g])  # reading twice is fine
    shared.step()


def test_memory_of_replaced_states_stays(dslib):
    """A step writes the states that the optimizer was made with, also where its lists were given others since."""
    p, g = torch.ones(70_000, device="cuda"), torch.full((70_000,), 1e-3, device="cuda")
    opt = dslib.AdamW([p], [g])
    held = opt.m[0]
    opt.m[0], opt.v[0] = None, None
    over = [torch.full((70_000,), 7.0, device="cuda") for _ in range(4)]
    opt.step()
    assert all(bool((t == 7).all()) for t in over) and bool((held != 0).all())


@pytest.mark.parametrize("state", [torch.float32, F8])
def test_memory_of_states_with_another_storage_stays(dslib, state):
    """Where a state was given other memory, the step goes on with what it was made with, which nothing else got."""
    n = 70_000
    p, g = torch.ones(n, device="cuda"), torch.full((n,), 1e-3, device="cuda")
    q = p.clone()
    a, b = dslib.AdamW([p], [g], state_dtype=state), dslib.AdamW([q], [g], state_dtype=state)
    a.step()
    b.step()
    for t in (a.m[0], a.v[0]):
        for x in (t if isinstance(t, tuple) else (t,)):
            x.data = x.clone()
    over = [torch.full((n,), 7, device="cuda", dtype=torch.uint8 if state == F8 else torch.float32) for _ in range(8)]
    scales = [torch.full((-(-n // 128),), 7.0, device="cuda") for _ in range(8)]
    a.step()
    b.step()
    assert torch.equal(p, q) and all(bool((t == 7).all()) for t in over + scales)


def test_copies_and_parameters_with_another_storage_are_refused(dslib):
    """Also where the step is given its gradients; nothing is written, and nothing else got the memory."""
    n = 70_000
    g = torch.full((n,), 1e-3, device="cuda")
    for which in (0, 1):
        for new in (None, [g.clone()]):
            p, c = torch.ones(n, device="cuda"), torch.ones(n, device="cuda", dtype=torch.bfloat16)
            opt = dslib.AdamW([p], [g], copies=[c])
            (p, c)[which].data = torch.zeros_like((p, c)[which])
            over = [torch.full_like((p, c)[which], 7.0) for _ in range(4)]
            for _ in range(2):
                with pytest.raises(ValueError, match="other memory"):
                    opt.step(new)
            assert opt.steps == 0 and all(bool((t == 7).all()) for t in over)
            assert bool((opt.m[0] == 0).all()) and bool(((p, c)[which] == 0).all()) and bool(((p, c)[1 - which] == 1).all())


@pytest.mark.parametrize("beta1,beta2", [(0.9, 0.999), (0.5, 0.75)])
def test_roots_and_quotients_are_correctly_rounded(dslib, beta1, beta2):
    """The roots and quotients of steps with 8-bit states, by one correction each, are those of correctly rounded operations:
    2^22 of them over all exponents that this path takes (v up to 2^67, m from 2^-74 to 2^60, roots from below eps = 2^-60
    on).  Without a gradient, decay and parameter a step is -(m / (sqrt(v) + eps)), m and v beta times what the states hold."""
    n, r = 1 << 22, _rng("exact", beta1, beta2)
    scale = lambda low, high: (np.exp2(r.integers(low, high, n // 128)) * r.uniform(1, 2, n // 128)).astype(np.float32)  # noqa: E731
    q = lambda codes: torch.from_numpy(r.choice(np.array(codes, np.uint8), n)).view(F8).cuda()  # noqa: E731
    positive = list(range(127))
    ms, vs = (q(positive + [c + 128 for c in positive]), scale(-65, 50)), (q(positive), scale(-68, 24))
    value = lambda s: _np(s[0]) * np.repeat(s[1], 128)  # noqa: E731
    m, root = value(ms), value(vs)
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    on_gpu = lambda s: (s[0], torch.from_numpy(s[1]).cuda())  # noqa: E731
    t = 1_000_000  # beta^t is 0: the factors of m and of the root are 1
    opt = dslib.AdamW([p], [g], m=[on_gpu(ms)], v=[on_gpu(vs)], lr=1.0, betas=(beta1, beta2), eps=2.0**-60, weight_decay=0.0, steps=t - 1)
    opt.step()
    with np.errstate(under="ignore"):
        want = X.adamw32(np.zeros(n, np.float32), np.zeros(n, np.float32), m, root * root, t, 1.0, (beta1, beta2), 2.0**-60, 0.0)[0]
    assert np.isfinite(want).all() and (want != 0).mean() > 0.9
    assert np.array_equal(_np(p), want)

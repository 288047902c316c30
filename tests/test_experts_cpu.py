"""The experts' operators and the optimizer step without a GPU: the oracle's own pins, and the refusals of the C ABI and
the helpers."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import experts_oracle as X
from test_f8_cpu import _m
from test_f8_devices_cpu import OnSecondGpu


@pytest.fixture(scope="module")
def ds():
    from paper_1905_13298_gb300 import build
    build.build_library()
    import paper_1905_13298_gb300 as ds
    ds.lib()
    return ds


# ------------------------------------------------------------------------------------------------------------- oracle


@pytest.mark.parametrize("align", [1, 16, 128])
def test_order_is_a_stable_sort(align):
    r = np.random.default_rng(1)
    ids = r.integers(-1, 8, (50, 3))
    rows = X.rows_needed(50, 3, 7, align)
    offsets, counts, position, slot = X.order(ids, 7, align, rows)
    flat = ids.reshape(-1)
    kept = np.flatnonzero((flat >= 0) & (flat < 7))
    want = kept[np.argsort(flat[kept], kind="stable")]
    assert np.array_equal(slot[slot >= 0], want) and counts.sum() == kept.size and offsets[-1] <= rows
    assert np.all(offsets % align == 0)
    for s in range(flat.size):
        p = position.reshape(-1)[s]
        assert (p < 0 and not 0 <= flat[s] < 7) or slot[p] == s


def test_rows_needed_are_enough_and_reached():
    """Over all ways to give 5 slots to 3 experts with segments of multiples of 4."""
    most = 0
    for n in np.ndindex(6, 6, 6):
        if sum(n) == 5:
            most = max(most, sum(-(-c // 4) * 4 for c in n))
    assert X.rows_needed(5, 1, 3, 4) == most == 12


def test_combine_gradient_against_differences():
    r = np.random.default_rng(2)
    ids = r.integers(-1, 3, (6, 2))
    rows = X.rows_needed(6, 2, 3, 1)
    _, _, position, slot = X.order(ids, 3, 1, rows)
    y, w, d = r.standard_normal((rows, 4)), r.standard_normal((6, 2)), r.standard_normal((6, 4))
    dy, dw, _ = X.combine_backward(d, y, position, rows, w)
    f = lambda: float((X.combine(y, position, w)[0] * d).sum())  # noqa: E731
    for a, g in ((y, dy), (w, dw)):
        for i in np.ndindex(*a.shape):
            old = a[i]
            a[i] = old + 0.5
            hi = f()
            a[i] = old - 0.5
            lo = f()
            a[i] = old
            assert abs(hi - lo - g[i]) < 1e-12  # linear: no truncation


def test_adamw_in_float32_follows_float64():
    r = np.random.default_rng(3)
    p, g, m = (r.standard_normal(4000).astype(np.float32) * s for s in (0.02, 1e-3, 1e-4))
    p, g, m = (a.astype(np.float32) for a in (p, g, m))
    v = ((r.standard_normal(4000) * 1e-3) ** 2).astype(np.float32)
    a = X.adamw32(p, g, m, v, 7, 1e-3, (0.9, 0.999), 1e-8, 0.1)
    b = X.adamw64(*(t.astype(np.float64) for t in (p, g, m, v)), 7, 1e-3, (0.9, 0.999), 1e-8, 0.1)
    terms = np.abs(0.9 * m) + np.abs(0.1 * g)
    update = terms * 1e-3 / (1 - 0.9**7) / (np.sqrt(b[2] / (1 - 0.999**7)) + 1e-8)
    assert np.all(np.abs(a[1] - b[1]) <= 4 * 2.0**-24 * terms)
    assert np.all(np.abs(a[0] - b[0]) <= 2.0**-24 * (4 * np.abs(p) + 20 * update))


def test_adamw64_is_torchs():
    """Against torch's own optimizer in float64, over five steps."""
    r = np.random.default_rng(4)
    p = torch.from_numpy(r.standard_normal(300)).requires_grad_()
    opt = torch.optim.AdamW([p], lr=0.01, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1)
    q, m, v = p.detach().numpy().copy(), np.zeros(300), np.zeros(300)
    for t in range(1, 6):
        g = r.standard_normal(300)
        p.grad = torch.from_numpy(g.copy())
        opt.step()
        q, m, v = X.adamw64(q, g, m, v, t, 0.01, (0.9, 0.99), 1e-6, 0.1)
        assert np.allclose(p.detach().numpy(), q, rtol=1e-12, atol=1e-14)


def test_random_bits_are_even():
    """Both halves of the hash, over 2^20 indices of several steps: each of 256 ranges within 6 standard deviations of its
    share, and neighbours, steps and tensors without correlation (below 6 / 2^10)."""
    n = 1 << 20
    first = None
    for t, number in ((1, 0), (2, 0), (1, 1), (1000, 77)):
        for half in X.random_bits(n, t, number, 5):
            share = np.bincount(half >> 8, minlength=256)
            assert np.all(np.abs(share - n / 256) < 6 * np.sqrt(n / 256))
            u = half.astype(np.float64) - 32767.5
            first = u if first is None else first
            scale = (u * u).mean()
            assert abs((u[1:] * u[:-1]).mean()) < 6 / 2**10 * scale
            if u is not first:
                assert abs((u * first).mean()) < 6 / 2**10 * scale


def test_states_round_to_neighbours_and_keep_the_mean():
    r = np.random.default_rng(5)
    v = (r.standard_normal(128 * 50) * 10.0 ** r.integers(-6, 1, 128 * 50)).astype(np.float32)
    mean = np.zeros(v.size)
    for t in range(200):
        q, s = X.state_to_f8(v, X.random_bits(v.size, t, 0, 0)[0], False)
        assert np.array_equal(q, torch.from_numpy(q).to(torch.float8_e4m3fn).float().numpy())  # e4m3 values
        each = np.repeat(s, 128)
        step = np.ldexp(1.0, np.maximum(np.frexp(np.abs(v) / each)[1] - 1, -6) - 3) * each
        assert np.all(np.abs(q * each - v) < step * (1 + 1e-5))
        mean += q * each / 200
    # a variance of at most a quarter step squared, 200 times: 6 standard deviations
    assert np.all(np.abs(mean - v) <= step * 6 * 0.5 / np.sqrt(200))
    root = np.abs(v)
    root[::128] = 1e6
    q, s = X.state_to_f8(root, np.zeros(v.size, np.uint32), True)
    assert np.all(q[root > 0] >= 2.0**-9) and np.all(q[root == 0] == 0)


def test_8bit_second_moment_is_above_the_recurrence_by_at_most_2_15():
    """The held root r of a value moves from r to a neighbour of sqrt(b r^2 + (1 - b) g^2), and is itself one (the block's
    scale stays).  Between neighbours d apart a rounding has the variance (u - r) (r + d - u) <= d |u - r|, with d <= u / 8
    and |u - r| = (1 - b) |g^2 - r^2| / (u + r): at most (1 - b) (g^2 + r^2) / 16 (u / (u + r) is 1/2 for b near 1).  So
    E r^2 = b E r^2 + (1 - b) E g^2 + that: E r^2 is at least E g^2, and at most 17/15 of it.  A value's square has a
    standard deviation below a half of it (a step adds 4 r^2 times the variance, which decays as b^2): 5 of the mean's."""
    r, n, b = np.random.default_rng(8), 128 * 32, np.float32(0.999)
    root, v = np.zeros(n, np.float32), np.zeros(n)
    root[::128] = 4  # with a gradient of 4: the blocks' scales stay
    v[::128] = 16
    for t in range(1, 2001):
        g = r.standard_normal(n).astype(np.float32)
        g[::128] = 4
        v = 0.999 * v + 0.001 * g.astype(np.float64) ** 2
        new = np.sqrt(root * root * b + g * g * (np.float32(1) - b))
        q, s = X.state_to_f8(new, X.random_bits(n, t, 0, 3)[1], True)
        root = q * np.repeat(s, 128)
    small = np.arange(n) % 128 != 0
    assert np.allclose(s, 4 / 448, rtol=1e-3)
    off = (root[small].astype(np.float64) ** 2).mean() / v[small].mean() - 1
    assert -5 * 0.5 / np.sqrt(small.sum()) <= off <= 2 / 15 + 5 * 0.5 / np.sqrt(small.sum()), off


@pytest.mark.parametrize("beta2", [0.501, 0.9, 0.999])
@pytest.mark.parametrize("top", [2.0**-57, 1e-16, 1.0])
def test_smallest_8bit_root_has_a_square(beta2, top):
    """Where the block's largest root is at least 2^-57, 2^-9 / 448 of it squared is above 2^-150: float32 holds 2^-149."""
    root = np.full(128, 1e-44, np.float32)
    root[0] = top
    q, s = X.state_to_f8(root, np.zeros(128, np.uint32), True)
    held = q * np.repeat(s, 128)
    assert np.all(held[1:] == np.float32(2.0**-9) * s[0]) and np.all(held * held * np.float32(beta2) > 0)


# ---------------------------------------------------------------------------------------------- refusals of the ABI


def _s(ds, tokens=6, top_k=2, experts=3, align=128, rows=None, **other):
    rows = X.rows_needed(tokens, top_k, experts, align) if rows is None else rows
    d = dict(offsets=1 << 30, counts=(1 << 30) + 4096, position=(1 << 30) + 8192, slot=1 << 31, tokens=tokens, rows=rows,
             top_k=top_k, experts=experts, align=align)
    d.update(other)
    return ds.ds_expert_slots(**d)


def test_rows(ds):
    assert ds.ds_expert_rows(6, 2, 3, 128) == X.rows_needed(6, 2, 3, 128) == 384
    assert ds.ds_expert_rows(0, 2, 3, 128) == 0 and ds.ds_expert_rows(1, 1, 1024, 16) == 16
    for bad in ((-1, 1, 1, 1), (1, 0, 1, 1), (1, 1, 0, 1), (1, 1, 1025, 1), (1, 1, 1, 0), (1, 1, 1, (1 << 20) + 1),
                (1 << 31, 1, 1, 1), (1 << 30, 2, 1, 1), ((1 << 31) - 300, 1, 1024, 1 << 20)):
        assert ds.ds_expert_rows(*bad) == -1


@pytest.mark.parametrize("change,status", [
    (dict(offsets=None), "INVALID_ARG"), (dict(counts=None), "INVALID_ARG"), (dict(position=None), "INVALID_ARG"),
    (dict(slot=None), "INVALID_ARG"), (dict(offsets=(1 << 30) + 2), "ALIGNMENT"), (dict(slot=(1 << 31) + 1), "ALIGNMENT"),
    (dict(rows=383), "BUFFER_TOO_SMALL"), (dict(rows=-1), "SHAPE"), (dict(tokens=-1, rows=0), "SHAPE"),
    (dict(top_k=0, rows=0), "SHAPE"), (dict(experts=0, rows=0), "SHAPE"), (dict(align=0, rows=0), "SHAPE"),
    (dict(experts=1025, rows=1 << 20), "UNSUPPORTED"), (dict(tokens=1 << 31, rows=1 << 30), "UNSUPPORTED"),
    (dict(rows=1 << 31), "UNSUPPORTED"), (dict(align=(1 << 20) + 128, rows=1 << 30), "UNSUPPORTED")])
def test_bad_slots_are_refused(ds, change, status):
    L, s, want = ds.lib(), _s(ds, **change), getattr(ds, "DS_ERR_" + status)
    x, w = _m(ds, 384, 256, 1 << 40), _m(ds, 3 * 128, 256, 1 << 42, blocks=1)
    assert L.ds_expert_order(1 << 35, 1, s, None) == want
    assert L.ds_expert_gather(1 << 40, 1, 256, 256, s, 1 << 45, 256, None) == want
    assert L.ds_expert_gather_f8(_m(ds, 6, 256), s, x, None) == want
    assert L.ds_expert_combine(1 << 40, 1, 256, 256, s, None, None, 0, 1 << 45, 256, None) == want
    assert L.ds_expert_combine_backward(1 << 40, 256, 1 << 41, 256, 1, 256, s, None, 1 << 45, 256, None, None) == want
    assert L.ds_expert_linear_f8(x, w, s, None, 1 << 45, 1, 128, None) == want
    assert L.ds_expert_weight_grad_f8(_m(ds, 128, 384, 1 << 40), _m(ds, 256, 384, 1 << 41), s, None, 0, 1 << 45, 256, None) == want
    assert ds.ds_last_error()
    assert L.ds_expert_order(1 << 35, 1, None, None) == ds.DS_ERR_INVALID_ARG


def test_bad_orders_are_refused(ds):
    L, s = ds.lib(), _s(ds)
    assert L.ds_expert_order(None, 1, s, None) == ds.DS_ERR_INVALID_ARG
    assert L.ds_expert_order(1 << 35, 2, s, None) == ds.DS_ERR_INVALID_ARG
    assert L.ds_expert_order((1 << 35) + 4, 1, s, None) == ds.DS_ERR_ALIGNMENT
    assert L.ds_expert_order((1 << 35) + 2, 0, s, None) == ds.DS_ERR_ALIGNMENT
    assert L.ds_expert_order(1 << 31, 1, s, None) == ds.DS_ERR_INVALID_ARG and "overlaps" in ds.ds_last_error()
    assert L.ds_expert_order(1 << 35, 1, _s(ds, counts=1 << 30), None) == ds.DS_ERR_INVALID_ARG


def test_bad_gathers_are_refused(ds):
    L, s = ds.lib(), _s(ds)
    call = lambda x=1 << 40, t=1, ldx=256, cols=256, out=1 << 45, ldo=256: L.ds_expert_gather(x, t, ldx, cols, s, out, ldo, None)  # noqa: E731
    assert call(x=None) == call(out=None) == call(t=3) == ds.DS_ERR_INVALID_ARG
    assert call(ldx=255) == call(ldo=255) == call(cols=-1) == ds.DS_ERR_SHAPE
    assert call(x=(1 << 40) + 1) == call(t=0, out=(1 << 45) + 2) == ds.DS_ERR_ALIGNMENT
    assert call(out=(1 << 40) + 512) == call(out=1 << 31) == ds.DS_ERR_INVALID_ARG  # over x, over slot
    assert call(cols=1 << 31) == ds.DS_ERR_UNSUPPORTED
    x, out = _m(ds, 6, 256), _m(ds, 384, 256, 1 << 40)
    f8 = lambda x=x, out=out: L.ds_expert_gather_f8(x, s, out, None)  # noqa: E731
    assert f8(x=None) == f8(out=None) == f8(x=_m(ds, 6, 256, blocks=1)) == f8(out=_m(ds, 384, 256, 1 << 40, blocks=1)) == ds.DS_ERR_INVALID_ARG
    assert f8(x=_m(ds, 7, 256)) == f8(out=_m(ds, 383, 256, 1 << 40)) == f8(out=_m(ds, 384, 255, 1 << 40)) == ds.DS_ERR_SHAPE
    assert f8(out=_m(ds, 384, 256, 1 << 40, format=1)) == f8(out=_m(ds, 384, 256)) == ds.DS_ERR_INVALID_ARG


def test_bad_combines_are_refused(ds):
    L, s = ds.lib(), _s(ds)

    def call(y=1 << 40, t=1, ldy=256, cols=256, w=1 << 35, add=None, ld_add=256, out=1 << 45, ldo=256):
        return L.ds_expert_combine(y, t, ldy, cols, s, w, add, ld_add, out, ldo, None)

    assert call(y=None) == call(out=None) == call(t=-1) == ds.DS_ERR_INVALID_ARG
    assert call(ldy=255) == call(ldo=255) == call(add=1 << 46, ld_add=255) == ds.DS_ERR_SHAPE
    assert call(w=(1 << 35) + 2) == call(add=(1 << 46) + 1) == ds.DS_ERR_ALIGNMENT
    assert call(out=1 << 40) == call(add=(1 << 45) + 2) == call(add=1 << 45, ld_add=257) == ds.DS_ERR_INVALID_ARG
    assert call(w=1 << 45) == ds.DS_ERR_INVALID_ARG

    def back(d=1 << 40, y=1 << 41, cols=256, ldy=256, w=1 << 35, dy=1 << 45, lddy=256, dw=1 << 36):
        return L.ds_expert_combine_backward(d, 256, y, ldy, 1, cols, s, w, dy, lddy, dw, None)

    assert back(d=None) == back(y=None) == back(dy=None) == ds.DS_ERR_INVALID_ARG
    assert back(cols=0) == back(lddy=255) == back(ldy=255) == ds.DS_ERR_SHAPE
    assert back(dw=(1 << 36) + 1) == ds.DS_ERR_ALIGNMENT
    assert back(dy=1 << 40) == back(dy=(1 << 41) + 2) == back(dy=1 << 41, lddy=264) == back(dw=1 << 35) == ds.DS_ERR_INVALID_ARG


def test_bad_products_are_refused(ds):
    L, s = ds.lib(), _s(ds)
    x, w = _m(ds, 384, 256, 1 << 40), _m(ds, 3 * 128, 256, 1 << 42, blocks=1)

    def call(x=x, w=w, s=s, bias=None, y=1 << 45, t=1, ldy=128):
        return L.ds_expert_linear_f8(x, w, s, bias, y, t, ldy, None)

    assert call(x=None) == call(w=None) == call(y=None) == call(t=9) == ds.DS_ERR_INVALID_ARG
    assert call(x=_m(ds, 383, 256, 1 << 40)) == call(w=_m(ds, 384, 255, 1 << 42)) == call(w=_m(ds, 385, 256, 1 << 42)) == ds.DS_ERR_SHAPE
    assert call(w=_m(ds, 3 * 100, 256, 1 << 42, blocks=1)) == ds.DS_ERR_SHAPE and "128" in ds.ds_last_error()
    assert call(ldy=127) == ds.DS_ERR_SHAPE
    assert call(x=_m(ds, 12, 256, 1 << 40, blocks=1), s=_s(ds, align=1)) == ds.DS_ERR_SHAPE  # tiles of several experts' rows
    assert call(bias=(1 << 35) + 2) == call(y=(1 << 45) + 1) == ds.DS_ERR_ALIGNMENT
    assert call(y=1 << 40) == call(bias=1 << 45) == ds.DS_ERR_INVALID_ARG
    d, xt = _m(ds, 128, 384, 1 << 40), _m(ds, 256, 384, 1 << 41)

    def grad(d=d, xt=xt, s=s, add=None, ld_add=256, dw=1 << 45, lddw=256):
        return L.ds_expert_weight_grad_f8(d, xt, s, add, ld_add, dw, lddw, None)

    assert grad(d=None) == grad(xt=None) == grad(dw=None) == ds.DS_ERR_INVALID_ARG
    assert grad(d=_m(ds, 128, 256, 1 << 40)) == grad(xt=_m(ds, 256, 400, 1 << 41)) == grad(lddw=255) == ds.DS_ERR_SHAPE
    assert L.ds_expert_weight_grad_f8(_m(ds, 128, 12, 1 << 40), _m(ds, 256, 12, 1 << 41), _s(ds, align=1), None, 0, 1 << 45, 256, None) == ds.DS_ERR_SHAPE
    assert grad(add=1 << 46, ld_add=255) == ds.DS_ERR_SHAPE
    assert grad(add=(1 << 45) + 4) == grad(add=1 << 45, ld_add=260) == grad(dw=1 << 40) == ds.DS_ERR_INVALID_ARG
    assert grad(dw=(1 << 45) + 2) == ds.DS_ERR_ALIGNMENT


def _t(ds, n=1000, at=1 << 40, **other):
    d = dict(p=at, g=at + (1 << 30), m=at + (1 << 31), v=at + (3 << 30), n=n, weight_decay=0.1)
    d.update(other)
    return ds.ds_adamw_tensor(**d)


def _o(ds, **other):
    return ds.ds_adamw_options(**{**dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1), **other})


def test_bad_optimizer_steps_are_refused(ds):
    L = ds.lib()

    def call(*tensors, count=None, options=None, **o):
        arr = (ds.ds_adamw_tensor * max(1, len(tensors)))(*tensors)
        return L.ds_adamw(arr, len(tensors) if count is None else count, options or _o(ds, **o), None)

    t = _t(ds)
    assert call(t, count=-1) == ds.DS_ERR_SHAPE
    assert L.ds_adamw(None, 1, _o(ds), None) == L.ds_adamw((ds.ds_adamw_tensor * 1)(t), 1, None, None) == ds.DS_ERR_INVALID_ARG
    for o in (dict(beta1=1.0), dict(beta2=-0.1), dict(beta1=float("nan")), dict(eps=-1.0), dict(eps=float("nan")), dict(step=0),
              dict(lr=-1.0), dict(lr=float("nan"))):
        assert call(t, **o) == ds.DS_ERR_INVALID_ARG, o
    assert call(t, step_dev=12) == call(t, grad_scale=2) == call(t, lr_dev=2) == ds.DS_ERR_ALIGNMENT
    for bad in (dict(p=None), dict(g=None), dict(m=None), dict(v=None), dict(p_type=3), dict(g_type=-1), dict(weight_decay=-0.1),
                dict(copy=1 << 50, copy_type=7), dict(m_scale=1 << 51), dict(v_scale=1 << 51)):
        assert call(_t(ds, **bad)) == ds.DS_ERR_INVALID_ARG, bad
    assert call(_t(ds, n=-1)) == ds.DS_ERR_SHAPE
    assert call(_t(ds, n=(1 << 40) + 1)) == ds.DS_ERR_UNSUPPORTED
    for bad in (dict(p=(1 << 40) + 2), dict(g=(1 << 41) + 1, g_type=1), dict(m=(1 << 42) + 3), dict(copy=(1 << 50) + 1, copy_type=1)):
        assert call(_t(ds, **bad)) == ds.DS_ERR_ALIGNMENT, bad
    eight = dict(m_scale=1 << 51, v_scale=1 << 52)
    assert call(t, _t(ds, at=1 << 44, **eight)) == ds.DS_ERR_INVALID_ARG and "kind" in ds.ds_last_error()
    # memory that is written overlaps nothing: the same tensor twice, p and g, one tensor's end and another's start, the
    # scales, a copy, what the options point to
    assert call(t, t) == ds.DS_ERR_INVALID_ARG and "overlaps" in ds.ds_last_error()
    for bad in ((_t(ds, g=1 << 40),), (t, _t(ds, at=1 << 44, p=(1 << 40) + 3996)), (_t(ds, m=(1 << 40) - 4),),
                (_t(ds, **{**eight, "v_scale": (1 << 51) + 28}),), (_t(ds, copy=(1 << 40) + (1 << 30)),),
                (t, _t(ds, at=1 << 44, g=1 << 40))):
        assert call(*bad) == ds.DS_ERR_INVALID_ARG and "overlaps" in ds.ds_last_error()
    assert call(t, grad_scale=(1 << 40) + 8) == call(t, step_dev=(1 << 40) + (1 << 31)) == ds.DS_ERR_INVALID_ARG


def test_nothing_to_do_needs_no_memory(ds):
    """Zero tokens and empty tensors launch nothing where nothing is written (there is no GPU here)."""
    L, s = ds.lib(), _s(ds, tokens=0, position=None, slot=None)
    none = dict(q=None, scale=None)
    assert L.ds_expert_gather(None, 1, 256, 256, s, None, 256, None) == ds.DS_OK
    assert L.ds_expert_gather_f8(_m(ds, 0, 256, **none), s, _m(ds, 0, 256, **none), None) == ds.DS_OK
    assert L.ds_expert_combine(None, 1, 256, 256, s, None, None, 0, None, 256, None) == ds.DS_OK
    assert L.ds_expert_combine_backward(None, 256, None, 256, 1, 256, s, None, None, 256, None, None) == ds.DS_OK
    assert L.ds_expert_linear_f8(_m(ds, 0, 256, **none), _m(ds, 384, 256), s, None, None, 1, 128, None) == ds.DS_OK
    assert L.ds_adamw(None, 0, _o(ds), None) == ds.DS_OK
    assert L.ds_adamw((ds.ds_adamw_tensor * 1)(_t(ds, n=0, p=None, g=None, m=None, v=None)), 1, _o(ds), None) == ds.DS_OK


def test_struct_layouts(ds):
    L = ds.lib()
    for which, st, size in ((3, ds.ds_expert_slots, 64), (4, ds.ds_adamw_tensor, 80), (5, ds.ds_adamw_options, 72)):
        assert L.ds_abi_struct_size(which) == ctypes.sizeof(st) == size


# ------------------------------------------------------------------------------------------------------------ helpers


@pytest.fixture()
def first_gpu(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)


class Gpu(OnSecondGpu):
    """What the helpers ask of a tensor on cuda:`device`."""

    def __init__(self, *shape, dtype=torch.bfloat16, device=0):
        super().__init__(*shape, dtype=dtype)
        self.index = device
        self.device = torch.device("cuda", device)

    def get_device(self):
        return self.index

    def numel(self):
        return int(np.prod(self.shape))


def _expert_order(ds, device=0, tokens=6, top_k=2, experts=3, align=128, rows=384):
    i = lambda *s: Gpu(*s, dtype=torch.int32, device=device)  # noqa: E731
    return ds.ExpertOrder(i(experts + 1), i(experts), i(tokens, top_k), i(rows), align=align)


def _f8(ds, rows, cols, device=0, tiles=False):
    return ds.F8Matrix(Gpu(rows, cols, dtype=torch.float8_e4m3fn, device=device),
                       Gpu(-(-rows // 128) if tiles else rows, -(-cols // 128), dtype=torch.float32, device=device), tiles)


def test_tensors_of_another_gpu_are_refused(ds, first_gpu):
    there, here = _expert_order(ds, 1), _expert_order(ds)
    f = lambda *s, device=1: Gpu(*s, dtype=torch.float32, device=device)  # noqa: E731
    for call in (lambda: ds.expert_order(Gpu(6, 2, dtype=torch.int64, device=1), 3), lambda: ds.expert_gather(f(6, 256), there),
                 lambda: ds.expert_gather(_f8(ds, 6, 256, 1), there), lambda: ds.expert_combine(f(384, 256), there),
                 lambda: ds.expert_combine_backward(f(6, 256), None, there), lambda: ds.expert_linear_f8(_f8(ds, 384, 256, 1), _f8(ds, 384, 256, 1), there),
                 lambda: ds.expert_weight_grad_f8(_f8(ds, 128, 384, 1), _f8(ds, 256, 384, 1), there), lambda: ds.AdamW([f(5)], [f(5)])):
        with pytest.raises(ValueError, match="is on cuda:1, the current device is cuda:0"):
            call()
    g = lambda *s: f(*s, device=0)  # noqa: E731
    for call in (lambda: ds.expert_gather(g(6, 256), there), lambda: ds.expert_combine(g(384, 256), there),
                 lambda: ds.expert_combine(g(384, 256), here, weights=f(6, 2)), lambda: ds.expert_combine(g(384, 256), here, add=f(6, 256)),
                 lambda: ds.expert_combine_backward(g(6, 256), f(384, 256), here, weights=g(6, 2)),
                 lambda: ds.expert_linear_f8(_f8(ds, 384, 256), _f8(ds, 384, 256, 1), here),
                 lambda: ds.expert_linear_f8(_f8(ds, 384, 256), _f8(ds, 384, 256), here, bias=f(3, 128), out=g(384, 128)),
                 lambda: ds.expert_weight_grad_f8(_f8(ds, 128, 384), _f8(ds, 256, 384, 1), here)):
        with pytest.raises(ValueError, match="cuda:1"):
            call()


def test_helpers_refuse_what_the_abi_cannot_see(ds, first_gpu):
    order = _expert_order(ds)
    f = lambda *s, dtype=torch.float32: Gpu(*s, dtype=dtype)  # noqa: E731
    i = lambda *s: f(*s, dtype=torch.int32)  # noqa: E731
    bad = [lambda: ds.expert_order(f(6, 2), 3), lambda: ds.expert_order(i(6), 3), lambda: ds.expert_order(i(6, 2), 0),
           lambda: ds.expert_order(i(6, 2), 3, align=0), lambda: ds.expert_order(torch.zeros((6, 2), dtype=torch.int64), 3),
           lambda: ds.expert_gather(f(7, 256), order), lambda: ds.expert_gather(f(6, 256, dtype=torch.float64), order),
           lambda: ds.expert_gather(f(6, 256), "order"), lambda: ds.expert_gather(_f8(ds, 7, 256), order),
           lambda: ds.expert_gather(_f8(ds, 6, 256, tiles=True), order), lambda: ds.expert_gather(_f8(ds, 6, 256), order, out=_f8(ds, 384, 256, tiles=True)),
           lambda: ds.expert_gather(f(6, 256), order, out=_f8(ds, 384, 256)), lambda: ds.expert_gather(_f8(ds, 6, 256), order, out=f(384, 256)),
           lambda: ds.expert_gather(f(6, 256), order, out=f(384, 255)), lambda: ds.expert_gather(f(6, 256), order, out=f(384, 256, dtype=torch.float16)),
           lambda: ds.expert_combine(f(383, 256), order), lambda: ds.expert_combine(f(384, 256), order, weights=f(6, 3)),
           lambda: ds.expert_combine(f(384, 256), order, weights=f(6, 2, dtype=torch.bfloat16)),
           lambda: ds.expert_combine(f(384, 256), order, add=f(6, 255)), lambda: ds.expert_combine(f(384, 256), order, out=f(5, 256)),
           lambda: ds.expert_combine_backward(f(5, 256), f(384, 256), order, f(6, 2)), lambda: ds.expert_combine_backward(f(6, 256), None, order, f(6, 2)),
           lambda: ds.expert_combine_backward(f(6, 256), f(384, 256, dtype=torch.float16), order, f(6, 2)),
           lambda: ds.expert_linear_f8(f(384, 256), _f8(ds, 384, 256), order), lambda: ds.expert_linear_f8(_f8(ds, 384, 256), _f8(ds, 384, 256), order, dtype=torch.int8),
           lambda: ds.expert_linear_f8(_f8(ds, 384, 256), _f8(ds, 384, 256), order, bias=f(128), out=f(384, 128)),
           lambda: ds.expert_linear_f8(_f8(ds, 384, 256), _f8(ds, 384, 256), order, out=f(384, 129)),
           lambda: ds.expert_weight_grad_f8(_f8(ds, 128, 384), _f8(ds, 256, 384), order, add=f(3, 128, 255)),
           lambda: ds.expert_weight_grad_f8(_f8(ds, 128, 384), _f8(ds, 256, 384), order, out=f(3, 128, 256, dtype=torch.float16)),
           lambda: ds.ExpertOrder(i(1), i(0), i(6, 2), i(12)), lambda: ds.ExpertOrder(i(4), i(4), i(6, 2), i(12)),
           lambda: ds.ExpertOrder(i(4), i(3), i(12), i(12)), lambda: ds.ExpertOrder(f(4), i(3), i(6, 2), i(12))]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("passed:", k)
    with pytest.raises(ds.DsError):
        ds.expert_order(i(6, 2), 1025)


def test_tensors_of_an_order_cannot_be_replaced(ds, first_gpu):
    """Its descriptor holds their addresses: another tensor would be passed over, and the memory of the first one lost."""
    order = _expert_order(ds)
    for name in ("offsets", "counts", "position", "slot"):
        held = getattr(order, name)
        with pytest.raises(AttributeError):
            setattr(order, name, Gpu(*held.shape, dtype=torch.int32))
        assert getattr(order, name) is held


def test_optimizer_refuses_before_any_launch(ds, first_gpu, monkeypatch):
    monkeypatch.setattr(torch.Tensor, "data_ptr", lambda t: t.data_ptr())
    f = lambda *s, dtype=torch.float32, device=0: Gpu(*s, dtype=dtype, device=device)  # noqa: E731
    p, g, m, v = f(300), f(300), f(300), f(300)
    q, s = f(300, dtype=torch.float8_e4m3fn), f(3)
    ok = ds.AdamW([p], [g], m=[m], v=[v])
    assert ok.steps == 0 and len(ok.params) == 1
    ds.AdamW([p], [g], m=[(q, s)], v=[(q, s)])  # the overlap is seen by the call
    for bad in (dict(params=[]), dict(grads=[]), dict(grads=[f(299)]), dict(grads=[f(300, dtype=torch.int32)]), dict(grads=[f(300, device=1)]),
                dict(m=[f(299)]), dict(m=[f(300, dtype=torch.float16)]), dict(m=[(q, f(2))]), dict(m=[(p, s)]), dict(m=[m, m]), dict(v=[]),
                dict(copies=[f(299)]), dict(copies=[q]), dict(copies=[]), dict(weight_decay=[0.1, 0.1]), dict(state_dtype=torch.float16)):
        with pytest.raises(ValueError):
            ds.AdamW(**{**dict(params=[p], grads=[g], m=[m], v=[v]), **bad})
    for bad in (dict(grads=[g, g]), dict(grads=[f(299)])):
        with pytest.raises(ValueError):
            ok.step(**bad)
    assert ok.grads == [g] and ok.steps == 0


def test_optimizer_refuses_memory_that_was_replaced(ds, first_gpu, monkeypatch):
    """A parameter, gradient or copy that lies elsewhere than it did, with the step's own gradients or with new ones."""
    monkeypatch.setattr(torch.Tensor, "data_ptr", lambda t: t.data_ptr())
    monkeypatch.setattr(ds.optimizer, "lib", None)  # nothing is launched

    class At(Gpu):
        at = 0

        def data_ptr(self):
            return self.at

    def moved(which, grads):
        tensors = []
        for k in range(6):
            tensors.append(At(300, dtype=torch.bfloat16 if k == 4 else torch.float32))
            tensors[k].at = (k + 1) << 40
        p, g, m, v, c, new = tensors
        opt = ds.AdamW([p], [g], m=[m], v=[v], copies=[c])
        tensors[which].at += 1 << 30
        with pytest.raises(ValueError, match="other memory"):
            opt.step([new] if grads else None)
        assert opt.steps == 0 and opt.grads == [g]

    for which, grads in ((0, False), (0, True), (1, False), (4, False), (4, True)):
        moved(which, grads)


def test_weight_decay_of_a_block_is_any_number(ds, monkeypatch):
    """One number of any type for all weights but the norm's, or one for each."""
    from paper_1905_13298_gb300 import feed_forward
    monkeypatch.setattr(feed_forward, "AdamW", lambda params, grads, weight_decay, **options: weight_decay)
    block = feed_forward.GatedFeedForward.__new__(feed_forward.GatedFeedForward)
    block.norm, block.gate_up, block.down = "norm", "gate_up", "down"
    grads = dict.fromkeys(block.masters())
    for number in (0.5, 1, np.float32(0.5), np.int64(1)):
        assert block.adamw(grads, weight_decay=number) == [0.0, number, number]
    assert block.adamw(grads) == [0.0, 0.01, 0.01]
    assert block.adamw(grads, weight_decay=[0.1, 0.2, 0.3]) == [0.1, 0.2, 0.3]

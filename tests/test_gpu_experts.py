"""Experts: gate, sort, gather, combine and their gradients against direct statements in doubles, and all of them in a row.

Tolerances.  A softmax weight in fp32: two exponentials off by at most 2 units of 2^-23, a sum of at most E terms of one sign (E additions,
2^-24 each), a division: (E + 8) * 2^-23 relative.  A gradient p (g - sum g p) adds a sum of at most k products: absolute
(2 E + k + 16) * 2^-23 * max|g|.  A combination of k rows: k fused multiply-adds of 2^-24 of the running sum of magnitudes each; a dot
product of D terms likewise.  Half a step of the output type comes on top of each."""
import numpy as np
import pytest

import packed_rows as pr

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF_STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
TINY = {"fp32": 0.0, "bf16": 0.0, "fp16": 2.0 ** -25}       # half a step of the smallest numbers


@pytest.fixture(scope="module")
def env():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2402_03694_b200 import build, binding as sf
    build.build()
    ctx = sf.sf_ctx_create(0, 0)
    yield sf, ctx
    sf.sf_ctx_poll(ctx, raise_on_error=False)
    sf.sf_ctx_destroy(ctx)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def num(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


# ---- gate -----------------------------------------------------------------------------------------------------
def gate_reference(x, k, mode):
    """Row by row: ids, weights and the weights of all experts (the softmax that the gradient needs)."""
    n, E = x.shape
    ids, w, full = np.full((n, k), -1), np.zeros((n, k)), np.zeros((n, E))
    for r in range(n):
        real = [e for e in range(E) if x[r, e] > -np.inf]            # False for NaN
        order = sorted(real, key=lambda e: (-x[r, e], e))[:k]
        base = {}
        if mode == 2:
            base = {e: x[r, e] for e in order}
        elif real:
            m = x[r, order[0]]
            base = {e: 1.0 if x[r, e] == m else np.exp(x[r, e] - m) for e in (real if mode == 0 else order)}
        total = sum(base.values())
        if total > 0:
            for e, b in base.items():
                full[r, e] = b / total
        for j, e in enumerate(order):
            ids[r, j] = e
            w[r, j] = full[r, e]
    return ids, w, full


def gate_gradient(x, ids, full, g, mode):
    n, E = x.shape
    d = np.zeros((n, E))
    for r in range(n):
        at = {e: g[r, j] for j, e in enumerate(ids[r]) if e >= 0}
        mean = sum(v * full[r, e] for e, v in at.items())
        if mode == 2:
            total = sum(x[r, e] for e in at)
            for e, v in at.items():
                d[r, e] = (v - mean) / total if total > 0 else 0.0
        else:
            for e in range(E):
                d[r, e] = full[r, e] * (at.get(e, 0.0) - mean)
    return d


def gate_scores(rng, n, E, mode, kind):
    x = rng.normal(size=(n, E)) * 2
    if mode == 2:
        x = np.exp(x) / np.exp(x).sum(-1, keepdims=True)
    x[rng.random((n, E)) < 0.15] = -np.inf
    if n > 3:
        x[1] = -np.inf                                   # nothing left
        x[2] = x[2, 0] if np.isfinite(x[2, 0]) else 0.5  # all the same: the lowest indices
        x[3, rng.random(E) < 0.5] = np.nan
    if n > 5:
        x[4] = -1.0                                      # shares of a sum that is not positive
        x[5, rng.random(E) < 0.5] = float(torch.finfo(TYPES[kind]).min)
    t = torch.from_numpy(x).to(TYPES[kind])
    return t, t.double().numpy()


@pytest.mark.parametrize("mode", [0, 1, 2])
@pytest.mark.parametrize("n,E,k,kind", [(1, 1, 1, "fp32"), (10, 8, 2, "fp32"), (200, 16, 2, "bf16"), (77, 3, 3, "fp16"), (65, 17, 5, "fp32"), (300, 5, 1, "bf16"),
                                        (40, 64, 8, "fp32"), (33, 128, 40, "fp16"), (21, 200, 200, "fp32"), (9, 1000, 6, "bf16"), (70, 32, 32, "fp32"), (50, 4, 2, "fp16")])
def test_gate_and_its_gradient(env, n, E, k, kind, mode):
    sf, ctx = env
    rng = np.random.default_rng(n + E * 10 + k)
    t, x = gate_scores(rng, n, E, mode, kind)
    g = rng.normal(size=(n, k)).astype(np.float32)
    want_ids, want_w, full = gate_reference(x, k, mode)
    want_d = gate_gradient(x, want_ids, full, g.astype(float), mode)
    for ld, at in ((E, 0), (E + 3, 1), (-(-E // 8) * 8 + 8, 8)):
        base = torch.full((n, ld + at), 99.0, dtype=TYPES[kind], device="cuda")
        base[:, at:at + E] = t.cuda()
        scores = base[:, at:at + E]
        ids, w = torch.full((n, k), 77, dtype=torch.int32, device="cuda"), torch.full((n, k), 77.0, device="cuda")
        sf.sf_expert_gate(ctx, scores, mode, ids, w)
        assert np.array_equal(num(ids), want_ids)
        err = np.abs(num(w) - want_w)
        assert (err <= (E + 8) * 2.0 ** -23 * want_w + 2.0 ** -126).all(), err.max()
        d = torch.full((n, ld + at), 5.0, dtype=TYPES[kind], device="cuda")
        sf.sf_expert_gate_backward(ctx, scores, mode, ids, dev(g), d[:, at:at + E])
        got = num(d[:, at:at + E])
        scale = np.abs(g).max()
        if mode == 2:                                    # (g - mean) / total: relative to 1 / total
            total = np.array([sum(x[r, e] for e in want_ids[r] if e >= 0) for r in range(n)])
            scale = scale / np.where(total > 0, total, 1.0)[:, None]
        tol = (2 * E + k + 16) * 2.0 ** -23 * scale
        err = np.abs(got - want_d)
        assert (err <= tol + HALF_STEP[kind] * (np.abs(want_d) + tol) + TINY[kind]).all(), err.max()
        assert (d[:, :at] == 5).all() and (d[:, at + E:] == 5).all()


@pytest.mark.parametrize("mode", [1, 2])
@pytest.mark.parametrize("E,k,kind", [(5, 1, "fp32"), (12, 1, "bf16"), (9, 6, "fp16"), (40, 9, "fp32")])
def test_gate_gradient_of_a_lone_pick_is_nothing(env, E, k, kind, mode):
    """One picked expert has weight 1 whatever its score, small ones too: its gradient is 0, not a rounding divided by the score."""
    sf, ctx = env
    rng = np.random.default_rng(E)
    n = 500
    x = np.full((n, E), -np.inf)
    x[np.arange(n), rng.integers(0, E, n)] = 10.0 ** rng.uniform(-4, 0, n)
    if k == 1:
        x = np.where(np.isinf(x), 10.0 ** rng.uniform(-4, 0, (n, E)), x)
    t = torch.from_numpy(x).to(TYPES[kind]).cuda()
    ids, w, d = torch.zeros(n, k, dtype=torch.int32, device="cuda"), torch.zeros(n, k, device="cuda"), torch.full((n, E), 7.0, dtype=TYPES[kind], device="cuda")
    sf.sf_expert_gate(ctx, t, mode, ids, w)
    assert (w[:, 0] == 1).all() and (w[:, 1:] == 0).all()
    sf.sf_expert_gate_backward(ctx, t, mode, ids, torch.randn(n, k, device="cuda"), d)
    assert (d == 0).all()


@pytest.mark.parametrize("mode", [0, 1, 2])
def test_gate_gradient_against_differences(env, mode):
    """Central differences of the reference gate in doubles, far from a change of the picks."""
    sf, ctx = env
    rng = np.random.default_rng(mode)
    n, E, k = 6, 7, 3
    x = np.stack([rng.permutation(E) for _ in range(n)]) * 0.7 + 0.3
    g = rng.normal(size=(n, k))
    x32, g32 = x.astype(np.float32), g.astype(np.float32)
    ids, d = torch.zeros(n, k, dtype=torch.int32, device="cuda"), torch.zeros(n, E, device="cuda")
    sf.sf_expert_gate(ctx, dev(x32), mode, ids, torch.zeros(n, k, device="cuda"))
    sf.sf_expert_gate_backward(ctx, dev(x32), mode, ids, dev(g32), d)
    loss = lambda v: (gate_reference(v, k, mode)[1] * g32).sum()  # noqa: E731
    h, num_d = 1e-5, np.zeros((n, E))
    for r in range(n):
        for e in range(E):
            hi, lo = x32.astype(float), x32.astype(float)
            hi[r, e] += h
            lo[r, e] -= h
            num_d[r, e] = (loss(hi) - loss(lo)) / (2 * h)
    # the difference itself is off by h^2 times a third derivative (below 10 here) and by 1e-16 / h
    assert np.abs(num(d) - num_d).max() < 1e-9 + 1e-10 + (2 * E + k + 16) * 2.0 ** -23 * np.abs(g).max() / min(1.0, x32.min() * k)


def test_gate_infinite_scores_and_device_count(env):
    sf, ctx = env
    x = torch.tensor([[1.0, float("inf"), 2.0, float("inf")], [0.0, 1.0, 2.0, 3.0], [5.0, 1.0, 2.0, 3.0]], device="cuda")
    ids, w = torch.full((3, 3), 9, dtype=torch.int32, device="cuda"), torch.full((3, 3), 9.0, device="cuda")
    sf.sf_expert_gate(ctx, x, sf.SF_GATE_SOFTMAX, ids, w, n_dev=torch.tensor([2], dtype=torch.int32, device="cuda"))
    assert ids.tolist() == [[1, 3, 2], [3, 2, 1], [9, 9, 9]]
    assert w[0].tolist() == [0.5, 0.5, 0.0] and (w[2] == 9).all()
    d = torch.full((3, 4), 9.0, device="cuda")
    sf.sf_expert_gate_backward(ctx, x, sf.SF_GATE_SOFTMAX, ids, torch.ones(3, 3, device="cuda"), d, n_dev=torch.tensor([1], dtype=torch.int32, device="cuda"))
    assert (d[0] == 0).all() and (d[1:] == 9).all()
    sf.sf_expert_gate(ctx, x, sf.SF_GATE_SOFTMAX, ids, w, n_dev=torch.tensor([0], dtype=torch.int32, device="cuda"))
    sf.sf_ctx_poll(ctx)


# ---- sort ------------------------------------------------------------------------------------------------------
def sort_reference(ids, E, align, capacity):
    n, k = ids.shape
    offsets, counts, rows, at = [0], [], [], np.full((n, k), -1)
    flow_of_row = np.full(capacity, -7)
    first = 0
    for e in range(E):
        pairs = [(f, j) for f, j in zip(*np.nonzero(ids == e))]
        for i, (f, j) in enumerate(pairs):
            if first + i < capacity:
                at[f, j], flow_of_row[first + i] = first + i, f
        end = first + -(-len(pairs) // align) * align
        flow_of_row[min(first + len(pairs), capacity):min(end, capacity)] = -1
        counts.append(min(len(pairs), capacity - min(first, capacity)))
        first = end
        offsets.append(min(first, capacity))
    return np.array(offsets), np.array(counts), flow_of_row, at


def sort(sf, ctx, ids, E, align, cap, **kw):
    n, k = ids.shape
    out = [torch.full(s, -7, dtype=torch.int32, device="cuda") for s in ((E + 1,), (E,), (cap,), (n, k))]
    work = torch.full((max(1, sf.sf_expert_sort_workspace(n, k, E) // 4),), -5, dtype=torch.int32, device="cuda")
    sf.sf_expert_sort(ctx, ids, E, align, *out, work, **kw)
    return out


def some_ids(rng, n, k, E, skew=1.0):
    p = np.exp(rng.normal(size=E) * skew)
    ids = rng.choice(E, size=(n, k), p=p / p.sum()).astype(np.int32)
    ids[rng.random((n, k)) < 0.05] = -1
    ids[rng.random((n, k)) < 0.01] = E
    return ids


@pytest.mark.parametrize("n,k,E,align", [(1, 1, 1, 1), (10, 1, 8, 128), (13, 3, 5, 16), (700, 2, 16, 1), (2048, 2, 3, 128), (4096, 1, 40, 64), (4097, 1, 40, 64),
                                         (20011, 2, 8, 128), (3000, 7, 1024, 4), (200001, 1, 256, 1), (400000, 2, 2, 128), (50000, 2, 1000, 8)])
def test_sort(env, n, k, E, align):
    sf, ctx = env
    ids = some_ids(np.random.default_rng(n + k + E), n, k, E)
    cap = n * k + E * (align - 1)
    want = sort_reference(ids, E, align, cap)
    for got, ref in zip(sort(sf, ctx, dev(ids), E, align, cap), want):
        assert np.array_equal(num(got), ref)
    sf.sf_ctx_poll(ctx)


@pytest.mark.parametrize("n,k,E,align,cap", [(50, 2, 4, 16, 40), (9000, 1, 6, 128, 5000), (9000, 1, 6, 128, 1), (20, 1, 3, 8, 0)])
def test_sort_cut_at_the_capacity(env, n, k, E, align, cap):
    sf, ctx = env
    ids = some_ids(np.random.default_rng(n), n, k, E, 0.3)
    sf.sf_ctx_poll(ctx, reset=True)
    for got, ref in zip(sort(sf, ctx, dev(ids), E, align, cap), sort_reference(ids, E, align, cap)):
        assert np.array_equal(num(got), ref)
    with pytest.raises(sf.SfError) as e:
        sf.sf_ctx_poll(ctx, reset=True)
    assert e.value.status == sf.SF_ERR_CAPACITY


def test_sort_device_count_and_nothing_to_sort(env):
    sf, ctx = env
    ids = some_ids(np.random.default_rng(1), 6000, 2, 9)
    for count in (0, 1, 4000, 6000):
        want = sort_reference(ids[:count], 9, 32, 13000)
        got = sort(sf, ctx, dev(ids), 9, 32, 13000, n_dev=torch.tensor([count], dtype=torch.int32, device="cuda"))
        for g, ref in zip(got[:3], want[:3]):
            assert np.array_equal(num(g), ref)
        assert np.array_equal(num(got[3])[:count], want[3]) and (num(got[3])[count:] == -7).all()
    none = np.full((100, 2), -1, np.int32)
    got = sort(sf, ctx, dev(none), 4, 128, 300)
    assert (num(got[0]) == 0).all() and (num(got[1]) == 0).all() and (num(got[2]) == -7).all() and (num(got[3]) == -1).all()
    got = sort(sf, ctx, dev(none[:0]), 4, 128, 300)
    assert (num(got[0]) == 0).all() and (num(got[1]) == 0).all()


# ---- gather, combine, gradients -------------------------------------------------------------------------------------
def plan(sf, ctx, rng, n, k, E, align, extra=5):
    ids = some_ids(rng, n, k, E)
    cap = n * k + E * (align - 1) + extra
    return sort(sf, ctx, dev(ids), E, align, cap), cap


def laid(x, kind, ld, at, fill=7.0):
    """x on the device with row pitch ld + at, first column at."""
    n, D = x.shape
    base = torch.full((n, ld + at), fill, dtype=TYPES[kind], device="cuda")
    base[:, at:at + D] = torch.from_numpy(x).to(TYPES[kind]).cuda()
    return base, base[:, at:at + D]


SHAPES = [(1, 1, 1, 1, 1), (10, 1, 8, 2048, 128), (13, 2, 8, 8, 16), (300, 2, 5, 100, 128), (257, 3, 4, 33, 1), (1500, 2, 16, 1024, 64), (5, 6, 9, 5000, 8), (3000, 1, 2, 3, 1), (40000, 2, 3, 17, 16), (9000, 3, 5, 50, 1), (7000, 1, 4, 114, 8)]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,k,E,D,align", SHAPES)
def test_gather_and_its_gradient(env, n, k, E, D, align, kind):
    sf, ctx = env
    rng = np.random.default_rng(n + D)
    (offsets, counts, flow_of_row, at), cap = plan(sf, ctx, rng, n, k, E, align)
    x = rng.normal(size=(n, D))
    flow, end, pairs = num(flow_of_row), int(offsets[-1]), num(at)
    for pad, first in ((0, 0), (16 - D % 8, 8), (3, 1)):
        _, xt = laid(x, kind, D + pad, first)
        base, rows = laid(np.full((cap, D), 7.0), kind, D + pad, first)
        sf.sf_expert_gather(ctx, xt, at, offsets, counts, rows)
        want = np.where((flow[:end] >= 0)[:, None], num(xt)[np.maximum(flow[:end], 0)], 0.0)
        assert np.array_equal(num(rows)[:end], want)
        assert (rows[end:] == 7).all() and (base[:, :first] == 7).all() and (base[:, first + D:] == 7).all()
        dr = rng.normal(size=(cap, D))
        dr[end:] = np.nan                                # rows that no pair has may hold anything
        _, drt = laid(dr, kind, D + pad, first)
        dbase, dx = laid(np.full((n, D), 7.0), kind, D + pad, first)
        sf.sf_expert_gather_backward(ctx, drt, at, dx)
        v = np.where((pairs >= 0)[..., None], np.nan_to_num(num(drt))[np.maximum(pairs, 0)], 0.0)
        slack = k * 2.0 ** -24 * np.abs(v).sum(1)
        err = np.abs(num(dx) - v.sum(1))
        assert (err <= slack + HALF_STEP[kind] * (np.abs(v.sum(1)) + slack) + TINY[kind]).all()
        assert (dbase[:, :first] == 7).all() and (dbase[:, first + D:] == 7).all()


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,k,E,D,align", SHAPES)
def test_combine_and_its_gradients(env, n, k, E, D, align, kind):
    sf, ctx = env
    rng = np.random.default_rng(n + D + 1)
    (offsets, counts, flow_of_row, at), cap = plan(sf, ctx, rng, n, k, E, align)
    pairs, end, flow = num(at), int(offsets[-1]), num(flow_of_row)
    real = pairs >= 0
    w = rng.random((n, k)).astype(np.float32)
    w[~real] = np.nan                                    # a pair without a row: its weight does not count
    rows = rng.normal(size=(cap, D))
    rows[end:] = np.nan
    for pad, first in ((0, 0), (16 - D % 8, 8), (3, 1)):
        _, rt = laid(rows, kind, D + pad, first)
        v = np.where(real[..., None], np.nan_to_num(num(rt))[np.maximum(pairs, 0)], 0.0)
        for weights in (w, None):
            ww = np.where(real, w if weights is not None else 1.0, 0.0).astype(float)
            base, y = laid(np.full((n, D), 7.0), kind, D + pad, first)
            sf.sf_expert_combine(ctx, rt, at, None if weights is None else dev(weights), y)
            want, mass = (ww[..., None] * v).sum(1), (np.abs(ww[..., None] * v)).sum(1)
            slack = (k + 1) * 2.0 ** -24 * mass
            assert (np.abs(num(y) - want) <= slack + HALF_STEP[kind] * (np.abs(want) + slack) + TINY[kind]).all()
            assert (base[:, :first] == 7).all() and (base[:, first + D:] == 7).all()
            _, dy = laid(rng.normal(size=(n, D)), kind, D + pad, first)
            g = num(dy)
            dbase, d_rows = laid(np.full((cap, D), 7.0), kind, D + pad, first)
            d_w = torch.full((n, k), 7.0, device="cuda")
            sf.sf_expert_combine_backward(ctx, dy, rt, at, None if weights is None else dev(weights), offsets, counts, d_rows, d_w)
            want_rows = np.zeros((end, D))
            f, j = np.nonzero(real)
            want_rows[pairs[f, j]] = ww[f, j, None] * g[f]
            tol = 2.0 ** -24 * np.abs(want_rows) + HALF_STEP[kind] * np.abs(want_rows) * (1 + 2.0 ** -24) + TINY[kind]
            assert (np.abs(num(d_rows)[:end] - want_rows) <= tol).all()
            assert (d_rows[end:] == 7).all() and (dbase[:, :first] == 7).all() and (dbase[:, first + D:] == 7).all()
            want_w = (g[:, None] * v).sum(-1)
            err = np.abs(num(d_w) - want_w)
            assert (err <= (D + 1) * 2.0 ** -24 * np.abs(g[:, None] * v).sum(-1)).all()
            only_w, only_rows = torch.zeros_like(d_w), torch.zeros_like(d_rows)
            sf.sf_expert_combine_backward(ctx, dy, rt, at, None if weights is None else dev(weights), offsets, counts, None, only_w)
            sf.sf_expert_combine_backward(ctx, dy, rt, at, None if weights is None else dev(weights), offsets, counts, only_rows, None)
            assert torch.equal(only_w, d_w) and torch.equal(only_rows[:end], d_rows[:end])


def test_gradients_against_differences(env):
    """The loss sum(c * y) of combine(gather(x)) with its weights, by central differences in doubles (it is bilinear: exact up to rounding)."""
    sf, ctx = env
    rng = np.random.default_rng(2)
    n, k, E, D = 5, 2, 3, 4
    (offsets, counts, flow_of_row, at), cap = plan(sf, ctx, rng, n, k, E, 4)
    pairs = num(at)
    x, w, c = rng.normal(size=(n, D)).astype(np.float32), rng.random((n, k)).astype(np.float32), rng.normal(size=(n, D)).astype(np.float32)
    rows = torch.zeros(cap, D, device="cuda")
    sf.sf_expert_gather(ctx, dev(x), at, offsets, counts, rows)
    d_rows, d_w, dx = torch.zeros_like(rows), torch.zeros(n, k, device="cuda"), torch.zeros(n, D, device="cuda")
    sf.sf_expert_combine_backward(ctx, dev(c), rows, at, dev(w), offsets, counts, d_rows, d_w)
    sf.sf_expert_gather_backward(ctx, d_rows, at, dx)

    def loss(xv, wv):
        return sum(c[f].astype(float) @ (wv[f, j] * xv[f]) for f in range(n) for j in range(k) if pairs[f, j] >= 0)
    h = 0.5
    for f in range(n):
        for i in range(D):
            hi, lo = x.astype(float), x.astype(float)
            hi[f, i] += h
            lo[f, i] -= h
            assert abs((loss(hi, w.astype(float)) - loss(lo, w.astype(float))) / (2 * h) - float(dx[f, i])) < 4e-6
        for j in range(k):
            hi, lo = w.astype(float), w.astype(float)
            hi[f, j] += h
            lo[f, j] -= h
            assert abs((loss(x.astype(float), hi) - loss(x.astype(float), lo)) / (2 * h) - float(d_w[f, j])) < 4e-6


def test_device_count_leaves_the_rest(env):
    sf, ctx = env
    rng = np.random.default_rng(3)
    n, k, E, D, m = 90, 2, 4, 24, 50
    cnt = torch.tensor([m], dtype=torch.int32, device="cuda")
    ids = some_ids(rng, n, k, E)
    cap = n * k + E * 15
    offsets, counts, flow, at = sort(sf, ctx, dev(ids), E, 16, cap, n_dev=cnt)
    at[m:] = 0                                           # stale rows of flows that are not there
    x = dev(rng.normal(size=(n, D)).astype(np.float32))
    rows = torch.full((cap, D), 7.0, device="cuda")
    sf.sf_expert_gather(ctx, x, at, offsets, counts, rows, n_dev=cnt)
    f, end = num(flow), int(offsets[-1])
    assert np.array_equal(num(rows)[:end], np.where((f[:end] >= 0)[:, None], num(x)[np.maximum(f[:end], 0)], 0.0)) and (rows[end:] == 7).all()
    w = torch.rand(n, k, device="cuda")
    for call in (lambda y: sf.sf_expert_combine(ctx, rows, at, w, y, n_dev=cnt), lambda y: sf.sf_expert_gather_backward(ctx, rows, at, y, n_dev=cnt)):
        y = torch.full((n, D), 7.0, device="cuda")
        call(y)
        assert (y[m:] == 7).all() and not (y[:m] == 7).all()
    d_rows, d_w = torch.full((cap, D), 7.0, device="cuda"), torch.full((n, k), 7.0, device="cuda")
    sf.sf_expert_combine_backward(ctx, x, rows, at, w, offsets, counts, d_rows, d_w, n_dev=cnt)
    assert (d_w[m:] == 7).all() and (d_rows[end:] == 7).all() and not (d_rows[:end] == 7).any()
    sf.sf_ctx_poll(ctx)
    sf.sf_expert_combine(ctx, rows, at, w, y, n_dev=torch.tensor([n + 1], dtype=torch.int32, device="cuda"))
    with pytest.raises(sf.SfError) as e:
        sf.sf_ctx_poll(ctx, reset=True)
    assert e.value.status == sf.SF_ERR_CAPACITY


def test_refusals(env):
    sf, ctx = env
    z = lambda *s, t=torch.int32: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
    ids, f = z(5000, 2), z(5000, 2, t=torch.float32)
    x, x16 = z(5000, 4, t=torch.float32), z(5000, 4, t=torch.bfloat16)
    small = z(3)
    with pytest.raises(sf.SfError):
        sf.sf_expert_gate(None, x, 0, ids, f)                                                        # no context
    wide = torch.zeros(1, dtype=torch.uint8, device="cuda").expand(1)
    assert sf._lib().sf_expert_combine(ctx, wide.data_ptr(), 0, 1, (1 << 24) + 1, (1 << 24) + 1, ids.data_ptr(), None, None, 1, 1, wide.data_ptr(),
                                       (1 << 24) + 1, None) == sf.SF_ERR_ARG                          # wider than SF_EXPERT_MAX_D
    for call in (lambda: sf.sf_expert_gate(ctx, z(5000, 1, t=torch.float32), 0, ids, f),            # k > E
                 lambda: sf.sf_expert_gate(ctx, x, 3, ids, f),
                 lambda: sf.sf_expert_gate(ctx, z(5000, 1025, t=torch.float32), 0, ids, f),
                 lambda: sf.sf_expert_gate(ctx, x, 0, ids[:4999], f),
                 lambda: sf.sf_expert_gate(ctx, x, 0, ids, f[:, :1]),
                 lambda: sf.sf_expert_gate(ctx, x, 0, z(5000, 0), z(5000, 0, t=torch.float32)),
                 lambda: sf.sf_expert_gate_backward(ctx, x, 0, ids, f, x16),
                 lambda: sf.sf_expert_sort(ctx, ids, 4, 3, z(5), z(4), z(20000), z(5000, 2), z(4000)),        # alignment
                 lambda: sf.sf_expert_sort(ctx, ids, 4, 0, z(5), z(4), z(20000), z(5000, 2), z(4000)),
                 lambda: sf.sf_expert_sort(ctx, ids, 0, 1, z(5), z(4), z(20000), z(5000, 2), z(4000)),
                 lambda: sf.sf_expert_sort(ctx, ids, 1025, 1, z(1026), z(1025), z(20000), z(5000, 2), z(40000)),
                 lambda: sf.sf_expert_sort(ctx, ids, 4, 1, z(5), z(4), z(20000), z(5000, 2), None),           # scratch
                 lambda: sf.sf_expert_sort(ctx, ids, 4, 1, z(5), z(4), z(20000), z(5000, 2), small),
                 lambda: sf.sf_expert_sort(ctx, ids, 4, 1, z(4), z(4), z(20000), z(5000, 2), z(4000)),
                 lambda: sf.sf_expert_gather(ctx, x, ids, z(5), z(4), x16),
                 lambda: sf.sf_expert_gather(ctx, x, ids[:10], z(5), z(4), x),
                 lambda: sf.sf_expert_gather(ctx, x.t(), ids, z(5), z(4), x),
                 lambda: sf.sf_expert_combine(ctx, x, ids, f[:1], x.clone()),
                 lambda: sf.sf_expert_combine(ctx, x, f, None, x.clone()),                                 # whole numbers are wanted
                 lambda: sf.sf_expert_combine(ctx, x, ids, ids, x.clone()),                                # real ones are wanted
                 lambda: sf.sf_expert_combine_backward(ctx, x, x, ids, f, z(5), z(4), None, None),
                 lambda: sf.sf_expert_combine_backward(ctx, x, x, ids, f, z(4), z(4), x.clone(), None)):
        with pytest.raises(sf.SfError) as e:
            call()
        assert e.value.status == sf.SF_ERR_ARG


def test_two_streams_of_one_context_at_once(env):
    """Each stream sorts, gathers, combines and takes gradients on its own data, many times over, with nothing between the two: every
    pass gives what the same calls give alone."""
    sf, ctx = env
    rng = np.random.default_rng(17)
    jobs = []
    for n, k, E, D in ((20000, 2, 16, 96), (15000, 3, 300, 50)):
        ids = dev(some_ids(rng, n, k, E))
        cap = n * k + E * 15
        i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
        x, dy, w = torch.randn(n, D, device="cuda"), torch.randn(n, D, device="cuda"), torch.rand(n, k, device="cuda")
        out = {"offsets": i32(E + 1), "counts": i32(E), "flow": i32(cap), "at": i32(n, k), "rows": torch.zeros(cap, D, device="cuda"),
               "y": torch.zeros(n, D, device="cuda"), "d_rows": torch.zeros(cap, D, device="cuda"), "d_w": torch.zeros(n, k, device="cuda")}
        work = i32(sf.sf_expert_sort_workspace(n, k, E) // 4 + 1)

        def step(stream, ids=ids, x=x, dy=dy, w=w, o=out, work=work, E=E):
            sf.sf_expert_sort(ctx, ids, E, 16, o["offsets"], o["counts"], o["flow"], o["at"], work, stream=stream)
            sf.sf_expert_gather(ctx, x, o["at"], o["offsets"], o["counts"], o["rows"], stream=stream)
            sf.sf_expert_combine(ctx, o["rows"], o["at"], w, o["y"], stream=stream)
            sf.sf_expert_combine_backward(ctx, dy, o["rows"], o["at"], w, o["offsets"], o["counts"], o["d_rows"], o["d_w"], stream=stream)
        step(torch.cuda.current_stream())
        torch.cuda.synchronize()
        jobs.append((step, out, {q: v.clone() for q, v in out.items()}))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for _, out, _ in jobs:
            for v in out.values():
                v.zero_()
        torch.cuda.synchronize()
        for _ in range(10):
            for (step, _, _), s in zip(jobs, streams):
                step(s)
        torch.cuda.synchronize()
        for _, out, want in jobs:
            for q in out:
                assert torch.equal(out[q], want[q]), q
    sf.sf_ctx_poll(ctx)


# ---- all of them in a row -----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n,E,k,K,N", [(1, 4, 1, 64, 8), (10, 8, 2, 1024, 256), (700, 5, 2, 416, 200)])
def test_experts_in_a_row(env, n, E, k, K, N):
    """Scores -> gate -> sort -> rows packed in the experts' order -> the experts' layer in 4 bits -> combine, captured and replayed
    on other inputs; against the definition, flow by flow."""
    sf, ctx = env
    rng = np.random.default_rng(n)
    cap = -(-(n * k) // 128) * 128 + 128 * E
    w = rng.normal(size=(E, N, K)) / np.sqrt(K)
    packed = [pr.pack(m) for m in w]
    rw = np.stack([pr.rounded(m) for m in w])
    wd, ws = dev(np.stack([p[0] for p in packed])), dev(np.stack([p[1] for p in packed]))
    bias = rng.normal(size=(E, N)).astype(np.float32)
    bd = dev(bias)
    scores, x = torch.zeros(n, E, device="cuda"), torch.zeros(n, K, dtype=torch.bfloat16, device="cuda")
    ids, wt = torch.zeros(n, k, dtype=torch.int32, device="cuda"), torch.zeros(n, k, device="cuda")
    offsets, counts, flow, at = [torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((E + 1,), (E,), (cap,), (n, k))]
    work = torch.zeros(sf.sf_expert_sort_workspace(n, k, E), dtype=torch.uint8, device="cuda")
    db, sb = sf.sf_mx4_sizes(cap, K)
    data, scales = torch.zeros(db, dtype=torch.uint8, device="cuda"), torch.zeros(sb, dtype=torch.uint8, device="cuda")
    hidden, y = torch.zeros(cap, N, device="cuda"), torch.zeros(n, N, device="cuda")

    def step():
        sf.sf_expert_gate(ctx, scores, sf.SF_GATE_SOFTMAX_PICKED, ids, wt)
        sf.sf_expert_sort(ctx, ids, E, 128, offsets, counts, flow, at, work)
        sf.sf_mx4_quantise(ctx, x, data, scales, row_ids=flow, n_rows_dev=offsets[E:])
        sf.sf_mx4_matmul_experts(ctx, data, scales, wd, ws, K, offsets, hidden, bias=bd, relu=True)
        sf.sf_expert_combine(ctx, hidden, at, wt, y)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(2):
        s = rng.normal(size=(n, E)).astype(np.float32)
        s[rng.random((n, E)) < 0.2] = -np.inf
        scores.copy_(dev(s))
        x.copy_(torch.from_numpy(rng.normal(size=(n, K))).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        sf.sf_ctx_poll(ctx)
        want_ids, want_w, _ = gate_reference(s.astype(float), k, 1)
        assert np.array_equal(num(ids), want_ids)
        rx = pr.rounded(num(x))
        want, tol = np.zeros((n, N)), np.zeros((n, N))
        for f in range(n):
            for j, e in enumerate(want_ids[f]):
                if e >= 0:
                    h = np.maximum(rw[e] @ rx[f] + bias[e], 0)
                    mass = np.abs(rw[e]) @ np.abs(rx[f]) + np.abs(bias[e])
                    want[f] += want_w[f, j] * h
                    tol[f] += want_w[f, j] * ((K + 2) * 2.0 ** -23 * mass + (E + k + 12) * 2.0 ** -23 * h)
        assert (np.abs(num(y) - want) <= tol + 2.0 ** -24 * np.abs(want)).all()


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,m,k,E,D", [(90, 50, 2, 4, 24), (90, 0, 2, 4, 24), (700, 699, 3, 5, 17), (40, 1, 2, 3, 3000), (300, 211, 1, 8, 1024)])
def test_device_count_values_of_the_flows_present(env, n, m, k, E, D, kind):
    """With fewer flows than the arrays hold, the present ones get the sums of the definition and the others stay as they were."""
    sf, ctx = env
    rng = np.random.default_rng(n + m + D)
    cnt = torch.tensor([m], dtype=torch.int32, device="cuda")
    cap = n * k + E * 15
    offsets, counts, flow, at = sort(sf, ctx, dev(some_ids(rng, n, k, E)), E, 16, cap, n_dev=cnt)
    at[m:] = 0                                           # stale rows of flows that are not there
    pairs, end = num(at)[:m], int(offsets[-1])
    real = pairs >= 0
    base, rows = laid(rng.normal(size=(cap, D)), kind, D, 0)
    v = np.where(real[..., None], num(rows)[np.maximum(pairs, 0)], 0.0)
    w = rng.random((n, k)).astype(np.float32)
    ww = np.where(real, w[:m], 0.0).astype(float)
    for weights, f in ((dev(w), ww), (None, real.astype(float))):
        y = torch.full((n, D), 7.0, dtype=TYPES[kind], device="cuda")
        sf.sf_expert_combine(ctx, rows, at, weights, y, n_dev=cnt)
        want, mass = (f[..., None] * v).sum(1), np.abs(f[..., None] * v).sum(1)
        slack = (k + 1) * 2.0 ** -24 * mass
        assert (np.abs(num(y)[:m] - want) <= slack + HALF_STEP[kind] * (np.abs(want) + slack) + TINY[kind]).all() and (y[m:] == 7).all()
        if weights is None:
            dx = torch.full((n, D), 7.0, dtype=TYPES[kind], device="cuda")
            sf.sf_expert_gather_backward(ctx, rows, at, dx, n_dev=cnt)
            assert torch.equal(dx, y)                    # the same sum of the same rows in the same order
    dy = laid(rng.normal(size=(n, D)), kind, D, 0)[1]
    g = num(dy)[:m]
    d_rows, d_w = torch.full((cap, D), 7.0, dtype=TYPES[kind], device="cuda"), torch.full((n, k), 7.0, device="cuda")
    sf.sf_expert_combine_backward(ctx, dy, rows, at, dev(w), offsets, counts, d_rows, d_w, n_dev=cnt)
    want = np.zeros((end, D))
    f, j = np.nonzero(real)
    want[pairs[f, j]] = ww[f, j, None] * g[f]
    assert (np.abs(num(d_rows)[:end] - want) <= (2.0 ** -24 + HALF_STEP[kind] * (1 + 2.0 ** -24)) * np.abs(want) + TINY[kind]).all() and (d_rows[end:] == 7).all()
    want_w = (g[:, None] * v).sum(-1)
    assert (np.abs(num(d_w)[:m] - want_w) <= (D + 1) * 2.0 ** -24 * np.abs(g[:, None] * v).sum(-1)).all() and (d_w[m:] == 7).all()
    sf.sf_ctx_poll(ctx)


@pytest.mark.parametrize("n,m,k,D,kind", [(20000, 19999, 3, 45, "fp32"), (152000, 151001, 2, 90, "bf16"), (152000, 152000, 1, 61, "fp16"), (76000, 75003, 2, 132, "fp32"),
                                          (80000, 80000, 3, 64, "bf16"), (80000, 7, 2, 64, "fp16"), (30000, 29990, 5, 17, "fp16"), (310000, 310000, 2, 8, "fp32"),
                                          (40000, 40000, 4, 512, "bf16"), (20001, 20001, 2, 256, "bf16"), (19000, 18999, 2, 33, "fp32"), (9000, 9000, 3, 50, "bf16")])
def test_many_flows_of_narrow_rows(env, n, m, k, D, kind):
    """Flows enough for several of them a thread, and just too few: gather, combine and their gradients against doubles on the device, m of n
    flows present."""
    sf, ctx = env
    rng = np.random.default_rng(n + D)
    E, T = 7, TYPES[kind]
    cnt = torch.tensor([m], dtype=torch.int32, device="cuda")
    cap = n * k + E * 15
    offsets, counts, flow, at = sort(sf, ctx, dev(some_ids(rng, n, k, E)), E, 16, cap, n_dev=cnt)
    end = int(offsets[-1])
    at[m:] = 0                                           # stale rows of flows that are not there
    pairs = at[:m].long()
    real, where = pairs >= 0, pairs.clamp(min=0)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n)
    new = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    x, dy, w = new(n, D).to(T), new(n, D).to(T), torch.rand(n, k, device="cuda", generator=gen)
    rows = torch.full((cap, D), 7.0, dtype=T, device="cuda")
    sf.sf_expert_gather(ctx, x, at, offsets, counts, rows, n_dev=cnt)
    f = flow[:end].long()
    assert torch.equal(rows[:end], torch.where((f >= 0)[:, None], x[f.clamp(min=0)], torch.zeros((), dtype=T, device="cuda"))) and (rows[end:] == 7).all()
    rows = new(cap, D).to(T)
    rows[end:] = float("nan")

    def within(got, want, slack):
        return bool(((got.double() - want).abs() <= slack + HALF_STEP[kind] * (want.abs() + slack) + TINY[kind]).all())
    for weights in (w, None):
        want, mass = torch.zeros(m, D, dtype=torch.float64, device="cuda"), torch.zeros(m, D, dtype=torch.float64, device="cuda")
        for j in range(k):
            t = torch.where(real[:, j, None], rows[where[:, j]].double() * (w[:m, j, None].double() if weights is not None else 1.0), 0.0)
            want, mass = want + t, mass + t.abs()
        y = torch.full((n, D), 7.0, dtype=T, device="cuda")
        sf.sf_expert_combine(ctx, rows, at, weights, y, n_dev=cnt)
        assert within(y[:m], want, (k + 1) * 2.0 ** -24 * mass) and (y[m:] == 7).all()
    dx = torch.full((n, D), 7.0, dtype=T, device="cuda")
    sf.sf_expert_gather_backward(ctx, rows, at, dx, n_dev=cnt)
    assert torch.equal(dx, y)
    d_rows, d_w = torch.full((cap, D), 7.0, dtype=T, device="cuda"), torch.full((n, k), 7.0, device="cuda")
    sf.sf_expert_combine_backward(ctx, dy, rows, at, w, offsets, counts, d_rows, d_w, n_dev=cnt)
    want = torch.zeros(end, D, dtype=torch.float64, device="cuda")
    for j in range(k):
        r = real[:, j]
        want[pairs[r, j]] = w[:m][r, j, None].double() * dy[:m][r].double()
        p = torch.where(r[:, None], rows[where[:, j]].double(), 0.0) * dy[:m].double()
        assert bool(((d_w[:m, j].double() - p.sum(-1)).abs() <= (D + 1) * 2.0 ** -24 * p.abs().sum(-1)).all())
    assert within(d_rows[:end], want, 2.0 ** -24 * want.abs()) and (d_rows[end:] == 7).all() and (d_w[m:] == 7).all()
    only_w, only_rows = torch.zeros_like(d_w), torch.zeros_like(d_rows)
    sf.sf_expert_combine_backward(ctx, dy, rows, at, w, offsets, counts, None, only_w, n_dev=cnt)
    sf.sf_expert_combine_backward(ctx, dy, rows, at, w, offsets, counts, only_rows, None, n_dev=cnt)
    assert torch.equal(only_w[:m], d_w[:m]) and torch.equal(only_rows[:end], d_rows[:end])
    sf.sf_ctx_poll(ctx)


def test_weights_gradient_alone_without_segments(env):
    sf, ctx = env
    rng = np.random.default_rng(8)
    (offsets, counts, flow, at), cap = plan(sf, ctx, rng, 300, 2, 5, 16)
    rows, dy = torch.randn(cap, 40, device="cuda"), torch.randn(300, 40, device="cuda")
    with_, without = torch.zeros(300, 2, device="cuda"), torch.zeros(300, 2, device="cuda")
    sf.sf_expert_combine_backward(ctx, dy, rows, at, None, offsets, counts, None, with_)
    sf.sf_expert_combine_backward(ctx, dy, rows, at, None, None, None, None, without)
    assert torch.equal(with_, without) and (with_ != 0).any()

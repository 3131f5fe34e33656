"""Causal convolution and selective scan over sequences of rows against direct statements in doubles, and together with what they are used with.

Tolerances, with e = 2^-24 (half a step of fp32) and M = the same statement with every term's magnitude.
 Convolution: W + 1 fused multiply-adds of e each; a sigmoid is off by (8 + 2 |x|) e (argument |x| e, exponential 4 e, sum and reciprocal 3 e), and silu
 takes an error of its argument 1.1 times: (W + 24 + 2 |x|) e.  Its slope takes it (1/2) |dpre| times; sums over rows add one e a row.
 Scan: a step is off by 16 e (softplus), so a decay by (4 + 20 |delta A|) e, a state adds two roundings: L rows (8 + 24 |delta A|) e; sums over N
 states, D channels or all rows one e a term; gates as above, 64 e for the rest.
Half a step of the output type comes on top."""
import numpy as np
import pytest

import sequences as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF_STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
TINY = {"fp32": 1e-37, "bf16": 1e-37, "fp16": 2.0 ** -24}
E = 2.0 ** -24
MARK = 7.0                                                 # what outputs hold before a call


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


def num(t):
    return t.double().cpu().numpy()


def rows_in(rng, n, d, kind, pitch=0, offset=0, scale=1.0):
    """A device tensor [n][d] of random values inside a wider one, which begins `offset` elements behind an allocation's start."""
    t = torch.from_numpy(rng.standard_normal(n * (d + pitch) + offset) * scale).to(TYPES[kind]).cuda()
    return t[offset:].view(n, d + pitch)[:, :d] if n else t.new_zeros(0, d)


def like(t):
    """An output beside t: same pitch and boundary, marked."""
    n, d = t.shape
    if n <= 1:
        return torch.full((n, d), MARK, dtype=t.dtype, device="cuda")
    return torch.full((n * t.stride(0) + 8,), MARK, dtype=t.dtype, device="cuda")[t.storage_offset() % 8:].as_strided((n, d), (t.stride(0), 1))


def lay_out(sf, rng, lengths, planes, with_slots):
    """offsets, counts, slots of sequences of these lengths: planes of the longest + 2 rows, or one behind the other."""
    S, most = len(lengths), max(max(lengths), 1)
    if planes:
        offsets, counts = np.arange(S + 1) * (most + 2), np.array(lengths)
    else:
        offsets, counts = np.concatenate([[0], np.cumsum(lengths)]), None
    slots = None
    if with_slots:
        slots = rng.permutation(S + 2)[:S]
        if S > 2:
            slots[1] = -1                                  # one sequence keeps no state
    dev = lambda a: None if a is None else torch.from_numpy(np.asarray(a, np.int32)).cuda()  # noqa: E731
    keep = dev(offsets), dev(counts), dev(slots)
    q = sf.make_sequences(keep[0], most, counts=keep[1], slots=keep[2])
    return q, offsets, int(offsets[-1]) + (3 if planes else 0), np.arange(S) if slots is None else slots


def close(name, got, want, tol, kind):
    bad = np.abs(got - want) > tol + HALF_STEP[kind] * np.abs(want) + TINY[kind]
    assert not bad.any(), (name, np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], (np.abs(got - want) / (tol + 1e-300)).max())


# ---- convolution ---------------------------------------------------------------------------------------------------------------------
CONV = [
    # W, silu, D, type, lengths, planes, slots, pitch, offset, bias
    (4, True, 64, "bf16", [5, 1, 0, 33, 2, 130], True, True, 0, 0, True),
    (4, True, 40, "bf16", [9, 3, 128, 129, 127], False, False, 8, 0, True),
    (4, False, 33, "fp16", [17, 4, 1], False, True, 1, 1, True),
    (3, True, 8, "fp32", [8, 7, 9, 2, 0, 16], True, True, 4, 0, False),
    (2, False, 130, "fp32", [1, 1, 1, 1], False, True, 2, 2, True),
    (1, True, 20, "bf16", [5, 2], False, False, 0, 0, True),
    (8, True, 24, "fp32", [3, 20, 7, 8], True, True, 0, 0, True),
    (5, False, 6, "bf16", [2, 300, 4], False, True, 2, 0, False),
    (4, True, 512, "bf16", [1] * 9, False, True, 0, 0, True),
    (4, True, 3, "fp16", [2] * 300, True, False, 0, 0, True),
    (7, True, 1, "fp32", [40], False, True, 0, 0, True),
]


@pytest.mark.parametrize("W,silu,D,kind,lengths,planes,slots,pitch,offset,with_bias", CONV)
def test_convolution(env, W, silu, D, kind, lengths, planes, slots, pitch, offset, with_bias):
    sf, ctx = env
    rng = np.random.default_rng(W * 1000 + D)
    q, first, R, slot = lay_out(sf, rng, lengths, planes, slots)
    S, act = len(lengths), sf.SF_ACT_SILU if silu else sf.SF_ACT_NONE
    x, dy = rows_in(rng, R, D, kind, pitch, offset), rows_in(rng, R, D, kind, pitch, offset)
    w, b = torch.from_numpy(rng.standard_normal((D, W)).astype(np.float32)).cuda(), torch.from_numpy(rng.standard_normal(D).astype(np.float32)).cuda() if with_bias else None
    pool = torch.from_numpy(rng.standard_normal((S + 2, W - 1, D))).to(TYPES[kind]).cuda()
    d_pool = torch.from_numpy(rng.standard_normal((S + 2, W - 1, D))).to(TYPES[kind]).cuda()
    y, dx = like(x), like(x)
    both = pool.clone()                                    # read and written by one call
    sf.sf_seq_conv(ctx, q, x, w, y, bias=b, act=act, state_in=both, state_out=both)
    dw, db, d_in = torch.full_like(w, MARK), torch.full((D,), MARK, device="cuda"), torch.full_like(pool, MARK)
    work = torch.zeros(sf.sf_seq_conv_backward_workspace(S, max(max(lengths), 1), D, W), dtype=torch.uint8, device="cuda")
    sf.sf_seq_conv_backward(ctx, q, x, w, dy, work, bias=b, act=act, state_in=pool, d_state=d_pool, dx_out=dx, dw_out=dw, dbias_out=db, d_state_in_out=d_in)
    sf.sf_ctx_poll(ctx)
    X, DY, P, DP, W_, B_ = num(x), num(dy), num(pool), num(d_pool), num(w), None if b is None else num(b)
    want_y, want_dx, want_pool, want_din = np.full((R, D), MARK), np.full((R, D), MARK), P.copy(), np.full(P.shape, MARK)
    tol_y, tol_dx, tol_din = np.zeros((R, D)), np.zeros((R, D)), np.zeros(P.shape)
    sums, mags = {"dw": 0, "dbias": 0}, {"dw": 0, "dbias": 0}
    for s, n in enumerate(lengths):
        at, own = slice(first[s], first[s] + n), slot[s]
        st = P[own] if own >= 0 else np.zeros(P.shape[1:])
        dst = DP[own] if own >= 0 else None
        r = ref.conv(X[at], W_, B_, silu, st, DY[at], dst)
        pre = ref.conv(X[at], W_, B_, False, st, ab=np.abs)["y"]
        m = ref.conv(X[at], W_, B_, False, st, DY[at] * (1.1 + pre if silu else 1.0), dst, ab=np.abs)
        c = (2 * W + 48 + 4 * pre.max(initial=0)) * E
        want_y[at], tol_y[at] = r["y"], 1.1 * (W + 24 + 2 * pre) * E * pre
        want_dx[at], tol_dx[at] = r["dx"], c * m["dx"]
        for k in sums:
            sums[k], mags[k] = sums[k] + r[k], mags[k] + m[k]
        if own >= 0 and W > 1:
            want_pool[own] = r["state"]
            want_din[own], tol_din[own] = r["d_state_in"], c * m["d_state_in"]
    close("y", num(y), want_y, tol_y, kind)
    assert np.array_equal(num(both), want_pool)
    close("dx", num(dx), want_dx, tol_dx, kind)
    close("d_state_in", num(d_in), want_din, tol_din, kind)
    c = (sum(lengths) + 2 * W + 48 + 4 * 20) * E
    close("dw", num(dw), sums["dw"], c * mags["dw"], "fp32")
    close("dbias", num(db), sums["dbias"], c * mags["dbias"], "fp32")


# ---- scan -------------------------------------------------------------------------------------------------------------------------------
SCAN = [
    # D, N, G, type, lengths, planes, slots, pitch, offset, z, softplus, skip, bias
    (32, 16, 1, "bf16", [5, 1, 0, 33, 2, 8], True, True, 0, 0, True, True, True, True),
    (64, 16, 2, "bf16", [9, 16, 17, 7], False, False, 0, 0, True, True, True, True),
    (33, 16, 1, "fp16", [17, 4, 1], False, True, 1, 1, True, True, True, True),
    (160, 16, 1, "bf16", [12, 3], False, True, 0, 0, True, True, True, False),
    (8, 4, 1, "fp32", [8, 7, 9, 2, 0, 16], True, True, 4, 0, False, True, False, False),
    (140, 3, 1, "fp32", [5, 18], False, True, 0, 0, True, False, True, False),
    (12, 1, 4, "fp32", [11, 1, 1], False, True, 0, 0, False, False, False, True),
    (70, 8, 1, "bf16", [10, 21], False, False, 2, 0, True, True, True, True),
    (24, 30, 3, "fp32", [6, 25], True, True, 0, 0, True, True, True, True),
    (20, 64, 1, "bf16", [7, 9], False, True, 0, 0, True, True, True, True),
    (16, 33, 2, "fp16", [14], False, True, 0, 0, False, True, True, True),
    (1, 16, 1, "fp32", [10, 1], False, True, 0, 0, True, True, True, True),
    (32, 16, 1, "bf16", [1] * 9, False, True, 0, 0, True, True, True, True),
    (40, 16, 1, "fp32", [1, 0, 1, 1], True, True, 0, 0, True, True, True, True),
    (9, 5, 1, "fp16", [1] * 3, False, True, 0, 1, False, True, True, False),
    (24, 16, 1, "fp32", [300], False, True, 0, 0, True, True, True, True),             # in parts
    (32, 4, 2, "bf16", [260, 0, 131], True, True, 0, 0, True, True, True, True),       # in parts, one empty
    (64, 16, 1, "bf16", [33, 16, 8, 9, 1, 17] * 50, False, False, 0, 0, True, True, True, True),      # too many for parts, too few to fill the machine
    (520, 4, 1, "fp32", [2, 9] + [1] * 158, False, False, 0, 0, True, True, True, True),       # a whole block of wide warps
    (1032, 3, 1, "bf16", [3] * 150, False, False, 0, 0, True, True, True, True),
]


def scan_case(sf, rng, D, N, G, kind, lengths, planes, slots, pitch, offset, z, softplus, skip, bias):
    q, first, R, slot = lay_out(sf, rng, lengths, planes, slots)
    f32 = lambda a: torch.from_numpy(np.asarray(a, np.float32)).cuda()  # noqa: E731
    t = {"u": rows_in(rng, R, D, kind, pitch, offset), "B": rows_in(rng, R, G * N, kind, pitch, offset), "C": rows_in(rng, R, G * N, kind, pitch, offset),
         "delta": rows_in(rng, R, D, kind, pitch, offset, 0.5), "dy": rows_in(rng, R, D, kind, pitch, offset),
         "z": rows_in(rng, R, D, kind, pitch, offset) if z else None, "A": f32(-rng.uniform(0.05, 2, (D, N))),
         "D": f32(rng.standard_normal(D)) if skip else None, "bias": f32(rng.uniform(-4, -1, D)) if bias else None}
    if not softplus:
        t["delta"].abs_().mul_(0.2)
        if bias:
            t["bias"] = f32(rng.uniform(0.01, 0.1, D))
    pool, d_pool = f32(rng.standard_normal((len(lengths) + 2, D, N))), f32(rng.standard_normal((len(lengths) + 2, D, N)))
    return q, first, R, slot, t, pool, d_pool


def scan_doubles(t, first, lengths, slot, pool, d_pool, softplus, G, grads=True):
    """Sequence by sequence: what the calls have to give and how far they may be off."""
    v = {k: None if x is None else num(x) for k, x in t.items()}
    N = v["A"].shape[1]
    R, D = v["u"].shape
    P, DP = num(pool), num(d_pool)
    shape = {"y": (R, D), "du": (R, D), "d_delta": (R, D), "dz": (R, D), "dB": (R, G * N), "dC": (R, G * N), "state": P.shape, "d_state_in": P.shape}
    want = {k: np.full(s, MARK) for k, s in shape.items()}
    want["state"] = P.copy()
    tol = {k: np.zeros(s) for k, s in shape.items()}
    sums = {k: [0, 0] for k in ("dA", "dD", "d_delta_bias")}
    for s, n in enumerate(lengths):
        at, own = slice(first[s], first[s] + n), slot[s]
        g3 = lambda a: a[at].reshape(n, G, N)  # noqa: E731
        z = None if v["z"] is None else v["z"][at]
        args = (v["u"][at], v["delta"][at], v["A"], g3(v["B"]), g3(v["C"]), v["D"], v["bias"])
        h0, dh = (P[own], DP[own]) if own >= 0 else (np.zeros(P.shape[1:]), None)
        dy = v["dy"][at] if grads else None
        r = ref.scan(*args, z, softplus, h0, dy, dh if grads else None)
        m = ref.scan(*args, z, softplus, h0, dy, dh if grads else None, ab=np.abs)
        raw = v["delta"][at] + (0 if v["bias"] is None else v["bias"])
        most = (np.abs(ref.softplus(raw) if softplus else raw).max(initial=0) * np.abs(v["A"]).max(initial=0))
        c = (n * (8 + 24 * most) + 4 * N + D + 64 + (0 if z is None else 4 * np.abs(z).max(initial=0))) * E
        if grads and z is not None:
            flat = ref.scan(*args, None, softplus, h0, ab=np.abs)["y"]
            m["dz"] = np.abs(v["dy"][at]) * flat * (1.1 + np.abs(z))
        for k in ("y", "du", "d_delta", "dz", "dB", "dC"):
            if k in r:
                want[k][at], tol[k][at] = r[k].reshape(n, shape[k][1]), c * m[k].reshape(n, shape[k][1])
        if own >= 0:
            want["state"][own], tol["state"][own] = r["state"], c * m["state"]
            if grads:
                want["d_state_in"][own], tol["d_state_in"][own] = r["d_state_in"], c * m["d_state_in"]
        for k in sums:
            if k in r:
                sums[k][0], sums[k][1] = sums[k][0] + r[k], sums[k][1] + (c + R * E) * m[k]
    return want, tol, sums


@pytest.mark.parametrize("D,N,G,kind,lengths,planes,slots,pitch,offset,z,softplus,skip,bias", SCAN)
def test_scan(env, D, N, G, kind, lengths, planes, slots, pitch, offset, z, softplus, skip, bias):
    sf, ctx = env
    rng = np.random.default_rng(D * 100 + N)
    q, first, R, slot, t, pool, d_pool = scan_case(sf, rng, D, N, G, kind, lengths, planes, slots, pitch, offset, z, softplus, skip, bias)
    S, most = len(lengths), max(max(lengths), 1)
    rest = dict(D=t["D"], delta_bias=t["bias"], z=t["z"], softplus=softplus)
    rows = (t["u"], t["delta"], t["A"], t["B"], t["C"])
    work = torch.full((sf.sf_seq_scan_workspace(S, most, R, D, N, G, backward=True),), 255, dtype=torch.uint8, device="cuda")
    want, tol, sums = scan_doubles(t, first, lengths, slot, pool, d_pool, softplus, G)
    # serving: no states kept for a backward pass; one pool read and written
    y, both = like(t["u"]), pool.clone()
    sf.sf_seq_scan(ctx, q, *rows, y, workspace=work, state_in=both, state_out=both, **rest)
    close("y", num(y), want["y"], tol["y"], kind)
    close("state", num(both), want["state"], tol["state"], "fp32")
    # training
    y2, after = like(t["u"]), pool.clone()
    starts = torch.zeros(sf.sf_seq_scan_starts(S, R, D, N), device="cuda")
    sf.sf_seq_scan(ctx, q, *rows, y2, workspace=work, state_in=pool, state_out=after, starts_out=starts, **rest)
    close("y kept", num(y2), want["y"], tol["y"], kind)
    close("state kept", num(after), want["state"], tol["state"], "fp32")
    g = {k: None if x is None else like(x) for k, x in (("du", t["u"]), ("d_delta", t["delta"]), ("dB", t["B"]), ("dC", t["C"]), ("dz", t["z"]))}
    p = {k: None if x is None else torch.full_like(x, MARK) for k, x in (("dA", t["A"]), ("dD", t["D"]), ("d_delta_bias", t["bias"]))}
    d_in = torch.full_like(pool, MARK)
    outs = {k + "_out": x for k, x in {**g, **p}.items()}
    sf.sf_seq_scan_backward(ctx, q, *rows, t["dy"], starts, work, d_state=d_pool, d_state_in_out=d_in, **outs, **rest)
    sf.sf_ctx_poll(ctx)
    for k, x in g.items():
        if x is not None:
            close(k, num(x), want[k], tol[k], kind)
    close("d_state_in", num(d_in), want["d_state_in"], tol["d_state_in"], "fp32")
    for k, x in p.items():
        if x is not None:
            close(k, num(x), sums[k][0] + np.zeros(x.shape), sums[k][1] + np.zeros(x.shape), "fp32")
    # twice the same
    again = {k: None if x is None else x.clone() for k, x in outs.items()}
    sf.sf_seq_scan_backward(ctx, q, *rows, t["dy"], starts, work, d_state=d_pool, d_state_in_out=d_in, **again, **rest)
    for k, x in outs.items():
        assert x is None or torch.equal(x, again[k]), k


def test_scan_row_by_row_is_the_whole_scan(env):
    """A stream: the next packet of every flow in a call of its own, states kept in a pool, against all of them in one call."""
    sf, ctx = env
    rng = np.random.default_rng(5)
    S, L, D, N = 7, 12, 48, 16
    q, first, R, slot, t, pool, _ = scan_case(sf, rng, D, N, 1, "fp32", [L] * S, False, True, 0, 0, True, True, True, True)
    rest = dict(D=t["D"], delta_bias=t["bias"], softplus=True)
    y, whole = like(t["u"]), pool.clone()
    sf.sf_seq_scan(ctx, q, t["u"], t["delta"], t["A"], t["B"], t["C"], y, z=t["z"], state_in=whole, state_out=whole, workspace=torch.zeros(
        sf.sf_seq_scan_workspace(S, L, R, D, N), dtype=torch.uint8, device="cuda"), **rest)
    steps, out = pool.clone(), torch.zeros_like(y)
    one = sf.make_sequences(torch.arange(S + 1, dtype=torch.int32, device="cuda"), 1, slots=torch.from_numpy(np.asarray(slot, np.int32)).cuda())
    for i in range(L):
        at = torch.arange(S, device="cuda") * L + i
        row = lambda k: t[k][at].contiguous()  # noqa: E731
        o = torch.zeros(S, D, device="cuda")
        before = steps.clone()
        if (slot < 0).any():                               # the sequence that keeps no state: a pool of its own to read
            spare = [k for k in range(S + 2) if k not in set(slot)][0]
            if i == 0:
                before[spare] = 0
            ids = torch.from_numpy(np.where(slot < 0, spare, slot).astype(np.int32)).cuda()
            one = sf.make_sequences(torch.arange(S + 1, dtype=torch.int32, device="cuda"), 1, slots=ids)
        sf.sf_seq_scan(ctx, one, row("u"), row("delta"), t["A"], row("B"), row("C"), o, z=row("z"), state_in=before, state_out=steps, **rest)
        out[at] = o
    want, tol, _ = scan_doubles({**t}, first, [L] * S, slot, pool, pool, True, 1, grads=False)
    close("rows one by one", num(out), want["y"], tol["y"], "fp32")
    close("all at once", num(y), want["y"], tol["y"], "fp32")
    keep = slot[slot >= 0]
    close("states", num(steps)[keep], want["state"][keep], tol["state"][keep], "fp32")


def test_long_memory_is_kept(env):
    """Thousands of rows whose decay is near one: the state is a sum over all of them (2000 e relative by the count of roundings)."""
    sf, ctx = env
    L, D, N = 2000, 64, 16
    rng = np.random.default_rng(9)
    u, b = torch.from_numpy(rng.uniform(0.5, 1, (L, D))).float().cuda(), torch.ones(L, N, device="cuda")
    delta, A = torch.full((L, D), 1e-3, device="cuda"), -torch.from_numpy(rng.uniform(0.01, 1, (D, N))).float().cuda()
    q = sf.make_sequences(torch.tensor([0, L], dtype=torch.int32, device="cuda"), L)
    state, y = torch.zeros(1, D, N, device="cuda"), torch.zeros(L, D, device="cuda")
    sf.sf_seq_scan(ctx, q, u, delta, A, b, b, y, state_out=state, workspace=torch.zeros(sf.sf_seq_scan_workspace(1, L, L, D, N), dtype=torch.uint8, device="cuda"))
    a, h = np.exp(np.float64(np.float32(1e-3)) * num(A)), np.zeros((D, N))
    for i in range(L):
        h = a * h + np.float64(np.float32(1e-3)) * num(u)[i][:, None]
    # roundings of single steps go either way, so they add up as their root: sqrt(2000) times 2 e, and the mean of the exponential's own error, below e / 8 a step
    assert (np.abs(num(state)[0] - h) / h).max() < (2 * np.sqrt(L) + L / 8) * E * 2


def test_more_sequences_than_a_grid_has_rows(env):
    """70,000 sequences of one row each, channels of a group over several blocks: h = delta u B, so dB = sum_d e C delta u and dC = sum_d e h in closed form."""
    sf, ctx = env
    S, D, N = 70_000, 136, 16
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    r = lambda d: torch.randn(S, d, device="cuda", generator=g)  # noqa: E731
    u, delta, B, C, dy, A = r(D), r(D).abs() * 0.3, r(N), r(N), r(D), -torch.ones(D, N, device="cuda")
    q = sf.make_sequences(torch.arange(S + 1, dtype=torch.int32, device="cuda"), 1)
    y, dB, dC, dx = torch.zeros_like(u), torch.zeros_like(B), torch.zeros_like(C), torch.zeros_like(u)
    starts = torch.zeros(sf.sf_seq_scan_starts(S, S, D, N), device="cuda")
    work = torch.zeros(sf.sf_seq_scan_workspace(S, 1, S, D, N, backward=True), dtype=torch.uint8, device="cuda")
    sf.sf_seq_scan(ctx, q, u, delta, A, B, C, y, starts_out=starts)
    sf.sf_seq_scan_backward(ctx, q, u, delta, A, B, C, dy, starts, work, dB_out=dB, dC_out=dC)
    in_, e = delta.double() * u.double(), dy.double()
    dot = (B.double() * C.double()).sum(1, keepdim=True)
    tol = (D + 64) * E
    assert ((y.double() - in_ * dot).abs() <= tol * (in_.abs() * (B.double() * C.double()).abs().sum(1, keepdim=True))).all()
    both, mag = (e * in_).sum(1, keepdim=True), (e * in_).abs().sum(1, keepdim=True)
    assert ((dB.double() - both * C.double()).abs() <= tol * mag * C.double().abs() + 1e-30).all()
    assert ((dC.double() - both * B.double()).abs() <= tol * mag * B.double().abs() + 1e-30).all()
    w = torch.randn(D, 4, device="cuda", generator=g)
    work = torch.zeros(sf.sf_seq_conv_backward_workspace(S, 1, D, 4), dtype=torch.uint8, device="cuda")
    dw = torch.zeros_like(w)
    sf.sf_seq_conv_backward(ctx, q, u, w, dy, work, dx_out=dx, dw_out=dw)
    assert ((dx.double() - w[:, 3].double() * e).abs() <= 4 * E * (w[:, 3].double() * e).abs()).all()
    assert ((dw[:, 3].double() - (e * u.double()).sum(0)).abs() <= S * E * (e * u.double()).abs().sum(0)).all() and bool((dw[:, :3] == 0).all())


# ---- both: what device memory says ------------------------------------------------------------------------------------------------------
def bad_sequences(sf):
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"rows behind the arrays": (sf.make_sequences(i32(0, 4, 100), 200), sf.SF_ERR_CAPACITY, [(0, 4), (4, 12)]),
            "first row behind the arrays": (sf.make_sequences(i32(0, 4, 50, 100), 200), sf.SF_ERR_CAPACITY, [(0, 4), (4, 12)]),
            "falling offsets": (sf.make_sequences(i32(0, 6, 4, 9), 12), sf.SF_ERR_ARG, [(0, 6), (4, 9)]),
            "counts beyond the offsets": (sf.make_sequences(i32(0, 4, 9), 12, counts=i32(9, 2)), sf.SF_ERR_CAPACITY, [(0, 4), (4, 6)]),
            "longer than max_len": (sf.make_sequences(i32(0, 9), 5), sf.SF_ERR_CAPACITY, [(0, 5)]),
            "nothing": (sf.make_sequences(i32(0), 5), sf.SF_OK, []), "nothing of long sequences": (sf.make_sequences(i32(0), 5000), sf.SF_OK, [])}


@pytest.mark.parametrize("which", ["rows behind the arrays", "first row behind the arrays", "falling offsets", "counts beyond the offsets", "longer than max_len", "nothing", "nothing of long sequences"])
def test_sequences_that_do_not_fit_are_cut(env, which):
    sf, ctx = env
    q, status, parts = bad_sequences(sf)[which]
    R, D, N, W = 12, 32, 16, 4
    rng = np.random.default_rng(3)
    r = lambda d: torch.from_numpy(rng.standard_normal((R, d))).float().cuda()  # noqa: E731
    x, w, dy = r(D), torch.from_numpy(rng.standard_normal((D, W))).float().cuda(), r(D)
    y, dx = torch.full_like(x, MARK), torch.full_like(x, MARK)
    sf.sf_ctx_poll(ctx, reset=True, raise_on_error=False)
    sf.sf_seq_conv(ctx, q, x, w, y)
    c = sf.sf_ctx_poll(ctx, reset=True, raise_on_error=False)
    assert c.device_error == status
    work = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    dw = torch.zeros_like(w)
    sf.sf_seq_conv_backward(ctx, q, x, w, dy, work, dx_out=dx, dw_out=dw)
    assert sf.sf_ctx_poll(ctx, reset=True, raise_on_error=False).device_error == status
    inside = np.zeros(R, bool)
    for a, b in parts:
        inside[a:b] = True
    assert (num(y)[~inside] == MARK).all() and (num(dx)[~inside] == MARK).all() and (num(y)[inside] != MARK).any(1).all()
    A, B, C = -torch.ones(D, N, device="cuda"), r(N), r(N)
    y, du, dA = torch.full_like(x, MARK), torch.full_like(x, MARK), torch.full_like(A, MARK)
    starts = torch.zeros(sf.sf_seq_scan_starts(q.n_seq, R, D, N), device="cuda")
    sf.sf_seq_scan(ctx, q, x, dy.abs() * 0.1, A, B, C, y, starts_out=starts, workspace=torch.zeros(sf.sf_seq_scan_workspace(q.n_seq, q.max_len, R, D, N), dtype=torch.uint8, device="cuda"))
    assert sf.sf_ctx_poll(ctx, reset=True, raise_on_error=False).device_error == status
    work = torch.zeros(sf.sf_seq_scan_workspace(q.n_seq, q.max_len, R, D, N, backward=True), dtype=torch.uint8, device="cuda")
    sf.sf_seq_scan_backward(ctx, q, x, dy.abs() * 0.1, A, B, C, dy, starts, work, du_out=du, dA_out=dA)
    assert sf.sf_ctx_poll(ctx, reset=True, raise_on_error=False).device_error == status
    assert (num(y)[~inside] == MARK).all() and (num(du)[~inside] == MARK).all()
    assert (num(y)[inside] != MARK).any(1).all()
    if not parts:
        assert (num(dA) == 0).all() and (num(dw) == 0).all()


def test_nan_and_infinity_stay_in_their_sequence(env):
    sf, ctx = env
    D, N = 32, 16
    rng = np.random.default_rng(4)
    r = lambda d: torch.from_numpy(rng.standard_normal((30, d))).float().cuda()  # noqa: E731
    x, delta, B, C = r(D), r(D), r(N), r(N)
    x[13, 3], B[14, 2], delta[15, 5] = float("nan"), float("inf"), float("nan")
    q = sf.make_sequences(torch.tensor([0, 10, 20, 30], dtype=torch.int32, device="cuda"), 10)
    y = torch.zeros_like(x)
    sf.sf_seq_scan(ctx, q, x, delta, -torch.ones(D, N, device="cuda"), B, C, y, softplus=True)
    v = num(y)
    assert np.isfinite(v[:13]).all() and np.isfinite(v[20:]).all() and np.isnan(v[13:20, 3]).all() and np.isnan(v[15:20, 5]).all()
    w = torch.ones(D, 4, device="cuda")
    sf.sf_seq_conv(ctx, q, x, w, y)
    v = num(y)
    assert np.isnan(v[13:17, 3]).all() and np.isfinite(np.delete(v, np.s_[13:17], 0)).all()


def test_captured_and_on_other_streams(env):
    """Both calls in a graph, replayed on new inputs; and two streams of one context at once with workspaces of their own."""
    sf, ctx = env
    S, L, D, N = 1, 700, 40, 16                            # in parts: the workspace is used
    rng = np.random.default_rng(6)
    q, first, R, slot, t, pool, d_pool = scan_case(sf, rng, D, N, 1, "fp32", [L], False, False, 0, 0, True, True, True, True)
    rest = dict(D=t["D"], delta_bias=t["bias"], z=t["z"], softplus=True)
    size = sf.sf_seq_scan_workspace(S, L, R, D, N, backward=True)

    def both(u, work, y, starts, du):
        sf.sf_seq_scan(ctx, q, u, t["delta"], t["A"], t["B"], t["C"], y, workspace=work, state_in=pool[:1], starts_out=starts, **rest)
        sf.sf_seq_scan_backward(ctx, q, u, t["delta"], t["A"], t["B"], t["C"], t["dy"], starts, work, du_out=du, **rest)

    def buffers():
        return [torch.zeros(size, dtype=torch.uint8, device="cuda"), torch.zeros(R, D, device="cuda"), torch.zeros(sf.sf_seq_scan_starts(S, R, D, N), device="cuda"), torch.zeros(R, D, device="cuda")]
    inputs = [t["u"].clone(), t["u"].flip(0).contiguous()]
    want = []
    for u in inputs:
        b = buffers()
        both(u, *b)
        want.append((b[1].clone(), b[3].clone()))
    u, b = inputs[0].clone(), buffers()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(u, *b)
    for k in (1, 0, 1):
        u.copy_(inputs[k])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(b[1], want[k][0]) and torch.equal(b[3], want[k][1])
    streams, sets = [torch.cuda.Stream(), torch.cuda.Stream()], [buffers(), buffers()]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, v, x in zip(streams, sets, inputs):
            with torch.cuda.stream(s):
                both(x, *v)
    torch.cuda.synchronize()
    for v, (y, du) in zip(sets, want):
        assert torch.equal(v[1], y) and torch.equal(v[3], du)


def test_far_rows_and_slots(env):
    """Rows and states behind 2^32 bytes."""
    sf, ctx = env
    D, N, W = 1024, 16, 4
    rows, slots = 1_100_000, 66_000                        # 2.25 GB of bf16 rows twice, 4.3 GB of states
    u = torch.zeros(rows, D, dtype=torch.bfloat16, device="cuda")
    y = torch.zeros(rows, D, dtype=torch.bfloat16, device="cuda")
    first = rows - 5
    u[first:] = torch.randn(5, D, device="cuda").bfloat16()
    q = sf.make_sequences(torch.tensor([first, rows], dtype=torch.int32, device="cuda"), 5, slots=torch.tensor([slots - 1], dtype=torch.int32, device="cuda"))
    w = torch.randn(D, W, device="cuda")
    sf.sf_seq_conv(ctx, q, u, w, y)
    want = ref.conv(num(u[first:]), num(w), None, False, np.zeros((W - 1, D)))["y"]
    mag = ref.conv(num(u[first:]), num(w), None, False, np.zeros((W - 1, D)), ab=np.abs)["y"]
    close("y", num(y[first:]), want, (W + 1) * E * mag, "bf16")
    B = torch.zeros(rows, N, dtype=torch.bfloat16, device="cuda")
    B[first:] = 1
    pool = torch.zeros(slots, D, N, device="cuda")
    pool[-1] = 2.0
    A = -torch.ones(D, N, device="cuda")
    sf.sf_seq_scan(ctx, q, u, torch.full_like(u, 0.5), A, B, B, y, state_in=pool, state_out=pool)
    r = ref.scan(num(u[first:]), np.full((5, D), 0.5), num(A), np.ones((5, 1, N)), np.ones((5, 1, N)), None, None, None, False, np.full((D, N), 2.0))
    m = ref.scan(num(u[first:]), np.full((5, D), 0.5), num(A), np.ones((5, 1, N)), np.ones((5, 1, N)), None, None, None, False, np.full((D, N), 2.0), ab=np.abs)
    c = (5 * 20 + 4 * N + 64) * E
    close("state", num(pool[-1]), r["state"], c * m["state"], "fp32")
    close("y", num(y[first:]), r["y"], c * m["y"], "bf16")
    assert (pool[0] == 0).all()


# ---- refusals ------------------------------------------------------------------------------------------------------------------------------
def test_pools_of_another_size_and_workspaces_too_small(env):
    sf, ctx = env
    D, N, L = 32, 16, 500
    x, bc, A = torch.zeros(L, D, device="cuda"), torch.zeros(L, N, device="cuda"), torch.zeros(D, N, device="cuda")
    q = sf.make_sequences(torch.tensor([0, L], dtype=torch.int32, device="cuda"), L)
    need = sf.sf_seq_scan_workspace(1, L, L, D, N)
    assert need > 0
    for work in (None, torch.zeros(need - 1, dtype=torch.uint8, device="cuda")):
        with pytest.raises(sf.SfError) as e:
            sf.sf_seq_scan(ctx, q, x, x, A, bc, bc, torch.zeros_like(x), workspace=work)
        assert e.value.status == sf.SF_ERR_ARG
    starts = torch.zeros(sf.sf_seq_scan_starts(1, L, D, N), device="cuda")
    need = sf.sf_seq_scan_workspace(1, L, L, D, N, backward=True)
    with pytest.raises(sf.SfError):
        sf.sf_seq_scan_backward(ctx, q, x, x, A, bc, bc, x, starts, torch.zeros(need // 2, dtype=torch.uint8, device="cuda"), du_out=torch.zeros_like(x))
    with pytest.raises(sf.SfError):
        sf.sf_seq_conv_backward(ctx, q, x, torch.zeros(D, 4, device="cuda"), x, None, dw_out=torch.zeros(D, 4, device="cuda"))
    sf.sf_seq_conv_backward(ctx, q, x, torch.zeros(D, 4, device="cuda"), x, None, dx_out=torch.zeros_like(x))          # the rows' gradient alone needs none


# ---- together ---------------------------------------------------------------------------------------------------------------------------------
def test_a_slow_model_that_reads_packets_served_and_trained(env):
    """Wide rows of flows -> convolution -> scan -> the last packet's row -> 4-bit layer -> scores -> thresholds; and the gradient of the loss back to
    the filters, held to differences of the same formulas in doubles."""
    sf, ctx = env
    S, P, D, N, W, V = 60, 20, 32, 16, 4, 8
    rng = np.random.default_rng(12)
    f32 = lambda a: torch.from_numpy(np.asarray(a, np.float32)).cuda()  # noqa: E731
    counts = rng.integers(1, P + 1, S)
    q = sf.make_sequences(torch.arange(S + 1, dtype=torch.int32, device="cuda") * P, P, counts=torch.from_numpy(counts.astype(np.int32)).cuda())
    R = S * P
    x, delta, B, C, z = (f32(rng.standard_normal((R, d))) for d in (D, D, N, N, D))
    w, wb, A, Dk, db = f32(rng.standard_normal((D, W)) / 2), f32(rng.standard_normal(D)), f32(-rng.uniform(0.1, 2, (D, N))), f32(rng.standard_normal(D)), f32(rng.uniform(-3, -1, D))
    head, labels = f32(rng.standard_normal((V, D)) / 4), torch.from_numpy(rng.integers(0, V, S).astype(np.int32)).cuda()
    u, y = torch.zeros_like(x), torch.zeros_like(x)
    starts = torch.zeros(sf.sf_seq_scan_starts(S, R, D, N), device="cuda")
    work = torch.zeros(max(sf.sf_seq_scan_workspace(S, P, R, D, N, backward=True), sf.sf_seq_conv_backward_workspace(S, P, D, W)), dtype=torch.uint8, device="cuda")
    rest = dict(D=Dk, delta_bias=db, z=z, softplus=True)
    sf.sf_seq_conv(ctx, q, x, w, u, bias=wb, act=sf.SF_ACT_SILU)
    sf.sf_seq_scan(ctx, q, u, delta, A, B, C, y, starts_out=starts, workspace=work, **rest)
    last = torch.from_numpy(np.arange(S) * P + counts - 1).cuda()
    # serving: a 4-bit layer on the last rows, scores of its logits, thresholds from the entropies
    packed, scales = (torch.zeros(b, dtype=torch.uint8, device="cuda") for b in sf.sf_mx4_sizes(S, D))
    pw, sw = (torch.zeros(b, dtype=torch.uint8, device="cuda") for b in sf.sf_mx4_sizes(V, D))
    sf.sf_mx4_quantise(ctx, y, packed, scales, row_ids=last.int())
    sf.sf_mx4_quantise(ctx, head, pw, sw)
    low = torch.zeros(S, V, device="cuda")
    sf.sf_mx4_matmul(ctx, packed, scales, pw, sw, D, low)
    entropy, ids, top, tau = torch.zeros(S, device="cuda"), torch.zeros(S, 2, dtype=torch.int32, device="cuda"), torch.zeros(S, 2, device="cuda"), torch.zeros(2, device="cuda")
    sf.sf_label_logprobs(ctx, low, None, None, entropy_out=entropy, top_ids_out=ids, top_logprobs_out=top)
    sf.sf_universal_thresholds_dev(ctx, entropy, S, [50, 76], 100, tau)
    f = ref.logprobs(num(low), 1.0, np.full(S, -1), 2)
    assert np.array_equal(ids.cpu().numpy(), f["top_ids"]) and np.abs(num(entropy) - f["entropy"]).max() < 200 * E
    assert num(tau)[0] == np.sort(num(entropy))[int(np.ceil(0.5 * S)) - 1]
    # training: full-precision head, loss = -mean log probability
    logits = y[last] @ head.T
    lp, lse, dl = torch.zeros(S, device="cuda"), torch.zeros(S, device="cuda"), torch.zeros_like(logits)
    sf.sf_label_logprobs(ctx, logits, labels, lp, lse_out=lse)
    sf.sf_label_logprobs_backward(ctx, logits, labels, lse, dl, d_logprob=torch.full((S,), -1.0 / S, device="cuda"))
    dy = torch.zeros_like(y)
    dy[last] = dl @ head
    du, dx, dw, dA = torch.zeros_like(u), torch.zeros_like(x), torch.zeros_like(w), torch.zeros_like(A)
    sf.sf_seq_scan_backward(ctx, q, u, delta, A, B, C, dy, starts, work, du_out=du, dA_out=dA, **rest)
    sf.sf_seq_conv_backward(ctx, q, x, w, du, work, bias=wb, act=sf.SF_ACT_SILU, dx_out=dx, dw_out=dw)
    sf.sf_ctx_poll(ctx)
    v = {k: num(t) for k, t in dict(x=x, w=w, wb=wb, delta=delta, A=A, B=B, C=C, Dk=Dk, db=db, z=z, head=head).items()}

    def loss():
        total = 0.0
        for s in range(S):
            at = slice(s * P, s * P + counts[s])
            c = ref.conv(v["x"][at], v["w"], v["wb"], True, np.zeros((W - 1, D)))["y"]
            o = ref.scan(c, v["delta"][at], v["A"], v["B"][at][:, None], v["C"][at][:, None], v["Dk"], v["db"], v["z"][at], True, np.zeros((D, N)))["y"]
            g = o[-1] @ v["head"].T
            total -= (g[int(labels[s])] - np.log(np.exp(g - g.max()).sum()) - g.max()) / S
        return total
    # Differences with step 1e-5 are off by 1e-10 of the third derivative and 2^-53 / 1e-5 = 1e-11 of the loss; the calls by some hundred roundings of
    # values of order 1 / S: 1e-4 of the largest gradient covers both
    for name, got in (("w", dw), ("A", dA), ("x", dx)):
        G = num(got)
        for i in [tuple(rng.integers(0, n) for n in G.shape) for _ in range(6)]:
            if name == "x" and i[0] % P >= counts[i[0] // P]:
                assert G[i] == 0
                continue
            keep = v[name][i]
            v[name][i] = keep + 1e-5
            hi = loss()
            v[name][i] = keep - 1e-5
            lo = loss()
            v[name][i] = keep
            assert abs((hi - lo) / 2e-5 - G[i]) < 1e-4 * np.abs(G).max(), (name, i)

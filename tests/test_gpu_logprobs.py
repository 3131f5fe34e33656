"""Label log probabilities, entropy, alternatives and their gradient against a direct statement in doubles.

Tolerances, with e = 2^-24 and span = the largest |x - max| that counts (below 104 an exponential in fp32 is not zero): an exponential is off by (4 + 2 span) e; a
thread adds at most V / 8 + 16 of them, a row's threads are joined in at most 32 steps: s is off by c = (V / 8 + 64 + 2 span) e relative, ln s by as much, w / s likewise
times H.  A log probability adds the roundings of its own terms, 4 e of each.  p is off by (c + 4 |lse| e) relative.  Half a step of the output type comes on top."""
import numpy as np
import pytest

import sequences as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF_STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
TINY = {"fp32": 1e-37, "bf16": 1e-37, "fp16": 2.0 ** -24}
E = 2.0 ** -24
MARK = 7.0


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
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def dev(a, kind=np.float32):
    return torch.from_numpy(np.ascontiguousarray(a, kind)).cuda()


def logits(rng, n, V, kind, pitch, offset, masked, values="normal"):
    x = rng.standard_normal((n, V)) * 2
    if values == "ties":
        x = rng.integers(-2, 3, (n, V)).astype(float)
    if values == "equal":
        x[:] = 1.5
    if values == "wide":
        x *= 40
    x[rng.random((n, V)) < masked] = -np.inf
    if masked and n > 1:
        x[n // 2] = -np.inf                                # a row with nothing
    t = torch.zeros(n * (V + pitch) + offset, dtype=TYPES[kind], device="cuda")[offset:].view(n, V + pitch)[:, :V]
    t.copy_(torch.from_numpy(x))
    return t


def run(sf, ctx, x, labels, k, scale, n_dev=None):
    n = x.shape[0]
    o = {q: torch.full((n,), MARK, device="cuda") for q in ("logprob", "entropy", "lse")}
    o["top_ids"], o["top_logprobs"] = torch.full((n, k), 77, dtype=torch.int32, device="cuda"), torch.full((n, k), MARK, device="cuda")
    sf.sf_label_logprobs(ctx, x, labels, o["logprob"], entropy_out=o["entropy"], lse_out=o["lse"], top_ids_out=o["top_ids"], top_logprobs_out=o["top_logprobs"],
                         scale=scale, n_dev=n_dev)
    return o


def span_of(X, scale):
    top = np.where(np.isneginf(X).all(1, keepdims=True), 0, X.max(1, keepdims=True))
    return min(np.where(np.isfinite(X), scale * (top - X), 0).max(initial=0), 104.0)


def compare(o, f, X, scale):
    V = X.shape[1]
    span = span_of(X, scale)
    c = (V / 8 + 64 + 2 * span) * E
    lse = np.where(np.isfinite(f["lse"]), np.abs(f["lse"]), 0)
    assert np.array_equal(num(o["top_ids"]), f["top_ids"])
    for q in ("lse", "entropy", "logprob", "top_logprobs"):
        got, want = num(o[q]), f[q]
        assert np.array_equal(np.isneginf(got), np.isneginf(want)) and np.array_equal(np.isnan(got), np.isnan(want)), q
        ok = np.isfinite(want)
        tol = {"lse": c + 4 * E * (lse + span), "entropy": c * (1 + np.abs(f["entropy"])), "logprob": c + 4 * E * np.abs(want)}.get(q, c + 4 * E * np.abs(want))
        with np.errstate(invalid="ignore"):
            assert (np.abs(got - want) <= tol + 2 * E * np.abs(want))[ok].all(), (q, np.nanmax(np.abs(got - want)[ok]), c)


CASES = [
    # n, V, k, kind, pitch, offset, masked, values, scale
    (5, 1, 1, "fp32", 0, 0, 0.3, "normal", 1.5), (300, 2, 2, "fp32", 0, 0, 0.0, "normal", 1.0), (70, 8, 3, "bf16", 0, 0, 0.2, "normal", 1.0),
    (33, 9, 9, "fp16", 0, 1, 0.5, "normal", 0.7), (40, 16, 2, "fp32", 0, 0, 0.1, "ties", 1.0), (21, 17, 5, "fp32", 3, 1, 0.0, "normal", 2.0),
    (9, 33, 8, "bf16", 1, 3, 0.9, "normal", 1.0), (7, 64, 1, "fp16", 0, 0, 0.0, "equal", 1.0), (6, 100, 32, "fp32", 0, 0, 0.3, "normal", 1.0),
    (5, 255, 4, "bf16", 0, 1, 0.0, "ties", 1.0), (5, 256, 6, "fp32", 0, 0, 0.0, "ties", 1.0), (4, 300, 20, "fp32", 1, 0, 0.2, "normal", 1.0), (4, 513, 24, "fp16", 0, 0, 0.0, "equal", 1.0),
    (4, 1000, 32, "fp32", 8, 0, 0.98, "normal", 1.0), (3, 1024, 5, "bf16", 0, 0, 0.0, "normal", 1.0), (3, 1025, 5, "bf16", 0, 0, 0.0, "normal", 1.0),
    (4, 1018, 3, "fp32", 3, 2, 0.1, "wide", 1.0), (4, 2050, 32, "fp32", 1, 1, 0.1, "normal", 0.5), (3, 8193, 8, "bf16", 0, 0, 0.0, "ties", 1.0), (2, 9000, 0, "fp16", 0, 0, 0.2, "normal", 1.0),
    (3, 5000, 31, "bf16", 0, 0, 0.9995, "normal", 1.0), (160, 4099, 4, "bf16", 0, 0, 0.0, "normal", 1.0), (1, 16384, 7, "fp32", 0, 0, 0.0, "normal", 1.0), (2, 20011, 32, "bf16", 0, 1, 0.1, "ties", 1.0),
    (1, 131075, 20, "fp16", 0, 0, 0.2, "wide", 0.3), (2, 70000, 3, "bf16", 0, 0, 0.0, "equal", 1.0), (1, 17000, 5, "fp32", 0, 0, 1.0, "normal", 1.0),
]


@pytest.mark.parametrize("n,V,k,kind,pitch,offset,masked,values,scale", CASES)
def test_scores_and_gradient(env, n, V, k, kind, pitch, offset, masked, values, scale):
    sf, ctx = env
    rng = np.random.default_rng(V * 10 + k)
    x = logits(rng, n, V, kind, pitch, offset, masked, values)
    X = num(x)
    labels = rng.integers(0, V, n)
    labels[rng.random(n) < 0.2] = -1
    if n > 3:
        labels[0] = V                                      # outside: none
    scale = float(np.float32(scale))
    f = ref.logprobs(X, scale, labels, k)
    o = run(sf, ctx, x, dev(labels, np.int32), k, scale)
    compare(o, f, X, scale)
    dl, de, dt = rng.standard_normal(n), rng.standard_normal(n), rng.standard_normal((n, k))
    span = span_of(X, scale)
    lse = np.where(np.isfinite(f["lse"]), np.abs(f["lse"]), 0)[:, None]
    with np.errstate(divide="ignore", invalid="ignore"):
        logp = np.where(f["p"] > 0, np.log(f["p"]), 0.0)
    for use in ((1, 0, 0), (0, 1, 0), (1, 1, 1)):
        g = [v.astype(np.float32).astype(float) if u else None for u, v in zip(use, (dl, de, dt))]
        if k == 0:
            g[2] = None
        d = torch.full((n * (V + pitch) + 16,), MARK, dtype=x.dtype, device="cuda")[offset:].as_strided((n, V), (V + pitch, 1))
        sf.sf_label_logprobs_backward(ctx, x, dev(labels, np.int32), o["lse"], d, d_logprob=None if g[0] is None else dev(g[0]), entropy=o["entropy"],
                                      d_entropy=None if g[1] is None else dev(g[1]), top_ids=o["top_ids"] if g[2] is not None else None,
                                      d_top_logprobs=None if g[2] is None else dev(g[2]), scale=scale)
        want = ref.logprobs_gradient(X, scale, labels, f, *g)
        pull = np.abs(dl) * (g[0] is not None) + (np.abs(dt).sum(1) if g[2] is not None else 0)
        mag = f["p"] * (pull[:, None] + (np.abs(de)[:, None] * (np.abs(logp) + np.abs(f["entropy"])[:, None] + 1) if g[1] is not None else 0))
        c = (V / 8 + 64 + 2 * span + 8 * lse) * E
        tol = scale * (c * mag + (k + 4) * E * pull[:, None])
        got = num(d)
        bad = np.abs(got - want) > tol + HALF_STEP[kind] * np.abs(want) + TINY[kind]
        assert not bad.any(), (use, np.argwhere(bad)[:3], got[bad][:3], want[bad][:3])
        assert (got[np.isneginf(X)] == 0).all()


@pytest.mark.parametrize("V", [16, 300, 5000])
def test_lowest_values_infinities_and_nan(env, V):
    """Rows of the type's lowest value (a mask that is not minus infinity), of one entry among them, with an infinity, with a NaN."""
    sf, ctx = env
    x = torch.zeros(6, V, device="cuda")
    low = float(np.finfo(np.float32).min)
    x[0] = low
    x[1] = low
    x[1, V // 2] = 3.0
    x[2, 1] = float("inf")
    x[3, 2] = float("nan")
    x[4, 5] = -0.0
    x[5] = -low                                            # the largest numbers
    x[3, 7] = -float("inf")
    labels = torch.full((6,), 1, dtype=torch.int32, device="cuda")
    o = run(sf, ctx, x, labels, 3, 1.0)
    lp, h, ids = num(o["logprob"]), num(o["entropy"]), num(o["top_ids"])
    c = (V / 8 + 64) * E
    for r in (0, 4, 5):                                    # equal entries
        assert abs(h[r] - np.log(V)) < c * (1 + np.log(V)) and abs(lp[r] + np.log(V)) < c + 4 * E * np.log(V) and ids[r].tolist() == [0, 1, 2], r
    assert h[1] == 0 and ids[1].tolist() == [V // 2, 0, 1] and num(o["lse"])[1] == 3 and num(o["top_logprobs"])[1, 0] == 0
    for r in (2, 3):
        assert np.isnan(h[r]) and np.isnan(lp[r]) and np.isnan(num(o["lse"])[r]), r
    assert ids[2, 0] == 1 and 2 not in ids[3]
    d = torch.zeros_like(x)
    sf.sf_label_logprobs_backward(ctx, x, labels, o["lse"], d, d_logprob=torch.ones(6, device="cuda"), entropy=o["entropy"], d_entropy=torch.ones(6, device="cuda"))
    g = num(d)
    assert np.isnan(g[2]).any() and np.isnan(g[3]).any() and np.isfinite(g[[0, 1, 4, 5]]).all()
    assert abs(g[4, 1] - (1 - 1 / V)) < 4 * c and g[3, 7] == 0          # masked: 0 in a row with a NaN too


def test_rows_behind_the_count_and_each_output_alone(env):
    sf, ctx = env
    rng = np.random.default_rng(2)
    for V in (8, 400, 3000):
        n, k = 11, 3
        x, labels = logits(rng, n, V, "fp32", 0, 0, 0.1), dev(rng.integers(0, V, n), np.int32)
        full = run(sf, ctx, x, labels, k, 1.0)
        some = run(sf, ctx, x, labels, k, 1.0, n_dev=torch.tensor([4], dtype=torch.int32, device="cuda"))
        for q in full:
            assert torch.equal(some[q][:4], full[q][:4]) and bool((some[q][4:] == (77 if q == "top_ids" else MARK)).all()), q
        d, part = torch.zeros_like(x), torch.full_like(x, MARK)
        args = dict(d_logprob=torch.ones(n, device="cuda"))
        sf.sf_label_logprobs_backward(ctx, x, labels, full["lse"], d, **args)
        sf.sf_label_logprobs_backward(ctx, x, labels, full["lse"], part, n_dev=torch.tensor([4], dtype=torch.int32, device="cuda"), **args)
        assert torch.equal(part[:4], d[:4]) and bool((part[4:] == MARK).all())
        sf.sf_ctx_poll(ctx, reset=True)
        run(sf, ctx, x, labels, k, 1.0, n_dev=torch.tensor([50], dtype=torch.int32, device="cuda"))
        assert sf.sf_ctx_poll(ctx, reset=True, raise_on_error=False).device_error == sf.SF_ERR_CAPACITY
        for q in ("logprob", "entropy", "lse", "top_ids", "top_logprobs"):
            alone = torch.zeros_like(full[q])
            kw = {q + "_out": alone} if q != "logprob" else {}
            sf.sf_label_logprobs(ctx, x, labels if q == "logprob" else None, alone if q == "logprob" else None, **kw)
            assert torch.equal(alone, full[q]), q


def test_captured_and_on_other_streams(env):
    sf, ctx = env
    rng = np.random.default_rng(3)
    for n, V in ((500, 16), (3, 40000)):                   # the second: clusters
        xs = [logits(rng, n, V, "bf16", 0, 0, 0.1) for _ in range(2)]
        labels = dev(rng.integers(0, V, n), np.int32)
        want = [run(sf, ctx, x, labels, 4, 1.0) for x in xs]
        x = xs[0].clone()
        o = {q: torch.zeros_like(v) for q, v in want[0].items()}
        call = lambda: sf.sf_label_logprobs(ctx, x, labels, o["logprob"], entropy_out=o["entropy"], lse_out=o["lse"], top_ids_out=o["top_ids"], top_logprobs_out=o["top_logprobs"])  # noqa: E731
        call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        for i in (1, 0):
            x.copy_(xs[i])
            g.replay()
            torch.cuda.synchronize()
            for q in o:
                assert torch.equal(o[q], want[i][q]), q
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        torch.cuda.synchronize()
        got = []
        for _ in range(3):
            for s, v in zip(streams, xs):
                with torch.cuda.stream(s):
                    got.append(run(sf, ctx, v, labels, 4, 1.0))
        torch.cuda.synchronize()
        for i, v in enumerate(got):
            for q in v:
                assert torch.equal(v[q], want[i % 2][q]), q


def test_entries_behind_2_to_the_32_bytes(env):
    """A row that lies far, and a row that is long."""
    sf, ctx = env
    V, n = 65536, 40000                                    # 5.2 GB of bf16
    x = torch.zeros(n, V, dtype=torch.bfloat16, device="cuda")
    x[n - 1, V - 3] = 20.0
    o = run(sf, ctx, x, torch.full((n,), V - 3, dtype=torch.int32, device="cuda"), 1, 1.0)
    p = np.exp(20.0) / (np.exp(20.0) + V - 1)
    assert num(o["top_ids"])[n - 1, 0] == V - 3 and abs(num(o["logprob"])[n - 1] - np.log(p)) < (V / 8 + 120) * E
    assert abs(num(o["entropy"])[5] - np.log(V)) < (V / 8 + 64) * E * 13
    d = torch.zeros_like(x)
    sf.sf_label_logprobs_backward(ctx, x, torch.full((n,), V - 3, dtype=torch.int32, device="cuda"), o["lse"], d, d_logprob=torch.ones(n, device="cuda"))
    assert abs(num(d[n - 1, V - 3]) - (1 - p)) < (V / 8 + 300) * E + 2.0 ** -8 * (1 - p) and abs(num(d[n - 2, V - 3]) - (1 - 1 / V)) < 2.0 ** -8
    one = x.view(1, -1)[:, :2 ** 30 + 5]
    o = run(sf, ctx, one, torch.zeros(1, dtype=torch.int32, device="cuda"), 2, 1.0)
    # a thread adds 2^30 / 4096 ones one by one: its sum is exact, and so is the row's count
    assert abs(num(o["lse"])[0] - np.log(2.0 ** 30 + 5)) < 64 * E * 21 and num(o["top_ids"])[0].tolist() == [0, 1]

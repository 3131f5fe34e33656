"""The calls on sequences and on logits with numbers that must not matter: scratch full of NaN, rows of no sequence full of NaN, a NaN in another sequence. Comparisons
here fail on a NaN wherever one comes out (a comparison by `>` does not)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import sequences as ref  # noqa: E402
import test_gpu_logprobs as scores  # noqa: E402
import test_gpu_sequences as base  # noqa: E402
from test_gpu_sequences import CONV, E, HALF_STEP, MARK, SCAN, TINY, TYPES, env, lay_out, like, num, rows_in, scan_case  # noqa: E402, F401

NAN = float("nan")


def strict(name, got, want, tol, kind):
    bad = ~(np.abs(got - want) <= tol + HALF_STEP[kind] * np.abs(want) + TINY[kind])
    assert not bad.any(), (name, np.argwhere(bad)[:4], got[bad][:4], want[bad][:4])


@pytest.mark.parametrize("case", CONV, ids=str)
def test_convolution_without_a_nan(env, monkeypatch, case):  # noqa: F811
    monkeypatch.setattr(base, "close", strict)
    base.test_convolution(env, *case)


@pytest.mark.parametrize("case", SCAN, ids=str)
def test_scan_without_a_nan(env, monkeypatch, case):  # noqa: F811
    monkeypatch.setattr(base, "close", strict)
    base.test_scan(env, *case)


@pytest.mark.parametrize("n,V,k,kind,pitch,offset,masked,values,scale", scores.CASES)
def test_logits_gradient_without_a_nan(env, n, V, k, kind, pitch, offset, masked, values, scale):  # noqa: F811
    sf, ctx = env
    rng = np.random.default_rng(V * 10 + k + 1)
    x = scores.logits(rng, n, V, kind, pitch, offset, masked, values)
    X, labels, scale = num(x), rng.integers(-1, V, n), float(np.float32(scale))
    f = ref.logprobs(X, scale, labels, k)
    o = scores.run(sf, ctx, x, scores.dev(labels, np.int32), k, scale)
    g = [v.astype(np.float32).astype(float) for v in (rng.standard_normal(n), rng.standard_normal(n), rng.standard_normal((n, k)))]
    d = torch.full((n, V + pitch), MARK, dtype=x.dtype, device="cuda")
    sf.sf_label_logprobs_backward(ctx, x, scores.dev(labels, np.int32), o["lse"], d[:, :V], d_logprob=scores.dev(g[0]), entropy=o["entropy"], d_entropy=scores.dev(g[1]),
                                  top_ids=o["top_ids"] if k else None, d_top_logprobs=scores.dev(g[2]) if k else None, scale=scale)
    want = ref.logprobs_gradient(X, scale, labels, f, g[0], g[1], g[2] if k else None)
    pull = np.abs(g[0]) + np.abs(g[2]).sum(1)
    with np.errstate(divide="ignore"):
        logp = np.where(f["p"] > 0, np.log(f["p"]), 0.0)
    mag = f["p"] * (pull[:, None] + np.abs(g[1])[:, None] * (np.abs(logp) + np.abs(f["entropy"])[:, None] + 1))
    lse = np.where(np.isfinite(f["lse"]), np.abs(f["lse"]), 0)[:, None]
    c = (V / 8 + 64 + 2 * scores.span_of(X, scale) + 8 * lse) * E      # as there
    strict("d_logits", num(d[:, :V]), want, scale * (c * mag + (k + 4) * E * pull[:, None]), kind)
    assert bool((d[:, V:] == MARK).all())


def conv_call(sf, ctx, q, S, most, x, dy, w, b, pool, d_pool, fill):
    """The convolution and its gradients with scratch full of `fill`: everything that comes out."""
    D, W = w.shape
    o = {"y": torch.full_like(x, MARK), "state": pool.clone(), "dx": torch.full_like(x, MARK), "dw": torch.full_like(w, MARK), "db": torch.full((D,), MARK, device="cuda"), "d_in": torch.full_like(pool, MARK)}
    work = torch.full((sf.sf_seq_conv_backward_workspace(S, most, D, W) // 4,), fill, device="cuda")
    sf.sf_seq_conv(ctx, q, x, w, o["y"], bias=b, act=sf.SF_ACT_SILU, state_in=pool, state_out=o["state"])
    sf.sf_seq_conv_backward(ctx, q, x, w, dy, work, bias=b, act=sf.SF_ACT_SILU, state_in=pool, d_state=d_pool, dx_out=o["dx"], dw_out=o["dw"], dbias_out=o["db"], d_state_in_out=o["d_in"])
    return o


def scan_call(sf, ctx, q, S, most, t, pool, d_pool, fill):
    R, D = t["u"].shape
    N, G = t["A"].shape[1], t["B"].shape[1] // t["A"].shape[1]
    rest, rows = dict(D=t["D"], delta_bias=t["bias"], z=t["z"], softplus=True), (t["u"], t["delta"], t["A"], t["B"], t["C"])
    work = torch.full((sf.sf_seq_scan_workspace(S, most, R, D, N, G, backward=True) // 4,), fill, device="cuda")
    starts = torch.full((sf.sf_seq_scan_starts(S, R, D, N),), fill, device="cuda")
    o = {"y": torch.full_like(t["u"], MARK), "serve": torch.full_like(t["u"], MARK), "state": pool.clone(), "d_in": torch.full_like(pool, MARK)}
    g = {k + "_out": torch.full_like(x, MARK) for k, x in (("du", t["u"]), ("d_delta", t["delta"]), ("dB", t["B"]), ("dC", t["C"]), ("dz", t["z"]), ("dA", t["A"]), ("dD", t["D"]), ("d_delta_bias", t["bias"]))}
    sf.sf_seq_scan(ctx, q, *rows, o["serve"], workspace=work, state_in=pool, **rest)
    work.fill_(fill)
    sf.sf_seq_scan(ctx, q, *rows, o["y"], workspace=work, state_in=pool, state_out=o["state"], starts_out=starts, **rest)
    work.fill_(fill)
    sf.sf_seq_scan_backward(ctx, q, *rows, t["dy"], starts, work, d_state=d_pool, d_state_in_out=o["d_in"], **g, **rest)
    return {**o, **g}


def same(a, b):
    for k in a:
        assert torch.equal(a[k], b[k]) and bool(torch.isfinite(b[k]).all()), k


SHAPES = [([300], 24, "fp32"), ([260, 0, 131], 33, "bf16"), ([9, 3, 0, 17, 8, 1] * 40, 64, "bf16"), ([1, 0, 1, 1], 130, "fp16"), ([40, 2, 16], 136, "fp32")]


@pytest.mark.parametrize("lengths,D,kind", SHAPES)
@pytest.mark.parametrize("planes", [False, True])
def test_scratch_and_rows_of_no_sequence_do_not_matter(env, lengths, D, kind, planes):  # noqa: F811
    """Twice the same into marked outputs: scratch of zeros and of NaN, rows behind the sequences' counts of zeros and of NaN."""
    sf, ctx = env
    S, most, N, W = len(lengths), max(lengths), 16, 4
    rng = np.random.default_rng(D + planes)
    q, first, R, slot, t, pool, d_pool = scan_case(sf, rng, D, N, 1, kind, lengths, planes, True, 0, 0, True, True, True, True)
    x, dy, w, b = rows_in(rng, R, D, kind), rows_in(rng, R, D, kind), torch.randn(D, W, device="cuda"), torch.randn(D, device="cuda")
    c_pool, cd_pool = (torch.from_numpy(rng.standard_normal((S + 2, W - 1, D))).to(TYPES[kind]).cuda() for _ in range(2))
    out = torch.ones(R, dtype=torch.bool, device="cuda")
    for s, n in enumerate(lengths):
        out[first[s]:first[s] + n] = False
    runs = []
    for junk in (0.0, NAN):
        for v in [x, dy] + [t[k] for k in ("u", "delta", "B", "C", "z", "dy")]:
            v[out] = junk
        runs.append((conv_call(sf, ctx, q, S, most, x, dy, w, b, c_pool, cd_pool, junk), scan_call(sf, ctx, q, S, most, t, pool, d_pool, junk)))
    same(runs[0][0], runs[1][0])
    same(runs[0][1], runs[1][1])
    sf.sf_ctx_poll(ctx)


def test_a_nan_goes_no_further_than_its_rows_reach_in_both_gradients(env):  # noqa: F811
    """Sequences of several tiles: a NaN in one row's gradient, input or step touches rows of its own sequence only, and of the convolution those within its taps."""
    sf, ctx = env
    S, L, D, N, W = 3, 40, 32, 16, 4
    rng = np.random.default_rng(8)
    q, first, R, slot, t, pool, _ = scan_case(sf, rng, D, N, 1, "fp32", [L] * S, False, False, 0, 0, True, True, True, True)
    x, dy, w, b = rows_in(rng, R, D, "fp32"), rows_in(rng, R, D, "fp32"), torch.randn(D, W, device="cuda"), torch.randn(D, device="cuda")
    c_pool = torch.zeros(S + 2, W - 1, D, device="cuda")
    at, ch = L + 17, 5
    for bad in ("dy", "x"):
        xx, gg = x.clone(), dy.clone()
        (gg if bad == "dy" else xx)[at, ch] = NAN
        o = conv_call(sf, ctx, q, S, L, xx, gg, w, b, c_pool, c_pool, NAN)
        dx, want = num(o["dx"]), np.zeros((R, D), bool)
        want[at - W + 1:at + (1 if bad == "dy" else W), ch] = True     # x: its own pre and the W - 1 after it, whose gradients reach W - 1 rows back
        assert np.array_equal(np.isnan(dx), want), bad
        nan_dw = np.isnan(num(o["dw"]))
        assert nan_dw[ch].all() and not np.delete(nan_dw, ch, 0).any() and np.isnan(num(o["db"])).sum() == 1 and bool(torch.isfinite(o["d_in"]).all())
    for bad in ("dy", "delta", "B"):
        v = {k: None if a is None else a.clone() for k, a in t.items()}
        v[bad][at, ch] = NAN
        o = scan_call(sf, ctx, q, S, L, v, pool, torch.zeros_like(pool), NAN)
        for k in ("du_out", "d_delta_out", "dB_out", "dC_out", "dz_out"):
            a = np.isnan(num(o[k])).any(1)
            assert not a[:L].any() and not a[2 * L:].any(), (bad, k)
            if bad == "dy":
                assert not a[at + 1:].any(), k             # gradients go from the last row to the first
        assert np.isnan(num(o["du_out"])[L:at + 1]).any() and bool(torch.isfinite(o["d_in"][[0, 2, 3, 4]]).all())


def test_convolution_captured_and_on_other_streams(env):  # noqa: F811
    """Forward and backward in a graph, replayed on new inputs; two streams of one context at once with workspaces of their own; states in one pool each."""
    sf, ctx = env
    lengths, D, W = [300, 2, 0, 65], 40, 4
    rng = np.random.default_rng(6)
    q, first, R, slot = lay_out(sf, rng, lengths, False, True)
    S = len(lengths)
    w, b, dy = torch.randn(D, W, device="cuda"), torch.randn(D, device="cuda"), rows_in(rng, R, D, "bf16")
    before, d_after = (torch.randn(S + 2, W - 1, D, device="cuda").bfloat16() for _ in range(2))

    def buffers():
        return {"work": torch.zeros(sf.sf_seq_conv_backward_workspace(S, 300, D, W), dtype=torch.uint8, device="cuda"), "y": torch.zeros(R, D, device="cuda").bfloat16(), "dx": torch.zeros(R, D, device="cuda").bfloat16(),
                "dw": torch.zeros(D, W, device="cuda"), "db": torch.zeros(D, device="cuda"), "pool": before.clone(), "d_pool": d_after.clone()}

    def both(x, o):
        o["pool"].copy_(before)
        o["d_pool"].copy_(d_after)
        sf.sf_seq_conv(ctx, q, x, w, o["y"], bias=b, act=sf.SF_ACT_SILU, state_in=o["pool"], state_out=o["pool"])
        sf.sf_seq_conv_backward(ctx, q, x, w, dy, o["work"], bias=b, act=sf.SF_ACT_SILU, state_in=before, d_state=o["d_pool"], dx_out=o["dx"], dw_out=o["dw"], dbias_out=o["db"], d_state_in_out=o["d_pool"])
    inputs = [rows_in(rng, R, D, "bf16") for _ in range(2)]
    want = [buffers(), buffers()]
    for x, o in zip(inputs, want):
        both(x, o)
    x, o = inputs[0].clone(), buffers()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(x, o)
    for i in (1, 0, 1):
        x.copy_(inputs[i])
        for k in ("y", "dx", "dw", "db"):
            o[k].fill_(MARK)
        graph.replay()
        torch.cuda.synchronize()
        for k in o:
            assert k == "work" or torch.equal(o[k], want[i][k]), (i, k)
    streams, sets = [torch.cuda.Stream(), torch.cuda.Stream()], [buffers(), buffers()]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, v, x in zip(streams, sets, inputs):
            with torch.cuda.stream(s):
                both(x, v)
    torch.cuda.synchronize()
    for v, o in zip(sets, want):
        for k in o:
            assert k == "work" or torch.equal(v[k], o[k]), k
    sf.sf_ctx_poll(ctx)

"""What the calls on logits promise at the ends of their range: rows of more than 2^30 entries, threads without a row, rows that lie far from zero."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import sequences as ref  # noqa: E402
from test_gpu_logprobs import E, HALF_STEP, MARK, TINY, TYPES, dev, env, num, run, span_of  # noqa: E402, F401


def test_gradient_of_a_row_of_more_than_a_billion_entries(env):  # noqa: F811
    """Threads behind the last row, and those of a row behind the count, do nothing: 1.3e9 entries by four chunks 3.2e8 entries apart reach beyond 2^31 from there."""
    sf, ctx = env
    V, k = 1_300_000_003, 2
    x = torch.zeros(2 * V, dtype=torch.bfloat16, device="cuda").view(2, V)
    x[:, 5], x[0, V - 1] = 20.0, 21.0
    n_dev = torch.ones(1, dtype=torch.int32, device="cuda")
    labels, ids = torch.tensor([7, 7], dtype=torch.int32, device="cuda"), torch.tensor([[V - 1, 5], [5, 0]], dtype=torch.int32, device="cuda")
    s = V - 2 + np.exp(20.0) + np.exp(21.0)
    lse = torch.full((2,), float(np.log(s)), device="cuda")
    g, gt = 0.5, (2.0, -1.0)
    d = torch.full_like(x, MARK)
    sf.sf_label_logprobs_backward(ctx, x, labels, lse, d, d_logprob=torch.full((2,), g, device="cuda"), top_ids=ids, d_top_logprobs=torch.tensor([gt, gt], device="cuda"), n_dev=n_dev)
    sf.sf_ctx_poll(ctx)
    total = g + sum(gt)
    p = np.exp([0.0, 20.0, 21.0]) / s
    # lse rounded to fp32 is off by e |lse|, an exponential by (4 + 2 span) e; half a step of bf16 on top
    for i, want in ((7, g - p[0] * total), (5, gt[1] - p[1] * total), (V - 1, gt[0] - p[2] * total), (0, -p[0] * total), (V - 2, -p[0] * total), (V // 2, -p[0] * total)):
        assert abs(float(d[0, i]) - want) <= 2.0 ** -8 * abs(want) + 100 * E * total, i
    rest = d[0].clone()
    rest[torch.tensor([5, 7, V - 1], device="cuda")] = d[0, 0]
    assert bool((rest == d[0, 0]).all()) and bool((d[1] == MARK).all())


FAR = [  # n, V, k, kind, scale, pitch
    (300, 1, 1, "fp32", 1.0, 0), (70, 2, 1, "bf16", 0.7, 0), (200, 16, 2, "fp32", 1.0, 0), (50, 17, 3, "fp16", 1.5, 1), (40, 100, 2, "fp32", 0.7, 3), (20, 511, 0, "bf16", 1.0, 0),
    (40, 515, 2, "fp32", 1.0, 1), (30, 600, 2, "bf16", 1.0, 0), (9, 5000, 4, "fp32", 0.7, 0), (5, 40000, 8, "bf16", 1.0, 0),
]


@pytest.mark.parametrize("n,V,k,kind,scale,pitch", FAR)
def test_gradient_of_rows_far_from_zero(env, n, V, k, kind, scale, pitch):  # noqa: F811
    """Rows of nothing but the type's lowest or largest value, and rows around a large number, between ordinary ones.  The tolerance is the one of ordinary rows without
    the rounding of lse where |lse| >= 1024: exponentials of differences from the row's maximum are off by (4 + 2 span) e each, their sum by one e a term."""
    sf, ctx = env
    rng = np.random.default_rng(V + k)
    low = float(torch.finfo(TYPES[kind]).min) if kind != "fp16" else -60000.0
    x = rng.standard_normal((n, V)) * 2
    for r in range(n):
        if r % 5 == 0:
            x[r] = low if r % 10 == 0 else -low
        elif r % 5 == 1:
            x[r] += (1e6 if kind == "fp32" else 2e4) * rng.choice([-1, 1])
        elif r % 5 == 2:
            x[r, rng.random(V) < 0.4] = low                # a mask by the lowest value
        elif r % 5 == 3:
            x[r] -= 5000
            x[r, rng.random(V) < 0.3] = -np.inf
    t = torch.zeros(n, V + pitch, dtype=TYPES[kind], device="cuda")[:, :V]
    t.copy_(torch.from_numpy(x))
    X, scale = num(t), float(np.float32(scale))
    labels = rng.integers(0, V, n)
    labels[rng.random(n) < 0.2] = -1
    f = ref.logprobs(X, scale, labels, k)
    o = run(sf, ctx, t, dev(labels, np.int32), k, scale)
    assert np.array_equal(num(o["top_ids"]), f["top_ids"])
    dl, de, dt = rng.standard_normal(n), rng.standard_normal(n), rng.standard_normal((n, k))
    quiet = rng.random(n) < 0.2                            # rows whose outputs nobody uses
    dl[quiet] = de[quiet] = 0
    span, lse = span_of(X, scale), np.abs(np.where(np.isfinite(f["lse"]), f["lse"], 0))[:, None]
    with np.errstate(divide="ignore", invalid="ignore"):
        logp = np.where(f["p"] > 0, np.log(f["p"]), 0.0)
    for use in ((1, 0, 0), (0, 1, 0), (1, 1, 1)):
        g = [v.astype(np.float32).astype(float) if u else None for u, v in zip(use, (dl, de, dt))]
        if k == 0:
            g[2] = None
        d = torch.full((n, V + pitch), MARK, dtype=t.dtype, device="cuda")[:, :V]
        sf.sf_label_logprobs_backward(ctx, t, dev(labels, np.int32), o["lse"], d, d_logprob=None if g[0] is None else dev(g[0]), entropy=o["entropy"],
                                      d_entropy=None if g[1] is None else dev(g[1]), top_ids=o["top_ids"] if g[2] is not None else None,
                                      d_top_logprobs=None if g[2] is None else dev(g[2]), scale=scale)
        want = ref.logprobs_gradient(X, scale, labels, f, *g)
        pull = np.abs(dl) * (g[0] is not None) + (np.abs(dt).sum(1) if g[2] is not None else 0)
        mag = f["p"] * (pull[:, None] + (np.abs(de)[:, None] * (np.abs(logp) + np.abs(f["entropy"])[:, None] + 1) if g[1] is not None else 0))
        c = (V / 8 + 64 + 2 * span + 8 * np.where(lse < 1024, lse, 0)) * E
        tol = scale * (c * mag + (k + 4) * E * pull[:, None])
        got = num(d)
        bad = ~(np.abs(got - want) <= tol + HALF_STEP[kind] * np.abs(want) + TINY[kind])
        assert not bad.any(), (use, np.argwhere(bad)[:3], got[bad][:3], want[bad][:3])
    again = torch.full((n, V + pitch), MARK, dtype=t.dtype, device="cuda")[:, :V]
    sf.sf_label_logprobs_backward(ctx, t, dev(labels, np.int32), o["lse"], again, d_logprob=dev(g[0]), entropy=o["entropy"], d_entropy=dev(g[1]),
                                  top_ids=o["top_ids"] if k else None, d_top_logprobs=dev(g[2]) if k else None, scale=scale)
    assert torch.equal(d, again)
    sf.sf_ctx_poll(ctx)


@pytest.mark.parametrize("n,V", [(n, V) for n in (1, 16, 17, 148, 149, 296, 297) for V in (12288, 12289, 32768, 32769)] + [(n, V) for n in (2, 16, 17) for V in (196607, 196608)])
def test_scores_on_both_sides_of_every_choice_of_threads(env, n, V):  # noqa: F811
    """Threads a row are chosen by n and V: labels, entropies and alternatives of rows that are alike but for their order have to come out alike, and right."""
    sf, ctx = env
    k = 5
    g = torch.Generator(device="cuda")
    g.manual_seed(V + n)
    row = (torch.randn(V, device="cuda", generator=g) * 2).bfloat16()
    shift = torch.arange(n, device="cuda") * 37 % V
    x = torch.stack([row.roll(int(s)) for s in shift])
    labels = ((shift + 3) % V).int()                       # entry 3 of the row wherever it lies now
    o = run(sf, ctx, x, labels, k, 1.0)
    z = num(row)
    lse = z.max() + np.log(np.exp(z - z.max()).sum())
    p = np.exp(z - lse)
    c = (V / 8 + 64 + 2 * (z.max() - z.min())) * E
    assert (np.abs(num(o["lse"]) - lse) <= c + 4 * E * np.abs(lse)).all()
    assert (np.abs(num(o["logprob"]) - (z[3] - lse)) <= c + 6 * E * np.abs(z[3] - lse)).all()
    h = -(p * (z - lse)).sum()
    assert (np.abs(num(o["entropy"]) - h) <= c * (1 + h)).all()
    X = num(x)
    order = np.argsort(-X, axis=1, kind="stable")[:, :k]   # ties to the lowest index
    assert np.array_equal(num(o["top_ids"]), order)
    top = np.take_along_axis(X, order, 1) - lse
    assert (np.abs(num(o["top_logprobs"]) - top) <= c + 6 * E * np.abs(top)).all()


@pytest.mark.parametrize("V,kind", [(11000, "bf16"), (700, "fp32")])      # (rows on 16-byte boundaries: sums in the same order wherever a row lies)
def test_gradient_of_rows_far_from_zero_among_many(env, V, kind):  # noqa: F811
    """More rows than the machine takes at once: each as it comes out among a few, where the rows above are compared with the formula."""
    sf, ctx = env
    few, times = 10, 5_000_000 // V // 10
    g = torch.Generator(device="cuda")
    g.manual_seed(V)
    x = torch.randn(few, V, device="cuda", generator=g) * 2
    x[::5] = float(torch.finfo(TYPES[kind]).min)
    x[1::5] += 20000
    x[3::5, ::3] = -float("inf")
    x = x.to(TYPES[kind])
    labels = torch.arange(few, device="cuda", dtype=torch.int32) * 7
    labels[4] = -1
    dl, de = torch.randn(few, device="cuda", generator=g), torch.randn(few, device="cuda", generator=g)

    def grad(times):
        many = lambda t: t.repeat(times, *[1] * (t.dim() - 1))  # noqa: E731
        z, y = many(x), many(labels)
        o = run(sf, ctx, z, y, 1, 1.0)
        d = torch.full_like(z, MARK)
        sf.sf_label_logprobs_backward(ctx, z, y, o["lse"], d, d_logprob=many(dl), entropy=o["entropy"], d_entropy=many(de))
        return o, d
    o, want = grad(1)
    p, got = grad(times)
    assert bool(torch.isfinite(want).all()) and torch.equal(got, want.repeat(times, 1))
    for k in o:
        assert torch.equal(p[k], o[k].repeat(times, *[1] * (o[k].dim() - 1))), k

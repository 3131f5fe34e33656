"""A slow model of sequence layers behind the assignment: fast model's probabilities -> sf_route -> the assigned flows' wide rows, read as planes of P rows of 16 a flow ->
convolution -> scan -> head -> entropies of the assigned flows -> a threshold for the next tier; everything is sized by the capacity, the number of assigned flows stays on the device."""
import numpy as np
import pytest

import flowgen
import oracle
import sequences as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_sequences import E, MARK, num  # noqa: E402


@pytest.fixture(scope="module")
def env():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2402_03694_b200 import binding as sf, build, harness as hz
    build.build()
    ctx = sf.sf_ctx_create(0, 0)
    yield sf, hz, ctx
    sf.sf_ctx_destroy(ctx)


def test_assigned_flows_through_sequence_layers(env):
    sf, hz, ctx = env
    n, C, P, D, N, W, V = 900, 6, 20, 16, 8, 4, 5
    rng = np.random.default_rng(21)
    prob = rng.dirichlet([0.5] * C, size=n).astype(np.float32)
    tau = np.full(C, 0.55, np.float32)
    want = oracle.route_lc(prob, tau)
    wide, valid = flowgen.gen_packets(22, n, P, 13), rng.integers(1, P + 1, n).astype(np.uint8)
    w = hz.upload_packets(wide, n_valid=valid)
    cap = want["n_esc"] + 40                               # more room than flows
    ids, n_esc = torch.zeros(n, dtype=torch.uint32, device="cuda"), torch.zeros(1, dtype=torch.uint32, device="cuda")
    rows = torch.full((cap, P * 16), float("nan"), device="cuda")
    sf.sf_route(ctx, sf.make_route_cfg(sf.SF_LC_GT, hz.dev(tau), sf.SF_MLP16, sf.SF_F32, P, cap), hz.dev(prob), n, C, w["struct"], ids, n_esc, rows)
    # planes of P rows a flow: as many sequences as there is room, of those behind the assigned flows none has a row
    at = torch.arange(cap, device="cuda")
    counts = torch.where(at < n_esc.to(torch.int64), torch.from_numpy(valid).cuda().long()[ids.to(torch.int64)[:cap]], 0).int()
    q = sf.make_sequences(torch.arange(cap + 1, dtype=torch.int32, device="cuda") * P, P, counts=counts)
    x, R = rows.view(cap * P, 16), cap * P
    f32 = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda()  # noqa: E731
    taps, bias, A, skip, step = f32(D, W) / 2, f32(D) / 4, -f32(D, N).abs() - 0.05, f32(D), f32(D) / 4 - 2
    to_delta, to_b, to_c, to_z, head = f32(D, D) / 8, f32(D, N) / 4, f32(D, N) / 4, f32(D, D) / 4, f32(V, D)
    u, y = torch.full((R, D), MARK, device="cuda"), torch.full((R, D), MARK, device="cuda")
    sf.sf_seq_conv(ctx, q, x, taps, u, bias=bias, act=sf.SF_ACT_SILU)
    delta, B, Cc, z = u @ to_delta, u @ to_b, u @ to_c, u @ to_z
    state = torch.zeros(cap, D, N, device="cuda")
    work = torch.zeros(sf.sf_seq_scan_workspace(cap, P, R, D, N), dtype=torch.uint8, device="cuda")
    sf.sf_seq_scan(ctx, q, u, delta, A, B, Cc, y, D=skip, delta_bias=step, z=z, softplus=True, state_out=state, workspace=work)
    last = y[(at * P + counts - 1).clamp(min=0)]
    logits = last @ head.T
    entropy, lse = torch.full((cap,), MARK, device="cuda"), torch.full((cap,), MARK, device="cuda")
    best, top = torch.full((cap, 1), -7, dtype=torch.int32, device="cuda"), torch.full((cap, 1), MARK, device="cuda")
    sf.sf_label_logprobs(ctx, logits, None, None, entropy_out=entropy, lse_out=lse, top_ids_out=best, top_logprobs_out=top, n_dev=n_esc)
    k = want["n_esc"]
    tau2 = torch.zeros(1, device="cuda")
    sf.sf_universal_thresholds_dev(ctx, entropy, k, [76], 100, tau2)
    sf.sf_ctx_poll(ctx)
    assert int(n_esc.cpu().numpy()[0]) == k and np.array_equal(ids.cpu().numpy()[:k], want["esc_ids"])
    X = oracle.wide_rows(0, want["esc_ids"], wide, P, False, n_valid=valid).reshape(k, P, 16).astype(np.float64)
    assert np.array_equal(num(x).reshape(cap, P, 16)[:k], X)
    U, Y, DE, B_, C_, Z = num(u).reshape(cap, P, D), num(y).reshape(cap, P, D), num(delta).reshape(cap, P, D), num(B).reshape(cap, P, 1, N), num(Cc).reshape(cap, P, 1, N), num(z).reshape(cap, P, D)
    for i in range(k):
        c = int(valid[want["esc_ids"][i]])
        r = ref.conv(X[i, :c], num(taps), num(bias), True, np.zeros((W - 1, D)))["y"]
        m = ref.conv(X[i, :c], num(taps), num(bias), False, np.zeros((W - 1, D)), ab=np.abs)["y"]
        assert (np.abs(U[i, :c] - r) <= 1.1 * (W + 24 + 2 * m) * E * m + E * np.abs(r)).all() and (U[i, c:] == MARK).all(), i
        args = (U[i, :c], DE[i, :c], num(A), B_[i, :c], C_[i, :c], num(skip), num(step), Z[i, :c], True, np.zeros((D, N)))
        r, m = ref.scan(*args), ref.scan(*args, ab=np.abs)
        most = ref.softplus(DE[i, :c] + num(step)).max() * np.abs(num(A)).max()
        tol = (c * (8 + 24 * most) + 4 * N + D + 64 + 4 * np.abs(Z[i, :c]).max()) * E
        assert (np.abs(Y[i, :c] - r["y"]) <= tol * m["y"] + E * np.abs(r["y"])).all() and (Y[i, c:] == MARK).all(), i
        assert (np.abs(num(state[i]) - r["state"]) <= tol * m["state"] + E * np.abs(r["state"])).all(), i
    f = ref.logprobs(num(logits)[:k], 1.0, np.full(k, -1), 1)
    span = (num(logits)[:k].max(1) - num(logits)[:k].min(1)).max()
    assert np.array_equal(best.cpu().numpy()[:k], f["top_ids"]) and (np.abs(num(entropy)[:k] - f["entropy"]) <= (V / 8 + 64 + 2 * span) * E * (1 + f["entropy"])).all()
    assert (num(entropy)[k:] == MARK).all() and (best.cpu().numpy()[k:] == -7).all() and bool((state[k:] == 0).all())
    assert num(tau2)[0] == np.sort(num(entropy)[:k])[int(np.ceil(0.76 * k)) - 1]

"""The slow model with its hidden layers in 4 bits (SF_MX4): the same bits as the staged calls give, an exact network, and the
model inside the composite call and the streaming table."""
import dataclasses

import numpy as np
import pytest

import flowgen
import oracle
import packed_rows as pr
from workload import make_workload

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2402_03694_b200 import build, binding as sf, harness as hz
    build.build()
    ctx = sf.sf_ctx_create(0, 0)
    yield sf, hz, ctx
    sf.sf_ctx_poll(ctx, raise_on_error=False)
    sf.sf_ctx_destroy(ctx)


def infer(sf, ctx, slow, rows, count, C):
    cap = rows.shape[0]
    logits, label = torch.full((cap, C), 7.0, device="cuda"), torch.full((cap,), 9, dtype=torch.uint8, device="cuda")
    sf.sf_slow_infer(ctx, slow, rows, torch.tensor([count], dtype=torch.int32, device="cuda"), cap, logits, label)
    torch.cuda.synchronize()
    return logits, label


@pytest.mark.parametrize("dims,cap,count", [((1024, 256, 4), 300, 300), ((2048, 1024, 1024, 1024, 8), 500, 10), ((2048, 1024, 1024, 1024, 8), 70000, 61234),
                                            ((64, 64, 2), 1, 1), ((128, 192, 320, 16), 1000, 0), ((1024, 192, 5), 40, 17), ((1024, 512, 512, 2), 30000, 29999),
                                            ((512, 256, 4), 20011, 20011), ((256, 320, 16), 25000, 24001), ((256, 704, 5), 19000, 300), ((128, 1024, 3), 40000, 40000)])
def test_same_bits_as_the_staged_calls(env, dims, cap, count):
    sf, hz, ctx = env
    m = flowgen.gen_mlp(7, dims)
    slow = sf.sf_mlp_create(ctx, sf.SF_MX4, m["dims"], m["W"], m["b"])
    g = torch.Generator(device="cuda")
    g.manual_seed(cap)
    rows = torch.rand(cap, dims[0], device="cuda", generator=g).to(torch.bfloat16)
    logits, label = infer(sf, ctx, slow, rows, count, dims[-1])
    assert (logits[count:] == 7).all() and (label[count:] == 9).all()
    n = torch.tensor([count], dtype=torch.int32, device="cuda")
    def packed(rows_, K):
        d, s = sf.sf_mx4_sizes(rows_, K)
        return torch.zeros(rows_, d // rows_, dtype=torch.uint8, device="cuda"), torch.zeros(s, dtype=torch.uint8, device="cuda")
    a, sa = packed(cap, dims[0])
    sf.sf_mx4_quantise(ctx, rows, a, sa, n_rows_dev=n)
    L = len(dims) - 2
    for l in range(L):
        N, K = dims[l + 1], dims[l]
        w, sw = packed(N, K)
        sf.sf_mx4_quantise(ctx, torch.from_numpy(m["W"][l]).cuda(), w, sw)
        b = torch.from_numpy(m["b"][l]).cuda()
        if l + 1 < L:
            o, so = packed(cap, N)
            sf.sf_mx4_matmul(ctx, a, sa, w, sw, K, o, bias=b, relu=True, n_rows_dev=n, out_scales=so, N=N)
            a, sa = o, so
        else:
            h = torch.zeros(cap, N, dtype=torch.bfloat16, device="cuda")
            sf.sf_mx4_matmul(ctx, a, sa, w, sw, K, h, bias=b, relu=True, n_rows_dev=n)
    # the head: products of bf16 values, each sum off by at most K * 2^-23 of the sum of magnitudes
    w = torch.from_numpy(m["W"][L]).to(torch.bfloat16).double()
    b = torch.from_numpy(m["b"][L]).double()
    h = h[:count].double().cpu()
    want = h @ w.T + b
    slack = (dims[-2] + 2) * 2.0 ** -23 * (h @ w.abs().T + b.abs())
    got = logits[:count].double().cpu()
    assert ((got - want).abs() <= slack).all()
    if count:
        assert torch.equal(label[:count].cpu().long(), logits[:count].cpu().argmax(-1))
    sf.sf_ctx_poll(ctx)
    sf.sf_slow_destroy(slow)


def test_a_network_of_permutations_is_exact(env):
    """Rows of 4-bit values, every hidden layer a signed permutation, a head of small integers: nothing is ever rounded."""
    sf, hz, ctx = env
    rng = np.random.default_rng(3)
    D, C, n = 256, 5, 700
    W = []
    for _ in range(3):
        p = np.zeros((D, D), np.float32)
        p[np.arange(D), rng.permutation(D)] = rng.choice([-1, 1, 1], D)
        W.append(p)
    W.append(rng.integers(-3, 4, (C, D)).astype(np.float32))
    b = [np.zeros(D, np.float32)] * 3 + [rng.integers(-5, 6, C).astype(np.float32)]
    x = rng.choice([0, .5, 1, 1.5, 2, 3, 4, 6], (n, D))
    x[:, rng.integers(0, D, 40)] = 6.0                 # any 32 values that hold a 4 or a 6 keep scale 1
    h = x.copy()
    for w in W[:3]:
        h = np.maximum(h @ w.T, 0)
        top = h.reshape(n, -1, 32).max(-1)
        assert (pr.rounded(h) == h).all() and top.min() >= 0
    slow = sf.sf_mlp_create(ctx, sf.SF_MX4, (D, D, D, D, C), W, b)
    logits, label = infer(sf, ctx, slow, torch.from_numpy(x).to(torch.bfloat16).cuda(), n, C)
    want = h @ W[3].T + b[3]
    assert np.array_equal(logits.cpu().numpy().astype(float), want)
    assert np.array_equal(label.cpu().numpy(), want.argmax(-1))
    sf.sf_slow_destroy(slow)


def test_creation_refuses_what_the_kernels_do_not_take(env):
    sf, hz, ctx = env
    for dims in ((64, 4), (100, 64, 4), (64, 100, 4), (64, 64, 17)):
        m = flowgen.gen_mlp(1, dims)
        with pytest.raises(sf.SfError) as e:
            sf.sf_mlp_create(ctx, sf.SF_MX4, m["dims"], m["W"], m["b"])
        assert e.value.status == sf.SF_ERR_UNSUPPORTED
    with pytest.raises(sf.SfError) as e:
        m = flowgen.gen_mlp(1, (64, 64, 4))
        sf.sf_mlp_create(ctx, sf.SF_F16, m["dims"], m["W"], m["b"])
    assert e.value.status == sf.SF_ERR_ARG


def test_inside_the_composite_call(env):
    """sf_serve_batch with a 4-bit slow model: the routing of the bf16 one, and the slow answers of sf_slow_infer on the same rows."""
    sf, hz, ctx = env
    n = 3000
    cfg = dataclasses.replace(flowgen.get_config(2), n=n, slow_dtype="mx4")
    wl = make_workload(cfg, n=n)
    ref = oracle.serve_batch(dataclasses.replace(cfg, slow_dtype="bf16"), wl["fast"], wl["wide"], wl["forest"], wl["slow"], wl["tau"], threads=8)
    forest, slow = hz.make_forest(ctx, wl["forest"]), hz.make_slow(ctx, cfg, wl["slow"])
    fast_d, wide_d = hz.upload_packets(wl["fast"], with_hdr=False), hz.upload_packets(wl["wide"])
    rcfg = hz.route_cfg_for(cfg, hz.dev(wl["tau"]), n)
    label, stage = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    n_esc = torch.zeros(1, dtype=torch.int32, device="cuda")
    sf.sf_serve_batch(ctx, forest, slow, fast_d["struct"], cfg.N, cfg.F, wide_d["struct"], rcfg, label, stage, n_esc)
    torch.cuda.synchronize()
    sf.sf_ctx_poll(ctx)
    k = int(n_esc[0])
    assert k == ref["n_esc"] and np.array_equal(stage.cpu().numpy(), ref["stage"])
    p = sf.sf_serve_batch_intermediates(ctx)
    logits = hz.ptr_tensor(p["logits"], (k, 8), torch.float32)
    rows = hz.ptr_tensor(p["rows"], (n, cfg.D), torch.bfloat16)
    again, lab = infer(sf, ctx, slow, rows, k, 8)
    assert torch.equal(logits, again[:k])
    fast = ref["stage"] == 1
    got = label.cpu().numpy()
    # the host entry point works in pieces of the assigned rows: the same answers
    fp, wp = hz.pinned_packets(wl["fast"], with_hdr=False), hz.pinned_packets(wl["wide"])
    hl, hs, he = np.zeros(n, np.uint8), np.zeros(n, np.uint8), np.zeros(1, np.uint32)
    hcfg = sf.make_route_cfg(sf.SF_LC_GT, wl["tau"], sf.SF_MLP16, sf.SF_BF16, cfg.P, n)
    sf.sf_serve_batch_host(ctx, forest, slow, fp["struct"], cfg.N, cfg.F, wp["struct"], hcfg, hl, hs, he)
    assert int(he[0]) == k and np.array_equal(hl, got) and np.array_equal(hs, ref["stage"])
    assert np.array_equal(got[fast], ref["label_final"][fast]) and np.array_equal(got[~fast], lab[:k].cpu().numpy())
    sf.sf_slow_destroy(slow)
    sf.sf_forest_destroy(forest)


def test_inside_the_streaming_table(env):
    """One flow of 64 packets after the other: its record holds the label of sf_slow_infer on its wide row."""
    sf, hz, ctx = env
    F, C, P, flows = 24, 4, 64, 60
    w = flowgen.gen_packets(5, 4096, 8, 0)
    feat = oracle.extract_features(w, 8, F, threads=4)
    forest = flowgen.gen_forest(5, "rf", 16, 8, F, C, feat)
    m = flowgen.gen_mlp(5, (1024, 256, 4))
    pk = flowgen.gen_packets(6, flows, P, 13)
    tau = np.full(C, -1.0, np.float32)                   # every flow goes to the slow model
    dirs = ((pk["dir_bits"][:, np.arange(P) // 32] >> (np.arange(P) % 32)) & 1).astype(np.uint8)
    slow = sf.sf_mlp_create(ctx, sf.SF_MX4, m["dims"], m["W"], m["b"])
    table = sf.sf_table_create(ctx, 10, 8, P, flows)
    fh = hz.make_forest(ctx, forest)
    rcfg = sf.make_route_cfg(sf.SF_LC_GT, hz.dev(tau), sf.SF_MLP16, sf.SF_BF16, P, 0, P_real=P)
    src = np.repeat(np.arange(1, flows + 1, dtype=np.uint32), P)
    d = {"src": src, "dst": src + 7, "sport": np.full(src.size, 9, np.uint16), "dport": np.full(src.size, 80, np.uint16),
         "proto": np.full(src.size, 6, np.uint8), "dir": dirs.reshape(-1), "size": pk["size"].reshape(-1), "iat_us": pk["iat_us"].reshape(-1),
         "hdr": pk["hdr"].reshape(-1, 13)}
    t = {k: hz.dev(v) for k, v in d.items()}
    res = torch.zeros(8, dtype=torch.int32, device="cuda")
    sf.sf_table_ingest(ctx, table, sf.make_pkt_batch(t["src"], t["dst"], t["sport"], t["dport"], t["proto"], t["dir"], t["size"], t["iat_us"], t["hdr"]),
                       fh, F, slow, rcfg, res)
    torch.cuda.synchronize()
    sf.sf_ctx_poll(ctx)
    assert int(res[4]) == flows
    keys = np.zeros(flows, sf.KEY_DTYPE)
    keys["src"], keys["dst"], keys["sport"], keys["dport"], keys["proto"] = np.arange(1, flows + 1), np.arange(1, flows + 1) + 7, 9, 80, 6
    out = torch.zeros((flows, 12), dtype=torch.uint8, device="cuda")
    sf.sf_table_lookup(ctx, table, torch.from_numpy(keys.view(np.uint8).reshape(flows, 16).copy()).cuda(), flows, out)
    got = out.cpu().numpy().reshape(-1).view(sf.FLOW_RESULT_DTYPE)
    rows = oracle.wide_rows(0, np.arange(flows, dtype=np.uint32), pk, P, True)
    _, want = infer(sf, ctx, slow, torch.from_numpy(rows).to(torch.bfloat16).cuda(), flows, 4)
    assert (got["stage"] == 3).all() and np.array_equal(got["label_slow"], want.cpu().numpy())
    sf.sf_table_destroy(table)
    sf.sf_slow_destroy(slow)
    sf.sf_forest_destroy(fh)


def test_inside_the_three_tier_cascade(env):
    """sf_serve_batch3 with a 4-bit slow model: stages, ids and the faster answers of the cascade, the slow answers of sf_slow_infer."""
    sf, hz, ctx = env
    n = 5000
    cfg = dataclasses.replace(flowgen.get_config(2), n=n, slow_dtype="mx4")
    wl = make_workload(cfg, n=n)
    feat = oracle.extract_features(wl["fast"], cfg.N, cfg.F, threads=8)
    fastest = flowgen.gen_forest(4242, "rf", 1, 7, cfg.F, cfg.C, feat)
    rng = np.random.default_rng(2)
    tau1 = rng.uniform(0.2, 0.7, cfg.C).astype(np.float32)
    tau2 = (wl["tau"] + rng.uniform(-0.05, 0.05, cfg.C)).astype(np.float32)
    ref = oracle.serve_batch3(dataclasses.replace(cfg, slow_dtype="bf16"), wl["fast"], wl["wide"], fastest, wl["forest"], wl["slow"], tau1, tau2, threads=8)
    h1, h2, slow = hz.make_forest(ctx, fastest), hz.make_forest(ctx, wl["forest"]), hz.make_slow(ctx, cfg, wl["slow"])
    fast_d, wide_d = hz.upload_packets(wl["fast"], with_hdr=False), hz.upload_packets(wl["wide"])
    cfg1, cfg2 = hz.route_cfg_for(cfg, hz.dev(tau1), n), hz.route_cfg_for(cfg, hz.dev(tau2), n)
    label, stage = torch.full((n,), 255, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    cnt = torch.zeros(2, dtype=torch.uint32, device="cuda")
    sf.sf_ctx_poll(ctx, reset=True)
    sf.sf_serve_batch3(ctx, h1, h2, slow, fast_d["struct"], cfg.N, cfg.F, wide_d["struct"], cfg1, cfg2, label, stage, cnt)
    torch.cuda.synchronize()
    c = sf.sf_ctx_poll(ctx, reset=True)
    k1, k2 = [int(x) for x in cnt.cpu().numpy()]
    assert (k1, k2) == (len(ref["ids1"]), len(ref["ids2"])) and 0 < k2 < k1 < n and c.n_slow_done == k2
    st, lab = stage.cpu().numpy(), label.cpu().numpy()
    assert np.array_equal(st, ref["stage"]) and np.array_equal(lab[st < 3], ref["label_final"][st < 3])
    p = sf.sf_serve_batch_intermediates(ctx)
    assert np.array_equal(hz.ptr_tensor(p["esc_ids"], (k2,), torch.uint32).cpu().numpy(), ref["ids2"])
    logits = hz.ptr_tensor(p["logits"], (k2, 8), torch.float32).clone()
    rows = torch.zeros(n, cfg.D, dtype=torch.bfloat16, device="cuda")
    rows[:k2] = hz.ptr_tensor(p["rows"], (k2, cfg.D), torch.bfloat16)
    assert np.array_equal(rows[:k2].float().cpu().numpy(), ref["rows"])
    again, lab_slow = infer(sf, ctx, slow, rows, k2, 8)
    assert torch.equal(logits, again[:k2])
    assert np.array_equal(lab[ref["ids2"]], lab_slow[:k2].cpu().numpy())
    sf.sf_slow_destroy(slow)
    sf.sf_forest_destroy(h2)
    sf.sf_forest_destroy(h1)

"""Rows in 4 bits: packing, unpacking and products against the format's definition in doubles.

Packing is exact arithmetic with one rounding that both sides take alike: bit equality.  A product is a sum of K exact products:
K additions that are each off by at most 2^-23 of the running sum of magnitudes (a truncated fp32 addition), so by at most
K * 2^-23 * sum |a w|, plus the bias addition, plus half a step of the output type."""
import numpy as np
import pytest

import packed_rows as pr

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF_STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


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


def values_for(rng, n, K, kind):
    """Blocks of all magnitudes the type has: ordinary, ties, zeros, the smallest and the largest values, negative zeros."""
    x = rng.normal(size=(n, K)) * 10.0 ** rng.uniform(-4, 4 if kind == "fp16" else 8, size=(n, 1))
    x[rng.random((n, K)) < 0.1] = 0.0
    x[rng.random((n, K)) < 0.05] = -0.0
    if n > 1:
        x[1] = rng.choice([0, .25, .5, .75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, -2.5, -5], size=K) * 2.0 ** rng.integers(-3, 4)
    if n > 2:
        x[2, ::2], x[2, 1::2] = 0.0, 2.0 ** -24 if kind == "fp16" else 2.0 ** -133
        x[2, : K // 2] = 0.0
    if n > 3:
        x[3] = np.where(rng.random(K) < 0.5, 1, -1) * float(torch.finfo(TYPES[kind]).max)
    t = torch.from_numpy(x).to(TYPES[kind])
    return t, t.double().numpy()


def quantise(sf, ctx, x, **kw):
    n, K = x.shape
    m = n if kw.get("row_ids") is None else kw["row_ids"].numel()
    db, sb = sf.sf_mx4_sizes(m, K)
    data = torch.full((m, db // max(m, 1)), 0xAA, dtype=torch.uint8, device="cuda")
    scales = torch.full((sb,), 0x55, dtype=torch.uint8, device="cuda")
    sf.sf_mx4_quantise(ctx, x, data, scales, **kw)
    torch.cuda.synchronize()
    return data, scales


def check_packed(data, scales, x64, rows=None):
    n, K = x64.shape
    code, byte = pr.quantise(x64)
    want = code[:, 0::2] | (code[:, 1::2] << 4)
    assert np.array_equal(data.cpu().numpy()[:n], want)
    full = np.full((n, -(-K // 128) * 4), 127, np.uint8)
    full[:, : byte.shape[1]] = byte
    got = scales.cpu().numpy()
    at = pr.scale_index(n, K)
    assert np.array_equal(got[at], full)
    rest = np.ones(got.size, bool)
    rest[at.reshape(-1)] = False
    assert (got[rest] == 0x55).all()                     # nothing else is written


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,K", [(1, 1), (1, 32), (3, 33), (129, 100), (130, 416), (257, 2048), (5, 4097), (300, 7), (2, 260), (40000, 2), (3001, 129), (500, 1066)])
def test_quantise_bit_exact(env, n, K, kind):
    sf, ctx = env
    x, x64 = values_for(np.random.default_rng(n * 31 + K), n, K, kind)
    data, scales = quantise(sf, ctx, x.cuda())
    check_packed(data, scales, x64)


@pytest.mark.parametrize("kind", list(TYPES))
def test_quantise_infinities_and_nans_stay_in_their_block(env, kind):
    sf, ctx = env
    x, x64 = values_for(np.random.default_rng(5), 6, 200, kind)
    for r, c, v in ((0, 0, np.inf), (4, 35, -np.inf), (4, 199, np.nan), (5, 64, np.nan)):
        x[r, c] = v
        x64[r, c] = v
    data, scales = quantise(sf, ctx, x.cuda())
    check_packed(data, scales, x64)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("ld,at", [(512, 0), (515, 0), (512, 1), (512, 8), (512, 3)])
def test_quantise_pitches_and_alignments(env, kind, ld, at):
    sf, ctx = env
    x, x64 = values_for(np.random.default_rng(ld + at), 70, 300, kind)
    base = torch.full((70, ld), 3.0, dtype=TYPES[kind], device="cuda")
    base[:, at:at + 300] = x.cuda()
    data, scales = quantise(sf, ctx, base[:, at:at + 300])
    check_packed(data, scales, x64)


def test_quantise_row_list_and_device_count(env):
    sf, ctx = env
    x, x64 = values_for(np.random.default_rng(8), 40, 96, "bf16")
    ids = np.random.default_rng(9).integers(0, 40, 200).astype(np.int32)
    ids[[3, 50, 199]] = -1
    ids[[4, 60]] = 40                                    # outside: a row of zeros as well
    want = np.where(((ids >= 0) & (ids < 40))[:, None], x64[np.clip(ids, 0, 39)], 0.0)
    data, scales = quantise(sf, ctx, x.cuda(), row_ids=dev(ids))
    check_packed(data, scales, want)
    for count in (0, 1, 131, 200):
        data, scales = quantise(sf, ctx, x.cuda(), row_ids=dev(ids), n_rows_dev=dev(np.array([count], np.int32)))
        check_packed(data, scales, want[:count])
        assert (data.cpu().numpy()[count:] == 0xAA).all()
    sf.sf_ctx_poll(ctx, reset=True)
    data, scales = quantise(sf, ctx, x.cuda(), n_rows_dev=dev(np.array([41], np.int32)))
    check_packed(data, scales, x64)
    with pytest.raises(sf.SfError) as e:
        sf.sf_ctx_poll(ctx, reset=True)
    assert e.value.status == sf.SF_ERR_CAPACITY
    quantise(sf, ctx, x.cuda()[:0])                      # no rows: nothing to do


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,K", [(1, 1), (3, 33), (129, 100), (257, 2048), (4, 4097)])
def test_unpack(env, n, K, kind):
    sf, ctx = env
    rng = np.random.default_rng(n + K)
    code = rng.integers(0, 16, (n, -(-K // 32) * 32)).astype(np.uint8)
    byte = rng.integers(0, 253, (n, code.shape[1] // 32)).astype(np.uint8)
    byte[rng.random(byte.shape) < 0.1] = 255
    if kind == "fp16":
        byte = np.where(byte == 255, 255, 100 + byte % 45).astype(np.uint8)
    scales = np.full(sf.sf_mx4_sizes(n, K)[1], 255, np.uint8)
    scales[pr.scale_index(n, K)[:, : byte.shape[1]]] = byte
    want = torch.from_numpy(pr.values(code, byte, K)).to(TYPES[kind])
    data = dev(code[:, 0::2] | (code[:, 1::2] << 4))
    for ld, at in ((K, 0), (K + 5, 2), (K + 16 - K % 8, 8)):
        out = torch.full((n, ld + at), 7.0, dtype=TYPES[kind], device="cuda")
        sf.sf_mx4_unpack(ctx, data, dev(scales), out[:, at:at + K])
        got = out.cpu()
        assert torch.equal(torch.nan_to_num(got[:, at:at + K], nan=1e4), torch.nan_to_num(want, nan=1e4))
        assert (got[:, :at] == 7).all() and (got[:, at + K:] == 7).all()
    out = torch.full((n, K), 7.0, dtype=TYPES[kind], device="cuda")
    sf.sf_mx4_unpack(ctx, data, dev(scales), out, n_rows_dev=dev(np.array([n - 1], np.int32)))
    assert (out[n - 1:] == 7).all()
    assert torch.equal(torch.nan_to_num(out[: n - 1].cpu(), nan=1e4), torch.nan_to_num(want[: n - 1], nan=1e4))


def test_rows_beyond_32_bits_of_elements(env):
    """70,000 rows 65,536 elements apart: offsets pass 2^32."""
    sf, ctx = env
    big = torch.zeros(70000 * 65536 + 64, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((70000, 64), (65536, 1))
    x.copy_(torch.randn(70000, 64, device="cuda"))
    near = x.contiguous()
    a, b = quantise(sf, ctx, x), quantise(sf, ctx, near)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    out = big.as_strided((70000, 64), (65536, 1))
    out.zero_()
    sf.sf_mx4_unpack(ctx, a[0], a[1], out)
    want = torch.empty_like(near)
    sf.sf_mx4_unpack(ctx, a[0], a[1], want)
    assert torch.equal(out.contiguous(), want)


# ---- products ---------------------------------------------------------------------------------------------------
def operands(rng, n, N, K):
    a, w = rng.normal(size=(n, K)), rng.normal(size=(N, K)) / np.sqrt(K)
    return a, w, pr.rounded(a), pr.rounded(w)


def check_product(got, a, w, bias, relu, kind):
    K = a.shape[1]
    exact = a @ w.T + (0 if bias is None else bias)
    slack = (K + 2) * 2.0 ** -23 * (np.abs(a) @ np.abs(w).T + (0 if bias is None else np.abs(bias)))
    if relu:
        exact = np.maximum(exact, 0)
    got = got.double().cpu().numpy()
    tol = slack + HALF_STEP[kind] * (np.abs(exact) + slack) + (2.0 ** -25 if kind == "fp16" else 0)
    bad = np.abs(got - exact) > tol
    assert not bad.any(), (np.abs(got - exact).max(), int(bad.sum()), np.argwhere(bad)[:5])


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,K,N", [(1, 32, 1), (1, 1, 3), (10, 1024, 1024), (713, 416, 200), (128, 100, 64), (129, 33, 65), (257, 2080, 130),
                                   (1, 8192, 24), (300, 256, 256), (17, 160, 1000), (1000, 512, 512), (40, 288, 384)])
def test_product(env, n, K, N, kind):
    sf, ctx = env
    rng = np.random.default_rng(n + 7 * K + 13 * N)
    a, w, ra, rw = operands(rng, n, N, K)
    pa, pw = [dev(v) for v in pr.pack(a)], [dev(v) for v in pr.pack(w)]
    bias = rng.normal(size=N).astype(np.float32)
    for b, relu in ((bias, True), (None, False)):
        out = torch.full((n, N), 7.0, dtype=TYPES[kind], device="cuda")
        sf.sf_mx4_matmul(ctx, pa[0], pa[1], pw[0], pw[1], K, out, bias=None if b is None else dev(b), relu=relu)
        check_product(out, ra, rw, b, relu, kind)
    wide = torch.full((n, N + 11), 7.0, dtype=TYPES[kind], device="cuda")
    sf.sf_mx4_matmul(ctx, pa[0], pa[1], pw[0], pw[1], K, wide[:, 3:3 + N])
    assert torch.equal(wide[:, 3:3 + N], out) and (wide[:, :3] == 7).all() and (wide[:, 3 + N:] == 7).all()
    sf.sf_ctx_poll(ctx)


@pytest.mark.parametrize("n,K,N", [(5, 64, 9), (300, 1024, 320), (1000, 96, 128)])
def test_product_of_small_integers_is_exact(env, n, K, N):
    """Values 0, +-1, 2, 3, 4, 6 with scale 1: every partial sum is an integer below 2^24."""
    sf, ctx = env
    rng = np.random.default_rng(K)
    pick = np.array([0, 1, -1, 2, -2, 3, 4, -6, 6])
    a, w = rng.choice(pick, (n, K)).astype(float), rng.choice(pick, (N, K)).astype(float)
    a[:, ::32], w[:, ::32] = 6, -6
    pa, pw = [dev(v) for v in pr.pack(a)], [dev(v) for v in pr.pack(w)]
    out = torch.zeros(n, N, device="cuda")
    sf.sf_mx4_matmul(ctx, pa[0], pa[1], pw[0], pw[1], K, out)
    assert np.array_equal(out.cpu().numpy().astype(float), a @ w.T)


def test_product_scales_of_all_sizes(env):
    """Scales from 2^-60 to 2^60 on both sides, every (row, block) with one of its own: a misplaced scale byte cannot hide."""
    sf, ctx = env
    rng = np.random.default_rng(3)
    n, N, K = 200, 136, 640
    a = rng.normal(size=(n, K)) * np.repeat(2.0 ** rng.integers(-30, 30, (n, K // 32)), 32, axis=1)
    w = rng.normal(size=(N, K)) * np.repeat(2.0 ** rng.integers(-30, 30, (N, K // 32)), 32, axis=1)
    pa, pw = [dev(v) for v in pr.pack(a)], [dev(v) for v in pr.pack(w)]
    out = torch.zeros(n, N, device="cuda")
    sf.sf_mx4_matmul(ctx, pa[0], pa[1], pw[0], pw[1], K, out)
    check_product(out, pr.rounded(a), pr.rounded(w), None, False, "fp32")


def test_product_count_and_rows_beyond_it(env):
    sf, ctx = env
    rng = np.random.default_rng(4)
    n, N, K = 300, 72, 320
    a, w, ra, rw = operands(rng, n, N, K)
    pa, pw = [dev(v) for v in pr.pack(a)], [dev(v) for v in pr.pack(w)]
    for count in (0, 1, 128, 129, 299, 300):
        pa[0][count:] = 0x77                             # rows beyond the count hold anything, their scales are NaN
        sc = pa[1].cpu().numpy().copy()
        sc[pr.scale_index(n, K)[count:]] = 255
        out = torch.full((n, N), 7.0, device="cuda")
        sf.sf_mx4_matmul(ctx, pa[0], dev(sc), pw[0], pw[1], K, out, n_rows_dev=dev(np.array([count], np.int32)))
        check_product(out[:count], ra[:count], rw, None, False, "fp32")
        assert (out[count:] == 7).all()
        pa[0].copy_(dev(pr.pack(a)[0]))
    sf.sf_ctx_poll(ctx, reset=True)
    sf.sf_mx4_matmul(ctx, pa[0], pa[1], pw[0], pw[1], K, out, n_rows_dev=dev(np.array([301], np.int32)))
    check_product(out, ra, rw, None, False, "fp32")
    with pytest.raises(sf.SfError) as e:
        sf.sf_ctx_poll(ctx, reset=True)
    assert e.value.status == sf.SF_ERR_CAPACITY
    sf.sf_mx4_matmul(ctx, pa[0], pa[1], pw[0], pw[1], K, out[:0])


def test_product_nan_blocks_stay_in_their_rows_and_columns(env):
    sf, ctx = env
    rng = np.random.default_rng(6)
    n, N, K = 140, 70, 200
    a, w, _, _ = operands(rng, n, N, K)
    a[5, 40], w[3, 199] = np.nan, np.inf
    pa, pw = [dev(v) for v in pr.pack(a)], [dev(v) for v in pr.pack(w)]
    for relu in (False, True):
        out = torch.zeros(n, N, device="cuda")
        sf.sf_mx4_matmul(ctx, pa[0], pa[1], pw[0], pw[1], K, out, relu=relu)
        bad = np.isnan(out.cpu().numpy())
        want = np.zeros((n, N), bool)
        want[5], want[:, 3] = True, True
        assert np.array_equal(bad, want)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("counts,K,N", [([1], 64, 8), ([200, 0, 1, 129, 0, 383], 416, 200), ([0, 0, 0], 128, 64), ([5] * 40, 96, 33), ([1000, 30, 257], 1024, 512),
                                        ([3] * 300, 64, 70), ([4000, 700, 9000, 300], 2304, 300)])
def test_product_by_expert(env, counts, K, N, kind):
    sf, ctx = env
    rng = np.random.default_rng(len(counts) + K)
    E = len(counts)
    offsets = np.concatenate([[0], np.cumsum([-(-c // 128) * 128 for c in counts])]).astype(np.int32)
    cap = int(offsets[-1]) + 77                          # rows behind the last expert
    a, w, ra, rw = operands(rng, cap, E * N, K)
    pa = [dev(v) for v in pr.pack(a)]
    packed = [pr.pack(w[e * N:(e + 1) * N]) for e in range(E)]
    wd, ws = dev(np.stack([p[0] for p in packed])), dev(np.stack([p[1] for p in packed]))
    bias = rng.normal(size=(E, N)).astype(np.float32)
    out = torch.full((cap, N), 7.0, dtype=TYPES[kind], device="cuda")
    sf.sf_mx4_matmul_experts(ctx, pa[0], pa[1], wd, ws, K, dev(offsets), out, bias=dev(bias), relu=True)
    for e in range(E):
        lo, hi = offsets[e], offsets[e + 1]
        if hi > lo:
            check_product(out[lo:hi], ra[lo:hi], rw[e * N:(e + 1) * N], bias[e], True, kind)
    assert (out[int(offsets[-1]):] == 7).all()
    sf.sf_ctx_poll(ctx)


def test_product_by_expert_cut_at_the_capacity_and_misplaced(env):
    sf, ctx = env
    rng = np.random.default_rng(12)
    N, K = 40, 128
    a, w, ra, rw = operands(rng, 300, 2 * N, K)
    pa = [dev(v) for v in pr.pack(a)]
    packed = [pr.pack(w[e * N:(e + 1) * N]) for e in range(2)]
    wd, ws = dev(np.stack([p[0] for p in packed])), dev(np.stack([p[1] for p in packed]))
    sf.sf_ctx_poll(ctx, reset=True)
    out = torch.full((300, N), 7.0, device="cuda")
    sf.sf_mx4_matmul_experts(ctx, pa[0], pa[1], wd, ws, K, dev(np.array([0, 256, 512], np.int32)), out)     # the last expert ends behind the rows
    check_product(out[:256], ra[:256], rw[:N], None, False, "fp32")
    check_product(out[256:], ra[256:], rw[N:], None, False, "fp32")
    sf.sf_ctx_poll(ctx)
    out.fill_(7.0)
    sf.sf_mx4_matmul_experts(ctx, pa[0], pa[1], wd, ws, K, dev(np.array([0, 100, 300], np.int32)), out)     # the second does not start on a tile
    check_product(out[:100], ra[:100], rw[:N], None, False, "fp32")
    assert (out[100:] == 7).all()
    with pytest.raises(sf.SfError) as e:
        sf.sf_ctx_poll(ctx, reset=True)
    assert e.value.status == sf.SF_ERR_ARG


def test_refusals(env):
    sf, ctx = env
    x = torch.zeros(8, 64, device="cuda")
    data, scales = torch.zeros(8, 32, dtype=torch.uint8, device="cuda"), torch.zeros(512, dtype=torch.uint8, device="cuda")
    out = torch.zeros(8, 8, device="cuda")
    wd = torch.zeros(8, 32, dtype=torch.uint8, device="cuda")
    for call in (lambda: sf.sf_mx4_quantise(ctx, x, data[:7].contiguous(), scales),           # too short
                 lambda: sf.sf_mx4_quantise(ctx, x, data, scales[:511]),
                 lambda: sf.sf_mx4_quantise(ctx, x.int(), data, scales),                       # a type it does not know
                 lambda: sf.sf_mx4_quantise(ctx, x.t(), data, scales),                         # rows that are not contiguous
                 lambda: sf.sf_mx4_quantise(ctx, x[:1].expand(8, 64), data, scales),
                 lambda: sf.sf_mx4_quantise(ctx, x, data.view(-1)[1:], scales),
                 lambda: sf.sf_mx4_quantise(ctx, x, data, scales, n_rows_dev=torch.zeros(1, dtype=torch.int64, device="cuda")),
                 lambda: sf.sf_mx4_unpack(ctx, data, scales, x.double()),
                 lambda: sf.sf_mx4_matmul(ctx, data, scales, wd[:7].contiguous(), scales, 64, out),
                 lambda: sf.sf_mx4_matmul(ctx, data, scales, wd, scales, 65, out),
                 lambda: sf.sf_mx4_matmul(ctx, data, scales, wd, scales, 64, out, bias=torch.zeros(7, device="cuda")),
                 lambda: sf.sf_mx4_matmul_experts(ctx, data, scales, wd, scales, 64, torch.zeros(3, dtype=torch.int32, device="cuda"), out)):
        with pytest.raises(sf.SfError) as e:
            call()
        assert e.value.status == sf.SF_ERR_ARG
    big = torch.zeros(1024, dtype=torch.uint8, device="cuda")
    with pytest.raises(sf.SfError):
        sf.sf_mx4_quantise(ctx, x[:1], big[1:], scales)       # not on a 16-byte boundary
    with pytest.raises(sf.SfError):
        sf.sf_mx4_quantise(ctx, x[:1], big, big[8:])


def check_rows(got, a, w, bias, relu, kind):
    """check_product on the GPU's doubles, for outputs that are long on the CPU."""
    K = a.shape[1]
    exact = a @ w.T + bias
    slack = (K + 2) * 2.0 ** -23 * (a.abs() @ w.abs().T + bias.abs())
    exact = exact.clamp(min=0) if relu else exact
    off = (got.double() - exact).abs() - slack - HALF_STEP[kind] * (exact.abs() + slack)
    assert float(off.max()) <= 0, float(off.max())


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("n,K,N,E", [(20011, 1024, 1024, 1), (5000, 2048, 1000, 1), (40000, 224, 257, 1), (19000, 4096, 512, 1), (30000, 512, 512, 7), (3000, 640, 160, 1), (9000, 300, 721, 3), (1200, 900, 1453, 2)])
def test_product_of_many_rows(env, n, K, N, E, kind):
    """Sizes that fill the machine (CTA pairs): packed by the library, whose packing the tests above hold to the definition."""
    sf, ctx = env
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    rng = np.random.default_rng(n)
    counts = rng.multinomial(n - 128 * E, np.ones(E) / E) if E > 1 else [n]
    offsets = np.concatenate([[0], np.cumsum([-(-c // 128) * 128 for c in counts])]).astype(np.int32) if E > 1 else np.array([0, n], np.int32)
    x, w = torch.randn(n, K, device="cuda", generator=g), torch.randn(E * N, K, device="cuda", generator=g) / K ** 0.5
    def packed(v):
        d, s = sf.sf_mx4_sizes(*v.shape)
        d, s = torch.zeros(d, dtype=torch.uint8, device="cuda"), torch.full((s,), 255, dtype=torch.uint8, device="cuda")
        sf.sf_mx4_quantise(ctx, v, d, s)
        r = torch.zeros_like(v)
        sf.sf_mx4_unpack(ctx, d, s, r)
        return d, s, r.double()
    a, sa, ra = packed(x)
    ws = [packed(w[e * N:(e + 1) * N]) for e in range(E)]
    bias = torch.randn(E, N, device="cuda", generator=g)
    out = torch.full((n, N), 7.0, dtype=TYPES[kind], device="cuda")
    if E == 1:
        sf.sf_mx4_matmul(ctx, a, sa, ws[0][0], ws[0][1], K, out, bias=bias, relu=True)
    else:
        sf.sf_mx4_matmul_experts(ctx, a, sa, torch.cat([v[0] for v in ws]), torch.cat([v[1] for v in ws]), K, dev(offsets), out, bias=bias, relu=True)
    sf.sf_ctx_poll(ctx)
    for e in range(E):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        check_rows(out[lo:hi], ra[lo:hi], ws[e][2], bias[e].double(), True, kind)
    assert (out[int(offsets[-1]):] == 7).all()


def check_packed_product(sf, ctx, data, scales, rows, N, a, w, bias):
    """Packed outputs against the definition applied to the exact product.  A sum that is off by `slack` may fall on the other side of
    a border between two codes (or, for the largest of a block, of a power of two): a value has to be what some sum within
    slack of the exact one is rounded to, with the scale that the kernel chose, and that scale what some largest magnitude gives."""
    K = a.shape[1]
    exact = np.maximum(a @ w.T + bias, 0)
    slack = (K + 2) * 2.0 ** -23 * (np.abs(a) @ np.abs(w).T + np.abs(bias))
    Np, kt = -(-N // 32) * 32, -(-N // 128)
    byte = scales.cpu().numpy()[pr.scale_index(len(exact), N)]
    assert (byte[:, Np // 32:] == 127).all()
    lo, hi = np.zeros((len(exact), Np)), np.zeros((len(exact), Np))
    lo[:, :N], hi[:, :N] = np.maximum(exact - slack, 0), exact + slack
    e = byte[:, :Np // 32].astype(int) - 127
    e_of = lambda m: pr.quantise(m.reshape(-1, 1))[1].reshape(m.shape).astype(int) - 127  # noqa: E731
    assert (e >= e_of(lo.reshape(len(exact), -1, 32).max(-1))).all() and (e <= e_of(hi.reshape(len(exact), -1, 32).max(-1))).all()
    d = data.cpu().numpy()
    code = np.stack([d & 15, d >> 4], -1).reshape(len(exact), Np)
    assert (code < 8).all()
    unit = np.repeat(2.0 ** e, 32, axis=1)
    assert (code >= pr.nearest_code(np.minimum(lo / unit, 6))).all() and (code <= pr.nearest_code(np.minimum(hi / unit, 6))).all()


@pytest.mark.parametrize("n,K,N", [(1, 32, 1), (10, 1024, 1024), (300, 416, 200), (129, 96, 130), (70, 2304, 64), (257, 256, 33), (2000, 640, 1024), (6000, 512, 1000)])
def test_product_packed_again(env, n, K, N):
    sf, ctx = env
    rng = np.random.default_rng(n + K + N)
    a, w, ra, rw = operands(rng, n, N, K)
    pa, pw = [dev(v) for v in pr.pack(a)], [dev(v) for v in pr.pack(w)]
    bias = rng.normal(size=N).astype(np.float32)
    data = torch.full((n, -(-N // 32) * 16), 0xAA, dtype=torch.uint8, device="cuda")
    scales = torch.full((sf.sf_mx4_sizes(n, N)[1],), 0x55, dtype=torch.uint8, device="cuda")
    count = max(1, n - 3)
    sf.sf_mx4_matmul(ctx, pa[0], pa[1], pw[0], pw[1], K, data, bias=dev(bias), relu=True, n_rows_dev=dev(np.array([count], np.int32)), out_scales=scales, N=N)
    check_packed_product(sf, ctx, data[:count], scales, count, N, ra[:count], rw, bias)
    got = scales.cpu().numpy()
    rest = np.ones(got.size, bool)
    rest[pr.scale_index(count, N).reshape(-1)] = False
    assert (got[rest] == 0x55).all() and (data[count:] == 0xAA).all()
    sf.sf_ctx_poll(ctx)


def test_product_packed_again_by_expert_and_nan(env):
    sf, ctx = env
    rng = np.random.default_rng(31)
    E, N, K = 3, 96, 160
    offsets = np.array([0, 128, 128, 512], np.int32)
    a, w, _, rw = operands(rng, 512, E * N, K)
    a[200, 3] = np.nan
    ra = pr.rounded(a)
    pa = [dev(v) for v in pr.pack(a)]
    packed = [pr.pack(w[e * N:(e + 1) * N]) for e in range(E)]
    bias = rng.normal(size=(E, N)).astype(np.float32)
    data = torch.full((512, N // 2), 0xAA, dtype=torch.uint8, device="cuda")
    scales = torch.full((sf.sf_mx4_sizes(512, N)[1],), 0x55, dtype=torch.uint8, device="cuda")
    sf.sf_mx4_matmul_experts(ctx, pa[0], pa[1], dev(np.stack([p[0] for p in packed])), dev(np.stack([p[1] for p in packed])), K, dev(offsets), data,
                             bias=dev(bias), relu=True, out_scales=scales, N=N)
    s = scales.cpu().numpy()[pr.scale_index(512, N)]
    assert (s[200, :3] == 255).all() and (np.delete(s, 200, 0) != 255).all()
    for e, lo, hi in ((0, 0, 128), (2, 128, 256), (2, 256, 384), (2, 384, 512)):
        keep = [r for r in range(lo, hi) if r != 200]
        at = scales[lo * 4:hi * 4]                       # a 128-row block of one k tile is 512 bytes
        sub = at.clone()
        if lo <= 200 < hi:
            continue
        check_packed_product(sf, ctx, data[lo:hi], sub, hi - lo, N, ra[lo:hi], rw[e * N:(e + 1) * N], bias[e])
        assert len(keep) == hi - lo
    with pytest.raises(sf.SfError):
        sf.sf_mx4_matmul(ctx, pa[0], pa[1], dev(packed[0][0]), dev(packed[0][1]), K, data[:, :32].contiguous(), out_scales=scales, N=N)
    sf.sf_ctx_poll(ctx)


def test_captured_replayed_and_on_another_stream(env):
    sf, ctx = env
    rng = np.random.default_rng(14)
    n, N, K = 150, 96, 224
    a, w, _, rw = operands(rng, n, N, K)
    pw = [dev(v) for v in pr.pack(w)]
    x = torch.zeros(n, K, device="cuda")
    data, scales = torch.zeros(n, K // 2, dtype=torch.uint8, device="cuda"), torch.zeros(1024 * 2, dtype=torch.uint8, device="cuda")
    out = torch.zeros(n, N, device="cuda")

    def step(stream=None):
        sf.sf_mx4_quantise(ctx, x, data, scales, stream=stream)
        sf.sf_mx4_matmul(ctx, data, scales, pw[0], pw[1], K, out, stream=stream)
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for k in range(2):
        x.copy_(dev((a * (k + 1) + k).astype(np.float32)))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        check_product(out, pr.rounded(x.double().cpu().numpy()), rw, None, False, "fp32")
    s = torch.cuda.Stream()
    out.zero_()
    torch.cuda.synchronize()
    step(stream=s)
    s.synchronize()
    check_product(out, pr.rounded(x.double().cpu().numpy()), rw, None, False, "fp32")


def test_products_without_pairs_at_once_on_two_streams(env):
    """Products of single CTAs that store by TMA, with nothing between them on two streams, each followed by packing, whose blocks take
    over the shared memory that the last boxes were stored from: every pass gives the bits of the same calls alone."""
    sf, ctx = env
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    jobs = []
    for n, K, N, kind in ((20000, 256, 128, "bf16"), (20000, 200, 128, "fp32"), (700, 416, 200, "fp32"), (129, 64, 64, "fp32")):
        x, w, bias = torch.randn(n, K, device="cuda", generator=g), torch.randn(N, K, device="cuda", generator=g) / K ** 0.5, torch.randn(N, device="cuda", generator=g)
        def packed(v):
            d, s = sf.sf_mx4_sizes(*v.shape)
            return torch.zeros(d, dtype=torch.uint8, device="cuda"), torch.zeros(s, dtype=torch.uint8, device="cuda")
        a, b = packed(x), packed(w)
        sf.sf_mx4_quantise(ctx, x, *a)
        sf.sf_mx4_quantise(ctx, w, *b)
        outs, spare = [torch.zeros(n, N, dtype=TYPES[kind], device="cuda") for _ in range(6)], packed(x)

        def step(stream, x=x, a=a, b=b, K=K, bias=bias, outs=outs, spare=spare):
            for o in outs:
                sf.sf_mx4_matmul(ctx, *a, *b, K, o, bias=bias, relu=True, stream=stream)
                sf.sf_mx4_quantise(ctx, x[:, :x.shape[1] - 1], *spare, stream=stream)        # (rows on no 16-byte boundary: turned round in shared memory)
        step(torch.cuda.current_stream())
        ra, rw = torch.zeros_like(x), torch.zeros_like(w)
        sf.sf_mx4_unpack(ctx, *a, ra)
        sf.sf_mx4_unpack(ctx, *b, rw)
        torch.cuda.synchronize()
        for o in outs:
            check_rows(o, ra.double(), rw.double(), bias.double(), True, kind)
        jobs.append((step, outs, outs[0].clone()))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for _, outs, _ in jobs:
            for o in outs:
                o.zero_()
        torch.cuda.synchronize()
        for i, (step, _, _) in enumerate(jobs):
            step(streams[i % 2])
        torch.cuda.synchronize()
        for _, outs, want in jobs:
            for o in outs:
                assert torch.equal(o, want)
    sf.sf_ctx_poll(ctx)


@pytest.mark.parametrize("n,K,N", [(128, 160, 96), (300, 416, 200), (20011, 512, 512)])
def test_rows_beside_a_nan_row_are_packed_as_if_alone(env, n, K, N):
    """Packed outputs of the rows that share tiles (and scale words) with rows of NaN: the codes and scales of the definition, and the
    bits that they get without the NaN."""
    sf, ctx = env
    rng = np.random.default_rng(n + K)
    a, w, _, rw = operands(rng, n, N, K)
    bad = np.unique(rng.integers(0, n, 5))
    keep = np.setdiff1d(np.arange(n), bad)
    b = a.copy()
    b[bad, rng.integers(0, K, bad.size)] = np.nan
    pw, bias = [dev(v) for v in pr.pack(w)], rng.normal(size=N).astype(np.float32)
    got = []
    for x in (a, b):
        data = torch.full((n, -(-N // 32) * 16), 0xAA, dtype=torch.uint8, device="cuda")
        scales = torch.full((sf.sf_mx4_sizes(n, N)[1],), 0x55, dtype=torch.uint8, device="cuda")
        sf.sf_mx4_matmul(ctx, *[dev(v) for v in pr.pack(x)], *pw, K, data, bias=dev(bias), relu=True, out_scales=scales, N=N)
        got.append((data.cpu().numpy(), scales.cpu().numpy()[pr.scale_index(n, N)]))
    (data, scale), (data_nan, scale_nan) = got
    blocks = -(-N // 32)
    assert (scale_nan[bad, :blocks] == 255).all() and (scale_nan[:, blocks:] == 127).all()
    assert np.array_equal(data_nan[keep], data[keep]) and np.array_equal(scale_nan[keep], scale[keep])
    few = keep[:200]                                     # (rows of the first NaN's tile among them; laid out again as rows of their own)
    laid = np.full(sf.sf_mx4_sizes(few.size, N)[1], 0x55, np.uint8)
    laid[pr.scale_index(few.size, N)] = scale_nan[few]
    check_packed_product(sf, ctx, torch.from_numpy(data_nan[few]), torch.from_numpy(laid), few.size, N, pr.rounded(a[few]), rw, bias)
    sf.sf_ctx_poll(ctx)

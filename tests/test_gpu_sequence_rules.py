"""What the calls on sequences promise beyond their values: pools that are read and written by one call, small steps and gates."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import sequences as ref  # noqa: E402
from test_gpu_sequences import E, MARK, TYPES, env, lay_out, like, num, rows_in, scan_case  # noqa: E402, F401


# ---- one pool, read and written by a call ----------------------------------------------------------------------------------------------
# Sequences shorter than a state, as long as one, of one tile and of many (few sequences: tiles of 8 rows), and a batch that is walked by tiles of 128.
POOLS = [
    (4, True, 24, "fp32", [1, 2, 0, 3, 10, 130, 300, 7], True), (4, False, 33, "bf16", [1, 2, 0, 3, 4, 5, 8, 9, 40], True), (2, True, 8, "fp16", [0, 1, 2, 17], False),
    (3, True, 130, "fp32", [1, 0, 2, 3, 100], True), (8, True, 16, "bf16", [3, 6, 7, 8, 0, 15, 16, 29], True), (5, False, 7, "fp32", [1, 3, 4, 5, 33], False),
    (4, True, 64, "bf16", [129, 1, 260, 2] * 150, False), (1, True, 8, "fp32", [3, 1], True), (7, True, 12, "fp32", [1] * 5, True),
]


@pytest.mark.parametrize("W,silu,D,kind,lengths,slots", POOLS)
def test_convolution_gradients_of_states_in_one_pool(env, W, silu, D, kind, lengths, slots):  # noqa: F811
    """The gradient of the states before the call over that of the states after it: the same as with a pool for each."""
    sf, ctx = env
    rng = np.random.default_rng(W * 100 + D)
    q, first, R, slot = lay_out(sf, rng, lengths, False, slots)
    S, act = len(lengths), sf.SF_ACT_SILU if silu else sf.SF_ACT_NONE
    x, dy = rows_in(rng, R, D, kind), rows_in(rng, R, D, kind)
    w, b = torch.from_numpy(rng.standard_normal((D, W)).astype(np.float32)).cuda(), torch.from_numpy(rng.standard_normal(D).astype(np.float32)).cuda()
    pool, after = (torch.from_numpy(rng.standard_normal((S + 2, W - 1, D))).to(TYPES[kind]).cuda() for _ in range(2))
    work = torch.full((sf.sf_seq_conv_backward_workspace(S, max(lengths), D, W),), 255, dtype=torch.uint8, device="cuda")

    def grads(into, **only):
        o = {"dx_out": like(x), "dw_out": torch.full_like(w, MARK), "dbias_out": torch.full((D,), MARK, device="cuda")}
        if only:
            o = {}
        sf.sf_seq_conv_backward(ctx, q, x, w, dy, work, bias=b, act=act, state_in=pool, d_state=into if into is not None else after, d_state_in_out=into if into is not None else apart, **o)
        return o
    apart = after.clone()                                  # (slots that no sequence names are left as they were: the same in both)
    want = grads(None)
    one = after.clone()
    got = grads(one)
    for k in want:
        assert torch.equal(got[k], want[k]) and bool(torch.isfinite(got[k]).all()), k
    assert torch.equal(one, apart) and bool(torch.isfinite(one).all())
    named = sorted(i for i in slot if i >= 0)
    if W > 1:
        assert not torch.equal(one[named], after[named])
        other = [i for i in range(S + 2) if i not in named]
        assert torch.equal(one[other], after[other])
        alone = after.clone()                              # nothing asked for but the states' (with one tap they have no rows: that would be nothing at all)
        grads(alone, states=True)
        assert torch.equal(alone, apart)
    sf.sf_ctx_poll(ctx)


@pytest.mark.parametrize("lengths,D,kind", [([300], 24, "fp32"), ([260, 0, 131], 32, "bf16"), ([9, 3, 0, 17] * 60, 40, "fp32"), ([1, 0, 1, 1], 33, "fp16")])
def test_scan_gradients_of_states_in_one_pool(env, lengths, D, kind):  # noqa: F811
    """Sequences in parts and in one go."""
    sf, ctx = env
    N, S = 16, len(lengths)
    rng = np.random.default_rng(D)
    q, first, R, slot, t, pool, after = scan_case(sf, rng, D, N, 1, kind, lengths, False, True, 0, 0, True, True, True, True)
    rest = dict(D=t["D"], delta_bias=t["bias"], z=t["z"], softplus=True)
    rows = (t["u"], t["delta"], t["A"], t["B"], t["C"])
    work = torch.full((sf.sf_seq_scan_workspace(S, max(lengths), R, D, N, backward=True),), 255, dtype=torch.uint8, device="cuda")
    starts = torch.full((sf.sf_seq_scan_starts(S, R, D, N),), float("nan"), device="cuda")
    sf.sf_seq_scan(ctx, q, *rows, like(t["u"]), workspace=work, state_in=pool, starts_out=starts, **rest)
    out = []
    for one in (False, True):
        d = after.clone()
        du = like(t["u"])
        sf.sf_seq_scan_backward(ctx, q, *rows, t["dy"], starts, work, d_state=d if one else after, d_state_in_out=d, du_out=du, **rest)
        out.append((d, du))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1]) and bool(torch.isfinite(out[1][0]).all())
    sf.sf_ctx_poll(ctx)


# ---- steps and gates of large arguments ----------------------------------------------------------------------------------------------------
# exp(-|x|) is off by 4 e (two units in the last place), 1 + it by e, a reciprocal by 2 e, each product by e.  Sigmoid: 7 e; the slope of softplus, e^-|x| / (1 + e^-|x|): 8 e;
# softplus itself, 2 q (1 + q^2 / 3 + ..) with q = e / (2 + e): 8 e for q, 3 e for the series, 2 e for the rest, 16 e with room.  All relative, wherever the argument lies.
def within(got, want, tol):
    got = num(got)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:3], got[bad][:3], want[bad][:3], (np.abs(got - want) / tol)[bad].max())


@pytest.mark.parametrize("D", [64, 33, 6])                 # rows on 16-byte boundaries, and not
def test_small_steps_and_gates_keep_their_relative_accuracy(env, D):  # noqa: F811
    sf, ctx = env
    S, N = 120, 2
    x = torch.linspace(-85, 85, S * D, dtype=torch.float64).float().view(S, D).cuda()
    X, one, ones, A = num(x), torch.ones(S, D, device="cuda"), torch.ones(S, N, device="cuda"), -torch.ones(D, N, device="cuda")
    half = ones / N                                        # N states of delta u / N each: y = delta u
    q = sf.make_sequences(torch.arange(S + 1, dtype=torch.int32, device="cuda"), 1)
    starts = torch.zeros(sf.sf_seq_scan_starts(S, S, D, N), device="cuda")
    work = torch.zeros(sf.sf_seq_scan_workspace(S, 1, S, D, N, backward=True), dtype=torch.uint8, device="cuda")
    step, slope = ref.softplus(X), np.exp(-np.maximum(-X, 0)) / (1 + np.exp(-np.abs(X)))
    for kept in (None, starts):                            # the single step's kernel, the scan's
        y = torch.zeros_like(x)
        sf.sf_seq_scan(ctx, q, one, x, A, ones, half, y, softplus=True, starts_out=kept)
        within(y, step, 18 * E * step)
    du, dd = torch.zeros_like(x), torch.zeros_like(x)
    sf.sf_seq_scan_backward(ctx, q, one, x, A, ones, half, one, starts, work, softplus=True, du_out=du, d_delta_out=dd)
    within(du, step, 20 * E * step)
    within(dd, slope, 12 * E * slope)
    s = np.exp(-np.maximum(-X, 0)) / (1 + np.exp(-np.abs(X)))
    gate, d_gate, mag = X * s, s * (1 + X * (1 - s)), s * (1 + np.abs(X) * (1 - s))
    for kept in (None, starts):
        y = torch.zeros_like(x)
        sf.sf_seq_scan(ctx, q, one, one, A, ones, half, y, z=x, starts_out=kept)
        within(y, gate, 12 * E * np.abs(gate))
    dz = torch.zeros_like(x)
    sf.sf_seq_scan_backward(ctx, q, one, one, A, ones, half, one, starts, work, z=x, du_out=du, dz_out=dz)
    within(du, gate, 12 * E * np.abs(gate))
    # slope: 1 - s is off by 7 e s + e (1 - s); for large x it is a difference of equals, off by a step of 1, and times x
    within(dz, d_gate, 14 * E * mag + 10 * E * np.abs(X) * s)
    b = x.bfloat16()                                       # rows of 16 bits, states of 32
    B, state = num(b), torch.zeros(S, D, N, device="cuda")
    for kept in (None, starts):
        sf.sf_seq_scan(ctx, q, one.bfloat16(), b, A, ones.bfloat16(), half.bfloat16(), torch.zeros_like(b), softplus=True, state_out=state, starts_out=kept)
        within(state, np.repeat(ref.softplus(B)[:, :, None], N, 2), 18 * E * ref.softplus(B)[:, :, None])
        state.zero_()
    w = torch.ones(D, 1, device="cuda")
    long = sf.make_sequences(torch.tensor([0, S], dtype=torch.int32, device="cuda"), S)
    for seq in (q, long):                                  # single rows and whole sequences: with one tap the same
        y, dx = torch.zeros_like(x), torch.zeros_like(x)
        sf.sf_seq_conv(ctx, seq, x, w, y, act=sf.SF_ACT_SILU)
        within(y, gate, 10 * E * np.abs(gate))
        sf.sf_seq_conv_backward(ctx, seq, x, w, one, None, act=sf.SF_ACT_SILU, dx_out=dx)
        within(dx, d_gate, 14 * E * mag + 10 * E * np.abs(X) * s)
    sf.sf_ctx_poll(ctx)

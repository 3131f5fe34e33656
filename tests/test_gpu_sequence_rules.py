"""What the calls on sequences promise beyond their values: pools that are read and written by one call."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import test_gpu_sequences as base  # noqa: E402
from test_gpu_sequences import MARK, TYPES, env, lay_out, like, rows_in, scan_case  # noqa: E402, F401


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

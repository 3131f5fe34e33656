"""The statements in doubles that the GPU tests go by: their gradients against differences, and closed forms."""
import numpy as np
import pytest

import sequences as ref


def differences(f, x, d=1e-6):
    g = np.zeros(x.shape)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + d
        hi = f()
        x[i] = keep - d
        lo = f()
        x[i] = keep
        g[i] = (hi - lo) / (2 * d)
    return g


# a central difference is off by d^2 / 6 times the third derivative (values of order one: 1e-11) and 2^-53 / d of the sum (1e-10 times its terms)
CLOSE = dict(rtol=1e-6, atol=1e-7)


@pytest.mark.parametrize("W,silu,L", [(1, True, 3), (2, False, 1), (4, True, 2), (4, True, 6), (7, True, 4), (3, True, 0)])
def test_convolution_gradients(W, silu, L):
    rng = np.random.default_rng(W * 10 + L)
    D = 3
    x, w, b, s = rng.standard_normal((L, D)), rng.standard_normal((D, W)), rng.standard_normal(D), rng.standard_normal((W - 1, D))
    dy, ds = rng.standard_normal((L, D)), rng.standard_normal((W - 1, D))
    r = ref.conv(x, w, b, silu, s, dy, ds)

    def total():
        o = ref.conv(x, w, b, silu, s)
        return (o["y"] * dy).sum() + (o["state"] * ds).sum()
    for name, v in (("dx", x), ("dw", w), ("dbias", b), ("d_state_in", s)):
        np.testing.assert_allclose(r[name], differences(total, v), **CLOSE, err_msg=name)


@pytest.mark.parametrize("N,G,gate,sp,skip,L", [(3, 1, True, True, True, 5), (2, 2, False, False, True, 4), (4, 1, True, True, False, 1), (1, 4, False, True, False, 3), (2, 1, True, True, True, 0)])
def test_scan_gradients(N, G, gate, sp, skip, L):
    rng = np.random.default_rng(N * 10 + G)
    D = 4
    u, z = rng.standard_normal((L, D)), rng.standard_normal((L, D)) if gate else None
    delta = rng.standard_normal((L, D)) if sp else rng.uniform(0.1, 0.9, (L, D))
    A, B, C = -rng.uniform(0.2, 2, (D, N)), rng.standard_normal((L, G, N)), rng.standard_normal((L, G, N))
    Dk, bias = (rng.standard_normal(D) if skip else None), (rng.standard_normal(D) if sp else None)
    h0, dy, dh = rng.standard_normal((D, N)), rng.standard_normal((L, D)), rng.standard_normal((D, N))
    r = ref.scan(u, delta, A, B, C, Dk, bias, z, sp, h0, dy, dh)

    def total():
        o = ref.scan(u, delta, A, B, C, Dk, bias, z, sp, h0)
        return (o["y"] * dy).sum() + (o["state"] * dh).sum()
    for name, v in (("du", u), ("d_delta", delta), ("dA", A), ("dB", B), ("dC", C), ("dD", Dk), ("d_delta_bias", bias), ("dz", z), ("d_state_in", h0)):
        if v is not None:
            np.testing.assert_allclose(r[name], differences(total, v), **CLOSE, err_msg=name)


def test_scan_closed_form():
    """A step that keeps half: h = 1 - 2^-t with delta u B = 1/2."""
    L = 20
    one = np.ones((L, 1))
    r = ref.scan(one * 0.5 / np.log(2), one * np.log(2), -np.ones((1, 1)), one[:, None], one[:, None], None, None, None, False, np.zeros((1, 1)))
    np.testing.assert_allclose(r["y"][:, 0], 1 - 0.5 ** np.arange(1, L + 1), rtol=1e-12)


@pytest.mark.parametrize("V,scale", [(5, 1.0), (3, 0.5)])
def test_logprob_gradients(V, scale):
    rng = np.random.default_rng(V)
    n, k = 4, 2
    x = rng.standard_normal((n, V))
    x[1, 0] = -np.inf
    labels = np.array([0, 2, -1, 1])
    dl, de, dt = rng.standard_normal(n), rng.standard_normal(n), rng.standard_normal((n, k))
    f = ref.logprobs(x, scale, labels, k)
    want = ref.logprobs_gradient(x, scale, labels, f, dl, de, dt)

    def total():
        o = ref.logprobs(x, scale, labels, k)
        return (o["logprob"] * dl).sum() + (o["entropy"] * de).sum() + (o["top_logprobs"] * dt).sum()
    got = np.zeros((n, V))
    for r in range(n):
        for i in range(V):
            if np.isinf(x[r, i]):
                continue
            keep = x[r, i]
            x[r, i] = keep + 1e-6
            hi = total()
            x[r, i] = keep - 1e-6
            lo = total()
            x[r, i] = keep
            got[r, i] = (hi - lo) / 2e-6
    np.testing.assert_allclose(want, got, **CLOSE)
    assert want[1, 0] == 0


def test_logprob_closed_forms():
    f = ref.logprobs(np.array([[0.0, 0, 0, 0], [5, -np.inf, -np.inf, -np.inf], [-np.inf] * 4]), 1.0, np.array([3, 0, 1]), 2)
    np.testing.assert_allclose(f["entropy"], [np.log(4), 0, 0])
    np.testing.assert_allclose(f["logprob"][:2], [-np.log(4), 0])
    assert f["logprob"][2] == f["lse"][2] == -np.inf and f["top_ids"].tolist() == [[0, 1], [0, -1], [-1, -1]]

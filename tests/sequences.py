"""Direct statements in doubles of the operators on sequences of rows: one sequence at a time, row by row, with their gradients.

Every function takes `ab`: the identity, or np.abs to get the sum of the magnitudes of everything that is added up, which bounds what roundings can do."""
import numpy as np


def same(x):
    return x


def sigmoid(x):
    return 1.0 / (1.0 + np.exp(-x))


def softplus(x):
    return np.maximum(x, 0) + np.log1p(np.exp(-np.abs(x)))


def conv(x, w, bias, silu, state, dy=None, d_state=None, ab=same):
    """x [L][D], w [D][W], state [W - 1][D]; y and the state after, and with dy the gradients of x, w, bias and the state before."""
    L, D = x.shape
    W = w.shape[1]
    b = np.zeros(D) if bias is None else bias
    full = np.concatenate([state, x])
    pre = np.zeros((L, D)) + ab(b)
    real = np.zeros((L, D)) + b
    for t in range(L):
        for k in range(W):
            pre[t] += ab(w[:, k]) * ab(full[t + k])
            real[t] += w[:, k] * full[t + k]
    s = sigmoid(real)
    r = {"y": pre * s if silu else pre, "state": full[L:]}
    if dy is None:
        return r
    g = ab(dy) * (ab(s * (1 + real * (1 - s))) if silu else 1.0)
    d = np.zeros((L + W - 1, D))
    if d_state is not None:
        d[L:] += ab(d_state)
    dw = np.zeros((D, W))
    for t in range(L):
        for k in range(W):
            d[t + k] += ab(w[:, k]) * g[t]
            dw[:, k] += g[t] * ab(full[t + k])
    r.update(dx=d[W - 1:], d_state_in=d[:W - 1], dw=dw, dbias=g.sum(0))
    return r


def scan(u, delta, A, B, C, Dk, bias, z, sp, state, dy=None, d_state=None, ab=same):
    """u, delta, z [L][D], B, C [L][G][N], A [D][N], state [D][N]; y and the state after, and with dy the gradients of everything."""
    L, D = u.shape
    N, G = A.shape[1], B.shape[1]
    of = np.arange(D) // (D // G)
    raw = delta + (0 if bias is None else bias)
    step = softplus(raw) if sp else raw
    a = np.exp(step[:, :, None] * A)
    skip = np.zeros(D) if Dk is None else ab(Dk)
    gate = np.ones((L, D)) if z is None else ab(z * sigmoid(z))
    h, hs = ab(state), []
    y = np.zeros((L, D))
    for t in range(L):
        h = a[t] * h + (ab(step[t]) * ab(u[t]))[:, None] * ab(B[t])[of]
        hs.append(h)
        y[t] = (h * ab(C[t])[of]).sum(-1) + skip * ab(u[t])
    r = {"y": y * gate, "state": h}
    if dy is None:
        return r
    e = ab(dy) * gate
    du, dd, dB, dC, dA = np.zeros((L, D)), np.zeros((L, D)), np.zeros(B.shape), np.zeros(C.shape), np.zeros(A.shape)
    g = np.zeros((D, N)) if d_state is None else ab(d_state)
    for t in range(L - 1, -1, -1):
        g = g + e[t][:, None] * ab(C[t])[of]
        for i in range(G):
            dC[t, i] = (e[t][:, None] * hs[t])[of == i].sum(0)
            dB[t, i] = (g * (ab(step[t]) * ab(u[t]))[:, None])[of == i].sum(0)
        s1 = (g * ab(B[t])[of]).sum(-1)
        g = g * a[t]
        x = g * (hs[t - 1] if t else ab(state))
        du[t] = skip * e[t] + ab(step[t]) * s1
        dd[t] = ab(u[t]) * s1 + (x * ab(A)).sum(-1)
        dA += x * ab(step[t])[:, None]
    if sp:
        dd = dd * sigmoid(raw)
    r.update(du=du, d_delta=dd, dA=dA, dB=dB, dC=dC, d_state_in=g, dD=(e * ab(u)).sum(0), d_delta_bias=dd.sum(0))
    if z is not None:
        s = sigmoid(z)
        r["dz"] = ab(dy) * y * ab(s * (1 + z * (1 - s)))
    return r


def logprobs(x, scale, labels, k):
    """Row by row: log probability of the label, entropy, lse, the k best entries and their log probabilities; p."""
    n, V = x.shape
    lp, h, lse = np.zeros(n), np.zeros(n), np.zeros(n)
    ids, top, p = np.full((n, k), -1), np.full((n, k), -np.inf), np.zeros((n, V))
    for r in range(n):
        z = scale * x[r]
        real = [i for i in range(V) if x[r, i] > -np.inf]                     # False for NaN
        order = sorted(real, key=lambda i: (-x[r, i], i))[:k]
        bad = np.isnan(x[r]).any() or np.isposinf(x[r]).any()
        label = labels[r] if 0 <= labels[r] < V else None
        if bad:
            lse[r] = h[r] = np.nan
            p[r] = np.nan
        elif not real:
            lse[r] = -np.inf
        else:
            m = max(z[i] for i in real)
            s = sum(np.exp(z[i] - m) for i in real)
            lse[r] = m + np.log(s)
            for i in real:
                p[r, i] = np.exp(z[i] - m) / s
            h[r] = np.log(s) - sum(p[r, i] * (z[i] - m) for i in real)
        for j, i in enumerate(order):
            ids[r, j], top[r, j] = i, z[i] - lse[r]
        if label is not None:
            lp[r] = -np.inf if np.isneginf(x[r, label]) else z[label] - lse[r]
    return {"logprob": lp, "entropy": h, "lse": lse, "top_ids": ids, "top_logprobs": top, "p": p}


def logprobs_gradient(x, scale, labels, f, d_logprob, d_entropy, d_top):
    n, V = x.shape
    d = np.zeros((n, V))
    for r in range(n):
        pick = {}
        if d_logprob is not None and 0 <= labels[r] < V:
            pick[labels[r]] = pick.get(labels[r], 0) + d_logprob[r]
        total = sum(pick.values())
        if d_top is not None:
            for j, i in enumerate(f["top_ids"][r]):
                if i >= 0:
                    pick[i] = pick.get(i, 0) + d_top[r, j]
                    total += d_top[r, j]
        for i in range(V):
            if np.isneginf(x[r, i]):
                continue
            p = f["p"][r, i]
            d[r, i] = pick.get(i, 0) - p * total
            if d_entropy is not None and p > 0:
                d[r, i] -= d_entropy[r] * p * (np.log(p) + f["entropy"][r])
    return d * scale

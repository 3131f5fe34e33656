"""Cases that measure the operators of a slow model that reads a flow's packets one after the other, and of its answers: what
each takes in, its plain form, the framework's calls and the values in 64 bits.

  conv     short causal convolution over the rows of each sequence (one filter a channel), with the rows before the sequence
           taken from and kept in a state; with the gradients of rows, filters and bias
  scan     selective state space scan: h = exp(delta A) h + delta B u, y = C h + D u, gated by silu(z); state in and out; with
           the gradients of everything that goes in
  answers  log probabilities of given labels, entropy and the k best alternatives of each row of logits; with the logits' gradient

A sequence is a run of rows: rows offsets[s] .. offsets[s + 1] - 1, of which the first counts[s] are there (all where there are
no counts). Rows that belong to no sequence stay as they are.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZES = {"bf16": 2, "fp16": 2, "fp32": 4}


# ---- cases -------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # the ten flows of a streaming batch that got another packet: one row each, states kept by flow
        {"name": "conv few tokens", "op": "conv", "S": 10, "L": 1, "D": 256, "W": 4, "silu": True, "state": True, "ragged": False, "train": False, "type": "bf16"},
        # training on flows of up to 128 packets, in planes of 128 packets a flow
        {"name": "conv flows train", "op": "conv", "S": 8192, "L": 128, "D": 256, "W": 4, "silu": True, "state": False, "ragged": True, "padded": True, "train": True, "type": "bf16"},
        # the same streaming batch, one row each
        {"name": "scan few tokens", "op": "scan", "S": 10, "L": 1, "D": 256, "N": 16, "G": 1, "z": True, "softplus": True, "state": True, "ragged": False, "train": False, "type": "bf16"},
        # a full batch of packets of different flows, one step of each flow's state
        {"name": "scan tokens", "op": "scan", "S": 4096, "L": 1, "D": 1024, "N": 16, "G": 1, "z": True, "softplus": True, "state": True, "ragged": False, "train": False, "type": "bf16"},
        # the assigned flows of a batch, up to 128 packets each, in planes of 128 packets a flow
        {"name": "scan flows", "op": "scan", "S": 4096, "L": 128, "D": 256, "N": 16, "G": 1, "z": True, "softplus": True, "state": False, "ragged": True, "padded": True, "train": False, "type": "bf16"},
        # one long monitored flow, its state kept
        {"name": "scan long", "op": "scan", "S": 1, "L": 8192, "D": 1024, "N": 16, "G": 1, "z": True, "softplus": True, "state": True, "ragged": False, "train": False, "type": "bf16"},
        # a training step over windows of 512 packets
        {"name": "scan train", "op": "scan", "S": 64, "L": 512, "D": 512, "N": 16, "G": 1, "z": True, "softplus": True, "state": False, "ragged": False, "train": True, "type": "bf16"},
        # few short sequences of odd sizes in full precision, one behind the other, without a gate
        {"name": "scan odd train", "op": "scan", "S": 7, "L": 301, "D": 77, "N": 5, "G": 1, "z": False, "softplus": True, "state": False, "ragged": True, "padded": False, "train": True, "type": "fp32"},
        # the logits of eight classes of a streaming batch's flows
        {"name": "answers few rows", "op": "answers", "n": 10, "V": 8, "k": 1, "masked": 0.0, "scale": 1.0, "train": False, "type": "fp32"},
        # loss, entropy and runner-up of a batch of a million flows, with the gradient
        {"name": "answers batch", "op": "answers", "n": 1000000, "V": 16, "k": 2, "masked": 0.1, "scale": 1.0, "train": True, "type": "fp32"},
        # rows over a large vocabulary of header tokens, in training
        {"name": "answers vocabulary train", "op": "answers", "n": 2048, "V": 32768, "k": 8, "masked": 0.0, "scale": 1.0, "train": True, "type": "bf16"},
        # one row over a larger, odd one
        {"name": "answers one row", "op": "answers", "n": 1, "V": 250001, "k": 20, "masked": 0.2, "scale": 0.7, "train": False, "type": "fp16"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def draw(rng):
    op = rng.choice(["conv", "scan", "scan", "answers"])
    kind = rng.choice(["bf16", "fp16", "fp32"])
    train = rng.random() < 0.5
    if op == "answers":
        V = _log(rng, 1, 262144)
        return {"op": op, "n": _log(rng, 1, max(1, min(10 ** 6, 2 ** 26 // V))), "V": V, "k": rng.randint(0, min(V, 24)),
                "masked": round(rng.uniform(0, 1) ** 2, 2), "scale": rng.choice([1.0, 0.7, 1.5]), "train": train, "type": kind}
    D, L = _log(rng, 1, 4096), rng.choice([1, _log(rng, 2, 128), _log(rng, 2, 512 if train else 8192)])
    c = {"op": op, "S": 1, "L": L, "D": D, "state": not train, "ragged": rng.random() < 0.7, "padded": rng.random() < 0.5, "train": train, "type": kind}
    if op == "conv":
        most = 10 ** 8 // (L * D)
        return {**c, "S": _log(rng, 1, max(1, min(65536, most))), "W": rng.randint(1, 8), "silu": rng.random() < 0.7}
    N = rng.choice([16, 16, _log(rng, 1, 64)])
    most = 2 ** 28 // (L * D * N) if train else min(2 ** 25 // (L * D), 2 ** 28 // (D * N))
    return {**c, "S": _log(rng, 1, max(1, min(16384, most))), "N": N, "G": rng.choice([g for g in (1, 1, 2, 4) if D % g == 0]),
            "z": rng.random() < 0.7, "softplus": rng.random() < 0.8}


# ---- inputs ----------------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 29)
    return g


def _lengths(case):
    """Rows of each sequence: all L, or evenly spread up to L with an empty one among eight and more."""
    S, L = case["S"], case["L"]
    if not case["ragged"]:
        return [L] * S
    return [0 if S >= 8 and i == 0 else -(-L * (i + 1) // S) for i in range(S)]


def _rows(case):
    lengths = _lengths(case)
    return case["S"] * case["L"] if case.get("padded") else sum(lengths)


def _sequences(case, g):
    """offsets, counts and slots: lengths in random order; in planes of L rows a sequence, or one behind the other."""
    S, L = case["S"], case["L"]
    length = torch.tensor(_lengths(case), dtype=torch.int64, device=DEV)[torch.randperm(S, device=DEV, generator=g)]
    if case.get("padded"):
        offsets, counts = torch.arange(S + 1, device=DEV) * L, length.int()
    else:
        offsets, counts = torch.cat([torch.zeros_like(length[:1]), length.cumsum(0)]), None
    slots = torch.randperm(S + 3, device=DEV, generator=g)[:S].int() if case["state"] else None
    return {"offsets": offsets.int(), "counts": counts, "slots": slots}


def _bind(s):
    """The handle that a program keeps beside its sequences."""
    if own:
        sf, _ = _library()
        s["seq"] = sf.make_sequences(s["offsets"], s["case"]["L"], counts=s["counts"], slots=s["slots"])


def prepare(case, seed):
    g, op, t = _gen(seed), case["op"], TYPES[case["type"]]
    s = {"case": case}
    rand = lambda *d: torch.randn(*d, device=DEV, generator=g)  # noqa: E731
    if op == "answers":
        n, V, k = case["n"], case["V"], case["k"]
        x = (rand(n, V) * 2).to(t)
        if case["masked"]:
            x.masked_fill_(torch.rand(n, V, device=DEV, generator=g) < case["masked"], -math.inf)
        s["logits"] = x
        s["labels"] = torch.randint(0, V, (n,), device=DEV, generator=g, dtype=torch.int32)
        s["labels"].masked_fill_(torch.rand(n, device=DEV, generator=g) < 0.02, -1)
        s["logprob"], s["entropy"], s["lse"] = (torch.zeros(n, device=DEV) for _ in range(3))
        s["top_ids"], s["top_logprobs"] = torch.zeros(n, k, dtype=torch.int32, device=DEV), torch.zeros(n, k, device=DEV)
        if case["train"]:
            s["d_logprob"], s["d_entropy"], s["d_logits"] = -torch.rand(n, device=DEV, generator=g), rand(n) * 0.1, torch.zeros_like(x)
        return s
    D, R = case["D"], _rows(case)
    s.update(_sequences(case, g))
    if op == "conv":
        W = case["W"]
        s["x"] = rand(R, D).to(t)
        s["w"], s["bias"] = rand(D, W) / math.sqrt(W), rand(D) * 0.1
        s["y"] = torch.zeros_like(s["x"])
        if case["state"]:
            s["state_in"] = rand(case["S"] + 3, W - 1, D).to(t)
            s["state_out"] = torch.zeros_like(s["state_in"])
        if case["train"]:
            s["dy"] = rand(R, D).to(t)
            s["dx"], s["dw"], s["dbias"] = torch.zeros_like(s["x"]), torch.zeros_like(s["w"]), torch.zeros_like(s["bias"])
    else:
        N, G = case["N"], case["G"]
        s["u"] = rand(R, D).to(t)
        step = torch.exp(torch.rand(D, device=DEV, generator=g) * math.log(100.0) + math.log(0.001))          # steps from 0.001 to 0.1
        raw = rand(R, D) * 0.5
        if case["softplus"]:
            s["delta"], s["delta_bias"] = raw.to(t), step + torch.log(-torch.expm1(-step))
        else:
            s["delta"], s["delta_bias"] = (torch.exp(raw) * step).to(t), None
        s["A"] = -torch.arange(1, N + 1, device=DEV) * torch.exp(rand(D, N) * 0.1)
        s["B"], s["C"] = rand(R, G * N).to(t), rand(R, G * N).to(t)
        s["D"] = 1 + rand(D) * 0.1
        s["z"] = rand(R, D).to(t) if case["z"] else None
        s["y"] = torch.zeros_like(s["u"])
        if case["state"]:
            s["state_in"] = rand(case["S"] + 3, D, N)
            s["state_out"] = torch.zeros_like(s["state_in"])
        if case["train"]:
            s["dy"] = rand(R, D).to(t)
            for q in ("u", "delta", "A", "B", "C", "D", "delta_bias", "z"):
                s["d_" + q] = None if s[q] is None else torch.zeros_like(s[q])
    _scratch(s)
    return s


def _scratch(s):
    """What a program allocates once: the sequences' handle, states for the backward pass, workspaces."""
    _bind(s)
    c = s["case"]
    if not own:
        return
    sf, _ = _library()
    byte = lambda b: torch.zeros(b, dtype=torch.uint8, device=DEV)  # noqa: E731
    if c["op"] == "conv" and c["train"]:
        s["work"] = byte(sf.sf_seq_conv_backward_workspace(c["S"], c["L"], c["D"], c["W"]))
    if c["op"] == "scan":
        R = s["u"].shape[0]
        s["work"] = byte(sf.sf_seq_scan_workspace(c["S"], c["L"], R, c["D"], c["N"], c["G"], backward=c["train"]))
        s["starts"] = torch.zeros(sf.sf_seq_scan_starts(c["S"], R, c["D"], c["N"]), device=DEV) if c["train"] else None


# ---- the plain forms ---------------------------------------------------------------------------------------------------------
def _planes(s):
    """Row of each sequence's place [S][L] and whether it is there."""
    at = torch.arange(s["case"]["L"], device=DEV)
    first, end = s["offsets"][:-1].long(), s["offsets"][1:].long()
    length = end - first if s["counts"] is None else torch.minimum(s["counts"].long(), end - first)
    there = at < length[:, None]
    return torch.where(there, first[:, None] + at, 0), there, length


def _spread(v, row, there):
    """[rows][D] -> [S][L][D] in 32 bits, zeros where there is no row."""
    return torch.where(there[..., None], v[row].float(), 0.0) if v.shape[0] else torch.zeros(*row.shape, v.shape[1], device=DEV)


def _back(v, row, there, like):
    out = torch.zeros_like(like)
    out[row[there]] = v[there].to(like.dtype)
    return out


def _sigmoid(x):
    return 1 / (1 + torch.exp(-x))


def _plain_conv(s):
    c = s["case"]
    D, W, L = c["D"], c["W"], c["L"]
    row, there, length = _planes(s)
    before = s["state_in"][s["slots"].long()].float() if c["state"] else torch.zeros(c["S"], W - 1, D, device=DEV)
    x = torch.cat([before, _spread(s["x"], row, there)], 1)
    pre = s["bias"].expand(c["S"], L, D)
    for k in range(W):
        pre = pre + s["w"][:, k] * x[:, k:k + L]
    y = pre * _sigmoid(pre) if c["silu"] else pre
    r = {"y": _back(y, row, there, s["x"])}
    if c["state"]:
        last = (length[:, None] + torch.arange(W - 1, device=DEV))[..., None].expand(-1, -1, D)
        r["state"] = torch.zeros_like(s["state_in"])
        r["state"][s["slots"].long()] = x.gather(1, last).to(s["x"].dtype)
    if c["train"]:
        d = _spread(s["dy"], row, there)
        if c["silu"]:
            g = _sigmoid(pre)
            d = d * g * (1 + pre * (1 - g))
        dx = torch.zeros_like(x)
        for k in range(W):
            dx[:, k:k + L] += s["w"][:, k] * d
        r["dx"] = _back(dx[:, W - 1:], row, there, s["x"])
        r["dw"] = torch.stack([(d * x[:, k:k + L]).sum((0, 1)) for k in range(W)], 1)
        r["dbias"] = d.sum((0, 1))
    return r


def _plain_scan(s):
    c = s["case"]
    S, L, D, N, G = c["S"], c["L"], c["D"], c["N"], c["G"]
    row, there, _ = _planes(s)
    wide = lambda v: _spread(v, row, there).view(S, L, G, -1)  # noqa: E731
    u, B, C = wide(s["u"]), wide(s["B"]), wide(s["C"])
    raw = wide(s["delta"])
    if c["softplus"]:
        raw = raw + s["delta_bias"].view(G, -1)
        delta = torch.clamp(raw, min=0) + torch.log1p(torch.exp(-raw.abs()))
    else:
        delta = raw
    delta = torch.where(there[:, :, None, None], delta, 0.0)
    A, Dk = s["A"].view(G, -1, N), s["D"].view(G, -1)
    h = (s["state_in"][s["slots"].long()] if c["state"] else torch.zeros(S, D, N, device=DEV)).view(S, G, -1, N)
    start, hs, y = h, [], torch.empty_like(u)
    for t in range(L):
        h = torch.exp(delta[:, t, ..., None] * A) * h + (delta[:, t] * u[:, t])[..., None] * B[:, t, :, None]
        y[:, t] = (h * C[:, t, :, None]).sum(-1)
        if c["train"]:
            hs.append(h)
    y = y + Dk * u
    z = wide(s["z"]) if c["z"] else None
    out = y * z * _sigmoid(z) if c["z"] else y
    r = {"y": _back(out.view(S, L, D), row, there, s["u"])}
    if c["state"]:
        r["state"] = torch.zeros_like(s["state_in"])
        r["state"][s["slots"].long()] = h.reshape(S, D, N)
    if not c["train"]:
        return r
    dy = wide(s["dy"])
    if c["z"]:
        g = _sigmoid(z)
        r["d_z"] = _back((dy * y * g * (1 + z * (1 - g))).view(S, L, D), row, there, s["z"])
        dy = dy * z * g
    du, dd, dB, dC = Dk * dy, torch.zeros_like(delta), torch.zeros_like(B), torch.zeros_like(C)
    dA, carry = torch.zeros_like(A), torch.zeros_like(h)
    for t in range(L - 1, -1, -1):
        carry = carry + dy[:, t, ..., None] * C[:, t, :, None]
        dC[:, t] = (dy[:, t, ..., None] * hs[t]).sum(2)
        dB[:, t] = (carry * (delta[:, t] * u[:, t])[..., None]).sum(2)
        dx = (carry * B[:, t, :, None]).sum(-1)
        carry = carry * torch.exp(delta[:, t, ..., None] * A)
        da = carry * (hs[t - 1] if t else start)
        dd[:, t] = dx * u[:, t] + (da * A).sum(-1)
        du[:, t] += dx * delta[:, t]
        dA = dA + (da * delta[:, t, ..., None]).sum(0)
    if c["softplus"]:
        dd = torch.where(there[:, :, None, None], dd * _sigmoid(raw), 0.0)
        r["d_delta_bias"] = dd.sum((0, 1)).view(D)
    flat = lambda v, like: _back(v.reshape(S, L, -1), row, there, like)  # noqa: E731
    r.update(d_u=flat(du, s["u"]), d_delta=flat(dd, s["delta"]), d_A=dA.view(D, N), d_B=flat(dB, s["B"]), d_C=flat(dC, s["C"]),
             d_D=(dy * u).sum((0, 1)).view(D))
    return r


def _plain_answers(s):
    c, k = s["case"], s["case"]["k"]
    x = s["logits"].float() * c["scale"]
    top = x.amax(-1, keepdim=True)
    m = torch.where(top > -math.inf, top, 0.0)
    e = torch.exp(x - m)
    total = e.sum(-1, keepdim=True)
    there = total > 0
    lse = torch.where(there, m + torch.log(total), -math.inf)
    p = torch.where(there, e / total, 0.0)
    entropy = torch.where(there, torch.log(total), 0.0) - torch.where(p > 0, p * (x - m), 0.0).sum(-1, keepdim=True)
    has = s["labels"] >= 0
    at = s["labels"].clamp(min=0).long()[:, None]
    own_x = x.gather(1, at)
    logprob = torch.where(has[:, None], torch.where(own_x > -math.inf, own_x - lse, -math.inf), 0.0)
    value, ids = torch.sort(s["logits"], dim=-1, descending=True, stable=True)
    value, ids = value[:, :k].float(), ids[:, :k]
    r = {"logprob": logprob[:, 0], "entropy": entropy[:, 0], "lse": lse[:, 0], "top_ids": torch.where(value > -math.inf, ids, -1).int(),
         "top_logprobs": torch.where(value > -math.inf, value * c["scale"] - lse, -math.inf)}
    if c["train"]:
        g = torch.where(has, s["d_logprob"], 0.0)[:, None]
        d = -g * p - s["d_entropy"][:, None] * torch.where(p > 0, p * (x - lse + entropy), 0.0)
        d = d.scatter_add_(1, at, g)
        r["d_logits"] = torch.where(x > -math.inf, d * c["scale"], 0.0).to(s["logits"].dtype)
    return r


PLAIN = {"conv": _plain_conv, "scan": _plain_scan, "answers": _plain_answers}


# ---- the framework's calls ------------------------------------------------------------------------------------------------------
_held = {}


def _library():
    """The library's binding and a context: a program has one context for its stream and keeps it."""
    if not _held:
        from paper_2402_03694_b200 import binding
        _held["sf"], _held["ctx"] = binding, binding.sf_ctx_create(0, 0)
    return _held["sf"], _held["ctx"]


def _own_conv(s):
    sf, ctx = _library()
    c = s["case"]
    act = sf.SF_ACT_SILU if c["silu"] else sf.SF_ACT_NONE
    sf.sf_seq_conv(ctx, s["seq"], s["x"], s["w"], s["y"], bias=s["bias"], act=act, state_in=s.get("state_in"), state_out=s.get("state_out"))
    r = {"y": s["y"]}
    if c["state"]:
        r["state"] = s["state_out"]
    if c["train"]:
        sf.sf_seq_conv_backward(ctx, s["seq"], s["x"], s["w"], s["dy"], s["work"], bias=s["bias"], act=act, dx_out=s["dx"],
                                dw_out=s["dw"], dbias_out=s["dbias"])
        r.update(dx=s["dx"], dw=s["dw"], dbias=s["dbias"])
    return r


def _own_scan(s):
    sf, ctx = _library()
    c = s["case"]
    rows = dict(D=s["D"], delta_bias=s["delta_bias"], z=s["z"], softplus=c["softplus"])
    sf.sf_seq_scan(ctx, s["seq"], s["u"], s["delta"], s["A"], s["B"], s["C"], s["y"], workspace=s["work"], state_in=s.get("state_in"),
                   state_out=s.get("state_out"), starts_out=s["starts"], **rows)
    r = {"y": s["y"]}
    if c["state"]:
        r["state"] = s["state_out"]
    if c["train"]:
        sf.sf_seq_scan_backward(ctx, s["seq"], s["u"], s["delta"], s["A"], s["B"], s["C"], s["dy"], s["starts"], s["work"],
                                du_out=s["d_u"], d_delta_out=s["d_delta"], dA_out=s["d_A"], dB_out=s["d_B"], dC_out=s["d_C"], dD_out=s["d_D"],
                                d_delta_bias_out=s["d_delta_bias"], dz_out=s["d_z"], **rows)
        r.update({q: s[q] for q in ("d_u", "d_delta", "d_A", "d_B", "d_C", "d_D", "d_delta_bias", "d_z") if s[q] is not None})
    return r


def _own_answers(s):
    sf, ctx = _library()
    c = s["case"]
    sf.sf_label_logprobs(ctx, s["logits"], s["labels"], s["logprob"], entropy_out=s["entropy"], lse_out=s["lse"], top_ids_out=s["top_ids"],
                         top_logprobs_out=s["top_logprobs"], scale=c["scale"])
    r = {q: s[q] for q in ("logprob", "entropy", "lse", "top_ids", "top_logprobs")}
    if c["train"]:
        sf.sf_label_logprobs_backward(ctx, s["logits"], s["labels"], s["lse"], s["d_logits"], d_logprob=s["d_logprob"], entropy=s["entropy"],
                                      d_entropy=s["d_entropy"], scale=c["scale"])
        r["d_logits"] = s["d_logits"]
    return r


OWN = {"conv": _own_conv, "scan": _own_scan, "answers": _own_answers}


def run(state):
    return (OWN if own else PLAIN)[state["case"]["op"]](state)


# ---- what cannot be done without ---------------------------------------------------------------------------------------------------
def work(case):
    op, size = case["op"], SIZES[case["type"]]
    if op == "answers":
        n, V, k = case["n"], case["V"], case["k"]
        b, f = n * (V * size + 16 + 8 * k), 6 * n * V
        return {"bytes": b + (n * (V * size + 8) if case["train"] else 0), "flops": f + (8 * n * V if case["train"] else 0)}
    S, D = case["S"], case["D"]
    rows = sum(_lengths(case))
    if op == "conv":
        W = case["W"]
        b = 2 * rows * D * size + (2 * S * (W - 1) * D * size if case["state"] else 0) + D * (W + 1) * 4
        f = rows * D * (2 * W + (5 if case["silu"] else 0))
        return {"bytes": b + (2 * rows * D * size + D * (W + 1) * 4 if case["train"] else 0), "flops": f + (rows * D * (6 * W + 8) if case["train"] else 0)}
    N, G = case["N"], case["G"]
    wide, params = 3 + case["z"], D * (N + 2) * 4
    b = rows * (wide * D + 2 * G * N) * size + params + (2 * S * D * N * 4 if case["state"] else 0)
    f = rows * D * (7 * N + 12)
    if case["train"]:
        b += rows * ((3 + case["z"]) * D + 2 * G * N) * size + params
        f += rows * D * (17 * N + 24)
    return {"bytes": b, "flops": f}


# ---- the same from the definitions, in 64 bits ----------------------------------------------------------------------------------------
def _exact_lengths(s):
    off = s["offsets"].tolist()
    counts = s["counts"].tolist() if s["counts"] is not None else [b - a for a, b in zip(off, off[1:])]
    return off[:-1], counts


def _exact_conv(s):
    """From the last row to the first: row i of the result takes row i - j of the sequence or, before it, of the state."""
    c = s["case"]
    first, counts = _exact_lengths(s)
    S, L, D, W = c["S"], c["L"], c["D"], c["W"]
    length = torch.tensor(counts, device=DEV)
    R = s["x"].shape[0]
    x = s["x"].double().requires_grad_(c["train"])
    w, bias = s["w"].double().requires_grad_(c["train"]), s["bias"].double().requires_grad_(c["train"])
    owner = torch.full((R,), -1, dtype=torch.int64, device=DEV)
    place = torch.zeros(R, dtype=torch.int64, device=DEV)
    where = torch.tensor(first, device=DEV).repeat_interleave(length)
    inside = torch.arange(where.shape[0], device=DEV) - (length.cumsum(0) - length).repeat_interleave(length)
    owner[where + inside], place[where + inside] = torch.arange(S, device=DEV).repeat_interleave(length), inside
    state = torch.zeros(S, W - 1, D, dtype=torch.float64, device=DEV)
    if c["state"]:
        state = s["state_in"][s["slots"].long()].double()
    real = owner >= 0
    pre = torch.zeros(R, D, dtype=torch.float64, device=DEV) + bias
    for j in range(W):
        tap = w[:, W - 1 - j]
        v = torch.cat([torch.zeros(j, D, dtype=torch.float64, device=DEV), x[:max(R - j, 0)]])[:R]
        v = torch.where((place >= j)[:, None], v, 0.0)
        if c["state"] and j:
            early = real & (place < j)
            v = v.clone()
            v[early] = state[owner[early], place[early] - j + W - 1]
        pre = pre + tap * v
    y = torch.where(real[:, None], torch.nn.functional.silu(pre) if c["silu"] else pre, 0.0)
    r = {"y": y.detach()}
    if c["state"]:
        out = torch.zeros(s["state_in"].shape, dtype=torch.float64, device=DEV)
        for i in range(W - 1):
            at = length - (W - 1) + i
            rows = x.detach()[(torch.tensor(first, device=DEV) + at).clamp(0, max(R - 1, 0))] if R else torch.zeros(S, D, dtype=torch.float64, device=DEV)
            old = state[torch.arange(S, device=DEV), (at + W - 1).clamp(0, W - 2)]
            out[s["slots"].long(), i] = torch.where((at >= 0)[:, None], rows, old)
        r["state"] = out
    if c["train"]:
        dy = torch.where(real[:, None], s["dy"].double(), 0.0)
        r["dx"], r["dw"], r["dbias"] = torch.autograd.grad(y, (x, w, bias), dy)
    return r


def _exact_scan(s):
    """State by state over padded planes, gradients by differentiating the loop."""
    c = s["case"]
    first, counts = _exact_lengths(s)
    S, L, D, N, G = c["S"], c["L"], c["D"], c["N"], c["G"]
    R = s["u"].shape[0]
    grad = c["train"]
    leaf = {q: None if s[q] is None else s[q].double().requires_grad_(grad) for q in ("u", "delta", "A", "B", "C", "D", "delta_bias", "z")}
    length = torch.tensor(counts, device=DEV)
    at = (torch.tensor(first, device=DEV)[None] + torch.arange(L, device=DEV)[:, None]).clamp(max=max(R - 1, 0))
    live = (torch.arange(L, device=DEV)[:, None] < length)[..., None]
    take = lambda v: v[at]  # noqa: E731
    step = torch.nn.functional.softplus(leaf["delta"] + leaf["delta_bias"], threshold=60) if c["softplus"] else leaf["delta"]
    group = torch.arange(D, device=DEV) // (D // G)
    h = torch.zeros(N, S, D, dtype=torch.float64, device=DEV)
    if c["state"]:
        h = s["state_in"][s["slots"].long()].double().permute(2, 0, 1)
    At = leaf["A"].t()[:, None]
    ys = []
    if R:
        du, u, B, C = torch.where(live, take(step), 0.0), take(leaf["u"]), take(leaf["B"]).view(L, S, G, N), take(leaf["C"]).view(L, S, G, N)
        for t in range(L):
            Bt = B[t].permute(2, 0, 1) if G == 1 else B[t].permute(2, 0, 1)[..., group]
            Ct = C[t].permute(2, 0, 1) if G == 1 else C[t].permute(2, 0, 1)[..., group]
            h = h * torch.exp(At * du[t]) + Bt * (du[t] * u[t])
            ys.append((h * Ct).sum(0))
    y = torch.zeros(R, D, dtype=torch.float64, device=DEV)
    if R:
        there = live[..., 0]
        y = y.index_put((at[there],), torch.stack(ys)[there])
        mine = torch.zeros(R, 1, dtype=torch.float64, device=DEV)
        mine[at[there]] = 1
        y = y + mine * leaf["D"] * leaf["u"]
        if c["z"]:
            y = y * torch.nn.functional.silu(leaf["z"])
    r = {"y": y.detach()}
    if c["state"]:
        r["state"] = torch.zeros(s["state_in"].shape, dtype=torch.float64, device=DEV)
        r["state"][s["slots"].long()] = h.permute(1, 2, 0).detach()
    if grad:
        names = [q for q in leaf if leaf[q] is not None]
        got = torch.autograd.grad(y, [leaf[q] for q in names], s["dy"].double(), allow_unused=True)
        r.update({"d_" + q: torch.zeros_like(leaf[q]) if v is None else v for q, v in zip(names, got)})
    return r


def _exact_answers(s):
    c, k = s["case"], s["case"]["k"]
    x = s["logits"].double() * c["scale"]
    n, V = x.shape
    lse = torch.logsumexp(x, -1)
    logp = torch.where(x > -math.inf, x - lse[:, None], -math.inf)
    p = torch.exp(logp)
    entropy = -torch.special.xlogy(p, p).sum(-1)
    label = s["labels"].long()
    rows = torch.arange(n, device=DEV)
    logprob = torch.where(label >= 0, logp[rows, label.clamp(min=0)], 0.0)
    # one after the other: the largest that is left, the first of equals
    left, ids, values = s["logits"].float().clone(), [], []
    for _ in range(k):
        best = left.amax(-1)
        at = (left == best[:, None]).to(torch.uint8).argmax(-1)
        ids.append(torch.where(best > -math.inf, at, -1))
        values.append(torch.where(best > -math.inf, logp[rows, at], -math.inf))
        left[rows, at] = -math.inf
    none = torch.zeros(n, 0, device=DEV)
    r = {"logprob": logprob, "entropy": entropy, "lse": lse, "top_ids": torch.stack(ids, 1).int() if k else none.int(),
         "top_logprobs": torch.stack(values, 1) if k else none.double()}
    if c["train"]:
        g = torch.where(label >= 0, s["d_logprob"].double(), 0.0)
        d = -p * (g[:, None] + s["d_entropy"].double()[:, None] * torch.where(p > 0, logp + entropy[:, None], 0.0))
        d[rows, label.clamp(min=0)] += g
        r["d_logits"] = torch.where(x > -math.inf, d * c["scale"], 0.0)
    return r


EXACT = {"conv": _exact_conv, "scan": _exact_scan, "answers": _exact_answers}


def exact(case, seed):
    return EXACT[case["op"]](prepare(case, seed))

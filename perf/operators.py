"""Cases that measure the operators of a slow model made of experts in 4-bit arithmetic: what each takes in, its plain
form, the framework's calls and the values in 64 bits.

  quantise   rows -> 4-bit floating point with one power-of-two scale per 32 values (packed), and back to values
  product    packed rows x packed weights (+ bias, ReLU): one weight matrix, or one per expert over sorted rows
  gate       a row's k best experts and their weights from its scores, with the gradient of the scores
  dispatch   (row, expert) pairs sorted by expert and the rows brought into that order, with the gradient of the rows
  combine    the experts' rows weighted and added back into one row per flow, with the gradients of rows and weights

Packed layout: two values a byte (the first in the low half), rows padded to whole blocks of 32; the blocks' scale bytes
(exponent + 127, 255 = not a number) in tiles of 128 rows x 4 blocks, byte (r % 32) * 16 + (r / 32) * 4 + b of a tile,
tiles row block by row block.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
GATES = {"softmax": 0, "softmax of picked": 1, "share": 2}


def up(v, to):
    return -(-v // to) * to


# ---- cases -------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one flow's wide row (128 packets x 16 fields) on its way into the slow model
        {"name": "quantise one row", "op": "quantise", "n": 1, "K": 2048, "type": "bf16"},
        # the assigned rows of a batch of a million flows
        {"name": "quantise assigned rows", "op": "quantise", "n": 240001, "K": 2048, "type": "bf16"},
        # about ten flows of a streaming batch reach the slow model: a hidden layer on them
        {"name": "product few rows", "op": "product", "n": 10, "K": 1024, "N": 1024, "experts": 1, "spread": 0.0, "type": "bf16"},
        # the first hidden layer on the assigned rows of a batch of a million flows
        {"name": "product assigned rows", "op": "product", "n": 240001, "K": 2048, "N": 1024, "experts": 1, "spread": 0.0, "type": "bf16"},
        # a few hundred flows over five experts, one without a flow; odd sizes, full-precision outputs
        {"name": "product experts odd", "op": "product", "n": 713, "K": 416, "N": 200, "experts": 5, "spread": 2.0, "type": "fp32"},
        # a hidden layer of sixteen class specialists
        {"name": "product experts", "op": "product", "n": 131072, "K": 1024, "N": 512, "experts": 16, "spread": 0.5, "type": "bf16"},
        # the streaming batch's handful of flows, two experts each
        {"name": "gate few rows", "op": "gate", "n": 10, "E": 8, "k": 2, "gate": "softmax of picked", "masked": 0.0, "type": "fp32"},
        # a million flows' class scores, classes without a specialist masked, as a training step takes it
        {"name": "gate batch", "op": "gate", "n": 1000000, "E": 16, "k": 2, "gate": "softmax", "masked": 0.2, "type": "fp32"},
        # the handful again, one expert each
        {"name": "dispatch few rows", "op": "dispatch", "n": 10, "D": 2048, "E": 8, "k": 1, "align": 128, "train": False, "type": "bf16"},
        # half of a batch's assigned rows, two experts each, in training
        {"name": "dispatch batch", "op": "dispatch", "n": 120003, "D": 2048, "E": 16, "k": 2, "align": 128, "train": True, "type": "bf16"},
        # logits of eight classes from two experts
        {"name": "combine few rows", "op": "combine", "n": 13, "D": 8, "E": 8, "k": 2, "train": False, "type": "fp32"},
        # hidden rows from two experts, in training
        {"name": "combine batch", "op": "combine", "n": 120003, "D": 1024, "E": 16, "k": 2, "train": True, "type": "bf16"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantise", "product", "gate", "dispatch", "combine"])
    kind = rng.choice(["bf16", "fp16", "fp32"])
    if op == "quantise":
        K = _log(rng, 1, 8192)
        return {"op": op, "n": _log(rng, 1, min(240000, 240000 * 1024 // K)), "K": K, "type": kind}
    if op == "product":
        K, E = _log(rng, 32, 8192), rng.choice([1, 1, 2, 5, 16, 40])
        N = _log(rng, 1, min(4096, 10 ** 8 // (K * E)))
        most = min(240000, 5 * 10 ** 11 // (2 * K * N), 2 * 10 ** 8 // max(K, N))
        return {"op": op, "n": _log(rng, 1, max(1, most)), "K": K, "N": N, "experts": E, "spread": round(rng.uniform(0, 2), 2),
                "type": rng.choice(["bf16", "fp32"])}
    E = _log(rng, 1, 256)
    k = rng.randint(1, min(E, 8))
    if op == "gate":
        return {"op": op, "n": _log(rng, 1, min(10 ** 6, 16 * 10 ** 6 // E)), "E": E, "k": k, "gate": rng.choice(sorted(GATES)),
                "masked": round(rng.uniform(0, 1) ** 2, 2), "type": kind}
    D = _log(rng, 1, 8192)
    c = {"op": op, "n": _log(rng, 1, max(1, min(10 ** 6, 10 ** 8 // (D * k)))), "D": D, "E": E, "k": k, "train": rng.random() < 0.5, "type": kind}
    return {**c, "align": rng.choice([1, 16, 128])} if op == "dispatch" else c


# ---- packed 4-bit rows ---------------------------------------------------------------------------------------------------
def blocks_of(x):
    """[n][K] in 32 bits -> [n][blocks][32], zeros behind the last value."""
    n, K = x.shape
    return torch.nn.functional.pad(x.float(), (0, up(K, 32) - K)).view(n, -1, 32)


def scale_value(byte):
    """The power of two that a scale byte stands for, in 32 bits."""
    b = byte.to(torch.int32)
    bits = torch.where(b == 0, 0x00400000, b << 23)
    return torch.where(b == 255, 0x7FC00000, bits).view(torch.float32)


def round4(x):
    """[n][K] -> codes [n][blocks][32] (bit 3 the sign) and scale bytes [n][blocks]: the exponent of the block's largest
    magnitude less 2, each value to the nearest of 0 .5 1 1.5 2 3 4 6 (ties to the even code), beyond 6 to 6."""
    x = blocks_of(x)
    top = x.abs().amax(-1).view(torch.int32) >> 23
    bad = (x.abs().amax(-1).view(torch.int32) >= 0x7F800000) | x.isnan().any(-1)
    byte = torch.where(bad, 255, (top - 2).clamp(0, 252))
    v = torch.where(bad[..., None], 0.0, x.abs() / scale_value(byte.clamp(max=254))[..., None])
    step = torch.where(v < 2, 0.5, torch.where(v < 4, 1.0, 2.0))
    v = (torch.round(v / step) * step).clamp(max=6)
    code = torch.where(v < 2, v * 2, torch.where(v < 4, v + 2, v / 2 + 4)).to(torch.uint8)
    return code | (torch.signbit(x) & ~bad[..., None]).to(torch.uint8) * 8, byte.to(torch.uint8)


def tiles_of(byte):
    """Scale bytes [n][blocks] in tiles of 128 rows x 4 blocks (127, a scale of one, where there is no block)."""
    n, nb = byte.shape
    b = torch.nn.functional.pad(byte, (0, up(nb, 4) - nb, 0, up(n, 128) - n), value=127)
    return b.view(-1, 4, 32, b.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).reshape(-1)


def rows_of(tiles, n, K):
    """tiles_of() the other way round."""
    nb = up(K, 32) // 32
    b = tiles.view(up(n, 128) // 128, up(nb, 4) // 4, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(up(n, 128), -1)
    return b[:n, :nb]


def pack(x):
    code, byte = round4(x)
    code = code.view(x.shape[0], -1)
    return (code[:, 0::2] | (code[:, 1::2] << 4)).contiguous(), tiles_of(byte)


def unpack(data, tiles, n, K):
    """The values that packed rows stand for, in 32 bits."""
    code = torch.stack([data & 15, data >> 4], -1).view(n, -1, 32)
    value = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=data.device)[code.int()]
    return (value * scale_value(rows_of(tiles, n, K))[..., None]).view(n, -1)[:, :K]


# ---- inputs ----------------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 17)
    return g


def _wide_rows(n, K, g):
    """Wide rows as the packet fields give them: length, logarithm of the inter-arrival time, direction, header bytes."""
    x = torch.randint(0, 256, (n, K), device=DEV, generator=g, dtype=torch.int16).float() / 256
    x[:, 0::16] *= 0.73
    x[:, 2::16] = (x[:, 2::16] > 0.5).float()
    return x


def _pairs(n, k, E, spread, g):
    """k different experts a flow, popular and unpopular ones; a few flows miss one."""
    liking = torch.randn(E, device=DEV, generator=g) * spread
    ids = (liking - torch.log(-torch.log(torch.rand(n, E, device=DEV, generator=g).clamp(1e-7, 1 - 1e-7)))).topk(k, -1).indices.int()
    return torch.where(torch.rand(n, k, device=DEV, generator=g) < 0.01, -1, ids)


def sort_plain(ids, E, align, capacity):
    """Offsets [E + 1], counts [E], flow of each sorted row [capacity] and row of each pair [n][k]; -1 where there is none."""
    n, k = ids.shape
    flat = ids.reshape(-1).long()
    real = (flat >= 0) & (flat < E)
    key = torch.where(real, flat, E)
    order = torch.sort(key, stable=True).indices
    counts = torch.zeros(E + 1, dtype=torch.int64, device=ids.device).index_add_(0, key, torch.ones_like(key))
    sizes = (counts[:E] + align - 1) // align * align
    offsets = torch.cat([torch.zeros_like(sizes[:1]), sizes.cumsum(0)])
    first = torch.cat([torch.zeros_like(sizes[:1]), counts[:E].cumsum(0)])
    key = key[order]
    row = torch.where(key < E, offsets[key] + torch.arange(n * k, device=ids.device) - first[key], capacity)
    flow_of_row = torch.full((capacity + 1,), -1, dtype=torch.int32, device=ids.device)
    flow_of_row[row] = (order // k).int()
    flow_of_row[capacity] = -1
    row_of_pair = torch.empty(n * k, dtype=torch.int32, device=ids.device)
    row_of_pair[order] = torch.where(row < capacity, row, -1).int()
    return offsets.int(), counts[:E].int(), flow_of_row[:capacity], row_of_pair.view(n, k)


def prepare(case, seed):
    g, op, n = _gen(seed), case["op"], case["n"]
    s = {"case": case}
    if op == "quantise":
        K = case["K"]
        s["x"] = _wide_rows(n, K, g).to(TYPES[case["type"]])
        s["data"] = torch.zeros(n, up(K, 32) // 2, dtype=torch.uint8, device=DEV)
        s["scales"] = torch.zeros(up(n, 128) * (up(K, 128) // 32), dtype=torch.uint8, device=DEV)
        s["values"] = torch.zeros(n, K, dtype=torch.bfloat16, device=DEV)
    elif op == "product":
        K, N, E = case["K"], case["N"], case["experts"]
        if E > 1:
            # the plan of a pass over experts: sorted rows, every expert's first row a multiple of 128
            cap = up(n, 128) + 128 * E
            ids = _pairs(n, 1, E, case["spread"], g)
            s["offsets"], s["counts"], s["flow_of_row"], _ = sort_plain(ids, E, 128, cap)
            s["most"] = int(s["counts"].max())
        else:
            cap = n
        x = torch.relu(torch.randn(cap, K, device=DEV, generator=g))
        if E > 1:
            x *= (s["flow_of_row"] >= 0)[:, None]
        s["a"], s["a_scales"] = pack(x)
        w = (torch.rand(E * N, K, device=DEV, generator=g) * 2 - 1) * math.sqrt(6.0 / (K + N))
        packed = [pack(m) for m in w.view(E, N, K)]
        s["w"] = torch.stack([d for d, _ in packed])
        s["w_scales"] = torch.stack([t for _, t in packed])
        s["bias"] = torch.rand(E, N, device=DEV, generator=g) * 0.2 - 0.1
        s["out"] = torch.zeros(cap, N, dtype=TYPES[case["type"]], device=DEV)
    elif op == "gate":
        E, k = case["E"], case["k"]
        x = torch.randn(n, E, device=DEV, generator=g) * 2
        if case["gate"] == "share":
            x = torch.softmax(x, -1)
        s["scores"] = torch.where(torch.rand(n, E, device=DEV, generator=g) < case["masked"], -math.inf, x).to(TYPES[case["type"]])
        s["d_weights"] = torch.randn(n, k, device=DEV, generator=g)
        s["ids"] = torch.zeros(n, k, dtype=torch.int32, device=DEV)
        s["weights"] = torch.zeros(n, k, device=DEV)
        s["d_scores"] = torch.zeros_like(s["scores"])
    else:
        D, E, k, t = case["D"], case["E"], case["k"], TYPES[case["type"]]
        align = case.get("align", 128)
        cap = n * k + E * (align - 1)
        s["ids"] = _pairs(n, k, E, 0.5, g)
        plan = sort_plain(s["ids"], E, align, cap)
        if op == "dispatch":
            s["x"] = _wide_rows(n, D, g).to(t)
            s["offsets"], s["counts"] = torch.zeros_like(plan[0]), torch.zeros_like(plan[1])
            s["flow_of_row"], s["row_of_pair"] = torch.full_like(plan[2], -1), torch.full_like(plan[3], -1)
            s["rows"] = torch.zeros(cap, D, dtype=t, device=DEV)
            s["work"] = torch.zeros(_sort_workspace(n, k, E), dtype=torch.uint8, device=DEV)
            if case["train"]:
                s["d_rows"] = torch.randn(cap, D, device=DEV, generator=g).to(t)
                s["dx"] = torch.zeros(n, D, dtype=t, device=DEV)
        else:
            s["offsets"], s["counts"], s["flow_of_row"], s["row_of_pair"] = plan
            s["rows"] = torch.randn(cap, D, device=DEV, generator=g).to(t)
            s["weights"] = torch.softmax(torch.randn(n, k, device=DEV, generator=g), -1)
            s["y"] = torch.zeros(n, D, dtype=t, device=DEV)
            if case["train"]:
                s["dy"] = torch.randn(n, D, device=DEV, generator=g).to(t)
                s["d_rows"], s["d_weights"] = torch.zeros_like(s["rows"]), torch.zeros(n, k, device=DEV)
    return s


def _sort_workspace(n, k, E):
    """Bytes of scratch that sorting n * k pairs over E experts takes at most."""
    return 4 * (E + 1) * (up(n * k, 1024) // 1024 + 2) + 1024


# ---- the plain forms ---------------------------------------------------------------------------------------------------------
def _plain_quantise(s):
    n, K = s["x"].shape
    data, scales = pack(s["x"])
    return {"values": unpack(data, scales, n, K).to(torch.bfloat16), "scales": rows_of(scales, n, K)}


def _plain_product(s):
    c = s["case"]
    K, N, E = c["K"], c["N"], c["experts"]
    cap = s["a"].shape[0]
    a = unpack(s["a"], s["a_scales"], cap, K)
    if E == 1:
        w = unpack(s["w"][0], s["w_scales"][0], N, K)
        return {"out": torch.relu(a @ w.T + s["bias"][0]).to(s["out"].dtype)}
    per = up(N, 128)
    w = unpack(torch.nn.functional.pad(s["w"], (0, 0, 0, per - N)).view(E * per, -1), s["w_scales"].view(-1), E * per, K).view(E, per, K)[:, :N]
    at = torch.arange(s["most"], device=DEV)
    inside = at < s["counts"][:, None]
    row = torch.where(inside, s["offsets"][:-1, None] + at, cap)
    y = torch.relu(torch.bmm(torch.nn.functional.pad(a, (0, 0, 0, 1))[row], w.transpose(1, 2)) + s["bias"][:, None])
    # rows that only fill an expert's last 128 hold zeros: they come out as the bias
    fill = torch.bucketize(torch.arange(cap, device=DEV), s["offsets"][1:].long(), right=True)
    out = torch.cat([torch.relu(s["bias"]), torch.zeros_like(s["bias"][:1])])[fill]
    out = torch.cat([out, out[:1]])
    out[row] = y
    return {"out": out[:cap].to(s["out"].dtype)}


def _order(x, k):
    """The k largest of each row in falling order, ties to the lowest index; -inf and NaN are never among them."""
    picked = torch.where(x > -math.inf, x, -math.inf)
    value, at = torch.sort(picked, dim=-1, descending=True, stable=True)
    return value[:, :k], torch.where(value[:, :k] > -math.inf, at[:, :k], -1)


def _plain_gate(s):
    c = s["case"]
    x, k, g = s["scores"].float(), c["k"], s["d_weights"]
    v, ids = _order(x, k)
    real = ids >= 0
    at = ids.clamp(min=0)
    g = torch.where(real, g, 0.0)
    if c["gate"] == "share":
        v = torch.where(real, v, 0.0)
        total = v.sum(-1, keepdim=True)
        w = torch.where(real & (total > 0), v / total, 0.0)
        d = torch.where(real & (total > 0), (g - (g * w).sum(-1, keepdim=True)) / total, 0.0)
        ds = torch.zeros_like(x).scatter_add_(1, at, d)
    else:
        m = v[:, :1]
        near = lambda t: torch.where(t == m, 1.0, torch.exp(t - m)) * (t > -math.inf)  # noqa: E731
        e = torch.where(x > -math.inf, near(x), 0.0)
        pick = torch.where(real, near(v), 0.0)
        total = (e if c["gate"] == "softmax" else pick).sum(-1, keepdim=True)
        w = torch.where(real, pick / total, 0.0)
        spread = torch.zeros_like(x).scatter_add_(1, at, g)
        chosen = torch.zeros_like(x).scatter_add_(1, at, w)
        p = torch.where(total > 0, e / total, 0.0) if c["gate"] == "softmax" else chosen
        ds = p * (spread - (g * w).sum(-1, keepdim=True))
    return {"ids": ids.int(), "weights": w, "d_scores": ds.to(s["scores"].dtype)}


def _plain_dispatch(s):
    c = s["case"]
    offsets, counts, flow_of_row, row_of_pair = sort_plain(s["ids"], c["E"], c["align"], s["rows"].shape[0])
    r = {"offsets": offsets, "counts": counts, "flow_of_row": flow_of_row, "row_of_pair": row_of_pair,
         "rows": torch.where(flow_of_row[:, None] >= 0, s["x"][flow_of_row.clamp(min=0).long()], 0.0).to(s["x"].dtype)}
    if c["train"]:
        r["dx"] = _weighted(s["d_rows"], row_of_pair, None).to(s["x"].dtype)
    return r


def _weighted(rows, row_of_pair, weights):
    """The sum over a flow's pairs of weight * row, in 32 bits; a pair without a row adds nothing."""
    real = row_of_pair >= 0
    v = torch.where(real[..., None], rows[row_of_pair.clamp(min=0).long()].float(), 0.0)
    return (v if weights is None else v * torch.where(real, weights, 0.0)[..., None]).sum(1)


def _plain_combine(s):
    rows, at, w = s["rows"], s["row_of_pair"], s["weights"]
    r = {"y": _weighted(rows, at, w).to(rows.dtype)}
    if s["case"]["train"]:
        real = at >= 0
        cap, D = rows.shape
        dy = s["dy"].float()
        spread = torch.zeros(cap + 1, D, device=DEV)
        spread[torch.where(real, at, cap).long()] = w[..., None] * dy[:, None]
        r["d_rows"] = spread[:cap].to(rows.dtype)
        r["d_weights"] = torch.where(real, (rows[at.clamp(min=0).long()].float() * dy[:, None]).sum(-1), 0.0)
    return r


PLAIN = {"quantise": _plain_quantise, "product": _plain_product, "gate": _plain_gate, "dispatch": _plain_dispatch, "combine": _plain_combine}


# ---- the framework's calls ------------------------------------------------------------------------------------------------------
_held = {}


def _library():
    """The library's binding and a context: a program has one context for its stream and keeps it."""
    if not _held:
        from paper_2402_03694_b200 import binding
        _held["sf"], _held["ctx"] = binding, binding.sf_ctx_create(0, 0)
    return _held["sf"], _held["ctx"]


def _own_quantise(s):
    sf, ctx = _library()
    n, K = s["x"].shape
    sf.sf_mx4_quantise(ctx, s["x"], s["data"], s["scales"])
    sf.sf_mx4_unpack(ctx, s["data"], s["scales"], s["values"])
    return {"values": s["values"], "scales": rows_of(s["scales"], n, K)}


def _own_product(s):
    sf, ctx = _library()
    c = s["case"]
    if c["experts"] == 1:
        sf.sf_mx4_matmul(ctx, s["a"], s["a_scales"], s["w"][0], s["w_scales"][0], c["K"], s["out"], bias=s["bias"], relu=True)
    else:
        sf.sf_mx4_matmul_experts(ctx, s["a"], s["a_scales"], s["w"], s["w_scales"], c["K"], s["offsets"], s["out"], bias=s["bias"], relu=True)
    return {"out": s["out"]}


def _own_gate(s):
    sf, ctx = _library()
    mode = GATES[s["case"]["gate"]]
    sf.sf_expert_gate(ctx, s["scores"], mode, s["ids"], s["weights"])
    sf.sf_expert_gate_backward(ctx, s["scores"], mode, s["ids"], s["d_weights"], s["d_scores"])
    return {"ids": s["ids"], "weights": s["weights"], "d_scores": s["d_scores"]}


def _own_dispatch(s):
    sf, ctx = _library()
    c = s["case"]
    sf.sf_expert_sort(ctx, s["ids"], c["E"], c["align"], s["offsets"], s["counts"], s["flow_of_row"], s["row_of_pair"], s["work"])
    sf.sf_expert_gather(ctx, s["x"], s["row_of_pair"], s["offsets"], s["counts"], s["rows"])
    r = {q: s[q] for q in ("offsets", "counts", "flow_of_row", "row_of_pair", "rows")}
    if c["train"]:
        sf.sf_expert_gather_backward(ctx, s["d_rows"], s["row_of_pair"], s["dx"])
        r["dx"] = s["dx"]
    return r


def _own_combine(s):
    sf, ctx = _library()
    sf.sf_expert_combine(ctx, s["rows"], s["row_of_pair"], s["weights"], s["y"])
    r = {"y": s["y"]}
    if s["case"]["train"]:
        sf.sf_expert_combine_backward(ctx, s["dy"], s["rows"], s["row_of_pair"], s["weights"], s["offsets"], s["counts"],
                                      s["d_rows"], s["d_weights"])
        r["d_rows"], r["d_weights"] = s["d_rows"], s["d_weights"]
    return r


OWN = {"quantise": _own_quantise, "product": _own_product, "gate": _own_gate, "dispatch": _own_dispatch, "combine": _own_combine}


def run(state):
    return (OWN if own else PLAIN)[state["case"]["op"]](state)


# ---- what cannot be done without ---------------------------------------------------------------------------------------------------
def work(case):
    op, n = case["op"], case["n"]
    size = {"bf16": 2, "fp16": 2, "fp32": 4}[case["type"]]
    if op == "quantise":
        K = case["K"]
        packed = n * up(K, 32) * 17 // 32
        return {"bytes": n * K * (size + 2) + packed, "flops": 4 * n * K}
    if op == "product":
        K, N, E = case["K"], case["N"], case["experts"]
        return {"bytes": (n + E * N) * up(K, 32) * 17 // 32 + E * N * 4 + n * N * size, "flops": 2 * n * N * K}
    if op == "gate":
        return {"bytes": n * (2 * case["E"] * size + case["k"] * 12), "flops": 8 * n * case["E"]}
    D, k, E = case["D"], case["k"], case["E"]
    if op == "dispatch":
        b = n * k * 12 + n * (1 + k) * D * size + 8 * E
        return {"bytes": b + (n * (1 + k) * D * size if case["train"] else 0), "flops": n * k * D if case["train"] else n * k}
    b = n * k * 8 + n * (1 + k) * D * size
    return {"bytes": b + (n * k * 4 + n * (1 + k) * D * size if case["train"] else 0), "flops": (6 if case["train"] else 2) * n * k * D}


# ---- the same from the definitions, in 64 bits ----------------------------------------------------------------------------------------
CODES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_values(data, tiles, n, K):
    """A byte holds two values, the first in its low half; a tile's byte for row r and block b is at (r % 32) * 16 + (r / 32) * 4 + b."""
    table = torch.tensor(CODES + tuple(-v for v in CODES), dtype=torch.float64, device=DEV)
    out = torch.empty(n, data.shape[1] * 2, dtype=torch.float64, device=DEV)
    out[:, 0::2], out[:, 1::2] = table[(data % 16).long()], table[(data // 16).long()]
    r, b = torch.arange(n, device=DEV)[:, None], torch.arange(data.shape[1] // 16, device=DEV)[None]
    tile = (r // 128) * (up(K, 128) // 128) + b // 4
    byte = tiles[tile * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4].double()
    out.view(n, -1, 32).mul_(torch.exp2(byte - 127)[..., None])
    return out[:, :K]


def _exact_quantise(s):
    n, K = s["x"].shape
    x = torch.zeros(n, up(K, 32), dtype=torch.float64, device=DEV)
    x[:, :K] = s["x"]
    x = x.view(n, -1, 32)
    e = (torch.frexp(x.abs().amax(-1)).exponent - 3).clamp(min=-127)
    e = torch.where(x.abs().amax(-1) == 0, -127, e)
    v = x / torch.exp2(e.double())[..., None]
    # a border between two codes goes to the even one: 0, 1, 2 and 4 are even
    low = torch.tensor([0.25, 1.25, 2.5, 5.0], dtype=torch.float64, device=DEV)
    high = torch.tensor([0.75, 1.75, 3.5], dtype=torch.float64, device=DEV)
    code = torch.bucketize(v.abs(), low) + torch.bucketize(v.abs(), high, right=True)
    y = torch.tensor(CODES, dtype=torch.float64, device=DEV)[code] * v.sign() * torch.exp2(e.double())[..., None]
    return {"values": y.view(n, -1)[:, :K].contiguous(), "scales": (e + 127).to(torch.uint8)}


def _exact_product(s):
    c = s["case"]
    K, N, E = c["K"], c["N"], c["experts"]
    cap = s["a"].shape[0]
    ends = s["offsets"].tolist() if E > 1 else [0, cap]
    out = torch.zeros(cap, N, dtype=torch.float64, device=DEV)
    a = _exact_values(s["a"], s["a_scales"], cap, K)
    for i in range(E):
        w = _exact_values(s["w"][i], s["w_scales"][i], N, K)
        out[ends[i]:ends[i + 1]] = (a[ends[i]:ends[i + 1]].matmul(w.t()) + s["bias"][i].double()).clamp(min=0)
    return {"out": out}


def _exact_gate(s):
    c, k = s["case"], s["case"]["k"]
    x, g = s["scores"].double(), s["d_weights"].double()
    n, E = x.shape
    # an expert's rank is the number of experts before it
    rank = torch.empty(n, E, dtype=torch.int64, device=DEV)
    lower = torch.ones(E, E, dtype=torch.bool, device=DEV).tril(-1)
    for i in range(0, n, max(1, 10 ** 8 // (E * E))):
        y = x[i:i + max(1, 10 ** 8 // (E * E))]
        rank[i:i + y.shape[0]] = ((y[:, None] > y[..., None]) | (y[:, None] == y[..., None]) & lower).sum(-1)
    picked = (rank < k) & (x > -math.inf)
    ids = torch.full((n, k + 1), -1, dtype=torch.int64, device=DEV)
    ids.scatter_(1, torch.where(picked, rank, k), torch.arange(E, device=DEV).expand(n, E).contiguous())
    ids = ids[:, :k]
    own_g = torch.where(picked, g.gather(1, rank.clamp(max=k - 1)), 0.0)
    if c["gate"] == "share":
        base = torch.where(picked, x, 0.0)
    else:
        base = torch.exp(x - x.amax(-1, keepdim=True).clamp(min=-1e300))
        if c["gate"] != "softmax":
            base = base * picked
    total = base.sum(-1, keepdim=True)
    full = torch.where(total > 0, base / total, 0.0)
    mean = (own_g * full).sum(-1, keepdim=True)
    if c["gate"] == "share":
        ds = torch.where(picked & (total > 0), (own_g - mean) / total, 0.0)
    else:
        ds = full * (own_g - mean)
    w = torch.where(ids >= 0, full.gather(1, ids.clamp(min=0)), 0.0)
    return {"ids": ids.int(), "weights": w, "d_scores": ds}


def _exact_dispatch(s):
    c, n, D = s["case"], s["x"].shape[0], s["x"].shape[1]
    ids, cap = s["ids"].long(), s["rows"].shape[0]
    offsets, counts, at = [0], [], torch.full_like(ids, -1)
    flow_of_row = torch.full((cap,), -1, dtype=torch.int64, device=DEV)
    for e in range(c["E"]):
        flow, j = (ids == e).nonzero(as_tuple=True)
        row = offsets[-1] + torch.arange(len(flow), device=DEV)
        at[flow, j], flow_of_row[row] = row, flow
        counts.append(len(flow))
        offsets.append(offsets[-1] + up(len(flow), c["align"]))
    rows = torch.zeros(cap, D, dtype=torch.float64, device=DEV)
    rows[flow_of_row >= 0] = s["x"][flow_of_row[flow_of_row >= 0]].double()
    whole = lambda v: torch.as_tensor(v, device=DEV).int()  # noqa: E731
    r = {"offsets": whole(offsets), "counts": whole(counts), "flow_of_row": whole(flow_of_row), "row_of_pair": whole(at), "rows": rows}
    if c["train"]:
        dx = torch.zeros(n, D, dtype=torch.float64, device=DEV)
        for j in range(c["k"]):
            have = at[:, j] >= 0
            dx[have] += s["d_rows"][at[have, j]].double()
        r["dx"] = dx
    return r


def _exact_combine(s):
    at, w, rows = s["row_of_pair"].long(), s["weights"].double(), s["rows"]
    n, k = at.shape
    train = s["case"]["train"]
    y = torch.zeros(n, rows.shape[1], dtype=torch.float64, device=DEV)
    d_rows = torch.zeros(rows.shape, dtype=torch.float64, device=DEV) if train else None
    d_weights = torch.zeros(n, k, dtype=torch.float64, device=DEV) if train else None
    for j in range(k):
        have = at[:, j] >= 0
        row = at[have, j]
        y[have] += w[have, j, None] * rows[row].double()
        if train:
            dy = s["dy"][have].double()
            d_rows[row] = w[have, j, None] * dy
            d_weights[have, j] = (dy * rows[row].double()).sum(-1)
    return {"y": y, "d_rows": d_rows, "d_weights": d_weights} if train else {"y": y}


EXACT = {"quantise": _exact_quantise, "product": _exact_product, "gate": _exact_gate, "dispatch": _exact_dispatch, "combine": _exact_combine}


def exact(case, seed):
    return EXACT[case["op"]](prepare(case, seed))

"""What a layer of experts on packed weights needs around and between its products: the choice of experts for each token,
the tokens' order by expert, the products of each expert's tokens with its packed matrix, and the sum of a token's results.

A server keeps every expert's matrices as packed codes, one blob an expert, stacked.  For each step or prompt it has the
router's logits, chooses, orders the choices by expert, multiplies (gate and up in one product with the gated activation,
then down) and adds up with the router's weights.  Widths and bit widths are those of the benchmark's decoder layer sets (4096 /
11008, 5120, 8192; 4, 3 and 2 bits in groups of 128, 64 and 32) and generic ones.

`run` gives the same outputs in a plain form (elementary torch operations in 32 bits, scores in 64, rounded once) or, where
`own` is true, by the library's calls.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
MOST_FLOPS = 1.4e12                   # of a drawn case
MOST_WEIGHTS = 6.0e8
MOST_VALUES = 1.5e8                   # of a plain form's tokens, gathered


def listed():
    return [
        # one token's choice: a call whose latency is all that counts
        {"name": "route_one_token", "kind": "route", "tokens": 1, "experts": 64, "top_k": 6, "type": "f32", "score": "softmax", "bias": False,
         "groups": 1, "top_groups": 1, "group_best": 1, "renormalise": True},
        # a long prompt: sigmoid scores, a bias for balance, experts in groups of which the best four take part, a few experts masked
        {"name": "route_prompt_groups", "kind": "route", "tokens": 8190, "experts": 192, "top_k": 7, "type": "bf16", "score": "sigmoid", "bias": True,
         "groups": 12, "top_groups": 4, "group_best": 2, "renormalise": True},
        # a decoding batch's choices by expert
        {"name": "plan_step", "kind": "plan", "tokens": 48, "experts": 32, "top_k": 4},
        # a long prompt's
        {"name": "plan_prompt", "kind": "plan", "tokens": 16383, "experts": 192, "top_k": 8},
        # one token through the gate and up matrices of two large experts: the weights are all there is to read
        {"name": "product_one_token", "kind": "product", "tokens": 1, "experts": 8, "top_k": 2, "K": 4096, "N": 11008, "gated": True, "bits": 4,
         "group": 128, "type": "f32"},
        # a small batch through narrow experts' down matrices, some 3 tokens an expert, 3 bits
        {"name": "product_step_down", "kind": "product", "tokens": 24, "experts": 32, "top_k": 4, "K": 1408, "N": 4096, "gated": False, "bits": 3,
         "group": 64, "type": "f32"},
        # an ordinary batch through narrow experts, short groups
        {"name": "product_step_up", "kind": "product", "tokens": 61, "experts": 64, "top_k": 6, "K": 2048, "N": 1408, "gated": True, "bits": 4,
         "group": 32, "type": "bf16"},
        # the largest: a prompt through large experts
        {"name": "product_prompt", "kind": "product", "tokens": 4096, "experts": 8, "top_k": 2, "K": 4096, "N": 11008, "gated": True, "bits": 4,
         "group": 128, "type": "bf16"},
        # a prompt of odd length through many narrow experts' down matrices, 2 bits, f16
        {"name": "product_prompt_down", "kind": "product", "tokens": 1023, "experts": 60, "top_k": 8, "K": 1792, "N": 5120, "gated": False, "bits": 2,
         "group": 64, "type": "f16"},
        # a batch's results, added up
        {"name": "combine_step", "kind": "combine", "tokens": 24, "experts": 32, "top_k": 4, "N": 4096, "type": "f32", "residual": False},
        # a prompt's, onto the residual stream
        {"name": "combine_prompt", "kind": "combine", "tokens": 4095, "experts": 60, "top_k": 8, "N": 5120, "type": "bf16", "residual": True},
        # the whole layer for a decoding batch: choice, order, two products, sum
        {"name": "layer_step", "kind": "layer", "tokens": 16, "experts": 32, "top_k": 4, "K": 4096, "N": 1408, "bits": 4, "group": 64, "type": "f32"},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(max(low, high))))))


def draw(rng):
    kind = rng.choice(("route", "route", "plan", "product", "product", "product", "product", "combine", "layer"))
    tokens, dtype = _log(rng, 1, 8192), rng.choice(("f32", "bf16", "f16"))
    if kind == "route":
        groups = rng.choice((1, 1, 4, 8, 12))
        experts = groups * _log(rng, 2, 512 // groups)
        top_groups = rng.randrange(1, groups + 1)
        best = rng.choice((1, 2))
        return {"kind": kind, "tokens": tokens, "experts": experts, "top_k": rng.randrange(1, min(12, top_groups * experts // groups) + 1), "type": dtype,
                "score": rng.choice(("softmax", "sigmoid")), "bias": rng.random() < 0.5, "groups": groups, "top_groups": top_groups,
                "group_best": best if groups > 1 else 1, "renormalise": rng.random() < 0.7}
    experts = _log(rng, 2, 192)
    top_k = rng.randrange(1, min(8, experts) + 1)
    if kind == "plan":
        return {"kind": kind, "tokens": 2 * tokens, "experts": experts, "top_k": top_k}
    if kind == "combine":
        N = rng.choice((2048, 4096, 5120, 8192, _log(rng, 64, 8192)))
        return {"kind": kind, "tokens": max(1, min(tokens, (20 << 20) // (N * top_k))), "experts": experts, "top_k": top_k, "N": N, "type": dtype,
                "residual": rng.random() < 0.5}
    bits, group = rng.choice((4, 4, 3, 2)), rng.choice((32, 64, 128))
    K = group * _log(rng, 512 // group, 8192 // group)
    N = _log(rng, 256, 11008)
    if kind == "layer":                   # its inputs' width is K, the experts' inner one N
        N = group * max(1, N // group)
    gated = kind == "layer" or rng.random() < 0.5
    experts = max(2, min(experts, int(MOST_WEIGHTS / (N * K * (1 + gated + (kind == "layer"))))))
    top_k = min(top_k, experts)
    tokens = max(1, min(tokens, int(MOST_FLOPS / 3 / (2 * top_k * N * K * (1 + gated))), int(MOST_VALUES / (top_k * (K + 2 * N)))))
    case = {"kind": kind, "tokens": min(tokens, 512) if kind == "layer" else tokens, "experts": experts, "top_k": top_k, "K": K, "N": N,
            "bits": bits, "group": group, "type": "f32" if kind == "layer" else dtype}
    return case if kind == "layer" else {**case, "gated": gated}


# --- inputs -----------------------------------------------------------------------------------------------------

def _logits(case, g):
    """Router's logits: some experts are more popular than others."""
    popular = torch.randn(case["experts"], generator=g, device="cuda")
    return 1.5 * torch.randn(case["tokens"], case["experts"], generator=g, device="cuda") + 0.7 * popular


def _choices(case, g):
    """Chosen experts of each token; every 64th token is padding, which chooses none."""
    ids = _logits(case, g).sort(1, descending=True)[1][:, : case["top_k"]].to(torch.int32)
    ids[63::64] = -1
    return ids.contiguous()


def _matrices(E, N, K, bits, group, g):
    """Quantized matrices of E experts: codes [E][N][K] and zero-points [E][N][K / group] in bytes, scales [E][N][K / group]."""
    q = torch.empty(E, N, K, dtype=torch.uint8, device="cuda")
    s = torch.empty(E, N, K // group, device="cuda")
    z = torch.empty(E, N, K // group, dtype=torch.uint8, device="cuda")
    top = 2 ** bits - 1
    for e in range(E):
        w = torch.randn(N, K // group, group, generator=g, device="cuda") / math.sqrt(K)
        low, high = w.amin(2).clamp(max=0), w.amax(2).clamp(min=0)
        s[e] = (high - low) / top
        zero = torch.round(-low / s[e]).clamp(0, top)
        z[e] = zero.to(torch.uint8)
        q[e] = (torch.round(w / s[e][..., None]) + zero[..., None]).clamp(0, top).view(N, K).to(torch.uint8)
    return q, s, z


CELL = {4: 8, 2: 16, 3: 32}


def _section(t):
    """Bytes of a blob's section, [E][bytes], filled up to a multiple of 256."""
    t = t.contiguous().view(torch.uint8).flatten(1)
    return torch.nn.functional.pad(t, (0, -t.shape[1] % 256))


def _packed(q, s, z, bits, group):
    """The blobs that qg_pack makes of these codes (QG_LAYOUT_DEVICE), one a row."""
    E, N, K = q.shape
    cell, tiles = CELL[bits], -(-N // 64)
    unit = 4 * cell
    padded = -(-K // (unit * (2 if bits == 3 else 4))) * unit * (2 if bits == 3 else 4)
    out = []
    for e in range(E):
        codes = torch.nn.functional.pad(q[e], (0, padded - K, 0, 64 * tiles - N)).view(tiles, 64, padded // unit, 4, cell).int()
        if bits == 3:
            a = codes.view(tiles, 64, -1, 4, 4, 2, 4)                       # word, low or high field, byte
            fields = a[..., 0, :] | a[..., 1, :] << 3
            rest = fields[..., 3, :]
            words = [sum((fields[..., w, i] | (rest[..., i] >> 2 * w & 3) << 6) << 8 * i for i in range(4)) for w in range(3)]
            words = torch.stack(words, 3).permute(0, 2, 3, 1, 4)            # [tile][unit][plane][lane][cell]
        else:
            words = sum(codes[..., i] << bits * i for i in range(cell)).permute(0, 2, 1, 3)
        zbits = 2 if bits == 2 else 4
        per = 32 // zbits
        groups = K // group
        scales = torch.nn.functional.pad(s[e], (0, 0, 0, 64 * tiles - N)).view(tiles, 64, groups).transpose(1, 2)
        zeros = torch.nn.functional.pad(z[e], (0, -groups % per, 0, 64 * tiles - N)).view(tiles, 64, -1, per).int()
        zeros = sum(zeros[..., i] << zbits * i for i in range(per)).transpose(1, 2)
        out.append(torch.cat([_section(t[None]) for t in (words, scales, zeros)], 1))
    return torch.cat(out)


def _order(ids, experts):
    """(offsets, tokens, slots) of the choices ordered by expert."""
    flat = torch.where((ids >= 0) & (ids < experts), ids, experts).flatten().long()
    by, order = flat.sort(dim=0, stable=True)
    real = by < experts
    offsets = torch.zeros(experts + 2, dtype=torch.long, device="cuda").scatter_add_(0, flat + 1, torch.ones_like(flat)).cumsum(0)[:-1]
    tokens = torch.where(real, order // ids.shape[1], -1)
    slots = torch.empty_like(flat)
    slots[order] = torch.where(real, torch.arange(flat.numel(), device="cuda"), -1)
    return offsets.int(), tokens.int(), slots.view(ids.shape).int()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    kind, T, E = case["kind"], case["tokens"], case["experts"]
    if kind == "route":
        logits = _logits(case, g)
        logits[:, :: 41][:, 1:] = -math.inf                                 # experts that are switched off
        logits[63::64] = -math.inf                                          # padding
        s["logits"] = logits.to(TYPES[case["type"]])
        s["balance"] = 0.2 * torch.randn(E, generator=g, device="cuda") if case["bias"] else None
        return s
    t = TYPES[case.get("type", "f32")]
    if kind == "layer":
        s["logits"] = _logits(case, g)
        s["x"] = torch.randn(T, case["K"], generator=g, device="cuda")
        s["up"] = _matrices(E, 2 * case["N"], case["K"], case["bits"], case["group"], g)
        s["down"] = _matrices(E, case["K"], case["N"], case["bits"], case["group"], g)
        s["up_packed"], s["down_packed"] = (_packed(*s[m], case["bits"], case["group"]) for m in ("up", "down"))
        return s
    ids = _choices(case, g)
    if kind == "plan":
        s["ids"] = ids
        return s
    s["offsets"], s["rows"], s["slots"] = _order(ids, E)
    if kind == "combine":
        s["y"] = torch.randn(ids.numel(), case["N"], generator=g, device="cuda").to(t)
        w = torch.rand(T, case["top_k"], generator=g, device="cuda") + 0.05
        s["weights"] = w / w.sum(1, keepdim=True)
        s["r"] = torch.randn(T, case["N"], generator=g, device="cuda").to(t) if case["residual"] else None
        return s
    # gate and up take a token's hidden state (a few channels far larger than the others), down takes what up left for each slot
    x = torch.randn(T if case["gated"] else ids.numel(), case["K"], generator=g, device="cuda")
    x[:, :: 97] *= 8
    s["x"] = x.to(t)
    s["matrix"] = _matrices(E, case["N"] * (2 if case["gated"] else 1), case["K"], case["bits"], case["group"], g)
    s["packed"] = _packed(*s["matrix"], case["bits"], case["group"])
    s["out"] = torch.zeros(ids.numel(), case["N"], dtype=t, device="cuda")  # a buffer that the server keeps
    if not case["gated"]:
        s["rows"] = None
    return s


def _library():
    from paper_2307_03738_amd import binding
    return binding


# --- the choice -------------------------------------------------------------------------------------------------

def _route(s):
    if own:
        ids, weights = _library().qg_route(s["logits"], s["top_k"], bias=s["balance"], score=s["score"], groups=s["groups"],
                                           top_groups=s["top_groups"], group_best=s["group_best"], renormalise=s["renormalise"])
        return {"ids": ids, "weights": weights}
    logits = s["logits"].double()
    masked = logits == -math.inf
    if s["score"] == "softmax":
        most = logits.amax(1, keepdim=True)
        p = torch.exp(logits - torch.where(most == -math.inf, 0.0, most))
        total = p.sum(1, keepdim=True)
        p = p / torch.where(total == 0, 1.0, total)
    else:
        p = 1 / (1 + torch.exp(-logits))
    value = p if s["balance"] is None else p + s["balance"].double()
    key = torch.where(masked, -math.inf, logits if s["balance"] is None else value)
    T, E, G = s["tokens"], s["experts"], s["groups"]
    if s["top_groups"] < G:
        if s["group_best"] == 2:
            two = torch.where(masked, -math.inf, value).view(T, G, -1).sort(2, descending=True)[0][..., :2]
            rank = torch.where(torch.isinf(two[..., 1:]), two[..., :1], two.sum(2, keepdim=True))[..., 0]
        else:
            rank = key.view(T, G, -1).amax(2)
        kept = torch.zeros(T, G, dtype=torch.bool, device="cuda")
        kept.scatter_(1, rank.sort(dim=1, descending=True, stable=True)[1][:, : s["top_groups"]], True)
        key = torch.where(kept[:, :, None], key.view(T, G, -1), -math.inf).view(T, E)
    best, ids = key.sort(dim=1, descending=True, stable=True)
    best, ids = best[:, : s["top_k"]], ids[:, : s["top_k"]]
    real = best > -math.inf
    w = torch.where(real, p.gather(1, ids), 0.0)
    if s["renormalise"]:
        total = w.sum(1, keepdim=True)
        w = w / torch.where(total == 0, 1.0, total)
    return {"ids": torch.where(real, ids, -1).int(), "weights": w.float()}


def _route_exact(s):
    l = s["logits"].double()
    p = l.softmax(1).nan_to_num(0) if s["score"] == "softmax" else l.sigmoid()
    c = l if s["balance"] is None else p + s["balance"].double()
    c = c.masked_fill(l == -math.inf, -math.inf)
    G = s["groups"]
    if s["top_groups"] < G:
        v = (p if s["balance"] is None else c).masked_fill(l == -math.inf, -math.inf).unflatten(1, (G, -1))
        top = (v if s["group_best"] == 2 else c.unflatten(1, (G, -1))).topk(s["group_best"], 2)[0]
        rank = top.masked_fill(top.isinf() & (torch.arange(s["group_best"], device="cuda") > 0), 0).sum(2)
        order = torch.argsort(-rank, dim=1, stable=True).argsort(1)
        c = c.masked_fill((order >= s["top_groups"]).repeat_interleave(s["experts"] // G, 1), -math.inf)
    order = torch.argsort(-c, dim=1, stable=True)[:, : s["top_k"]]
    gone = c.take_along_dim(order, 1).isinf()
    w = p.take_along_dim(order, 1).masked_fill(gone, 0)
    if s["renormalise"]:
        w = torch.nn.functional.normalize(w, p=1, dim=1, eps=1e-300)
    return {"ids": None, "weights": w}


# --- the order --------------------------------------------------------------------------------------------------

def _plan(s):
    if own:
        offsets, tokens, slots = _library().qg_expert_plan(s["ids"], s["experts"])
    else:
        offsets, tokens, slots = _order(s["ids"], s["experts"])
    return {"offsets": offsets, "tokens": tokens, "slots": slots}


# --- the products -----------------------------------------------------------------------------------------------

def _plain_product(x, matrix, offsets, rows, group, gated, out):
    """Products of every used expert's tokens, filled up to the longest expert's, with its dequantized matrix."""
    counts = offsets[1:] - offsets[:-1]
    used = counts.nonzero()[:, 0]
    if used.numel() == 0:
        return out
    most = int(counts.max())
    at = offsets[:-1][used].long()[:, None] + torch.arange(most, device="cuda")
    real = torch.arange(most, device="cuda") < counts[used][:, None]
    slot = torch.where(real, at, 0)
    row = slot if rows is None else rows[slot].long()
    q, s, z = (m[used] for m in matrix)
    U, N, K = q.shape
    w = ((q.view(U, N, -1, group).float() - z[..., None].float()) * s[..., None]).view(U, N, K).transpose(1, 2).contiguous()
    y = torch.matmul(x.float()[row.clamp(min=0)], w)
    if gated:
        gate, up = y.chunk(2, 2)
        y = gate / (1 + torch.exp(-gate)) * up
    out[slot[real]] = y[real].to(out.dtype)
    return out


def _product(s):
    if own:
        return {"y": _library().qg_experts_product(s["packed"], s["N"] * (2 if s["gated"] else 1), s["K"], s["bits"], s["group"], s["x"], s["offsets"],
                                                   rows=s["rows"], gated=s["gated"], y=s["out"])}
    return {"y": _plain_product(s["x"], s["matrix"], s["offsets"], s["rows"], s["group"], s["gated"], s["out"])}


def _exact_expert(x, q, s, z, gated):
    groups = s.shape[1]
    w = q.double().unflatten(1, (groups, -1)).sub_(z.double().unsqueeze(2)).mul_(s.double().unsqueeze(2)).flatten(1)
    y = x.double() @ w.t()
    if gated:
        half = y.shape[1] // 2
        y = torch.nn.functional.silu(y[:, :half]) * y[:, half:]
    return y


def _product_exact(s):
    y = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    ends = s["offsets"].tolist()
    for e, (begin, end) in enumerate(zip(ends, ends[1:])):
        if begin < end:
            x = s["x"][begin:end] if s["rows"] is None else s["x"][s["rows"][begin:end].long()]
            y[begin:end] = _exact_expert(x, *(m[e] for m in s["matrix"]), s["gated"])
    return {"y": y}


# --- the sum ----------------------------------------------------------------------------------------------------

def _plain_combine(y, slots, weights, residual, dtype):
    taken = torch.where((slots >= 0)[..., None], y.float()[slots.clamp(min=0).long()], 0.0)
    out = (weights[..., None] * taken).sum(1)
    return (out if residual is None else out + residual.float()).to(dtype)


def _combine(s):
    if own:
        return {"out": _library().qg_experts_combine(s["y"], s["slots"], s["weights"], residual=s["r"])}
    return {"out": _plain_combine(s["y"], s["slots"], s["weights"], s["r"], s["y"].dtype)}


def _combine_exact(s):
    out = torch.zeros(s["tokens"], s["N"], dtype=torch.float64, device="cuda") if s["r"] is None else s["r"].double()
    for j in range(s["top_k"]):
        slot = s["slots"][:, j].long()
        t = (slot >= 0).nonzero()[:, 0]
        out.index_add_(0, t, s["y"][slot[t]].double() * s["weights"][t, j].double().unsqueeze(1))
    return {"out": out}


# --- the layer --------------------------------------------------------------------------------------------------

def _layer(s):
    K, N = s["K"], s["N"]
    if own:
        qg = _library()
        ids, weights = qg.qg_route(s["logits"], s["top_k"])
        offsets, tokens, slots = qg.qg_expert_plan(ids, s["experts"])
        h = qg.qg_experts_product(s["up_packed"], 2 * N, K, s["bits"], s["group"], s["x"], offsets, rows=tokens, gated=True)
        y = qg.qg_experts_product(s["down_packed"], K, N, s["bits"], s["group"], h, offsets)
        return {"out": qg.qg_experts_combine(y, slots, weights)}
    choice = _route({**s, "score": "softmax", "balance": None, "groups": 1, "top_groups": 1, "renormalise": True})
    offsets, tokens, slots = _order(choice["ids"], s["experts"])
    pairs = tokens.numel()
    h = _plain_product(s["x"], s["up"], offsets, tokens, s["group"], True, torch.zeros(pairs, N, device="cuda"))
    y = _plain_product(h, s["down"], offsets, None, s["group"], False, torch.zeros(pairs, K, device="cuda"))
    return {"out": _plain_combine(y, slots, choice["weights"], None, torch.float32)}


def _layer_exact(s):
    best, ids = s["logits"].double().topk(s["top_k"], 1)
    w = best.softmax(1)
    out = torch.zeros(s["tokens"], s["K"], dtype=torch.float64, device="cuda")
    for e in range(s["experts"]):
        t, j = (ids == e).nonzero(as_tuple=True)
        if t.numel():
            h = _exact_expert(s["x"][t], *(m[e] for m in s["up"]), True)
            out.index_add_(0, t, _exact_expert(h, *(m[e] for m in s["down"]), False) * w[t, j].unsqueeze(1))
    return {"out": out}


def run(state):
    return {"route": _route, "plan": _plan, "product": _product, "combine": _combine, "layer": _layer}[state["kind"]](state)


def exact(case, seed):
    kind = case["kind"]
    if kind == "plan":
        return None                       # whole numbers
    return {"route": _route_exact, "product": _product_exact, "combine": _combine_exact, "layer": _layer_exact}[kind](prepare(case, seed))


def _used(pairs, experts):
    """Experts that so many choices are expected to name (popular ones count more, which this leaves out)."""
    return experts * (1 - (1 - 1 / experts) ** pairs)


def _matrix_bytes(N, K, bits, group):
    return N * K * bits / 8 + N * (K / group) * (4 + (2 if bits == 2 else 4) / 8)


def work(case):
    kind, T, E, k = case["kind"], case["tokens"], case["experts"], case["top_k"]
    if kind == "route":
        return {"bytes": T * E * BYTES[case["type"]] + 8 * T * k, "flops": 4 * T * E}
    pairs = k * (T - (T // 64 if kind != "layer" else 0))
    if kind == "plan":
        return {"bytes": 4 * (3 * T * k + E + 1), "flops": 0}
    size = BYTES[case["type"]]
    if kind == "combine":
        return {"bytes": size * case["N"] * (pairs + T * (2 if case["residual"] else 1)) + 8 * T * k, "flops": 2 * pairs * case["N"]}
    K, N = case["K"], case["N"]
    used = _used(pairs, E)
    if kind == "layer":
        weights = used * (_matrix_bytes(2 * N, K, case["bits"], case["group"]) + _matrix_bytes(K, N, case["bits"], case["group"]))
        return {"bytes": round(weights) + 4 * T * (2 * K + E), "flops": 6 * pairs * K * N}
    outputs = N * (2 if case["gated"] else 1)
    x = K * (T if case["gated"] else pairs)
    return {"bytes": round(used * _matrix_bytes(outputs, K, case["bits"], case["group"])) + size * (x + pairs * N), "flops": 2 * pairs * outputs * K}

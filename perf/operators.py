"""What a token's step needs between the products of packed weights: the norm in front of them, the paged
key-value cache (writing it, attention over it) and the pages' bookkeeping.

A server keeps a pool of pages shared by a batch of sequences.  Every step it norms the residual stream, multiplies
(not measured here), rotates q and k and stores k and v in the pages, attends, and, between steps, grows, forks, ends and
packs sequences.  Head counts and widths are those of the benchmark's decoder layer sets (4096 = 32 x 128, 5120 = 40 x 128,
8192 = 64 x 128) with one key head per head or one for several, and generic ones.

`run` gives the same outputs in a plain form (elementary torch operations in 32 bits, rounded once) or, where `own`
is true, by the library's calls.
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1}
E4M3_MOST = 448.0
EPS = 1e-5
WORKSPACE = 48 << 20                  # what a server keeps for attention, whatever the batch
LARGEST_CACHE = 1.5e9                 # bytes of keys and values that attention reads, at most


def listed():
    return [
        # one token's residual stream in front of a product: a call whose latency is all that counts
        {"name": "norm_one_row", "kind": "norm", "rows": 1, "K": 4096, "type": "f32", "out": "f32", "group": 0, "residual": True},
        # a long prompt's rows, handed on in 8 bits with a scale per 128 values
        {"name": "norm_prompt_e4m3", "kind": "norm", "rows": 4099, "K": 8192, "type": "bf16", "out": "e4m3", "group": 128, "residual": True},
        # one sequence's new token, fresh from the products, into a cache in 16 bits
        {"name": "append_one", "kind": "append", "rows": 1, "max_len": 1, "heads": 32, "kv_heads": 32, "head_dim": 128, "rope": 128,
         "interleaved": False, "type": "f32", "cache": "bf16", "page": 16, "start": 700},
        # a batch of prompts of uneven length, padding tokens among them, into a cache in 8 bits
        {"name": "append_prompts_e4m3", "kind": "append", "rows": 12, "max_len": 2048, "heads": 64, "kv_heads": 8, "head_dim": 128,
         "rope": 128, "interleaved": True, "type": "bf16", "cache": "e4m3", "page": 32, "start": 0},
        # one chat on its own: a key head for every head, a cache that ends inside a page
        {"name": "attend_one_short", "kind": "attend", "rows": 1, "max_len": 777, "heads": 32, "kv_heads": 32, "head_dim": 128,
         "type": "f32", "cache": "bf16", "page": 16, "window": 0, "padded": False},
        # an ordinary batch: lengths from none to some thousands, cache in 8 bits, prompts padded on the left
        {"name": "attend_ragged_e4m3", "kind": "attend", "rows": 32, "max_len": 4093, "heads": 64, "kv_heads": 8, "head_dim": 128,
         "type": "f32", "cache": "e4m3", "page": 32, "window": 0, "padded": True},
        # one long document, whose length is all there is to split the work over
        {"name": "attend_one_long", "kind": "attend", "rows": 1, "max_len": 131071, "heads": 40, "kv_heads": 8, "head_dim": 128,
         "type": "f16", "cache": "f16", "page": 64, "window": 0, "padded": False},
        # the largest batch
        {"name": "attend_large_batch", "kind": "attend", "rows": 128, "max_len": 8190, "heads": 64, "kv_heads": 8, "head_dim": 128,
         "type": "bf16", "cache": "bf16", "page": 16, "window": 0, "padded": False},
        # every sequence of a batch grows by a token: a few need a page, some share their last one with a branch
        {"name": "pages_step", "kind": "resize", "rows": 64, "max_pages": 256, "pages": 8192, "page": 16, "kv_heads": 8, "head_dim": 128,
         "layers": 1, "cache": "bf16", "grow": 1, "shared": True},
        # sequences branch and end: rows are taken over from others, their pages shared
        {"name": "pages_fork", "kind": "fork", "rows": 128, "max_pages": 512, "pages": 65536, "page": 16, "kv_heads": 1, "head_dim": 16,
         "layers": 1, "cache": "bf16", "grow": 0, "shared": False},
        # a small pool packed to its lower end
        {"name": "pages_compact_small", "kind": "compact", "rows": 8, "max_pages": 64, "pages": 1024, "page": 16, "kv_heads": 8,
         "head_dim": 64, "layers": 1, "cache": "f16", "grow": 0, "shared": False},
        # a large one, several layers of it
        {"name": "pages_compact_large", "kind": "compact", "rows": 96, "max_pages": 256, "pages": 16384, "page": 32, "kv_heads": 8,
         "head_dim": 128, "layers": 2, "cache": "e4m3", "grow": 0, "shared": True},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _heads(rng):
    group = rng.choice((1, 1, 2, 4, 5, 8, 8, 16))
    kv_heads = _log(rng, 1, 64 // group)
    return group * kv_heads, kv_heads


def draw(rng):
    kind = rng.choice(("norm", "append", "attend", "attend", "attend", "resize", "fork", "compact"))
    cache = rng.choice(("bf16", "f16", "e4m3"))
    page = rng.choice((16, 32, 64, 128))
    if kind == "norm":
        K = rng.choice((512, 4096, 5120, 8192, _log(rng, 64, 16384)))
        out = rng.choice(("f32", "bf16", "f16", "e4m3"))
        group = rng.choice([0] + [g for g in (64, 128) if K % g == 0]) if out == "e4m3" else 0
        return {"kind": kind, "rows": _log(rng, 1, min(16384, (32 << 20) // K)), "K": K, "type": rng.choice(("f32", "bf16", "f16")),
                "out": out, "group": group, "residual": rng.random() < 0.75}
    heads, kv_heads = _heads(rng)
    head_dim = rng.choice((64, 80, 96, 128, 128, 128, 256))
    if kind == "append":
        max_len = _log(rng, 1, 4096)
        rows = _log(rng, 1, max(1, min(128, (12 << 20) // (max_len * heads * head_dim // 8))))
        return {"kind": kind, "rows": rows, "max_len": max_len, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim,
                "rope": rng.choice((0, head_dim, head_dim, head_dim // 2)), "interleaved": rng.random() < 0.5,
                "type": rng.choice(("f32", "bf16", "f16")), "cache": cache, "page": page, "start": rng.choice((0, _log(rng, 1, 4096)))}
    if kind == "attend":
        most = LARGEST_CACHE / 4 / (2 * kv_heads * head_dim * BYTES[cache])       # keys
        max_len = _log(rng, 1, min(131072, most))
        rows = _log(rng, 1, max(1, min(128, most / max_len)))
        return {"kind": kind, "rows": rows, "max_len": max_len, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim,
                "type": rng.choice(("f32", "bf16", "f16")), "cache": cache, "page": page,
                "window": rng.choice((0, 0, 0, _log(rng, 16, 4096))), "padded": rng.random() < 0.3}
    rows = _log(rng, 1, 128)
    max_pages = _log(rng, 4, 512)
    pages = rows * max_pages + rng.randrange(1, 4096)
    kv_heads, layers = min(kv_heads, 16), rng.choice((1, 2, 4))
    while 2 * layers * pages * page * kv_heads * head_dim * BYTES[cache] > 1.0e9 and max_pages * rows > 64:
        rows, max_pages = max(1, rows * 2 // 3), max(4, max_pages * 2 // 3)
        pages = rows * max_pages + rng.randrange(1, 64)
    return {"kind": kind, "rows": rows, "max_pages": max_pages, "pages": pages, "page": page, "kv_heads": kv_heads, "head_dim": head_dim,
            "layers": layers, "cache": cache, "grow": rng.choice((1, 1, 7, page)) if kind == "resize" else 0, "shared": rng.random() < 0.5}


def _lengths(case):
    """The batch's lengths, the same for every seed: one of the full length, the others uneven between a sixteenth of it and
    it, and, from four sequences on, one of none and one of a single token."""
    n, most = case["rows"], case["max_len"]
    lens = [most] + [max(1, round(most * 16.0 ** -((i * 0.6180339887) % 1.0))) for i in range(1, n)]
    if n >= 4:
        lens[1], lens[2] = 0, 1
    return lens


def _firsts(case, lens):
    """Where a sequence's keys begin: a left-padded prompt's padding is left out."""
    return [length // 7 if case["padded"] and i % 3 == 1 else 0 for i, length in enumerate(lens)]


def _shuffled(values, seed):
    values = list(values)
    random.Random(seed).shuffle(values)
    return values


def _cells(shape, kind, g):
    """Cache contents: values of about one, in 8 bits as codes with a scale for each cell of a head."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16 if kind != "f16" else torch.float16)
    if kind != "e4m3":
        return x, None
    s = 0.25 + torch.rand(shape[:-1], generator=g, device="cuda")
    return (x * 100).clamp(-E4M3_MOST, E4M3_MOST).to(torch.float8_e4m3fn), s / 100


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    if case["kind"] == "norm":
        t = TYPES[case["type"]]
        # a residual stream: a few channels far larger than the others
        x = randn(case["rows"], case["K"])
        x[:, :: 97] *= 20
        s["x"], s["r"] = x.to(t), randn(case["rows"], case["K"]).to(t) if case["residual"] else None
        s["w"] = 1 + 0.1 * randn(case["K"])
        return s
    if case["kind"] in ("resize", "fork", "compact"):
        return _prepare_book(s, case, g, seed)
    H, Hkv, D, page = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    lens = _lengths(case)
    start = case.get("start", 0)
    most_pages = -(-(start + case["max_len"]) // page)
    need = [-(-(start + n) // page) for n in lens]
    total = sum(need) + 3
    lens = _shuffled(lens, seed)
    # pages of a sequence lie anywhere in the pool; table entries past its end are stale
    ids = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    s["tables"] = torch.randint(0, total, (case["rows"], most_pages), generator=g, device="cuda", dtype=torch.int32)
    at, where, which = 0, [], []
    for b, n in enumerate(lens):
        k = -(-(start + n) // page)
        where.append(torch.arange(b * most_pages, b * most_pages + k, device="cuda"))
        which.append(ids[at:at + k])
        at += k
    s["tables"].view(-1)[torch.cat(where)] = torch.cat(which)
    shape = (total, Hkv, page, D)
    if case["kind"] == "attend":
        s["k"], s["k_scale"] = _cells(shape, case["cache"], g)
        s["v"], s["v_scale"] = _cells(shape, case["cache"], g)
        s["lens"] = _ints(lens)
        s["first"] = _ints(_firsts(case, lens)) if case["padded"] else None
        s["q"] = randn(case["rows"], H, D).to(TYPES[case["type"]])
        s["scale"] = 1 / math.sqrt(D)
        s["workspace"] = torch.full((WORKSPACE,), 255, dtype=torch.uint8, device="cuda")
        return s
    s["k"], s["v"] = (torch.zeros(shape, device="cuda").to(TYPES[case["cache"]]) for _ in "kv")
    e4m3 = case["cache"] == "e4m3"
    s["k_scale"], s["v_scale"] = (torch.zeros(shape[:-1], device="cuda") if e4m3 else None for _ in "kv")
    # tokens of the sequences one after the other; every 64th is padding, which belongs to none
    rows = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), torch.tensor(lens, device="cuda"))
    begins = torch.tensor([0] + lens[:-1], device="cuda").cumsum(0)
    T = rows.numel()
    s["positions"] = (start + torch.arange(T, device="cuda") - begins[rows]).to(torch.int32)
    s["rows_of"] = torch.where(torch.arange(T, device="cuda") % 64 == 63, -1, rows).to(torch.int32)
    # the three products' outputs as one stacked product leaves them
    qkv = randn(T, (H + 2 * Hkv) * D).to(TYPES[case["type"]])
    s["q"] = qkv[:, : H * D].view(T, H, D)
    s["new_k"] = qkv[:, H * D: (H + Hkv) * D].view(T, Hkv, D)
    s["new_v"] = qkv[:, (H + Hkv) * D:].view(T, Hkv, D)
    s["cos_sin"] = None
    if case["rope"]:
        half = case["rope"] // 2
        angles = torch.arange(start + case["max_len"], device="cuda").double()[:, None] * \
            10000.0 ** (-torch.arange(half, device="cuda").double() / half)
        s["cos_sin"] = torch.cat((angles.cos(), angles.sin()), 1).float()
    return s


def _book(case):
    """Pages of each row, before: uneven, and no more than half of the pool in all; the same for every seed."""
    n = case["rows"]
    most = min(case["max_pages"] - 2, max(1, case["pages"] // (2 * n)))
    held = [max(1, round(most * (0.35 + 0.65 * ((i * 0.6180339887) % 1.0)))) for i in range(n)]
    if n >= 8:
        held[3] = 0
    return held


def _tails(case, held):
    """Cells used of each row's last page: some pages are full, so that the next token needs a new one."""
    return [case["page"] - (i * 7) % case["page"] if k else 0 for i, k in enumerate(held)]


def _copied(case):
    """Pages that a call copies."""
    held = _book(case)
    if case["kind"] == "compact":
        # of u pages anywhere among the first n, those past the u-th are expected to be u (n - u) / n
        n = min(case["pages"], 2 * sum(held))
        u = sum(k for i, k in enumerate(held) if not case["shared"] or i % 8 != 1)
        return round(u * (n - u) / n)
    if case["kind"] == "resize" and case["shared"]:
        tails = _tails(case, held)
        return 2 * sum(1 for i in range(1, case["rows"], 8) if held[i - 1] and tails[i - 1] < case["page"])
    return 0


def _prepare_book(s, case, g, seed):
    n, page = case["rows"], case["page"]
    held = _book(case)
    tails = _tails(case, held)
    perm = torch.randperm(case["pages"], generator=g, device="cuda").to(torch.int32)
    if case["kind"] == "compact":         # in use: about half of the pages up to twice their number
        perm = torch.randperm(min(case["pages"], 2 * sum(held)), generator=g, device="cuda").to(torch.int32)
    tables = torch.full((n, case["max_pages"]), -1, dtype=torch.int32, device="cuda")
    heldt = _ints(held)
    live = torch.arange(case["max_pages"], device="cuda") < heldt[:, None]
    tables[live] = perm[: sum(held)]
    lens = [max(0, (k - 1) * page + t) for k, t in zip(held, tails)]
    if case["shared"]:                    # every eighth row is a branch of the one before it
        odd = torch.arange(1, n, 8, device="cuda")
        tables[odd] = tables[odd - 1]
        for i in range(1, n, 8):
            lens[i] = lens[i - 1]
    s["tables"], s["lens"] = tables, _ints(lens)
    s["refs"] = torch.bincount(tables[tables >= 0].long(), minlength=case["pages"]).to(torch.int32)
    if case["kind"] == "resize":          # most rows grow, one in sixteen ends, one loses its second half
        s["new_lens"] = _ints([0 if i % 16 == 5 else x // 2 if i % 16 == 7 else min(x + case["grow"], case["max_pages"] * page)
                               for i, x in enumerate(lens)])
    if case["kind"] == "fork":            # half of the rows go on, the others branch from one of them or end
        r = random.Random(seed)
        s["parents"] = _ints([i if r.random() < 0.5 else r.randrange(-1, n) for i in range(n)])
    shape = (case["layers"], case["pages"], case["kv_heads"], page, case["head_dim"])
    s["k"], s["k_scale"] = _cells(shape, case["cache"], g)
    s["v"], s["v_scale"] = _cells(shape, case["cache"], g)
    return s


def _library():
    from paper_2307_03738_amd import binding
    return binding


# --- norm -------------------------------------------------------------------------------------------------------

def _norm(s):
    if own:
        y, h, scales = _library().qg_rms_norm(s["x"], s["w"], EPS, residual=s["r"], dtype=TYPES[s["out"]], group=s["group"])
        return {"y": y, "h": h, "scales": scales}
    h = s["x"].float() + s["r"].float() if s["residual"] else s["x"].float()
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["w"]
    scales = None
    if s["out"] == "e4m3":
        y = y.view(s["rows"], -1, s["group"] or s["K"])
        scales = y.abs().amax(2) / E4M3_MOST
        scales = torch.where(scales == 0, 1.0, scales)
        y = (y / scales[:, :, None]).clamp(-E4M3_MOST, E4M3_MOST).view(s["rows"], s["K"])
    return {"y": y.to(TYPES[s["out"]]), "h": h.to(s["x"].dtype) if s["residual"] else None, "scales": scales}


def _norm_exact(s):
    h = s["x"].double()
    if s["residual"]:
        h = h + s["r"].double()
    y = s["w"].double() * h / (h.pow(2).sum(-1, keepdim=True) / s["K"] + EPS).sqrt()
    scales = None
    if s["out"] == "e4m3":
        parts = y.unflatten(1, (-1, s["group"] or s["K"]))
        scales = torch.linalg.vector_norm(parts, ord=math.inf, dim=-1) / E4M3_MOST
        scales[scales == 0] = 1
        y = (parts / scales.unsqueeze(-1)).flatten(1)
    return {"y": y, "h": h if s["residual"] else None, "scales": scales}


# --- writing the cache ------------------------------------------------------------------------------------------

def _turn(x, cos, sin, interleaved):
    r = 2 * cos.shape[-1]
    turned, rest = x[..., :r], x[..., r:]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if interleaved else (turned[..., : r // 2], turned[..., r // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    return torch.cat((torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1), rest), -1)


def _store(cells, scales, page, slot, x):
    if scales is not None:
        s = x.abs().amax(-1) / E4M3_MOST
        s = torch.where(s == 0, 1.0, s)
        scales[page, :, slot] = s
        x = (x / s[..., None]).clamp(-E4M3_MOST, E4M3_MOST)
    if cells.dtype == torch.float8_e4m3fn:
        cells.view(torch.uint8)[page, :, slot] = x.to(cells.dtype).view(torch.uint8)
    else:
        cells[page, :, slot] = x.to(cells.dtype)


def _append(s):
    if own:
        q = _library().qg_kv_append(s["k"], s["v"], s["tables"], s["rows_of"], s["positions"], s["new_k"], s["new_v"], q=s["q"],
                                    cos_sin=s["cos_sin"], interleaved=s["interleaved"], k_scale=s["k_scale"], v_scale=s["v_scale"])
    else:
        q, k, v = s["q"].float(), s["new_k"].float(), s["new_v"].float()
        at = s["positions"].long()
        if s["rope"]:
            cos, sin = s["cos_sin"][at, None].chunk(2, -1)
            q, k = _turn(q, cos, sin, s["interleaved"]), _turn(k, cos, sin, s["interleaved"])
        real = s["rows_of"] >= 0
        q = torch.where(real[:, None, None], q, 0.0).to(s["q"].dtype)
        at = at[real]
        page = s["tables"][s["rows_of"][real].long(), at // s["page"]].long()
        _store(s["k"], s["k_scale"], page, at % s["page"], k[real])
        _store(s["v"], s["v_scale"], page, at % s["page"], v[real])
    return {"q": q, "k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _append_exact(s):
    H, Hkv, D, r, page = s["heads"], s["kv_heads"], s["head_dim"], s["rope"], s["page"]
    both = torch.cat((s["q"], s["new_k"]), 1).double()
    if r:
        c, n = s["cos_sin"].double()[s["positions"].long()].split(r // 2, 1)
        turn = torch.complex(c, n)[:, None]
        order = torch.arange(r, device="cuda").view(-1, 2) if s["interleaved"] else torch.arange(r, device="cuda").view(2, -1).t()
        pairs = torch.view_as_complex(both[:, :, order].contiguous())
        both[:, :, order] = torch.view_as_real(pairs * turn)
    gone = (s["rows_of"] < 0).nonzero()[:, 0]
    out = {"q": both[:, :H].index_fill(0, gone, 0.0)}
    kept = (s["rows_of"] >= 0).nonzero()[:, 0]
    at = s["positions"].long().index_select(0, kept)
    cell = s["tables"].flatten().long()[s["rows_of"].long()[kept] * s["tables"].shape[1] + torch.div(at, page, rounding_mode="floor")]
    cell = (cell[:, None] * Hkv + torch.arange(Hkv, device="cuda")) * page + at.remainder(page)[:, None]
    for name, x in (("k", both[:, H:]), ("v", s["new_v"].double())):
        x = x.index_select(0, kept).reshape(-1, D)
        cells = s[name].double().reshape(-1, D)
        out[name + "_scale"] = None
        if s[name + "_scale"] is not None:
            scale = torch.linalg.vector_norm(x, ord=math.inf, dim=1) / E4M3_MOST
            scale[scale == 0] = 1
            out[name + "_scale"] = s[name + "_scale"].double().flatten().index_copy(0, cell.flatten(), scale).view(s[name + "_scale"].shape)
            x = x / scale[:, None]
        out[name] = cells.index_copy(0, cell.flatten(), x).view(s[name].shape)
    return out


# --- reading it -------------------------------------------------------------------------------------------------

def _attend(s):
    if own:
        out, lse = _library().qg_paged_attention(s["q"], s["k"], s["v"], s["tables"], s["lens"], s["scale"], first=s["first"],
                                                 window=s["window"], k_scale=s["k_scale"], v_scale=s["v_scale"], lse=True,
                                                 workspace=s["workspace"])
        return {"out": out, "lse": lse}
    B, H, Hkv, D = s["rows"], s["heads"], s["kv_heads"], s["head_dim"]
    tables = s["tables"].long()
    keys = torch.arange(tables.shape[1] * s["page"], device="cuda")
    begin = torch.zeros_like(s["lens"]) if s["first"] is None else s["first"]
    if s["window"]:
        begin = torch.maximum(begin, s["lens"] - s["window"])
    seen = ((keys >= begin[:, None]) & (keys < s["lens"][:, None]))[:, None, :, None]         # [B][1][keys][1]

    def cells(pool, scale):
        x = pool.view(torch.uint8)[tables].view(pool.dtype).float() if scale is not None else pool[tables].float()
        if scale is not None:
            x = x * scale[tables][..., None]
        return torch.where(seen, x.transpose(1, 2).reshape(B, Hkv, -1, D), 0.0)

    q = s["q"].float().view(B, Hkv, H // Hkv, D)
    score = torch.matmul(q, cells(s["k"], s["k_scale"]).transpose(2, 3).contiguous()) * s["scale"]
    score = torch.where(seen.transpose(2, 3), score, -math.inf)
    most = score.amax(3, keepdim=True)
    p = torch.exp(score - torch.where(most == -math.inf, 0.0, most))
    total = p.sum(3, keepdim=True)
    out = torch.matmul(p, cells(s["v"], s["v_scale"])) / torch.where(total == 0, 1.0, total)
    return {"out": out.view(B, H, D).to(s["q"].dtype), "lse": (most + torch.log(total)).view(B, H)}


def _attend_exact(s):
    H, Hkv, D, page = s["heads"], s["kv_heads"], s["head_dim"], s["page"]
    out = torch.zeros(s["rows"], H, D, dtype=torch.float64, device="cuda")
    lse = torch.full((s["rows"], H), -math.inf, dtype=torch.float64, device="cuda")
    lens = s["lens"].tolist()
    firsts = s["first"].tolist() if s["padded"] else [0] * len(lens)
    for b, (length, first) in enumerate(zip(lens, firsts)):
        if s["window"]:
            first = max(first, length - s["window"])
        if first >= length:
            continue
        at = torch.arange(first, length, device="cuda")
        row = s["tables"][b].long()[at // page] * page + at % page
        for h in range(Hkv):
            def head(pool, scale):
                x = pool[:, h].contiguous().view(-1, D)
                x = (x.view(torch.uint8)[row].view(x.dtype) if x.dtype == torch.float8_e4m3fn else x[row]).double()
                return x if scale is None else x * scale[:, h].reshape(-1)[row, None].double()
            heads = slice(h * (H // Hkv), (h + 1) * (H // Hkv))
            score = s["scale"] * (head(s["k"], s["k_scale"]) @ s["q"][b, heads].double().t())          # [keys][heads]
            lse[b, heads] = torch.logsumexp(score, 0)
            out[b, heads] = torch.softmax(score, 0).t() @ head(s["v"], s["v_scale"])
    return {"out": out, "lse": lse}


# --- the pages' book --------------------------------------------------------------------------------------------

def _planes(s):
    return [s[name] for name in ("k", "v", "k_scale", "v_scale") if s[name] is not None]


def _move(s, source, target):
    for plane in _planes(s):
        plane = plane.view(torch.uint8) if plane.dtype == torch.float8_e4m3fn else plane
        plane[:, target] = plane[:, source]


def _count(pages, n):
    """How often each page from 0 to n - 1 is named."""
    return torch.zeros(n + 1, dtype=torch.int32, device="cuda").scatter_add_(
        0, torch.where(pages < 0, n, pages).flatten().long(), torch.ones_like(pages).flatten())[:n]


def _resize(s):
    if own:
        tables, lens, refs, short = _library().qg_pages_resize(s["tables"], s["lens"], s["refs"], s["page"], s["new_lens"], planes=_planes(s))
        return {"tables": tables, "lens": lens, "refs": refs, "short": short}
    page, old, new = s["page"], s["lens"], s["new_lens"]
    column = torch.arange(s["max_pages"], device="cuda")
    had, has = (old + page - 1) // page, (new + page - 1) // page
    dropped = (column >= has[:, None]) & (column < had[:, None])
    refs = s["refs"] - _count(torch.where(dropped, s["tables"], -1), s["pages"])
    tables = torch.where(dropped, -1, s["tables"])
    # the last page of a row that grows inside it, where others hold it too
    last = (column == (had - 1)[:, None]) & ((new > old) & (old % page != 0))[:, None]
    copied = last & (refs[tables.clamp(min=0).long()] > 1)
    wanted = copied | ((column >= had[:, None]) & (column < has[:, None]))
    free = (refs == 0).nonzero()[:, 0]
    rank = wanted.flatten().int().cumsum(0).view(wanted.shape) - 1
    short = (wanted.sum() - free.numel()).clamp(min=0).int().view(1)         # none here: the pools have pages enough
    source = tables[copied].long()
    tables[wanted] = free[rank[wanted].long()].int()
    refs = refs - _count(source.int(), s["pages"]) + _count(torch.where(wanted, tables, -1), s["pages"])
    _move(s, source, tables[copied].long())
    return {"tables": tables, "lens": new.clone(), "refs": refs, "short": short}


def _fork(s):
    if own:
        tables, lens, refs = _library().qg_pages_fork(s["tables"], s["lens"], s["refs"], s["parents"])
        return {"tables": tables, "lens": lens, "refs": refs}
    kept = (s["parents"] >= 0)
    rows = s["parents"].clamp(min=0).long()
    tables = torch.where(kept[:, None], s["tables"][rows], -1)
    lens = torch.where(kept, s["lens"][rows], 0)
    return {"tables": tables, "lens": lens, "refs": s["refs"] - _count(s["tables"], s["pages"]) + _count(tables, s["pages"])}


def _compact(s):
    if own:
        tables, refs, live = _library().qg_pages_compact(s["tables"], s["refs"], planes=_planes(s))
    else:
        used = s["refs"] > 0
        live = used.sum().int().view(1)
        above = torch.arange(s["pages"], device="cuda") >= live
        source = (used & above).nonzero()[:, 0]
        target = (~used & ~above).nonzero()[:, 0]
        to = torch.arange(s["pages"], dtype=torch.int32, device="cuda")
        to[source] = target.int()
        tables = torch.where(s["tables"] >= 0, to[s["tables"].clamp(min=0).long()], -1)
        refs = s["refs"].clone()
        refs[target] = refs[source]
        refs[source] = 0
        _move(s, source, target)
    return {"tables": tables, "refs": refs, "live": live}


def run(state):
    kind = state["kind"]
    if kind in ("resize", "compact"):
        return {**(_resize if kind == "resize" else _compact)(state), **dict(zip(("p0", "p1", "p2", "p3"), _planes(state)))}
    return {"norm": _norm, "append": _append, "attend": _attend, "fork": _fork}[kind](state)


def exact(case, seed):
    kind = case["kind"]
    if kind in ("resize", "fork", "compact"):
        return None                       # whole numbers, and pages as they are
    if kind == "attend" and sum(_lengths(case)) * case["kv_heads"] * case["head_dim"] > 1 << 29:
        return None                       # too slow
    return {"norm": _norm_exact, "append": _append_exact, "attend": _attend_exact}[kind](prepare(case, seed))


def work(case):
    kind = case["kind"]
    if kind == "norm":
        n = case["rows"] * case["K"]
        scales = 4 * n // (case["group"] or case["K"]) if case["out"] == "e4m3" else 0
        return {"bytes": n * (BYTES[case["type"]] * (3 if case["residual"] else 1) + BYTES[case["out"]]) + scales + 4 * case["K"], "flops": 5 * n}
    if kind in ("resize", "fork", "compact"):
        cell = case["kv_heads"] * case["page"] * (case["head_dim"] * BYTES[case["cache"]] + (4 if case["cache"] == "e4m3" else 0))
        book = 2 * 4 * (case["rows"] * case["max_pages"] + case["rows"] + case["pages"])
        return {"bytes": book + 2 * _copied(case) * 2 * case["layers"] * cell, "flops": 0}
    H, Hkv, D = case["heads"], case["kv_heads"], case["head_dim"]
    cell = 2 * Hkv * (D * BYTES[case["cache"]] + (4 if case["cache"] == "e4m3" else 0))       # of one token, k and v
    lens = _lengths(case)
    size = BYTES[case["type"]]
    if kind == "append":
        T = sum(lens)
        return {"bytes": T * (size * (2 * H + 2 * Hkv) * D + cell + 4 * case["rope"] + 8), "flops": T * 3 * case["rope"] * (H + Hkv)}
    keys = sum(max(0, min(n - f, case["window"] or n)) for n, f in zip(lens, _firsts(case, lens)))
    return {"bytes": keys * cell + case["rows"] * H * (2 * D * size + 4) + 4 * (keys // case["page"]), "flops": 4 * keys * H * D}

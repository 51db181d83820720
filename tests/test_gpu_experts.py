"""A layer of experts -- choice, order, products, sum -- against plain implementations in 64 bits.

Tolerances (U = 2^-24, the unit roundoff of fp32), set before any of these ran:
  weights   a score is computed in 64 bits and rounded once: U of it (2 U: the scale's product may be rounded before).
  product   with A = sum |What x|: the terms of a group of G add up, then K / G groups and at most 16 wavefronts' parts, in fp32, where a matrix
            instruction's additions may be cut off instead of rounded (2 U each): 2 (G + K / G + 16) U A; x may go in as parts that
            leave out 2^-22 of it, and 2^-39 of its row's largest.
  gated     silu' is at most 1.1 and silu is off by 8 U of itself (exp by 4 U of its own).
  sum       top_k + 1 fused multiply-adds: (top_k + 2) U sum |w y|.
  storing   half a unit of the type's last place: U, 2^-8 (bf16), 2^-11 (f16) of the value, and half of the smallest step.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
REL = {F32: U, BF16: 2.0 ** -8, F16: 2.0 ** -11}
STEP = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -25}
INF = math.inf


@pytest.fixture(scope="module")
def qg():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2307_03738_amd import binding
    binding.lib()
    return binding


def case(*what):
    print("[case]", *what, flush=True)


def near(got, want, slack, dtype):
    err = (got.double() - want).abs()
    bound = slack + (want.abs() + slack) * REL[dtype] + STEP[dtype]
    # from max + half of its last place on, max (1 + eps / 4) at least, values are rounded to infinity
    over = (want.abs() + slack >= torch.finfo(dtype).max * (1 + torch.finfo(dtype).eps / 4)) & (got.double() == want.sign() * INF)
    err = torch.where(over, 0.0, err)
    worst = (err - bound).max().item() if err.numel() else -1.0
    assert not torch.isnan(err).any() and worst <= 0, f"off by {worst:.3e} more than allowed; largest error {err.max().item():.3e}"


def gen(seed):
    return torch.Generator().manual_seed(seed)


# --- choice -----------------------------------------------------------------------------------------------------

def plain_route(logits, k, bias, score, groups, top_groups, best, renormalise, scale):
    """Ids and weights, token by token."""
    E = logits.shape[1]
    ids, weights = [], []
    for l in logits.double():
        bad = torch.isnan(l) | (torch.isnan(bias) if bias is not None else False)
        off = (l == -INF) | bad | ((bias == -INF) if bias is not None else False)
        nan = bool((bad & (l != -INF)).any())
        l = torch.where(torch.isnan(l), -INF, l)
        if score == "sigmoid":
            p = 1 / (1 + torch.exp(-l))
        else:
            most = l.max()
            e = (l == INF).double() if most == INF else torch.where(l == -INF, 0.0, torch.exp(l - (0 if most == -INF else most)))
            p = e / e.sum() if e.sum() > 0 else e
        value = p if bias is None else p + bias.double()
        key = [(-INF if off[i] else float(l[i] if bias is None else value[i])) for i in range(E)]
        if top_groups < groups:
            size, rank = E // groups, []
            for g in range(groups):
                at = range(g * size, (g + 1) * size)
                if best == 2:
                    v = sorted((float(value[i]) for i in at if not off[i]), reverse=True)[:2]
                    rank.append(sum(v) if v else -INF)
                else:
                    rank.append(max(key[i] for i in at))
            kept = sorted(range(groups), key=lambda g: (-rank[g], g))[:top_groups]
            key = [key[i] if i // size in kept else -INF for i in range(E)]
        order = [i for i in sorted(range(E), key=lambda i: (-key[i], i)) if key[i] > -INF][:k]
        w = [float(p[i]) for i in order]
        if renormalise and sum(w) > 0:
            w = [v / sum(w) for v in w]
        ids.append(order + [-1] * (k - len(order)))
        weights.append([math.nan] * k if nan else [v * scale for v in w] + [0.0] * (k - len(w)))
    return torch.tensor(ids, dtype=torch.int32), torch.tensor(weights, dtype=torch.float64)


ROUTES = [
    # tokens, experts, k, type, score, bias, groups, top groups, best, renormalise, scale, gap between rows
    (1, 64, 6, F32, "softmax", False, 1, 1, 1, True, 1.0, 0),
    (1, 1, 1, F32, "softmax", False, 1, 1, 1, True, 1.0, 0),
    (1, 2, 2, BF16, "sigmoid", True, 1, 1, 1, False, 2.5, 0),
    (37, 192, 7, BF16, "sigmoid", True, 12, 4, 2, True, 1.0, 0),
    (19, 96, 8, F16, "softmax", True, 8, 3, 2, False, 0.5, 3),
    (21, 96, 8, F32, "sigmoid", False, 8, 3, 2, True, 1.0, 1),
    (33, 60, 5, F32, "softmax", False, 12, 2, 1, True, 1.0, 4),
    (17, 130, 20, F32, "softmax", True, 1, 1, 1, True, 1.0, 0),
    (9, 511, 33, BF16, "softmax", False, 1, 1, 1, False, 1.0, 0),
    (5, 1024, 64, F32, "sigmoid", True, 128, 9, 2, True, 1.0, 0),
    (4, 1000, 12, F16, "softmax", False, 1000, 12, 1, True, 1.0, 8),
    (6, 1024, 5, F32, "softmax", True, 1024, 9, 2, True, 1.0, 0),
    (7, 256, 32, BF16, "sigmoid", True, 256, 40, 1, False, 1.0, 0),
    (300, 8, 8, F16, "softmax", False, 1, 1, 1, True, 1.0, 0),
    (65, 16, 4, F32, "sigmoid", False, 4, 4, 2, False, 3.0, 0),
]


@pytest.mark.parametrize("tokens,experts,k,dt,score,bias,groups,top_groups,best,renormalise,scale,gap", ROUTES)
def test_route_matches_64_bits(qg, tokens, experts, k, dt, score, bias, groups, top_groups, best, renormalise, scale, gap):
    case("route", tokens, experts, k, dt, score, bias, groups, top_groups, best)
    g = gen(tokens + 7 * experts + k)
    full = (2 * torch.randn(tokens, experts + gap, generator=g)).to(dt)
    if tokens > 3:
        full[1] = -INF                                    # padding
        full[2, : experts // 2 + 1] = -INF
        full[3, : experts // 3] = full[3, experts - experts // 3: experts].clone()     # ties
    logits = full[:, :experts]
    b = 0.3 * torch.randn(experts, generator=g) if bias else None
    ids, weights = qg.qg_route(full.cuda()[:, :experts], k, bias=None if b is None else b.cuda(), score=score, groups=groups, top_groups=top_groups, group_best=best,
                               renormalise=renormalise, scale=scale)
    want, w = plain_route(logits, k, b, score, groups, top_groups, best, renormalise, scale)
    assert torch.equal(ids.cpu(), want)
    near(weights.cpu(), w, 2 * U * w.abs(), F32)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [False, True])
def test_route_of_values_that_are_no_numbers(qg, score, bias):
    logits = torch.randn(9, 12, generator=gen(3))
    logits[0, 3] = math.nan
    logits[1] = math.nan
    logits[2, 4] = INF
    logits[3, [4, 7]] = INF
    logits[4] = -INF
    logits[5, :11] = -INF
    logits[6] = torch.finfo(F32).min
    logits[7] = 1e30
    b = 0.1 * torch.randn(12, generator=gen(4)) if bias else None
    for groups, top in ((1, 1), (4, 2)):
        ids, w = qg.qg_route(logits.cuda(), 4, bias=None if b is None else b.cuda(), score=score, groups=groups, top_groups=top)
        want, ww = plain_route(logits, 4, b, score, groups, top, 1, True, 1.0)
        assert torch.equal(ids.cpu(), want)
        assert torch.equal(torch.isnan(w.cpu()), torch.isnan(ww))
        near(w.cpu().nan_to_num(0), ww.nan_to_num(0), 2 * U, F32)
    if bias:
        b[2], b[5] = -INF, math.nan
        ids, w = qg.qg_route(logits.cuda(), 4, bias=b.cuda(), score=score)
        assert not ((ids == 2) | (ids == 5)).any()


@pytest.mark.parametrize("score,renormalise", [("softmax", True), ("softmax", False), ("sigmoid", False)])
@pytest.mark.parametrize("bias", [False, True])
def test_route_of_every_magnitude(qg, score, renormalise, bias):
    # exponentials from 1 to what 64 bits do not hold, of 40 experts all chosen, and of equal, huge and tiny logits
    case("route magnitudes", score, renormalise, bias)
    row = torch.tensor([0.0, 1e-40, -1e-40, 2.0 ** -24, 1e-3, 0.3465735, -0.3465736, 0.69314718, 1.0, -1.0, 5.5, -5.5, 16.6, -16.6, 37.0, -37.0, 87.3, -87.3, 88.8, -88.8, -103.9, -104.1,
                        300.0, -300.0, 708.0, -708.0, -745.0, 746.0, -801.0, 1e4, -1e4, 3e38, -3e38, 2.0, 2.0, 3.25, -3.25, 10.0, -10.0, 0.125])
    logits = torch.stack([row, row.clamp(-60, 60), row.clamp(-1, 1), torch.full((40,), -3e38), torch.full((40,), 7.0), row.clamp(max=0)])
    b = 0.3 * torch.randn(40, generator=gen(3)) if bias else None
    ids, weights = qg.qg_route(logits.cuda(), 40, bias=None if b is None else b.cuda(), score=score, renormalise=renormalise)
    want, w = plain_route(logits, 40, b, score, 1, 1, 1, renormalise, 1.0)
    assert torch.equal(ids.cpu(), want)
    near(weights.cpu(), w, 2 * U * w.abs(), F32)


def test_sigmoids_that_tie_rank_by_their_logits(qg):
    logits = torch.tensor([[50.0, 60.0, 40.0, 70.0, 45.0, 38.0, 80.0, 39.0]])
    ids, w = qg.qg_route(logits.cuda(), 4, score="sigmoid", groups=2, top_groups=2, group_best=2)
    assert ids.tolist() == [[6, 3, 1, 0]] and w.tolist() == [[0.25] * 4]
    ids, _ = qg.qg_route(logits.cuda(), 3, score="sigmoid", groups=2, top_groups=1, group_best=2)
    assert ids.tolist() == [[3, 1, 0]]                    # both groups' sums are 2: the lower one, its experts by their logits


# --- order ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("tokens,k,experts", [(1, 1, 1), (1, 8, 8), (48, 4, 32), (1000, 3, 7), (2049, 1, 192), (5000, 8, 1024), (3000, 4, 963), (1100, 15, 1000), (40000, 2, 3), (70001, 8, 100)])
def test_plan_is_a_stable_sort(qg, tokens, k, experts):
    case("plan", tokens, k, experts)
    g = gen(tokens + k)
    ids = torch.randint(-1, experts + 1, (tokens, k), generator=g, dtype=torch.int32)
    ids[::7] = experts // 2
    ids[tokens // 2] = torch.tensor([-(1 << 31), (1 << 31) - 1] * k, dtype=torch.int32)[:k]
    offsets, slot_tokens, slots = (t.cpu() for t in qg.qg_expert_plan(ids.cuda(), experts))
    flat = torch.where((ids >= 0) & (ids < experts), ids, experts).flatten().long()
    by, order = flat.sort(stable=True)
    count = torch.bincount(flat, minlength=experts + 1)[:experts]
    assert offsets.tolist() == [0] + count.cumsum(0).tolist()
    assert torch.equal(slot_tokens, torch.where(by < experts, order // k, -1).int())
    want = torch.empty(tokens * k, dtype=torch.int32)
    want[order] = torch.where(by < experts, torch.arange(tokens * k), -1).int()
    assert torch.equal(slots.flatten(), want)


def test_plan_of_no_tokens(qg):
    offsets, slot_tokens, slots = qg.qg_expert_plan(torch.empty(0, 4, dtype=torch.int32, device="cuda"), 5)
    assert offsets.tolist() == [0] * 6 and slot_tokens.numel() == 0 and slots.shape == (0, 4)


# --- products ---------------------------------------------------------------------------------------------------

def blobs(qg, E, N, K, bits, group, seed, spread=0):
    """(packed [E][bytes] with rows `spread` bytes further apart, dequantized matrices in 64 bits)"""
    g = gen(seed)
    q = torch.randint(0, 2 ** bits, (E, N, K), generator=g, dtype=torch.uint8)
    s = (0.5 + torch.rand(E, N, K // group, generator=g)) / math.sqrt(K)
    s[:, ::5] *= 1e-3
    z = torch.randint(0, 2 ** bits, (E, N, K // group), generator=g, dtype=torch.uint8)
    nbytes = qg.qg_packed_bytes(N, K, bits, group)
    packed = torch.full((E, nbytes + spread), 255, dtype=torch.uint8, device="cuda")
    for e in range(E):
        packed[e, :nbytes] = qg.qg_pack(q[e].cuda(), s[e].cuda(), z[e].cuda(), bits, group)[:nbytes]
    wide = lambda t: t.double().repeat_interleave(group, 2)  # noqa: E731
    return packed[:, :nbytes] if spread else packed, wide(s) * (q.double() - wide(z))


def product_want(W, x, offsets, rows, gated, group):
    """(y, slack) of the slots that offsets name."""
    E, N, K = W.shape
    slots = offsets[-1]
    y = torch.zeros(slots, N // 2 if gated else N, dtype=torch.float64)
    slack = torch.zeros_like(y)
    xd = x.cpu().double()
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        if a == b:
            continue
        take = torch.arange(a, b) if rows is None else rows[a:b].long()
        real = (take >= 0) & (take < len(xd))
        xe = torch.where(real[:, None], xd[take.clamp(0, len(xd) - 1)], 0.0)
        out, A = xe @ W[e].t(), xe.abs() @ W[e].abs().t()
        err = (2 * (group + K / group + 16) * U + 2.0 ** -22) * A + 2.0 ** -39 * xe.abs().amax(1, keepdim=True) * W[e].abs().sum(1)
        if gated:
            gate, up = out.chunk(2, 1)
            eg, eu = err.chunk(2, 1)
            sil = gate / (1 + torch.exp(-gate))
            out, err = sil * up, 1.1 * eg * (up.abs() + eu) + sil.abs() * eu + 10 * U * (sil * up).abs()
        y[a:b], slack[a:b] = out, err
    return y, slack


def offsets_of(counts):
    return [0] + torch.tensor(counts).cumsum(0).tolist()


ODD = [0, 1, 5, 0, 17, 2]
PRODUCTS = [
    # N, K, bits, group, slots of each expert, gated, x type, y type, rows given, gap between rows of x
    (64, 128, 4, 128, [1], False, F32, F32, False, 0),
    (1, 32, 4, 32, [1, 0], False, F32, F32, False, 0),
    (2, 64, 2, 32, [0, 1, 3], True, F32, BF16, True, 0),
    (130, 256, 4, 64, ODD, False, F32, F32, True, 8),
    (130, 256, 4, 64, ODD, True, BF16, BF16, True, 8),
    (130, 256, 4, 32, ODD, True, F16, F16, True, 8),
    (96, 384, 3, 128, ODD, False, F16, F32, False, 0),
    (97, 480, 3, 96, ODD, False, BF16, F16, True, 0),
    (70, 352, 3, 32, ODD, False, F32, F32, True, 16),
    (70, 352, 2, 32, ODD, False, BF16, F32, True, 16),
    (258, 192, 2, 64, ODD, True, F16, BF16, False, 0),
    (129, 640, 2, 128, ODD, False, F32, F32, True, 0),
    (66, 96, 4, 96, ODD, True, F32, F32, True, 0),
    (100, 1024, 4, 1024, ODD, False, F32, F32, True, 0),
    (100, 512, 3, 256, ODD, False, F16, F16, True, 0),
    (64, 72, 4, 8, ODD, False, F32, F32, True, 0),
    (66, 80, 4, 16, ODD, True, BF16, BF16, True, 0),
    (64, 48, 2, 16, ODD, False, F16, F32, True, 0),
    (64, 240, 4, 40, ODD, False, BF16, F32, False, 0),
    (200, 1408, 3, 64, [3] * 33, False, F32, F32, False, 0),
    (320, 2048, 4, 32, [7, 0, 90, 33, 1, 16], True, BF16, BF16, True, 0),
    (320, 1024, 4, 128, [700, 0, 3, 130, 64, 65], True, BF16, BF16, True, 0),
    (322, 1056, 2, 32, [300, 1, 129], True, F16, F16, True, 8),
    (300, 1056, 3, 32, [128, 257, 0], False, F32, F32, True, 0),
    (260, 1792, 2, 64, [140, 120, 0, 150], False, F16, F16, False, 0),
    (514, 1280, 4, 64, [255, 400], True, F32, F32, True, 0),
    (256, 768, 3, 128, [513], False, BF16, F32, True, 0),
    (2050, 160, 4, 32, [200], False, F32, BF16, True, 0),
]

# wide matrices and rows enough for the tiles of 64 and of 32 slots, every width, scales for 32, 64, 128 k and odd numbers of 32, K that ends inside 128
WIDE = [
    (5130, 160, 4, 32, [300, 419], False, F32, F32, True, 0),
    (2570 * 2, 352, 4, 32, [419, 300, 1], True, BF16, BF16, True, 8),
    (5130, 320, 4, 64, [419, 300], False, F16, F32, False, 0),
    (2562 * 2, 192, 4, 64, [300, 419], True, F32, F32, True, 0),
    (5130, 384, 4, 128, [129, 600], False, BF16, F32, True, 0),
    (5130, 256, 4, 256, [129, 600], False, F32, F16, True, 0),
    (5130, 288, 4, 96, [129, 600], False, F16, F16, True, 0),
    (5130, 384, 4, 192, [129, 600], False, BF16, BF16, True, 0),
    (5130, 160, 3, 32, [300, 419], False, F32, F32, True, 0),
    (5130, 320, 3, 64, [300, 419], False, BF16, F32, True, 0),
    (2562 * 2, 384, 3, 128, [300, 419], True, F16, F16, True, 0),
    (5130, 160, 2, 32, [300, 419], False, F16, F32, True, 0),
    (5130, 320, 2, 64, [300, 419], False, F32, BF16, True, 0),
    (2562 * 2, 384, 2, 128, [300, 419], True, BF16, F32, True, 0),
    (5130, 288, 2, 96, [300, 419], False, F32, F32, False, 0),
    (7170, 160, 4, 32, [40, 33, 0, 64, 31], False, F32, F32, True, 0),
    (3590 * 2, 192, 4, 64, [40, 33, 0, 64, 31], True, BF16, BF16, True, 0),
    (7170, 384, 4, 128, [40, 33, 2, 64, 31], False, F16, F32, True, 0),
    (7170, 192, 4, 96, [40, 33, 2, 64, 31], False, BF16, F32, True, 0),
    (7170, 160, 3, 32, [40, 33, 2, 64, 31], False, BF16, F16, True, 0),
    (7170, 192, 3, 64, [40, 33, 2, 64, 31], False, F32, F32, True, 0),
    (7170, 384, 3, 384, [40, 33, 2, 64, 31], False, F16, F32, True, 0),
    (7170, 160, 2, 32, [40, 33, 2, 64, 31], False, F32, F32, True, 0),
    (3590 * 2, 192, 2, 64, [40, 33, 2, 64, 31], True, F16, F16, True, 0),
    (7170, 256, 2, 128, [40, 33, 2, 64, 31], False, BF16, F32, True, 0),
]
# many experts of few rows: workgroups of four wavefronts, one, two and four tiles of outputs each, with and without a conversion of rows of its own
def some(E, often, most):
    return [(7 * e * e + e) % (most + 1) if e % often == 0 else 0 for e in range(E)]


FEW = [
    (2050, 160, 4, 32, some(24, 1, 7), False, F32, F32, True, 0),
    (2050 * 2, 192, 4, 64, some(24, 1, 12), True, BF16, BF16, True, 8),
    (2050, 288, 4, 96, some(24, 1, 9), False, F16, F32, True, 0),
    (2050, 256, 4, 128, some(60, 1, 5), False, F32, F32, True, 0),
    (2050, 96, 3, 32, some(60, 1, 5), False, BF16, F32, True, 0),
    (1030 * 2, 192, 3, 64, some(60, 1, 5), True, F32, F32, True, 0),
    (2050, 128, 3, 128, some(100, 1, 5), False, F16, F16, False, 0),
    (1030 * 2, 96, 2, 32, some(100, 1, 5), True, F32, F32, True, 0),
    (2050, 192, 2, 64, some(100, 1, 5), False, BF16, F32, True, 0),
    (2050, 96, 2, 96, some(24, 1, 9), False, F32, F32, True, 0),
    (2050, 352, 4, 32, some(60, 3, 2), False, F32, F32, True, 8),
    (1030 * 2, 192, 4, 64, some(60, 3, 2), True, BF16, F32, True, 8),
    (2050, 256, 4, 128, some(60, 4, 3), False, F16, F32, True, 0),
    (2050, 160, 3, 32, some(60, 4, 3), False, F32, BF16, True, 0),
    (2050, 288, 3, 96, some(60, 4, 3), False, BF16, F32, False, 0),
    (2050, 160, 2, 32, some(60, 4, 3), False, F32, F32, True, 0),
    (1030 * 2, 320, 2, 64, some(60, 4, 3), True, F16, F16, True, 0),
    (1290, 192, 4, 64, some(130, 1, 60), False, BF16, F32, True, 0),              # many experts of many rows
    (645 * 2, 128, 2, 32, some(70, 1, 300), True, F32, F32, True, 8),
    (300, 384, 3, 128, some(200, 3, 500), False, F16, F32, True, 0),
    (64, 9600, 4, 128, [0, 1, 0, 0, 2, 0, 0, 0], False, F32, F32, True, 0),       # rows too long for a workgroup's own conversion of two
    (64, 4992, 2, 64, [0, 1, 0, 0, 2, 0, 0, 1], False, F32, F32, True, 0),        # ... of three
]


# workgroups for less than a round: K in three slices, of different lengths, that end inside 128
SLICED = [
    (5130, 1056, 4, 32, [100, 77], False, F32, F32, True, 8),
    (2570 * 2, 1152, 4, 64, [90, 3, 60], True, BF16, BF16, True, 0),
    (5130, 1280, 4, 128, [33, 120], False, F16, F32, True, 0),
    (5130, 1408, 4, 128, [33, 120], False, F32, F32, True, 0),
    (5130, 1344, 4, 96, [128, 1], False, BF16, F32, False, 0),
    (5130, 1056, 3, 32, [100, 77], False, BF16, F32, True, 0),
    (2570 * 2, 1216, 3, 64, [100, 77], True, F32, F32, True, 8),
    (5130, 1024, 3, 128, [100, 77], False, F16, F16, True, 0),
    (5130, 1120, 2, 32, [100, 77], False, F16, F32, True, 0),
    (2570 * 2, 1600, 2, 64, [100, 77], True, F32, BF16, True, 0),
    (5130, 1024, 2, 256, [100, 77], False, BF16, BF16, True, 8),
]
# groups that are no whole 32 k: pieces of 8 and of 16 k, words of zero-points that end inside 128 k, K that ends inside 32, few rows and many
CELLS = [
    (130, 1000, 4, 8, ODD, False, F32, F32, True, 8),
    (70, 1024, 4, 8, [1, 0, 0, 0], True, BF16, F32, False, 0),
    (2050, 96, 4, 8, some(60, 4, 3), False, F16, F32, True, 0),
    (130, 1104, 4, 24, ODD, True, F16, F16, True, 0),
    (67, 40, 4, 40, [3, 200, 0, 1], False, F32, F32, True, 0),
    (2050, 360, 4, 72, some(24, 1, 12), False, BF16, F32, True, 8),
    (1030 * 2, 176, 4, 88, some(60, 3, 2), True, F32, F32, True, 8),
    (130, 1040, 4, 16, ODD, False, F32, F32, True, 0),
    (130, 1040, 4, 16, [300, 2, 129], True, BF16, BF16, True, 0),
    (2050, 272, 4, 16, some(24, 1, 12), False, F32, F32, True, 0),
    (70, 2064, 4, 48, [1, 0, 1, 0, 0, 0], False, F16, F32, True, 0),
    (2050, 336, 4, 112, some(60, 1, 5), False, BF16, F32, False, 0),
    (130, 1040, 2, 16, ODD, True, F32, F32, True, 8),
    (2050, 272, 2, 16, some(24, 1, 12), False, BF16, F32, True, 0),
    (70, 2064, 2, 16, [1, 0, 0, 0], False, F16, F16, False, 0),
    (1030 * 2, 336, 2, 48, some(60, 4, 3), True, F32, F32, True, 0),
    (130, 1200, 2, 80, [90, 0, 33, 5], False, F16, F32, True, 0),
]


@pytest.mark.parametrize("N,K,bits,group,counts,gated,xt,yt,given,gap", PRODUCTS + WIDE + FEW + SLICED + CELLS)
def test_products_match_64_bits(qg, N, K, bits, group, counts, gated, xt, yt, given, gap):
    case("product", N, K, bits, group, counts[:6], gated, xt, yt, given)
    g = gen(N + K + len(counts))
    packed, W = blobs(qg, len(counts), N, K, bits, group, N * 3 + K, spread=256 if given else 0)
    offsets = offsets_of(counts)
    slots, tokens = offsets[-1] + 5, max(offsets[-1] // 2, 3) if given else offsets[-1] + 5
    x = torch.randn(tokens, K + gap, generator=g)
    x[:, ::17] *= 8
    x[0] *= 1e-6
    x[-1] *= 1e4 if xt is not F16 else 1.0
    x = x.to(xt)
    rows = torch.randint(0, tokens, (slots,), generator=g, dtype=torch.int32) if given else None
    if given:
        rows[0], rows[offsets[-1] - 1] = 0, tokens - 1
        if offsets[-1] > 8:
            rows[3], rows[5] = -1, tokens
    y = torch.full((slots, N // 2 if gated else N), 7.0, dtype=yt, device="cuda")
    out = qg.qg_experts_product(packed, N, K, bits, group, x.cuda()[:, :K], torch.tensor(offsets, dtype=torch.int32).cuda(),
                                rows=None if rows is None else rows.cuda(), gated=gated, y=y)
    assert out is y
    want, slack = product_want(W, x[:, :K], offsets, rows, gated, group)
    near(y[: offsets[-1]].cpu(), want, slack, yt)
    assert (y[offsets[-1]:] == 7).all()                   # behind the last expert's slots
    if given and offsets[-1] > 8:
        assert (y[[3, 5]] == 0).all()


@pytest.mark.parametrize("N,counts", [(96, [1, 0, 0, 2, 0, 0, 0, 0]), (96, [2, 3]), (96, [40, 3]), (96, [300, 9]), (7168, [64, 90]), (5120, [400, 300]), (5120, [100, 77])])
@pytest.mark.parametrize("dt", [F32, BF16, F16])
def test_values_that_are_no_numbers_stay_in_their_rows(qg, N, counts, dt):
    case("nan", N, counts, dt)
    K, group = 1152 if counts == [100, 77] else 256, 64
    packed, W = blobs(qg, len(counts), N, K, 4, group, 5)
    offsets = offsets_of(counts)
    x = torch.randn(offsets[-1], K, generator=gen(1)).to(dt)
    x[1, 5], x[2, 250] = math.nan, INF
    y = qg.qg_experts_product(packed, N, K, 4, group, x.cuda(), torch.tensor(offsets, dtype=torch.int32).cuda()).cpu()
    assert torch.isnan(y[1]).all() and not torch.isfinite(y[2]).any()
    assert torch.isfinite(y[[i for i in range(offsets[-1]) if i not in (1, 2)]]).all()


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("N,count", [(70, 1), (70, 20), (70, 200), (5120, 700)])
def test_rows_of_every_magnitude(qg, dt, N, count):
    # the largest and smallest numbers that leave the result's terms within fp32's range, rows of zeros
    case("magnitudes", dt, N, count)
    K, group = 384, 128
    packed, W = blobs(qg, 1, N, K, 4, group, 9)
    x = torch.randn(count, K, generator=gen(2))
    x *= torch.tensor([2.0 ** e for e in (0, 100, -100, 60, -60, -110)])[torch.arange(count) % 6, None]
    if count > 7:
        x[7] = 0
    x = x.to(dt)
    offsets = [0, count]
    y = qg.qg_experts_product(packed, N, K, 4, group, x.cuda(), torch.tensor(offsets, dtype=torch.int32).cuda(), dtype=F32)
    want, slack = product_want(W, x, offsets, None, False, group)
    near(y.cpu(), want, slack + 2.0 ** -140, F32)         # (sums below the normal numbers may be cut off)


def test_offsets_that_no_plan_makes_stay_in_range(qg):
    N, K, group = 64, 128, 64
    packed, W = blobs(qg, 3, N, K, 4, group, 11)
    x = torch.randn(10, K, generator=gen(3)).cuda()
    for offsets in ([-5, 4, 6, 1 << 30], [3, 1, 9, 2], [20, 30, 40, 50]):
        guard = torch.full((14, N), 7.0, device="cuda")
        qg.qg_experts_product(packed, N, K, 4, group, x, torch.tensor(offsets, dtype=torch.int32).cuda(), y=guard[2:12])
        assert (guard[:2] == 7).all() and (guard[12:] == 7).all()


def test_empty_calls(qg):
    packed, _ = blobs(qg, 2, 64, 128, 4, 64, 1)
    zero = torch.zeros(3, dtype=torch.int32, device="cuda")
    y = qg.qg_experts_product(packed, 64, 128, 4, 64, torch.empty(0, 128, device="cuda"), zero)
    assert y.shape == (0, 64)
    y = torch.full((4, 64), 7.0, device="cuda")
    qg.qg_experts_product(packed, 64, 128, 4, 64, torch.randn(4, 128, device="cuda"), zero, y=y)
    assert (y == 7).all()
    y = qg.qg_experts_product(packed, 64, 128, 4, 64, torch.empty(0, 128, device="cuda"), torch.tensor([0, 1, 3], dtype=torch.int32, device="cuda"),
                              rows=torch.zeros(3, dtype=torch.int32, device="cuda"))
    assert (y == 0).all()                                 # there are no rows: all count as zeros
    out = qg.qg_experts_combine(torch.empty(0, 64, device="cuda"), torch.zeros(2, 1, dtype=torch.int32, device="cuda"), torch.ones(2, 1, device="cuda"))
    assert (out == 0).all()


# --- sum --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("tokens,k,N,dt,ot,residual,gap", [
    (1, 1, 1, F32, F32, False, 0), (24, 4, 4096, F32, F32, False, 0), (33, 8, 5120, BF16, BF16, True, 0), (7, 6, 1408, F16, F32, True, 8), (5, 3, 1001, BF16, BF16, True, 0),
    (9, 2, 66, F16, F16, True, 3), (3, 64, 264, F32, BF16, False, 0), (1000, 2, 64, BF16, F16, True, 8), (2, 5, 20000, F32, F32, True, 4), (6, 7, 4099, F16, F16, False, 0)])
def test_sums_match_64_bits(qg, tokens, k, N, dt, ot, residual, gap):
    case("combine", tokens, k, N, dt, ot, residual, gap)
    g = gen(tokens + N)
    y = torch.randn(tokens * k, N, generator=g).to(dt)
    slots = torch.randperm(tokens * k, generator=g).int().view(tokens, k)
    if tokens > 4:
        slots[1], slots[2, 0], slots[3, 0] = -1, tokens * k, -(1 << 31)
        y[slots[4].long()] = y[slots[4].long()] * 100
    w = torch.rand(tokens, k, generator=g)
    r = torch.randn(tokens, N + gap, generator=g).to(ot) if residual else None
    out = qg.qg_experts_combine(y.cuda(), slots.cuda(), w.cuda(), residual=None if r is None else r.cuda()[:, :N], dtype=ot)
    real = ((slots >= 0) & (slots < tokens * k))[..., None]
    terms = torch.where(real, w.double()[..., None] * y.double()[slots.clamp(0, tokens * k - 1).long()], 0.0)
    base = r[:, :N].double() if residual else torch.zeros(tokens, N, dtype=torch.float64)
    near(out.cpu(), base + terms.sum(1), (k + 2) * U * (base.abs() + terms.abs().sum(1)), ot)


def test_sum_over_the_residual(qg):
    y, r = torch.randn(12, 200, generator=gen(1)).cuda(), torch.randn(6, 200, generator=gen(2)).cuda()
    slots, w = torch.randperm(12, generator=gen(3)).int().view(6, 2).cuda(), torch.rand(6, 2, generator=gen(4)).cuda()
    want = qg.qg_experts_combine(y, slots, w, residual=r)
    assert qg.qg_experts_combine(y, slots, w, residual=r, out=r) is r and torch.equal(r, want)


def test_a_weight_of_zero_does_not_hide_what_is_no_number(qg):
    y = torch.tensor([[1.0], [math.nan]]).cuda()
    out = qg.qg_experts_combine(y, torch.tensor([[0, 1], [0, -1]], dtype=torch.int32).cuda(), torch.tensor([[1.0, 0.0], [1.0, 0.0]]).cuda())
    assert torch.isnan(out[0]).all() and out[1].item() == 1.0


# --- together ---------------------------------------------------------------------------------------------------

def layer(qg, up, down, N, K, bits, group, x, logits, k):
    ids, weights = qg.qg_route(logits, k)
    offsets, tokens, slots = qg.qg_expert_plan(ids, up.shape[0])
    h = qg.qg_experts_product(up, 2 * N, K, bits, group, x, offsets, rows=tokens, gated=True)
    y = qg.qg_experts_product(down, K, N, bits, group, h, offsets)
    return qg.qg_experts_combine(y, slots, weights, residual=x)


def layer_want(Wu, Wd, x, logits, k):
    out = x.double().clone()
    best, ids = logits.double().topk(k, 1)
    w = best.softmax(1)
    for t in range(len(x)):
        for j in range(k):
            if best[t, j] > -INF:
                gate, up = (Wu[ids[t, j]] @ x[t].double()).chunk(2)
                out[t] += w[t, j] * (Wd[ids[t, j]] @ (gate / (1 + torch.exp(-gate)) * up))
    return out


@pytest.mark.parametrize("tokens,bits,group", [(1, 4, 32), (13, 3, 64), (150, 2, 64)])
def test_a_layer_in_a_graph_with_eager_work_between_replays(qg, tokens, bits, group):
    case("layer", tokens, bits, group)
    E, N, K, k = 9, 192, 256, 3
    up, Wu = blobs(qg, E, 2 * N, K, bits, group, 1)
    down, Wd = blobs(qg, E, K, N, bits, group, 2)
    g = gen(tokens)
    x, logits = torch.empty(tokens, K, device="cuda"), torch.empty(tokens, E, device="cuda")

    def fill():
        hx, hl = torch.randn(tokens, K, generator=g), 2 * torch.randn(tokens, E, generator=g)
        hl[:, 4] = -INF
        x.copy_(hx)
        logits.copy_(hl)
        return hx, hl

    fill()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        layer(qg, up, down, N, K, bits, group, x, logits, k)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer(qg, up, down, N, K, bits, group, x, logits, k)
    for _ in range(4):
        hx, hl = fill()
        graph.replay()
        got = out.clone()
        eager = layer(qg, up, down, N, K, bits, group, x, logits, k)
        torch.cuda.synchronize()
        assert torch.equal(got, eager)
        want = layer_want(Wu, Wd, hx, hl, k)
        # two products in fp32 one after the other: their slack is far below 2^-12 of the norm at these sizes
        assert (got.cpu().double() - want).norm() <= 2.0 ** -12 * want.norm()


def test_two_streams_at_once(qg):
    E, N, K = 5, 320, 512
    packed, W = blobs(qg, E, N, K, 4, 64, 7)
    streams, outs, wants = [torch.cuda.Stream() for _ in range(2)], [], []
    for i, st in enumerate(streams):
        counts = [[30, 2, 0, 70, 1], [1, 200, 3, 0, 9]][i]
        offsets = torch.tensor(offsets_of(counts), dtype=torch.int32).cuda()
        x = torch.randn(offsets_of(counts)[-1], K, generator=gen(i)).cuda()
        st.wait_stream(torch.cuda.current_stream())
        outs.append((x, offsets, counts))
    got = []
    for _ in range(5):
        for st, (x, offsets, counts) in zip(streams, outs):
            with torch.cuda.stream(st):
                got.append(qg.qg_experts_product(packed, N, K, 4, 64, x, offsets))
    torch.cuda.synchronize()
    for i, y in enumerate(got):
        x, _, counts = outs[i % 2]
        want, slack = product_want(W, x.cpu(), offsets_of(counts), None, False, 64)
        near(y.cpu(), want, slack, F32)


def test_refused_tensors(qg):
    packed, _ = blobs(qg, 2, 64, 128, 4, 64, 1)
    x, offsets = torch.randn(4, 128).cuda(), torch.tensor([0, 2, 4], dtype=torch.int32).cuda()
    with pytest.raises(ValueError):
        qg.qg_experts_product(packed, 64, 128, 4, 64, x.double(), offsets)
    with pytest.raises(ValueError):
        qg.qg_experts_product(packed, 64, 128, 4, 64, x.t().contiguous().t(), offsets)
    with pytest.raises(ValueError):
        qg.qg_experts_product(packed, 64, 128, 4, 64, x, offsets[:2])
    with pytest.raises(ValueError):
        qg.qg_experts_product(packed, 64, 128, 4, 64, x, offsets, y=torch.empty(4, 63, device="cuda"))
    with pytest.raises(RuntimeError):
        qg.qg_experts_product(packed[:, :100], 64, 128, 4, 64, x, offsets)
    with pytest.raises(RuntimeError):
        qg.qg_experts_product(packed, 64, 128, 4, 64, x[:, :64], offsets)
    with pytest.raises(RuntimeError):
        qg.qg_route(torch.randn(2, 8).cuda(), 9)
    with pytest.raises(ValueError):
        qg.qg_route(torch.randn(2, 8).cuda(), 2, score="relu")
    with pytest.raises(ValueError):
        qg.qg_expert_plan(torch.zeros(2, 2, dtype=torch.int64, device="cuda"), 4)
    with pytest.raises(ValueError):
        qg.qg_experts_combine(x, torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.ones(2, 3, device="cuda"))


def test_tensors_that_the_current_device_does_not_hold_are_refused(qg, monkeypatch):
    packed, _ = blobs(qg, 2, 64, 128, 4, 64, 1)
    x, offsets = torch.randn(4, 128).cuda(), torch.tensor([0, 2, 4], dtype=torch.int32).cuda()
    need = qg.qg_experts_workspace_bytes(4, 128)
    for workspace in (torch.empty(need, dtype=torch.uint8), torch.empty(1, dtype=torch.uint8, device="cuda").expand(need)):
        with pytest.raises(ValueError):
            qg.qg_experts_product(packed, 64, 128, 4, 64, x, offsets, workspace=workspace)
    ids, weights = qg.qg_route(torch.randn(4, 2).cuda(), 1)
    _, rows, slots = qg.qg_expert_plan(ids, 2)
    torch.cuda.synchronize()
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)          # the calls see a current device that none of the tensors is on
    calls = (lambda: qg.qg_route(x, 1), lambda: qg.qg_expert_plan(ids, 2), lambda: qg.qg_experts_product(packed, 64, 128, 4, 64, x, offsets, rows=rows),
             lambda: qg.qg_experts_combine(x, slots, weights))
    for call in calls:
        with pytest.raises(ValueError, match="current device"):
            call()


# --- distances past 32 bits -------------------------------------------------------------------------------------

def test_route_past_32_bits(qg):
    case("route far", 1200001, 1900)
    logits = torch.zeros(1200001, 1900, dtype=BF16, device="cuda")
    last = torch.randn(5, 64, generator=gen(1)).to(BF16)
    logits[-5:, :64] = last.cuda()
    ids, weights = qg.qg_route(logits[:, :64], 6)
    want, w = plain_route(last, 6, None, "softmax", 1, 1, 1, True, 1.0)
    assert torch.equal(ids[-5:].cpu(), want)
    near(weights[-5:].cpu(), w, 2 * U * w.abs(), F32)
    assert (ids[:-5] == torch.arange(6, device="cuda")).all()


@pytest.mark.parametrize("counts", [[2], [40]])
def test_experts_past_32_bits(qg, counts):
    case("experts far", counts)
    N, K, group, E = 96, 256, 64, 700
    one, W = blobs(qg, 1, N, K, 4, group, 4)
    packed = torch.empty(E, 7 << 20, dtype=torch.uint8, device="cuda")
    packed[E - 1, : one.shape[1]] = one[0]
    x = torch.randn(counts[0], K, generator=gen(5))
    offsets = [0] * E + counts
    y = qg.qg_experts_product(packed, N, K, 4, group, x.cuda(), torch.tensor(offsets, dtype=torch.int32).cuda())
    want, slack = product_want(W, x, [0] + counts, None, False, group)
    near(y.cpu(), want, slack, F32)


@pytest.mark.parametrize("E,N,slots", [(2, 4096, 600000), (1024, 220000, 10240)])
def test_rows_past_32_bits(qg, E, N, slots):
    # X's rows, those of its f16 parts and those of y: by the kernel of many rows and by that of few
    case("rows far", E, N, slots)
    K, group, stride, tokens = 32, 32, 8192, 300000
    one, W = blobs(qg, 1, N, K, 4, group, 6)
    packed = one.expand(E, one.shape[1]).contiguous()
    x = torch.zeros(tokens, stride, dtype=BF16, device="cuda")[:, :K]
    x[-1] = torch.randn(K, generator=gen(7)).to(BF16).cuda()
    rows = torch.zeros(slots, dtype=torch.int32)
    rows[-3:] = torch.tensor([tokens - 1, 0, tokens - 1])
    offsets = torch.arange(E + 1) * slots // E
    y = qg.qg_experts_product(packed, N, K, 4, group, x, offsets.int().cuda(), rows=rows.cuda())
    want, slack = product_want(W, x[-1:].cpu(), [0, 1], None, False, group)
    for at in (-3, -1):
        near(y[at:][:1].cpu(), want, slack, BF16)
    assert (y[-2] == 0).all() and not y[:-3].any()


def test_sum_past_32_bits(qg):
    case("sum far", 600000, 4096)
    y = torch.empty(600000, 4096, dtype=BF16, device="cuda")
    last = torch.randn(4, 4096, generator=gen(8)).to(BF16)
    y[-4:] = last.cuda()
    slots = torch.full((540000, 2), -1, dtype=torch.int32, device="cuda")
    slots[-1], slots[-3] = torch.tensor([599999, 599996]), torch.tensor([599997, 599998])
    out = qg.qg_experts_combine(y, slots, torch.tensor([0.25, 2.0], device="cuda").expand(540000, 2).contiguous())
    for at, (a, b) in ((-1, (3, 0)), (-3, (1, 2))):
        want, size = 0.25 * last[a].double() + 2 * last[b].double(), 0.25 * last[a].double().abs() + 2 * last[b].double().abs()
        near(out[at].cpu(), want, 4 * U * size, BF16)
    assert not out[:-3].any() and not out[-2].any()

"""A layer of experts at its edges: gates far below zero, small values beside large ones, values that are no numbers for every width of a token's lanes, offsets that no plan makes for the kernels of many rows, more workgroups than a launch has in one dimension, the layer's wiring within what its parts may be off by.

U = 2^-24, the unit roundoff of fp32; each test derives its bound, set before any of these ran."""
import math

import pytest
import torch

from tests.test_gpu_experts import BF16, F16, F32, INF, U, blobs, case, gen, layer, near, offsets_of, plain_route, product_want

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qg():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2307_03738_amd import binding
    binding.lib()
    return binding


# --- gates ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("columns,tokens", [(70, 1), (70, 12), (1600, 400)])
def test_gates_far_below_zero(qg, columns, tokens):
    # Gates are the row's first x, exactly (numbers of eleven bits, weights of one), ups 2^60 of it, so that y is an ordinary number where the gate's silu is not.
    # silu: e^-|v| by the series' instruction 2 U and what its argument is rounded by 1/3 U, in numerator and (at half, at most) denominator, 1 + t 1 U,
    # its reciprocal 2 U, two products: 8 U; and half a step of the numbers below the normal ones, once.
    case("gates", columns, tokens)
    group = K = 32
    q = torch.full((2 * columns, K), 8, dtype=torch.uint8)
    s = torch.ones(2 * columns, 1)
    s[columns:] = 2.0 ** 60
    z = torch.full((2 * columns, 1), 7, dtype=torch.uint8)
    packed = qg.qg_pack(q.cuda(), s.cuda(), z.cuda(), 4, group)[None]
    v = torch.cat([-torch.arange(1280, 1665) / 16, torch.tensor([0.0, -200.0, -201.0, -300.0, -1000.0, -60000.0, 1.0, -1.0, 0.125, 88.0, 104.0, 1000.0, 3.0, -3.0, -20.0])])
    pieces = v.split(tokens)
    offsets = torch.tensor([0, tokens], dtype=torch.int32).cuda()
    for piece in pieces if tokens > 1 else pieces[::5]:
        x = torch.zeros(tokens, K)
        x[:len(piece), 0] = piece
        y = qg.qg_experts_product(packed, 2 * columns, K, 4, group, x.cuda(), offsets, gated=True).cpu()
        gate = x[:, :1].double()
        want = (gate / (1 + torch.exp(-gate)) * (gate * 2.0 ** 60)).expand(-1, columns)
        near(y, want, 8 * U * want.abs() + 2.0 ** -150 * (gate * 2.0 ** 60).abs(), F32)


def test_infinite_gates(qg):
    q, s, z = torch.full((128, 32), 8, dtype=torch.uint8).cuda(), torch.ones(128, 1).cuda(), torch.full((128, 1), 7, dtype=torch.uint8).cuda()
    x = torch.zeros(3, 32)
    x[:, 0] = torch.tensor([INF, -INF, 1.0])
    y = qg.qg_experts_product(qg.qg_pack(q, s, z, 4, 32)[None], 128, 32, 4, 32, x.cuda(), torch.tensor([0, 3], dtype=torch.int32).cuda(), gated=True).cpu()
    assert (y[0] == INF).all() and torch.isnan(y[1]).all() and torch.isfinite(y[2]).all()      # v / (1 + e^-v) at -infinity is a quotient of infinities


# --- fp32 rows of wide range ------------------------------------------------------------------------------------

@pytest.mark.parametrize("N,K,bits,group,counts", [
    (64, 64, 4, 32, [0, 1, 0, 0]), (70, 256, 4, 128, [3, 12]), (70, 160, 3, 32, [3, 12]), (70, 192, 2, 64, [3, 12]), (70, 96, 4, 16, [3, 12]), (70, 80, 4, 8, [3, 12]), (70, 96, 2, 16, [3, 12]),
    (7170, 160, 4, 32, [40, 33, 64]), (7170, 192, 3, 64, [40, 33, 64]), (7170, 256, 2, 128, [40, 33, 64]),
    (5130, 384, 4, 128, [129, 600]), (5130, 320, 2, 64, [300, 419]), (5130, 160, 3, 32, [300, 419]), (5130, 1056, 4, 32, [100, 77]), (5130, 1280, 2, 128, [100, 77])])
def test_small_values_beside_a_large_one_count_in_full(qg, N, K, bits, group, counts):
    # A channel 2^20 to 2^21 above the others, whose weights are zero (q = z), and one other value a row: y is one product.  An x is off by 2^-23 of itself or 2^-51 of the row's
    # largest (2^-30 here); its parts' products add up with one rounding (2 U, if cut off), the scale's and the sum of a row's parts are one each.
    case("wide range", N, K, bits, group, counts)
    E, g = len(counts), gen(N + K)
    q = torch.randint(0, 2 ** bits, (E, N, K), generator=g, dtype=torch.uint8)
    s = 0.5 + torch.rand(E, N, K // group, generator=g)
    z = torch.randint(0, 2 ** bits, (E, N, K // group), generator=g, dtype=torch.uint8)
    q[:, :, 0] = z[:, :, 0]
    packed = torch.stack([qg.qg_pack(q[e].cuda(), s[e].cuda(), z[e].cuda(), bits, group) for e in range(E)])
    offsets = offsets_of(counts)
    x = torch.zeros(offsets[-1], K)
    x[:, 0] = 2.0 ** 20 * (1 + torch.rand(len(x), generator=g))
    at = 1 + 7 * torch.arange(len(x)) % (K - 1)
    small = 1 + torch.rand(len(x), generator=g)
    x[torch.arange(len(x)), at] = small
    y = qg.qg_experts_product(packed, N, K, bits, group, x.cuda(), torch.tensor(offsets, dtype=torch.int32).cuda()).cpu()
    expert = torch.repeat_interleave(torch.arange(E), torch.tensor(counts))
    w = s[expert, :, at // group].double() * (q[expert, :, at].double() - z[expert, :, at // group].double())
    near(y, small.double()[:, None] * w, (6 * U * small.double()[:, None] + 2.0 ** -30) * w.abs(), F32)


# --- choices of values that are no numbers ----------------------------------------------------------------------

@pytest.mark.parametrize("experts,groups,top_groups", [(12, 1, 1), (12, 4, 2), (100, 10, 7), (150, 1, 1), (150, 10, 6), (250, 10, 6), (300, 1, 1), (300, 12, 5), (600, 12, 5)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("best", [1, 2])
@pytest.mark.parametrize("bias", ["none", "numbers", "switched off", "no number"])
def test_choices_of_values_that_are_no_numbers(qg, experts, groups, top_groups, score, best, bias):
    # every width of a token's lanes; of neighbouring tokens one has a NaN; an expert that its logit switches off does not show that its bias is NaN
    case("route nan", experts, groups, score, best, bias)
    g = gen(experts + groups)
    logits = torch.randn(11, experts, generator=g)
    logits[1, 3] = math.nan
    logits[3, experts - 1] = math.nan
    logits[5] = math.nan
    logits[6, 5] = -INF
    logits[7] = -INF
    logits[8, [4, 7]] = INF
    logits[9, experts // 2:] = -INF
    b = None if bias == "none" else 0.2 * torch.randn(experts, generator=g)
    if bias == "switched off":
        b[[2, experts - 1]] = -INF
    if bias == "no number":
        b[5] = math.nan
    for renormalise in (True, False):
        ids, w = qg.qg_route(logits.cuda(), 4, bias=None if b is None else b.cuda(), score=score, groups=groups, top_groups=top_groups, group_best=best, renormalise=renormalise)
        want, ww = plain_route(logits, 4, b, score, groups, top_groups, best, renormalise, 1.0)
        assert torch.equal(ids.cpu(), want)
        assert torch.equal(torch.isnan(w.cpu()), torch.isnan(ww))
        assert torch.isnan(ww).any() and not torch.isnan(ww[6:8]).any()
        near(w.cpu().nan_to_num(0), ww.nan_to_num(0), 2 * U * ww.nan_to_num(0).abs(), F32)


# --- offsets ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("E,N,K,slots,dt", [(3, 7170, 192, 200, F32), (3, 7170, 192, 140, BF16), (2, 5130, 320, 719, F16), (2, 5130, 1056, 177, BF16), (70, 2600, 64, 4000, BF16), (70, 2600, 64, 5000, F32),
                                            (9, 130, 64, 40, F32)])
def test_offsets_that_no_plan_makes(qg, E, N, K, slots, dt):
    # tiles of 32 and of 64 slots, K in slices, more experts than a wavefront has lanes, few rows
    case("offsets", E, N, K, slots, dt)
    group, guard = 64 if K % 64 == 0 else 32, 5
    one, W = blobs(qg, 1, N, K, 4, group, 12)
    packed = one.expand(E, one.shape[1]).contiguous()
    x = torch.randn(slots, K, generator=gen(E)).to(dt)
    want, slack = product_want(W, x, [0, slots], None, False, group)
    plan = torch.arange(E + 1) * slots // E
    far = plan.clone()
    far[1::3], far[2::3] = 1 << 30, -(1 << 31)
    for offsets in (plan.flip(0), plan + slots, plan - slots, far, torch.cat([plan[1:], plan[:1]]), torch.full((E + 1,), (1 << 31) - 1), torch.where(torch.arange(E + 1) % 2 == 0, 0, slots)):
        y = torch.full((slots + 2 * guard, N), 7.0, device="cuda")
        qg.qg_experts_product(packed, N, K, 4, group, x.cuda(), offsets.int().cuda(), y=y[guard: slots + guard], dtype=F32)
        y = y.cpu()
        assert (y[:guard] == 7).all() and (y[-guard:] == 7).all()
        # all experts have the same matrix: a row that any of them has taken holds its product
        rows = (y[guard:-guard] != 7).any(1)
        near(y[guard:-guard][rows], want[rows], slack[rows], F32)


# --- the most workgroups ----------------------------------------------------------------------------------------

def test_more_workgroups_than_a_dimension_has(qg):
    # 2^23 workgroups and 48892 more, of 64 rows each; every row is one of three
    case("workgroups", 540000000)
    N, K, group, slots = 8, 32, 32, 540000000
    packed, W = blobs(qg, 2, N, K, 4, group, 13)
    x = torch.randn(3, K, generator=gen(14)).to(BF16)
    rows = torch.arange(3, dtype=torch.int32, device="cuda").repeat(slots // 3)
    offsets = torch.tensor([0, slots // 2, slots], dtype=torch.int32, device="cuda")
    y = qg.qg_experts_product(packed, N, K, 4, group, x.cuda(), offsets, rows=rows)
    for e in range(2):
        got = y[e * slots // 2: (e + 1) * slots // 2].view(-1, 3, N)
        assert bool((got == got[:1]).all())
        want, slack = product_want(W[e: e + 1], x, [0, 3], None, False, group)
        near(got[0].cpu(), want, slack, BF16)


# --- together ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("tokens,bits,group", [(1, 4, 32), (13, 3, 64), (150, 2, 64), (40, 4, 16)])
def test_a_layer_is_off_by_no_more_than_its_parts(qg, tokens, bits, group):
    # h within the gated product's slack; y within that through |What| and its own product's; each weight 2 U; the sum's k + 2 roundings
    case("layer parts", tokens, bits, group)
    E, N, K, k = 9, 192, 256, 3
    up, Wu = blobs(qg, E, 2 * N, K, bits, group, 1)
    down, Wd = blobs(qg, E, K, N, bits, group, 2)
    x, logits = torch.randn(tokens, K, generator=gen(tokens)), 2 * torch.randn(tokens, E, generator=gen(tokens + 1))
    logits[:, 4] = -INF
    got = layer(qg, up, down, N, K, bits, group, x.cuda(), logits.cuda(), k).cpu()
    best, ids = logits.double().topk(k, 1)
    weights = best.softmax(1)
    want, slack, size = x.double().clone(), torch.zeros(tokens, K, dtype=torch.float64), x.double().abs()
    for j in range(k):
        for e in range(E):
            t = (ids[:, j] == e).nonzero()[:, 0]
            if len(t) == 0:
                continue
            h, eh = product_want(Wu[e: e + 1], x[t], [0, len(t)], None, True, group)
            eh = eh + U * (h.abs() + eh) + 2.0 ** -149
            y, ey = product_want(Wd[e: e + 1], h, [0, len(t)], None, False, group)
            ey = ey + eh @ Wd[e].abs().t()
            ey = ey + U * (y.abs() + ey)
            w = weights[t, j: j + 1]
            want[t] += w * y
            slack[t] += w * ey + 2 * U * w * (y.abs() + ey)
            size[t] += w * (y.abs() + ey)
    near(got, want, slack + (k + 2) * U * size, F32)

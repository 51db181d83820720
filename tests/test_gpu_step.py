"""The calls between the products of a token's step -- norm, cache writing, attention over the paged cache, the pages' book --
against plain implementations: in 64 bits for what is computed, with loops over rows and pages for the book.

Tolerances (U = 2^-24, the unit roundoff of fp32), set before any of these ran:
  norm      a sum of K squares in pieces of at most 64 terms and ten levels of a tree errs by at most 74 U of itself, half of that
            under the root, six roundings around it: 43 U of |y|.
  rotation  two products, one sum: 3 U of |a cos| + |b sin|.
  attention a score sums D products: (D + 8) U of scale * sum |q k| (times |k scale|); exp of a difference of scores adds
            4 U and U of the scores; the p_i are kept to 2^-16; n of them add up with sqrt(n) U.  Two sums of this kind
            are divided: 2 (delta + 2^-16 + sqrt(n) U) max |v|.
  storing   half a unit of the type's last place: 2^-8 (bf16: 8 bits of significand), 2^-11 (f16: 11), 2^-4 (e4m3: 4) of the value, and half of the
            smallest step, 2^-25 for f16 and 2^-10 scales for e4m3, the rounding of the scale itself included in 2^-4.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F8 = torch.float8_e4m3fn
REL = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, F8: 2.0 ** -4}
STEP = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25, F8: 2.0 ** -10}


@pytest.fixture(scope="module")
def qg():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2307_03738_amd import binding
    binding.lib()
    return binding


def case(*what):
    print("[case]", *what, flush=True)


def near(got, want, slack, dtype, scale=1.0):
    """got (as stored, times its scale) within slack of want before rounding and half a last place after it."""
    err = (got - want).abs()
    bound = slack + (want.abs() + slack) * REL[dtype] + STEP[dtype] * scale
    worst = (err - bound).max().item() if err.numel() else -1.0
    assert not torch.isnan(err).any() and worst <= 0, f"off by {worst:.3e} more than allowed; largest error {err.max().item():.3e}"


def gen(seed):
    return torch.Generator().manual_seed(seed)


# --- norm -------------------------------------------------------------------------------------------------------

NORMS = [
    # rows, K, type, residual, weight type, out, group, row stride beyond K
    (1, 4096, torch.float32, True, torch.float32, torch.float32, 0, 0),
    (3, 4096, torch.bfloat16, True, torch.bfloat16, torch.bfloat16, 0, 0),
    (5, 5120, torch.float16, True, torch.float32, torch.float16, 0, 64),
    (2, 8192, torch.bfloat16, False, torch.float32, torch.float32, 0, 8),
    (7, 1, torch.float32, True, torch.float32, torch.float32, 0, 0),
    (4, 7, torch.float16, True, torch.float16, torch.bfloat16, 0, 0),
    (3, 1001, torch.bfloat16, True, torch.float32, torch.float32, 0, 3),
    (2, 20000, torch.float32, True, torch.float32, torch.float16, 0, 0),
    (2, 33333, torch.float32, True, torch.float32, F8, 0, 0),
    (130, 4096, torch.float32, True, torch.float32, F8, 128, 0),
    (9, 5120, torch.bfloat16, True, torch.float32, F8, 64, 0),
    (33, 192, torch.float16, False, torch.float32, F8, 24, 0),
    (6, 4096, torch.float16, True, torch.float32, F8, 0, 16),
    (3, 90, torch.float32, False, torch.bfloat16, F8, 9, 5),
    (2, 65536, torch.bfloat16, True, torch.float32, F8, 1024, 0),
    (1024, 512, torch.float32, True, torch.float32, torch.bfloat16, 0, 0),
    (5, 8, torch.float32, True, torch.float32, F8, 1, 0),
    (300, 64, torch.bfloat16, True, torch.float32, torch.bfloat16, 0, 0),
    (2, 16384, torch.float32, True, torch.float32, F8, 512, 0),
]


def norm_want(x, r, w, eps, group):
    h = x.double() + (r.double() if r is not None else 0)
    y = h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * w.double()
    return h, y


@pytest.mark.parametrize("rows,K,dt,residual,wt,out,group,gap", NORMS)
def test_norm_matches_64_bits(qg, rows, K, dt, residual, wt, out, group, gap):
    case("norm", rows, K, dt, out, group, gap)
    g = gen(rows * 7 + K)
    x = torch.randn(rows, K + gap, generator=g)
    x[:, ::13] *= 30
    x[-1] *= 1e-3
    x, w = x.to(dt)[:, :K], (1 + 0.2 * torch.randn(K, generator=g)).to(wt)
    r = torch.randn(rows, K + 2 * gap, generator=g).to(dt)[:, :K] if residual else None
    dx = x.cuda() if gap == 0 else torch.empty(rows, K + gap, dtype=dt, device="cuda")[:, :K].copy_(x)
    dr = None if r is None else (r.cuda() if gap == 0 else torch.empty(rows, K + 2 * gap, dtype=dt, device="cuda")[:, :K].copy_(r))
    y, h, s = qg.qg_rms_norm(dx, w.cuda(), 1e-5, residual=dr, dtype=out, group=group)
    h64, y64 = norm_want(x, r, w, 1e-5, group)
    if residual:
        near(h.cpu().double(), h64, 2 * U * (x.double().abs() + r.double().abs()), dt)
    got = y.cpu().double()
    if out is not F8:
        assert s is None
        near(got, y64, 43 * U * y64.abs(), out)
        return
    size = group or K
    s64 = y64.view(rows, -1, size).abs().amax(2) / 448
    assert s.shape == s64.shape
    near(s.cpu().double(), s64, 45 * U * s64, torch.float32)
    wide = s.cpu().double().repeat_interleave(size, 1)
    near(got * wide, y64, 45 * U * y64.abs(), F8, wide)


def test_norm_writes_h_over_its_inputs(qg):
    for which in ("x", "residual"):
        x, r, w = (torch.randn(*n, generator=gen(i)).cuda() for i, n in enumerate(((37, 4096), (37, 4096), (4096,))))
        y0, h0, _ = qg.qg_rms_norm(x, w, 1e-6, residual=r)
        y, h, _ = qg.qg_rms_norm(x, w, 1e-6, residual=r, h=x if which == "x" else r)
        assert torch.equal(y, y0) and torch.equal(h, h0) and h.data_ptr() == (x if which == "x" else r).data_ptr()


def test_norm_of_rows_that_are_zero_or_hold_no_numbers(qg):
    x = torch.randn(6, 256, generator=gen(3))
    x[0] = 0
    x[1, 5], x[2, 250], x[3, 100] = math.nan, math.inf, -math.inf
    y, _, s = qg.qg_rms_norm(x.cuda(), torch.ones(256).cuda(), dtype=F8, group=64)
    y, s = y.cpu().float(), s.cpu()
    assert (y[0] == 0).all() and (s[0] == 1).all()
    assert torch.isnan(s[1]).all() and torch.isnan(y[1]).all()            # the sum of squares is NaN
    for row, at in ((2, 3), (3, 1)):                                       # infinity / infinity; the other values come out 0
        assert torch.isnan(s[row, at]) and torch.isnan(y[row, at * 64:(at + 1) * 64]).all()
        assert (s[row, [i for i in range(4) if i != at]] == 1).all()
    assert torch.isfinite(y[4:]).all()
    y, _, _ = qg.qg_rms_norm(x.cuda(), torch.ones(256).cuda())
    assert torch.isfinite(y[[0, 4, 5]]).all() and torch.isnan(y[1]).all() and torch.isnan(y[2, 250]) and (y[2, :250] == 0).all()


def test_empty_batches_are_fine(qg):
    y, h, s = qg.qg_rms_norm(torch.empty(0, 64, device="cuda"), torch.ones(64, device="cuda"), residual=torch.empty(0, 64, device="cuda"))
    assert y.shape == (0, 64) and h.shape == (0, 64) and s is None
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16, device="cuda")
    t, none = torch.zeros(1, 4, dtype=torch.int32, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    q = torch.empty(0, 4, 64, device="cuda")
    assert qg.qg_kv_append(k, k.clone(), t, none, none, q[:, :2], q[:, :2], q=q).shape == (0, 4, 64)
    out, lse = qg.qg_paged_attention(q, k, k, t, none, 0.1, lse=True)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)


# --- writing the cache ------------------------------------------------------------------------------------------

APPENDS = [
    # heads, kv heads, head_dim, rope, interleaved, type, cache, page, lengths, start
    (32, 32, 128, 128, False, torch.float32, torch.bfloat16, 16, [1], 700),
    (8, 2, 128, 128, True, torch.bfloat16, F8, 32, [40, 0, 1, 33], 0),
    (4, 4, 64, 64, False, torch.float16, torch.float16, 16, [17, 16, 15], 5),
    (5, 1, 80, 40, True, torch.float32, F8, 64, [70, 3], 64),
    (6, 3, 96, 96, False, torch.bfloat16, torch.bfloat16, 128, [9, 130], 1),
    (2, 1, 256, 256, False, torch.float32, torch.float16, 16, [33], 0),
    (2, 2, 8, 2, True, torch.float32, F8, 16, [20, 20], 3),
    (0, 3, 40, 0, False, torch.float32, torch.bfloat16, 16, [5, 6], 0),
    (3, 3, 72, 20, False, torch.float16, F8, 4096, [50], 4090),
    (16, 16, 248, 100, True, torch.bfloat16, torch.float16, 32, [12], 0),
]


@pytest.mark.parametrize("H,Hkv,D,rope,inter,dt,ct,page,lens,start", APPENDS)
def test_append_matches_64_bits(qg, H, Hkv, D, rope, inter, dt, ct, page, lens, start):
    case("append", H, Hkv, D, rope, inter, dt, ct, page, lens, start)
    g = gen(H + D + page)
    need = [-(-(start + n) // page) for n in lens]
    pages = sum(need) + 2
    ids = torch.randperm(pages, generator=g)[:sum(need)].tolist()
    most = max(need)
    tables = torch.full((len(lens), most + 1), -1, dtype=torch.int32)
    for b, n in enumerate(need):
        for j in range(n):
            tables[b, j] = ids.pop()
    tokens = [(b, start + i) for b, n in enumerate(lens) for i in range(n)]
    order = torch.randperm(len(tokens), generator=g).tolist()
    tokens = [tokens[i] for i in order] + [(-1, 0), (len(lens), 0), (0, (most + 1) * page), (0, -1), (0, most * page)]      # the last ones have no page
    T, real = len(tokens), len(order)
    qkv = torch.randn(T, (H + 2 * Hkv) * D + 8, generator=g)
    qkv[0, H * D: (H + Hkv) * D] = 0                                        # a token whose k is zero
    qkv = qkv.to(dt)
    q, k, v = (qkv[:, a * D: b * D].view(T, b - a, D) for a, b in ((0, H), (H, H + Hkv), (H + Hkv, H + 2 * Hkv)))
    cs = None
    if rope:
        ang = torch.arange((most + 1) * page + 1).double()[:, None] * 100.0 ** (-torch.arange(rope // 2).double() / rope)
        cs = torch.cat((ang.cos(), ang.sin()), 1).float()
    shape = (pages, Hkv, page, D)
    kc, vc = torch.full(shape, 7.0).to(ct).cuda(), torch.full(shape, 7.0).to(ct).cuda()
    ks = vs = None
    if ct is F8:
        ks, vs = torch.full(shape[:3], 3.0).cuda(), torch.full(shape[:3], 3.0).cuda()
    d = qkv.cuda()
    dq, dk, dv = (d[:, a * D: b * D].view(T, b - a, D) for a, b in ((0, H), (H, H + Hkv), (H + Hkv, H + 2 * Hkv)))
    out = qg.qg_kv_append(kc, vc, tables.cuda(), torch.tensor([b for b, _ in tokens], dtype=torch.int32).cuda(),
                          torch.tensor([p for _, p in tokens], dtype=torch.int32).cuda(), dk, dv, q=dq if H else None,
                          cos_sin=None if cs is None else cs.cuda(), interleaved=inter, k_scale=ks, v_scale=vs)

    def turned(x):
        x, size = x[:real].double().clone(), x[:real].double().abs()
        for j in range(rope // 2):
            a, b = (2 * j, 2 * j + 1) if inter else (j, j + rope // 2)
            at = torch.tensor([p for _, p in tokens[:real]])
            c, s = cs[at, j].double()[:, None], cs[at, rope // 2 + j].double()[:, None]
            u, w = x[..., a].clone(), x[..., b].clone()
            x[..., a], x[..., b] = u * c - w * s, w * c + u * s
            size[..., a], size[..., b] = (u * c).abs() + (w * s).abs(), (w * c).abs() + (u * s).abs()
        return x, 3 * U * size

    if H:
        x, slack = turned(q)
        near(out.cpu()[:real].double(), x, slack, dt)
        assert (out[real:] == 0).all()
    for cache, scales, (x, slack) in ((kc, ks, turned(k)), (vc, vs, (v[:real].double(), torch.zeros(real, Hkv, D, dtype=torch.float64)))):
        cache = cache.cpu().double()
        where = [(int(tables[b, p // page]), p % page) for b, p in tokens[:real]]
        got = torch.stack([cache[i, :, j] for i, j in where]) if where else cache[:0, :, 0]
        rest = torch.ones(pages, page, dtype=torch.bool)
        for i, j in where:
            rest[i, j] = False
        assert (cache.transpose(1, 2)[rest] == 7).all(), "a cell of no token was written"
        if scales is None:
            near(got, x, slack, ct)
            continue
        sc = torch.stack([scales.cpu().double()[i, :, j] for i, j in where])
        want = x.abs().amax(2) / 448
        want = torch.where(want == 0, 1.0, want)
        near(sc, want, 4 * U * want, torch.float32)
        near(got * sc[..., None], x, slack + 4 * U * x.abs(), F8, sc[..., None])
        assert (scales.cpu().transpose(1, 2)[rest] == 3).all()


# --- attention --------------------------------------------------------------------------------------------------

def cache_of(lens, Hkv, D, page, ct, g, extra=3):
    """(k, v, k_scale, v_scale, tables, K64, V64): used cells random, all others NaN, stale table entries."""
    need = [-(-n // page) for n in lens]
    pages = sum(need) + extra
    ids = torch.randperm(pages, generator=g).tolist()
    columns = max(max(need), 1) + 2
    # stale entries: pages of nobody, and ids that are none
    tables = torch.tensor([[(-1, 0x7fffffff, pages - 1, 0)[(b + j) % 4] for j in range(columns)] for b in range(len(lens))], dtype=torch.int32)
    shape = (pages, Hkv, page, D)
    kv, scales, wide = [], [], []
    for b, n in enumerate(need):
        for j in range(n):
            tables[b, j] = ids.pop()
    for which in range(2):
        x = torch.full(shape, math.nan)
        s = torch.full(shape[:3], math.nan) if ct is F8 else None
        for b, n in enumerate(lens):
            for j in range(need[b]):
                used = min(page, n - j * page)
                i = int(tables[b, j])
                x[i, :, :used] = torch.randn(Hkv, used, D, generator=g) * (100 if ct is F8 else 1)
                if s is not None:
                    s[i, :, :used] = (0.5 + torch.rand(Hkv, used, generator=g)) / 100
        x = x.clamp(-448, 448).to(ct) if ct is F8 else x.to(ct)
        kv.append(x)
        scales.append(s)
        wide.append(x.double() if s is None else x.double() * s.double()[..., None])
    return kv[0], kv[1], scales[0], scales[1], tables, wide[0], wide[1]


def attention_want(q, K, V, tables, lens, firsts, window, page, scale):
    """(out, lse, slack of out, slack of lse) in 64 bits, sequence by sequence."""
    B, H, D = q.shape
    Hkv = K.shape[1]
    out, lse = torch.zeros(B, H, D, dtype=torch.float64), torch.full((B, H), -math.inf, dtype=torch.float64)
    so, sl = torch.zeros(B, H, 1, dtype=torch.float64), torch.zeros(B, H, dtype=torch.float64)
    for b in range(B):
        first = max(firsts[b], lens[b] - window) if window else firsts[b]
        at = torch.arange(first, max(first, lens[b]))
        if not len(at):
            continue
        cells = (tables[b, at // page].long(), at % page)
        for h in range(H):
            k, v = K[:, h * Hkv // H][cells], V[:, h * Hkv // H][cells]
            x = q[b, h].double()
            s = k @ x * scale
            p = torch.softmax(s, 0)
            out[b, h], lse[b, h] = p @ v, torch.logsumexp(s, 0)
            delta = (D + 8) * U * scale * (k.abs() @ x.abs()).max() + 4 * U + 2 * U * s.abs().max()
            e = 2 * (delta + 2.0 ** -16 + math.sqrt(len(at)) * U)
            so[b, h], sl[b, h] = e * v.abs().max(), e + 2 * U * lse[b, h].abs()
    return out, lse, so, sl


ATTENTIONS = [
    # heads, kv heads, head_dim, page, cache, q type, lengths, firsts, window
    (32, 32, 128, 16, torch.bfloat16, torch.float32, [777], None, 0),
    (8, 8, 128, 16, torch.bfloat16, torch.bfloat16, [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129], None, 0),
    (16, 2, 128, 32, F8, torch.float32, [300, 0, 1, 513, 64], [42, 0, 0, 73, 64], 0),
    (10, 2, 128, 64, torch.float16, torch.float16, [2049, 100], None, 0),
    (4, 1, 64, 16, torch.float16, torch.float32, [129, 47, 1], None, 0),
    (4, 2, 64, 128, F8, torch.bfloat16, [1000, 3], None, 0),
    (6, 2, 80, 16, torch.bfloat16, torch.float16, [95, 200], None, 0),
    (3, 3, 96, 32, F8, torch.float16, [31, 65, 500], None, 0),
    (2, 1, 256, 16, torch.bfloat16, torch.float32, [70, 333], None, 0),
    (4, 4, 256, 64, F8, torch.float32, [130], None, 0),
    (2, 2, 256, 16, torch.float16, torch.bfloat16, [65], None, 0),
    (16, 1, 128, 16, torch.float16, torch.float32, [600], None, 0),
    (40, 2, 64, 16, torch.bfloat16, torch.float32, [150, 7], None, 0),
    (71, 1, 64, 16, torch.bfloat16, torch.bfloat16, [260], None, 0),
    (5, 5, 8, 16, torch.bfloat16, torch.float32, [40, 5], None, 0),
    (4, 2, 136, 16, torch.float16, torch.float32, [77, 40], None, 0),
    (4, 2, 24, 16, F8, torch.float32, [77, 40], None, 0),
    (2, 2, 200, 32, F8, torch.float16, [77, 33], None, 0),
    (8, 2, 128, 16, torch.bfloat16, torch.float32, [500, 20, 0, 17], None, 17),
    (8, 2, 128, 16, torch.bfloat16, torch.float32, [500, 20, 700, 17], [490, 30, 5, 17], 200),
    (8, 8, 128, 4096, F8, torch.bfloat16, [5000, 4096], None, 0),
    (64, 8, 128, 16, torch.bfloat16, torch.bfloat16, [4100] + [33 * i for i in range(31)], None, 0),
    (8, 1, 128, 64, torch.bfloat16, torch.float32, [20011], None, 0),
    (2, 2, 128, 16, torch.float16, torch.float16, [7 * i for i in range(300)], None, 0),
]


@pytest.mark.parametrize("H,Hkv,D,page,ct,dt,lens,firsts,window", ATTENTIONS)
def test_attention_matches_64_bits(qg, H, Hkv, D, page, ct, dt, lens, firsts, window):
    case("attention", H, Hkv, D, page, ct, dt, len(lens), lens[:8], firsts, window)
    g = gen(H * 3 + D + page + len(lens))
    k, v, ks, vs, tables, K, V = cache_of(lens, Hkv, D, page, ct, g)
    B, scale = len(lens), 1.3 / math.sqrt(D)
    # q as a stacked product leaves it: followed by other things
    qkv = torch.randn(B, H * D + 24, generator=g).to(dt)
    q, dq = qkv[:, :H * D].view(B, H, D), qkv.cuda()[:, :H * D].view(B, H, D)
    on = lambda t: None if t is None else t.cuda()  # noqa: E731
    i32 = lambda t: None if t is None else torch.tensor(t, dtype=torch.int32, device="cuda")  # noqa: E731
    args = (dq, on(k), on(v), on(tables), i32(lens), scale)
    kw = dict(first=i32(firsts), window=window, k_scale=on(ks), v_scale=on(vs), lse=True)
    workspace = qg.new_workspace(qg.qg_paged_attention_workspace_bytes(B, H, Hkv, D))
    out, lse = qg.qg_paged_attention(*args, **kw, workspace=workspace)
    want, wlse, so, sl = attention_want(q, K, V, tables, lens, firsts or [0] * B, window, page, scale)
    near(out.cpu().double(), want, so, dt)
    empty = torch.isinf(wlse)
    assert torch.equal(torch.isinf(lse.cpu()), empty) and (lse.cpu()[empty] < 0).all() and (out.cpu()[empty] == 0).all()
    near(lse.cpu().double()[~empty], wlse[~empty], sl[~empty], torch.float32)
    # the workspace is left prepared, and the bits are the same each time
    for _ in range(3):
        again, lse2 = qg.qg_paged_attention(*args, **kw, workspace=workspace)
        assert torch.equal(again, out) and torch.equal(lse2, lse)


def test_attention_with_scores_far_apart(qg):
    # one key outweighs all others by e^200, some score -1e4: nothing overflows, the small ones vanish
    for ct in (torch.bfloat16, torch.float16):
        lens, D = [200, 1, 65], 128
        k, v, _, _, tables, K, V = cache_of(lens, 2, D, 16, ct, gen(5))
        q = torch.randn(3, 4, D, generator=gen(6)) * 40
        out, lse = qg.qg_paged_attention(q.cuda(), k.cuda(), v.cuda(), tables.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), 1.0, lse=True)
        want, wlse, so, sl = attention_want(q, K, V, tables, lens, [0] * 3, 0, 16, 1.0)
        near(out.cpu().double(), want, so, torch.float32)
        near(lse.cpu().double(), wlse, sl, torch.float32)


@pytest.mark.parametrize("size", [1e-30, 1e-5, 1e4, 1e30])
def test_attention_on_queries_of_any_size(qg, size):
    # scale times q is what counts: q far outside of 16-bit ranges, in a cache of 16-bit floats
    for ct in (torch.bfloat16, torch.float16, F8):
        lens, D = [100, 33], 64
        k, v, ks, vs, tables, K, V = cache_of(lens, 1, D, 16, ct, gen(7))
        q = torch.randn(2, 3, D, generator=gen(8)) * size
        on = lambda t: None if t is None else t.cuda()  # noqa: E731
        out, lse = qg.qg_paged_attention(q.cuda(), on(k), on(v), tables.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), 0.2 / size,
                                         k_scale=on(ks), v_scale=on(vs), lse=True)
        want, wlse, so, sl = attention_want(q, K, V, tables, lens, [0] * 2, 0, 16, 0.2 / size)
        near(out.cpu().double(), want, so, torch.float32)
        near(lse.cpu().double(), wlse, sl, torch.float32)


def test_attention_values_of_any_size_and_scale(qg):
    # V scales from 1e-30 to 1e30 beside each other, a zero one among them
    lens, D = [130], 128
    k, v, ks, vs, tables, K, _ = cache_of(lens, 1, D, 16, F8, gen(9))
    for low, high in ((-30, -28), (28, 30), (-3, 3)):
        s = 10.0 ** (low + (high - low) * torch.rand(vs.shape, generator=gen(10)))
        s[int(tables[0, 0]), 0, 3] = 0
        V = v.double() * s.double()[..., None]
        q = torch.randn(1, 2, D, generator=gen(11))
        out, _ = qg.qg_paged_attention(q.cuda(), k.cuda(), v.cuda(), tables.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), 0.1,
                                       k_scale=ks.cuda(), v_scale=s.cuda())
        want, _, so, _ = attention_want(q, K, V, tables, lens, [0], 0, 16, 0.1)
        near(out.cpu().double(), want, so, torch.float32)


def test_attention_past_32_bit_offsets(qg):
    # a pool of more than 2^32 bytes and cells, of which only the last pages are in use
    page, Hkv, D = 64, 8, 128
    pages = (1 << 32) // (page * Hkv * D) + 8
    lens = [300]
    for ct in (F8, torch.bfloat16):
        case("offsets", ct, pages)
        small = cache_of(lens, Hkv, D, page, ct, gen(12), extra=0)
        n = small[0].shape[0]
        big = []
        for x in small[:4]:
            if x is None:
                big.append(None)
                continue
            t = torch.empty((pages,) + x.shape[1:], dtype=x.dtype, device="cuda")
            t[pages - n:] = x.cuda()
            big.append(t)
        q = torch.randn(1, 16, D, generator=gen(13))
        tables = torch.where((small[4] >= 0) & (small[4] < n), small[4] + pages - n, small[4])
        at = torch.tensor(lens, dtype=torch.int32).cuda()
        out, _ = qg.qg_paged_attention(q.cuda(), big[0], big[1], tables.cuda(), at, 0.1, k_scale=big[2], v_scale=big[3])
        want, _, so, _ = attention_want(q, small[5], small[6], small[4], lens, [0], 0, page, 0.1)
        near(out.cpu().double(), want, so, torch.float32)
        # ... and written there
        new = torch.randn(1, Hkv, D, generator=gen(14))
        qg.qg_kv_append(big[0], big[1], tables.cuda(), torch.zeros(1, dtype=torch.int32).cuda(), at - 1, new.cuda(), new.cuda(), k_scale=big[2], v_scale=big[3])
        cell = big[0][int(tables[0, (lens[0] - 1) // page]), :, (lens[0] - 1) % page].cpu().double()
        if ct is torch.bfloat16:
            near(cell, new[0].double(), torch.zeros(1, dtype=torch.float64), ct)
        else:
            s = big[2][int(tables[0, (lens[0] - 1) // page]), :, (lens[0] - 1) % page].cpu().double()[:, None]
            near(cell * s, new[0].double(), 4 * U * new[0].double().abs(), ct, s)
        del big
        torch.cuda.empty_cache()


def test_attention_workspace_serves_smaller_batches_in_any_order(qg):
    workspace = qg.new_workspace(qg.qg_paged_attention_workspace_bytes(40, 16, 2, 128))
    for lens, H, Hkv in (([900] * 40, 16, 2), ([5000], 8, 8), ([64, 0], 16, 1), ([3] * 17, 2, 2), ([2500, 1], 16, 2)):
        k, v, _, _, tables, K, V = cache_of(lens, Hkv, 128, 16, torch.bfloat16, gen(len(lens)))
        q = torch.randn(len(lens), H, 128, generator=gen(1))
        assert qg.qg_paged_attention_workspace_bytes(len(lens), H, Hkv, 128) <= workspace.numel()
        out, _ = qg.qg_paged_attention(q.cuda(), k.cuda(), v.cuda(), tables.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), 0.08, workspace=workspace)
        want, _, so, _ = attention_want(q, K, V, tables, lens, [0] * len(lens), 0, 16, 0.08)
        near(out.cpu().double(), want, so, torch.float32)


def test_step_calls_in_a_graph_and_on_another_stream(qg):
    # norm, append, attention captured once and replayed on growing sequences, with eager work in between
    B, H, Hkv, D, page = 3, 8, 2, 64, 16
    g = gen(21)
    k, v = (torch.zeros(64, Hkv, page, D, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    tables = torch.randperm(60, generator=g).to(torch.int32).view(B, 20).cuda()
    rows, positions = torch.arange(B, dtype=torch.int32).cuda(), torch.zeros(B, dtype=torch.int32).cuda()
    lens, x, w = torch.ones(B, dtype=torch.int32).cuda(), torch.zeros(B, (H + 2 * Hkv) * D).cuda(), torch.ones((H + 2 * Hkv) * D).cuda()
    workspace = qg.new_workspace(qg.qg_paged_attention_workspace_bytes(B, H, Hkv, D))

    def step(kc, vc):
        y, _, _ = qg.qg_rms_norm(x, w)
        q, nk, nv = (y[:, a * D: b * D].view(B, b - a, D) for a, b in ((0, H), (H, H + Hkv), (H + Hkv, H + 2 * Hkv)))
        q = qg.qg_kv_append(kc, vc, tables, rows, positions, nk, nv, q=q)
        return qg.qg_paged_attention(q, kc, vc, tables, lens, 0.125, workspace=workspace)[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(k, v)                                                          # also: a stream of its own
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(k, v)
    k2, v2 = torch.zeros_like(k), torch.zeros_like(v)
    k.zero_(), v.zero_()
    for i in range(40):
        x.copy_(torch.randn(x.shape, generator=g))
        positions.fill_(i)
        lens.fill_(i + 1)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, step(k2, v2)) and torch.equal(k, k2) and torch.equal(v, v2)
        torch.cuda.synchronize()


# --- the pages' book --------------------------------------------------------------------------------------------

def resize_plain(tables, lens, refs, page, new, planes):
    tables, lens, refs = tables.copy(), lens.copy(), refs.copy()
    rows, columns = tables.shape
    has_id = lambda i: 0 <= i < len(refs)  # noqa: E731
    old = np.clip(lens, 0, columns * page)
    new = np.clip(new, 0, columns * page)
    had, has = -(-old // page), -(-new // page)
    before = refs.copy()
    t0 = tables.copy()
    for b in range(rows):
        for j in range(has[b], had[b]):
            if has_id(tables[b, j]):
                refs[tables[b, j]] -= 1
            tables[b, j] = -1
    wants = []
    for b in range(rows):
        if new[b] > old[b] and old[b] % page and has_id(tables[b, had[b] - 1]) and refs[tables[b, had[b] - 1]] > 1:
            wants.append((b, had[b] - 1, True))
        wants += [(b, j, False) for j in range(had[b], has[b])]
    free = [i for i in range(len(refs)) if refs[i] == 0]
    if len(free) < len(wants):
        return t0, lens, before, len(wants) - len(free), planes
    planes = [p.copy() for p in planes]
    moves = []
    for (b, j, copy), i in zip(wants, free):
        if copy:
            moves.append((tables[b, j], i))
        tables[b, j] = i
    for a, i in moves:
        refs[a] -= 1
        for p in planes:
            p[:, i] = p[:, a]
    for (_, _, _), i in zip(wants, free):
        refs[i] += 1
    return tables, new.astype(np.int32), refs, 0, planes


def book(seed, rows, columns, pages, page, fill=0.6, shared=True):
    r = np.random.default_rng(seed)
    ids = list(r.permutation(pages))
    tables, lens = np.full((rows, columns), -1, np.int32), np.zeros(rows, np.int32)
    for b in range(rows):
        if shared and b and r.random() < 0.4:
            n = int(r.integers(0, lens[b - 1] + 1))
            k = -(-n // page)
            tables[b, :k], lens[b] = tables[b - 1, :k], n
            continue
        k = min(int(r.integers(0, max(1, int(columns * fill)) + 1)), len(ids))
        tables[b, :k] = [ids.pop() for _ in range(k)]
        lens[b] = max(0, k * page - int(r.integers(0, page))) if k else 0
    refs = np.bincount(tables[tables >= 0], minlength=pages).astype(np.int32)
    if len(ids) > 3:
        refs[ids.pop()] += 2                                                # pages held by others
    return tables, lens, refs


BOOKS = [(1, 1, 1, 16), (1, 4, 9, 16), (5, 8, 64, 16), (64, 33, 3000, 32), (300, 20, 7001, 16), (7, 600, 5000, 128), (1500, 5, 9000, 16), (3, 70, 40000, 64)]


def planes_of(seed, pages, shapes=((2, 48), (1, 4112), (3, 16))):
    r = np.random.default_rng(seed)
    return [r.integers(0, 255, (layers, pages, size), dtype=np.uint8) for layers, size in shapes]


def up(*arrays):
    return [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in arrays]


@pytest.mark.parametrize("rows,columns,pages,page", BOOKS)
@pytest.mark.parametrize("in_place", [False, True])
def test_resize_matches_the_loops(qg, rows, columns, pages, page, in_place):
    case("resize", rows, columns, pages, page, in_place)
    r = np.random.default_rng(rows + pages)
    tables, lens, refs = book(rows + 1, rows, columns, pages, page)
    for what in ("step", "random", "much", "end"):
        new = {"step": lens + 1, "random": r.integers(-5, columns * page + 9, rows), "much": np.full(rows, columns * page), "end": np.zeros(rows)}[what].astype(np.int32)
        planes = planes_of(3, pages) if pages <= 9000 else []
        want = resize_plain(tables, lens, refs, page, new, planes)
        t, n, f, nw = up(tables, lens, refs, new)
        p = up(*planes)
        got = qg.qg_pages_resize(t, n, f, page, nw, planes=p, out=(t, n, f) if in_place else None)
        assert int(got[3]) == want[3], what
        for a, b in zip(got[:3], want[:3]):
            assert np.array_equal(a.cpu().numpy(), b), what
        for a, b in zip(p, want[4]):
            assert np.array_equal(a.cpu().numpy(), b), what
        if not in_place:
            assert all(np.array_equal(a.cpu().numpy(), b) for a, b in ((t, tables), (n, lens), (f, refs)))
        if want[3] == 0:
            tables, lens, refs = want[:3]


@pytest.mark.parametrize("rows,columns,pages,page", BOOKS)
def test_fork_matches_the_loops(qg, rows, columns, pages, page):
    case("fork", rows, columns, pages, page)
    r = np.random.default_rng(rows)
    tables, lens, refs = book(rows + 2, rows, columns, pages, page)
    for parents in (np.arange(rows), r.integers(-2, rows + 2, rows), np.full(rows, -1), np.zeros(rows)):
        parents = parents.astype(np.int32)
        got = [a.cpu().numpy() for a in qg.qg_pages_fork(*up(tables, lens, refs, parents))]
        t, n, f = np.full_like(tables, -1), np.zeros_like(lens), refs.copy()
        for b, parent in enumerate(parents):
            if 0 <= parent < rows:
                t[b], n[b] = tables[parent], lens[parent]
        np.subtract.at(f, tables[tables >= 0], 1)
        np.add.at(f, t[t >= 0], 1)
        assert np.array_equal(got[0], t) and np.array_equal(got[1], n) and np.array_equal(got[2], f)


@pytest.mark.parametrize("rows,columns,pages,page", BOOKS)
@pytest.mark.parametrize("in_place", [False, True])
def test_compact_matches_the_loops(qg, rows, columns, pages, page, in_place):
    case("compact", rows, columns, pages, page, in_place)
    for fill in (0.0, 0.3, 1.0):
        tables, lens, refs = book(rows + 3, rows, columns, pages, page, fill)
        planes = planes_of(4, pages) if pages <= 9000 else []
        t, f = up(tables, refs)
        p = up(*planes)
        got = qg.qg_pages_compact(t, f, planes=p, out=(t, f) if in_place else None)
        used = [i for i in range(pages) if refs[i] > 0]
        n = len(used)
        to = {a: b for a, b in zip([i for i in used if i >= n], [i for i in range(n) if refs[i] <= 0])}
        wt = np.vectorize(lambda i: to.get(i, i), otypes=[np.int32])(tables)
        wf = np.array([refs[i] if i < n else 0 for i in range(pages)], np.int32)
        for a, b in to.items():
            wf[b] = refs[a]
            for q in planes:
                q[:, b] = q[:, a]
        assert int(got[2]) == n and np.array_equal(got[0].cpu().numpy(), wt) and np.array_equal(got[1].cpu().numpy(), wf)
        for a, b in zip(p, planes):
            assert np.array_equal(a.cpu().numpy(), b)


def test_copy_pages(qg):
    planes = planes_of(5, 100, ((1, 16), (4, 65536), (2, 4096 + 16), (1, 8208)))
    p = up(*planes)
    pairs = np.array([[3, 50], [3, 51], [99, 0], [-1, 60], [5, 100], [7, 99 - 9]], np.int32)
    qg.qg_pages_copy([t[..., None] for t in p], up(pairs)[0])
    for a, b in pairs:
        if 0 <= a < 100 and 0 <= b < 100:
            for q in planes:
                q[:, b] = q[:, a]
    assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(p, planes))


def test_numbers_that_are_none_stay_with_their_head(qg):
    # an 8-bit cell of a head with a NaN or infinity is NaN, scale and codes; its neighbours are as they would be; attention over such a
    # cell is NaN for the heads that read it, and only where it is read
    H, D, page = 3, 64, 16
    k, v = (torch.zeros(4, H, page, D).to(F8).cuda() for _ in "kv")
    ks, vs = (torch.ones(4, H, page).cuda() for _ in "kv")
    t = torch.tensor([[2, 1]], dtype=torch.int32).cuda()
    new = torch.randn(20, H, D, generator=gen(31))
    new[5, 1, 7], new[9, 2, 60] = math.nan, math.inf
    at = torch.arange(20, dtype=torch.int32).cuda()
    qg.qg_kv_append(k, v, t, torch.zeros_like(at), at, new.cuda(), new.cuda(), k_scale=ks, v_scale=vs)
    for cells, scales in ((k, ks), (v, vs)):
        cells, scales = cells.cpu().float(), scales.cpu()
        bad = torch.zeros(4, H, page, dtype=torch.bool)
        bad[2, 1, 5] = bad[2, 2, 9] = True
        assert torch.equal(torch.isnan(scales), bad) and torch.equal(torch.isnan(cells).all(-1), bad) and torch.equal(torch.isnan(cells).any(-1), bad)
    q, n = torch.randn(1, H, D, generator=gen(32)).cuda(), torch.tensor([20], dtype=torch.int32).cuda()
    for first, none in ((0, [False, True, True]), (6, [False, False, True]), (10, [False, False, False])):
        out, lse = qg.qg_paged_attention(q, k, v, t, n, 0.1, first=torch.tensor([first], dtype=torch.int32).cuda(), k_scale=ks, v_scale=vs, lse=True)
        assert torch.isnan(out[0]).all(-1).tolist() == none == torch.isnan(out[0]).any(-1).tolist() == torch.isnan(lse[0]).tolist()


@pytest.mark.parametrize("lens", [[40, 7], [9000, 130]])
def test_queries_that_are_no_numbers_come_out_as_none(qg, lens):
    # a head whose q holds a NaN or an infinity has no score that is a number: its output is NaN, whether its keys are looked at by one
    # workgroup or many; the other heads and sequences are as they would be
    for ct in (torch.bfloat16, torch.float16):
        k, v, _, _, tables, _, _ = cache_of(lens, 2, 64, 16, ct, gen(41))
        q = torch.randn(2, 6, 64, generator=gen(42))
        args = (k.cuda(), v.cuda(), tables.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), 0.1)
        good, glse = qg.qg_paged_attention(q.cuda(), *args, lse=True)
        q[0, 1, 5], q[0, 4], q[1, 3, 63] = math.nan, math.nan, math.inf
        out, lse = qg.qg_paged_attention(q.cuda(), *args, lse=True)
        none = torch.zeros(2, 6, dtype=torch.bool)
        none[0, 1] = none[0, 4] = none[1, 3] = True
        assert torch.equal(torch.isnan(out).all(-1).cpu(), none) and torch.equal(torch.isnan(lse).cpu(), none)
        assert torch.equal(out.cpu()[~none], good.cpu()[~none]) and torch.equal(lse.cpu()[~none], glse.cpu()[~none])


def test_books_in_a_graph(qg):
    # a step, a fork and a compaction captured once and replayed on changing books, with the caller's own work in between
    rows, columns, pages, page = 40, 12, 700, 16
    planes = planes_of(8, pages)
    held = [torch.from_numpy(a).cuda() for a in book(77, rows, columns, pages, page)]
    p = up(*planes)
    new, parents = torch.zeros(rows, dtype=torch.int32).cuda(), torch.zeros(rows, dtype=torch.int32).cuda()
    space = torch.empty(qg.qg_pages_workspace_bytes(rows, columns, pages), dtype=torch.uint8, device="cuda")

    def step():
        t, n, f, lacking = qg.qg_pages_resize(*held, page, new, planes=p, workspace=space)
        t, n, f = qg.qg_pages_fork(t, n, f, parents)
        t, f, live = qg.qg_pages_compact(t, f, planes=p, workspace=space)
        return t, n, f, lacking, live

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    r = np.random.default_rng(5)
    for i in range(6):
        new.copy_(torch.from_numpy(np.minimum(held[1].cpu().numpy() + r.integers(-3, 20, rows), columns * page).astype(np.int32)))
        parents.copy_(torch.from_numpy(np.where(r.random(rows) < 0.8, np.arange(rows), r.integers(-1, rows, rows)).astype(np.int32)))
        before = [t.clone() for t in p]
        graph.replay()
        torch.cuda.synchronize()
        got, moved = [t.clone() for t in out], [t.clone() for t in p]
        for a, b in zip(p, before):
            a.copy_(b)
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(a, b) for a, b in zip(moved, p))
        for a, b in zip(held, got):
            a.copy_(b)


# --- refusals of the Python entry points ------------------------------------------------------------------------

def test_wrong_arguments_are_refused(qg):
    f = lambda *n: torch.zeros(*n, device="cuda")  # noqa: E731
    i = lambda *n: torch.zeros(*n, dtype=torch.int32, device="cuda")  # noqa: E731
    x, w = f(4, 64), f(64)
    for bad in (lambda: qg.qg_rms_norm(x.cpu(), w), lambda: qg.qg_rms_norm(x, w[:63]), lambda: qg.qg_rms_norm(x.t(), f(4)),
                lambda: qg.qg_rms_norm(x, w, residual=f(4, 63)), lambda: qg.qg_rms_norm(x, w, residual=x.half()),
                lambda: qg.qg_rms_norm(x, w, dtype=F8, group=48), lambda: qg.qg_rms_norm(x, w, group=32), lambda: qg.qg_rms_norm(x, w, dtype=torch.int8),
                lambda: qg.qg_rms_norm(x, w, h=f(4, 64)), lambda: qg.qg_rms_norm(x, w, scales=f(4, 1)), lambda: qg.qg_rms_norm(x.double(), w),
                lambda: qg.qg_rms_norm(x, w, y=f(4, 65)[:, :64])):
        with pytest.raises((ValueError, RuntimeError)):
            bad()
    k = f(6, 2, 16, 64).bfloat16()
    t, n, q, kv = i(3, 2), i(3), f(3, 4, 64), f(3, 2, 64)
    for bad in (lambda **a: qg.qg_paged_attention(q, k.float(), k.float(), t, n, 1.0), lambda: qg.qg_paged_attention(q, k, k[:5], t, n, 1.0),
                lambda: qg.qg_paged_attention(f(3, 5, 64), k, k, t, n, 1.0), lambda: qg.qg_paged_attention(f(3, 4, 32), k, k, t, n, 1.0),
                lambda: qg.qg_paged_attention(q, k, k, t, i(2), 1.0), lambda: qg.qg_paged_attention(q, k, k, t.long(), n, 1.0),
                lambda: qg.qg_paged_attention(f(4, 4, 64), k, k, t, i(4), 1.0), lambda: qg.qg_paged_attention(q, k, k, t, n, 1.0, window=-1),
                lambda: qg.qg_paged_attention(q, k.to(F8), k.to(F8), t, n, 1.0), lambda: qg.qg_paged_attention(q.transpose(0, 1), k, k, t, n, 1.0),
                lambda: qg.qg_paged_attention(q, f(6, 2, 24, 64).bfloat16(), f(6, 2, 24, 64).bfloat16(), t, n, 1.0),
                lambda: qg.qg_paged_attention(q, k, k, t, n, 1.0, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")),
                lambda: qg.qg_paged_attention(q, k, k, t, n, 1.0, out=q.half()), lambda: qg.qg_paged_attention(q[:, :, ::2], k[..., :32].contiguous(), k[..., :32].contiguous(), t, n, 1.0),
                lambda: qg.qg_kv_append(k, k, t, n, n, kv, kv.half()), lambda: qg.qg_kv_append(k, k, t, n[:2], n, kv, kv),
                lambda: qg.qg_kv_append(k, k, t, n, n, kv, kv, cos_sin=f(9, 66)), lambda: qg.qg_kv_append(k, k, t, n, n, kv, kv, cos_sin=f(9, 7)),
                lambda: qg.qg_kv_append(k, k, t, n, n, kv, f(3, 2, 32)), lambda: qg.qg_kv_append(k, k, t, n, n, f(3, 130)[:, 1:129].view(3, 2, 64), kv)):
        with pytest.raises((ValueError, RuntimeError)):
            bad()
    r = i(9)
    for bad in (lambda: qg.qg_pages_resize(t, n, r, 0, n), lambda: qg.qg_pages_resize(t, n, r, 16, i(2)), lambda: qg.qg_pages_fork(t, n, r, n, out=(t, n, r)),
                lambda: qg.qg_pages_resize(t, n, r, 16, n, planes=[f(1, 8, 4)]), lambda: qg.qg_pages_resize(t, n, r, 16, n, planes=[f(1, 9, 3)]),
                lambda: qg.qg_pages_resize(t, n, r, 16, n, planes=[f(1, 9, 4)] * 9), lambda: qg.qg_pages_compact(t, r, workspace=i(1).view(torch.uint8)),
                lambda: qg.qg_pages_copy([f(1, 9, 4)], i(3, 3))):
        with pytest.raises((ValueError, RuntimeError)):
            bad()
    torch.cuda.synchronize()

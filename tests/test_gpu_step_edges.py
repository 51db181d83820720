"""The calls between the products of a token's step where values lie on the edge of what their types hold: quotients in the middle of two codes,
numbers so small that their scale would be zero, small probabilities beside large ones,
infinite cells, the longest rows, the most of them.

Exact comparisons unless a test derives a bound of its own."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def qg():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2307_03738_amd import binding
    binding.lib()
    return binding


def gen(seed):
    return torch.Generator().manual_seed(seed)


def codes(y, scales):
    """y / scale in fp32, then to nearest even."""
    return (y / scales).clamp(-448, 448).to(F8).view(torch.uint8)


@pytest.mark.parametrize("size", [1.0, 3e-30, 2e30])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16, torch.float32])
def test_codes_of_the_cache_are_the_quotients_to_nearest_even(qg, dt, size):
    # values and their largest one have 8 bits each in bf16, so a quotient in the middle of two codes is common
    print("[case] append codes", dt, size, flush=True)
    if dt is torch.float16:
        size = min(max(size, 1e-2), 100.0)
    T, H, D, page = 2000, 4, 128, 64
    x = (torch.randn(T, 2, H, D, generator=gen(1)) * size).to(dt)
    x[:, 1, 1] = x[:, 1, 1].to(torch.bfloat16).to(dt)
    pages = -(-T // page)
    k, v = (torch.zeros(pages, H, page, D).to(F8).cuda() for _ in "kv")
    ks, vs = (torch.zeros(pages, H, page).cuda() for _ in "kv")
    at, d = torch.arange(T, dtype=torch.int32).cuda(), x.cuda()
    tables = torch.arange(pages, dtype=torch.int32).view(1, -1).cuda()
    qg.qg_kv_append(k, v, tables, torch.zeros_like(at), at, d[:, 0], d[:, 1], k_scale=ks, v_scale=vs)
    for cells, scales, want in ((k, ks, x[:, 0]), (v, vs, x[:, 1])):
        s = scales.cpu().transpose(1, 2).reshape(-1, H)[:T, :, None]
        got = cells.cpu().view(torch.uint8).transpose(1, 2).reshape(-1, H, D)[:T]
        assert torch.equal(s[..., 0], want.float().abs().amax(2) / 448)
        off = got != codes(want.float(), s)
        assert not off.any(), f"{int(off.sum())} of {off.numel()} codes"


@pytest.mark.parametrize("rows,K,group", [(64, 4096, 128), (3, 4096, 0), (700, 512, 64), (2, 16384, 0), (5, 4099, 0), (40, 96, 24), (3, 20000, 8)])
def test_codes_of_the_norm_are_the_quotients_to_nearest_even(qg, rows, K, group):
    # tiny rows under eps = 1: 1 / sqrt(mean + eps) is 1, and y is x
    x = (torch.randn(rows, K, generator=gen(2)) * 1e-6).to(torch.bfloat16)
    y, _, s = qg.qg_rms_norm(x.cuda(), torch.ones(K).cuda(), 1.0, dtype=F8, group=group)
    wide = s.cpu().repeat_interleave(group or K, 1)
    assert torch.equal(s.cpu(), x.float().abs().view(rows, -1, group or K).amax(2) / 448)
    off = y.cpu().view(torch.uint8) != codes(x.float(), wide)
    assert not off.any(), f"{int(off.sum())} of {off.numel()} codes"


# the largest of a group: its scale is 0 in fp32 up to 224 steps of 2^-149 (1 is taken), then a multiple of 2^-149
TINY = [(1e-44, True), (224 * 2.0 ** -149, True), (225 * 2.0 ** -149, False), (448 * 2.0 ** -149, False), (1e-41, False)]


@pytest.mark.parametrize("most,one", TINY)
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_tiny_heads_are_stored_as_numbers(qg, most, one, dt):
    print("[case] append tiny", dt, most, flush=True)
    H, D, page = 3, 64, 16
    x = torch.zeros(4, H, D)
    x[1, 1, 5], x[2, 0], x[3, 2, :9] = most, torch.linspace(-most, most, D), most
    x = x.to(dt)
    x[0] = torch.randn(H, D, generator=gen(3)).to(dt)
    k, v = (torch.zeros(1, H, page, D).to(F8).cuda() for _ in "kv")
    ks, vs = (torch.zeros(1, H, page).cuda() for _ in "kv")
    at = torch.arange(4, dtype=torch.int32).cuda()
    qg.qg_kv_append(k, v, torch.zeros(1, 1, dtype=torch.int32).cuda(), torch.zeros_like(at), at, x.cuda(), x.cuda(), k_scale=ks, v_scale=vs)
    want = x.float().abs().amax(2) / 448
    want = torch.where(want == 0, 1.0, want)
    if dt is torch.float32:
        assert (want[1, 1] == 1) == one
    for cells, scales in ((k, ks), (v, vs)):
        s = scales.cpu()[0, :, :4].t()
        assert torch.equal(s, want)
        assert torch.equal(cells.cpu().view(torch.uint8)[0, :, :4].transpose(0, 1) & 0x7f, codes(x.float(), s[..., None]) & 0x7f)
    q = torch.randn(1, H, D, generator=gen(4)).cuda()
    out, lse = qg.qg_paged_attention(q, k, v, torch.zeros(1, 1, dtype=torch.int32).cuda(), at[:1] + 4, 0.1, k_scale=ks, v_scale=vs, lse=True)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("most,one", TINY)
@pytest.mark.parametrize("K,group", [(128, 32), (128, 0), (90, 9), (75, 0), (4096, 0)])
def test_tiny_rows_of_the_norm_are_stored_as_numbers(qg, most, one, K, group):
    # rows of one under a tiny weight: y is the weight
    print("[case] norm tiny", most, K, group, flush=True)
    w = torch.zeros(K)
    w[3], w[K // 2] = most, -most
    x = torch.ones(5, K)
    y, _, s = qg.qg_rms_norm(x.cuda(), w.cuda(), 0.0, dtype=F8, group=group)
    want = w.abs().view(-1, group or K).amax(1) / 448
    assert (want[0] == 0) == one
    want = torch.where(want == 0, 1.0, want).expand(5, -1)
    assert torch.equal(s.cpu(), want)
    assert torch.equal(y.cpu().view(torch.uint8) & 0x7f, codes(w, want.repeat_interleave(group or K, 1)) & 0x7f)


@pytest.mark.parametrize("D,H,n", [(64, 4, 900), (128, 4, 5000), (128, 1, 70), (256, 2, 2000), (80, 16, 3000)])
@pytest.mark.parametrize("nats", [6, 9, 12, 15, 17, 20])
@pytest.mark.parametrize("ct", [torch.bfloat16, torch.float16, F8])
def test_many_small_probabilities_beside_large_ones(qg, ct, nats, D, H, n):
    # Every 16th key is `nats` above the others and has values of 0, the others have 1: out is the others' share alone, and has to be right relative to
    # itself.  Scores are exact; exp errs by 4 U and U of the score, the sums by sqrt(n) U each, p by 2^-22 of itself or 2^-43 of the largest, and
    # out is rounded once.
    print("[case] small p", ct, nats, D, H, n, flush=True)
    page, pages = 16, -(-n // 16)
    k, v = torch.zeros(pages, 1, page, D), torch.ones(pages, 1, page, D)
    k[:, :, 0, 0], v[:, :, 0] = nats, 0
    s = torch.ones(pages, 1, page).cuda() if ct is F8 else None
    q = torch.zeros(1, H, D)
    q[..., 0] = 1
    out, lse = qg.qg_paged_attention(q.cuda(), k.to(ct).cuda(), v.to(ct).cuda(), torch.arange(pages, dtype=torch.int32).view(1, -1).cuda(),
                                     torch.tensor([n], dtype=torch.int32).cuda(), 1.0, k_scale=s, v_scale=s, lse=True)
    big, nats = pages, k.to(ct).float().max().item()                        # (17 is 16 in e4m3)
    total = big * math.exp(nats) + n - big
    want = (n - big) / total
    e = 2 * (2.0 ** -22 + 2.0 ** -43 * math.exp(nats) + (4 + 2 * nats + math.sqrt(n)) * U) + U
    off = (out.cpu().double() / want - 1).abs().max().item()
    assert off <= e, f"off by {off:.2e} of itself, {e:.2e} allowed"
    assert (lse.cpu().double() - math.log(total)).abs().max().item() <= e + 2 * U * math.log(total)


def formula(q, K, V, scale):
    """(out, lse, largest error of a score) of one head over keys K, V [n][D], infinities and all."""
    q, K, V = q.double(), K.double(), V.double()
    s = (K * q).sum(1) * scale
    p = torch.softmax(s, 0)
    finite = torch.isfinite(K).all(1)
    delta = (len(q) + 8) * U * scale * (K[finite].abs() @ q.abs()).max() + 4 * U + 2 * U * s[finite].abs().max()
    return (p[:, None] * V).sum(0), torch.logsumexp(s, 0), float(delta)


def same(got, want, slack, dtype):
    """NaN and infinities where they belong, other values near."""
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"NaN: {int(torch.isnan(got).sum())}, not {int(torch.isnan(want).sum())}"
    assert torch.equal(torch.isinf(got), torch.isinf(want)) and torch.equal(got[torch.isinf(want)], want[torch.isinf(want)])
    at = torch.isfinite(want)
    bound = slack + (want.abs() + slack) * {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype] + 2.0 ** -25
    assert ((got - want).abs() <= bound)[at].all(), float(((got - want).abs() - bound)[at].max())


@pytest.mark.parametrize("lens", [[40, 7, 129], [9000, 600, 1]])
@pytest.mark.parametrize("D", [64, 80, 128, 256])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("ct", [torch.bfloat16, torch.float16])
def test_infinite_cells_are_what_they_are_in_the_formula(qg, ct, dt, D, lens):
    print("[case] infinite cells", ct, dt, D, lens, flush=True)
    H, Hkv, page, scale = 6, 2, 16, 0.1
    B, need = len(lens), [-(-n // page) for n in lens]
    pages = sum(need)
    tables = torch.full((B, max(need)), -1, dtype=torch.int32)
    order, at = torch.randperm(pages, generator=gen(5)).to(torch.int32), 0
    for b, n in enumerate(need):
        tables[b, :n], at = order[at:at + n], at + n
    g = gen(6)
    k, v = (torch.randn(pages, Hkv, page, D, generator=g).to(ct) for _ in "kv")
    q = torch.randn(B, H, D, generator=g).to(dt)
    q[:, :, 3], q[:, :, 7] = 1, -2                                       # one part each, whose others are 0
    q[:, 1, 11] = 0
    cell = lambda b, i: (int(tables[b, i // page]), slice(None), i % page)  # noqa: E731
    for b, n in enumerate(lens):
        for i, d, x in ((0, 5, math.inf), (n - 1, 9, -math.inf), (n // 2, 20, math.inf), (n // 3, 20, -math.inf), (n // 4, 21, math.inf), (n // 5, 21, math.inf)):
            v[cell(b, i)][:, d] = x
        if n > 30:
            k[cell(b, 17)][:, 3] = -math.inf                               # q is positive there: the key counts for nothing
            k[cell(b, 18)][:, 7] = math.inf                                # q is negative
            k[cell(b, n - 2)][0, 12] = math.inf                            # one key head: of heads 0, 1 and 2 those with positive q are NaN
            k[cell(b, n - 4)][1, 11] = -math.inf
            # a key far below the others, whose p has no place in fp32, has an infinite value
            k[cell(b, 25)][:, 3], v[cell(b, 25)][:, 30] = -3000, math.inf
    out, lse = qg.qg_paged_attention(q.cuda(), k.cuda(), v.cuda(), tables.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), scale, lse=True)
    for b, n in enumerate(lens):
        at = torch.arange(n)
        for h in range(H):
            cells = (tables[b, at // page].long(), h // (H // Hkv), at % page)
            want, wlse, delta = formula(q[b, h], k[cells], v[cells], scale)
            e = 2 * (delta + 2.0 ** -16 + math.sqrt(n) * U)
            same(out[b, h].cpu().double(), want, e * v[torch.isfinite(v)].abs().max().item(), dt)
            if not torch.isnan(want).all():
                same(lse[b, h].cpu().double(), wlse, e + 2 * U * float(wlse.abs()), torch.float32)


def test_values_past_the_range_of_f16_come_out_infinite(qg):
    H, D, page, n = 2, 64, 16, 300
    k, v = (torch.zeros(-(-n // page), H, page, D, dtype=torch.float16).cuda() for _ in "kv")
    at, tables = torch.arange(n, dtype=torch.int32).cuda(), torch.arange(-(-n // page), dtype=torch.int32).view(1, -1).cuda()
    new = torch.randn(n, H, D, generator=gen(7))
    new[100, 1, 6], new[299, 0, 2] = 7e4, -1e30
    qg.qg_kv_append(k, v, tables, torch.zeros_like(at), at, torch.randn(n, H, D, generator=gen(8)).cuda(), new.cuda())
    q = torch.randn(1, H, D, generator=gen(9)).cuda()
    for window in (0, 250, 190):
        out, _ = qg.qg_paged_attention(q, k, v, tables, at[-1:] + 1, 0.1, window=window)
        want = torch.zeros(H, D)
        want[0, 2], want[1, 6] = -math.inf, math.inf if window != 190 else 0
        assert torch.equal(torch.where(torch.isinf(out[0].cpu()), out[0].cpu(), 0.0), want) and not torch.isnan(out).any()


@pytest.mark.parametrize("value", [3.3, 1.1, 0.9])
@pytest.mark.parametrize("rows,K,residual", [(2, 65536 + 7, False), (2, (1 << 20) + 3, True), (1, 1 << 24, False), (1, (1 << 24) - 1, True)])
def test_norm_of_the_longest_rows(qg, rows, K, residual, value):
    # equal values, whose sum's roundings do not average out.  A sum of K squares in pieces of at most 64 terms and ten levels of a tree errs
    # by at most 74 U of itself, half of that under the root, six roundings around it: 43 U of |y|
    print("[case] long rows", rows, K, residual, value, flush=True)
    x = torch.full((rows, K), value)
    r = torch.full((rows, K), value / 2) if residual else None
    y, _, _ = qg.qg_rms_norm(x.cuda(), torch.ones(K).cuda(), 0.0, residual=None if r is None else r.cuda())
    assert (y.double() - 1).abs().max().item() <= 43 * U + U


def test_norm_of_more_rows_than_one_launch_takes(qg):
    rows, K = (1 << 23) + 5, 3
    print("[case] rows", rows, K, flush=True)
    g = torch.Generator(device="cuda").manual_seed(11)
    x = torch.randn(rows, K, generator=g, device="cuda").to(torch.float16)
    r = torch.randn(rows, K, generator=g, device="cuda").to(torch.float16)
    w = torch.tensor([1.0, 0.5, 2.0]).cuda()
    at = torch.tensor([0, 1, rows // 2, (1 << 23) - 1, 1 << 23, rows - 1]).cuda()
    y, h, _ = qg.qg_rms_norm(x, w, residual=r)
    part = qg.qg_rms_norm(x[at].contiguous(), w, residual=r[at].contiguous())
    assert torch.equal(y[at], part[0]) and torch.equal(h[at], part[1]) and torch.equal(h[-1 << 20:], (x[-1 << 20:].float() + r[-1 << 20:].float()).half())
    y, _, s = qg.qg_rms_norm(x, w, dtype=F8, group=1)
    part = qg.qg_rms_norm(x[at].contiguous(), w, dtype=F8, group=1)
    assert torch.equal(y.view(torch.uint8)[at], part[0].view(torch.uint8)) and torch.equal(s[at], part[2])


def test_append_of_more_tokens_than_one_launch_takes(qg):
    T, D, page, n = (1 << 23) + 5, 8, 16, 48
    print("[case] tokens", T, flush=True)
    g = torch.Generator(device="cuda").manual_seed(12)
    q, k, v = (torch.randn(T, 1, D, generator=g, device="cuda").to(torch.bfloat16) for _ in "qkv")
    rows, positions = torch.full((T,), -1, dtype=torch.int32).cuda(), torch.zeros(T, dtype=torch.int32).cuda()
    at = torch.cat((torch.arange(n - 10), torch.arange(T - 10, T))).cuda()
    rows[at], positions[at] = 0, torch.arange(n, dtype=torch.int32).cuda()
    kc, vc = (torch.zeros(n // page, 1, page, D, dtype=torch.bfloat16).cuda() for _ in "kv")
    angles = torch.rand(64, 2, generator=g, device="cuda")
    turn = torch.cat((angles.cos(), angles.sin()), 1)
    tables = torch.arange(n // page, dtype=torch.int32).view(1, -1).cuda()
    out = qg.qg_kv_append(kc, vc, tables, rows, positions, k, v, q=q, cos_sin=turn)
    k2, v2 = torch.zeros_like(kc), torch.zeros_like(vc)
    out2 = qg.qg_kv_append(k2, v2, tables, rows[at], positions[at], k[at], v[at], q=q[at], cos_sin=turn)
    assert torch.equal(kc, k2) and torch.equal(vc, v2) and torch.equal(out[at], out2) and torch.equal(vc.view(n, D), v[at, 0])
    assert (out[n:-10] == 0).all()


def test_fork_of_more_rows_than_one_launch_takes(qg):
    rows, pages = (1 << 23) + 5, 64
    print("[case] rows", rows, flush=True)
    tables = (torch.arange(rows, dtype=torch.int32) % pages).view(-1, 1).cuda()
    lens, refs = torch.arange(rows, dtype=torch.int32).cuda() % 7, torch.bincount(tables.view(-1), minlength=pages).to(torch.int32)
    parents = torch.arange(rows, dtype=torch.int32).flip(0).cuda()
    parents[-3] = -1
    t, n, r = qg.qg_pages_fork(tables, lens, refs, parents)
    want = tables.flip(0)
    want[-3] = -1
    wlens = lens.flip(0)
    wlens[-3] = 0
    assert torch.equal(t, want) and torch.equal(n, wlens) and torch.equal(r, torch.bincount(want[want >= 0], minlength=pages).to(torch.int32))


@pytest.mark.parametrize("D", [8, 64, 128, 200, 256])
@pytest.mark.parametrize("ct", [torch.bfloat16, torch.float16, F8])
def test_probabilities_keep_fp32_for_fp32(qg, ct, D):
    # Two keys, with scores 0 and s and values 0 and 1: out = p / (1 + p).  Scores are exact (s has 8 bits, or is the scale of a key of 1); exp errs by 4 U
    # and U of the score, p by 2^-22 of itself in f16 and 2^-24 in bf16 (in two parts of 8 bits it would be off by 107 U here), out is rounded once.
    print("[case] p", ct, D, flush=True)
    s = torch.linspace(-1, 1, 65).to(torch.bfloat16).float()
    n, page = len(s), 16
    k, v = torch.zeros(n, 1, page, D), torch.zeros(n, 1, page, D)
    k[:, 0, 1, 0], v[:, 0, 1] = 1 if ct is F8 else s, 1
    ks = vs = None
    if ct is F8:
        ks, vs = torch.ones(n, 1, page), torch.ones(n, 1, page).cuda()
        ks[:, 0, 1] = s
        ks = ks.cuda()
    q = torch.zeros(n, 2, D)
    q[..., 0] = 1
    out, lse = qg.qg_paged_attention(q.cuda(), k.to(ct).cuda(), v.to(ct).cuda(), torch.arange(n, dtype=torch.int32).view(-1, 1).cuda(),
                                     torch.full((n,), 2, dtype=torch.int32).cuda(), 1.0, k_scale=ks, v_scale=vs, lse=True)
    p = torch.exp(s.double())
    want = (p / (1 + p))[:, None, None]
    e = 2 * (2.0 ** -22 + 6 * U) + U
    assert ((out.cpu().double() / want - 1).abs() <= e).all(), float((out.cpu().double() / want - 1).abs().max() / U)
    assert ((lse.cpu().double() - torch.log(1 + p)[:, None]).abs() <= e).all()


@pytest.mark.parametrize("rows,K,dt,out,group", [(37, 4099, torch.float32, torch.float32, 0), (5, 20000, torch.bfloat16, torch.float16, 0),
                                                 (9, 90, torch.float16, F8, 9), (3, 4099, torch.bfloat16, F8, 0), (300, 1, torch.float32, F8, 1)])
def test_norm_writes_h_over_its_inputs_element_by_element(qg, rows, K, dt, out, group):
    for which in ("x", "residual"):
        x, r = (torch.randn(rows, K, generator=gen(i)).to(dt).cuda() for i in (13, 14))
        w = torch.randn(K, generator=gen(15)).cuda()
        y0, h0, s0 = qg.qg_rms_norm(x, w, 1e-6, residual=r, dtype=out, group=group)
        y, h, s = qg.qg_rms_norm(x, w, 1e-6, residual=r, h=x if which == "x" else r, dtype=out, group=group)
        assert torch.equal(y.view(torch.uint8), y0.view(torch.uint8)) and torch.equal(h, h0) and h.data_ptr() == (x if which == "x" else r).data_ptr()
        assert s is None or torch.equal(s, s0)

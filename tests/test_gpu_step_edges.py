"""The calls between the products of a token's step where values lie on the edge of what their types hold: quotients in the middle of two codes.

Exact comparisons unless a test derives a bound of its own."""
import pytest
import torch

pytestmark = pytest.mark.gpu

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

"""The decoder example with layers of experts against a plain implementation in 64 bits that keeps no cache.

Every token takes all experts, so that what is rounded before the choice cannot change it.  Tolerance on the 2-norm of a row: as in the example without experts (2^-5
with a bf16 cache and two layers); the experts' products round nothing that counts beside that, and the router's product rounds its input to bf16, 2^-8 of a
logit's terms, whose softmax changes by as much at most: one more rounding of the ones counted there, 2^-5 (1 + 1/8) < 2^-4."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

HIDDEN, INNER, H, HKV, D, GROUP, ROWS, PAGE, E = 256, 320, 4, 2, 64, 64, 4, 16, 3


@pytest.fixture(scope="module")
def decoder():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2307_03738_amd import decoder
    return decoder


def wide(m):
    q, s, z = (t.cpu().double() for t in m)
    return s.repeat_interleave(q.shape[1] // s.shape[1], 1) * (q - z.repeat_interleave(q.shape[1] // z.shape[1], 1))


def gated(y, up, down):
    gate, up = (y @ wide(up).t()).chunk(2, 1)
    return gate / (1 + torch.exp(-gate)) * up @ wide(down).t()


def plain(weights, final, xs, eps=1e-5):
    """Hidden state of the last of the tokens xs [n][hidden]."""
    n, h = len(xs), xs.double()
    norm = lambda h, w: h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * w.cpu().double()  # noqa: E731
    ang = torch.arange(n).double()[:, None] * 10000.0 ** (-torch.arange(D // 2).double() / (D // 2))
    c, s = ang.cos()[:, None], ang.sin()[:, None]
    turn = lambda x: torch.cat((x[..., :D // 2] * c - x[..., D // 2:] * s, x[..., D // 2:] * c + x[..., :D // 2] * s), -1)  # noqa: E731
    for w in weights:
        qkv = norm(h, w["norm"]) @ wide(w["qkv"]).t()
        q, k, v = turn(qkv[:, :H * D].view(n, H, D)), turn(qkv[:, H * D:(H + HKV) * D].view(n, HKV, D)), qkv[:, (H + HKV) * D:].view(n, HKV, D)
        k, v = k.repeat_interleave(H // HKV, 1), v.repeat_interleave(H // HKV, 1)
        score = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(D)
        score = score.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -math.inf)
        h = h + torch.einsum("hij,jhd->ihd", score.softmax(-1), v).reshape(n, H * D) @ wide(w["out"]).t()
        y = norm(h, w["norm2"])
        if "router" in w:
            p = (y @ wide(w["router"]).t()).softmax(1)
            h = h + sum(p[:, e, None] * gated(y, w["experts_gate_up"][e], w["experts_down"][e]) for e in range(E))
        else:
            h = h + gated(y, w["gate_up"], w["down"])
    return norm(h, final)[-1]


@pytest.mark.parametrize("bits", [4, 3, 2])
def test_decoder_with_experts_matches_the_whole_history(decoder, bits):
    print("[case] decoder with experts", bits, flush=True)
    weights, final = decoder.random_weights(2, HIDDEN, INNER, H, HKV, D, bits, GROUP, seed=bits, experts=E)
    assert "router" in weights[1] and "router" not in weights[0]
    model = decoder.Decoder(weights, final, H, HKV, D, bits, GROUP, ROWS, pages=24, max_pages=6, page=PAGE, top_k=E)
    history, g = [[] for _ in range(ROWS)], torch.Generator().manual_seed(7)
    for t in range(20):
        live = torch.tensor([True, t < 5, t % 2 == 0, False])
        assert int(model.resize((model.lens.cpu() + live).to(torch.int32).cuda())) == 0
        x = torch.randn(ROWS, HIDDEN, generator=g)
        y = model.step(x.cuda(), live.cuda()).cpu().double()
        for b in range(ROWS):
            if live[b]:
                history[b].append(x[b])
                if t in (0, 1, 4, 18):
                    want = plain(weights, final, torch.stack(history[b]))
                    assert (y[b] - want).norm() <= 2.0 ** -4 * want.norm(), (b, t, float((y[b] - want).norm() / want.norm()))


def test_rows_that_are_passed_over_choose_no_expert(decoder):
    weights, final = decoder.random_weights(2, HIDDEN, INNER, H, HKV, D, 4, GROUP, experts=E)
    model = decoder.Decoder(weights, final, H, HKV, D, 4, GROUP, ROWS, pages=24, max_pages=6, page=PAGE, top_k=2)
    layer, y = model.layers[1], torch.randn(ROWS, HIDDEN, generator=torch.Generator().manual_seed(1)).cuda()
    live = torch.tensor([True, False, True, False]).cuda()
    out = model._experts(layer, y, live)
    assert (out[~live] == 0).all() and torch.isfinite(out).all() and (out[live] != 0).any(1).all()
    # what the others do does not depend on them
    y[~live] = math.nan
    assert torch.equal(model._experts(layer, y, live), out)

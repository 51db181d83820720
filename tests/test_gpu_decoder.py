"""The decoder example against a plain implementation in 64 bits that keeps no cache: every sequence's whole history is
computed anew with the dequantized weights.

Tolerance, on the 2-norm of a row: products of several rows round their input to bf16, 2^-8 of an element at most; the cache's
cells are rounded once, 2^-8 in bf16 and 2^-4 in e4m3.  A layer has three rounded inputs one after the other on each of its
two branches and the cells' rounding in one of them; two layers: 2 (3 + 1) 2^-8 = 2^-5 with a bf16 cache.  Roundings
of e4m3 cells are as independent as values are: at most 2^-4 each, about 2^-5 together after the softmax's averaging, and again so in the
second layer: 2^-5 + 2 * 2^-5 < 2^-3."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

HIDDEN, INNER, H, HKV, D, GROUP, ROWS, PAGE = 256, 512, 4, 2, 64, 64, 5, 16


@pytest.fixture(scope="module")
def decoder():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2307_03738_amd import decoder
    return decoder


def plain(weights, final, xs, eps=1e-5):
    """Hidden state of the last of the tokens xs [n][hidden]."""
    n = len(xs)
    wide = lambda m: (m[1].cpu().double().repeat_interleave(m[0].shape[1] // m[1].shape[1], 1) *  # noqa: E731
                      (m[0].cpu().double() - m[2].cpu().double().repeat_interleave(m[0].shape[1] // m[2].shape[1], 1)))
    norm = lambda h, w: h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * w.cpu().double()  # noqa: E731
    h = xs.double()
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
        gate, up = (norm(h, w["norm2"]) @ wide(w["gate_up"]).t()).chunk(2, 1)
        h = h + (gate / (1 + torch.exp(-gate)) * up) @ wide(w["down"]).t()
    return norm(h, final)[-1]


@pytest.mark.parametrize("cache,bits,bound", [(torch.bfloat16, 4, 2.0 ** -5), (torch.float16, 3, 2.0 ** -5), (torch.float8_e4m3fn, 2, 2.0 ** -3)])
def test_decoder_matches_the_whole_history(decoder, cache, bits, bound):
    print("[case] decoder", cache, bits, flush=True)
    weights, final = decoder.random_weights(2, HIDDEN, INNER, H, HKV, D, bits, GROUP, seed=bits)
    model = decoder.Decoder(weights, final, H, HKV, D, bits, GROUP, ROWS, pages=24, max_pages=6, page=PAGE, cache=cache)
    history = [[] for _ in range(ROWS)]
    g = torch.Generator().manual_seed(7)

    def step(live):
        live = torch.tensor(live)
        lacking = model.resize((model.lens.cpu() + live).to(torch.int32).cuda())
        x = torch.randn(ROWS, HIDDEN, generator=g)
        y = model.step(x.cuda(), live.cuda()).cpu().double()
        assert int(lacking) == 0
        for b in range(ROWS):
            if live[b]:
                history[b].append(x[b])
        return y, live

    def check(y, live):
        for b in range(ROWS):
            if live[b]:
                want = plain(weights, final, torch.stack(history[b]))
                assert (y[b] - want).norm() <= bound * want.norm(), (b, len(history[b]), float((y[b] - want).norm() / want.norm()))

    for t in range(21):
        y, live = step([True, t < 5, t % 2 == 0, False, False])
        if t in (0, 1, 16):
            check(y, live)
    # two branches of row 0 (which share a page that is not full), row 1 ends
    model.fork(torch.tensor([0, -1, 2, 0, 2], dtype=torch.int32).cuda())
    history[3], history[4], history[1] = list(history[0]), list(history[2]), []
    for t in range(14):
        y, live = step([True, False, t < 3, True, True])
        if t in (0, 2, 13):
            check(y, live)
    # row 0 falls back to its first tokens, row 3 ends, the pool is packed, row 1 begins anew
    lens = model.lens.clone()
    lens[0], lens[3] = 9, 0
    model.resize(lens)
    history[0], history[3] = history[0][:9], []
    used = model.compact()
    assert int(model.tables.max()) < int(used) == int((model.refs > 0).sum())
    for t in range(9):
        y, live = step([True, True, False, False, True])
    check(y, live)
    assert model.lens.tolist() == [len(h) for h in history]


def test_example_runs(decoder, capsys):
    decoder.main()
    assert "pages in use" in capsys.readouterr().out


def test_a_full_pool_leaves_the_cells_alone(decoder):
    # 4 pages: two rows fill them, a third row shares one's pages; a resize that lacks pages changes nothing, and neither does the step after it
    print("[case] full pool", flush=True)
    weights, final = decoder.random_weights(1, HIDDEN, INNER, H, HKV, D, 4, GROUP)
    model = decoder.Decoder(weights, final, H, HKV, D, 4, GROUP, 3, pages=4, max_pages=6, page=PAGE)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    g = torch.Generator(device="cuda").manual_seed(3)
    x = lambda: torch.randn(3, HIDDEN, generator=g, device="cuda")  # noqa: E731
    for t in range(32):
        assert int(model.resize(ints(t + 1, t + 1, 0))) == 0
        model.step(x(), ints(1, 1, 0).bool())
    model.fork(ints(0, 1, 0))
    before = [t.clone() for t in [*model.planes, model.tables, model.lens, model.refs]]
    assert int(model.resize(ints(33, 33, 33))) == 3
    model.step(x(), ints(1, 1, 1).bool())
    assert all(torch.equal(a, b) for a, b in zip(before, [*model.planes, model.tables, model.lens, model.refs]))
    # once a row has ended the others go on
    assert int(model.resize(ints(33, 0, 32))) == 0
    at = (int(model.tables[0, 2]), slice(None), 0)
    y = model.step(x(), ints(1, 0, 0).bool())
    assert torch.isfinite(y[0]).all() and not torch.equal(model.k[0][at], before[0][0][at])

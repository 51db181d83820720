"""A decoder's step on packed weights, from the library's calls: how they go together in a server.

    python -m paper_2307_03738_amd.decoder

runs a small batch with random weights: sequences begin, grow token by token, branch, end, and the pool is packed.
Every layer is norm -> q/k/v product -> rotate and store -> attention -> output product -> norm -> gate/up product -> down
product on 2-, 3- or 4-bit weights; hidden states come in and go out (no vocabulary: embedding and sampling are the caller's).
"""
import math
from typing import Dict, List, Sequence

import torch

from . import binding as qg


class Decoder:
    """Layers of packed weights, a paged cache for all of them, and the book of a batch of `rows` sequences (at most 128).

    weights: for each layer a dict of qkv, out, gate_up, down -- (codes, scales, zero-points) of qg_quantize, q, k and v
    and gate and up stacked along the outputs -- and norm, norm2 (fp32 [hidden]); final_norm (fp32 [hidden])."""

    def __init__(self, weights: Sequence[Dict], final_norm: torch.Tensor, heads: int, kv_heads: int, head_dim: int, bits: int, group: int,
                 rows: int, pages: int, max_pages: int, page: int = 16, cache: torch.dtype = torch.bfloat16, base: float = 10000.0,
                 eps: float = 1e-5):
        self.heads, self.kv_heads, self.head_dim, self.bits, self.group, self.eps = heads, kv_heads, head_dim, bits, group, eps
        self.rows, self.page, self.final_norm = rows, page, final_norm
        device = final_norm.device
        self.layers: List[Dict] = []
        spaces: Dict = {}
        for w in weights:
            layer = {"norm": w["norm"], "norm2": w["norm2"]}
            for name in ("qkv", "out", "gate_up", "down"):
                codes, scales, zeros = w[name]
                N, K = codes.shape
                if (N, K) not in spaces:              # one for each shape: products of a stream do not overlap
                    spaces[N, K] = qg.new_workspace(qg.qg_workspace_bytes(N, K, bits, group, rows), device)
                layer[name] = (qg.qg_pack(codes, scales, zeros, bits, group), N, K, spaces[N, K])
            self.layers.append(layer)
        # a page has the same id in all layers
        shape = (len(self.layers), pages, kv_heads, page, head_dim)
        self.k, self.v = (torch.zeros(shape, device=device).to(cache) for _ in "kv")
        scaled = cache is torch.float8_e4m3fn
        self.k_scale, self.v_scale = (torch.zeros(shape[:-1], device=device) if scaled else None for _ in "kv")
        self.planes = [t for t in (self.k, self.v, self.k_scale, self.v_scale) if t is not None]
        self.tables = torch.full((rows, max_pages), -1, dtype=torch.int32, device=device)
        self.lens = torch.zeros(rows, dtype=torch.int32, device=device)
        self.refs = torch.zeros(pages, dtype=torch.int32, device=device)
        half = head_dim // 2
        angles = torch.arange(max_pages * page, device=device).double()[:, None] * base ** (-torch.arange(half, device=device).double() / half)
        self.cos_sin = torch.cat((angles.cos(), angles.sin()), 1).float()
        self.workspace = qg.new_workspace(qg.qg_paged_attention_workspace_bytes(rows, heads, kv_heads, head_dim), device)
        self.order = torch.arange(rows, dtype=torch.int32, device=device)
        self.lacking = torch.zeros(1, dtype=torch.int32, device=device)

    def resize(self, new_lens: torch.Tensor) -> torch.Tensor:
        """Begins (from 0), grows, cuts and ends (0) sequences; the number of pages that were missing, 0 if it was done.  If some were,
        nothing has changed, and step() passes over all rows until a resize has been done."""
        self.lacking = qg.qg_pages_resize(self.tables, self.lens, self.refs, self.page, new_lens, planes=self.planes,
                                          out=(self.tables, self.lens, self.refs))[3]
        return self.lacking

    def fork(self, parents: torch.Tensor) -> None:
        """Row b goes on from where row parents[b] is (-1: is empty)."""
        self.tables, self.lens, self.refs = qg.qg_pages_fork(self.tables, self.lens, self.refs, parents)

    def compact(self) -> torch.Tensor:
        """Moves the pages in use to the pool's lower end; how many there are."""
        return qg.qg_pages_compact(self.tables, self.refs, planes=self.planes, out=(self.tables, self.refs))[2]

    def _product(self, packed, x: torch.Tensor) -> torch.Tensor:
        blob, N, K, space = packed
        return qg.qg_gemm_small(blob, N, K, self.bits, self.group, x, workspace=space)

    def step(self, x: torch.Tensor, live: torch.Tensor) -> torch.Tensor:
        """Hidden states after the last layer of one new token for each row of x [rows][hidden] (fp32) that `live` (bool) marks; its
        place, the last cell of its row, has been made by resize().  The other rows are passed over: nothing is stored
        for them and what comes out is of no use.  Where the last resize lacked pages that holds for all rows, as their last cells are
        those of tokens before (and maybe of other rows)."""
        H, Hkv, D, rows = self.heads, self.kv_heads, self.head_dim, self.rows
        live = live & (self.lacking == 0)
        where = torch.where(live, self.order, -1)
        positions, lens = self.lens - 1, torch.where(live, self.lens, 0)
        update, stream = x, None
        for i, layer in enumerate(self.layers):
            y, stream, _ = qg.qg_rms_norm(update, layer["norm"], self.eps, residual=stream)
            stream = update if stream is None else stream
            qkv = self._product(layer["qkv"], y)
            q, k, v = (qkv[:, a * D: b * D].view(rows, b - a, D) for a, b in ((0, H), (H, H + Hkv), (H + Hkv, H + 2 * Hkv)))
            scales = {} if self.k_scale is None else {"k_scale": self.k_scale[i], "v_scale": self.v_scale[i]}
            q = qg.qg_kv_append(self.k[i], self.v[i], self.tables, where, positions, k, v, q=q, cos_sin=self.cos_sin, **scales)
            seen, _ = qg.qg_paged_attention(q, self.k[i], self.v[i], self.tables, lens, 1 / math.sqrt(D), workspace=self.workspace, **scales)
            update = self._product(layer["out"], seen.view(rows, H * D))
            y, stream, _ = qg.qg_rms_norm(update, layer["norm2"], self.eps, residual=stream)
            gate, up = self._product(layer["gate_up"], y).chunk(2, 1)
            update = self._product(layer["down"], torch.nn.functional.silu(gate) * up)
        return qg.qg_rms_norm(update, self.final_norm, self.eps, residual=stream)[0]


def random_weights(layers: int, hidden: int, inner: int, heads: int, kv_heads: int, head_dim: int, bits: int, group: int, seed: int = 0):
    """Quantized random weights of the right shapes, and the final norm's."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def matrix(N, K):
        return qg.qg_quantize(torch.randn(N, K, generator=g, device="cuda") / math.sqrt(K), bits, group)

    def norm():
        return 1 + 0.1 * torch.randn(hidden, generator=g, device="cuda")

    return [{"qkv": matrix((heads + 2 * kv_heads) * head_dim, hidden), "out": matrix(hidden, heads * head_dim),
             "gate_up": matrix(2 * inner, hidden), "down": matrix(hidden, inner), "norm": norm(), "norm2": norm()} for _ in range(layers)], norm()


def main() -> None:
    hidden, inner, heads, kv_heads, head_dim, bits, group, rows = 1024, 2816, 8, 2, 128, 4, 128, 6
    weights, final = random_weights(2, hidden, inner, heads, kv_heads, head_dim, bits, group)
    model = Decoder(weights, final, heads, kv_heads, head_dim, bits, group, rows, pages=96, max_pages=16, cache=torch.float8_e4m3fn)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    g = torch.Generator(device="cuda").manual_seed(1)
    ends = torch.tensor([40, 17, 3, 0, 0, 25], device="cuda")             # two rows stay empty for branches
    for t in range(60):
        if t == 45:                                                        # rows 3 and 4 branch from row 0, row 2 ends
            model.fork(ints(0, 1, -1, 0, 0, 5))
            ends[3:5] = 60
        grows = (t < ends) | (t >= 45) & (model.lens > 0)
        lacking = model.resize(torch.where(grows, model.lens + 1, model.lens))
        if int(lacking):
            raise SystemExit("the pool is full")
        y = model.step(torch.randn(rows, hidden, generator=g, device="cuda"), grows)
        if not bool(torch.isfinite(y[grows]).all()):
            raise SystemExit("the step gave values that are no numbers")
    live = model.compact()
    print(f"lengths {model.lens.tolist()}, pages in use {int(live)}, the highest {int(model.tables.max())}, shared {int((model.refs > 1).sum())}")


if __name__ == "__main__":
    main()

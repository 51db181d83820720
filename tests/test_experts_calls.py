"""Host side of the calls of a layer of experts: descriptions are laid out as the header has them, and bad ones are refused before
anything is enqueued.  No kernel is launched here."""
import os
import struct
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

ROUTE = dict(logits=64, bias=0, ids=64, weights=64, tokens=3, logits_stride=32, type=0, experts=32, top_k=4, score=0, groups=1, top_groups=1, group_best=1,
             renormalise=1, scale=1.0)
EXPERTS = dict(packed=64, x=64, offsets=64, rows=64, y=128, N=128, K=256, expert_stride=1 << 20, x_rows=5, x_stride=256, slots=9, bits=4, group=64, experts=4,
               x_type=0, y_type=0, gated=0, workspace=64, workspace_bytes=1 << 40)
COMBINE = dict(y=64, slots=64, weights=64, residual=0, out=128, y_rows=9, tokens=3, N=64, residual_stride=0, type=0, out_type=0, top_k=2)
OK, NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = range(6)


@pytest.fixture(scope="module")
def qg():
    from paper_2307_03738_amd import binding
    binding.lib()
    return binding


def test_descriptions_are_laid_out_as_the_header_has_them(qg, tmp_path):
    src = tmp_path / "sizes.c"
    src.write_text("""#include <stddef.h>
#include <stdio.h>
#include "qg.h"
int main(void)
{
    printf("%zu %zu %zu\\n", sizeof(qg_route_desc), sizeof(qg_experts_desc), sizeof(qg_combine_desc));
    printf("%zu %zu %zu\\n", offsetof(qg_route_desc, scale), offsetof(qg_experts_desc, gated), offsetof(qg_combine_desc, top_k));
    return 0;
}
""")
    subprocess.run(["gcc", "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "sizes")], check=True)
    sizes, at = [[int(v) for v in line.split()] for line in subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True, check=True).stdout.splitlines()]
    packed = [qg._ROUTE(*ROUTE.values()), qg._EXPERTS(*{**EXPERTS, "gated": 7}.values()), qg._COMBINE(*COMBINE.values())]
    assert [len(p) for p in packed] == sizes
    assert struct.unpack_from("f", packed[0], at[0])[0] == 1.0
    assert struct.unpack_from("i", packed[1], at[1])[0] == 7 and struct.unpack_from("i", packed[2], at[2])[0] == 2


@pytest.mark.parametrize("change,status", [
    (dict(logits=0), NULL), (dict(ids=0), NULL), (dict(weights=0), NULL), (dict(type=3), UNSUPPORTED), (dict(type=-1), UNSUPPORTED), (dict(score=2), UNSUPPORTED),
    (dict(group_best=0), UNSUPPORTED), (dict(group_best=3), UNSUPPORTED), (dict(experts=1025, logits_stride=1025), UNSUPPORTED), (dict(experts=128, logits_stride=128, top_k=65), UNSUPPORTED),
    (dict(tokens=-1), SHAPE), (dict(experts=0), SHAPE), (dict(top_k=0), SHAPE), (dict(top_k=33), SHAPE), (dict(groups=0), SHAPE), (dict(groups=5), SHAPE),
    (dict(groups=4, top_groups=0), SHAPE), (dict(groups=4, top_groups=5), SHAPE), (dict(groups=8, top_groups=1, top_k=5), SHAPE), (dict(logits_stride=31), SHAPE),
    (dict(tokens=1 << 29), SHAPE), (dict(logits=66), ALIGN), (dict(bias=66), ALIGN), (dict(ids=66), ALIGN), (dict(weights=65), ALIGN), (dict(tokens=0, logits=0, ids=0), OK)])
def test_route_refuses(qg, change, status):
    assert qg.lib().qg_route(qg._ROUTE(*{**ROUTE, **change}.values()), None) == status


def test_plan_refuses(qg):
    plan = qg.lib().qg_expert_plan
    good = [64, 3, 2, 4, 64, 64, 64, None]
    for at, value, status in ((0, 0, NULL), (4, 0, NULL), (5, 0, NULL), (6, 0, NULL), (1, -1, SHAPE), (2, 0, SHAPE), (3, 0, SHAPE), (3, 1025, UNSUPPORTED), (1, 1 << 29, SHAPE),
                              (0, 66, ALIGN), (4, 65, ALIGN), (5, 66, ALIGN), (6, 66, ALIGN)):
        bad = list(good)
        bad[at] = value
        assert plan(*bad) == status, (at, value)


@pytest.mark.parametrize("change,status", [
    (dict(packed=0), NULL), (dict(x=0), NULL), (dict(offsets=0), NULL), (dict(y=0), NULL), (dict(bits=5), UNSUPPORTED), (dict(x_type=3), UNSUPPORTED), (dict(y_type=3), UNSUPPORTED),
    (dict(experts=1025), UNSUPPORTED), (dict(experts=0), SHAPE), (dict(N=0), SHAPE), (dict(K=250), SHAPE), (dict(group=12), SHAPE), (dict(slots=-1), SHAPE), (dict(slots=1 << 31), SHAPE),
    (dict(x_rows=-1), SHAPE), (dict(x_rows=1 << 31), SHAPE), (dict(x_stride=248), SHAPE), (dict(expert_stride=1024), SHAPE), (dict(N=127, gated=1), SHAPE), (dict(packed=72), ALIGN),
    (dict(x=72), ALIGN), (dict(x_stride=260), ALIGN), (dict(expert_stride=(1 << 20) + 8), ALIGN), (dict(offsets=66), ALIGN), (dict(rows=66), ALIGN), (dict(y=130), ALIGN),
    (dict(N=1 << 24, K=1 << 16, x_stride=1 << 16, expert_stride=1 << 42, gated=1), SHAPE),             # ups further behind the gates than 32 bits reach
    (dict(workspace=72), ALIGN), (dict(workspace=0), WORKSPACE), (dict(workspace_bytes=6 * (2 * 256 * 2 + 4) - 1), WORKSPACE), (dict(slots=0, x=0, packed=0), OK)])
def test_product_refuses(qg, change, status):
    assert qg.lib().qg_experts_product(qg._EXPERTS(*{**EXPERTS, **change}.values()), None) == status


@pytest.mark.parametrize("change,status", [
    (dict(y=0), NULL), (dict(slots=0), NULL), (dict(weights=0), NULL), (dict(out=0), NULL), (dict(type=3), UNSUPPORTED), (dict(out_type=3), UNSUPPORTED), (dict(top_k=65), UNSUPPORTED),
    (dict(tokens=-1), SHAPE), (dict(N=0), SHAPE), (dict(top_k=0), SHAPE), (dict(y_rows=-1), SHAPE), (dict(residual=64, residual_stride=63), SHAPE), (dict(tokens=1 << 30, top_k=2), SHAPE),
    (dict(y=66), ALIGN), (dict(out=130), ALIGN), (dict(slots=66), ALIGN), (dict(weights=65), ALIGN), (dict(residual=66, residual_stride=64), ALIGN), (dict(tokens=0, y=0, out=0), OK)])
def test_combine_refuses(qg, change, status):
    assert qg.lib().qg_experts_combine(qg._COMBINE(*{**COMBINE, **change}.values()), None) == status


def test_workspace_sizes(qg):
    import torch
    size = qg.qg_experts_workspace_bytes
    assert size(5, 256) == 6 * (2 * 256 * 2 + 4) and size(0, 32, torch.bfloat16) == 128 * 2 + 4          # rows of whole 128 k, and one of zeros
    assert size(-1, 256) == 0 and size(4, 0) == 0 and qg.lib().qg_experts_workspace_bytes(4, 256, 3) == 0
    assert size(1 << 30, 1 << 20) == ((1 << 30) + 1) * (4 * (1 << 20) + 4)

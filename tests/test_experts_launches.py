"""Launches of a layer of experts, looked at without a GPU (tests/hip_stub.c): which kernels a call takes, and that its workgroups see
every tile that the choices could make, in launches of less than 2^32 lanes and no more LDS than there is."""
import ctypes
import json
import os
import re
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
BASE = 1 << 40                             # of every buffer; nothing is read
F32, BF16, F16 = range(3)


def _run(stub_path, lib_path, call, packed):
    stub, L = ctypes.CDLL(stub_path, mode=ctypes.RTLD_GLOBAL), ctypes.CDLL(lib_path)
    stub.stub_name.restype = ctypes.c_char_p
    vp = ctypes.c_void_p
    if call == "qg_expert_plan":
        tokens, top_k, experts = json.loads(packed.decode())
        L.qg_expert_plan.argtypes = [vp, ctypes.c_int64, ctypes.c_int, ctypes.c_int, vp, vp, vp, vp]
        status = L.qg_expert_plan(BASE, tokens, top_k, experts, BASE, BASE, BASE, None)
    else:
        function = getattr(L, call)
        function.argtypes = [ctypes.c_char_p, vp]
        status = function(packed, None)
    out = []
    for i in range(stub.stub_launches()):
        shape = (ctypes.c_uint32 * 5)()
        stub.stub_shape(i, shape)
        length, rest = re.match(r"_ZN12_GLOBAL__N_1(\d\d?)(\D.*)", stub.stub_name(i).decode()).groups()
        name, tail = rest[:int(length)], rest[int(length):]
        out.append([name, [int(v.replace("n", "-")) for v in re.findall(r"L[ib](n?\d+)E", tail)], list(shape)])
    json.dump([status, out], sys.stdout)


def _launches(tmp_path, call, packed):
    from paper_2307_03738_amd import build
    stub = os.path.join(str(tmp_path), "hip_stub.so")
    subprocess.run(["gcc", "-O1", "-w", "-shared", "-fPIC", os.path.join(HERE, "hip_stub.c"), "-o", stub], check=True)
    done = subprocess.run([sys.executable, os.path.abspath(__file__), stub, os.environ.get("QG_LIBRARY", build.OUT), call, packed.hex()],
                          capture_output=True, text=True, timeout=120)
    assert done.returncode == 0, done.stderr
    status, launches = json.loads(done.stdout)
    assert status == 0 and launches
    assert all(x * lanes < 1 << 32 and y < 1 << 16 and z == 1 and lds <= 160 << 10 for _, _, (x, y, z, lanes, lds) in launches), launches
    return launches


def _product(slots, experts, N, K, bits, group, x_type, gated):
    from paper_2307_03738_amd import binding as qg
    size = qg.qg_packed_bytes(N, K, bits, group)
    return qg._EXPERTS(BASE, BASE, BASE, BASE, 2 * BASE, N, K, size, slots, K, slots, bits, group, experts, x_type, x_type, gated, BASE, 1 << 50)


def most_tiles(slots, experts, rows):
    # as many slots as there are in tiles of `rows`, any split among the experts
    used = min(slots, experts)
    return (slots - used) // rows + used if slots < used * rows else (slots + used * (rows - 1)) // rows


PRODUCTS = [
    # slots, experts, N, K, bits, group, type, gated: kernels, slots of a tile, columns of a workgroup
    (2, 8, 22016, 4096, 4, 128, F32, 1, [("experts_few", [4, 4, 2, 4, 1])], None),                           # a row for each expert that is used
    (2, 8, 22016, 1 << 16, 4, 128, F32, 1, [("prepare_rows", [4, 256]), ("experts_few", [4, 4, 2, 4, 0])], None),
    (96, 32, 4096, 1408, 3, 64, F32, 0, [("prepare_rows", [3, 256]), ("experts_few", [3, 2, 2, 4, 0])], 8),
    (96, 32, 4096, 1440, 2, 96, BF16, 0, [("prepare_rows", [2, 256]), ("experts_few", [2, 0, 2, 4, 0])], 16),
    (366, 64, 2816, 2048, 4, 32, BF16, 1, [("prepare_rows", [4, 256]), ("experts_few", [4, 1, 2, 4, 0])], 16),
    (8192, 8, 22016, 4096, 4, 128, BF16, 1, [("prepare_rows", [4, 64]), ("experts_many", [4, 4, 1, 2, 1])], 64),
    (1280, 32, 4096, 4096, 4, 64, F32, 1, [("prepare_rows", [4, 256]), ("experts_many", [4, 2, 2, 1, 1])], 32),
    (8184, 60, 5120, 1792, 2, 64, F16, 0, [("prepare_rows", [2, 64]), ("experts_many", [2, 2, 1, 2, 1])], 64),
    (719, 2, 5130, 160, 4, 32, F32, 0, [("prepare_rows", [4, 256]), ("experts_many", [4, 1, 2, 2, 1])], 64),
    (173, 5, 7170, 192, 3, 64, F32, 0, [("prepare_rows", [3, 256]), ("experts_many", [3, 2, 2, 1, 1])], 32),
    (177, 2, 5130, 1056, 4, 32, F32, 0, [("prepare_rows", [4, 256]), ("experts_many", [4, 1, 2, 1, 3])], 32),     # less than a round of workgroups: K in slices
    (300, 2, 1000, 8192, 4, 128, BF16, 0, [("prepare_rows", [4, 256]), ("experts_few", [4, 4, 2, 8, 0])], 16),
    (4, 32, 2816, 4096, 4, 64, F32, 1, [("experts_few", [4, 2, 2, 8, 1])], 2),                              # not many workgroups: eight wavefronts each
    (16, 8, 4096, 4096, 4, 128, BF16, 0, [("prepare_rows", [4, 256]), ("experts_few", [4, 4, 2, 8, 0])], 16),
    (9, 4, 128, 320, 4, 40, F32, 0, [("prepare_rows", [4, 256]), ("experts_few", [4, -4, 2, 8, 0])], 8),     # groups that are no whole 32 k
    (2, 8, 22016, 4096, 4, 16, F32, 1, [("experts_few", [4, -2, 2, 4, 1])], None),
    (5000, 8, 4096, 4096, 2, 16, BF16, 0, [("prepare_rows", [2, 64]), ("experts_few", [2, -2, 2, 4, 0])], 16),
    (1 << 24, 64, 22016, 4096, 4, 16, F16, 1, [("prepare_rows", [4, 64]), ("experts_few", [4, -2, 2, 4, 0])], 16),
]


@pytest.mark.parametrize("slots,experts,N,K,bits,group,x_type,gated,kernels,tile", PRODUCTS)
def test_products_take_the_kernels_that_are_meant(tmp_path, slots, experts, N, K, bits, group, x_type, gated, kernels, tile):
    launches = _launches(tmp_path, "qg_experts_product", _product(slots, experts, N, K, bits, group, x_type, gated))
    assert [(n, t) for n, t, _ in launches] == kernels
    name, template, (x, y, _, lanes, _) = launches[-1]
    columns = N // 2 if gated else N
    if tile:
        if name == "experts_many":
            assert x * y >= most_tiles(slots, experts, tile) * -(-columns // (128 if gated else 256)) and lanes == 256 * template[4]
        elif y == 1:                           # 1, 2 or 4 tiles of 64 outputs
            assert x % most_tiles(slots, experts, tile) == 0
            wide = [-(-columns // (w * (32 if gated else 64))) for w in (1, 2, 4)]
            assert x // most_tiles(slots, experts, tile) in wide and lanes == 64 * template[3]
        else:
            assert x * y >= most_tiles(slots, experts, tile) * -(-columns // (4 * (32 if gated else 64))) and x % 8 == 0


@pytest.mark.parametrize("tokens,top_k,experts,kernels", [(1, 1, 1, ["plan"]), (48, 4, 32, ["plan"]), (2048, 8, 1024, ["plan"]), (16383, 8, 192, ["plan_count", "plan", "plan_tokens"]),
                                                          ((1 << 27) - 1, 8, 1024, ["plan_count", "plan", "plan_tokens"])])
def test_orders(tmp_path, tokens, top_k, experts, kernels):
    launches = _launches(tmp_path, "qg_expert_plan", json.dumps([tokens, top_k, experts]).encode())
    assert [n for n, _, _ in launches] == kernels
    if len(kernels) > 1:
        parts = launches[0][2][0]
        assert parts * experts <= tokens * top_k and launches[2][2][0] * 256 >= tokens * top_k        # the counts fit into what will be the slots' tokens


@pytest.mark.parametrize("tokens,N", [(1, 1), (5, 4099), ((1 << 24) + 5, 8), (1 << 20, 1 << 16), (2, 1 << 24)])
def test_sums_see_every_column_of_every_token(tmp_path, tokens, N):
    from paper_2307_03738_amd import binding as qg
    launches = _launches(tmp_path, "qg_experts_combine", qg._COMBINE(BASE, BASE, BASE, 0, BASE, 100, tokens, N, 0, BF16, F32, 3))
    assert sum(x for _, _, (x, _, _, _, _) in launches) == tokens * -(-N // 2048)


@pytest.mark.parametrize("tokens,experts,top_k,lanes", [(1, 64, 6, 16), (3, 128, 16, 16), (9, 128, 17, 32), (5, 256, 32, 32), (5, 256, 33, 64), (7, 512, 9, 64), (3, 1024, 64, 64), ((1 << 27) + 3, 8, 2, 16)])
def test_choices_see_every_token(tmp_path, tokens, experts, top_k, lanes):
    from paper_2307_03738_amd import binding as qg
    launches = _launches(tmp_path, "qg_route", qg._ROUTE(BASE, 0, BASE, BASE, tokens, experts, BF16, experts, top_k, 0, 1, 1, 1, 1, 1.0))
    assert all(n == "route" and t[0] == lanes for n, t, _ in launches)
    per = 256 // lanes
    assert sum(x for _, _, (x, _, _, _, _) in launches) == -(-tokens // per)


if __name__ == "__main__":
    _run(*sys.argv[1:4], bytes.fromhex(sys.argv[4]))

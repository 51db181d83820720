"""Launches of the calls between the products, looked at without a GPU (tests/hip_stub.c): a launch has less than 2^32 lanes in a
dimension, however many rows or tokens a call has, and all of its workgroups together see every one of them."""
import ctypes
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
BASE = 1 << 40                             # of every buffer; nothing is read


def _run(stub_path, lib_path, call, packed):
    stub, L = ctypes.CDLL(stub_path, mode=ctypes.RTLD_GLOBAL), ctypes.CDLL(lib_path)
    vp = ctypes.c_void_p
    function = getattr(L, call)
    function.argtypes = [ctypes.c_char_p] + [vp] * (2 if call == "qg_pages_fork" else 1)
    status = function(packed, BASE, None) if call == "qg_pages_fork" else function(packed, None)
    shapes = []
    for i in range(stub.stub_launches()):
        shape = (ctypes.c_uint32 * 5)()
        stub.stub_shape(i, shape)
        shapes.append(list(shape[:4]))
    json.dump([status, shapes], sys.stdout)


def _cases():
    from paper_2307_03738_amd import binding as qg
    norm = lambda rows, K, y, group: ("qg_rms_norm", qg._NORM(BASE, BASE, BASE, BASE, BASE, BASE, rows, K, K, K, 2, 0, y, group, 1e-5))  # noqa: E731
    append = lambda tokens, heads, rope: ("qg_kv_append", qg._APPEND(  # noqa: E731
        BASE, BASE, BASE, BASE, BASE, 4, 8, 2, 4, 1, 16, 8, 3, BASE, BASE, 2 * BASE, BASE, BASE, BASE, BASE, tokens, 8 * max(heads, 1), 8, 8, 64, 1, heads, rope, 0))
    fork = lambda rows: ("qg_pages_fork", qg._BOOK(BASE, BASE, BASE, 2 * BASE, 2 * BASE, 2 * BASE, 9, rows, 1, 16))  # noqa: E731
    return [(n, *c) for n, c in [
        (5, norm(5, 7, 0, 0)), ((1 << 24) + 5, norm((1 << 24) + 5, 7, 0, 0)), (0x7fffffff, norm(0x7fffffff, 1, 3, 0)), ((1 << 25) - 1, norm((1 << 25) - 1, 30, 3, 3)),
        (5, append(5, 2, 8)), ((1 << 24) + 5, append((1 << 24) + 5, 0, 0)), (0x7fffffff, append(0x7fffffff, 1, 4)),
        (5, fork(5)), ((1 << 24) + 5, fork((1 << 24) + 5)), (0x3fffffff, fork(0x3fffffff))]]


@pytest.mark.parametrize("n", range(10))
def test_launches_stay_below_2_to_the_32_lanes(tmp_path, n):
    from paper_2307_03738_amd import build
    items, call, packed = _cases()[n]
    stub = os.path.join(str(tmp_path), "hip_stub.so")
    subprocess.run(["gcc", "-O1", "-w", "-shared", "-fPIC", os.path.join(HERE, "hip_stub.c"), "-o", stub], check=True)
    done = subprocess.run([sys.executable, os.path.abspath(__file__), stub, os.environ.get("QG_LIBRARY", build.OUT), call, packed.hex()],
                          capture_output=True, text=True, timeout=120)
    assert done.returncode == 0, done.stderr
    status, shapes = json.loads(done.stdout)
    assert status == 0 and shapes
    assert all(x * lanes < 1 << 32 and y < 1 << 16 and z == 1 for x, y, z, lanes in shapes), shapes
    of_rows = shapes[1:] if call == "qg_pages_fork" else shapes
    assert sum(x for x, _, _, _ in of_rows) == items


if __name__ == "__main__":
    _run(*sys.argv[1:4], bytes.fromhex(sys.argv[4]))

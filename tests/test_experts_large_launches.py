"""Launches of experts' products of the most rows that a GPU's memory holds, looked at without a GPU: whether a call is taken does not hang on the kernel that its rows choose."""
import pytest

from tests.test_experts_launches import BF16, F16, F32, _launches, _product, most_tiles


@pytest.mark.parametrize("slots,experts,N,K,bits,group,x_type,gated", [
    (6200000, 8, 22016, 4096, 4, 128, BF16, 1),            # just below and just above 2^23 workgroups
    (6300000, 8, 22016, 4096, 4, 128, BF16, 1),
    (7000001, 8, 22016, 4096, 4, 128, F32, 1),
    (12000000, 1024, 22016, 64, 2, 32, F16, 0),
    ((1 << 31) - 1, 3, 255, 96, 3, 96, BF16, 0),
    (6300000, 8, 22016, 4096, 4, 16, BF16, 1),             # the kernel of few rows takes them all along
])
def test_products_of_the_most_rows(tmp_path, slots, experts, N, K, bits, group, x_type, gated):
    launches = _launches(tmp_path, "qg_experts_product", _product(slots, experts, N, K, bits, group, x_type, gated))
    assert [n for n, _, _ in launches] == ["prepare_rows", "experts_few" if group % 32 else "experts_many"]
    name, template, (x, y, _, lanes, _) = launches[-1]
    columns = N // 2 if gated else N
    tiles = most_tiles(slots, experts, 64 if name == "experts_many" else 16)
    wide = (128 if gated else 256)
    assert x * y >= tiles * -(-columns // wide) and x * y < 1 << 31
    assert y == 1 or x % 8 == 0                            # a workgroup's number still says on which die it runs

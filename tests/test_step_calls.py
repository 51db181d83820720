"""Host side of the calls between the products: descriptions are laid out as the header has them, and bad ones are refused
before anything is enqueued.  No kernel is launched here."""
import os
import struct
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

NORM = dict(x=64, residual=0, weight=64, h=0, y=64, scales=0, rows=2, K=64, x_stride=64, residual_stride=0, type=0, weight_type=0, y_type=0, group=0, eps=1e-5)
CACHE = dict(k=64, v=64, k_scale=0, v_scale=0, tables=64, table_stride=4, pages=8, max_rows=2, max_pages=4, kv_heads=2, page=16, head_dim=64, cache_type=1)
APPEND = dict(CACHE, rows=64, positions=64, q=64, new_k=64, new_v=64, q_out=128, cos_sin=64, tokens=3, q_stride=256, k_stride=128, v_stride=128, cos_sin_rows=9,
              type=0, heads=4, rope_dim=64, interleaved=0)
ATTENTION = dict(CACHE, lens=64, first=0, q=64, out=64, lse=0, q_stride=256, batch=2, heads=4, type=0, window=0, scale=1.0, workspace=64, workspace_bytes=1 << 40)
BOOK = dict(tables=64, lens=64, refs=64, tables_out=128, lens_out=128, refs_out=128, pages=9, rows=2, max_pages=3, page=16)
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
    printf("%zu %zu %zu %zu %zu\\n", sizeof(qg_norm_desc), sizeof(qg_append_desc), sizeof(qg_attention_desc), sizeof(qg_page_book), sizeof(qg_page_plane));
    printf("%zu %zu %zu %zu\\n", offsetof(qg_norm_desc, eps), offsetof(qg_append_desc, interleaved), offsetof(qg_attention_desc, scale), offsetof(qg_page_book, page));
    return 0;
}
""")
    subprocess.run(["gcc", "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "sizes")], check=True)
    sizes, at = [[int(v) for v in line.split()] for line in subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True, check=True).stdout.splitlines()]
    packed = [qg._NORM(*NORM.values()), qg._APPEND(*APPEND.values()), qg._ATTENTION(*ATTENTION.values()), qg._BOOK(*BOOK.values()), qg._PLANE(1, 2, 3)]
    assert [len(p) for p in packed] == sizes
    assert struct.unpack_from("f", packed[0], at[0])[0] == pytest.approx(1e-5) and struct.unpack_from("f", packed[2], at[2])[0] == 1.0
    assert struct.unpack_from("i", packed[1], at[1])[0] == 0 and struct.unpack_from("i", packed[3], at[3])[0] == 16


@pytest.mark.parametrize("change,status", [
    (dict(x=0), NULL), (dict(weight=0), NULL), (dict(y=0), NULL), (dict(h=64), NULL), (dict(y_type=3), NULL), (dict(type=3), UNSUPPORTED), (dict(type=-1), UNSUPPORTED),
    (dict(weight_type=3), UNSUPPORTED), (dict(y_type=4), UNSUPPORTED), (dict(rows=-1), SHAPE), (dict(K=0), SHAPE), (dict(x_stride=63), SHAPE),
    (dict(residual=64, residual_stride=9), SHAPE), (dict(group=32), SHAPE), (dict(y_type=3, scales=64, group=48), SHAPE), (dict(rows=1 << 31), SHAPE),
    (dict(x=65), ALIGN), (dict(y=66), ALIGN), (dict(rows=0, x=0), OK)])
def test_norm_refuses(qg, change, status):
    assert qg.lib().qg_rms_norm(qg._NORM(*{**NORM, **change}.values()), None) == status


BAD_CACHES = [
    (dict(k=0), NULL), (dict(v=0), NULL), (dict(tables=0), NULL), (dict(cache_type=3), NULL), (dict(cache_type=0), UNSUPPORTED), (dict(cache_type=4), UNSUPPORTED),
    (dict(page=8), UNSUPPORTED), (dict(page=24), UNSUPPORTED), (dict(page=8192), UNSUPPORTED), (dict(head_dim=60), UNSUPPORTED), (dict(head_dim=264), UNSUPPORTED),
    (dict(head_dim=0), UNSUPPORTED), (dict(pages=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(max_pages=0), SHAPE), (dict(table_stride=3), SHAPE),
    (dict(max_pages=1 << 28), SHAPE), (dict(k=72), ALIGN), (dict(tables=66), ALIGN)]


@pytest.mark.parametrize("change,status", BAD_CACHES + [
    (dict(type=3), UNSUPPORTED), (dict(tokens=-1), SHAPE), (dict(rope_dim=63), SHAPE), (dict(rope_dim=66), SHAPE), (dict(heads=-1), SHAPE),
    (dict(q_stride=255), SHAPE), (dict(k_stride=120), SHAPE), (dict(rows=0), NULL), (dict(positions=0), NULL), (dict(new_k=0), NULL), (dict(q=0), NULL),
    (dict(q_out=0), NULL), (dict(q_out=128, q=128), UNSUPPORTED), (dict(cos_sin=0), NULL), (dict(q=72), ALIGN), (dict(new_v=68), ALIGN), (dict(q_stride=260), ALIGN), (dict(tokens=0, rows=0, q=0), OK)])
def test_append_refuses(qg, change, status):
    assert qg.lib().qg_kv_append(qg._APPEND(*{**APPEND, **change}.values()), None) == status


@pytest.mark.parametrize("change,status", BAD_CACHES + [
    (dict(type=3), UNSUPPORTED), (dict(batch=-1), SHAPE), (dict(batch=3), SHAPE), (dict(heads=3), SHAPE), (dict(heads=0), SHAPE), (dict(window=-1), SHAPE),
    (dict(q_stride=255), SHAPE), (dict(lens=0), NULL), (dict(q=0), NULL), (dict(out=0), NULL), (dict(q=72), ALIGN), (dict(q_stride=260), ALIGN), (dict(lse=66), ALIGN),
    (dict(workspace=0), WORKSPACE), (dict(workspace_bytes=16), WORKSPACE), (dict(workspace=72), ALIGN), (dict(batch=0, lens=0, q=0), OK)])
def test_attention_refuses(qg, change, status):
    assert qg.lib().qg_paged_attention(qg._ATTENTION(*{**ATTENTION, **change}.values()), None) == status


def test_attention_workspace_sizes(qg):
    size = qg.qg_paged_attention_workspace_bytes
    assert size(1, 8, 3, 64) == 0 and size(1, 8, 2, 60) == 0 and size(-1, 8, 2, 64) == 0 and size(1, 0, 2, 64) == 0
    assert 0 < size(1, 32, 32, 128) <= size(128, 32, 32, 128) and size(64, 64, 8, 128) % 256 == 0


@pytest.mark.parametrize("change,status", [
    (dict(refs=0), NULL), (dict(refs_out=0), NULL), (dict(tables=0), NULL), (dict(tables_out=0), NULL), (dict(pages=0), SHAPE), (dict(rows=-1), SHAPE),
    (dict(max_pages=0), SHAPE), (dict(page=0), SHAPE), (dict(max_pages=1 << 28), SHAPE), (dict(refs=66), ALIGN), (dict(tables_out=65), ALIGN)])
def test_books_are_refused(qg, change, status):
    L, book = qg.lib(), qg._BOOK(*{**BOOK, **change}.values())
    assert L.qg_pages_resize(book, 64, b"", 0, 64, 64, 1 << 40, None) == status
    assert L.qg_pages_compact(book, b"", 0, 64, 64, 1 << 40, None) == status
    assert L.qg_pages_fork(book, 64, None) == status


def test_page_calls_refuse(qg):
    L, book = qg.lib(), qg._BOOK(*BOOK.values())
    plane = qg._PLANE
    assert L.qg_pages_resize(None, 64, b"", 0, 64, 64, 1 << 40, None) == NULL
    assert L.qg_pages_resize(book, None, b"", 0, 64, 64, 1 << 40, None) == NULL
    assert L.qg_pages_resize(book, 64, b"", 0, None, 64, 1 << 40, None) == NULL
    assert L.qg_pages_resize(book, 64, None, 1, 64, 64, 1 << 40, None) == NULL
    assert L.qg_pages_resize(book, 64, b"", 9, 64, 64, 1 << 40, None) == UNSUPPORTED
    assert L.qg_pages_resize(book, 64, plane(64, 1, 24), 1, 64, 64, 1 << 40, None) == ALIGN
    assert L.qg_pages_resize(book, 64, plane(72, 1, 32), 1, 64, 64, 1 << 40, None) == ALIGN
    assert L.qg_pages_resize(book, 64, plane(64, 0, 32), 1, 64, 64, 1 << 40, None) == SHAPE
    assert L.qg_pages_resize(book, 64, b"", 0, 64, 64, qg.qg_pages_workspace_bytes(2, 3, 9) - 1, None) == WORKSPACE
    assert L.qg_pages_compact(book, b"", 0, None, 64, 1 << 40, None) == NULL
    assert L.qg_pages_compact(book, b"", 0, 64, None, 1 << 40, None) == WORKSPACE
    assert L.qg_pages_fork(book, None, None) == NULL
    for half in ({"tables_out": 64}, {"lens_out": 64}):                    # tables and lens in place both or neither
        assert L.qg_pages_resize(qg._BOOK(*{**BOOK, **half}.values()), 64, b"", 0, 64, 64, 1 << 40, None) == UNSUPPORTED
    assert L.qg_pages_fork(qg._BOOK(*{**BOOK, "refs_out": 64}.values()), 64, None) == UNSUPPORTED
    assert L.qg_pages_copy(plane(64, 1, 32), 1, 9, None, 3, None) == NULL
    assert L.qg_pages_copy(plane(64, 1, 32), 1, 9, 64, -1, None) == SHAPE
    assert L.qg_pages_copy(plane(64, 1, 32), 1, 0, 64, 3, None) == SHAPE
    assert L.qg_pages_copy(plane(64, 1, 32), 1, 9, 64, 0, None) == OK
    assert qg.qg_pages_workspace_bytes(2, 0, 9) == 0 and qg.qg_pages_workspace_bytes(-1, 3, 9) == 0

// The paged key-value cache as the kernels see it, and its checks.
#pragma once

#include "qg_types.h"

#define QG_MAX_HEADS 4096

namespace {

struct QgKv {
    void *k, *v;
    float *k_scale, *v_scale;
    const int32_t *tables;
    int64_t table_stride, pages;
    int rows, max_pages, kv_heads, page, page_shift, head_dim, type;
};

static inline int qg_check_cache(const qg_kv_cache &c, QgKv *kv)
{
    if (c.type != QG_BF16 && c.type != QG_F16 && c.type != QG_E4M3) return QG_ERR_UNSUPPORTED;
    if (c.page < 16 || c.page > 4096 || (c.page & (c.page - 1))) return QG_ERR_UNSUPPORTED;
    if (c.head_dim < 8 || c.head_dim > 256 || c.head_dim % 8) return QG_ERR_UNSUPPORTED;
    if (c.rows < 0 || c.max_pages <= 0 || c.kv_heads <= 0 || c.kv_heads > QG_MAX_HEADS || c.pages <= 0 || c.pages > 0x7fffffff) return QG_ERR_SHAPE;
    if ((int64_t)c.max_pages * c.page > 0x7ffffe00) return QG_ERR_SHAPE;        // positions are 32-bit, with room to round up
    if (c.rows > 1 && c.table_stride < c.max_pages) return QG_ERR_SHAPE;
    if (!c.k || !c.v || !c.tables || (c.type == QG_E4M3 && (!c.k_scale || !c.v_scale))) return QG_ERR_NULL;
    if (!qg_aligned16(c.k) || !qg_aligned16(c.v) || !qg_aligned_to(c.tables, 4) || !qg_aligned16(c.k_scale) || !qg_aligned16(c.v_scale)) return QG_ERR_ALIGN;
    *kv = {c.k, c.v, c.k_scale, c.v_scale, c.tables, c.table_stride, c.pages, c.rows, c.max_pages, c.kv_heads, c.page,
           __builtin_ctz((unsigned)c.page), c.head_dim, c.type};
    return QG_OK;
}

// Page of a sequence's token, -1 if it has none.
__device__ inline int64_t qg_page_of(const QgKv &c, int row, int64_t position)
{
    if (row < 0 || row >= c.rows || position < 0) return -1;
    const int64_t column = position >> c.page_shift;
    if (column >= c.max_pages) return -1;
    const int64_t page = c.tables[row * c.table_stride + column];
    return page < c.pages ? page : -1;        // (a negative id is none either)
}

}  // namespace

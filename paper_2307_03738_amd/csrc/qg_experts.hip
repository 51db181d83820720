// qg_experts_product: y[p] = What_e x[rows[p]] for the slots p of each expert e.
#include "qg_experts_few.h"
#include "qg_experts_many.h"

namespace {

// Of the rows of X as f16, and their powers of two.
struct RowsSpace {
    int64_t padded, bytes, total;
    int parts;
};
RowsSpace rows_space(int64_t x_rows, int64_t K, int x_type)
{
    RowsSpace s;
    s.parts = x_type == QG_F32 ? 2 : 1;
    s.padded = (K + 127) / 128 * 128;
    s.bytes = (x_rows + 1) * s.parts * s.padded * 2;
    s.total = s.bytes + (x_rows + 1) * 4;
    return s;
}

// Slots of a workgroup of the kernel of many rows, 64 or 32, or 0: the kernel of few rows.
//
// By the rows of an expert, on average: few rows up to 20 operand rows (two of fp32 each); beyond, tiles of 32 slots, three workgroups a compute unit, up to
// 48 rows (128 of fp32, whose two parts make as much of a weight unpacked).  Each side measured, us a call, matrices that no cache holds, random choices (some experts have twice the average):
// 32 experts' 4096 x 4096 4-bit matrices, groups of 64, few rows against tiles of 32: fp32 8 rows 84, 82, 10 rows 92, 111, 12 rows 108, 116, 16 rows 128, 120; bf16 16 rows 86, 94 (tiles of 64: 76),
// 20 rows 95, 84 (64: 104), 24 rows 112, 88; tiles of 32 against 64: bf16, groups of 128, 43 rows 109, 117, 51 rows 125, 127, 59 rows 130, 126; groups of 32, 43 rows 139, 149,
// 51 rows 164, 152; fp32, groups of 64, 98 rows 304, 314, 134 rows 382, 395, 158 rows 430, 449; 8 experts' gated 8192 x 4096, 504 rows: bf16, groups of 32, 495, 404, fp32, groups of 128, 568, 501.
//
// And by workgroups: with fewer than one a compute unit tiles of 32, and where those are not 9 to 16 units the wavefronts of few rows, which also divide K.  Few rows, tiles of 32 (with K in
// slices, where many_plan has them so) and of 64, groups of 128, bf16: 2 experts' 148 rows of 1000 x 8192 34, 50, 83; two's 197 of 4096 x 4096 48, 32, 47; four's 492 of 400 x 4096 39, 38, 54 (fp32 57, 43, 74: the slices
// came after this limit, which fp32 would have lower); three's 1969 of 1000 x 1024 59, 44, 35.
int many_rows_of(const QgExpertsArgs &a, int parts)
{
    if (a.group % 32 || a.slots * parts <= (int64_t)20 * a.experts) return 0;
    const int width = a.gated ? 128 : 256;
    const int64_t across = (a.columns + width - 1) / width;
    if (qg_most_tiles(a.slots, a.experts, 32) * across * 16 <= (int64_t)9 * qg_compute_units()) return 0;
    if (a.slots <= (int64_t)(parts == 2 ? 128 : 48) * a.experts || qg_most_tiles(a.slots, a.experts, 64) * across < qg_compute_units()) return 32;
    return 64;
}

int few_plan(const QgExpertsArgs &a, int bits, const RowsSpace &s, const QgPrepareArgs &p, hipStream_t st)
{
    QgFewArgs f = {};
    f.e = a;
    f.xh = p.xh;
    f.up = p.up;
    f.padded = s.padded;
    f.parts = s.parts;
    f.tile_rows = FEW_ROWS / s.parts;
    // about one row for each expert that is used, and room for two of them: without prepare_rows
    const int64_t row_bytes = s.parts * (s.padded * 2 + 16);
    if (a.slots * 2 <= a.experts && 2 * row_bytes <= FEW_LDS) {
        f.stride = (int)(s.padded * 2 + 16);
        if (f.tile_rows * row_bytes > FEW_LDS) f.tile_rows = (int)(FEW_LDS / row_bytes);
    }
    f.e.row_tiles = (int)qg_most_tiles(a.slots, a.experts, f.tile_rows);
    const int64_t used = a.experts < a.slots ? a.experts : a.slots;
    // as few tiles as leave one and a half rounds of workgroups, four on a compute unit (61 tokens' 2816 x 2048 matrices 59.2 us, with one round at most 68.2; 24 tokens'
    // 4096 x 1408 28.2, with two 31.3)
    const int shift = a.gated ? 5 : 6;
    f.tile_shift = 0;
    while (f.tile_shift < 2 && used * ((a.columns + (1 << (shift + f.tile_shift)) - 1) >> (shift + f.tile_shift)) > 6 * qg_compute_units()) ++f.tile_shift;
    // where not even the tiles that could be needed make two and a half workgroups a compute unit, K goes to twice as many wavefronts (8 experts' 4096 x 4096 4-bit matrices, 2 rows
    // each: fp32 24.7 us, 21.4 so, bf16 4 rows 26.4, 23.0; beyond, fp32 4 rows 27.0, 29.2)
    f.waves = 2 * (int64_t)f.e.row_tiles * ((a.columns + (1 << shift) - 1) >> shift) <= 5 * qg_compute_units() ? 8 : 4;
    const int width = 1 << (shift + f.tile_shift);
    if (a.group % 32) {
        f.cells = a.group % 16 ? a.group / 8 : a.group / 16;
    } else {
        f.g32 = a.group / 32;
        f.gshift = f.g32 & (f.g32 - 1) ? -1 : __builtin_ctz(f.g32);
    }
    f.quanta = (a.K + 127) / 128;
    const int64_t blocks = (int64_t)f.e.row_tiles * ((a.columns + width - 1) / width);
    if (blocks > 0x7fffffff - QG_MOST_GROUPS) return QG_ERR_SHAPE;
    f.blocks = (int)blocks;
    (bits == 4 ? qg_few_launch_b4 : bits == 3 ? qg_few_launch_b3 : qg_few_launch_b2)(f, p, st);
    return QG_OK;
}

// Workgroups of 32 slots that make less than a round (three a compute unit) take K in three slices, where it has eight steps at least: 130 tokens' three of three 2646 x 7104 3-bit
// matrices, groups of 64, bf16, 50 us, without 69; 100 tokens' two of four 4096 x 4096 fp32 36, 47.  (Tiles of 64 where those make one to two workgroups a compute unit stay: 1305 tokens' seven
// of 26 497 x 2432 64, in 32 sliced 75.)
constexpr int MANY_SLICED = 3, MANY_SLICED_K = 1024;

int many_plan(const QgExpertsArgs &a, int bits, int tile_rows, const RowsSpace &s, const QgPrepareArgs &p, hipStream_t st)
{
    QgManyArgs f = {};
    f.e = a;
    f.tile_rows = tile_rows;
    f.e.row_tiles = (int)qg_most_tiles(a.slots, a.experts, f.tile_rows);
    f.xh = p.xh;
    f.up = p.up;
    f.padded = s.padded;
    f.parts = s.parts;
    f.g32 = a.group / 32;
    f.gshift = f.g32 & (f.g32 - 1) ? -1 : __builtin_ctz(f.g32);
    const int width = a.gated ? 128 : 256;
    f.column_blocks = (a.columns + width - 1) / width;
    const int64_t blocks = (int64_t)f.e.row_tiles * f.column_blocks;
    if (blocks > 0x7fffffff - QG_MOST_GROUPS) return QG_ERR_SHAPE;
    f.blocks = (int)blocks;
    f.slices = tile_rows == 32 && blocks < (int64_t)MANY_SLICED * qg_compute_units() && a.K >= MANY_SLICED_K ? 3 : 1;
    return (bits == 4 ? qg_many_launch_b4 : bits == 3 ? qg_many_launch_b3 : qg_many_launch_b2)(f, p, st);
}

}  // namespace

extern "C" size_t qg_experts_workspace_bytes(int64_t x_rows, int64_t K, int x_type)
{
    if (x_rows < 0 || x_rows > 0x7fffffff || K <= 0 || K > (int64_t)1 << 24 || !qg_float_type(x_type)) return 0;
    return (size_t)rows_space(x_rows, K, x_type).total;
}

extern "C" int qg_experts_product(const qg_experts_desc *d, void *stream)
{
    if (!d) return QG_ERR_NULL;
    QgLayout L;
    const int status = qg_make_layout(d->N, d->K, d->bits, d->group, &L);
    if (status != QG_OK) return status;
    if (!qg_float_type(d->x_type) || !qg_float_type(d->y_type) || d->experts > QG_MAX_EXPERTS) return QG_ERR_UNSUPPORTED;
    if (d->experts <= 0 || d->slots < 0 || d->slots > 0x7fffffff || d->x_rows < 0 || d->x_rows > 0x7fffffff || (d->gated && d->N % 2)) return QG_ERR_SHAPE;
    if ((d->x_rows > 1 && d->x_stride < d->K) || (d->experts > 1 && (d->expert_stride < 0 || (size_t)d->expert_stride < L.total))) return QG_ERR_SHAPE;
    if (d->slots == 0) return QG_OK;
    if (!d->packed || (!d->x && d->x_rows) || !d->offsets || !d->y) return QG_ERR_NULL;
    if (!qg_aligned16(d->packed) || d->expert_stride % 16 || !qg_aligned16(d->x) || (d->x_rows > 1 && d->x_stride % 8) || !qg_aligned_to(d->offsets, 4) ||
        !qg_aligned_to(d->rows, 4) || !qg_aligned_to(d->y, qg_type_bytes(d->y_type)) || !qg_aligned16(d->workspace)) return QG_ERR_ALIGN;
    if (!d->workspace || d->workspace_bytes < qg_experts_workspace_bytes(d->x_rows, d->K, d->x_type)) return QG_ERR_WORKSPACE;
    QgExpertsArgs a = {};
    a.packed = (const char *)d->packed;
    a.x = (const char *)d->x;
    a.offsets = d->offsets;
    a.rows = d->rows;
    a.y = d->y;
    a.expert_stride = d->expert_stride;
    a.x_rows = d->x_rows;
    a.x_stride = d->x_stride;
    a.slots = d->slots;
    a.scales_off = (int64_t)L.scales_off;
    a.zeros_off = (int64_t)L.zeros_off;
    a.tile_codes = (int64_t)L.units * L.planes * 1024;
    a.tile_scales = L.ngroups * 256;
    a.tile_zeros = L.zwords * 256;
    a.N = (int)d->N;
    a.K = (int)d->K;
    a.gated = d->gated != 0;
    a.columns = a.gated ? a.N / 2 : a.N;
    a.group = d->group;
    a.experts = d->experts;
    a.x_type = d->x_type;
    a.y_type = d->y_type;
    // (the lanes of a wavefront that take ups lie up to so far behind the gates, in 32 bits)
    if (a.gated && ((a.columns + 63) / 64 + 2) * a.tile_codes >= (int64_t)1 << 32) return QG_ERR_SHAPE;
    const hipStream_t st = (hipStream_t)stream;
    const RowsSpace s = rows_space(a.x_rows, a.K, a.x_type);
    const QgPrepareArgs p = {a.x, (char *)d->workspace, (int32_t *)((char *)d->workspace + s.bytes), a.x_rows, a.x_stride, s.padded, a.K, a.x_type};
    const int many = many_rows_of(a, s.parts);
    const int launched = many ? many_plan(a, d->bits, many, s, p, st) : few_plan(a, d->bits, s, p, st);
    return launched != QG_OK ? launched : qg_launch_status();
}

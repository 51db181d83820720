// The experts' products where an expert has few rows: bound by reading the packed matrices once.
//
// A workgroup of eight wavefronts takes 64 or 128 outputs (two tiles of 64; gated: the gates and the ups of 64 columns) of up to 32
// operand rows of an expert, K cut into slices of whole quanta (128 k, 256 at 2 bits) over its wavefronts.  X goes through LDS as f16 (rows of two parts if it is fp32),
// in the order in which the codes come out of their words; the weights go from memory into registers, a quantum ahead, and into the 16 x 16 x 32
// matrix instruction as q - z.  fp32 sums of a group (or 128 k of it) are multiplied by its scale; slices meet in LDS.
#pragma once

#include "qg_experts_codes.h"

constexpr int FEW_LDS = (64 << 10) - 256;      // for rows of X; and 35 KB at the end
constexpr int FEW_ROWS = 32;                   // operand rows
constexpr int FEW_PAD = 68;                    // floats from one row of sums to the next: rows 4 apart on other banks

struct QgFewArgs {
    QgExpertsArgs e;
    int tile_rows;             // rows of X a workgroup takes
    int tiles;                 // tiles of 64 outputs a workgroup takes: 2, or 1 where it takes 8 slices
    int g32, gshift;           // group / 32, its logarithm or -1
    int quanta;                // of K
    int blocks;
};

#ifdef QG_EXPERTS_KERNELS
namespace {

template <int BITS> constexpr int few_quantum() { return BITS == 2 ? 256 : 128; }
template <int BITS> constexpr int few_loads() { return BITS == 3 ? 3 : 4; }

// Weights of a quantum, as loaded.
template <int BITS, int FOLDS>
struct FewWeights {
    uint4 v[few_loads<BITS>()];
    uint32_t s[FOLDS], z[FOLDS];               // scale, and the word with the zero-point (shifted where it is used: a shift here would wait)
    int shift[FOLDS];
};

template <int BITS, int GP, int MB>
__device__ inline void few_rows(const QgFewArgs &f, const ExpertTile &t, int64_t column0, char *smem, uint32_t *most, int rows, int parts)
{
    using F = Fmt<BITS>;
    constexpr int QK = few_quantum<BITS>(), LOADS = few_loads<BITS>(), FOLDS = QK / 32 / GP, ZPER = 32 / F::ZBITS;
    constexpr int OCT = BITS == 2 ? 16 : 8;
    const QgExpertsArgs &a = f.e;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = f.tiles == 2 ? wave & 1 : 0, slices = f.tiles == 2 ? 4 : 8, slice = f.tiles == 2 ? wave >> 1 : wave;
    const int vrows = rows * parts;

    // this lane's output
    const int64_t column = column0 + (a.gated ? 0 : tile * 64) + lane;
    const int64_t n = (column < a.columns ? column : a.columns - 1) + (a.gated ? (int64_t)tile * a.columns : 0);
    const char *blob = a.packed + t.expert * a.expert_stride;
    const char *codes = blob + (n >> 6) * a.tile_codes + (n & 63) * 16;
    const char *scales = blob + a.scales_off + (n >> 6) * a.tile_scales + (n & 63) * 4;
    const char *zeros = blob + a.zeros_off + (n >> 6) * a.tile_zeros + (n & 63) * 4;
    const int last_group = a.K / a.group - 1;

    // quanta of X that fit, a whole number for each slice
    int chunk = FEW_LDS / vrows / 2 / QK;                    // (of 16 bytes a row for bank offsets: QK >= 128 leaves them room below)
    while (chunk > 1 && vrows * (chunk * QK * 2 + 16) > FEW_LDS) --chunk;
    chunk = chunk >= f.quanta ? f.quanta : chunk > slices ? chunk / slices * slices : chunk;
    const int stride = chunk * QK * 2 + 16;

    auto first_of = [&](int c) {                             // first quantum of this slice in the chunk that begins at c
        const int here = f.quanta - c < chunk ? f.quanta - c : chunk;
        return c + here * slice / slices;
    };
    auto load = [&](int q, FewWeights<BITS, FOLDS> &w) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) w.v[i] = *(const uint4 *)(codes + ((int64_t)q * LOADS + i) * 1024);
#pragma unroll
        for (int i = 0; i < FOLDS; ++i) {
            const int k32 = q * (QK / 32) + i * GP;
            int g = f.gshift >= 0 ? k32 >> f.gshift : k32 / f.g32;
            g = g < last_group ? g : last_group;
            w.s[i] = *(const uint32_t *)(scales + (int64_t)g * 256);
            w.z[i] = *(const uint32_t *)(zeros + (int64_t)(g / ZPER) * 256);
            w.shift[i] = g % ZPER * F::ZBITS;
        }
    };

    FewWeights<BITS, FOLDS> next;
    int held = min(first_of(0), f.quanta - 1);               // the quantum in `next`
    load(held, next);

    float4v y[MB][4];
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int b = 0; b < 4; ++b) y[m][b] = 0.0f;
    const HalfConst hc = half_constants<BITS>();

    for (int c0 = 0; c0 < f.quanta; c0 += chunk) {
        const int here = f.quanta - c0 < chunk ? f.quanta - c0 : chunk;
        // X of the chunk into LDS: a wavefront takes 64 x OCT k of a row at a time
        const int pieces = (here * QK + 64 * OCT - 1) / (64 * OCT);
        auto take = [&](int i, float *v, int &row, int &k) {
            row = i / pieces;
            k = (i - row * pieces) * 64 * OCT + lane * OCT;
            const int64_t at = t.begin + row;
            const int64_t from = a.rows ? a.rows[at] : at;
            const bool real = from >= 0 && from < a.x_rows;
#pragma unroll
            for (int o = 0; o < OCT; o += 8) {
                const int64_t kk = (int64_t)c0 * QK + k + o;
                if (real && kk < a.K) {
                    if (a.x_type == QG_F32) load_eight<QG_F32>(a.x, from * a.x_stride + kk, v + o);
                    else if (a.x_type == QG_BF16) load_eight<QG_BF16>(a.x, from * a.x_stride + kk, v + o);
                    else load_eight<QG_F16>(a.x, from * a.x_stride + kk, v + o);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[o + e] = 0.0f;
                }
            }
        };
        float first[OCT];
        int first_row = 0, first_k = 0;
        if (wave < rows * pieces) take(wave, first, first_row, first_k);
        if (a.x_type != QG_F16) {
            for (int i = wave; i < rows * pieces; i += 8) {
                float v[OCT];
                int row = first_row, k = first_k;
                if (i == wave) {
#pragma unroll
                    for (int e = 0; e < OCT; ++e) v[e] = first[e];
                } else {
                    take(i, v, row, k);
                }
                uint32_t m = 0;
#pragma unroll
                for (int e = 0; e < OCT; ++e) m = max(m, magnitude_bits(v[e]));
                m = most_of(m, 64);
                if (lane == 0) atomicMax(&most[row], m);
            }
            __syncthreads();
        }
        for (int i = wave; i < rows * pieces; i += 8) {
            float v[OCT];
            int row = first_row, k = first_k;
            if (i == wave) {
#pragma unroll
                for (int e = 0; e < OCT; ++e) v[e] = first[e];
            } else {
                take(i, v, row, k);
            }
            const int up = a.x_type == QG_F16 ? 0 : row_exponent(most[row]);
            float p[OCT];
#pragma unroll
            for (int e = 0; e < OCT; ++e) p[k_position<BITS>(e)] = a.x_type == QG_F16 ? v[e] : __builtin_amdgcn_ldexpf(v[e], up);
            if (k < here * QK) {
                char *to = smem + row * parts * stride + k * 2;
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    if (part < parts) {
#pragma unroll
                        for (int o = 0; o < OCT; o += 8)
                            *(uint4 *)(to + o * 2) = make_uint4(two_halves(p[o], p[o + 1]), two_halves(p[o + 2], p[o + 3]), two_halves(p[o + 4], p[o + 5]), two_halves(p[o + 6], p[o + 7]));
                        to += stride;
#pragma unroll
                        for (int e = 0; e < OCT; ++e) p[e] = left_over(p[e]);
                    }
                }
            }
        }
        __syncthreads();

        // this wavefront's quanta
        const int q0 = first_of(c0), q1 = c0 + here * (slice + 1) / slices;
        float4v part_y[MB][4];
#pragma unroll
        for (int m = 0; m < MB; ++m)
#pragma unroll
            for (int b = 0; b < 4; ++b) part_y[m][b] = 0.0f;
        const char *xa[MB];
#pragma unroll
        for (int m = 0; m < MB; ++m) {
            const int v = 16 * m + (lane & 15);
            xa[m] = smem + (v < vrows ? v : vrows - 1) * stride + (lane >> 4) * 16;
        }
        if (q0 < q1 && held != q0) load(q0, next);           // (after a chunk of fewer quanta than slices)
        for (int q = q0; q < q1; ++q) {
            const FewWeights<BITS, FOLDS> w = next;
            held = min(q + 1 < q1 ? q + 1 : c0 + chunk < f.quanta ? first_of(c0 + chunk) : q, f.quanta - 1);
            load(held, next);
#pragma unroll
            for (int i = 0; i < FOLDS; ++i) {
                uint32_t s[4], zw[4];
                spread_16(w.s[i], s);
                spread_16((w.z[i] >> w.shift[i]) & ((1u << F::ZBITS) - 1), zw);
                uint32_t ops[GP][4];
                HalfOperand x[GP][MB];
#pragma unroll
                for (int g = 0; g < GP; ++g) {
                    uint32_t words[4];
                    words_of<BITS>(w.v, i * GP + g, words);
                    words_16<BITS>(words, ops[g]);
#pragma unroll
                    for (int m = 0; m < MB; ++m) x[g][m].q = *(const uint4 *)(xa[m] + ((q - c0) * QK + (i * GP + g) * 32) * 2);
                }
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    uint32_t zc[4];
                    zero_operands<BITS>(zw[b], zc);
                    float4v sum[MB];
#pragma unroll
                    for (int m = 0; m < MB; ++m) sum[m] = 0.0f;
#pragma unroll
                    for (int g = 0; g < GP; ++g) {
                        HalfOperand o;
                        unpack_halves<BITS>(ops[g][b], hc, zc, o);
#pragma unroll
                        for (int m = 0; m < MB; ++m) sum[m] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[g][m].v, o.v, sum[m], 0, 0, 0);
                    }
#pragma unroll
                    for (int m = 0; m < MB; ++m)
#pragma unroll
                        for (int e = 0; e < 4; ++e) part_y[m][b][e] = __builtin_fmaf(__uint_as_float(s[b]), sum[m][e], part_y[m][b][e]);
                }
            }
        }
        // back from the rows' scales
#pragma unroll
        for (int m = 0; m < MB; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int v = 16 * m + 4 * (lane >> 4) + e;
                const int down = a.x_type == QG_F16 || v >= vrows ? 0 : -row_exponent(most[parts == 2 ? v >> 1 : v]);
#pragma unroll
                for (int b = 0; b < 4; ++b) y[m][b][e] += __builtin_amdgcn_ldexpf(part_y[m][b][e], down);
            }
        __syncthreads();
        if (threadIdx.x < FEW_ROWS) most[threadIdx.x] = 0;
        __syncthreads();
    }

    // slices meet, 16 operand rows at a time
    float *sums = (float *)smem;
#pragma unroll
    for (int m = 0; m < MB; ++m) {
        if (m > 0) __syncthreads();
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[(wave * 16 + 4 * (lane >> 4) + e) * FEW_PAD + 16 * b + (lane & 15)] = y[m][b][e];
        __syncthreads();
        const int first = 16 * m / parts, here = min(16 / parts, rows - first);
        const int wide = a.gated ? 64 : 64 * f.tiles;
        for (int i = threadIdx.x; i < here * wide; i += 512) {
            const int r = i / wide, col = i - r * wide;
            auto total = [&](int which) {
                float v = 0.0f;
                for (int sl = 0; sl < slices; ++sl) {
                    const int w = f.tiles == 2 ? 2 * sl + which : sl;
                    for (int p = 0; p < parts; ++p) v += sums[(w * 16 + r * parts + p) * FEW_PAD + (col & 63)];
                }
                return v;
            };
            const int64_t at = column0 + col;
            if (at >= a.columns) continue;
            const float v = a.gated ? silu(total(0)) * total(1) : total(col >> 6);
            store_typed(a.y_type, a.y, (t.begin + first + r) * a.columns + at, v);
        }
    }
}

template <int BITS, int GP>
__global__ __launch_bounds__(512, 4) void experts_few(const QgFewArgs f)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ uint32_t most[FEW_ROWS];
    // workgroup i runs on die i % 8: a die's workgroups take neighbouring pieces, so that an expert's tiles of rows share its weights
    int block = blockIdx.x;
    {
        const int die = block & 7, each = f.blocks >> 3, more = f.blocks & 7;
        block = die * each + (die < more ? die : more) + (block >> 3);
    }
    const int columns = block / f.e.row_tiles;
    const ExpertTile t = expert_tile(f.e, block - columns * f.e.row_tiles, f.tile_rows);
    if (t.rows == 0) return;
    if (threadIdx.x < FEW_ROWS) most[threadIdx.x] = 0;
    __syncthreads();
    const int expert = __builtin_amdgcn_readfirstlane(t.expert), rows = __builtin_amdgcn_readfirstlane(t.rows);
    const ExpertTile u = {expert, rows, (int64_t)__builtin_amdgcn_readfirstlane((int)t.begin)};
    const int64_t column0 = (int64_t)columns * (f.e.gated || f.tiles == 1 ? 64 : 128);
    const int parts = f.e.x_type == QG_F32 ? 2 : 1;
    if (rows * parts <= 16) few_rows<BITS, GP, 1>(f, u, column0, smem, most, rows, parts);
    else few_rows<BITS, GP, 2>(f, u, column0, smem, most, rows, parts);
}

template <int BITS>
void few_launch(const QgFewArgs &f, hipStream_t st)
{
    if (f.g32 % 4 == 0) experts_few<BITS, 4><<<f.blocks, 512, FEW_LDS, st>>>(f);
    else if (f.g32 % 2 == 0) experts_few<BITS, 2><<<f.blocks, 512, FEW_LDS, st>>>(f);
    else experts_few<BITS, 1><<<f.blocks, 512, FEW_LDS, st>>>(f);
}

}  // namespace
#endif

void qg_few_launch_b2(const QgFewArgs &f, hipStream_t st);
void qg_few_launch_b3(const QgFewArgs &f, hipStream_t st);
void qg_few_launch_b4(const QgFewArgs &f, hipStream_t st);

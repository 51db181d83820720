// The experts' products where an expert has few rows: bound by reading the packed matrices once.
//
// A workgroup of eight wavefronts takes 1, 2, 4 or 8 tiles of 64 outputs (gated: gates and ups of half as many columns) of up to 16
// operand rows of an expert, K cut into 8, 4, 2 or 1 slices of whole 128 k over its wavefronts.  X goes through LDS as f16 (rows of two parts if it is fp32),
// in the order in which the codes come out of their words; the weights go from memory into registers, in a ring of a few times 128 k that no register leaves by a
// copy (which would wait for it), and into the 16 x 16 x 32 matrix instruction as q - z.  fp32 sums of a group (or 128 k of it) are multiplied by its scale; slices meet in LDS.
//
// A workgroup waits for offsets, rows and X, one after the other, before it multiplies, and for its wavefronts at the end: so it takes
// as many tiles as leave the chip one round of workgroups (few_plan).
#pragma once

#include "qg_experts_codes.h"

constexpr int FEW_LDS = (64 << 10) - 256;      // for rows of X; and 35 KB at the end
constexpr int FEW_ROWS = 16;                   // operand rows
constexpr int FEW_PAD = 68;                    // floats from one row of sums to the next: rows 4 apart on other banks

struct QgFewArgs {
    QgExpertsArgs e;
    int tile_rows;             // rows of X a workgroup takes
    int tiles, tile_shift;     // tiles of 64 outputs a workgroup takes: 1, 2, 4 or 8, and its logarithm
    int g32, gshift;           // group / 32, its logarithm or -1
    int quanta;                // of K
    int blocks;
};

#ifdef QG_EXPERTS_KERNELS
namespace {

// Weights of 128 k, as loaded: GP times 32 k share a scale; GP 0: groups of an odd number of 32 k (or of pairs), a scale for each 32 k.
template <int BITS, int GP>
struct FewWeights {
    static constexpr int FOLDS = GP ? 4 / GP : 4, ZEROS = GP ? 1 : FOLDS;
    uint4 v[BITS];
    uint32_t s[FOLDS], z[ZEROS];               // scales, and the words with the zero-points (shifted where they are used: a shift here would wait)
    int shift[FOLDS];
};

// RING: how many times 128 k are under way.
template <int BITS, int GP, int RING>
__device__ inline void few_rows(const QgFewArgs &f, const ExpertTile &t, int64_t column0, char *smem, uint32_t *most, int rows, int parts)
{
    using F = Fmt<BITS>;
    using Weights = FewWeights<BITS, GP>;
    constexpr int QK = 128, FOLDS = Weights::FOLDS, PER = 4 / FOLDS, ZPER = 32 / F::ZBITS;
    constexpr int OCT = BITS == 2 ? 16 : 8;
    const QgExpertsArgs &a = f.e;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = wave & (f.tiles - 1), slices = 8 >> f.tile_shift, slice = wave >> f.tile_shift;
    const int vrows = rows * parts;

    // this lane's output
    const int64_t column = column0 + (a.gated ? tile >> 1 : tile) * 64 + lane;
    const int64_t n = (column < a.columns ? column : a.columns - 1) + (a.gated ? (int64_t)(tile & 1) * a.columns : 0);
    const OutputWeights at_n = output_weights(a, t.expert, n);
    const int last_group = a.K / a.group - 1;

    // quanta of X that fit, a whole number for each slice
    int chunk = FEW_LDS / vrows / 2 / QK;                    // (of 16 bytes a row for bank offsets: QK >= 128 leaves them room below)
    while (chunk > 1 && vrows * (chunk * QK * 2 + 16) > FEW_LDS) --chunk;
    chunk = chunk >= f.quanta ? f.quanta : chunk > slices ? chunk / slices * slices : chunk;
    const int stride = chunk * QK * 2 + 16;

    auto load = [&](int q, Weights &w) {
#pragma unroll
        for (int i = 0; i < BITS; ++i) w.v[i] = *(const uint4 *)(at_n.codes + ((int64_t)q * BITS + i) * 1024 + at_n.codes_lane);
#pragma unroll
        for (int i = 0; i < FOLDS; ++i) {
            const int k32 = q * 4 + i * PER;
            int g = GP ? k32 >> f.gshift : k32 / f.g32;
            g = g < last_group ? g : last_group;
            w.s[i] = *(const uint32_t *)(at_n.scales + (int64_t)g * 256 + at_n.scales_lane);
            // (a scale for 32, 64 or whole multiples of 128 k: 128 k's zero-points lie in one word)
            if (i < Weights::ZEROS) w.z[i] = *(const uint32_t *)(at_n.zeros + (int64_t)(g / ZPER) * 256 + at_n.zeros_lane);
            w.shift[i] = g % ZPER * F::ZBITS;
        }
    };

    float4v y[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) y[b] = 0.0f;
    const HalfConst hc = half_constants<BITS>();
    int up_y[4];                                             // powers of two that y's rows are multiplied by

    for (int c0 = 0; c0 < f.quanta; c0 += chunk) {
        const int here = f.quanta - c0 < chunk ? f.quanta - c0 : chunk;
        // this wavefront's part
        const int q0 = c0 + here * slice / slices, q1 = c0 + here * (slice + 1) / slices;
        Weights ring[RING];
#pragma unroll
        for (int i = 0; i < RING; ++i)
            if (q0 + i < q1) load(q0 + i, ring[i]);
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
        if (a.x_type != QG_F16) {
            for (int i = wave; i < rows * pieces; i += 8) {
                float v[OCT];
                int row, k;
                take(i, v, row, k);
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
            int row, k;
            take(i, v, row, k);
            const int up = a.x_type == QG_F16 ? 0 : row_exponent(most[row]);      // of the largest |x| so far
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

        // y of the chunks before goes over to this one's powers of two, which are not above theirs
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int v = 4 * (lane >> 4) + e;
            const int up = a.x_type == QG_F16 || v >= vrows ? 0 : row_exponent(most[parts == 2 ? v >> 1 : v]);
            if (c0 > 0)
#pragma unroll
                for (int b = 0; b < 4; ++b) y[b][e] = __builtin_amdgcn_ldexpf(y[b][e], up - up_y[e]);
            up_y[e] = up;
        }
        const char *xa = smem + ((lane & 15) < vrows ? lane & 15 : vrows - 1) * stride + (lane >> 4) * 16;
        for (int q = q0; q < q1; q += RING) {
#pragma unroll
            for (int at = 0; at < RING; ++at) {
                if (at > 0 && q + at >= q1) break;
                Weights &w = ring[at];
#pragma unroll
                for (int i = 0; i < FOLDS; ++i) {
                    // A branch that is always taken keeps the next scale's operands out of this one's code: the compiler would
                    // begin with all of them at once, in registers that there are not (up to 400 spilled).
                    int go = 1;
                    if (i > 0) asm volatile("" : "+s"(go));
                    if (!go) continue;
                    uint32_t s[4], zw[4];
                    spread_16(w.s[i], s);
                    spread_16((w.z[i < Weights::ZEROS ? i : 0] >> w.shift[i]) & ((1u << F::ZBITS) - 1), zw);
                    uint32_t zc[4][zero_constants<BITS>()];
                    float4v sum[4];
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        zero_operands<BITS>(zw[b], zc[b]);
                        sum[b] = 0.0f;
                    }
#pragma unroll
                    for (int g = 0; g < PER; ++g) {
                        uint32_t words[4], ops[4];
                        words_of<BITS>(w.v, i * PER + g, words);
                        words_16<BITS>(words, ops);
                        HalfOperand x;
                        x.q = *(const uint4 *)(xa + ((q + at - c0) * QK + (i * PER + g) * 32) * 2);
#pragma unroll
                        for (int b = 0; b < 4; ++b) {
                            HalfOperand o;
                            unpack_halves<BITS>(ops[b], hc, zc[b], o);
                            sum[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x.v, o.v, sum[b], 0, 0, 0);
                        }
                    }
#pragma unroll
                    for (int b = 0; b < 4; ++b)
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[b][e] = __builtin_fmaf(__uint_as_float(s[b]), sum[b][e], y[b][e]);
                }
                if (q + at + RING < q1) load(q + at + RING, w);
            }
        }
        __syncthreads();
    }

    // slices meet
    float *sums = (float *)smem;
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[(wave * 16 + 4 * (lane >> 4) + e) * FEW_PAD + 16 * b + (lane & 15)] = __builtin_amdgcn_ldexpf(y[b][e], -up_y[e]);
    __syncthreads();
    const int wide_shift = 6 + f.tile_shift - a.gated, wide = 1 << wide_shift;
    for (int i = threadIdx.x; i < rows * wide; i += 512) {
        const int r = i >> wide_shift, col = i & (wide - 1);
        auto total = [&](int which) {
            float v = 0.0f;
            for (int sl = 0; sl < slices; ++sl)
                for (int p = 0; p < parts; ++p) v += sums[((sl * f.tiles + which) * 16 + r * parts + p) * FEW_PAD + (col & 63)];
            return v;
        };
        const int64_t at = column0 + col;
        if (at >= a.columns) continue;
        const float v = a.gated ? silu(total(col >> 6 << 1)) * total((col >> 6 << 1) + 1) : total(col >> 6);
        store_typed(a.y_type, a.y, (t.begin + r) * a.columns + at, v);
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
    const int64_t column0 = (int64_t)columns << (6 + f.tile_shift - f.e.gated);
    const int parts = f.e.x_type == QG_F32 ? 2 : 1;
    few_rows<BITS, GP, BITS == 4 ? 2 : 3>(f, u, column0, smem, most, rows, parts);
}

template <int BITS>
void few_launch(const QgFewArgs &f, hipStream_t st)
{
    if (f.gshift < 0) experts_few<BITS, 0><<<f.blocks, 512, FEW_LDS, st>>>(f);
    else if (f.g32 % 4 == 0) experts_few<BITS, 4><<<f.blocks, 512, FEW_LDS, st>>>(f);
    else if (f.g32 == 2) experts_few<BITS, 2><<<f.blocks, 512, FEW_LDS, st>>>(f);
    else experts_few<BITS, 1><<<f.blocks, 512, FEW_LDS, st>>>(f);
}

}  // namespace
#endif

void qg_few_launch_b2(const QgFewArgs &f, hipStream_t st);
void qg_few_launch_b3(const QgFewArgs &f, hipStream_t st);
void qg_few_launch_b4(const QgFewArgs &f, hipStream_t st);

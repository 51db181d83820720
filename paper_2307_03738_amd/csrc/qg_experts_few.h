// The experts' products where an expert has few rows: bound by reading the packed matrices once.
//
// A wavefront takes a tile of 64 outputs (gated: gates and ups of 32 columns) of up to 16 operand rows of an expert (8 of fp32, in two parts
// each) and a slice of K; a workgroup of four wavefronts is 1, 2 or 4 tiles by 4, 2 or 1 slices, which meet in LDS (of eight: one tile by
// eight slices).  Rows of X come as prepare_rows leaves them, from cache straight into the operands; the weights go from memory into registers,
// in a ring of twice 128 k that no register leaves by a copy (which would wait for it; rings of 1, 2, 3, 4 times: 22.9, 22.5, 23.2, 24.9 us for one token, 57.5, 59.1 for 61 tokens), and into the
// 16 x 16 x 32 matrix instruction as q - z.  fp32 sums of a group (or 128 k of it) are multiplied by its scale.
// Measured: 61 tokens' six of 64 2816 x 2048 4-bit matrices in groups of 32, 237 MB: 49 us, 4.8 TB/s (a copy 5.4); one token's two of eight
// 22016 x 4096, 91 MB: 22 us as a caller sees it; 24 tokens' four of 32 4096 x 1408 3-bit, 80 MB: 22.5 us, of which 3 are the launch and the meeting.  (With the same matrices
// call after call; with matrices in turn that no cache holds 55, 22 and 25 us.)
//
// A call with about one row for each expert that it uses does without prepare_rows: its workgroups convert their rows into LDS themselves (SELF), which is a kernel less
// (one token, two of eight 22016 x 4096 4-bit matrices: 23.5 us against 28.1; four of 32 2816 x 4096: 15.1, 18.4).  With more rows that costs every workgroup more than
// the kernel costs the call (61 tokens' 2816 x 2048 matrices, groups of 32: 73 to 86 us against 67.8, 20 to 36 of them before the first multiplication).
//
// Groups that are no whole 32 k take the matrix instruction twice for every 32 k (four times, where not even 16 k share a scale), with what other scales have set
// to zero in X: at groups of 16 and eight 4096 x 4096 4-bit matrices, 105 MB, 43 us with a row each, 47 with four, 119 with 32 (multiply-adds on the vector ALU, four rows
// at a time: 92, 179, 664).  They come here with any number of rows.
#pragma once

#include "qg_experts_rows.h"

constexpr int FEW_ROWS = 16;                   // operand rows
constexpr int FEW_LDS = 39 << 10;              // four workgroups a compute unit
constexpr int FEW_PAD = 80;                    // floats from one row of sums to the next: four rows on other banks

struct QgFewArgs {
    QgExpertsArgs e;
    const char *xh;            // of prepare_rows
    const int32_t *up;
    int64_t padded;
    int parts;
    int tile_rows;             // rows of X a workgroup takes
    int stride;                // SELF: bytes from one operand row to the next
    int waves;                 // of a workgroup: 4, or 8
    int tile_shift;            // logarithm of a workgroup's tiles
    int g32, gshift;           // group / 32, its logarithm or -1
    int cells;                 // > 0: groups that are no whole 32 k, in pieces of 16 k or, where that does not do, of 8
    int quanta;                // times 128 k
    int blocks;
};

#ifdef QG_EXPERTS_KERNELS
namespace {

// Weights of 128 k, as loaded: GP times 32 k share a scale; GP 0: groups of an odd number of 32 k (or of pairs), a scale for each 32 k;
// GP -2, -4: groups that are no whole 32 k, two or four scales for each 32 k.
template <int BITS, int GP>
struct FewWeights {
    static constexpr int SUB = GP < 0 ? -GP : 1, FOLDS = GP < 0 ? 4 * SUB : GP ? 4 / GP : 4, ZEROS = GP < 0 ? 2 : GP ? 1 : FOLDS;
    uint4 v[BITS];
    uint32_t s[FOLDS], z[ZEROS];               // scales, and the words with the zero-points (shifted where they are used: a shift here would wait)
    int shift[FOLDS];                          // GP < 0: which of the zero-points of both words
};

// RING: how many times 128 k are under way.
template <int BITS, int GP, int RING, int WAVES, bool SELF>
__global__ __launch_bounds__(64 * WAVES, GP < 0 ? 2 : 4) void experts_few(const QgFewArgs f)
{
    using F = Fmt<BITS>;
    using Weights = FewWeights<BITS, GP>;
    constexpr int SUB = Weights::SUB, FOLDS = Weights::FOLDS, TURNS = FOLDS / SUB, PER = 4 / TURNS, ZPER = 32 / F::ZBITS;
    extern __shared__ __attribute__((aligned(16))) char smem[];      // SELF: rows of X; then sums
    const QgExpertsArgs &a = f.e;
    // workgroup i runs on die i % 8: a die's workgroups take neighbouring pieces, so that an expert's tiles of rows share its weights
    int block = blockIdx.y * gridDim.x + blockIdx.x;
    if (block >= f.blocks) return;
    {
        const int die = block & 7, each = f.blocks >> 3, more = f.blocks & 7;
        block = die * each + (die < more ? die : more) + (block >> 3);
    }
    const int columns = block / a.row_tiles;
    const ExpertTile t = expert_tile(a, block - columns * a.row_tiles, f.tile_rows);
    if (t.rows == 0) return;
    const int expert = __builtin_amdgcn_readfirstlane(t.expert), rows = __builtin_amdgcn_readfirstlane(t.rows);
    const int64_t begin = __builtin_amdgcn_readfirstlane((int)t.begin);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tiles = 1 << f.tile_shift, tile = wave & (tiles - 1), slices = WAVES >> f.tile_shift, slice = wave >> f.tile_shift;

    // this lane's output
    const int width_shift = 6 - a.gated, tile_columns = 1 << width_shift;
    const int64_t column0 = (int64_t)columns << (width_shift + f.tile_shift);
    const int64_t column = column0 + tile * tile_columns + (lane & (tile_columns - 1));
    const int64_t n = (column < a.columns ? column : a.columns - 1) + (a.gated && lane >= 32 ? (int64_t)a.columns : 0);
    const OutputWeights at_n = output_weights(a, expert, n);
    const int last_group = a.K / a.group - 1;

    // this lane's operand row (row and part of it), and its quarter of every 32 k.  Row v is the instruction's row 4 (v % 4) + v / 4, so that the first
    // four come out in one register of every lane, the next four in the second, and only as many are added up as there are.
    const int v = (lane & 3) * 4 + (lane >> 2 & 3), quarter = lane >> 4, row_of = f.parts == 2 ? v >> 1 : v;
    int64_t row = a.x_rows;
    if (row_of < rows) {
        row = a.rows ? a.rows[begin + row_of] : begin + row_of;
        row = row >= 0 && row < a.x_rows ? row : a.x_rows;
    }
    const int octet = BITS == 2 ? 2 * (quarter & 1) + (quarter >> 1) : quarter;
    int up = 0;
    const char *x;
    if constexpr (SELF) x = smem + (row_of < rows ? v : 0) * f.stride + octet * 16;
    else {
        up = f.up[row];
        x = f.xh + ((row * f.parts + (f.parts == 2 ? v & 1 : 0)) * f.padded + octet * 8) * 2;
    }

    auto load = [&](int q, Weights &w) {
#pragma unroll
        for (int i = 0; i < BITS; ++i) w.v[i] = *(const uint4 *)(at_n.codes + ((int64_t)q * BITS + i) * 1024 + at_n.codes_lane);
        if constexpr (GP < 0) {
            // (128 k have zero-points of two words at most: whole words of them at groups of a cell, half as many at longer ones)
            int g = q * FOLDS / f.cells, in = q * FOLDS - g * f.cells;
            const int word = min(g, last_group) / ZPER;
#pragma unroll
            for (int i = 0; i < 2; ++i) w.z[i] = *(const uint32_t *)(at_n.zeros + (int64_t)min(word + i, last_group / ZPER) * 256 + at_n.zeros_lane);
#pragma unroll
            for (int i = 0; i < FOLDS; ++i) {
                const int at = min(g, last_group);
                w.s[i] = *(const uint32_t *)(at_n.scales + (int64_t)at * 256 + at_n.scales_lane);
                w.shift[i] = at - word * ZPER;
                if (++in == f.cells) {
                    in = 0;
                    ++g;
                }
            }
            return;
        }
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
    const int vrows = rows * f.parts;
    const int q0 = f.quanta * slice / slices, q1 = f.quanta * (slice + 1) / slices;
    Weights ring[RING];
#pragma unroll
    for (int i = 0; i < RING; ++i)
        if (q0 + i < q1) load(q0 + i, ring[i]);
    uint4 xs[SELF ? 1 : 4];                    // X of 128 k
    if constexpr (!SELF) {
#pragma unroll
        for (int i = 0; i < 4; ++i) xs[i] = *(const uint4 *)(x + ((int64_t)min(q0, f.quanta - 1) * 4 + i) * 64);
    }
    if constexpr (SELF) {
        __shared__ uint32_t mosts[WAVES];
        for (int r = 0; r < rows; ++r) {
            int64_t from = a.rows ? a.rows[begin + r] : begin + r;
            const bool real = from >= 0 && from < a.x_rows;
            from *= a.x_stride;
            constexpr int OCT = row_piece<BITS>();
            float p[OCT];
            auto take = [&](int k) {
#pragma unroll
                for (int o = 0; o < OCT; o += 8) eight_of_row(a.x, a.x_type, from, k + o, a.K, real, p + o);
            };
            uint32_t most = 0;
            if (a.x_type != QG_F16) {
                for (int k = threadIdx.x * OCT; k < a.K; k += 64 * WAVES * OCT) {
                    take(k);
#pragma unroll
                    for (int e = 0; e < OCT; ++e) most = max(most, magnitude_bits(p[e]));
                }
                most = most_of(most, 64);
                if (r > 0) __syncthreads();
                if (lane == 0) mosts[wave] = most;
                __syncthreads();
                most = mosts[0];
#pragma unroll
                for (int w = 1; w < WAVES; ++w) most = max(most, mosts[w]);
            }
            const int row_up = a.x_type == QG_F16 ? 0 : row_exponent(most);
            if (row_of == r) up = row_up;
            for (int k = threadIdx.x * OCT; k < f.quanta * 128; k += 64 * WAVES * OCT) {
                take(k);
                store_piece<BITS>(p, a.x_type, row_up, smem + r * f.parts * f.stride, f.stride, k);
            }
        }
        __syncthreads();
    }
    for (int q = q0; q < q1; q += RING) {
#pragma unroll
        for (int at = 0; at < RING; ++at) {
            if (at > 0 && q + at >= q1) break;
            Weights &w = ring[at];
#pragma unroll
            for (int i = 0; i < TURNS; ++i) {
                // A branch that is always taken keeps the next scale's operands out of this one's code: the compiler would
                // begin with all of them at once, in registers that there are not (up to 400 spilled).
                int go = 1;
                if (i > 0) asm volatile("" : "+s"(go));
                if (!go) continue;
                if constexpr (GP < 0) {
                    // every quarter of an operand has its own zero-points; the sums of a scale's k come from X with the other k zero
                    HalfOperand xo, o[4];
                    uint32_t words[4], ops[4], z[4];
                    if constexpr (SELF) xo.q = *(const uint4 *)(x + ((q + at) * 4 + i) * 64);
                    else xo.q = xs[i];
#pragma unroll
                    for (int k = 0; k < words_of_32<BITS>(); ++k) {
                        const int place = w.shift[i * SUB + k * SUB / words_of_32<BITS>()];
                        const uint32_t zero = ((place < ZPER ? w.z[0] : w.z[1]) >> (place % ZPER * F::ZBITS)) & ((1u << F::ZBITS) - 1);
                        words[k] = BITS == 2 ? zero * 0x101u : zero;
                    }
                    words_16<BITS>(words, z);
                    words_of<BITS>(w.v, i, words);
                    words_16<BITS>(words, ops);
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        uint32_t zc[zero_constants<BITS>()];
                        zero_operands<BITS>(BITS == 2 ? z[b] & 0xff : z[b], zc);
                        unpack_halves<BITS>(ops[b], hc, zc, o[b]);
                    }
#pragma unroll
                    for (int j = 0; j < SUB; ++j) {
                        uint32_t s[4];
                        spread_16(w.s[i * SUB + j], s);
                        HalfOperand part;
#pragma unroll
                        for (int e = 0; e < 4; ++e) part.r[e] = quarter * SUB / 4 == j ? xo.r[e] : 0;
#pragma unroll
                        for (int b = 0; b < 4; ++b) {
                            float4v sum = 0.0f;
                            sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(part.v, o[b].v, sum, 0, 0, 0);
                            y[b][0] = __builtin_fmaf(__uint_as_float(s[b]), sum[0], y[b][0]);
                            if (vrows > 4) y[b][1] = __builtin_fmaf(__uint_as_float(s[b]), sum[1], y[b][1]);
                            if (vrows > 8)
#pragma unroll
                                for (int e = 2; e < 4; ++e) y[b][e] = __builtin_fmaf(__uint_as_float(s[b]), sum[e], y[b][e]);
                        }
                    }
                    if constexpr (!SELF) xs[i] = *(const uint4 *)(x + ((int64_t)min(q + at + 1, f.quanta - 1) * 4 + i) * 64);
                    continue;
                }
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
                    HalfOperand xo;
                    if constexpr (SELF) xo.q = *(const uint4 *)(x + ((q + at) * 4 + i * PER + g) * 64);
                    else xo.q = xs[i * PER + g];
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        HalfOperand o;
                        unpack_halves<BITS>(ops[b], hc, zc[b], o);
                        sum[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xo.v, o.v, sum[b], 0, 0, 0);
                    }
                    if constexpr (!SELF) xs[i * PER + g] = *(const uint4 *)(x + ((int64_t)min(q + at + 1, f.quanta - 1) * 4 + i * PER + g) * 64);
                }
                auto fold = [&](int e) {
#pragma unroll
                    for (int b = 0; b < 4; ++b) y[b][e] = __builtin_fmaf(__uint_as_float(s[b]), sum[b][e], y[b][e]);
                };
                fold(0);
                if (vrows > 4) fold(1);
                if (vrows > 8) {
                    fold(2);
                    fold(3);
                }
            }
            if (q + at + RING < q1) load(q + at + RING, w);
        }
    }

    // slices meet; a row's second part was SECOND_UP higher than its first
    if (f.parts == 2 && (v & 1)) up += SECOND_UP;
    float *sums = (float *)smem;
    if constexpr (SELF) __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int down = -__shfl(up, 4 * quarter + e);
#pragma unroll
        for (int b = 0; b < 4; ++b) sums[(wave * 16 + 4 * e + quarter) * FEW_PAD + 16 * b + (lane & 15)] = __builtin_amdgcn_ldexpf(y[b][e], down);
    }
    __syncthreads();
    const int wide_shift = width_shift + f.tile_shift, wide = 1 << wide_shift;
    for (int i = threadIdx.x; i < rows * wide; i += 64 * WAVES) {
        const int r = i >> wide_shift, col = i & (wide - 1);
        auto total = [&](int output) {
            float sum = 0.0f;
            for (int sl = 0; sl < slices; ++sl)
                for (int p = 0; p < f.parts; ++p) sum += sums[((sl * tiles + (output >> 6)) * 16 + r * f.parts + p) * FEW_PAD + (output & 63)];
            return sum;
        };
        const int64_t at = column0 + col;
        if (at >= a.columns) continue;
        const float out = a.gated ? silu(total((col >> 5) * 64 + (col & 31))) * total((col >> 5) * 64 + 32 + (col & 31)) : total(col);
        store_typed(a.y_type, a.y, (begin + r) * a.columns + at, out);
    }
}

template <int BITS, int WAVES, bool SELF>
void few_typed(const QgFewArgs &f, hipStream_t st)
{
    constexpr int RING = 2;
    constexpr size_t of_sums = WAVES * 16 * FEW_PAD * 4;
    const size_t of_rows = (size_t)f.tile_rows * f.parts * f.stride, lds = SELF && of_rows > of_sums ? of_rows : of_sums;
    const unsigned across = (unsigned)(f.blocks < QG_MOST_GROUPS / 2 ? f.blocks : QG_MOST_GROUPS / 2);
    const dim3 grid(across, (f.blocks + across - 1) / across);
    if (f.cells) {
        if constexpr (BITS == 4) {
            if (f.cells * 8 == f.e.group) {
                experts_few<BITS, -4, RING, WAVES, SELF><<<grid, 64 * WAVES, lds, st>>>(f);
                return;
            }
        }
        if constexpr (BITS != 3) experts_few<BITS, -2, RING, WAVES, SELF><<<grid, 64 * WAVES, lds, st>>>(f);
    } else if (f.gshift < 0) experts_few<BITS, 0, RING, WAVES, SELF><<<grid, 64 * WAVES, lds, st>>>(f);
    else if (f.g32 % 4 == 0) experts_few<BITS, 4, RING, WAVES, SELF><<<grid, 64 * WAVES, lds, st>>>(f);
    else if (f.g32 == 2) experts_few<BITS, 2, RING, WAVES, SELF><<<grid, 64 * WAVES, lds, st>>>(f);
    else experts_few<BITS, 1, RING, WAVES, SELF><<<grid, 64 * WAVES, lds, st>>>(f);
}

template <int BITS>
void few_launch(const QgFewArgs &f, const QgPrepareArgs &p, hipStream_t st)
{
    if (f.stride) {
        if (f.waves == 4) few_typed<BITS, 4, true>(f, st);
        else few_typed<BITS, 8, true>(f, st);
    } else {
        prepare_launch<BITS>(p, st);
        if (f.waves == 4) few_typed<BITS, 4, false>(f, st);
        else few_typed<BITS, 8, false>(f, st);
    }
}

}  // namespace
#endif

void qg_few_launch_b2(const QgFewArgs &f, const QgPrepareArgs &p, hipStream_t st);
void qg_few_launch_b3(const QgFewArgs &f, const QgPrepareArgs &p, hipStream_t st);
void qg_few_launch_b4(const QgFewArgs &f, const QgPrepareArgs &p, hipStream_t st);

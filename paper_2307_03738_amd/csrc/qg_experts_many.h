// The experts' products where an expert has many rows: bound by the matrix cores and by what turns codes into operands.
//
// Rows of X come as prepare_rows leaves them.  A workgroup of four wavefronts takes up to 64 slots of an expert (or 32: many_rows_of) and 256 outputs, a wavefront all of the
// slots and 64 outputs of its own (gated: gate and up of 32 columns), so that every weight is unpacked once per workgroup.  X's rows, gathered
// by slot, go from memory to LDS without passing through registers, 128 k ahead, codes to registers; a wavefront reads each operand
// of X for two 32 x 32 x 16 matrix instructions (half of LDS's rate at full speed of the matrix cores).  Two workgroups share a compute unit: with 128
// slots and one wavefront a SIMD nothing covers what a wavefront waits for (4096 tokens, two of eight gated 22016 x 4096 4-bit matrices: 2.55 ms against 1.71 at that time).
//
// Where workgroups are few they have twelve wavefronts, four for each third of K, which add their sums up in LDS at the end (many_plan says when).
//
// That prompt now takes 1.48 to 1.57 ms, 0.93 to 0.98 PFLOP/s, in fp32 2.5; a library's product of bf16 matrices reaches 1.20.  Both are held by power (the clock falls to 2.0 GHz; a loop of nothing but
// matrix instructions reaches 1.65), here by 9 vector instructions beside each matrix instruction: a loop of just these and no memory makes 1.17 to 1.33.  Codes unpacked once for a
// whole workgroup by way of LDS make 0.95 to 1.04 in such a loop.  8184 slots of 60 5120 x 1792 2-bit matrices, groups of 64: 209 us (0.71 PFLOP/s; 14 steps of 128 k, 10.5 vector instructions and more in the last tiles).
#pragma once

#include <type_traits>

#include "qg_experts_rows.h"

struct QgManyArgs {
    QgExpertsArgs e;
    const char *xh;            // rows of f16, [x_rows + 1][parts][padded]: the last one zeros
    const int32_t *up;         // [x_rows + 1]: their powers of two
    int64_t padded;            // k a row is filled up to: a multiple of 128
    int parts;
    int g32, gshift;
    int tile_rows;             // slots of a workgroup: 32 or 64
    int slices;                // of K: 1, or 3, four wavefronts each
    int column_blocks;         // of 256 outputs
    int blocks;
};

#ifdef QG_EXPERTS_KERNELS
namespace {

// MB: blocks of 32 slots.
template <int BITS, int GP, int PARTS, int MB, int SLICES>
__device__ inline void many_rows(const QgManyArgs &f, const ExpertTile &t, int64_t column0, char *smem, int32_t *ups)
{
    using F = Fmt<BITS>;
    constexpr int LOADS = BITS, FOLDS = 4 / GP, ZPER = 32 / F::ZBITS;      // of 128 k
    constexpr int ROWS = 32 * MB, STAGE = ROWS * 256 * PARTS;
    constexpr int COPIES = ROWS * PARTS / 16;                              // of 4 rows, a wavefront's
    const QgExpertsArgs &a = f.e;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6 & 3);
    const int slice = SLICES == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
    const int half = lane >> 5;

    // this lane's output
    const int64_t wave_column = column0 + wave * (a.gated ? 32 : 64);
    const int64_t column = wave_column + (a.gated ? lane & 31 : lane);
    const int64_t n = (column < a.columns ? column : a.columns - 1) + (a.gated && half ? (int64_t)a.columns : 0);
    const OutputWeights at_n = output_weights(a, t.expert, n);
    const int last_group = a.K / a.group - 1;
    const int steps = (a.K + 127) / 128, begin = steps * slice / SLICES, end = steps * (slice + 1) / SLICES;
    char *const stages = smem + slice * 2 * STAGE;

    // the rows it copies: 16 bytes of row 4 j + lane / 16 each, octet (lane % 16) ^ (row % 16) of the 128 k, so that 16 rows' octets of the same k
    // lie on distinct banks
    uint64_t from[COPIES];
#pragma unroll
    for (int j = 0; j < COPIES; ++j) {
        const int at = (wave * COPIES + j) * 4 + (lane >> 4), part = at / ROWS, r = at % ROWS;
        int64_t row = a.x_rows;
        if (r < t.rows) {
            row = a.rows ? a.rows[t.begin + r] : t.begin + r;
            row = row >= 0 && row < a.x_rows ? row : a.x_rows;
        }
        if (part == 0 && (lane & 15) == 0 && slice == 0) ups[r] = f.up[row];
        from[j] = (uint64_t)(uintptr_t)(f.xh + ((row * PARTS + part) * f.padded) * 2 + (((lane & 15) ^ (r & 15)) * 16));
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)stages;
    auto copy = [&](int step, int stage) {
#pragma unroll
        for (int j = 0; j < COPIES; ++j) {
            const uint64_t src = from[j] + (uint64_t)step * 256;
            const uint32_t dst = __builtin_amdgcn_readfirstlane(lds0 + stage * STAGE + (wave * COPIES + j) * 1024);
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(dst), "v"(src) : "memory", "m0");
        }
    };
    struct Weights {
        uint4 v[LOADS];
        uint32_t s[FOLDS], z[FOLDS];           // scale, and the word with the zero-point (shifted where it is used: a shift here would wait)
        int shift[FOLDS];
    };
    auto load = [&](int step, Weights &w) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) w.v[i] = *(const uint4 *)(at_n.codes + ((int64_t)step * LOADS + i) * 1024 + at_n.codes_lane);
#pragma unroll
        for (int i = 0; i < FOLDS; ++i) {
            const int k32 = step * 4 + i * GP;
            int g = f.gshift >= 0 ? k32 >> f.gshift : k32 / f.g32;
            g = g < last_group ? g : last_group;
            w.s[i] = *(const uint32_t *)(at_n.scales + (int64_t)g * 256 + at_n.scales_lane);
            w.z[i] = *(const uint32_t *)(at_n.zeros + (int64_t)(g / ZPER) * 256 + at_n.zeros_lane);
            w.shift[i] = g % ZPER * F::ZBITS;
        }
    };

    float16v y[MB][2];
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int b = 0; b < 2; ++b) y[m][b] = 0.0f;
    const HalfConst hc = half_constants<BITS>();
    const int r0 = lane & 31;

    Weights next;
    if (begin < end) {
        copy(begin, 0);
        load(begin, next);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    const int turns = (steps + SLICES - 1) / SLICES;               // as many for every slice, for their barriers
    for (int turn = 0; turn < turns; ++turn) {
        const int step = begin + turn;
        if (SLICES > 1 && step >= end) {
            __builtin_amdgcn_s_barrier();
            continue;
        }
        const Weights w = next;
        const char *x = stages + (turn & 1) * STAGE;
        if (step + 1 < end) {
            copy(step + 1, (turn + 1) & 1);
            load(step + 1, next);
        }
        // sixteens of k: operands of X are read AHEAD sixteens before they are multiplied (one where two would not fit into the registers: fp32 with a scale for each 32 k,
        // 390 slots of three 2646 x 7104 3-bit matrices, groups of 96, in slices: 82 us, with two 89), codes unpacked right before
        constexpr int KS = 2 * GP, AHEAD = PARTS == 2 && GP == 1 ? 1 : 2;
        HalfOperand xo[8][MB * PARTS];
        auto read = [&](int k) {
#pragma unroll
            for (int m = 0; m < MB; ++m)
#pragma unroll
                for (int part = 0; part < PARTS; ++part)
                    xo[k][m * PARTS + part].q = *(const uint4 *)(x + (part * ROWS + m * 32 + r0) * 256 + (((2 * k + half) ^ (r0 & 15)) * 16));
        };
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) read(k);
#pragma unroll
        for (int i = 0; i < FOLDS; ++i) {
            const auto s = __builtin_amdgcn_permlane32_swap(w.s[i], w.s[i], false, false);
            const uint32_t z = (w.z[i] >> w.shift[i]) & ((1u << F::ZBITS) - 1);
            const auto zz = __builtin_amdgcn_permlane32_swap(z, z, false, false);
            uint32_t zc[2][4];
            zero_operands<BITS>(zz[0], zc[0]);
            zero_operands<BITS>(zz[1], zc[1]);
            float16v sum[MB][2];
#pragma unroll
            for (int m = 0; m < MB; ++m)
#pragma unroll
                for (int b = 0; b < 2; ++b) sum[m][b] = 0.0f;
#pragma unroll
            for (int g = 0; g < GP; ++g) {
                uint32_t words[4];
                words_of<BITS>(w.v, i * GP + g, words);
                const auto p2 = __builtin_amdgcn_permlane32_swap(words[0], words[1], false, false);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int k = i * KS + 2 * g + h;
                    if (k + AHEAD < 8) read(k + AHEAD);
                    HalfOperand o[2];
                    if constexpr (BITS == 2) {
#pragma unroll
                        for (int b = 0; b < 2; ++b) unpack_halves<BITS>(p2[b] >> (8 * h), hc, zc[b], o[b]);
                    } else {
                        const auto p = h == 0 ? p2 : __builtin_amdgcn_permlane32_swap(words[2 % words_of_32<BITS>()], words[3 % words_of_32<BITS>()], false, false);
#pragma unroll
                        for (int b = 0; b < 2; ++b) unpack_halves<BITS>(p[b], hc, zc[b], o[b]);
                    }
#pragma unroll
                    for (int part = 0; part < PARTS; ++part) {
                        // (in place: 2 to 5 % of an fp32 call's time, with a scale for each 32 k up to 11; operands of their own up to 14 and 20)
                        if (part)
#pragma unroll
                            for (int b = 0; b < 2; ++b) second_weights(o[b]);
#pragma unroll
                        for (int m = 0; m < MB; ++m)
#pragma unroll
                            for (int b = 0; b < 2; ++b) sum[m][b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(xo[k][m * PARTS + part].v, o[b].v, sum[m][b], 0, 0, 0);
                    }
                }
            }
#pragma unroll
            for (int m = 0; m < MB; ++m)
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int e = 0; e < 16; ++e) y[m][b][e] = __builtin_fmaf(__uint_as_float(s[b]), sum[m][b][e], y[m][b][e]);
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
    }

    if constexpr (SLICES > 1) {
        // slices meet: the first adds the others' sums in order (every wavefront is behind the last barrier: the stages are free)
        float *sums = (float *)smem;
        constexpr int OF_WAVE = MB * 32 * 64;
        if (slice > 0) {
            float *to = sums + ((slice - 1) * 4 + wave) * OF_WAVE + lane;
#pragma unroll
            for (int m = 0; m < MB; ++m)
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int e = 0; e < 16; ++e) to[((m * 2 + b) * 16 + e) * 64] = y[m][b][e];
        }
        __syncthreads();
        if (slice > 0) return;
        for (int sl = 1; sl < SLICES; ++sl) {
            const float *from = sums + ((sl - 1) * 4 + wave) * OF_WAVE + lane;
#pragma unroll
            for (int m = 0; m < MB; ++m)
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int e = 0; e < 16; ++e) y[m][b][e] += from[((m * 2 + b) * 16 + e) * 64];
        }
    }
    // powers of two back, gates into their ups; then out: the type is asked for once, rows lie in scalar addresses, a lane's column and half beside them
    auto finish = [&](auto gated) {
#pragma unroll
        for (int m = 0; m < MB; ++m)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int r = 32 * m + 8 * (e / 4) + e % 4;
                if (r >= t.rows) continue;
                const int down = -ups[r + 4 * half];
                const float v0 = __builtin_amdgcn_ldexpf(y[m][0][e], down), v1 = __builtin_amdgcn_ldexpf(y[m][1][e], down);
                y[m][0][e] = decltype(gated)::value ? silu(v0) * v1 : v0;
                y[m][1][e] = v1;
            }
    };
    if (a.gated) finish(std::true_type());
    else finish(std::false_type());
    const int64_t c = wave_column + r0;
    const bool first = c < a.columns, second = !a.gated && c + 32 < a.columns;
    auto store = [&](auto type) {
        constexpr int TYPE = decltype(type)::value, SIZE = TYPE == QG_F32 ? 4 : 2;
        const uint32_t lane_at = ((uint32_t)(4 * half) * (uint32_t)a.columns + r0) * SIZE;
#pragma unroll
        for (int m = 0; m < MB; ++m)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int r = 32 * m + 8 * (e / 4) + e % 4;
                if (r >= t.rows) continue;
                char *to = (char *)a.y + ((t.begin + r) * a.columns + wave_column) * SIZE + lane_at;
                if (r + 4 * half < t.rows) {
                    if (first) store_float<TYPE>(to, 0, y[m][0][e]);
                    if (second) store_float<TYPE>(to, 32, y[m][1][e]);
                }
            }
    };
    if (a.y_type == QG_F32) store(std::integral_constant<int, QG_F32>());
    else if (a.y_type == QG_BF16) store(std::integral_constant<int, QG_BF16>());
    else store(std::integral_constant<int, QG_F16>());
}

// MOST: 32 slots in registers for three workgroups a compute unit, or 64 for two.  SLICES: a workgroup has so many times four wavefronts, each four a slice of K.
template <int BITS, int GP, int PARTS, int MOST, int SLICES>
__global__ __launch_bounds__(256 * SLICES, MOST == 1 ? 3 : 2) void experts_many(const QgManyArgs f)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ int32_t ups[32 * MOST];
    // A die's workgroups (number % 8) take neighbouring pieces, eight blocks of columns by as many tiles of slots: they share X's rows and weights in its L2.
    // Shares are of the tiles that there are, not of those that there could be: otherwise a die had up to 13 % more than its part (8184 slots of 60 experts: 236 us, 209 so).
    // (up to 64 experts are looked at once, for the number of tiles and for the workgroup's own)
    const ExpertTiles first(f.e, 0, 32 * MOST);
    const int tiles = f.e.experts > 64 ? expert_tiles(f.e, 32 * MOST) : first.total() < 0 || first.total() > f.e.row_tiles ? f.e.row_tiles : first.total();
    const int number = blockIdx.y * gridDim.x + blockIdx.x;
    int block = number >> 3;
    {
        const int blocks = tiles * f.column_blocks, die = number & 7, each = blocks >> 3, more = blocks & 7;
        if (block >= each + (die < more)) return;
        block += die * each + (die < more ? die : more);
    }
    const int band = block / (8 * tiles), across = min(8, f.column_blocks - 8 * band);
    const int rest = block - band * 8 * tiles;
    ExpertTile t = {0, 0, 0};
    if (f.e.experts > 64) t = expert_tile(f.e, rest / across, 32 * MOST);
    else first.take(rest / across, 32 * MOST, t);
    if (t.rows == 0) return;
    const int expert = __builtin_amdgcn_readfirstlane(t.expert), rows = __builtin_amdgcn_readfirstlane(t.rows);
    const ExpertTile u = {expert, rows, (int64_t)__builtin_amdgcn_readfirstlane((int)t.begin)};
    const int64_t column0 = (int64_t)(8 * band + rest % across) * (f.e.gated ? 128 : 256);
    if (rows <= 32) many_rows<BITS, GP, PARTS, 1, SLICES>(f, u, column0, smem, ups);
    else if constexpr (MOST == 2) many_rows<BITS, GP, PARTS, 2, SLICES>(f, u, column0, smem, ups);
}

template <int BITS, int GP, int PARTS, int MOST, int SLICES>
int many_sized(const QgManyArgs &f, hipStream_t st)
{
    constexpr size_t of_stages = (size_t)SLICES * 2 * 32 * MOST * 256 * PARTS, of_sums = (size_t)(SLICES - 1) * 4 * 32 * MOST * 64 * 4;
    constexpr size_t lds = of_stages > of_sums ? of_stages : of_sums;
    if (lds > 63 << 10) {
        static std::atomic<bool> prepared[64];      // once per device (devices past the table: every time)
        int dev = -1;
        if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) dev = -1;
        if (dev < 0 || !prepared[dev].load(std::memory_order_acquire)) {
            if (hipFuncSetAttribute((const void *)experts_many<BITS, GP, PARTS, MOST, SLICES>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) {
                (void)hipGetLastError();
                return QG_ERR_DEVICE;
            }
            if (dev >= 0) prepared[dev].store(true, std::memory_order_release);
        }
    }
    // (K is in slices where workgroups are few: lanes of a dimension number less than 2^32)
    const unsigned across = (unsigned)(f.blocks < QG_MOST_GROUPS ? f.blocks : QG_MOST_GROUPS);
    const dim3 grid(across, (f.blocks + across - 1) / across);
    experts_many<BITS, GP, PARTS, MOST, SLICES><<<grid, 256 * SLICES, lds, st>>>(f);
    return QG_OK;
}

template <int BITS, int GP, int PARTS>
int many_typed(const QgManyArgs &f, hipStream_t st)
{
    if (f.slices > 1) return many_sized<BITS, GP, PARTS, 1, 3>(f, st);
    return f.tile_rows == 32 ? many_sized<BITS, GP, PARTS, 1, 1>(f, st) : many_sized<BITS, GP, PARTS, 2, 1>(f, st);
}

template <int BITS>
int many_launch(const QgManyArgs &f, const QgPrepareArgs &p, hipStream_t st)
{
    prepare_launch<BITS>(p, st);
    if (f.parts == 2) return f.g32 % 4 == 0 ? many_typed<BITS, 4, 2>(f, st) : f.g32 % 2 == 0 ? many_typed<BITS, 2, 2>(f, st) : many_typed<BITS, 1, 2>(f, st);
    return f.g32 % 4 == 0 ? many_typed<BITS, 4, 1>(f, st) : f.g32 % 2 == 0 ? many_typed<BITS, 2, 1>(f, st) : many_typed<BITS, 1, 1>(f, st);
}

}  // namespace
#endif

int qg_many_launch_b2(const QgManyArgs &f, const QgPrepareArgs &p, hipStream_t st);
int qg_many_launch_b3(const QgManyArgs &f, const QgPrepareArgs &p, hipStream_t st);
int qg_many_launch_b4(const QgManyArgs &f, const QgPrepareArgs &p, hipStream_t st);

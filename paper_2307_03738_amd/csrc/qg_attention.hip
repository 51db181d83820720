// qg_paged_attention: attention of one new token of each sequence over a paged cache.
//
// out = sum_i p_i v_i / sum_i p_i over a sequence's keys, p_i = exp(scale q.k_i), in one pass with a running maximum.  Keys and
// values are read once and nothing else is of their size, so memory bounds it; the matrix instruction does both products
// with the (up to 16) heads that share a key head as one side of the 16 x 16 x 32 tile, and is busy for 5 % (16-bit
// cells) to 16 % (fp32 q on 8-bit cells) of the time, however few of the 16 there are.
//
// A wavefront takes 32 keys at a time, and nothing goes through LDS until it has seen all its keys:
//   S^T (keys x heads) = K Q^T   two products of 16 keys.  Lane l = 16 j + i loads elements of key 8 (i / 4) + 4 t + i % 4 in
//                                product t (rows of the left operand may be any keys): the accumulators of lane 16 j + i are then head
//                                i's scores of keys 8 j + 4 t + 0 ... 3,
//   O^T (dims x heads) = V^T P^T which is how the right operand of the second product wants them: head i, keys 8 j ... 8 j + 7.  Its left
//                                operand's rows are dims, which lie side by side in memory: lane 16 j + i loads 8 dims of each of its 8 keys
//                                and swaps halves of registers (one byte permutation for every two values).
// So maxima, sums and scaling factors of a head are in the lanes that need them; the 4 lanes of a head exchange their
// maximum only when some score exceeds the running one by 8 (a factor of 2^8 that fp32 sums do not feel).
//
// q goes in as it is: as one, two or three parts of 8 (bf16 instruction) or 11 bits (f16, with a power of two for each head
// taken out first); p as two or, for fp32 outputs on the bf16 instruction, three.  f16 has steps of 2^-24, below which many small p_i
// beside a large one would be lost: there p is kept 2^7 times as large, and its second part 2^11 times as large again, in products of its
// own that are added with 2^-11 (p to 2^-22 of itself or 2^-43 of the largest; 32 multiplications for 32 keys of 128 dims; 0 ... 2 % longer).
// 8-bit keys and values are exact in bf16; their scales are applied to the scores and to the p_i.
//
// An infinite cell times a part that is 0 or of the other sign is NaN where the whole is not.  So a workgroup that has seen a head's keys looks
// for NaN and infinity in what it has and, if there is one, sees them again with infinite cells in products of their own: with signs of q, and with
// 1 for each p_i.  (8-bit cells have no infinities.  Looking costs 0.2 us where there is little to do and up to 2 % where each head
// has keys of its own; f16 cells of other than 64, 128 or 256 dims lose 4 % to the registers that the second look takes.)
//
// Measured: 128 sequences of up to 8190 tokens, 64 heads on 8, bf16, 1.45 GB of cells: 253 us (5.8 TB/s; a workgroup per head with a key at a time:
// 8200); one sequence of 131071, 40 heads on 8, f16: 106 us (5.1 TB/s); 757 MB of 8-bit cells 167 ... 180 us; one sequence of 777, 32 key
// heads: 12.3 us, of which, by the clock in a copy, lengths take 1.5, page ids and q 2.5, cells 1.4, adding up in LDS 1.0, parts written and counted 0.8, their sum 3.
#include "qg_kv.h"

namespace {

constexpr int WAVES = 4;                   // wavefronts of a workgroup
constexpr int SPAN = 32 * WAVES;           // keys they take together
constexpr int MAX_WORKERS = 512;           // workgroups of a launch at most (sizes the counters in the workspace)
constexpr int COUNTER_BYTES = 4 * MAX_WORKERS;
constexpr float SLACK = 8.0f;
// Workgroups that a compute unit holds, by the registers that a head's dims take (three of 64 dims would spill and be no faster)
constexpr int groups_per_unit(int head_dim) { return head_dim <= 128 ? 2 : 1; }

struct AttentionArgs {
    QgKv kv;
    const int32_t *lens, *first;
    const void *q;
    void *out;
    float *lse;
    int64_t q_stride;
    int batch, heads, window, group;       // group: heads of a key head
    int blocks;                            // of at most 16 heads, that make up a group
    float scale;
    uint32_t *arrived;                     // [worker]
    float *parts;                          // [2 * worker + ...]: rows x head_dim sums, then rows x (maximum, sum of p)
    int part_floats;
    uint32_t parts_bytes;
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

union Operand {
    bf16x8 b;
    f16x8 h;
    uint32_t r[4];
};

template <bool F16>
__device__ inline floatx4 mma(const Operand &a, const Operand &b, floatx4 c)
{
    if constexpr (F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.h, b.h, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.b, b.b, c, 0, 0, 0);
}

// Two floats as a pair of bf16 or f16 to nearest, and what is left of them.
template <bool F16>
__device__ inline uint32_t take_part(float &a, float &b)
{
    if constexpr (F16) {
        const _Float16 x = (_Float16)a, y = (_Float16)b;
        a -= (float)x;
        b -= (float)y;
        return (uint32_t)__builtin_bit_cast(uint16_t, x) | (uint32_t)__builtin_bit_cast(uint16_t, y) << 16;
    } else {
        const bf16x2 v = {(__bf16)a, (__bf16)b};
        const uint32_t r = __builtin_bit_cast(uint32_t, v);
        a -= __uint_as_float(r << 16);
        b -= __uint_as_float(r & 0xffff0000u);
        return r;
    }
}

// Parts are written and read past the caches of the chip's dies.
constexpr int SC1 = 16;
typedef __amdgpu_buffer_rsrc_t rsrc_t;
__device__ inline rsrc_t buffer_of(const void *p, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, bytes, 0x00020000);
}

// Cells are read once, so they need not stay in the caches.
template <bool ONCE, typename T>
__device__ inline T load_cells(const char *p)
{
    if constexpr (ONCE) {
        typedef uint32_t words __attribute__((ext_vector_type(sizeof(T) / 4)));
        return __builtin_bit_cast(T, __builtin_nontemporal_load((const words *)p));
    } else {
        return *(const T *)p;
    }
}

// What a head's sums of values at maximum m are multiplied by to be at `top`: never 0 if there is a maximum, so that infinities stay
// (2^-149 of a finite one is nothing beside the largest value).
__device__ inline float value_weight(float m, float top) { return m == -INFINITY ? 0.0f : fmaxf(__builtin_amdgcn_exp2f(m - top), 0x1p-149f); }

// What a sum of p relative to maximum m counts relative to maximum `top`.  Without a score above -infinity the sum is 0, or NaN where
// scores were none, which has to come through.
__device__ inline float weight_of(float m, float top) { return m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - top); }

__device__ inline float across_quads_max(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}

// What a workgroup takes of a sequence: keys [base, len) in spans, of which those before `begin` are left out.
struct Keys {
    int begin, len, base, spans;
};

__device__ inline Keys keys_of(const AttentionArgs &a, int b)
{
    Keys k;
    const int limit = a.kv.max_pages << a.kv.page_shift;
    k.len = min(max(a.lens[b], 0), limit);
    k.begin = a.first ? max(a.first[b], 0) : 0;
    if (a.window) k.begin = max(k.begin, k.len - a.window);
    k.begin = min(k.begin, k.len);
    k.base = k.begin & ~31;
    k.spans = max(1, (k.len - k.base + SPAN - 1) / SPAN);         // a sequence without keys takes one, empty
    return k;
}

template <int TYPE, int CACHE, int DPAD, bool FULL>
struct Attend {
    static constexpr bool F16 = CACHE == QG_F16, E4M3 = CACHE == QG_E4M3;
    static constexpr int Q_PARTS = TYPE == QG_F32 ? 3 : TYPE == QG_F16 && !F16 ? 2 : 1;
    static constexpr int P_PARTS = TYPE == QG_F32 && !F16 ? 3 : 2;
    static constexpr float LIFT = F16 ? 7.0f : 0.0f;               // p is 2^LIFT times what it is to the maximum, so 2^15 at most in f16
    static constexpr float REST = 2048.0f;                         // what p's second part in f16 is larger by
    static constexpr int CHUNKS = DPAD / 32;                       // products of 32 dims in a score
    static constexpr int SIZE = E4M3 ? 1 : 2;
    static constexpr int K_LOADS = DPAD * SIZE / 64;               // of 16 bytes, for each key of a lane
    static constexpr int PIECE = DPAD == 64 ? 4 : 8;               // neighbouring dims a lane loads of a value
    static constexpr int PIECES = DPAD / 16 / PIECE;               // 128 dims apart
    static constexpr int V_WORDS = DPAD / 16 * SIZE / 4;           // registers of a value in a lane
    static constexpr int DIMS = DPAD / 16;                         // products of 16 dims in an output
    static constexpr int LDS_DIMS = DPAD < 128 ? DPAD : 128;       // the wavefronts' sums are added 128 dims at a time
    static constexpr int LDS_ROW = LDS_DIMS + 4;

    // whole lines are read past the caches' replacement order (16-bit cells: 273 us with ordinary loads, so 252); parts of lines, which
    // several instructions ask for, are not (8-bit values and padded heads lose 10 % by it)
    static constexpr bool ONCE_K = FULL, ONCE_V = FULL && !E4M3;

    static constexpr uint32_t EXPONENT = F16 ? 0x7c00u : 0x7f80u, ONE = F16 ? 0x3c00u : 0x3f80u;

    u32x4 kr[2][K_LOADS];
    uint32_t vr[8][V_WORDS];
    float ks[8], vs[8];
    // q's operands wait in LDS, where the four wavefronts share them (in registers: up to 96 more)
    static constexpr int Q_VECTORS = Q_PARTS * CHUNKS * 64;
    floatx4 o[DIMS];
    float m, l, factor;                                            // m: running maximum less LIFT; factor: of a score, for exp2

    // First dim of load c of a key's elements by the lanes of quad j (of 8 elements, or 16 bytes of e4m3).
    __device__ static int k_dim(int c, int j) { return E4M3 ? 64 * c + 16 * j : 32 * c + 8 * j; }

    // Elements of operand c of q's head that are this lane's.
    __device__ static void load_q(const AttentionArgs &a, int64_t b, int head, bool real, int c, int j, float x[8])
    {
        const int D = FULL ? DPAD : a.kv.head_dim;
        const char *row = (const char *)a.q + (b * a.q_stride + (int64_t)head * D) * (TYPE == QG_F32 ? 4 : 2);
        const int d = E4M3 ? k_dim(c / 2, j) + 8 * (c % 2) : k_dim(c, j);
        const bool some = real && (FULL || d < D);
        if constexpr (TYPE == QG_F32) {
            floatx4 v[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
            if (some) {
                v[0] = *(const floatx4 *)(row + 4 * d);
                v[1] = *(const floatx4 *)(row + 4 * d + 16);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = v[e / 4][e % 4];
        } else {
            u32x4 v = {0, 0, 0, 0};
            if (some) v = *(const u32x4 *)(row + 2 * d);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t bits = e % 2 ? v[e / 2] >> 16 : v[e / 2] & 0xffffu;
                x[e] = TYPE == QG_BF16 ? bf16_to_float(bits) : f16_to_float(bits);
            }
        }
    }

    // Of q's CHUNKS operands a wavefront makes every fourth and puts its parts into LDS.
    __device__ void share_q(const AttentionArgs &a, int64_t b, int head, bool real, u32x4 *shared_q, int wave, int lane)
    {
        auto load = [&](int c, float x[8]) { load_q(a, b, head, real, c, lane >> 4, x); };
        factor = a.scale * 1.4426950408889634f;
        int up = 0;
        if constexpr (F16) {
            // the largest element to [2^14, 2^15), so that what f16 cannot hold is below 2^-38 of it
            float most = 0.0f, x[8];
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                load(c, x);
#pragma unroll
                for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x[e]));
            }
            most = across_quads_max(most);
            up = most > 0.0f && most < INFINITY ? 14 - ilogbf(most) : 0;
            factor = ldexpf(factor, -up);
        }
        for (int c = wave; c < CHUNKS; c += WAVES) {
            float x[8];
            load(c, x);
            if constexpr (F16) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = ldexpf(x[e], up);
            }
#pragma unroll
            for (int p = 0; p < Q_PARTS; ++p) {
                u32x4 part;
#pragma unroll
                for (int e = 0; e < 4; ++e) part[e] = take_part<F16>(x[2 * e], x[2 * e + 1]);
                shared_q[(p * CHUNKS + c) * 64 + lane] = part;
            }
        }
    }

    // ... and the elements' signs, as 1, -1, 0 or, where they are no finite numbers, NaN.
    __device__ static void share_signs(const AttentionArgs &a, int64_t b, int head, bool real, u32x4 *shared_signs, int wave, int lane)
    {
        for (int c = wave; c < CHUNKS; c += WAVES) {
            float x[8];
            load_q(a, b, head, real, c, lane >> 4, x);
            uint32_t bits[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) bits[e] = x[e] == 0.0f ? 0u : !(fabsf(x[e]) < INFINITY) ? EXPONENT | EXPONENT >> 1 : ONE | (x[e] < 0.0f ? 0x8000u : 0u);
            shared_signs[c * 64 + lane] = u32x4{bits[0] | bits[1] << 16, bits[2] | bits[3] << 16, bits[4] | bits[5] << 16, bits[6] | bits[7] << 16};
        }
    }

    __device__ void load_k(const AttentionArgs &a, const char *cell, int j)      // cell: of the lane's first key
    {
        const int D = FULL ? DPAD : a.kv.head_dim;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < K_LOADS; ++c) {
                const int d = k_dim(c, j);
                const char *p = cell + (4 * t * D + d) * SIZE;
                if constexpr (FULL) {
                    kr[t][c] = load_cells<ONCE_K, u32x4>(p);
                } else if constexpr (E4M3) {
                    const uint2 none = {0, 0};
                    const uint2 x = d < D ? load_cells<false, uint2>(p) : none, y = d + 8 < D ? load_cells<false, uint2>(p + 8) : none;
                    kr[t][c] = u32x4{x.x, x.y, y.x, y.y};
                } else {
                    kr[t][c] = d < D ? load_cells<false, u32x4>(p) : u32x4{0, 0, 0, 0};
                }
            }
    }

    __device__ void load_v(const AttentionArgs &a, const char *cell, int i)      // cell: of the lane's first key
    {
        const int D = FULL ? DPAD : a.kv.head_dim;
        typedef typename QgRaw<PIECE * SIZE>::t raw;
        constexpr int W = PIECE * SIZE / 4;
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int h = 0; h < PIECES; ++h) {
                const int d = 128 * h + PIECE * i;
                raw x = raw{};
                if (FULL || d < D) x = load_cells<ONCE_V, raw>(cell + (e * D + d) * SIZE);
                __builtin_memcpy(&vr[e][h * W], &x, sizeof x);
            }
    }

    __device__ void load_scales(float *to, const float *from)
    {
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
            const floatx4 x = *(const floatx4 *)(from + e);
#pragma unroll
            for (int k = 0; k < 4; ++k) to[e + k] = x[k];
        }
    }

    // Two bf16 of a pair of 8-bit values: the lower or upper half of a word.
    __device__ static uint32_t widen(uint32_t w, bool upper)
    {
        const bf16x2 v = upper ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, false);
        return __builtin_bit_cast(uint32_t, v);
    }

    __device__ void scores(floatx4 s[2], const u32x4 *shared_q, int lane)
    {
        asm volatile("" : "+v"(lane));                              // read anew for every tile, not kept in registers
        s[0] = s[1] = floatx4{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            Operand part[Q_PARTS];
#pragma unroll
            for (int p = 0; p < Q_PARTS; ++p) {
                const u32x4 v = shared_q[(p * CHUNKS + c) * 64 + lane];
#pragma unroll
                for (int r = 0; r < 4; ++r) part[p].r[r] = v[r];
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                Operand k;
                if constexpr (E4M3) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) k.r[r] = widen(kr[t][c / 2][2 * (c % 2) + r / 2], r % 2);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r) k.r[r] = kr[t][c][r];
                }
#pragma unroll
                for (int p = Q_PARTS - 1; p >= 0; --p) s[t] = mma<F16>(k, part[p], s[t]);
            }
        }
    }

    // The halves of a word that are no finite numbers; the others are 0.
    __device__ static uint32_t not_finite(uint32_t w)
    {
        return ((w & EXPONENT) == EXPONENT ? w & 0xffffu : 0u) | ((w & EXPONENT << 16) == EXPONENT << 16 ? w & 0xffff0000u : 0u);
    }

    // Scores that are NaN are anew what the infinite elements of a key make of q's signs, if it has any.
    __device__ void correct_scores(floatx4 s[2], const u32x4 *shared_signs, int lane)
    {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            floatx4 x = {0, 0, 0, 0};
            for (int c = 0; c < CHUNKS; ++c) {
                Operand k, sign;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    k.r[r] = not_finite(kr[t][c][r]);
                    sign.r[r] = shared_signs[c * 64 + lane][r];
                }
                x = mma<F16>(k, sign, x);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) s[t][e] = s[t][e] != s[t][e] && x[e] != 0.0f ? x[e] : s[t][e];
        }
    }

    // Takes the values that are no finite numbers out of the registers and adds them up, each by 1 (0 where the score is -infinity, NaN where it is).
    __device__ void add_infinities(const floatx4 s[2], int key, int begin, int len)
    {
        Operand ones;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            ones.r[r] = 0;
#pragma unroll
            for (int e = 2 * r; e < 2 * r + 2; ++e) {
                const float x = s[e / 4][e % 4] * factor;
                const bool seen = key + e >= begin && key + e < len;
                const uint32_t one = !seen || x == -INFINITY ? 0u : x != x ? EXPONENT | EXPONENT >> 1 : ONE;
                ones.r[r] |= one << 16 * (e & 1);
#pragma unroll
                for (int w = 0; w < V_WORDS; ++w) vr[e][w] = seen ? vr[e][w] : 0u;
            }
        }
#pragma unroll
        for (int n = 0; n < DIMS; n += 2) {
            Operand lower, upper;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint32_t x = not_finite(vr[2 * r][n / 2]), y = not_finite(vr[2 * r + 1][n / 2]);
                lower.r[r] = __builtin_amdgcn_perm(y, x, 0x05040100u);
                upper.r[r] = __builtin_amdgcn_perm(y, x, 0x07060302u);
                vr[2 * r][n / 2] ^= x;
                vr[2 * r + 1][n / 2] ^= y;
            }
            o[n] = mma<F16>(lower, ones, o[n]);
            o[n + 1] = mma<F16>(upper, ones, o[n + 1]);
        }
    }

    // The running maximum, and s as p.  The keys are key ... key + 7; those outside [begin, len) count for nothing.
    template <bool PARTIAL>
    __device__ void soften(floatx4 s[2], float p[8], int key, int begin, int len)
    {
        float most = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            p[e] = s[e / 4][e % 4] * factor;
            if constexpr (E4M3) p[e] *= ks[e];
            if constexpr (PARTIAL) p[e] = key + e >= begin && key + e < len ? p[e] : -INFINITY;
            most = fmaxf(most, p[e]);
        }
        if (__any(most > m + (SLACK + LIFT))) {
            most = fmaxf(m, across_quads_max(most) - LIFT);
            const float keep = most == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - most), keep_o = fmaxf(keep, 0x1p-149f);
            l *= keep;
#pragma unroll
            for (int n = 0; n < DIMS; ++n) o[n] *= keep_o;
            m = most;
        }
        const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            p[e] = __builtin_amdgcn_exp2f(p[e] - base);
            l += p[e];
            if constexpr (E4M3) p[e] *= PARTIAL && !(key + e >= begin && key + e < len) ? 0.0f : vs[e];
        }
    }

    template <bool PARTIAL>
    __device__ void add_values(float p[8], int key, int begin, int len)
    {
        Operand parts[P_PARTS];
#pragma unroll
        for (int k = 0; k < P_PARTS; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                parts[k].r[e] = take_part<F16>(p[2 * e], p[2 * e + 1]);
                if constexpr (F16) {
                    p[2 * e] *= REST;
                    p[2 * e + 1] *= REST;
                }
            }
        if constexpr (PARTIAL) {                                    // 0 times what lies there could be NaN
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int w = 0; w < V_WORDS; ++w) vr[e][w] = key + e >= begin && key + e < len ? vr[e][w] : 0u;
        }
        // (product n: dims 128 (n / PIECE) + PIECE i + n % PIECE)
#pragma unroll
        for (int n = 0; n < DIMS; n += 2) {
            Operand lower, upper;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if constexpr (E4M3) {
                    // two dims of both keys in one word, side by side
                    const uint32_t both = __builtin_amdgcn_perm(vr[2 * r + 1][n / 4], vr[2 * r][n / 4], n % 4 ? 0x07030602u : 0x05010400u);
                    lower.r[r] = widen(both, false);
                    upper.r[r] = widen(both, true);
                } else {
                    const uint32_t x = vr[2 * r][n / 2], y = vr[2 * r + 1][n / 2];
                    lower.r[r] = __builtin_amdgcn_perm(y, x, 0x05040100u);
                    upper.r[r] = __builtin_amdgcn_perm(y, x, 0x07060302u);
                }
            }
            if constexpr (F16) {
                auto add = [&](const Operand &v, floatx4 &to) {
                    const floatx4 rest = mma<F16>(v, parts[1], floatx4{0, 0, 0, 0});
                    to = mma<F16>(v, parts[0], to);
#pragma unroll
                    for (int r = 0; r < 4; ++r) to[r] = __builtin_fmaf(rest[r], 1.0f / REST, to[r]);
                };
                add(lower, o[n]);
                add(upper, o[n + 1]);
            } else {
#pragma unroll
                for (int k = P_PARTS - 1; k >= 0; --k) {
                    o[n] = mma<F16>(lower, parts[k], o[n]);
                    o[n + 1] = mma<F16>(upper, parts[k], o[n + 1]);
                }
            }
        }
    }
};

// Sum of the values of the lanes up to this one.
__device__ inline int sum_up_to_lane(int v)
{
#define QG_UP(CTRL, ROWS) v += __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
    QG_UP(0x111, 0xf) QG_UP(0x112, 0xf) QG_UP(0x114, 0xf) QG_UP(0x118, 0xf)          // row_shr 1, 2, 4, 8
    QG_UP(0x142, 0xa) QG_UP(0x143, 0xc)                                            // row_bcast 15, 31
#undef QG_UP
    return v;
}

// n / d rounded up, for n below 2^16 and d below 2^8.
__device__ inline uint32_t divided(uint32_t n, uint32_t d) { return d == 1 ? n : __umulhi(n + d - 1, 0xffffffffu / d + 1); }

constexpr int FEW = 24;                    // spans for each worker up to which pieces are looked at

// n / d, in 32 bits where they do (a division in 64 bits is a hundred instructions and more, all of them one after the other).
__device__ inline int64_t quotient(int64_t n, int64_t d)
{
    return ((uint64_t)n | (uint64_t)d) >> 32 ? n / d : (int64_t)((uint32_t)n / (uint32_t)d);
}

// The list of units in as many runs as there are workers, the first `larger` of them a unit longer than the others.
struct Runs {
    int64_t size;
    int larger;
    __device__ Runs(int64_t total, int workers)
    {
        size = total == workers ? 1 : quotient(total, workers);
        larger = (int)(total - size * workers);
    }
    __device__ int64_t begin(int worker) const { return size * worker + min(worker, larger); }
    __device__ int of(int64_t unit) const
    {
        if (size == 1 && larger == 0) return (int)unit;
        const int64_t cut = (size + 1) * larger;
        return unit < cut ? (int)quotient(unit, size + 1) : larger + (int)quotient(unit - cut, size);
    }
};

template <int TYPE, int CACHE, int DPAD, bool FULL>
__global__ __launch_bounds__(64 * WAVES, groups_per_unit(DPAD)) void attend(AttentionArgs a)
{
    typedef Attend<TYPE, CACHE, DPAD, FULL> A;
    // the wavefronts' sums [wavefront][head][LDS_ROW]; of a head's parts, the maxima [part][head]
    constexpr int SHARED_FLOATS = WAVES * 16 * A::LDS_ROW;
    __shared__ float shared[SHARED_FLOATS];
    __shared__ u32x4 shared_q[A::Q_VECTORS];
    __shared__ float wave_m[16][16], wave_l[16][16];
    __shared__ int is_last, found_b, wave_sums[3][WAVES];
    __shared__ int64_t found_at, not_finite_at;                     // not_finite_at: the segment whose sums are not all finite
    __shared__ float head_m[16], head_l[16];
    const rsrc_t parts = buffer_of(a.parts, a.parts_bytes);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int D = FULL ? DPAD : a.kv.head_dim;
    const int heads = a.kv.kv_heads * a.blocks;                     // blocks of heads of a sequence
    const int worker = blockIdx.x;

    // The work is a list of units: sequence by sequence, block of heads by block of heads.  The lengths are gone over 256 sequences at a
    // time, a lane each; unless the batch is larger, once.
    int mine = 0, up_to_mine = 0, chunk = 0;                        // units of sequence tid of the chunk, of it and those before it, of the chunk
    auto scan = [&](int n, int *of_waves) {
        mine = n;
        up_to_mine = sum_up_to_lane(n);
        if (lane == 63) of_waves[wave] = up_to_mine;
        __syncthreads();
        chunk = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) up_to_mine += of_waves[w];
            chunk += of_waves[w];
        }
    };
    auto spans_of = [&](int b) { return b < a.batch ? keys_of(a, b).spans : 0; };
    scan(spans_of(tid), wave_sums[0]);
    int64_t total = chunk;
    for (int b0 = 256; b0 < a.batch; b0 += 256) {
        __syncthreads();
        scan(spans_of(b0 + tid), wave_sums[0]);
        total += chunk;
    }
    total *= heads;

    // Two ways to cut it.  In equal runs of spans (piece = 0): a worker's run may end one head's keys and begin another's, and every such
    // beginning (first page ids, first keys, adding up) costs as much as some spans.  Or a unit is a piece of at most `piece` spans of one
    // head's keys and every worker takes one: the longest take a little more, but each begins once.  Pieces it is where the workers suffice for those of
    // one span more than the longest run, or of three more in 8 bits, whose spans are half as long.  (One sequence of 14000, 8 key heads, bf16: runs 30.3 us,
    // pieces 26.6; 16 in 8 bits: 45.1 and 39.5; but with pieces of 25 spans for runs of 21, 16 of 30000 in bf16, 115.7 and 132.6, of 21 for 17 with 32 key heads
    // 91.7 and 111.2.  Where neither fits, the question costs half a microsecond.)
    int piece = 0;
    const int64_t least = total <= gridDim.x ? 1 : quotient(total + gridDim.x - 1, gridDim.x);
    if (a.batch <= 256 && least <= FEW) {
        // the shortest that will do; the units of two lengths are added up in one word
        const uint32_t exact = (uint32_t)least;
        const int spans = mine;
        int shift = 0;
        for (int c = 0; c < (A::E4M3 ? 2 : 1) && !piece; ++c) {
            const uint32_t shorter = exact + 2 * c, longer = shorter + 1;
            scan((int)(divided(spans, shorter) | divided(spans, longer) << 16), wave_sums[1 + c]);
            const int low = chunk & 0xffff, high = chunk >> 16;
            piece = low * heads <= (int)gridDim.x ? shorter : high * heads <= (int)gridDim.x ? longer : 0;
            shift = piece == (int)shorter ? 0 : 16;
        }
        if (piece) {
            mine = mine >> shift & 0xffff;
            up_to_mine = up_to_mine >> shift & 0xffff;
            chunk = chunk >> shift & 0xffff;
            total = (int64_t)chunk * heads;
        } else {
            __syncthreads();
            scan(spans, wave_sums[0]);
        }
    }
    auto units_of = [&](int spans) { return piece ? (int)divided(spans, piece) : spans; };
    const int workers = total < gridDim.x ? (int)total : (int)gridDim.x;        // each has a unit at least
    if (worker >= workers) return;                                  // the whole workgroup
    const Runs runs(total, workers);
    const int64_t begin_at = runs.begin(worker), end_at = runs.begin(worker + 1);

    // the sequence that this worker's units begin in, and where that sequence's begin in the list
    int64_t before = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 256) {
        if (a.batch > 256) {                                        // (else the only chunk is at hand)
            __syncthreads();
            scan(spans_of(b0 + tid), wave_sums[0]);
        }
        if (begin_at < (before + up_to_mine) * heads && begin_at >= (before + up_to_mine - mine) * heads) {
            found_b = b0 + tid;
            found_at = (before + up_to_mine - mine) * heads;
        }
        before += chunk;
    }
    __syncthreads();
    int b = found_b;
    int64_t sequence_at = found_at;
    b = __builtin_amdgcn_readfirstlane(b);
    Keys keys = keys_of(a, b);

    A t;
    if (tid == 0) not_finite_at = -1;                               // (the first segment's barrier is before its first use)
    for (int64_t at = begin_at; at < end_at;) {
        int tid = (int)threadIdx.x;
        asm volatile("" : "+v"(tid));                               // (so that nothing made of it waits in registers through the loop over the keys)
        const int lane = tid & 63, i = lane & 15, j = lane >> 4;
        int units = units_of(keys.spans);
        while (at - sequence_at >= (int64_t)units * heads) {
            sequence_at += (int64_t)units * heads;
            keys = keys_of(a, ++b);
            units = units_of(keys.spans);
        }
        const int hb = (int)quotient(at - sequence_at, units);           // key head and block of heads
        const int64_t segment_at = sequence_at + (int64_t)hb * units;
        const int unit = (int)(at - segment_at), past = (int)(end_at - segment_at < units ? end_at - segment_at : units);
        const int from = piece ? (int)((uint32_t)(keys.spans * unit) / (uint32_t)units) : unit;
        const int to = piece ? (int)((uint32_t)(keys.spans * past) / (uint32_t)units) : past;
        const int kv_head = hb / a.blocks, head0 = kv_head * a.group + (hb - kv_head * a.blocks) * 16;
        const int rows = min(16, a.group - (hb - kv_head * a.blocks) * 16);

        // tiles of 32 keys: first, first + WAVES, ...
        const int first = from * WAVES + wave, end_key = min(keys.len, keys.base + to * SPAN);
        const int tiles = keys.base + 32 * first < end_key ? (end_key - keys.base - 32 * first + SPAN - 1) / SPAN : 0;
        const int32_t *table = a.kv.tables + b * a.kv.table_stride;
        const int per_page_shift = a.kv.page_shift - 4, mask = a.kv.page - 1;
        const int64_t page_cells = (int64_t)a.kv.kv_heads << a.kv.page_shift, head_cells = (int64_t)kv_head << a.kv.page_shift;
        int32_t ids = 0;                                            // lane l: page of tile (l / 2) of the next 32, its 16 keys l % 2
        auto pages_from = [&](int n) {
            const int unit = (keys.base >> 4) + 2 * (first + WAVES * (n + (lane >> 1))) + (lane & 1);
            const int column = min(unit >> per_page_shift, a.kv.max_pages - 1);
            ids = (int32_t)min((uint32_t)table[column], (uint32_t)(a.kv.pages - 1));
        };
        // cell of key `local` of tile n, whose half of the tile is `half`
        auto cell_of = [&](int n, int half, int local) {
            const int64_t page = (uint32_t)__shfl(ids, 2 * (n & 31) + half);
            const int key0 = keys.base + 32 * (first + WAVES * n);
            return page * page_cells + head_cells + (key0 & mask) + (local & mask);
        };
        auto fetch_k = [&](int n) {
            t.load_k(a, (const char *)a.kv.k + cell_of(n, i >> 3, 8 * (i >> 2) + (i & 3)) * (D * A::SIZE), j);
            // (loads arrive in the order of their requests: scales are asked for before the values, which are used after them)
            if constexpr (A::E4M3) {
                const int64_t cell = cell_of(n, j >> 1, 8 * j);
                t.load_scales(t.ks, a.kv.k_scale + cell);
                t.load_scales(t.vs, a.kv.v_scale + cell);
            }
        };
        auto fetch_v = [&](int n) { t.load_v(a, (const char *)a.kv.v + cell_of(n, j >> 1, 8 * j) * (D * A::SIZE), i); };
        if (tiles) pages_from(0);
        t.share_q(a, b, head0 + i, i < rows, shared_q, wave, lane);
        if (tiles) {
            fetch_k(0);
            fetch_v(0);
        }
        __syncthreads();
        t.m = -INFINITY;
        t.l = 0.0f;
#pragma unroll
        for (int n = 0; n < A::DIMS; ++n) t.o[n] = floatx4{0, 0, 0, 0};
        for (int n = 0; n < tiles; ++n) {
            floatx4 s[2];
            float p[8];
            const int tile_key = keys.base + 32 * (first + WAVES * n), key = tile_key + 8 * j;
            const bool whole = tile_key >= keys.begin && tile_key + 32 <= keys.len;
            t.scores(s, shared_q, lane);
            if (whole) t.template soften<false>(s, p, key, keys.begin, keys.len);
            else t.template soften<true>(s, p, key, keys.begin, keys.len);
            if (n + 1 < tiles) {
                if (((n + 1) & 31) == 0) pages_from(n + 1);
                fetch_k(n + 1);
            }
            if (whole) t.template add_values<false>(p, key, keys.begin, keys.len);
            else t.template add_values<true>(p, key, keys.begin, keys.len);
            if (n + 1 < tiles) fetch_v(n + 1);
        }

        // the four wavefronts' parts: sums at one maximum
        auto share_sums = [&] {
            t.l += __shfl_xor(t.l, 16);
            t.l += __shfl_xor(t.l, 32);
            if (j == 0) {
                wave_m[wave][i] = t.m;
                wave_l[wave][i] = t.l;
            }
        };
        share_sums();
        if constexpr (!A::E4M3) {
            float rest = 0.0f * t.l;                                // 0 unless something is NaN, or infinite (a comparison each takes 1 % longer)
#pragma unroll
            for (int n = 0; n < A::DIMS; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) rest = __builtin_fmaf(t.o[n][r], 0.0f, rest);
            if (__any(rest != rest && i < rows)) not_finite_at = segment_at;       // (any lane's write is as good as another's)
        }
        __syncthreads();
        if constexpr (!A::E4M3) {
            if (not_finite_at == segment_at) {                        // (of the whole workgroup)
                u32x4 *signs = (u32x4 *)shared;
                t.share_signs(a, b, head0 + i, i < rows, signs, wave, lane);
                t.m = -INFINITY;
                t.l = 0.0f;
#pragma unroll
                for (int n = 0; n < A::DIMS; ++n) t.o[n] = floatx4{0, 0, 0, 0};
                __syncthreads();
                for (int n = 0; n < tiles; ++n) {
                    floatx4 s[2];
                    float p[8];
                    const int key = keys.base + 32 * (first + WAVES * n) + 8 * j;
                    if ((n & 31) == 0) pages_from(n);
                    fetch_k(n);
                    t.scores(s, shared_q, lane);
                    t.correct_scores(s, signs, lane);
                    t.template soften<true>(s, p, key, keys.begin, keys.len);
                    asm volatile("" ::: "memory");                  // (keys and values in registers one after the other: this is no place to hurry)
                    fetch_v(n);
                    t.add_infinities(s, key, keys.begin, keys.len);
                    t.template add_values<true>(p, key, keys.begin, keys.len);
                }
                share_sums();
                __syncthreads();
            }
        }
        float most = -INFINITY;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) most = fmaxf(most, wave_m[w][i]);
        const float keep = value_weight(t.m, most);
        const bool whole = from == 0 && to == keys.spans;
        // a worker's first part of a head's keys goes into its slot 0 unless it begins them
        const uint32_t part = 4u * (2 * worker + (from == 0)) * a.part_floats;
        for (int half = 0; half < DPAD / A::LDS_DIMS; ++half) {
            if (half) __syncthreads();
            if (i < rows) {
                // lane 16 j + i: products' rows 4 j + r are dims PIECE (4 j + r) + n of the half
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int n = 0; n < A::PIECE; n += 4) {
                        const int d = A::PIECE * (4 * j + r) + n;
                        floatx4 v;
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[k] = (DPAD > 128 && half ? t.o[A::DIMS / 2 * (DPAD > 128) + n + k][r] : t.o[n + k][r]) * keep;
                        *(floatx4 *)&shared[(wave * 16 + i) * A::LDS_ROW + d] = v;
                    }
            }
            __syncthreads();
            const int quads = min(D - half * A::LDS_DIMS, A::LDS_DIMS) / 4;
            for (int x = tid; x < rows * quads; x += 64 * WAVES) {
                const int row = x / quads, d = 4 * (x - row * quads);
                floatx4 v = *(const floatx4 *)&shared[row * A::LDS_ROW + d];
                float sum_l = 0.0f, top = -INFINITY;
#pragma unroll
                for (int w = 1; w < WAVES; ++w) v += *(const floatx4 *)&shared[(w * 16 + row) * A::LDS_ROW + d];
                if (whole) {
#pragma unroll
                    for (int w = 0; w < WAVES; ++w) top = fmaxf(top, wave_m[w][row]);
#pragma unroll
                    for (int w = 0; w < WAVES; ++w) sum_l += wave_l[w][row] * weight_of(wave_m[w][row], top);
                    const int64_t at_out = ((int64_t)b * a.heads + head0 + row) * D + half * A::LDS_DIMS + d;
#pragma unroll
                    for (int k = 0; k < 4; ++k) store_float<TYPE>(a.out, at_out + k, sum_l == 0.0f ? 0.0f : v[k] / sum_l);
                } else {
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), parts, part + 4 * (row * D + half * A::LDS_DIMS + d), 0, SC1);
                }
            }
        }
        if (tid < rows) {
            float top = -INFINITY, sum_l = 0.0f;
            for (int w = 0; w < WAVES; ++w) top = fmaxf(top, wave_m[w][tid]);
            for (int w = 0; w < WAVES; ++w) sum_l += wave_l[w][tid] * weight_of(wave_m[w][tid], top);
            if (whole) {
                if (a.lse) a.lse[(int64_t)b * a.heads + head0 + tid] = sum_l == 0.0f ? -INFINITY : top * 0.6931471805599453f + logf(sum_l);
            } else {
                __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(top), __float_as_uint(sum_l)}, parts, part + 4 * (rows * D + 2 * tid), 0, SC1);
            }
        }
        if (!whole) {
            // Every worker writes its part past the caches of the dies (agent scope), waits until it is written, and counts itself
            // in; the one that finds all others there adds the parts, in their order.  Nobody waits for anybody.  The counter is
            // that of the worker that begins the head's keys: a worker begins at most one that it does not end.
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            const int w0 = runs.of(segment_at), w1 = runs.of(segment_at + units - 1);
            const int n = w1 - w0 + 1;
            if (tid == 0) {
                const uint32_t was = __hip_atomic_fetch_add(a.arrived + w0, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                is_last = was + 1 == (uint32_t)(n - 1);             // (it starts at 0xffffffff)
                if (is_last) __hip_atomic_store(a.arrived + w0, 0xffffffffu, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            if (is_last) {
                auto part_of = [&](int k) { return 4u * (2 * (w0 + k) + (k == 0)) * a.part_floats; };
                // outputs, four dims a lane; where that leaves lanes over, several share the parts of one
                const int quads = rows * D / 4;
                int shares = 1;
                while (2 * shares * quads <= 64 * WAVES) shares *= 2;
                const int share = shares > 1 ? tid / quads : 0;
                constexpr int AT_ONCE = 8;
                u32x4 y[AT_ONCE];
                auto request = [&](int k0, int x) {
#pragma unroll
                    for (int c = 0; c < AT_ONCE; ++c)
                        if (k0 + c * shares < n) y[c] = __builtin_amdgcn_raw_buffer_load_b128(parts, part_of(k0 + c * shares) + 16 * x, 0, SC1);
                };
                if (share < shares) request(share, shares > 1 ? tid % quads : min(tid, quads - 1));       // on its way while the maxima are looked at
                // maxima and sums of p: 16 lanes for each head, each over every 16th part, then over each other
                {
                    const int row = tid & 15, share = tid >> 4;
                    float top = -INFINITY, sum_l = 0.0f;
                    if (row < rows)
                        for (int k = share; k < n; k += 16) {
                            const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(parts, part_of(k) + 4 * (rows * D + 2 * row), 0, SC1);
                            const float m = __uint_as_float(x[0]), next = fmaxf(top, m);
                            if (k * rows + row < SHARED_FLOATS) shared[k * rows + row] = m;
                            sum_l = sum_l * weight_of(top, next) + __uint_as_float(x[1]) * weight_of(m, next);
                            top = next;
                        }
                    wave_m[share][row] = top;
                    wave_l[share][row] = sum_l;
                }
                __syncthreads();
                if (tid < 16) {
                    float top = -INFINITY, sum_l = 0.0f;
                    for (int w = 0; w < 16; ++w) top = fmaxf(top, wave_m[w][tid]);
                    for (int w = 0; w < 16; ++w) sum_l += wave_l[w][tid] * weight_of(wave_m[w][tid], top);
                    head_m[tid] = top;
                    head_l[tid] = sum_l;
                    if (a.lse && tid < rows) a.lse[(int64_t)b * a.heads + head0 + tid] = sum_l == 0.0f ? -INFINITY : top * 0.6931471805599453f + logf(sum_l);
                }
                __syncthreads();
                for (int x0 = 0; x0 < quads; x0 += 64 * WAVES) {
                    const int x = shares > 1 ? tid % quads : x0 + tid;
                    const bool mine = shares > 1 ? share < shares : x < quads;
                    const int row = mine ? x / (D / 4) : 0;
                    floatx4 v = {0, 0, 0, 0};
                    if (mine) {
                        const float top = head_m[row];
                        for (int k0 = share; k0 < n; k0 += AT_ONCE * shares) {
                            if (x0 || k0 != share) request(k0, x);
#pragma unroll
                            for (int c = 0; c < AT_ONCE; ++c)
                                if (k0 + c * shares < n) {
                                    const int at_m = (k0 + c * shares) * rows + row;
                                    const float m = at_m < SHARED_FLOATS ? shared[at_m] : __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(
                                                                                              parts, part_of(k0 + c * shares) + 4 * (rows * D + 2 * row), 0, SC1));
                                    v += value_weight(m, top) * __builtin_bit_cast(floatx4, y[c]);
                                }
                        }
                    }
                    if (shares > 1) {
                        __syncthreads();                            // the maxima have been read
                        if (mine) *(floatx4 *)&shared[4 * tid] = v;
                        __syncthreads();
                        if (share == 0)
                            for (int k = 1; k < shares; ++k) v += *(const floatx4 *)&shared[4 * (tid + k * quads)];
                    }
                    if (mine && share == 0) {
                        const float sum_l = head_l[row];
                        const int64_t at_out = ((int64_t)b * a.heads + head0) * D + 4 * x;
#pragma unroll
                        for (int k = 0; k < 4; ++k) store_float<TYPE>(a.out, at_out + k, sum_l == 0.0f ? 0.0f : v[k] / sum_l);
                    }
                }
            }
        }
        __syncthreads();
        at = segment_at + past;
    }
}

int workers_for(int head_dim)
{
    const int n = qg_compute_units() * groups_per_unit(head_dim);
    return n < MAX_WORKERS ? n : MAX_WORKERS;
}

// Floats of a part: rows x head_dim sums, rows x (maximum, sum of p).
int part_floats(int heads, int kv_heads, int head_dim)
{
    const int group = heads / kv_heads, rows = group < 16 ? group : 16;
    return (rows * (head_dim + 2) + 3) / 4 * 4;
}

template <int TYPE, int CACHE, int DPAD>
int launch_dims(const AttentionArgs &a, hipStream_t st)
{
    const dim3 grid((unsigned)workers_for(a.kv.head_dim));
    if (a.kv.head_dim == DPAD) hipLaunchKernelGGL((attend<TYPE, CACHE, DPAD, true>), grid, dim3(64 * WAVES), 0, st, a);
    else hipLaunchKernelGGL((attend<TYPE, CACHE, DPAD, false>), grid, dim3(64 * WAVES), 0, st, a);
    return qg_launch_status();
}

template <int TYPE, int CACHE>
int launch_cache(const AttentionArgs &a, hipStream_t st)
{
    if (a.kv.head_dim <= 64) return launch_dims<TYPE, CACHE, 64>(a, st);
    if (a.kv.head_dim <= 128) return launch_dims<TYPE, CACHE, 128>(a, st);
    return launch_dims<TYPE, CACHE, 256>(a, st);
}

template <int TYPE>
int launch_attention(const AttentionArgs &a, hipStream_t st)
{
    return a.kv.type == QG_BF16 ? launch_cache<TYPE, QG_BF16>(a, st) : a.kv.type == QG_F16 ? launch_cache<TYPE, QG_F16>(a, st)
                                                                                          : launch_cache<TYPE, QG_E4M3>(a, st);
}

}  // namespace

extern "C" size_t qg_paged_attention_workspace_bytes(int batch, int heads, int kv_heads, int head_dim)
{
    if (batch < 0 || heads <= 0 || kv_heads <= 0 || heads > QG_MAX_HEADS || heads % kv_heads || head_dim < 8 || head_dim > 256 || head_dim % 8) return 0;
    // (as much for any number of key heads, so that a buffer for the most heads serves them all)
    return qg_round_up(COUNTER_BYTES + (size_t)2 * workers_for(head_dim) * part_floats(heads, 1, head_dim) * 4, 256);
}

extern "C" int qg_paged_attention(const qg_attention_desc *desc, void *stream)
{
    if (!desc) return QG_ERR_NULL;
    const qg_attention_desc &d = *desc;
    QgKv kv;
    const int rc = qg_check_cache(d.cache, &kv);
    if (rc != QG_OK) return rc;
    if (!qg_float_type(d.type)) return QG_ERR_UNSUPPORTED;
    const int D = kv.head_dim;
    if (d.batch < 0 || d.batch > 65535 || d.batch > kv.rows || d.heads <= 0 || d.heads > QG_MAX_HEADS || d.heads % kv.kv_heads || d.window < 0) return QG_ERR_SHAPE;
    if (d.batch == 0) return QG_OK;
    if (d.batch > 1 && d.q_stride < (int64_t)d.heads * D) return QG_ERR_SHAPE;
    if (!d.lens || !d.q || !d.out) return QG_ERR_NULL;
    if (!qg_aligned16(d.q) || !qg_aligned16(d.out) || (d.batch > 1 && d.q_stride % 8) || !qg_aligned_to(d.lens, 4) || !qg_aligned_to(d.first, 4) ||
        !qg_aligned_to(d.lse, 4) || !qg_aligned16(d.workspace)) return QG_ERR_ALIGN;
    if (!d.workspace || d.workspace_bytes < qg_paged_attention_workspace_bytes(d.batch, d.heads, kv.kv_heads, D)) return QG_ERR_WORKSPACE;
    const int group = d.heads / kv.kv_heads;
    const AttentionArgs a = {kv, d.lens, d.first, d.q, d.out, d.lse, d.q_stride, d.batch, d.heads, d.window, group, (group + 15) / 16, d.scale, (uint32_t *)d.workspace, (float *)((char *)d.workspace + COUNTER_BYTES),
                             part_floats(d.heads, kv.kv_heads, D), (uint32_t)(2 * workers_for(D) * part_floats(d.heads, kv.kv_heads, D) * 4)};
    hipStream_t st = (hipStream_t)stream;
    return d.type == QG_F32 ? launch_attention<QG_F32>(a, st) : d.type == QG_BF16 ? launch_attention<QG_BF16>(a, st) : launch_attention<QG_F16>(a, st);
}

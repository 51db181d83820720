// qg_paged_attention: attention of one new token of each sequence over a paged cache.
//
// out = sum_i p_i v_i / sum_i p_i over a sequence's keys, p_i = exp(scale q.k_i), in one pass with a running maximum.  Keys and
// values are read once and nothing else is of their size, so memory bounds it; the matrix instruction does both products
// with the (up to 16) heads that share a key head as one side of the 16 x 16 x 32 tile, and is busy for less than a
// fifth of the time memory takes even with one head in 16.
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
// taken out first); p as two or, for fp32 outputs on the bf16 instruction, three.  8-bit keys and values are exact in
// bf16; their scales are applied to the scores and to the p_i.
#include "qg_kv.h"

namespace {

constexpr int WAVES = 4;                   // wavefronts of a workgroup
constexpr int SPAN = 32 * WAVES;           // keys they take together
constexpr int MAX_WORKERS = 512;           // workgroups of a launch at most (sizes the counters in the workspace and the maxima in LDS)
constexpr int COUNTER_BYTES = 4 * MAX_WORKERS;
constexpr float SLACK = 8.0f;

struct AttentionArgs {
    QgKv kv;
    const int32_t *lens, *first;
    const void *q;
    void *out;
    float *lse;
    int64_t q_stride;
    int batch, heads, window, group;       // group: heads of a key head
    int blocks, rows;                      // blocks of at most 16 heads that make up a group, and the heads of one
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
    static constexpr int CHUNKS = DPAD / 32;                       // products of 32 dims in a score
    static constexpr int SIZE = E4M3 ? 1 : 2;
    static constexpr int K_LOADS = DPAD * SIZE / 64;               // of 16 bytes, for each key of a lane
    static constexpr int PIECE = DPAD == 64 ? 4 : 8;               // neighbouring dims a lane loads of a value
    static constexpr int PIECES = DPAD / 16 / PIECE;               // 128 dims apart
    static constexpr int V_WORDS = DPAD / 16 * SIZE / 4;           // registers of a value in a lane
    static constexpr int DIMS = DPAD / 16;                         // products of 16 dims in an output
    static constexpr int LDS_DIMS = DPAD < 128 ? DPAD : 128;       // the wavefronts' sums are added 128 dims at a time
    static constexpr int LDS_ROW = LDS_DIMS + 4;

    u32x4 kr[2][K_LOADS];
    uint32_t vr[8][V_WORDS];
    float ks[8], vs[8];
    Operand q[Q_PARTS][CHUNKS];
    floatx4 o[DIMS];
    float m, l, factor;                                            // factor: of a score, for exp2

    // First dim of load c of a key's elements by the lanes of quad j (of 8 elements, or 16 bytes of e4m3).
    __device__ static int k_dim(int c, int j) { return E4M3 ? 64 * c + 16 * j : 32 * c + 8 * j; }

    float x[CHUNKS][8];                                            // q on its way into the operands

    // (most sequences' first loads: issued before what depends on the page ids, used after it)
    __device__ void load_q(const AttentionArgs &a, int64_t b, int head, bool real, int j)
    {
        const int D = FULL ? DPAD : a.kv.head_dim;
        const char *row = (const char *)a.q + (b * a.q_stride + (int64_t)head * D) * (TYPE == QG_F32 ? 4 : 2);
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int d = E4M3 ? k_dim(c / 2, j) + 8 * (c % 2) : k_dim(c, j);
            const bool some = real && (FULL || d < D);
            if constexpr (TYPE == QG_F32) {
                floatx4 v[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
                if (some) {
                    v[0] = *(const floatx4 *)(row + 4 * d);
                    v[1] = *(const floatx4 *)(row + 4 * d + 16);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) x[c][e] = v[e / 4][e % 4];
            } else {
                u32x4 v = {0, 0, 0, 0};
                if (some) v = *(const u32x4 *)(row + 2 * d);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t bits = e % 2 ? v[e / 2] >> 16 : v[e / 2] & 0xffffu;
                    x[c][e] = TYPE == QG_BF16 ? bf16_to_float(bits) : f16_to_float(bits);
                }
            }
        }
    }

    __device__ void split_q(const AttentionArgs &a)
    {
        factor = a.scale * 1.4426950408889634f;
        if constexpr (F16) {
            // the largest element to [2^14, 2^15), so that what f16 cannot hold is below 2^-38 of it
            float most = 0.0f;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x[c][e]));
            most = across_quads_max(most);
            const int up = most > 0.0f && most < INFINITY ? 14 - ilogbf(most) : 0;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[c][e] = ldexpf(x[c][e], up);
            factor = ldexpf(factor, -up);
        }
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int p = 0; p < Q_PARTS; ++p)
#pragma unroll
                for (int e = 0; e < 4; ++e) q[p][c].r[e] = take_part<F16>(x[c][2 * e], x[c][2 * e + 1]);
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
                    kr[t][c] = *(const u32x4 *)p;
                } else if constexpr (E4M3) {
                    const uint2 none = {0, 0};
                    const uint2 x = d < D ? *(const uint2 *)p : none, y = d + 8 < D ? *(const uint2 *)(p + 8) : none;
                    kr[t][c] = u32x4{x.x, x.y, y.x, y.y};
                } else {
                    kr[t][c] = d < D ? *(const u32x4 *)p : u32x4{0, 0, 0, 0};
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
                if (FULL || d < D) x = *(const raw *)(cell + (e * D + d) * SIZE);
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

    __device__ void scores(floatx4 s[2])
    {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = floatx4{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                Operand k;
                if constexpr (E4M3) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) k.r[r] = widen(kr[t][c / 2][2 * (c % 2) + r / 2], r % 2);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r) k.r[r] = kr[t][c][r];
                }
#pragma unroll
                for (int p = Q_PARTS - 1; p >= 0; --p) s[t] = mma<F16>(k, q[p][c], s[t]);
            }
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
        if (__any(most > m + SLACK)) {
            most = fmaxf(m, across_quads_max(most));
            const float keep = most == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - most);
            l *= keep;
#pragma unroll
            for (int n = 0; n < DIMS; ++n) o[n] *= keep;
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
            for (int e = 0; e < 4; ++e) parts[k].r[e] = take_part<F16>(p[2 * e], p[2 * e + 1]);
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
                uint32_t x, y;
                if constexpr (E4M3) {
                    x = widen(vr[2 * r][n / 4], n % 4 != 0);
                    y = widen(vr[2 * r + 1][n / 4], n % 4 != 0);
                } else {
                    x = vr[2 * r][n / 2];
                    y = vr[2 * r + 1][n / 2];
                }
                lower.r[r] = __builtin_amdgcn_perm(y, x, 0x05040100u);
                upper.r[r] = __builtin_amdgcn_perm(y, x, 0x07060302u);
            }
#pragma unroll
            for (int k = P_PARTS - 1; k >= 0; --k) {
                o[n] = mma<F16>(lower, parts[k], o[n]);
                o[n + 1] = mma<F16>(upper, parts[k], o[n + 1]);
            }
        }
    }
};

// Range of the flattened list of (sequence, key head, block of heads, span) that a worker takes.
__device__ inline int64_t worker_begin(int64_t total, int worker, int workers) { return total * worker / workers; }
__device__ inline int worker_of(int64_t total, int64_t at, int workers)
{
    return (int)(((at + 1) * workers - 1) / total);                 // the last worker that begins at or before it
}

template <int TYPE, int CACHE, int DPAD, bool FULL>
__global__ __launch_bounds__(64 * WAVES, DPAD == 256 ? 1 : 2) void attend(AttentionArgs a)
{
    typedef Attend<TYPE, CACHE, DPAD, FULL> A;
    // the wavefronts' sums [wavefront][head][LDS_ROW]; of a head's parts, the maxima [part][head]
    constexpr int SHARED_FLOATS = WAVES * 16 * A::LDS_ROW > 16 * MAX_WORKERS ? WAVES * 16 * A::LDS_ROW : 16 * MAX_WORKERS;
    __shared__ float shared[SHARED_FLOATS];
    __shared__ float wave_m[16][16], wave_l[16][16];
    __shared__ int64_t found_before;
    __shared__ int found_b, scan[WAVES], is_last;
    __shared__ float head_m[16], head_l[16];
    const rsrc_t parts = buffer_of(a.parts, a.parts_bytes);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i = lane & 15, j = lane >> 4;
    const int D = FULL ? DPAD : a.kv.head_dim;
    const int heads = a.kv.kv_heads * a.blocks;                     // blocks of heads of a sequence
    const int worker = blockIdx.x;

    // spans of all sequences, and the sequence that this worker's part of them begins in (the batch 256 at a time)
    int64_t total = 0;
    int mine = 0, up_to_mine = 0;                                   // of the chunk at hand: spans of sequence tid, and with those before it
    auto scan_chunk = [&](int b0) {
        mine = up_to_mine = b0 + tid < a.batch ? keys_of(a, b0 + tid).spans : 0;
        for (int off = 1; off < 64; off <<= 1) {
            const int x = __shfl_up(up_to_mine, off);
            if (lane >= off) up_to_mine += x;
        }
        if (lane == 63) scan[wave] = up_to_mine;
        __syncthreads();
        int all = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) up_to_mine += scan[w];
            all += scan[w];
        }
        return all;
    };
    for (int b0 = 0; b0 < a.batch; b0 += 64 * WAVES) {
        if (b0) __syncthreads();                                    // scan is free again
        total += scan_chunk(b0);
    }
    total *= heads;
    const int workers = total < gridDim.x ? (int)total : (int)gridDim.x;        // each has a span at least
    if (worker >= workers) return;                                  // the whole workgroup
    const int64_t begin_at = worker_begin(total, worker, workers), end_at = worker_begin(total, worker + 1, workers);
    int64_t before = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 64 * WAVES) {
        int all = 0;
        if (a.batch > 64 * WAVES) {                                 // (else the only chunk is at hand)
            __syncthreads();
            all = scan_chunk(b0);
        }
        if (begin_at < (before + up_to_mine) * heads && begin_at >= (before + up_to_mine - mine) * heads) {
            found_b = b0 + tid;
            found_before = (before + up_to_mine - mine) * heads;
        }
        before += all;
    }
    __syncthreads();
    int b = found_b;
    int64_t sequence_at = found_before;                             // where sequence b's spans begin in the list
    Keys keys = keys_of(a, b);

    A t;
    for (int64_t at = begin_at; at < end_at;) {
        while (at - sequence_at >= (int64_t)keys.spans * heads) {
            sequence_at += (int64_t)keys.spans * heads;
            keys = keys_of(a, ++b);
        }
        const int hb = (int)((at - sequence_at) / keys.spans);      // key head and block of heads
        const int64_t segment_at = sequence_at + (int64_t)hb * keys.spans;
        const int from = (int)(at - segment_at);
        const int to = (int)(end_at - segment_at < keys.spans ? end_at - segment_at : keys.spans);
        const int kv_head = hb / a.blocks, head0 = kv_head * a.group + (hb - kv_head * a.blocks) * 16;
        const int rows = min(16, a.group - (hb - kv_head * a.blocks) * 16);

        t.m = -INFINITY;
        t.l = 0.0f;
#pragma unroll
        for (int n = 0; n < A::DIMS; ++n) t.o[n] = floatx4{0, 0, 0, 0};

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
            if constexpr (A::E4M3) t.load_scales(t.ks, a.kv.k_scale + cell_of(n, j >> 1, 8 * j));
        };
        auto fetch_v = [&](int n) {
            const int64_t cell = cell_of(n, j >> 1, 8 * j);
            t.load_v(a, (const char *)a.kv.v + cell * (D * A::SIZE), i);
            if constexpr (A::E4M3) t.load_scales(t.vs, a.kv.v_scale + cell);
        };
        if (tiles) {
            pages_from(0);
            t.load_q(a, b, head0 + i, i < rows, j);
            fetch_k(0);
            fetch_v(0);
            t.split_q(a);
        }
        for (int n = 0; n < tiles; ++n) {
            floatx4 s[2];
            float p[8];
            const int tile_key = keys.base + 32 * (first + WAVES * n), key = tile_key + 8 * j;
            const bool whole = tile_key >= keys.begin && tile_key + 32 <= keys.len;
            t.scores(s);
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
        t.l += __shfl_xor(t.l, 16);
        t.l += __shfl_xor(t.l, 32);
        if (j == 0) {
            wave_m[wave][i] = t.m;
            wave_l[wave][i] = t.l;
        }
        __syncthreads();
        float most = -INFINITY;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) most = fmaxf(most, wave_m[w][i]);
        const float keep = t.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(t.m - most);
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
                    for (int w = 0; w < WAVES; ++w) sum_l += wave_m[w][row] == -INFINITY ? 0.0f : wave_l[w][row] * __builtin_amdgcn_exp2f(wave_m[w][row] - top);
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
            for (int w = 0; w < WAVES; ++w) sum_l += wave_m[w][tid] == -INFINITY ? 0.0f : wave_l[w][tid] * __builtin_amdgcn_exp2f(wave_m[w][tid] - top);
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
            const int w0 = worker_of(total, segment_at, workers), w1 = worker_of(total, segment_at + keys.spans - 1, workers);
            const int n = w1 - w0 + 1;
            if (tid == 0) {
                const uint32_t was = __hip_atomic_fetch_add(a.arrived + w0, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                is_last = was + 1 == (uint32_t)(n - 1);             // (it starts at 0xffffffff)
                if (is_last) __hip_atomic_store(a.arrived + w0, 0xffffffffu, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            if (is_last) {
                auto part_of = [&](int k) { return 4u * (2 * (w0 + k) + (k == 0)) * a.part_floats; };
                // maxima and sums of p: 16 lanes for each head, each over every 16th part, then over each other
                {
                    const int row = tid & 15, share = tid >> 4;
                    float top = -INFINITY, sum_l = 0.0f;
                    if (row < rows)
                        for (int k = share; k < n; k += 16) {
                            const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(parts, part_of(k) + 4 * (rows * D + 2 * row), 0, SC1);
                            const float m = __uint_as_float(x[0]), next = fmaxf(top, m);
                            shared[k * 16 + row] = m;
                            if (m != -INFINITY) sum_l = (top == -INFINITY ? 0.0f : sum_l * __builtin_amdgcn_exp2f(top - next)) +
                                                        __uint_as_float(x[1]) * __builtin_amdgcn_exp2f(m - next);
                            top = next;
                        }
                    wave_m[share][row] = top;
                    wave_l[share][row] = sum_l;
                }
                __syncthreads();
                if (tid < 16) {
                    float top = -INFINITY, sum_l = 0.0f;
                    for (int w = 0; w < 16; ++w) top = fmaxf(top, wave_m[w][tid]);
                    for (int w = 0; w < 16; ++w) sum_l += wave_m[w][tid] == -INFINITY ? 0.0f : wave_l[w][tid] * __builtin_amdgcn_exp2f(wave_m[w][tid] - top);
                    head_m[tid] = top;
                    head_l[tid] = sum_l;
                    if (a.lse && tid < rows) a.lse[(int64_t)b * a.heads + head0 + tid] = sum_l == 0.0f ? -INFINITY : top * 0.6931471805599453f + logf(sum_l);
                }
                __syncthreads();
                // outputs, four dims a lane; where that leaves lanes over, several share the parts of one
                const int quads = rows * D / 4;
                int shares = 1;
                while (2 * shares * quads <= 64 * WAVES) shares *= 2;
                for (int x0 = 0; x0 < quads; x0 += 64 * WAVES) {
                    const int x = shares > 1 ? tid % quads : x0 + tid, share = shares > 1 ? tid / quads : 0;
                    const bool mine = shares > 1 ? share < shares : x < quads;
                    const int row = mine ? x / (D / 4) : 0;
                    floatx4 v = {0, 0, 0, 0};
                    if (mine) {
                        const float top = head_m[row];
                        constexpr int AT_ONCE = 8;
                        for (int k0 = share; k0 < n; k0 += AT_ONCE * shares) {
                            u32x4 y[AT_ONCE];
#pragma unroll
                            for (int c = 0; c < AT_ONCE; ++c)
                                if (k0 + c * shares < n) y[c] = __builtin_amdgcn_raw_buffer_load_b128(parts, part_of(k0 + c * shares) + 16 * x, 0, SC1);
#pragma unroll
                            for (int c = 0; c < AT_ONCE; ++c)
                                if (k0 + c * shares < n) {
                                    const float m = shared[(k0 + c * shares) * 16 + row];
                                    v += (m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - top)) * __builtin_bit_cast(floatx4, y[c]);
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
        at = segment_at + to;
    }
}

int workers_for(int head_dim)
{
    const int n = qg_compute_units() * (head_dim > 128 ? 1 : 2);
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
    const AttentionArgs a = {kv, d.lens, d.first, d.q, d.out, d.lse, d.q_stride, d.batch, d.heads, d.window, group, (group + 15) / 16,
                             group < 16 ? group : 16, d.scale, (uint32_t *)d.workspace, (float *)((char *)d.workspace + COUNTER_BYTES),
                             part_floats(d.heads, kv.kv_heads, D), (uint32_t)(2 * workers_for(D) * part_floats(d.heads, kv.kv_heads, D) * 4)};
    hipStream_t st = (hipStream_t)stream;
    return d.type == QG_F32 ? launch_attention<QG_F32>(a, st) : d.type == QG_BF16 ? launch_attention<QG_BF16>(a, st) : launch_attention<QG_F16>(a, st);
}

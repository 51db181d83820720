// qg_kv_append: rotates q and k of new tokens and stores k and v in the pages of a cache.
#include "qg_kv.h"

namespace {

struct AppendArgs {
    QgKv kv;
    const int32_t *rows, *positions;
    const void *q, *k, *v;
    void *q_out;
    const float *cos_sin;
    int64_t q_stride, k_stride, v_stride, cos_sin_rows;
    int heads, rope_dim, interleaved;
};

// A team of 1, 2, 4 ... 32 lanes, eight neighbouring elements each, takes heads of q, k and v of one token in turn and keeps the position's
// cosines and sines in registers.  Memory bounds it: every element crosses once, the pair's other half a second time from the caches.
// (7551 tokens of 64 + 16 heads of 128, bf16 into 8 bits: 54 us, 5.5 TB/s; a wavefront a head, an element at a time: 244.)
// WHOLE: the rotated elements and their halves are whole eights (and the angles aligned); otherwise angles and partners are loaded one by one.
template <int TYPE, int CACHE, bool WHOLE>
__global__ __launch_bounds__(256) void append_eights(AppendArgs a, int team_shift)
{
    const int64_t token = blockIdx.x;
    const int team = 1 << team_shift, teams = 256 >> team_shift, i = 8 * (threadIdx.x & (team - 1));
    const int D = a.kv.head_dim, items = a.heads + 2 * a.kv.kv_heads, half = a.rope_dim / 2;
    const int64_t position = a.positions[token];
    int64_t page = qg_page_of(a.kv, a.rows[token], position);
    if (a.rope_dim && position >= a.cos_sin_rows) page = -1;
    const bool real = i < D, turned = i < a.rope_dim, second = i >= half;
    float cosine[8], sine[8];
    if (turned && page >= 0) {
        const float *angle = a.cos_sin + position * a.rope_dim;
        if constexpr (!WHOLE) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int k = i + e, pair = a.interleaved ? k >> 1 : k < half ? k : k - half;
                const bool late = a.interleaved ? k & 1 : k >= half;
                cosine[e] = k < a.rope_dim ? angle[pair] : 1.0f;
                sine[e] = k < a.rope_dim ? (late ? angle[half + pair] : -angle[half + pair]) : 0.0f;
            }
        } else if (a.interleaved) {                                 // four pairs
            const float4 c = *(const float4 *)(angle + i / 2), s = *(const float4 *)(angle + half + i / 2);
            cosine[0] = c.x; cosine[1] = c.y; cosine[2] = c.z; cosine[3] = c.w;
            sine[0] = s.x; sine[1] = s.y; sine[2] = s.z; sine[3] = s.w;
        } else {
            load_eight<QG_F32>(angle, second ? i - half : i, cosine);
            load_eight<QG_F32>(angle, second ? i : i + half, sine);
            if (!second) {
#pragma unroll
                for (int e = 0; e < 8; ++e) sine[e] = -sine[e];
            }
        }
    }
    const int64_t cell0 = page * a.kv.kv_heads * a.kv.page + (position & (a.kv.page - 1));
    // (all lanes of a wavefront go round as often: the largest of a team is found across lanes)
    for (int item0 = blockIdx.y * teams; item0 < items; item0 += gridDim.y * teams) {
        const int item = item0 + (threadIdx.x >> team_shift);
        const bool mine = real && item < items, is_q = item < a.heads, is_v = item >= a.heads + a.kv.kv_heads;
        const int head = is_q ? item : is_v ? item - a.heads - a.kv.kv_heads : item - a.heads;
        const void *src = is_q ? a.q : is_v ? a.v : a.k;
        const int64_t at = token * (is_q ? a.q_stride : is_v ? a.v_stride : a.k_stride) + (int64_t)head * D;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.0f;
        if (mine && page >= 0) {
            load_eight<TYPE>(src, at + i, x);
            if (turned && !is_v) {
                if constexpr (!WHOLE) {
                    float other[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        other[e] = x[e ^ 1];
                        if (!a.interleaved && i + e < a.rope_dim) other[e] = load_as_float<TYPE>(src, at + (i + e >= half ? i + e - half : i + e + half));
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = i + e < a.rope_dim ? x[e] * cosine[e] + other[e] * sine[e] : x[e];
                } else if (a.interleaved) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float u = x[2 * e], w = x[2 * e + 1];
                        x[2 * e] = u * cosine[e] - w * sine[e];
                        x[2 * e + 1] = w * cosine[e] + u * sine[e];
                    }
                } else {
                    float other[8];
                    load_eight<TYPE>(src, at + (second ? i - half : i + half), other);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = x[e] * cosine[e] + other[e] * sine[e];
                }
            }
        }
        if (mine && is_q) store_eight<TYPE>(a.q_out, (token * a.heads + head) * D + i, x);
        if (page < 0) continue;                                     // (of the whole workgroup: its token)
        const int64_t cell = cell0 + (int64_t)head * a.kv.page;
        if constexpr (CACHE == QG_E4M3) {
            uint32_t most = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) most = max(most, magnitude_bits(x[e]));
            const float scale = e4m3_scale(most_of(most, team));
            if (mine && !is_q && i == 0) (is_v ? a.kv.v_scale : a.kv.k_scale)[cell] = scale;
            scale_eight(x, scale);
        }
        if (mine && !is_q) store_eight<CACHE>(is_v ? a.kv.v : a.kv.k, cell * D + i, x);
    }
}

template <int TYPE, int CACHE>
int launch_heads(int64_t all_tokens, const AppendArgs &all, hipStream_t st)
{
    const int items = all.heads + 2 * all.kv.kv_heads, D = all.kv.head_dim, size = qg_type_bytes(TYPE);
    int shift = 0;
    while ((8 << shift) < D) ++shift;
    const bool whole = all.rope_dim % (all.interleaved ? 8 : 16) == 0 && qg_aligned16(all.cos_sin);
    for (int64_t token = 0; token < all_tokens; token += QG_MOST_GROUPS) {
        const int64_t tokens = all_tokens - token < QG_MOST_GROUPS ? all_tokens - token : QG_MOST_GROUPS;
        AppendArgs a = all;
        a.rows += token;
        a.positions += token;
        a.k = (const char *)a.k + token * a.k_stride * size;
        a.v = (const char *)a.v + token * a.v_stride * size;
        if (a.heads) {
            a.q = (const char *)a.q + token * a.q_stride * size;
            a.q_out = (char *)a.q_out + token * a.heads * D * size;
        }
        // a workgroup takes all heads of a token (its angles are loaded once), or, where tokens are few, as many as it has teams
        const int teams = 256 >> shift, most = (items + teams - 1) / teams;
        const int64_t want = 4 * (int64_t)qg_compute_units() / tokens;
        const dim3 grid((unsigned)tokens, (unsigned)(want < 1 ? 1 : want < most ? want : most));
        if (whole) hipLaunchKernelGGL((append_eights<TYPE, CACHE, true>), grid, dim3(256), 0, st, a, shift);
        else hipLaunchKernelGGL((append_eights<TYPE, CACHE, false>), grid, dim3(256), 0, st, a, shift);
        const int rc = qg_launch_status();
        if (rc != QG_OK) return rc;
    }
    return QG_OK;
}

template <int TYPE>
int launch_append(int64_t tokens, const AppendArgs &a, hipStream_t st)
{
    return a.kv.type == QG_BF16 ? launch_heads<TYPE, QG_BF16>(tokens, a, st) : a.kv.type == QG_F16 ? launch_heads<TYPE, QG_F16>(tokens, a, st)
                                                                                                  : launch_heads<TYPE, QG_E4M3>(tokens, a, st);
}

}  // namespace

extern "C" int qg_kv_append(const qg_append_desc *desc, void *stream)
{
    if (!desc) return QG_ERR_NULL;
    const qg_append_desc &d = *desc;
    QgKv kv;
    const int rc = qg_check_cache(d.cache, &kv);
    if (rc != QG_OK) return rc;
    if (!qg_float_type(d.type)) return QG_ERR_UNSUPPORTED;
    const int D = kv.head_dim;
    if (d.tokens < 0 || d.tokens > 0x7fffffff || d.heads < 0 || d.heads > QG_MAX_HEADS || d.rope_dim < 0 || d.rope_dim > D || d.rope_dim % 2 ||
        (d.rope_dim && d.cos_sin_rows < 0)) return QG_ERR_SHAPE;
    if (d.tokens == 0) return QG_OK;
    if (d.tokens > 1 && ((d.heads && d.q_stride < (int64_t)d.heads * D) || d.k_stride < (int64_t)kv.kv_heads * D || d.v_stride < (int64_t)kv.kv_heads * D))
        return QG_ERR_SHAPE;
    if (!d.rows || !d.positions || !d.k || !d.v || (d.heads && (!d.q || !d.q_out)) || (d.rope_dim && !d.cos_sin)) return QG_ERR_NULL;
    if (!qg_aligned16(d.k) || !qg_aligned16(d.v) || (d.heads && (!qg_aligned16(d.q) || !qg_aligned16(d.q_out))) || !qg_aligned_to(d.cos_sin, 4) ||
        !qg_aligned_to(d.rows, 4) || !qg_aligned_to(d.positions, 4) ||
        (d.tokens > 1 && (d.k_stride % 8 || d.v_stride % 8 || (d.heads && d.q_stride % 8)))) return QG_ERR_ALIGN;
    if (d.heads && d.q == d.q_out) return QG_ERR_UNSUPPORTED;     // a lane reads what another has written
    const AppendArgs a = {kv, d.rows, d.positions, d.q, d.k, d.v, d.q_out, d.cos_sin, d.q_stride, d.k_stride, d.v_stride, d.cos_sin_rows,
                          d.heads, d.rope_dim, d.interleaved != 0};
    hipStream_t st = (hipStream_t)stream;
    return d.type == QG_F32 ? launch_append<QG_F32>(d.tokens, a, st) : d.type == QG_BF16 ? launch_append<QG_BF16>(d.tokens, a, st)
                                                                                       : launch_append<QG_F16>(d.tokens, a, st);
}

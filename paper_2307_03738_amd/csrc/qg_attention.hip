// qg_paged_attention: attention of one new token of each sequence over a paged cache.
#include "qg_kv.h"

namespace {

struct AttentionArgs {
    QgKv kv;
    const int32_t *lens, *first;
    const void *q;
    void *out;
    float *lse;
    int64_t q_stride;
    int heads, window;
    float scale;
};

// One workgroup per sequence and head; a wavefront takes every fourth key, its lanes hold the elements of a head.
template <int TYPE, int CACHE>
__global__ __launch_bounds__(256) void attend_simple(AttentionArgs a)
{
    __shared__ float part_o[4][256], part_m[4], part_l[4];
    const int head = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t b = blockIdx.y;
    const int D = a.kv.head_dim, kv_head = head / (a.heads / a.kv.kv_heads);
    const int len = min(max(a.lens[b], 0), a.kv.max_pages * a.kv.page);
    int first = a.first ? max(a.first[b], 0) : 0;
    if (a.window) first = max(first, len - a.window);
    float q[4], o[4] = {0, 0, 0, 0}, m = -INFINITY, l = 0.0f;
    for (int c = 0; c < 4; ++c) q[c] = lane + 64 * c < D ? load_as_float<TYPE>(a.q, b * a.q_stride + (int64_t)head * D + lane + 64 * c) : 0.0f;
    for (int i = first + wave; i < len; i += 4) {
        const int64_t page = min((uint32_t)a.kv.tables[b * a.kv.table_stride + (i >> a.kv.page_shift)], (uint32_t)(a.kv.pages - 1));
        const int64_t cell = (page * a.kv.kv_heads + kv_head) * a.kv.page + (i & (a.kv.page - 1));
        float s = 0.0f;
        for (int c = 0; c < 4; ++c)
            if (lane + 64 * c < D) s += q[c] * load_as_float<CACHE>(a.kv.k, cell * D + lane + 64 * c);
        for (int off = 32; off; off >>= 1) s += __shfl_xor(s, off);
        s *= a.scale;
        float vs = 1.0f;
        if constexpr (CACHE == QG_E4M3) {
            s *= a.kv.k_scale[cell];
            vs = a.kv.v_scale[cell];
        }
        const float most = fmaxf(m, s), keep = m == -INFINITY ? 0.0f : expf(m - most), p = most == -INFINITY ? 0.0f : expf(s - most);
        l = l * keep + p;
        for (int c = 0; c < 4; ++c)
            if (lane + 64 * c < D) o[c] = o[c] * keep + p * vs * load_as_float<CACHE>(a.kv.v, cell * D + lane + 64 * c);
        m = most;
    }
    for (int c = 0; c < 4; ++c)
        if (lane + 64 * c < D) part_o[wave][lane + 64 * c] = o[c];
    if (lane == 0) { part_m[wave] = m; part_l[wave] = l; }
    __syncthreads();
    float most = -INFINITY, total = 0.0f;
    for (int w = 0; w < 4; ++w) most = fmaxf(most, part_m[w]);
    for (int w = 0; w < 4; ++w) total += part_l[w] * (part_m[w] == -INFINITY ? 0.0f : expf(part_m[w] - most));
    const int64_t row = b * a.heads + head;
    for (int i = threadIdx.x; i < D; i += 256) {
        float v = 0.0f;
        for (int w = 0; w < 4; ++w) v += part_o[w][i] * (part_m[w] == -INFINITY ? 0.0f : expf(part_m[w] - most));
        store_float<TYPE>(a.out, row * D + i, total == 0.0f ? 0.0f : v / total);
    }
    if (a.lse && threadIdx.x == 0) a.lse[row] = most + logf(total);
}

template <int TYPE>
int launch_attention(int batch, const AttentionArgs &a, hipStream_t st)
{
    const dim3 grid((unsigned)a.heads, (unsigned)batch);
    switch (a.kv.type) {
    case QG_BF16: hipLaunchKernelGGL((attend_simple<TYPE, QG_BF16>), grid, dim3(256), 0, st, a); break;
    case QG_F16: hipLaunchKernelGGL((attend_simple<TYPE, QG_F16>), grid, dim3(256), 0, st, a); break;
    default: hipLaunchKernelGGL((attend_simple<TYPE, QG_E4M3>), grid, dim3(256), 0, st, a); break;
    }
    return qg_launch_status();
}

}  // namespace

extern "C" size_t qg_paged_attention_workspace_bytes(int batch, int heads, int kv_heads, int head_dim)
{
    if (batch < 0 || heads <= 0 || kv_heads <= 0 || heads > QG_MAX_HEADS || heads % kv_heads || head_dim < 8 || head_dim > 256 || head_dim % 8) return 0;
    return 256;
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
    const AttentionArgs a = {kv, d.lens, d.first, d.q, d.out, d.lse, d.q_stride, d.heads, d.window, d.scale};
    hipStream_t st = (hipStream_t)stream;
    return d.type == QG_F32 ? launch_attention<QG_F32>(d.batch, a, st) : d.type == QG_BF16 ? launch_attention<QG_BF16>(d.batch, a, st)
                                                                                         : launch_attention<QG_F16>(d.batch, a, st);
}

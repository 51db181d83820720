// qg_rms_norm: rows' root-mean-square norm with the residual's addition, output in 32, 16 or 8 bits.
#include "qg_types.h"

namespace {

struct NormArgs {
    const void *x, *residual, *weight;
    void *h, *y;
    float *scales;
    int64_t x_stride, residual_stride;
    int K, group;
    float eps;
};

__device__ inline float load_any(int type, const void *p, int64_t i)
{
    return type == QG_F32 ? load_as_float<QG_F32>(p, i) : type == QG_BF16 ? load_as_float<QG_BF16>(p, i) : load_as_float<QG_F16>(p, i);
}

__device__ inline float sum_of_block(float v, float *part)
{
    for (int off = 32; off; off >>= 1) v += __shfl_xor(v, off);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.0f;
    for (unsigned w = 0; w < blockDim.x / 64; ++w) s += part[w];
    return s;
}

// One workgroup per row; x + residual is read again for the output.
template <int TYPE, int YTYPE>
__global__ __launch_bounds__(256) void norm_rows(NormArgs a, int weight_type)
{
    __shared__ float part[4];
    const int64_t row = blockIdx.x;
    const int K = a.K;
    const int64_t xo = row * a.x_stride, ro = row * a.residual_stride, o = row * K;
    float sum = 0.0f;
    for (int k = threadIdx.x; k < K; k += 256) {
        float h = load_as_float<TYPE>(a.x, xo + k);
        if (a.residual) h += load_as_float<TYPE>(a.residual, ro + k);
        sum += h * h;
    }
    const float rs = 1.0f / sqrtf(sum_of_block(sum, part) / (float)K + a.eps);
    const int group = YTYPE == QG_E4M3 ? a.group : K, groups = K / group;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    // each wavefront takes whole groups: first their largest value, then the output
    for (int g = YTYPE == QG_E4M3 ? wave : 0; g < groups; g += YTYPE == QG_E4M3 ? 4 : 1) {
        float scale = 1.0f;
        if constexpr (YTYPE == QG_E4M3) {
            uint32_t most = 0;
            for (int k = lane; k < group; k += 64) {
                float h = load_as_float<TYPE>(a.x, xo + g * group + k);
                if (a.residual) h += load_as_float<TYPE>(a.residual, ro + g * group + k);
                most = max(most, magnitude_bits(h * rs * load_any(weight_type, a.weight, g * group + k)));
            }
            for (int off = 32; off; off >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, off));
            scale = e4m3_scale(most);
            if (lane == 0) a.scales[row * groups + g] = scale;
        }
        for (int k = YTYPE == QG_E4M3 ? lane : (int)threadIdx.x; k < group; k += YTYPE == QG_E4M3 ? 64 : 256) {
            const int at = g * group + k;
            float h = load_as_float<TYPE>(a.x, xo + at);
            if (a.residual) h += load_as_float<TYPE>(a.residual, ro + at);
            if (a.h) store_float<TYPE>(a.h, o + at, h);
            const float y = h * rs * load_any(weight_type, a.weight, at);
            store_float<YTYPE>(a.y, o + at, YTYPE == QG_E4M3 ? limit_e4m3(y / scale) : y);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <int TYPE>
int launch_norm(const qg_norm_desc &d, const NormArgs &a, hipStream_t st)
{
    const dim3 grid((unsigned)d.rows);
    switch (d.y_type) {
    case QG_F32: hipLaunchKernelGGL((norm_rows<TYPE, QG_F32>), grid, dim3(256), 0, st, a, d.weight_type); break;
    case QG_BF16: hipLaunchKernelGGL((norm_rows<TYPE, QG_BF16>), grid, dim3(256), 0, st, a, d.weight_type); break;
    case QG_F16: hipLaunchKernelGGL((norm_rows<TYPE, QG_F16>), grid, dim3(256), 0, st, a, d.weight_type); break;
    default: hipLaunchKernelGGL((norm_rows<TYPE, QG_E4M3>), grid, dim3(256), 0, st, a, d.weight_type); break;
    }
    return qg_launch_status();
}

}  // namespace

extern "C" int qg_rms_norm(const qg_norm_desc *desc, void *stream)
{
    if (!desc) return QG_ERR_NULL;
    const qg_norm_desc &d = *desc;
    if (!qg_float_type(d.type) || !qg_float_type(d.weight_type) || (!qg_float_type(d.y_type) && d.y_type != QG_E4M3)) return QG_ERR_UNSUPPORTED;
    if (d.rows < 0 || d.K <= 0 || d.rows > 0x7fffffff || d.K > (int64_t)1 << 24 || d.group < 0) return QG_ERR_SHAPE;
    if (d.y_type != QG_E4M3 ? d.group != 0 : d.group != 0 && d.K % d.group != 0) return QG_ERR_SHAPE;
    if (d.rows == 0) return QG_OK;
    if (d.rows > 1 && (d.x_stride < d.K || (d.residual && d.residual_stride < d.K))) return QG_ERR_SHAPE;
    if (!d.x || !d.weight || !d.y || (d.y_type == QG_E4M3 && !d.scales) || (d.h && !d.residual)) return QG_ERR_NULL;
    const int size = qg_type_bytes(d.type);
    if (!qg_aligned_to(d.x, size) || !qg_aligned_to(d.residual, size) || !qg_aligned_to(d.h, size) || !qg_aligned_to(d.scales, 4) ||
        !qg_aligned_to(d.weight, qg_type_bytes(d.weight_type)) || !qg_aligned_to(d.y, qg_type_bytes(d.y_type))) return QG_ERR_ALIGN;
    const NormArgs a = {d.x, d.residual, d.weight, d.h, d.y, d.scales, d.x_stride, d.residual_stride, (int)d.K, d.group ? d.group : (int)d.K, d.eps};
    hipStream_t st = (hipStream_t)stream;
    return d.type == QG_F32 ? launch_norm<QG_F32>(d, a, st) : d.type == QG_BF16 ? launch_norm<QG_BF16>(d, a, st) : launch_norm<QG_F16>(d, a, st);
}

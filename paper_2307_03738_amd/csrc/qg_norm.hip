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

// Rows whose length, alignment or groups the kernel below does not take: one workgroup per row, x + residual is read again for the output.
template <int TYPE, int YTYPE>
__global__ __launch_bounds__(256) void norm_rows(NormArgs a, int weight_type)
{
    __shared__ float part[4];
    const int64_t row = blockIdx.x;
    const int K = a.K;
    const int64_t xo = row * a.x_stride, ro = row * a.residual_stride, o = row * K;
    // A lane's squares in runs of 32, the runs in 64 bits: one after the other in 32 bits the 65536 of the longest rows lose 13 bits.
    double sum = 0.0;
    for (int k0 = threadIdx.x; k0 < K; k0 += 32 * 256) {
        const int end = min(K, k0 + 32 * 256);
        float run = 0.0f;
        for (int k = k0; k < end; k += 256) {
            float h = load_as_float<TYPE>(a.x, xo + k);
            if (a.residual) h += load_as_float<TYPE>(a.residual, ro + k);
            run += h * h;
        }
        sum += run;
    }
    const float rs = 1.0f / sqrtf(sum_of_block((float)sum, part) / (float)K + a.eps);
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

// Sum of a wavefront, in its last lane.
__device__ inline float sum_of_wave(float v)
{
#define QG_UP(CTRL, ROWS) v += __uint_as_float(dpp<CTRL, ROWS>(__float_as_uint(v)));
    QG_UP(0x111, 0xf) QG_UP(0x112, 0xf) QG_UP(0x114, 0xf) QG_UP(0x118, 0xf)          // row_shr 1, 2, 4, 8
    QG_UP(0x142, 0xa) QG_UP(0x143, 0xc)                                            // row_bcast 15, 31
#undef QG_UP
    return v;
}

// A row in the registers of `team` lanes (64 ... 1024), eight neighbouring elements at a time, R times; rows, residual, h and y cross memory
// once.  Memory bounds it from some hundred rows on, the one way through loads, two sums and stores below.  A workgroup takes rows
// in turn, keeps the weight and asks for the next row before it adds up this one.  (A workgroup of 256 per row that reads the row again for
// its output: 8.7 us for one row of 4096, 238 for 4099 x 8192 bf16 to e4m3; this 2.6 and 48, 5.0 TB/s, 102 for 8192 x 4096 fp32, 5.3 TB/s.)
template <int TYPE, int YTYPE, int R>
__global__ __launch_bounds__(1024, 4) void norm_rows8(NormArgs a, int weight_type, int64_t rows, int team)
{
    __shared__ float part[2][16];
    __shared__ uint32_t most_part[2][16];
    const int K = a.K, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int member = threadIdx.x & (team - 1), waves = team >> 6, first_wave = wave & ~(waves - 1);
    const int per_block = blockDim.x / team;
    const int64_t step = (int64_t)gridDim.x * per_block;
    int64_t row = (int64_t)blockIdx.x * per_block + threadIdx.x / team;
    int at[R];
    float w[R][8], x[R][8], r[R][8];
#pragma unroll
    for (int c = 0; c < R; ++c) at[c] = 8 * (member + c * team);
    auto load = [&](int64_t row) {
#pragma unroll
        for (int c = 0; c < R; ++c)
            if (at[c] < K && row < rows) {
                load_eight<TYPE>(a.x, row * a.x_stride + at[c], x[c]);
                if (a.residual) load_eight<TYPE>(a.residual, row * a.residual_stride + at[c], r[c]);
            }
    };
#pragma unroll
    for (int c = 0; c < R; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[c][e] = r[c][e] = w[c][e] = 0.0f;
    load(row);
#pragma unroll
    for (int c = 0; c < R; ++c)
        if (at[c] < K) {
            if (weight_type == QG_F32) load_eight<QG_F32>(a.weight, at[c], w[c]);
            else if (weight_type == QG_BF16) load_eight<QG_BF16>(a.weight, at[c], w[c]);
            else load_eight<QG_F16>(a.weight, at[c], w[c]);
        }
    int turn = 0;
    // (every lane of the workgroup goes round as often as the first row's)
    for (int64_t row0 = (int64_t)blockIdx.x * per_block; row0 < rows; row0 += step, row += step, turn ^= 1) {
        float h[R][8], sum = 0.0f;
#pragma unroll
        for (int c = 0; c < R; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                h[c][e] = a.residual ? x[c][e] + r[c][e] : x[c][e];
                sum += h[c][e] * h[c][e];
            }
        load(row + step);
        sum = sum_of_wave(sum);
        if (waves > 1) {
            if (lane == 63) part[turn][wave] = sum;
            __syncthreads();                                        // (two of them in turn: the last row's are still being read)
            sum = 0.0f;
            for (int k = 0; k < waves; ++k) sum += part[turn][first_wave + k];
        } else {
            sum = __shfl(sum, 63);
        }
        const float rs = 1.0f / sqrtf(sum / (float)K + a.eps);
        if (a.h && row < rows) {
#pragma unroll
            for (int c = 0; c < R; ++c)
                if (at[c] < K) store_eight<TYPE>(a.h, row * K + at[c], h[c]);
        }
#pragma unroll
        for (int c = 0; c < R; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) h[c][e] = h[c][e] * rs * w[c][e];
        if constexpr (YTYPE == QG_E4M3) {
            uint32_t most[R], of_row = 0;
#pragma unroll
            for (int c = 0; c < R; ++c) {
                most[c] = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) most[c] = max(most[c], magnitude_bits(h[c][e]));
                of_row = max(of_row, most[c]);
            }
            if (a.group == K) {
                of_row = most_of(of_row, 64);
                if (waves > 1) {
                    if (lane == 0) most_part[turn][wave] = of_row;
                    __syncthreads();
                    for (int k = 0; k < waves; ++k) of_row = max(of_row, most_part[turn][first_wave + k]);
                }
                if (member == 0 && row < rows) a.scales[row] = e4m3_scale(of_row);
            }
#pragma unroll
            for (int c = 0; c < R; ++c) {
                uint32_t top = of_row;
                if (a.group != K)                                   // group / 8 neighbouring lanes share a scale
                    top = most_of(most[c], a.group / 8);
                const float scale = e4m3_scale(top);
                if (a.group != K && at[c] < K && row < rows && at[c] % a.group == 0) a.scales[row * (K / a.group) + at[c] / a.group] = scale;
                scale_eight(h[c], scale);
            }
        }
        if (row < rows) {
#pragma unroll
            for (int c = 0; c < R; ++c)
                if (at[c] < K) store_eight<YTYPE>(a.y, row * K + at[c], h[c]);
        }
    }
}

template <int TYPE, int YTYPE>
int launch_rows(const qg_norm_desc &d, const NormArgs &a, hipStream_t st)
{
    const int K = a.K, group = a.group;
    bool eight = K % 8 == 0 && K <= 2 * 8 * 1024 && qg_aligned16(d.x) && qg_aligned16(d.residual) && qg_aligned16(d.weight) && qg_aligned16(d.h) && qg_aligned16(d.y) &&
                 (d.rows == 1 || (d.x_stride % 8 == 0 && d.residual_stride % 8 == 0));
    if (YTYPE == QG_E4M3 && group != K) eight = eight && group % 8 == 0 && group <= 512 && (group & (group - 1)) == 0;
    if (!eight) {
        const int size = qg_type_bytes(TYPE);
        for (int64_t row = 0; row < d.rows; row += QG_MOST_GROUPS) {
            const int64_t rows = d.rows - row < QG_MOST_GROUPS ? d.rows - row : QG_MOST_GROUPS;
            NormArgs turn = a;
            turn.x = (const char *)a.x + row * a.x_stride * size;
            if (a.residual) turn.residual = (const char *)a.residual + row * a.residual_stride * size;
            if (a.h) turn.h = (char *)a.h + row * K * size;
            turn.y = (char *)a.y + row * K * qg_type_bytes(YTYPE);
            if (a.scales) turn.scales = a.scales + row * (K / group);
            hipLaunchKernelGGL((norm_rows<TYPE, YTYPE>), dim3((unsigned)rows), dim3(256), 0, st, turn, d.weight_type);
            const int rc = qg_launch_status();
            if (rc != QG_OK) return rc;
        }
        return QG_OK;
    }
    // few rows: as many lanes as there are eights; many: two eights a lane (four would spill: a row asked for ahead doubles the registers)
    const int units = qg_compute_units();
    int team = 64, each = d.rows < 2 * units ? 8 : 16;
    while (team < 1024 && team * each < K) team *= 2;
    const int turns = (K / 8 + team - 1) / team, block = team < 256 ? 256 : team;
    const int64_t blocks = (d.rows + block / team - 1) / (block / team), most = (int64_t)units * (2048 / block);
    const dim3 grid((unsigned)(blocks < most ? blocks : most));
    if (turns == 1) hipLaunchKernelGGL((norm_rows8<TYPE, YTYPE, 1>), grid, dim3(block), 0, st, a, d.weight_type, d.rows, team);
    else hipLaunchKernelGGL((norm_rows8<TYPE, YTYPE, 2>), grid, dim3(block), 0, st, a, d.weight_type, d.rows, team);
    return qg_launch_status();
}

template <int TYPE>
int launch_norm(const qg_norm_desc &d, const NormArgs &a, hipStream_t st)
{
    switch (d.y_type) {
    case QG_F32: return launch_rows<TYPE, QG_F32>(d, a, st);
    case QG_BF16: return launch_rows<TYPE, QG_BF16>(d, a, st);
    case QG_F16: return launch_rows<TYPE, QG_F16>(d, a, st);
    default: return launch_rows<TYPE, QG_E4M3>(d, a, st);
    }
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

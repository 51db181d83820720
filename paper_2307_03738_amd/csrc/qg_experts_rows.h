// Rows of X as the experts' products take them, made once a call: f16 in the order in which codes come out of their words, one part or,
// fp32, two, and the power of two that the row was multiplied by.  A last row of zeros stands for rows that there are not.
#pragma once

#include "qg_experts_codes.h"

struct QgPrepareArgs {
    const char *x;
    char *xh;                  // [x_rows + 1][parts][padded] f16
    int32_t *up;               // [x_rows + 1]
    int64_t x_rows, x_stride, padded;
    int K, type;
};

#ifdef QG_EXPERTS_KERNELS
namespace {

// Position of k (0 ... 31) in two operands of 16 k: operand position / 16, lanes of half position / 8 % 2, element position % 8.
template <int BITS>
__device__ inline int k_position_32(int k)
{
    if constexpr (BITS == 2) {
        const int w = k >> 4, r = k & 15;
        return ((r & 7) >> 2) * 16 + w * 8 + 2 * (r & 3) + (r >> 3);
    } else {
        return k_position<BITS>(k);
    }
}

// Eight k of a row from k on, zeros from K on.
__device__ inline void eight_of_row(const char *x, int type, int64_t from, int64_t k, int K, bool real, float *v)
{
    if (real && k < K) {
        if (type == QG_F32) load_eight<QG_F32>(x, from + k, v);
        else if (type == QG_BF16) load_eight<QG_BF16>(x, from + k, v);
        else load_eight<QG_F16>(x, from + k, v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    }
}

// LANES lanes a row, a wavefront or a workgroup; a lane takes 32 k at a time, which it keeps where K ends there (a workgroup: 8192).  Bound by memory where rows are many
// (read once, from cache a second time where K is longer; written once), by one load and a meeting where they are few.
template <int BITS, int LANES>
__global__ __launch_bounds__(256) void prepare_rows(const QgPrepareArgs a)
{
    __shared__ uint32_t mosts[4];
    const int lane = threadIdx.x % LANES;
    const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (256 / LANES) + threadIdx.x / LANES;
    if (row > a.x_rows) return;                       // (a workgroup of one row, or a wavefront, as a whole)
    const int parts = a.type == QG_F32 ? 2 : 1;
    char *to = a.xh + row * parts * a.padded * 2;
    const bool real = row < a.x_rows;
    const int64_t from = row * a.x_stride;
    float v[32];
    auto take = [&](int64_t k, float *to) {
#pragma unroll
        for (int o = 0; o < 32; o += 8) eight_of_row(a.x, a.type, from, k + o, a.K, real, to + o);
    };
    take(lane * 32, v);
    int up = 0;
    if (a.type != QG_F16) {
        uint32_t most = 0;
#pragma unroll
        for (int e = 0; e < 32; ++e) most = max(most, magnitude_bits(v[e]));
        for (int64_t k = (LANES + lane) * 32; k < a.K; k += LANES * 32) {
            float u[32];
            take(k, u);
#pragma unroll
            for (int e = 0; e < 32; ++e) most = max(most, magnitude_bits(u[e]));
        }
        most = most_of(most, 64);
        if constexpr (LANES > 64) {
            if ((threadIdx.x & 63) == 0) mosts[threadIdx.x >> 6] = most;
            __syncthreads();
            most = max(max(mosts[0], mosts[1]), max(mosts[2], mosts[3]));
        }
        up = row_exponent(most);
    }
    if (lane == 0) a.up[row] = up;
    for (int64_t k = lane * 32; k < a.padded; k += LANES * 32) {
        if (k != lane * 32) take(k, v);
        float p[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) p[k_position_32<BITS>(e)] = a.type == QG_F16 ? v[e] : __builtin_amdgcn_ldexpf(v[e], up);
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            if (part < parts) {
#pragma unroll
                for (int o = 0; o < 32; o += 8)
                    *(uint4 *)(to + (part * a.padded + k + o) * 2) =
                        make_uint4(two_halves(p[o], p[o + 1]), two_halves(p[o + 2], p[o + 3]), two_halves(p[o + 4], p[o + 5]), two_halves(p[o + 6], p[o + 7]));
#pragma unroll
                for (int e = 0; e < 32; ++e) p[e] = left_over(p[e]);
            }
        }
    }
}

template <int BITS>
void prepare_launch(const QgPrepareArgs &p, hipStream_t st)
{
    // few rows: a workgroup each, whose loads are under way at once
    const bool wide = p.x_rows < 2048;
    const int64_t blocks = wide ? p.x_rows + 1 : (p.x_rows + 4) / 4;
    const unsigned across = (unsigned)(blocks < QG_MOST_GROUPS ? blocks : QG_MOST_GROUPS);
    const dim3 grid(across, (unsigned)((blocks + across - 1) / across));
    if (wide) prepare_rows<BITS, 256><<<grid, 256, 0, st>>>(p);
    else prepare_rows<BITS, 64><<<grid, 256, 0, st>>>(p);
}

}  // namespace
#endif

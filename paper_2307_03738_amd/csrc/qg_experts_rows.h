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
__device__ inline int k_position(int k)
{
    if constexpr (BITS == 2) {                 // word, and upper or lower four fields of its bytes 0, 2 or 1, 3
        const int w = k >> 4, r = k & 15;
        return ((r & 7) >> 2) * 16 + w * 8 + 2 * (r & 3) + (r >> 3);
    } else if constexpr (BITS == 4) {
        return (k & 24) + 2 * (k & 3) + ((k >> 2) & 1);
    } else {                                   // byte b: code b below, code 4 + b above
        const int c = k & 7;
        return (k & 24) + 4 * (c & 1) + 2 * (c >> 2) + ((c & 3) >> 1);
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

// Values of a row that a lane takes together, as many as decide an operand's eight, from k on, and where they go: 2 bits, two eights 16 positions apart.
template <int BITS> constexpr int row_piece() { return BITS == 2 ? 16 : 8; }

template <int BITS>
__device__ inline void store_piece(const float *v, int type, int up, char *row, int64_t apart, int64_t k)
{
    constexpr int OCT = row_piece<BITS>();
    char *to = row + (BITS == 2 ? (k & ~31) + (k >> 1 & 8) : k) * 2;
    float h[2 * OCT];
#pragma unroll
    for (int e = 0; e < OCT; ++e) h[k_position<BITS>(e)] = type == QG_F16 ? v[e] : __builtin_amdgcn_ldexpf(v[e], up);
#pragma unroll
    for (int part = 0; part < 2; ++part) {
        if (part == 0 || type == QG_F32) {
#pragma unroll
            for (int j = 0; j < OCT / 8; ++j) {
                float *o = h + 16 * j;
                *(uint4 *)(to + part * apart + j * 32) = make_uint4(two_halves(o[0], o[1]), two_halves(o[2], o[3]), two_halves(o[4], o[5]), two_halves(o[6], o[7]));
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = left_over(o[e]);
            }
        }
    }
}

// LANES lanes a row, a wavefront or a workgroup, which keep 32 values each (a workgroup: rows up to 8192 are read once).  Bound by memory where rows are many,
// by one load and a meeting where they are few (4096 rows of 4096 bf16: 16 us, 4.2 TB/s; 61 of 2048: 2 to 4).
template <int BITS, int LANES>
__global__ __launch_bounds__(256) void prepare_rows(const QgPrepareArgs a)
{
    constexpr int OCT = row_piece<BITS>(), KEPT = 32 / OCT;
    __shared__ uint32_t mosts[4];
    const int lane = threadIdx.x % LANES;
    const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (256 / LANES) + threadIdx.x / LANES;
    if (row > a.x_rows) return;                       // (a workgroup of one row, or a wavefront, as a whole)
    const int parts = a.type == QG_F32 ? 2 : 1;
    char *to = a.xh + row * parts * a.padded * 2;
    const bool real = row < a.x_rows;
    const int64_t from = row * a.x_stride;
    auto take = [&](int64_t k, float *v) {
#pragma unroll
        for (int o = 0; o < OCT; o += 8) eight_of_row(a.x, a.type, from, k + o, a.K, real, v + o);
    };
    float v[KEPT][OCT];
#pragma unroll
    for (int i = 0; i < KEPT; ++i) take((i * LANES + lane) * OCT, v[i]);
    int up = 0;
    if (a.type != QG_F16) {
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < KEPT; ++i)
#pragma unroll
            for (int e = 0; e < OCT; ++e) most = max(most, magnitude_bits(v[i][e]));
        for (int64_t k = (KEPT * LANES + lane) * OCT; k < a.K; k += LANES * OCT) {
            float u[OCT];
            take(k, u);
#pragma unroll
            for (int e = 0; e < OCT; ++e) most = max(most, magnitude_bits(u[e]));
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
#pragma unroll
    for (int i = 0; i < KEPT; ++i) {
        const int64_t k = (i * LANES + lane) * OCT;
        if (k < a.padded) store_piece<BITS>(v[i], a.type, up, to, a.padded * 2, k);
    }
    for (int64_t k = (KEPT * LANES + lane) * OCT; k < a.padded; k += LANES * OCT) {
        take(k, v[0]);
        store_piece<BITS>(v[0], a.type, up, to, a.padded * 2, k);
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

// Weights of the experts' products as f16 operands of the matrix instructions: exact integers q - z, the scale applied to fp32 sums.
// A lane holds the code words of its own output (device layout); operands want 16 outputs x 4 lanes, so words change lanes first
// (permlane swaps of whole words, 4 for 4), and are unpacked where they are needed.
//
// f16 1024 + 2^f q is the pattern 0x6400 with a field f bits up in the mantissa, so a field is taken where it stands by one and-or, and
// one packed fused multiply-add by 2^-f with -(1024 2^-f + z) leaves q - z, exact.
#pragma once

#include "qg_experts.h"

namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));

union HalfOperand {
    half8v v;
    half2v h[4];
    uint32_t r[4];
    uint4 q;
};

// 32 k of 64 outputs are 32 / CELL cells: 4 words a lane at 3 (three planes and their spare bits) and 4 bits, 2 at 2 bits.
template <int BITS> constexpr int words_of_32() { return BITS == 2 ? 2 : 4; }
// fields of a 16-bit half that a word, shifted by 8 or not, is read with
template <int BITS> constexpr int zero_constants() { return BITS == 2 ? 4 : 2; }

struct HalfConst {
    uint32_t mask[4], magic;
};
template <int BITS>
__device__ inline HalfConst half_constants()
{
    HalfConst c;
    constexpr uint32_t one = BITS == 4 ? 0x000f000fu : BITS == 3 ? 0x00070007u : 0x00030003u;
#pragma unroll
    for (int f = 0; f < 4; ++f) {
        c.mask[f] = one << (BITS * (f < zero_constants<BITS>() ? f : 0));
        asm("" : "+s"(c.mask[f]));             // what the optimiser cannot see through becomes one and-or
    }
    c.magic = 0x64006400u;
    asm("" : "+v"(c.magic));
    return c;
}

// -(1024 2^-f + z), twice, for the fields f = 0, BITS, ...
template <int BITS>
__device__ inline void zero_operands(uint32_t z, uint32_t *c)
{
    const uint32_t two = z << 16 | z;
#pragma unroll
    for (int i = 0; i < zero_constants<BITS>(); ++i) {
        const uint32_t f = BITS * i;
        c[i] = (two << f) + (0xe400e400u - (f << 10) * 0x00010001u);
    }
}

// One word (for 2 bits its byte 0 and 2, shifted there) to eight q - z.
template <int BITS>
__device__ inline void unpack_halves(uint32_t w, const HalfConst &k, const uint32_t *zc, HalfOperand &op)
{
    const uint32_t up = w >> 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int field = BITS == 2 ? i : i & 1;
        const uint32_t src = BITS == 2 || i < 2 ? w : up;
        const uint32_t raw = and_or(src, k.mask[field], k.magic);
        const _Float16 down = (_Float16)(1.0f / (float)(1 << (BITS * field)));
        const half2v by = {down, down};
        const half2v c = __builtin_bit_cast(half2v, zc[field]);
        op.h[i] = __builtin_elementwise_fma(__builtin_bit_cast(half2v, raw), by, c);
    }
}

// A lane's value of its output to the lanes of a block of 16 outputs: out[b] holds output 16 b + lane % 16.
__device__ inline void spread_16(uint32_t v, uint32_t *out)
{
    const auto h = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    const auto a = __builtin_amdgcn_permlane16_swap(h[0], h[0], false, false);
    const auto b = __builtin_amdgcn_permlane16_swap(h[1], h[1], false, false);
    out[0] = a[0];
    out[1] = a[1];
    out[2] = b[0];
    out[3] = b[1];
}

// Words of 32 k of 64 outputs (lane = output) to operands' words: out[b] holds, for output 16 b + lane % 16, the word of quarter lane / 16.
template <int BITS>
__device__ inline void words_16(const uint32_t *w, uint32_t *out)
{
    if constexpr (BITS == 2) {
        const auto h = __builtin_amdgcn_permlane32_swap(w[0], w[1], false, false);
        const auto a = __builtin_amdgcn_permlane16_swap(h[0], h[0], false, false);
        const auto b = __builtin_amdgcn_permlane16_swap(h[1], h[1], false, false);
        const uint32_t down = (threadIdx.x & 16) >> 1;
        out[0] = a[0] >> down;
        out[1] = a[1] >> down;
        out[2] = b[0] >> down;
        out[3] = b[1] >> down;
    } else {
        const auto p = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
        const auto q = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
        const auto a = __builtin_amdgcn_permlane16_swap(p[0], q[0], false, false);
        const auto b = __builtin_amdgcn_permlane16_swap(p[1], q[1], false, false);
        out[0] = a[0];
        out[1] = a[1];
        out[2] = b[0];
        out[3] = b[1];
    }
}

// Words of 32 k number `i` of a quantum's loads (4 bits: a vector each; 2 bits: half a vector; 3 bits: cell i of three planes).
template <int BITS>
__device__ inline void words_of(const uint4 *v, int i, uint32_t *w)
{
    if constexpr (BITS == 4) {
        w[0] = v[i].x; w[1] = v[i].y; w[2] = v[i].z; w[3] = v[i].w;
    } else if constexpr (BITS == 2) {
        w[0] = word_of(v[i / 2], 2 * (i & 1));
        w[1] = word_of(v[i / 2], 2 * (i & 1) + 1);
    } else {
        const int u = i / 4;
        const uint32_t a = word_of(v[3 * u], i & 3), b = word_of(v[3 * u + 1], i & 3), c = word_of(v[3 * u + 2], i & 3);
        w[0] = a;
        w[1] = b;
        w[2] = c;
        w[3] = ((a >> 6) & 0x03030303u) | ((b >> 4) & 0x0c0c0c0cu) | ((c >> 2) & 0x30303030u);
    }
}

// A row of X enters as f16: f16 as it is; bf16 and fp32 times a power of two that puts the largest |x| of the row into [2^14, 2^15).  f16's smallest step is
// 2^-24, so that a bf16's eight bits are whole down to 2^-31 of that largest, and what is left out of it below that is 2^-39 of the largest at most.
// fp32 goes in two parts, x less the first in the second, which is 2^SECOND_UP times as large as it would be (at most 2^3 before, 2^15 so: it fits), with weights or sums that are as
// much smaller: its 2^-25 then are 2^-51 of the largest, and 2^-23 of x is left out, or 2^-51 of the row's largest if that is more.  (Without the power 2^-39: ordinary values beside one that
// is 2^20 times as large kept 19 bits.)  Rows with NaN or infinity are not scaled.
constexpr int SECOND_UP = 12;
__device__ inline int row_exponent(uint32_t most)          // most: pattern of the largest |x|
{
    return most == 0 || most >= 0x7f800000u ? 0 : 141 - (most < 0x00800000u ? 1 : (int)(most >> 23));
}
__device__ inline uint32_t two_halves(float a, float b)    // both rounded to nearest even
{
    return __builtin_bit_cast(uint16_t, (_Float16)a) | (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)b) << 16;
}
__device__ inline float left_over(float x)                  // of the first part
{
    const float h = (float)(_Float16)x;
    return __builtin_fabsf(h) == __builtin_inff() ? 0.0f : (x - h) * (float)(1 << SECOND_UP);
}
// Weights for the second part: q - z is a whole number below 16, exact so, too.
__device__ inline void second_weights(HalfOperand &o)
{
    const _Float16 down = (_Float16)(1.0f / (float)(1 << SECOND_UP));
#pragma unroll
    for (int i = 0; i < 4; ++i) o.h[i] *= half2v{down, down};
}

}  // namespace

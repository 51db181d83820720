// Element types of the calls between the products (qg_type): loading and storing them as fp32.
#pragma once

#include "qg_common.h"

namespace {

static inline bool qg_float_type(int t) { return t == QG_F32 || t == QG_BF16 || t == QG_F16; }
static inline int qg_type_bytes(int t) { return t == QG_F32 ? 4 : t == QG_E4M3 ? 1 : 2; }
static inline bool qg_aligned_to(const void *p, int bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

constexpr float QG_E4M3_MOST = 448.0f;

// Workgroups of 256 of one launch, whose lanes have to number less than 2^32; what needs more is launched in turns.
constexpr int64_t QG_MOST_GROUPS = 1 << 23;

// Vectors of 4, 8 or 16 bytes, loaded as they lie in memory.
template <int BYTES> struct QgRaw;
template <> struct QgRaw<4> { typedef uint32_t t; };
template <> struct QgRaw<8> { typedef uint2 t; };
template <> struct QgRaw<16> { typedef uint4 t; };

__device__ inline float bf16_to_float(uint32_t b) { return __uint_as_float(b << 16); }
__device__ inline uint32_t float_to_bf16(float v)
{
    return __builtin_bit_cast(uint16_t, (__bf16)v);           // to nearest even, NaN kept
}
__device__ inline float f16_to_float(uint32_t b) { return (float)__builtin_bit_cast(_Float16, (uint16_t)b); }
__device__ inline uint32_t float_to_f16(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }

// |v| <= 448 or NaN; the hardware's conversion of two
__device__ inline uint32_t floats_to_e4m3x2(float a, float b)
{
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xffffu;
}
// NaN stays NaN
__device__ inline float limit_e4m3(float v)
{
    return v > QG_E4M3_MOST ? QG_E4M3_MOST : v < -QG_E4M3_MOST ? -QG_E4M3_MOST : v;
}

template <int TYPE>
__device__ inline float load_as_float(const void *p, int64_t i)
{
    if constexpr (TYPE == QG_F32) return ((const float *)p)[i];
    else if constexpr (TYPE == QG_BF16) return bf16_to_float(((const uint16_t *)p)[i]);
    else return f16_to_float(((const uint16_t *)p)[i]);
}

template <int TYPE>
__device__ inline void store_float(void *p, int64_t i, float v)
{
    if constexpr (TYPE == QG_F32) ((float *)p)[i] = v;
    else if constexpr (TYPE == QG_BF16) ((uint16_t *)p)[i] = (uint16_t)float_to_bf16(v);
    else if constexpr (TYPE == QG_F16) ((uint16_t *)p)[i] = (uint16_t)float_to_f16(v);
    else ((uint8_t *)p)[i] = (uint8_t)floats_to_e4m3x2(v, 0.0f);
}

// Largest |v| of values that share a scale, where NaN and infinity have to be seen: as integers, the patterns of |v| are
// ordered like the numbers, with infinity and NaN above them all.
__device__ inline uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ inline float e4m3_scale(uint32_t most)
{
    if (most >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
    const float scale = __uint_as_float(most) / QG_E4M3_MOST;
    return scale == 0.0f ? 1.0f : scale;                            // (it is for the smallest of numbers, too: up to 224 x 2^-149)
}

// Eight neighbouring elements as floats, and back.
template <int TYPE>
__device__ inline void load_eight(const void *p, int64_t i, float *v)
{
    if constexpr (TYPE == QG_F32) {
        const float4 a = ((const float4 *)((const float *)p + i))[0], b = ((const float4 *)((const float *)p + i))[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
        const uint4 a = *(const uint4 *)((const uint16_t *)p + i);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t bits = e % 2 ? w[e / 2] >> 16 : w[e / 2] & 0xffffu;
            v[e] = TYPE == QG_BF16 ? bf16_to_float(bits) : f16_to_float(bits);
        }
    }
}

template <int TYPE>
__device__ inline void store_eight(void *p, int64_t i, const float *v)
{
    if constexpr (TYPE == QG_F32) {
        ((float4 *)((float *)p + i))[0] = make_float4(v[0], v[1], v[2], v[3]);
        ((float4 *)((float *)p + i))[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else if constexpr (TYPE == QG_E4M3) {
        uint32_t w[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) w[e] = floats_to_e4m3x2(v[4 * e], v[4 * e + 1]) | floats_to_e4m3x2(v[4 * e + 2], v[4 * e + 3]) << 16;
        *(uint2 *)((uint8_t *)p + i) = make_uint2(w[0], w[1]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w[e] = TYPE == QG_BF16 ? float_to_bf16(v[2 * e]) | float_to_bf16(v[2 * e + 1]) << 16 : float_to_f16(v[2 * e]) | float_to_f16(v[2 * e + 1]) << 16;
        *(uint4 *)((uint16_t *)p + i) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

template <int CTRL, int ROWS>
__device__ inline uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false); }

// Largest of `lanes` (1, 2, 4 ... 64) neighbouring lanes, in all of them: exchanges inside a row of 16 lanes on the vector ALU (pairs, quads,
// mirrored halves and rows), rows by lane exchanges.
__device__ inline uint32_t most_of(uint32_t v, int lanes)
{
    if (lanes >= 2) v = max(v, dpp<0xb1, 0xf>(v));
    if (lanes >= 4) v = max(v, dpp<0x4e, 0xf>(v));
    if (lanes >= 8) v = max(v, dpp<0x141, 0xf>(v));
    if (lanes >= 16) v = max(v, dpp<0x140, 0xf>(v));
    if (lanes >= 32) {
        const auto x = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = max(x[0], x[1]);
    }
    if (lanes >= 64) {
        const auto x = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        v = max(x[0], x[1]);
    }
    return v;
}

// Eight values over their scale, rounded as a division rounds them, and within e4m3's range.  Values of 8 or 11 bits over a scale taken of one of
// them lie in the middle of two codes often enough to see (the reciprocal's product alone moved 5 in 10000 codes of bf16 heads), so the
// quotient is corrected: the reciprocal, refined once, is the nearest there is, and what the first quotient is over v, exact in a fused
// multiplication, times it makes the nearest quotient.  Scales below 2^-80, beside which that rest could underflow in a value that matters,
// divide, and NaN goes that way too.
__device__ inline void scale_eight(float *v, float scale)
{
    if (__any(!(scale >= 0x1p-80f))) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = limit_e4m3(v[e] / scale);
    } else {
        float inverse = __builtin_amdgcn_rcpf(scale);
        inverse = __builtin_fmaf(__builtin_fmaf(-scale, inverse, 1.0f), inverse, inverse);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float quotient = v[e] * inverse;
            const float over = __builtin_fmaf(quotient, scale, -v[e]);         // (this way round -0 stays -0)
            v[e] = __builtin_amdgcn_fmed3f(__builtin_fmaf(-over, inverse, quotient), -QG_E4M3_MOST, QG_E4M3_MOST);
        }
    }
}

}  // namespace

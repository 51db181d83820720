// Element types of the calls between the products (qg_type): loading and storing them as fp32.
#pragma once

#include "qg_common.h"

namespace {

static inline bool qg_float_type(int t) { return t == QG_F32 || t == QG_BF16 || t == QG_F16; }
static inline int qg_type_bytes(int t) { return t == QG_F32 ? 4 : t == QG_E4M3 ? 1 : 2; }
static inline bool qg_aligned_to(const void *p, int bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

constexpr float QG_E4M3_MOST = 448.0f;

// Vectors of N elements of 1, 2 or 4 bytes, loaded and stored as they lie in memory.
template <int BYTES> struct QgRaw;
template <> struct QgRaw<1> { typedef uint8_t t; };
template <> struct QgRaw<2> { typedef uint16_t t; };
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
__device__ inline float e4m3_to_float(uint32_t b) { return __builtin_amdgcn_cvt_f32_fp8((int)b, 0); }
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
    else if constexpr (TYPE == QG_F16) return f16_to_float(((const uint16_t *)p)[i]);
    else return e4m3_to_float(((const uint8_t *)p)[i]);
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
    return most == 0 ? 1.0f : __uint_as_float(most) / QG_E4M3_MOST;
}

}  // namespace

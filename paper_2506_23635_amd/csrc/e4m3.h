// e4m3.h -- 8-bit floating-point codes (1 sign, 4 exponent and 3 mantissa bits,
// bias 7, largest value 448) with power-of-two scales.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "moe_common.h"

namespace moe {

constexpr int kExpMin = -100;      // exponents of a scale
constexpr int kExpMax = 119;        // 448 * 2^119 is the largest such that is a bf16

// The least exponent e of kExpMin .. kExpMax with amax <= 448 * 2^e = 1.75 *
// 2^(e + 8), from the bits of a finite amax >= 0: the carry of the addition is
// 1 where the mantissa is past 1.75.  (Past kExpMax values end at 448.)
__device__ inline int scale_exponent(float amax)
{
    const int e = (int)((__float_as_uint(amax) + (0x7FFFFFu - 0x600000u)) >> 23) - 127 - 8;
    return min(max(e, kExpMin), kExpMax);
}

__device__ inline float exp2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

__device__ inline bool finite(float v) { return (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u; }

// four values times 2^-e as e4m3 codes; what is not finite becomes NaN
__device__ inline uint32_t code4(const float* v, float inv)
{
    float w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = finite(v[i]) ? fminf(fmaxf(v[i] * inv, -448.f), 448.f) : NAN;
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(w[0], w[1], 0, false);
    c = __builtin_amdgcn_cvt_pk_fp8_f32(w[2], w[3], c, true);
    return (uint32_t)c;
}

// |v| as bits: ordered like the values, what is not finite from kInfBits on
constexpr uint32_t kInfBits = 0x7F800000u;
__device__ inline uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// code4 of finite values
__device__ inline uint32_t code4_finite(const float* v, float inv)
{
    float w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_fmed3f(v[i] * inv, -448.f, 448.f);
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(w[0], w[1], 0, false);
    c = __builtin_amdgcn_cvt_pk_fp8_f32(w[2], w[3], c, true);
    return (uint32_t)c;
}

// eight e4m3 codes as eight bf16 of code * scale (exact: a power of two)
__device__ inline u32x4_t decode8(uint32_t c0, uint32_t c1, float scale)
{
    return u32x4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c0, scale, false)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c0, scale, true)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c1, scale, false)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c1, scale, true))};
}

// Eight values with scale 2^e as the bf16 values that their codes stand for.
__device__ __forceinline__ u32x4_t round8(const float* v, int e)
{
    const float inv = exp2i(-e);
    return decode8(code4(v, inv), code4(v + 4, inv), exp2i(e));
}

// The exponent of the block of 128 whose elements 16 consecutive lanes hold, 8 each.
__device__ __forceinline__ int block_exponent(const float* v)
{
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (finite(v[i])) amax = fmaxf(amax, fabsf(v[i]));
#pragma unroll
    for (int o = 8; o >= 1; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o, 16));
    return scale_exponent(amax);
}

__device__ __forceinline__ void unpack8(const u32x4_t p, float* v)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(p[i] << 16);
        v[2 * i + 1] = __uint_as_float(p[i] & 0xFFFF0000u);
    }
}

}  // namespace moe

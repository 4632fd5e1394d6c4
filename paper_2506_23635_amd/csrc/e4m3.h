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

// The largest of 16 consecutive lanes' values, for all of them: rotations within
// the row of 16 (row_ror), which the maximum takes as its operand.
__device__ __forceinline__ uint32_t max16(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xF, 0xF, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xF, 0xF, false));
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xF, 0xF, false));
}

// The block of 128 whose elements 16 consecutive lanes hold, 8 each: its scale's
// exponent, and this lane's codes.  The maximum is taken of the bits, so a value
// that is not finite shows in it, and only then do the lanes look at them one by
// one (which takes as long as the rest).
struct Coded {
    int e;
    uint32_t lo, hi;
};
__device__ __forceinline__ Coded code_block(const float* v)
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, abs_bits(v[i]));
    m = max16(m);
    Coded c;
    if (m < kInfBits) {
        c.e = scale_exponent(__uint_as_float(m));
        const float inv = exp2i(-c.e);
        c.lo = code4_finite(v, inv);
        c.hi = code4_finite(v + 4, inv);
        return c;
    }
    m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, finite(v[i]) ? abs_bits(v[i]) : 0u);
    c.e = scale_exponent(__uint_as_float(max16(m)));
    const float inv = exp2i(-c.e);
    c.lo = code4(v, inv);
    c.hi = code4(v + 4, inv);
    return c;
}

// The same as the bf16 values that the codes stand for.
__device__ __forceinline__ u32x4_t round_block(const float* v)
{
    const Coded c = code_block(v);
    return decode8(c.lo, c.hi, exp2i(c.e));
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

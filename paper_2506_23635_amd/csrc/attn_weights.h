// attn_weights.h -- the weights of a softmax whose scores arrive in pieces,
// each with a running maximum (attn.hip, attn_paged.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>

namespace moe {

// A weight is 2^(s scale2 - M), M a base-2 maximum of the row, in one fused
// multiply-add: M is m * scale2 with the product's one rounding, everywhere,
// so that p, the rescaling and the merges refer to the same value, and what
// the rounding left out is a factor that all of the row's weights share.  From
// |M| = 2^31 on that factor alone can leave fp32's range, so from kFar on M is
// m * scale2 exactly, in two parts (base2, base2_rest), and the weights are
// 2^((s - m) scale2) (far_scores): the difference first.
__device__ inline float base2(float m, float scale2)
{
#pragma clang fp contract(off)
    return m * scale2;
}

constexpr float kFar = 16777216.f;           // 2^24: below, the factor is in [2^-1/2, 2^1/2]

__device__ inline float base2_rest(float m, float scale2)
{
    const float b = base2(m, scale2);
    return fabsf(b) < kFar ? 0.f : fmaf(m, scale2, -b);
}

// 2^(M' - M) of the maxima m <= mx: what sums that refer to m are multiplied by
__device__ __forceinline__ float decay(float m, float mx, float scale2)
{
    if (m == -INFINITY) return 0.f;
    return __builtin_amdgcn_exp2f((base2(m, scale2) - base2(mx, scale2)) + (base2_rest(m, scale2) - base2_rest(mx, scale2)));
}

// Scores of rows whose maximum m is far, less m; and what is to be subtracted
// from their product with scale2 (ms = base2(m), or 0 where m is -inf).  S is
// float or a vector of floats.
template <class S, int N>
__device__ __forceinline__ float far_scores(S (&sc)[N], float m, float ms)
{
    if (!__ballot(!(fabsf(ms) < kFar))) return ms;
    const bool far = !(fabsf(ms) < kFar);
    const float less = far ? m : 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (sizeof(S) == 4) {
            sc[i] -= less;
        } else {
#pragma unroll
            for (int e = 0; e < (int)(sizeof(S) / 4); ++e) sc[i][e] -= less;
        }
    }
    return far ? 0.f : ms;
}

}  // namespace moe

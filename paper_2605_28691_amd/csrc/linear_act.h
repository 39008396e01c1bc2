// Activations of the linear layer and their slopes, in float32.
//     gelu_tanh(z) = z / (1 + exp(-2u)),  u = sqrt(2/pi) (z + 0.044715 z^3)      ( = z (1 + tanh u) / 2, without the cancellation at negative u)
//     silu(z)      = z / (1 + exp(-z))
// Both are z s with s = 1 / (1 + exp(-v)); the slope is s + z s (1 - s) v'(z).  exp(-v) is 2^e, e = -v log2(e), whose factor is in the constants.
#pragma once
#include <hip/hip_runtime.h>

#include "kernels.h"

namespace skiparse {

constexpr float GELU_C0 = 0.7978845608028654f, GELU_C1 = 0.044715f;  // sqrt(2 / pi)

constexpr float LOG2E = 1.4426950408889634f;

// e = -v log2(e)
__device__ inline float act_exponent(int act, float z) { return act == ACT_SILU ? -LOG2E * z : z * fmaf(z * z, -2.f * LOG2E * GELU_C0 * GELU_C1, -2.f * LOG2E * GELU_C0); }
// 1 / (1 + 2^e): the power overflows to infinity for e above 128, the quotient is 0 then
__device__ inline float act_share(float e) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(e)); }

// Far out s or s (1 - s) is 0 and so is the product with an infinite z, not 0 * inf: the other factor is kept finite.  (A z that is not a number makes s one that is none.)
constexpr float ACT_FAR = 3.4028234663852886e38f;

__device__ inline float act_value(int act, float z) {
    if (act == ACT_NONE) return z;
    return fmaxf(z, -ACT_FAR) * act_share(act_exponent(act, z));
}
__device__ inline float act_slope(int act, float z) {
    const float dv = act == ACT_SILU ? 1.f : fmaf(z * z, 6.f * GELU_C0 * GELU_C1, 2.f * GELU_C0);
    const float s = act_share(act_exponent(act, z)), t = s * (1.f - s);
    return s + t * __builtin_amdgcn_fmed3f(z * dv, -ACT_FAR, ACT_FAR);
}

}  // namespace skiparse

// Activations of the linear layer and their slopes, in float32.
//     gelu_tanh(z) = z / (1 + exp(-2u)),  u = sqrt(2/pi) (z + 0.044715 z^3)      ( = z (1 + tanh u) / 2, without the cancellation at negative u)
//     silu(z)      = z / (1 + exp(-z))
// Both are z s with s = 1 / (1 + exp(-v)); the slope is s + z s (1 - s) v'(z).
#pragma once
#include <hip/hip_runtime.h>

#include "kernels.h"

namespace skiparse {

constexpr float GELU_C0 = 0.7978845608028654f, GELU_C1 = 0.044715f;  // sqrt(2 / pi)

// 1 / (1 + exp(-v)): exp overflows to infinity for v below -88, the quotient is 0 then
__device__ inline float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -1.4426950408889634f)); }

// z s without 0 * inf: where v is -inf the product is the limit 0
__device__ inline float act_value(int act, float z) {
    if (act == ACT_NONE) return z;
    const float v = act == ACT_SILU ? z : 2.f * GELU_C0 * (z + GELU_C1 * z * z * z);
    const float s = sigmoid(v);
    return s == 0.f ? 0.f * s : z * s;
}
__device__ inline float act_slope(int act, float z) {
    const float v = act == ACT_SILU ? z : 2.f * GELU_C0 * (z + GELU_C1 * z * z * z);
    const float dv = act == ACT_SILU ? 1.f : 2.f * GELU_C0 * (1.f + 3.f * GELU_C1 * z * z);
    const float s = sigmoid(v), t = s * (1.f - s);
    return t == 0.f ? s : s + z * t * dv;  // far out the second term is 0, not 0 * inf
}

}  // namespace skiparse

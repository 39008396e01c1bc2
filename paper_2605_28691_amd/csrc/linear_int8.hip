// The linear layer in 8-bit integers: out = act(sx[m] sw[n] sum_k x[m][k] w[n][k] + bias) + residual, x and w int8, sums exact in int32, the rest in float32, rounded once to bf16.
#include "kernels.h"
#include "linear_act.h"

namespace skiparse {

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;

// A wavefront has 16 rows and 64 channels, and reads its fragments from memory: lane l 16 bytes of row l % 16 from k = 16 (l / 16).
__global__ __launch_bounds__(256) void linear_int8_kernel(LinearInt8Args a, uint32_t blocks_m) {
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, li = lane & 15u, g = lane >> 4;
    const uint32_t m = (blockIdx.x % blocks_m * 4u + wave) * 16u + li, n0 = blockIdx.x / blocks_m * 64u;
    const uint32_t mc = m < a.M ? m : a.M - 1u;
    const uint32_t from = a.order == 1 ? source_row<TO_SPARSE>(a.rows, mc, 0u) : a.order == 2 ? source_row<TO_ORIGINAL>(a.rows, mc, 0u) : mc;
    const char* const x = (const char*)a.x + (size_t)from * a.K;
    const i32x4 zero = {0, 0, 0, 0};
    i32x4 acc[4] = {zero, zero, zero, zero};
    for (uint32_t k = 0; k < a.K; k += 64u) {
        const uint32_t at = k + 16u * g;
        const i32x4 p = at < a.K ? *(const i32x4*)(x + at) : zero;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint32_t n = n0 + 16u * j + li;
            const i32x4 q = at < a.K && n < a.N ? *(const i32x4*)((const char*)a.w + (size_t)n * a.K + at) : zero;
            acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q, p, acc[j], 0, 0, 0);
        }
    }
    if (m >= a.M) return;
    const float sx = a.x_scales[from];
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const uint32_t n = n0 + 16u * j + 4u * g;
        if (n >= a.N) continue;
        bf16x4 y;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            float z = fmaf((float)acc[j][e] * sx, a.w_scales[n + e], a.bias != nullptr ? (float)((const __bf16*)a.bias)[n + e] : 0.f);
            z = act_value(a.act, z);
            if (a.residual != nullptr) z += (float)((const __bf16*)a.residual)[(size_t)m * a.N + n + e];
            y[e] = (__bf16)z;
        }
        *(bf16x4*)((__bf16*)a.out + (size_t)m * a.N + n) = y;
    }
}

size_t linear_int8_workspace(uint32_t, uint32_t, uint32_t) { return 0; }

hipError_t launch_linear_int8(const LinearInt8Args& a, hipStream_t stream) {
    const uint64_t bm = ((uint64_t)a.M + 63u) / 64u, bn = ((uint64_t)a.N + 63u) / 64u;
    if (!fits_grid(bm * bn, 256u)) return hipErrorInvalidConfiguration;
    linear_int8_kernel<<<(uint32_t)(bm * bn), 256, 0, stream>>>(a, (uint32_t)bm);
    return hipGetLastError();
}

}  // namespace skiparse

// The linear layer in 8-bit integers: out = act(sx[m] sw[n] sum_k x[m][k] w[n][k] + bias) + residual, x and w int8, sums exact in int32, the rest in float32, rounded once to bf16.
// The products are those of linear_tiles.h with v_mfma_i32_16x16x64_i8: its operands are 16 bytes a lane, as those of the bf16 product are, and k is summed over, so the walk over k, what it
// loads and how it lies in LDS are the same bytes, two codes in the place of one number.  What is left of the sums on the way out are scales: those of a wavefront's rows and channels are asked for before
// its walk begins.  Parts of a sum are whole numbers too: however a product is cut, a row's bits are the same.
// Large products are bound by the matrix cores at the board's power limit: 16,384^3 2925 TOP/s (a library's product without an epilogue 2384), 80,640 x 5120 -> 20,480 2.68 POP/s without an epilogue and
// 2.45 to 2.62 with GELU (6.3 and 6.44 to 6.9 ms: cards differ).  Small ones by what stands outside the walk: 32,760 x 1536 -> 1536, three rounds of 256 tiles, 77 to 84 us.  A tile of it has 1.5 until its loads leave, 2.5 until they land, 5 for its
// results, 12 with a residual, which all CUs move at once, and the rest for twelve steps (20 to 23 with two buffers, 14 on codes of zero; without any results the product took 71 of then 87).  Loads sent off
// earlier in a step and waited for later, in a second barrier, were 3 % slower, results past the caches as well, and first tiles that begin at four different times no faster.
#include "linear_tiles.h"

namespace skiparse {

// One row: a wavefront has two channels and reads 2048 codes of each at once; four products an instruction (v_dot4_i32_i8).  Bound by reading w, and by what a launch takes.  (us, 1 / 2 / 4 channels: 5120 -> 5120
// 7.4 / 7.2 / 8.0, 1536 -> 8960 6.2 / 5.0 / 5.3, 8960 -> 1536 7.6 / 6.0 / 6.6, 5120 -> 30,720, 157 MB, 32.1 / 29.5 / 29.5.)
constexpr int ROW8_CHANNELS = 2;
__global__ __launch_bounds__(256) void linear_int8_row_kernel(LinearArgs a) {
    typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
    constexpr int CH = ROW8_CHANNELS, AT_ONCE = 2;  // times 1024 codes
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t n0 = (blockIdx.x * 4u + wave) * CH;
    if (n0 >= a.N) return;
    const uint32_t ld = a.K * 2u;  // bytes
    int acc[CH];
#pragma unroll
    for (int c = 0; c < CH; c++) acc[c] = 0;
#if defined(__HIP_DEVICE_COMPILE__)
    // N is a multiple of 8, so a wavefront's channels are all there
    const auto wb = __builtin_amdgcn_make_buffer_rsrc((char*)a.q + (size_t)n0 * ld, 0, LIN_RECORDS, 0x27000);
    const auto xb = __builtin_amdgcn_make_buffer_rsrc((char*)a.p, 0, LIN_RECORDS, 0x27000);
    for (uint32_t k = 0; k < ld; k += 1024u * AT_ONCE) {
        u32x4 w[AT_ONCE][CH], x[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; u++) {
            const uint32_t at = k + 1024u * u + lane * 16u;  // behind the end: zeros
#pragma unroll
            for (int c = 0; c < CH; c++) w[u][c] = __builtin_amdgcn_raw_buffer_load_b128(wb, at < ld ? at + c * ld : LIN_OUTSIDE, 0, 0);
            x[u] = __builtin_amdgcn_raw_buffer_load_b128(xb, at < ld ? at : LIN_OUTSIDE, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; u++)
#pragma unroll
            for (int e = 0; e < 4; e++)
#pragma unroll
                for (int c = 0; c < CH; c++) acc[c] = __builtin_amdgcn_sdot4((int)w[u][c][e], (int)x[u][e], acc[c], false);
    }
#endif
    int sum = 0;  // lane c takes that of channel c
#pragma unroll
    for (int c = 0; c < CH; c++) {
        int s = acc[c];
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) s += __shfl_xor(s, off);
        if (lane == (uint32_t)c) sum = s;
    }
    if (lane >= CH) return;
    const uint32_t n = n0 + lane;
    const LinearEpilogue& e = a.e;
    float z = act_value(e.act, int8_value_far(sum, a.x_scales[0], a.w_scales[n], e.bias != nullptr ? (float)((const __bf16*)e.bias)[n] : 0.f));
    if (e.residual != nullptr) z = int8_plus(z, (float)((const __bf16*)e.residual)[n]);
    ((__bf16*)e.out)[n] = (__bf16)z;
}

static hipError_t launch_row8(const LinearArgs& a, hipStream_t stream) {
    constexpr uint32_t per = ROW8_CHANNELS * 4u;
    linear_int8_row_kernel<<<(a.N + per - 1u) / per, 256, 0, stream>>>(a);
    return hipGetLastError();
}
template <int FM, int FN>
static hipError_t launch_few8(const LinearArgs& a, hipStream_t stream) {
    constexpr uint32_t per = 16u * FN;
    linear_few_kernel<FM, FN, false, LINEAR_INT8><<<(a.N + per - 1u) / per, 64 * FEW_WAVES, 0, stream>>>(a);
    return hipGetLastError();
}
static hipError_t launch_few8(const LinearArgs& a, hipStream_t stream) {
    if (a.M == 1u) return launch_row8(a, stream);  // moved or not, row 0
    if (few_blocks8(a.M, a.N, a.K * 2u) == 2u) return a.M <= 16u ? launch_few8<1, 2>(a, stream) : launch_few8<2, 2>(a, stream);
    return a.M <= 16u ? launch_few8<1, 1>(a, stream) : launch_few8<2, 1>(a, stream);
}

template <bool EXTRAS>
static hipError_t launch_int8(const LinearArgs& a, hipStream_t stream) {
    const LinearPlan p = plan_linear8(a.M, a.N, a.K, a.e.act != ACT_NONE);
    switch (p.shape) {
        case T256: return launch_tiles<T256, LINEAR_INT8, EXTRAS>(a, p, stream);
        case T128: return launch_tiles<T128, LINEAR_INT8, EXTRAS>(a, p, stream);
        default: return launch_tiles<T64, LINEAR_INT8, EXTRAS>(a, p, stream);
    }
}

// for either, with an activation and without
size_t linear_int8_workspace(uint32_t M, uint32_t N, uint32_t K) {
    if (linear_few8(M, N, K)) return 0u;
    const size_t without = plan_linear8(M, N, K / 2u, false).workspace(), with = plan_linear8(M, N, K / 2u, true).workspace();
    return without > with ? without : with;
}

hipError_t launch_linear_int8(const LinearArgs& a, hipStream_t stream) {
    if (linear_few8(a.M, a.N, a.K * 2u)) return launch_few8(a, stream);
    return a.e.act != ACT_NONE || a.e.residual ? launch_int8<true>(a, stream) : launch_int8<false>(a, stream);
}

}  // namespace skiparse

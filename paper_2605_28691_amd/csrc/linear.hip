// Products of the linear layer on the matrix cores, bf16 in and out, float32 sums: C[m][n] = sum_k P(m, k) Q(n, k), and its epilogue
//     z = C + bias (kept, if asked for, in bf16 or as an 8-bit checkpoint),  out = act(z) + residual
// Three forms:  out = x w^T (neither operand transposed),  dx = dz w (Q = w given as [k][n]),  dw = dz^T x (both given as [k][..]).
//
//   * v_mfma_f32_16x16x32_bf16: the board's power sets the clock on real data, and this form takes less of it than 32x32x16, which reads and writes twice the accumulators
//     a product (products alone, operands N(0,1): 2041 and 1820 TFLOP/s; on zeros 2419 and 2453).  Q's rows are its A operand, P's its B.
//   * A workgroup is 4 wavefronts, 2 x 2, one a SIMD; at 256 x 256 each has 128 x 128 of C in 256 accumulation registers, so that a fragment read from LDS feeds 8
//     products.
//   * Tiles go from memory straight into LDS (buffer_load_dwordx4 ... lds), 64 of k a step, double buffered.  Operands with k along the row are laid out in rows of
//     128 bytes and read 16 bytes at a time; transposed ones in rows of 256 and read with ds_read_b64_tr_b16; no read has bank conflicts.
//   * Ends: a 16-byte piece behind the end of k is given an offset outside the buffer and reads as zero; transposed operands end with the buffer; rows
//     past the last read the last one, columns past the last whatever lies there, and neither is stored.
// Bound by the matrix cores at the board's power limit: 8192^3 720 us (1526 TFLOP/s), 743 both operands transposed; 80,640 x 5120 -> 5120 2992 us (1413).
#include "linear_tiles.h"

namespace skiparse {

// x w^T for one row, which reads w once and is bound by that: a wavefront has CH channels, and reads 1024 of k of each at once, whole lines; x is read with them and comes out of the
// caches.  Its sums are added up over the lanes at the end.  (5120 -> 5120: 9.5 us; reading w as the products' fragments, 64 bytes of 16 rows at once, 15.6.)
// KEPT: z is kept as a checkpoint, of whose blocks of 32 channels a workgroup has one.  A channel's sum does not depend on either.  (us with a checkpoint written, so / in tiles: 5120 -> 5120
// 13.1 / 21.8, 1536 -> 8960 9.3 / 20.3, 8960 -> 1536 15.3 / 19.4, 64 -> 11,200 4.3 / 4.4.)
constexpr int row_waves(int channels, bool kept) { return kept ? CKPT_BLOCK / channels : 4; }
template <int CH, bool KEPT>
__global__ __launch_bounds__(64 * row_waves(CH, KEPT)) void linear_row_kernel(LinearArgs a) {
    typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
    constexpr int AT_ONCE = 2;  // times 512 of k
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t n0 = (blockIdx.x * row_waves(CH, KEPT) + wave) * CH;
    if (!KEPT && n0 >= a.N) return;
    __shared__ __attribute__((aligned(16))) float block[KEPT ? CKPT_BLOCK : 4];
    const uint32_t ld = a.K * 2u, end = !KEPT || n0 < a.N ? a.K : 0u;  // a wavefront behind the last channel reads nothing, and has zeros
    float acc[CH];
#pragma unroll
    for (int c = 0; c < CH; c++) acc[c] = 0.f;
#if defined(__HIP_DEVICE_COMPILE__)
    // N is a multiple of 8, so a wavefront's channels are all there
    const auto wb = __builtin_amdgcn_make_buffer_rsrc((char*)a.q + (size_t)n0 * ld, 0, LIN_RECORDS, 0x27000);
    const auto xb = __builtin_amdgcn_make_buffer_rsrc((char*)a.p, 0, LIN_RECORDS, 0x27000);
    for (uint32_t k = 0; k < end; k += 512u * AT_ONCE) {
        u32x4 w[AT_ONCE][CH], x[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; u++) {
            const uint32_t at = k + 512u * u + lane * 8u;  // behind the end: zeros
#pragma unroll
            for (int c = 0; c < CH; c++) w[u][c] = __builtin_amdgcn_raw_buffer_load_b128(wb, at < a.K ? at * 2u + c * ld : LIN_OUTSIDE, 0, 0);
            x[u] = __builtin_amdgcn_raw_buffer_load_b128(xb, at < a.K ? at * 2u : LIN_OUTSIDE, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; u++)
#pragma unroll
            for (int e = 0; e < 8; e++) {
                auto value = [&](const u32x4& v) __attribute__((always_inline)) -> float { return __uint_as_float(e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16); };
                const float xv = value(x[u]);
#pragma unroll
                for (int c = 0; c < CH; c++) acc[c] = fmaf(value(w[u][c]), xv, acc[c]);
            }
    }
#endif
    // lane c takes the sum of channel c
    float z = 0.f;
#pragma unroll
    for (int c = 0; c < CH; c++) {
        float s = acc[c];
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) s += __shfl_xor(s, off);
        if (lane == (uint32_t)c) z = s;
    }
    const uint32_t n = n0 + lane;
    const bool on = lane < CH && (!KEPT || n0 < a.N);
    const LinearEpilogue& e = a.e;
    if (on && e.bias != nullptr) z += (float)((const __bf16*)e.bias)[n];
    if (KEPT) {
        if (lane < CH) block[wave * CH + lane] = z;
        __syncthreads();
        if (threadIdx.x < CKPT_BLOCK / 4u) {  // 4 channels each, the block's largest from all of them
            const f32x4 own = *(const f32x4*)(block + threadIdx.x * 4u);
            const uint32_t c = blockIdx.x * CKPT_BLOCK + threadIdx.x * 4u;
            uint32_t top = ckpt_largest(own);
#pragma unroll
            for (int off = 1; off <= 4; off <<= 1) {
                const uint32_t o = (uint32_t)__shfl_xor((int)top, off);
                top = o > top ? o : top;
            }
            const uint32_t byte = ckpt_byte(top);
            if (c < a.N) *(uint32_t*)((unsigned char*)e.pre + c) = ckpt_codes(own[0], own[1], own[2], own[3], ckpt_down(byte));
            if (threadIdx.x == 0u) ((unsigned char*)e.pre_scales)[blockIdx.x] = (unsigned char)byte;
        }
    }
    if (!on) return;
    if (!KEPT && e.pre != nullptr) ((__bf16*)e.pre)[n] = (__bf16)z;
    z = act_value(e.act, z);
    if (e.residual != nullptr) z += (float)((const __bf16*)e.residual)[n];
    ((__bf16*)e.out)[n] = (__bf16)z;
}

template <int CH, bool KEPT = false>
static hipError_t launch_row(const LinearArgs& a, hipStream_t stream) {
    constexpr uint32_t waves = row_waves(CH, KEPT), per = CH * waves;
    linear_row_kernel<CH, KEPT><<<(a.N + per - 1u) / per, 64 * waves, 0, stream>>>(a);
    return hipGetLastError();
}
template <int FM, int FN, bool KEPT = false>
static hipError_t launch_few(const LinearArgs& a, hipStream_t stream) {
    constexpr uint32_t per = 16u * FN;
    linear_few_kernel<FM, FN, KEPT><<<(a.N + per - 1u) / per, 64 * FEW_WAVES, 0, stream>>>(a);
    return hipGetLastError();
}
static hipError_t launch_few(const LinearArgs& a, hipStream_t stream) {
    const bool kept = a.e.pre_scales != nullptr;
    if (a.M == 1u) {  // moved or not, row 0
        if (kept) return launch_row<4, true>(a, stream);
        const uint32_t channels = row_channels(a.N);
        return channels == 1u ? launch_row<1>(a, stream) : channels == 2u ? launch_row<2>(a, stream) : launch_row<4>(a, stream);
    }
    if (kept) return a.M <= 16u ? launch_few<1, 2, true>(a, stream) : launch_few<2, 2, true>(a, stream);
    if (few_blocks(a.M, a.N, a.K) == 2u) return a.M <= 16u ? launch_few<1, 2>(a, stream) : launch_few<2, 2>(a, stream);
    return a.M <= 16u ? launch_few<1, 1>(a, stream) : launch_few<2, 1>(a, stream);
}

template <int FORM, bool EXTRAS = false>
static hipError_t launch_form(const LinearArgs& a, hipStream_t stream) {
    if (FORM == LINEAR_FWD && linear_few(a.M, a.K)) return launch_few(a, stream);
    const LinearPlan p = plan_linear(a.M, a.N, a.K);
    switch (p.shape) {
        case T256: return launch_tiles<T256, FORM, EXTRAS>(a, p, stream);
        case T128: return launch_tiles<T128, FORM, EXTRAS>(a, p, stream);
        case T128X256: return launch_tiles<T128X256, FORM, EXTRAS>(a, p, stream);
        default: return launch_tiles<T64, FORM, EXTRAS>(a, p, stream);
    }
}

size_t linear_workspace(int form, uint32_t M, uint32_t N, uint32_t K) {
    return form == LINEAR_FWD && linear_few(M, K) ? 0u : plan_linear(M, N, K).workspace();
}

hipError_t launch_linear(int form, const LinearArgs& a, hipStream_t stream) {
    switch (form) {
        case LINEAR_FWD: return a.e.act != ACT_NONE || a.e.residual || a.e.pre ? launch_form<LINEAR_FWD, true>(a, stream) : launch_form<LINEAR_FWD>(a, stream);
        case LINEAR_DX: return launch_form<LINEAR_DX>(a, stream);
        default: return launch_form<LINEAR_DW>(a, stream);
    }
}

}  // namespace skiparse

// Products of the linear layer on the matrix cores, bf16 in and out, float32 sums: C[m][n] = sum_k P(m, k) Q(n, k), and its epilogue
//     z = C + bias (kept, if asked for, in bf16 or as an 8-bit checkpoint),  out = act(z) + residual
// Three forms:  out = x w^T (neither operand transposed),  dx = dz w (Q = w given as [k][n]),  dw = dz^T x (both given as [k][..]).
//
//   * The MFMA takes Q's rows as its A operand and P's as B, so that a lane's accumulators are 16 channels of ONE row of C: bias, residual and the blocks of a
//     checkpoint are its own.
//   * Tiles go from memory straight into LDS (buffer_load_dwordx4 ... lds), 64 of k a step, double buffered.  Operands with k along the row are laid out in rows of
//     128 bytes and read 16 bytes at a time; transposed ones in rows of 256 and read with ds_read_b64_tr_b16; swizzles as in lds_layout.h.
//   * Ends: a 16-byte piece behind the end of k is given an offset outside the buffer and reads as zero; transposed operands end with the buffer; rows
//     past the last read the last one, columns past the last whatever lies there, and neither is stored.
#include "checkpoint.h"
#include "kernels.h"
#include "lds_layout.h"
#include "linear_act.h"

namespace skiparse {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;

#define LDS_PTR(T) __attribute__((address_space(3))) T*

constexpr uint32_t LIN_KT = 64;           // of k a step
constexpr uint32_t LIN_OUTSIDE = ~0u;     // an offset outside every buffer
constexpr uint32_t LIN_RECORDS = 0xfffffff0u;

// One operand's side of a workgroup's tile: ROWS of m (or n) by 64 of k.
template <int ROWS, bool T, int NW>
struct Side {
    static constexpr int INSTR = ROWS * 128 / 1024 / NW;  // direct loads of a wavefront and step, 1 KiB each
    static constexpr int BYTES = ROWS * 128;
    uint32_t off[INSTR];  // of the lane's piece from the step's base
    uint32_t kofs[INSTR]; // !T: where in the step's k it lies
    // row_off: byte offset of row r of the tile from the base (!T), row_bytes: of a row of k (T)
    template <typename F>
    __device__ __attribute__((always_inline)) inline void init(uint32_t wave, uint32_t lane, uint32_t row_bytes, F row_off) {
#pragma unroll
        for (int i = 0; i < INSTR; i++) {
            const uint32_t n = wave * INSTR + i;  // of the tile's
            if (!T) {
                const uint32_t r = n * 8u + lane / 8u;
                kofs[i] = ((lane % 8u) ^ lds_swizzle<64>(r)) * 8u;
                off[i] = row_off(r) + kofs[i] * 2u;
            } else {
                const uint32_t part = n / 16u, r = n % 16u * 4u + lane / 16u;  // 128 columns a part
                kofs[i] = 0u;
                off[i] = r * row_bytes + part * 256u + ((lane % 16u) ^ lds_swizzle<128>(r)) * 16u;
            }
        }
    }
    __device__ __attribute__((always_inline)) inline void issue(const char* base, uint32_t records, uint32_t k_left, char* buf, uint32_t wave) const {
#if defined(__HIP_DEVICE_COMPILE__)  // the host pass does not know the buffer's type, and would drop the kernel without a word
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, records, 0x27000);
#pragma unroll
        for (int i = 0; i < INSTR; i++)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (LDS_PTR(void))(buf + (wave * INSTR + i) * 1024u), 16, T || kofs[i] < k_left ? off[i] : LIN_OUTSIDE, 0, 0, 0);
#endif
    }
};

// Fragment of 32 rows from `row0` (a multiple of 32) and 16 of k: lane l has row l % 32, k = 16 ks + 8 (l / 32) ...
template <bool T>
__device__ __attribute__((always_inline)) inline bf16x8 read_fragment(const char* buf, uint32_t row0, uint32_t ks, uint32_t lane) {
    const uint32_t h = lane >> 5;
    if (!T) {
        const uint32_t r = lane & 31u;
        return *(const bf16x8*)(buf + (row0 + r) * 128u + ((2u * ks + h) ^ lds_swizzle<64>(r)) * 16u);
    }
    const uint32_t li = lane & 15u, group = lane >> 4 & 1u;
    const char* const part = buf + row0 / 128u * 16384u;
    bf16x4 v[2];
#pragma unroll
    for (uint32_t sec = 0; sec < 2; sec++) {
        const uint32_t r = 16u * ks + 8u * h + 4u * sec + (li >> 2);
        const uint32_t c = row0 % 128u / 8u + group * 2u + ((li & 3u) >> 1);
        const char* const at = part + r * 256u + ((c ^ lds_swizzle<128>(r)) * 16u) + 8u * (li & 1u);
        v[sec] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(LDS_PTR(char))at);
    }
    return __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
}

// Row m of C, channels n .. n + 3 of a block of 32: z = acc + bias; the result's value, without the residual.
__device__ __attribute__((always_inline)) inline f32x4 with_bias(const LinearEpilogue& e, f32x4 z, uint32_t n) {
    if (e.bias != nullptr) {
        const bf16x4 b = *(const bf16x4*)((const __bf16*)e.bias + n);
#pragma unroll
        for (int i = 0; i < 4; i++) z[i] += (float)b[i];
    }
    return z;
}

template <int BM, int BN, int FORM>
__global__ __launch_bounds__(256) void linear_kernel(LinearArgs a, uint32_t tiles_n) {
    constexpr bool PT = FORM == LINEAR_DW, QT = FORM != LINEAR_FWD;
    constexpr int NW = 4, FM = BM / 64, FN = BN / 64;  // wavefronts 2 x 2; blocks of 32 that each has
    using SP = Side<BM, PT, NW>;
    using SQ = Side<BN, QT, NW>;
    __shared__ __attribute__((aligned(1024))) char pbuf[2][SP::BYTES];
    __shared__ __attribute__((aligned(1024))) char qbuf[2][SQ::BYTES];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = wave & 1u, wn = wave >> 1;
    const uint32_t tm = blockIdx.x / tiles_n, tn = blockIdx.x - tm * tiles_n;
    const uint32_t m0 = tm * BM, n0 = tn * BN;
    const uint32_t ldp = (PT ? a.M : a.K) * 2u, ldq = (QT ? a.N : a.K) * 2u;  // bytes
    const bool mapped = FORM == LINEAR_FWD && a.order != 0;
    SP sp;
    SQ sq;
    sp.init(wave, lane, ldp, [&](uint32_t r) __attribute__((always_inline)) -> uint32_t {
        const uint32_t last = a.M - 1u - m0;
        const uint32_t m = r < last ? r : last;
        if (!mapped) return m * ldp;
        return (a.order == 1 ? source_row<TO_SPARSE>(a.rows, m0 + m, 0u) : source_row<TO_ORIGINAL>(a.rows, m0 + m, 0u)) * ldp;
    });
    sq.init(wave, lane, ldq, [&](uint32_t r) __attribute__((always_inline)) -> uint32_t {
        const uint32_t last = a.N - 1u - n0;
        return (r < last ? r : last) * ldq;
    });
    const char* const p0 = (const char*)a.p + (PT ? (size_t)m0 * 2u : mapped ? 0 : (size_t)m0 * ldp);
    const char* const q0 = (const char*)a.q + (QT ? (size_t)n0 * 2u : (size_t)n0 * ldq);
    auto records = [&](bool t, uint32_t k, uint32_t ld, uint32_t col0) __attribute__((always_inline)) -> uint32_t {
        if (!t) return LIN_RECORDS;
        const uint64_t left = (uint64_t)(a.K - k) * ld - col0 * 2u;
        return left < LIN_RECORDS ? (uint32_t)left : LIN_RECORDS;
    };
    auto issue = [&](uint32_t k, int b) __attribute__((always_inline)) {
        sp.issue(p0 + (PT ? (size_t)k * ldp : (size_t)k * 2u), records(PT, k, ldp, m0), a.K - k, pbuf[b], wave);
        sq.issue(q0 + (QT ? (size_t)k * ldq : (size_t)k * 2u), records(QT, k, ldq, n0), a.K - k, qbuf[b], wave);
    };
    f32x16 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; i++)
#pragma unroll
        for (int j = 0; j < FN; j++)
#pragma unroll
            for (int r = 0; r < 16; r++) acc[i][j][r] = 0.f;
    issue(0, 0);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    int b = 0;
    for (uint32_t k = 0; k < a.K; k += LIN_KT) {
        if (k + LIN_KT < a.K) issue(k + LIN_KT, b ^ 1);
#pragma unroll
        for (uint32_t ks = 0; ks < 4; ks++) {
            bf16x8 pf[FM], qf[FN];
#pragma unroll
            for (int i = 0; i < FM; i++) pf[i] = read_fragment<PT>(pbuf[b], (wm * FM + i) * 32u, ks, lane);
#pragma unroll
            for (int j = 0; j < FN; j++) qf[j] = read_fragment<QT>(qbuf[b], (wn * FN + j) * 32u, ks, lane);
#pragma unroll
            for (int i = 0; i < FM; i++)
#pragma unroll
                for (int j = 0; j < FN; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[j], pf[i], acc[i][j], 0, 0, 0);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        b ^= 1;
    }
    // the epilogue: a lane has row m and, of every block of 32 channels, 8 g + 4 h .. + 3
    const LinearEpilogue& e = a.e;
    const uint32_t h = lane >> 5;
#pragma unroll
    for (int i = 0; i < FM; i++) {
        const uint32_t m = m0 + (wm * FM + i) * 32u + (lane & 31u);
        const bool row_in = m < a.M;
        const size_t row = (size_t)(row_in ? m : 0u) * a.N;
#pragma unroll
        for (int j = 0; j < FN; j++) {
            const uint32_t nb = n0 + (wn * FN + j) * 32u;
            f32x4 z[4];
            uint32_t top = 0u;
#pragma unroll
            for (int g = 0; g < 4; g++) {
                const uint32_t n = nb + 8u * g + 4u * h;
                z[g] = f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
                if (n < a.N) {
                    z[g] = with_bias(e, z[g], n);
#pragma unroll
                    for (int x = 0; x < 4; x++) {
                        const uint32_t s = ckpt_size(z[g][x]);
                        top = s > top ? s : top;
                    }
                }
            }
            uint32_t byte = 0u;
            if (e.pre_scales != nullptr) {
                const uint32_t o = (uint32_t)__shfl_xor((int)top, 32);
                byte = ckpt_byte(o > top ? o : top);
                if (row_in && nb < a.N && h == 0u) ((unsigned char*)e.pre_scales)[(size_t)m * ((a.N + 31u) / 32u) + nb / 32u] = (unsigned char)byte;
            }
#pragma unroll
            for (int g = 0; g < 4; g++) {
                const uint32_t n = nb + 8u * g + 4u * h;
                if (!row_in || n >= a.N) continue;
                if (e.pre_scales != nullptr) *(uint32_t*)((char*)e.pre + row + n) = ckpt_codes(z[g][0], z[g][1], z[g][2], z[g][3], ckpt_down(byte));
                else if (e.pre != nullptr) {
                    bf16x4 o;
#pragma unroll
                    for (int x = 0; x < 4; x++) o[x] = (__bf16)z[g][x];
                    *(bf16x4*)((__bf16*)e.pre + row + n) = o;
                }
                f32x4 y;
#pragma unroll
                for (int x = 0; x < 4; x++) y[x] = act_value(e.act, z[g][x]);
                if (e.residual != nullptr) {
                    const bf16x4 r = *(const bf16x4*)((const __bf16*)e.residual + row + n);
#pragma unroll
                    for (int x = 0; x < 4; x++) y[x] += (float)r[x];
                }
                bf16x4 o;
#pragma unroll
                for (int x = 0; x < 4; x++) o[x] = (__bf16)y[x];
                *(bf16x4*)((__bf16*)e.out + row + n) = o;
            }
        }
    }
}

template <int FORM>
static hipError_t launch_form(const LinearArgs& a, hipStream_t stream) {
    constexpr int BM = 128, BN = 128;
    const uint32_t tiles_m = (a.M + BM - 1u) / BM, tiles_n = (a.N + BN - 1u) / BN;
    if (!fits_grid((uint64_t)tiles_m * tiles_n, 256u)) return hipErrorInvalidConfiguration;
    linear_kernel<BM, BN, FORM><<<tiles_m * tiles_n, 256, 0, stream>>>(a, tiles_n);
    return hipGetLastError();
}

hipError_t launch_linear(int form, const LinearArgs& a, hipStream_t stream) {
    switch (form) {
        case LINEAR_FWD: return launch_form<LINEAR_FWD>(a, stream);
        case LINEAR_DX: return launch_form<LINEAR_DX>(a, stream);
        default: return launch_form<LINEAR_DW>(a, stream);
    }
}

}  // namespace skiparse

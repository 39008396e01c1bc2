// What stands in front of a linear layer's backward products: dz = dy act'(z), written in the order of the input's rows, and the bias's gradient, the sum of dz over
// the rows.  Bound by HBM bandwidth: dy and z are read once, dz written once; the sums are of the float32 values, before dz is rounded to bf16 for the products.
// The rounding is off by 2^-8 of a value at most and independent from row to row, so in a product's result it is as large as that of its own output.
//
// A workgroup takes the rows of a part by 256 channels: 32 lanes of 8 channels, 8 rows at a time.  One row a thread at a time is best: what is in flight lies close together then
// (us, 6426 x 4008 with a checkpoint of z / 3840 x 5120 with z in bf16, both in parts of 32 rows: one row 30.2 / 28.0, two at once 34.1 / -, four 39.7 / 35.8; parts of 128 41.4
// / -).  The sums of a part go to memory and are added up in order by a second launch: the same bits every time, without atomics.  80,640 x 5120, 2.1 GB, 430 us.
#include "checkpoint.h"
#include "kernels.h"
#include "linear_act.h"
#include "linear_plan.h"

namespace skiparse {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

constexpr uint32_t LANES_X = 32, COLS = LANES_X * 8, ROWS_AT_ONCE = 256 / LANES_X;
static_assert(COLS == 256, "what linear_rows_per_part() counts on");

__device__ inline void unpack8(const u32x4& x, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; e++) {
        v[2 * e] = __uint_as_float(x[e] << 16);
        v[2 * e + 1] = __uint_as_float(x[e] & 0xffff0000u);
    }
}

template <bool ACT, bool CHECKPOINT>
__global__ __launch_bounds__(256) void linear_rows_kernel(LinearRowsArgs a, uint32_t col_blocks, uint32_t per_part) {
    __shared__ float sums[ROWS_AT_ONCE][COLS];
    const uint32_t part = blockIdx.x / col_blocks, cb = blockIdx.x - part * col_blocks;
    const uint32_t lane = threadIdx.x % LANES_X, ty = threadIdx.x / LANES_X;
    const uint32_t n = cb * COLS + lane * 8u;
    const bool in = n < a.N;
    const uint32_t blocks = (a.N + CKPT_BLOCK - 1u) / CKPT_BLOCK;
    float sum[8] = {};
    for (uint32_t r = ty; r < per_part; r += ROWS_AT_ONCE) {
        const uint32_t row = part * per_part + r;
        if (!in || row >= a.M) break;
        uint32_t from = row;
        if (a.order == 1) from = source_row<TO_SPARSE>(a.rows, row, 0u);
        if (a.order == 2) from = source_row<TO_ORIGINAL>(a.rows, row, 0u);
        const size_t at = (size_t)from * a.N + n;
        float g[8];
        unpack8(*(const u32x4*)((const unsigned short*)a.dy + at), g);
        if (ACT) {
            float z[8];
            if (CHECKPOINT) {
                const u32x2 c = *(const u32x2*)((const unsigned char*)a.pre + at);
                const float up = ckpt_up(((const unsigned char*)a.pre_scales)[(size_t)from * blocks + n / CKPT_BLOCK]);
                float lo[4], hi[4];
                ckpt_values(c[0], up, lo);
                ckpt_values(c[1], up, hi);
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    z[e] = lo[e];
                    z[4 + e] = hi[e];
                }
            } else {
                unpack8(*(const u32x4*)((const unsigned short*)a.pre + at), z);
            }
#pragma unroll
            for (int e = 0; e < 8; e++) g[e] *= act_slope(a.act, z[e]);
        }
        if (a.dz != nullptr) {
            bf16x8 y;
#pragma unroll
            for (int e = 0; e < 8; e++) y[e] = (__bf16)g[e];
            *(bf16x8*)((__bf16*)a.dz + (size_t)row * a.N + n) = y;
        }
#pragma unroll
        for (int e = 0; e < 8; e++) sum[e] += g[e];
    }
    if (a.db_part == nullptr) return;
#pragma unroll
    for (int e = 0; e < 8; e++) sums[ty][lane * 8u + e] = sum[e];
    __syncthreads();
    const uint32_t c = cb * COLS + threadIdx.x;
    if (c >= a.N) return;
    float s = 0.f;
#pragma unroll
    for (uint32_t i = 0; i < ROWS_AT_ONCE; i++) s += sums[i][threadIdx.x];
    if (gridDim.x == col_blocks) ((__bf16*)a.db)[c] = (__bf16)s;  // one part
    else a.db_part[(size_t)part * a.N + c] = s;
}

// The parts' sums, 64 channels a workgroup, 16 parts at a time.
__global__ __launch_bounds__(1024) void linear_db_kernel(const float* __restrict__ part, __bf16* __restrict__ db, uint32_t parts, uint32_t N) {
    __shared__ float sums[16][64];
    const uint32_t lane = threadIdx.x & 63u, ty = threadIdx.x >> 6, n = blockIdx.x * 64u + lane;
    float s = 0.f;
    if (n < N) {
#pragma unroll 8
        for (uint32_t p = ty; p < parts; p += 16u) s += part[(size_t)p * N + n];
    }
    sums[ty][lane] = s;
    __syncthreads();
    if (ty != 0u || n >= N) return;
    s = 0.f;
#pragma unroll
    for (uint32_t i = 0; i < 16u; i++) s += sums[i][lane];
    db[n] = (__bf16)s;
}

hipError_t launch_linear_rows(const LinearRowsArgs& a, hipStream_t stream) {
    const uint32_t col_blocks = (a.N + COLS - 1u) / COLS, parts = linear_rows_parts(a.M, a.N);
    if (!fits_grid((uint64_t)col_blocks * parts, 256u)) return hipErrorInvalidConfiguration;
    const uint32_t per = linear_rows_per_part(a.M, a.N);
    if (a.pre == nullptr) linear_rows_kernel<false, false><<<col_blocks * parts, 256, 0, stream>>>(a, col_blocks, per);
    else if (a.pre_scales == nullptr) linear_rows_kernel<true, false><<<col_blocks * parts, 256, 0, stream>>>(a, col_blocks, per);
    else linear_rows_kernel<true, true><<<col_blocks * parts, 256, 0, stream>>>(a, col_blocks, per);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.db_part == nullptr || parts == 1u) return e;
    linear_db_kernel<<<(a.N + 63u) / 64u, 1024, 0, stream>>>(a.db_part, (__bf16*)a.db, parts, a.N);
    return hipGetLastError();
}

}  // namespace skiparse

// Root-mean-square norm of rows, with the residual's addition in front of it and, if asked for, its result in 8-bit integers; rows in 8-bit integers without a norm; and the
// norm's gradients.  All sums in float32.
//     h = x + residual,  r = 1 / sqrt(mean(h^2) + eps),  y = h r w          int8: codes and scale of h w (int8_rows.h), the scale times r: r is the same for a row and changes no code
//     g = dy w,  u = h r,  dx = r (g - u mean(g u)) + dx_add,  dw = sum over the rows of dy u
// Bound by HBM bandwidth: every tensor is moved once, a row stays in its workgroup's registers between its sum and its result.
#include "int8_rows.h"
#include "kernels.h"
#include "row_pieces.h"

namespace skiparse {

constexpr uint32_t NORM_WAVES = 16;  // of a workgroup, at most
constexpr int NORM_CH = 4;           // pieces of 8 channels of a lane
static_assert(NORM_WAVES * 64 * NORM_CH * 8 == NORM_MAX_COLS, "a row is in registers");

// Sums over a workgroup, the same in every lane, in an order that depends on nothing.
template <int N>
struct Together {
    float v[NORM_WAVES][N];
    double d[NORM_WAVES][N];
};
template <typename S>
__device__ inline S wave_sum(S v) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
    return v;
}
template <typename S, int N>
__device__ inline void group_sum(S (&v)[N], S (*all)[N]) {
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = wave_sum(v[i]);
    const uint32_t waves = blockDim.x >> 6;
    if (waves == 1u) return;
    __syncthreads();  // what was there has been read
    if ((threadIdx.x & 63u) == 0u) {
#pragma unroll
        for (int i = 0; i < N; i++) all[threadIdx.x >> 6][i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; i++) {
        v[i] = all[0][i];
        for (uint32_t w = 1; w < waves; w++) v[i] += all[w][i];
    }
}
__device__ inline uint32_t group_max(uint32_t v, float (*all)[1]) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
        const uint32_t o = (uint32_t)__shfl_xor((int)v, off);
        v = o > v ? o : v;
    }
    const uint32_t waves = blockDim.x >> 6;
    if (waves == 1u) return v;
    __syncthreads();
    if ((threadIdx.x & 63u) == 0u) all[threadIdx.x >> 6][0] = __uint_as_float(v);
    __syncthreads();
    for (uint32_t w = 0; w < waves; w++) {
        const uint32_t o = __float_as_uint(all[w][0]);
        v = o > v ? o : v;
    }
    return v;
}

// Squares of values beyond 2^63 or so are infinite in float32, and those below 2^-63 lose digits: a row whose sum says so is summed again in 64 bits.
__device__ inline bool out_of_range(float squares, float per_n, float eps) { return !(squares <= 1e38f) || squares * per_n + eps < 1e-30f; }
__device__ inline float inverse_size(float squares, float per_n, float eps) { return 1.f / sqrtf(squares * per_n + eps); }

template <typename T, int KIND>
__global__ __launch_bounds__(64 * NORM_WAVES) void norm_rows_kernel(NormArgs a) {
    __shared__ Together<1> all;
    const uint32_t row = a.first + blockIdx.x;
    const uint32_t from = a.order == 1 ? source_row<TO_SPARSE>(a.rows, row, 0u) : a.order == 2 ? source_row<TO_ORIGINAL>(a.rows, row, 0u) : row;
    const size_t at = (size_t)from * a.cols, to = (size_t)row * a.cols;
    float h[NORM_CH][8];
    float sum[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NORM_CH; i++) {
        const uint32_t c = (threadIdx.x + i * blockDim.x) * 8u;
#pragma unroll
        for (int e = 0; e < 8; e++) h[i][e] = 0.f;
        if (c >= a.cols) continue;
        const Piece<T> x = load_piece<T>(a.x, at + c);
#pragma unroll
        for (int e = 0; e < 8; e++) h[i][e] = x.get(e);
        if (a.residual != nullptr) {
            const Piece<T> r = load_piece<T>(a.residual, at + c);
#pragma unroll
            for (int e = 0; e < 8; e++) h[i][e] += r.get(e);
        }
        if (a.sum != nullptr) {
            Piece<T> s;
            s.set(h[i]);
            store_piece<T>(a.sum, at + c, s);
        }
#pragma unroll
        for (int e = 0; e < 8; e++) sum[0] += h[i][e] * h[i][e];
    }
    float r = 1.f;
    if (KIND != ROWS_QUANTIZED) {
        group_sum(sum, all.v);
        r = inverse_size(sum[0], a.per_n, a.eps);
        if (out_of_range(sum[0], a.per_n, a.eps)) {
            double d[1] = {0.};
#pragma unroll
            for (int i = 0; i < NORM_CH; i++)
#pragma unroll
                for (int e = 0; e < 8; e++) d[0] += (double)h[i][e] * h[i][e];
            group_sum(d, all.d);
            r = (float)(1. / sqrt(d[0] / a.cols + a.eps));
        }
    }
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < NORM_CH; i++) {
        const uint32_t c = (threadIdx.x + i * blockDim.x) * 8u;
        if (KIND == ROWS_NORM) {
#pragma unroll
            for (int e = 0; e < 8; e++) h[i][e] *= r;
        }
        if (c < a.cols && KIND != ROWS_QUANTIZED && a.weight != nullptr) {
            const Piece<T> w = load_piece<T>(a.weight, c);
#pragma unroll
            for (int e = 0; e < 8; e++) h[i][e] *= w.get(e);
        }
        if (KIND == ROWS_NORM && c < a.cols) {
            Piece<T> y;
            y.set(h[i]);
            store_piece<T>(a.out, to + c, y);
        }
#pragma unroll
        for (int e = 0; e < 8; e++) top = int8_size(h[i][e]) > top ? int8_size(h[i][e]) : top;
    }
    if (KIND == ROWS_NORM) return;
    const Int8Row q(group_max(top, all.v), r);
#pragma unroll
    for (int i = 0; i < NORM_CH; i++) {
        const uint32_t c = (threadIdx.x + i * blockDim.x) * 8u;
        if (c < a.cols)
            *(piece_u32x2*)((char*)a.out + to + c) = piece_u32x2{q.codes(h[i][0], h[i][1], h[i][2], h[i][3]), q.codes(h[i][4], h[i][5], h[i][6], h[i][7])};
    }
    if (threadIdx.x == 0u) a.scales[row] = q.scale;
}

template <typename T>
static void launch_rows_t(const NormArgs& a, uint32_t blocks, uint32_t threads, hipStream_t stream) {
    switch (a.kind) {
        case ROWS_NORM: norm_rows_kernel<T, ROWS_NORM><<<blocks, threads, 0, stream>>>(a); break;
        case ROWS_NORM_QUANTIZED: norm_rows_kernel<T, ROWS_NORM_QUANTIZED><<<blocks, threads, 0, stream>>>(a); break;
        default: norm_rows_kernel<T, ROWS_QUANTIZED><<<blocks, threads, 0, stream>>>(a); break;
    }
}

static uint32_t threads_of(uint32_t cols) {
    const uint32_t waves = (cols / 8u + 63u) / 64u;
    return 64u * (waves < NORM_WAVES ? waves : NORM_WAVES);
}

hipError_t launch_norm_rows(const NormArgs& all, hipStream_t stream) {
    const uint32_t threads = threads_of(all.cols);
    NormArgs a = all;
    a.per_n = 1.f / (float)a.cols;
    constexpr uint32_t AT_ONCE = 1u << 21;  // a grid has less than 2^32 threads
    for (a.first = 0; a.first < a.n_rows; a.first += AT_ONCE) {
        const uint32_t n = a.n_rows - a.first < AT_ONCE ? a.n_rows - a.first : AT_ONCE;
        if (a.f32) launch_rows_t<float>(a, n, threads, stream);
        else launch_rows_t<__bf16>(a, n, threads, stream);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// ---- gradients

uint32_t norm_bwd_parts(uint32_t rows, uint32_t) { return rows < 512u ? rows : 512u; }

// A workgroup takes a contiguous part of the rows, and has the sums of its part for the weights' gradient.
template <typename T>
__global__ __launch_bounds__(64 * NORM_WAVES) void norm_bwd_kernel(NormBwdArgs a) {
    __shared__ Together<2> all;
    const uint32_t first = (uint32_t)((uint64_t)blockIdx.x * a.n_rows / gridDim.x), end = (uint32_t)((uint64_t)(blockIdx.x + 1u) * a.n_rows / gridDim.x);
    float dw[NORM_CH][8] = {};
    for (uint32_t row = first; row < end; row++) {
        const uint32_t from = a.order == 1 ? source_row<TO_SPARSE>(a.rows, row, 0u) : a.order == 2 ? source_row<TO_ORIGINAL>(a.rows, row, 0u) : row;
        const size_t at = (size_t)row * a.cols, in = (size_t)from * a.cols;
        float h[NORM_CH][8], g[NORM_CH][8], sum[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NORM_CH; i++) {
            const uint32_t c = (threadIdx.x + i * blockDim.x) * 8u;
#pragma unroll
            for (int e = 0; e < 8; e++) h[i][e] = g[i][e] = 0.f;
            if (c >= a.cols) continue;
            const Piece<T> x = load_piece<T>(a.h, at + c), y = load_piece<T>(a.dy, in + c);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                h[i][e] = x.get(e);
                g[i][e] = y.get(e);
            }
        }
        auto weight = [&](int i, float (&w)[8]) __attribute__((always_inline)) {
            const uint32_t c = (threadIdx.x + i * blockDim.x) * 8u;
#pragma unroll
            for (int e = 0; e < 8; e++) w[e] = 1.f;
            if (a.weight == nullptr || c >= a.cols) return;
            const Piece<T> p = load_piece<T>(a.weight, c);
#pragma unroll
            for (int e = 0; e < 8; e++) w[e] = p.get(e);
        };
#pragma unroll
        for (int i = 0; i < NORM_CH; i++) {
            float w[8];
            weight(i, w);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                sum[0] += h[i][e] * h[i][e];
                sum[1] += g[i][e] * w[e] * h[i][e];
            }
        }
        group_sum(sum, all.v);
        float r = inverse_size(sum[0], a.per_n, a.eps), mean = sum[1] * a.per_n * r;
        if (out_of_range(sum[0], a.per_n, a.eps) || !(fabsf(sum[1]) <= 1e38f)) {
            double d[2] = {0., 0.};
#pragma unroll
            for (int i = 0; i < NORM_CH; i++) {
                float w[8];
                weight(i, w);
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    d[0] += (double)h[i][e] * h[i][e];
                    d[1] += (double)g[i][e] * w[e] * h[i][e];
                }
            }
            group_sum(d, all.d);
            const double s = 1. / sqrt(d[0] / a.cols + a.eps);
            r = (float)s;
            mean = (float)(d[1] / a.cols * s);
        }
#pragma unroll
        for (int i = 0; i < NORM_CH; i++) {
            const uint32_t c = (threadIdx.x + i * blockDim.x) * 8u;
            float w[8];
            weight(i, w);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float u = h[i][e] * r;
                dw[i][e] += g[i][e] * u;
                g[i][e] = r * (g[i][e] * w[e] - u * mean);
            }
            if (c >= a.cols || a.dx == nullptr) continue;
            if (a.dx_add != nullptr) {
                const Piece<T> p = load_piece<T>(a.dx_add, at + c);
#pragma unroll
                for (int e = 0; e < 8; e++) g[i][e] += p.get(e);
            }
            Piece<T> y;
            y.set(g[i]);
            store_piece<T>(a.dx, at + c, y);
        }
    }
    if (a.dw == nullptr) return;
#pragma unroll
    for (int i = 0; i < NORM_CH; i++) {
        const uint32_t c = (threadIdx.x + i * blockDim.x) * 8u;
        if (c >= a.cols) continue;
        Piece<float> p;
        p.set(dw[i]);
        store_piece<float>(a.parts, (size_t)blockIdx.x * a.cols + c, p);
    }
}

// The parts' sums, 64 channels a workgroup, 16 parts at a time, in an order that depends on nothing.
template <typename T>
__global__ __launch_bounds__(1024) void norm_dw_kernel(const float* __restrict__ part, T* __restrict__ dw, uint32_t parts, uint32_t cols) {
    __shared__ float sums[16][64];
    const uint32_t lane = threadIdx.x & 63u, ty = threadIdx.x >> 6, n = blockIdx.x * 64u + lane;
    float s = 0.f;
    if (n < cols) {
#pragma unroll 8
        for (uint32_t p = ty; p < parts; p += 16u) s += part[(size_t)p * cols + n];
    }
    sums[ty][lane] = s;
    __syncthreads();
    if (ty != 0u || n >= cols) return;
    s = 0.f;
#pragma unroll
    for (uint32_t i = 0; i < 16u; i++) s += sums[i][lane];
    dw[n] = (T)s;
}

hipError_t launch_norm_bwd(const NormBwdArgs& all, hipStream_t stream) {
    NormBwdArgs a = all;
    a.per_n = 1.f / (float)a.cols;
    const uint32_t parts = norm_bwd_parts(a.n_rows, a.cols), threads = threads_of(a.cols);
    if (a.f32) norm_bwd_kernel<float><<<parts, threads, 0, stream>>>(a);
    else norm_bwd_kernel<__bf16><<<parts, threads, 0, stream>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.dw == nullptr) return e;
    const uint32_t blocks = (a.cols + 63u) / 64u;
    if (a.f32) norm_dw_kernel<float><<<blocks, 1024, 0, stream>>>(a.parts, (float*)a.dw, parts, a.cols);
    else norm_dw_kernel<__bf16><<<blocks, 1024, 0, stream>>>(a.parts, (__bf16*)a.dw, parts, a.cols);
    return hipGetLastError();
}

}  // namespace skiparse

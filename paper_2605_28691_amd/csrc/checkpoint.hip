// 8-bit activation checkpoints (format: checkpoint.h): what a training step keeps of a bf16 or float32 tensor until its backward pass, in 33 / 64 of the
// bytes of bf16.  Bound by HBM bandwidth.  A lane has 8 channels, four lanes a block, whose maximum takes two exchanges between neighbours.
// (80,640 x 5120 of bf16, 1.25 GB: saved in 206 us, loaded in 203, 6.1 TB/s.)
#include "checkpoint.h"
#include "kernels.h"

namespace skiparse {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;

constexpr int CKPT_THREADS = 256;
// Pieces of 8 channels that a lane saves: few in flight are best but for large tensors (us, 1 / 2 / 4 a lane: 6426 x 1000 in float32 7.1 / 7.2 / 8.5, 3840 x 5120 in bf16 11.6 / 12.2 /
// 14.1, 32,760 x 1536 30.4 / 29.7 / 34.4, 80,640 x 5120 216 / 201 / 213).  A lane loads one (32,760 x 1536 28.0 / 29.3 / 31.3).
constexpr uint64_t CKPT_TWO = 1ull << 22;  // from this many pieces on, two a lane

struct CkptArgs {
    uint64_t first;    // piece that a launch begins with
    uint64_t pieces;   // 8-channel places of all rows, those behind the end of a short last block included
    Div32 per_row;     // of a row: 4 * blocks
    uint32_t cols;
};

// Where piece i lies: element offset and block; false: behind the row's end.  !RAGGED: rows are whole blocks, so that the tensor is one run of them.
template <bool RAGGED>
__device__ inline bool piece_at(const CkptArgs& a, uint64_t i, uint64_t& elem, uint64_t& block) {
    block = i >> 2;
    elem = i * 8u;
    if (!RAGGED) return true;
    const uint64_t row = a.pieces >> 32 ? i / a.per_row.d : a.per_row.div((uint32_t)i);  // the same way for the whole launch
    const uint32_t c = (uint32_t)(i - row * a.per_row.d) * 8u;
    elem = row * a.cols + c;
    return c < a.cols;
}

template <typename T>
__device__ inline void load8(const T* p, float (&v)[8]);
template <>
__device__ inline void load8<__bf16>(const __bf16* p, float (&v)[8]) {
    const u32x4 x = *(const u32x4*)p;
#pragma unroll
    for (int e = 0; e < 4; e++) {
        v[2 * e] = __uint_as_float(x[e] << 16);
        v[2 * e + 1] = __uint_as_float(x[e] & 0xffff0000u);
    }
}
template <>
__device__ inline void load8<float>(const float* p, float (&v)[8]) {
    const u32x4 x = *(const u32x4*)p, y = *(const u32x4*)(p + 4);
#pragma unroll
    for (int e = 0; e < 4; e++) {
        v[e] = __uint_as_float(x[e]);
        v[4 + e] = __uint_as_float(y[e]);
    }
}
__device__ inline void store8(__bf16* p, const float (&v)[8]) {
    typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
    bf16x8 y;
#pragma unroll
    for (int e = 0; e < 8; e++) y[e] = (__bf16)v[e];
    *(bf16x8*)p = y;
}
__device__ inline void store8(float* p, const float (&v)[8]) {
    typedef __attribute__((ext_vector_type(4))) float f32x4;
    *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]};
    *(f32x4*)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}

template <typename T, bool RAGGED, int UNROLL>
__global__ __launch_bounds__(CKPT_THREADS) void checkpoint_save_kernel(const T* __restrict__ x, unsigned char* __restrict__ codes, unsigned char* __restrict__ scales, CkptArgs a) {
    const uint64_t first = a.first + (uint64_t)blockIdx.x * (CKPT_THREADS * UNROLL) + threadIdx.x;
    float v[UNROLL][8];
    uint64_t elem[UNROLL], block[UNROLL];
    bool real[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; u++) {
        const uint64_t i = first + u * CKPT_THREADS;
        real[u] = i < a.pieces && piece_at<RAGGED>(a, i, elem[u], block[u]);
#pragma unroll
        for (int e = 0; e < 8; e++) v[u][e] = 0.f;
        if (real[u]) load8(x + elem[u], v[u]);
    }
#pragma unroll
    for (int u = 0; u < UNROLL; u++) {
        uint32_t m = 0u;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const uint32_t s = ckpt_size(v[u][e]);
            m = s > m ? s : m;
        }
#pragma unroll
        for (int off = 1; off <= 2; off <<= 1) {  // a block's four lanes are neighbours: pieces of a row come in fours
            const uint32_t o = (uint32_t)__shfl_xor((int)m, off);
            m = o > m ? o : m;
        }
        const uint32_t byte = ckpt_byte(m);
        const float down = ckpt_down(byte);
        if (real[u]) {
            *(u32x2*)(codes + elem[u]) = u32x2{ckpt_codes(v[u][0], v[u][1], v[u][2], v[u][3], down), ckpt_codes(v[u][4], v[u][5], v[u][6], v[u][7], down)};
            if ((threadIdx.x & 3u) == 0u) scales[block[u]] = (unsigned char)byte;
        }
    }
}

template <typename T, bool RAGGED>
__global__ __launch_bounds__(CKPT_THREADS) void checkpoint_load_kernel(const unsigned char* __restrict__ codes, const unsigned char* __restrict__ scales, T* __restrict__ out, CkptArgs a) {
    const uint64_t i = a.first + (uint64_t)blockIdx.x * CKPT_THREADS + threadIdx.x;
    uint64_t elem, block;
    if (i >= a.pieces || !piece_at<RAGGED>(a, i, elem, block)) return;
    const u32x2 c = *(const u32x2*)(codes + elem);
    const float up = ckpt_up(scales[block]);
    float lo[4], hi[4];
    ckpt_values(c[0], up, lo);
    ckpt_values(c[1], up, hi);
    const float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    store8(out + elem, v);
}

static CkptArgs make_args(uint32_t rows, uint32_t cols) {
    const uint32_t blocks = (cols + CKPT_BLOCK - 1u) / CKPT_BLOCK;
    return {0u, (uint64_t)rows * blocks * 4u, make_div32(blocks * 4u), cols};
}

// f(arguments, workgroups of `each` pieces) for every launch: a grid has less than 2^32 threads
template <typename F>
static hipError_t in_launches(CkptArgs a, uint64_t each, F f) {
    constexpr uint64_t AT_ONCE = 1ull << 31;
    for (; a.first < a.pieces; a.first += AT_ONCE) {
        const uint64_t left = a.pieces - a.first, n = left < AT_ONCE ? left : AT_ONCE;
        f(a, (uint32_t)((n + each - 1) / each));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, bool RAGGED>
static hipError_t save_t(const void* x, void* codes, void* scales, const CkptArgs& all, hipStream_t stream) {
    const bool two = all.pieces >= CKPT_TWO;
    return in_launches(all, two ? 2 * CKPT_THREADS : CKPT_THREADS, [&](const CkptArgs& a, uint32_t blocks) {
        if (two) checkpoint_save_kernel<T, RAGGED, 2><<<blocks, CKPT_THREADS, 0, stream>>>((const T*)x, (unsigned char*)codes, (unsigned char*)scales, a);
        else checkpoint_save_kernel<T, RAGGED, 1><<<blocks, CKPT_THREADS, 0, stream>>>((const T*)x, (unsigned char*)codes, (unsigned char*)scales, a);
    });
}
template <typename T>
static hipError_t load_t(const void* codes, const void* scales, void* out, const CkptArgs& all, hipStream_t stream) {
    return in_launches(all, CKPT_THREADS, [&](const CkptArgs& a, uint32_t blocks) {
        if (a.cols % CKPT_BLOCK) checkpoint_load_kernel<T, true><<<blocks, CKPT_THREADS, 0, stream>>>((const unsigned char*)codes, (const unsigned char*)scales, (T*)out, a);
        else checkpoint_load_kernel<T, false><<<blocks, CKPT_THREADS, 0, stream>>>((const unsigned char*)codes, (const unsigned char*)scales, (T*)out, a);
    });
}

hipError_t launch_checkpoint_save(const void* x, void* codes, void* scales, uint32_t rows, uint32_t cols, bool f32, hipStream_t stream) {
    const CkptArgs a = make_args(rows, cols);
    if (cols % CKPT_BLOCK) return f32 ? save_t<float, true>(x, codes, scales, a, stream) : save_t<__bf16, true>(x, codes, scales, a, stream);
    return f32 ? save_t<float, false>(x, codes, scales, a, stream) : save_t<__bf16, false>(x, codes, scales, a, stream);
}

hipError_t launch_checkpoint_load(const void* codes, const void* scales, void* out, uint32_t rows, uint32_t cols, bool f32, hipStream_t stream) {
    const CkptArgs a = make_args(rows, cols);
    return f32 ? load_t<float>(codes, scales, out, a, stream) : load_t<__bf16>(codes, scales, out, a, stream);
}

}  // namespace skiparse

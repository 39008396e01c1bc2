// Eight channels of a row as a lane of the passes over rows has them: 16 bytes of bf16, or twice 16 bytes of float32.  An instruction moves 16 bytes a lane, neighbours' next to each other, so that lines are moved
// as a whole: a lane's two halves in float32 lie apart by all the lanes' first halves.  (32 bytes a lane in one place: 6426 x 4008 with residual 79.5 us, and 89.7 past the caches; so 75.8.)
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace skiparse {

typedef __attribute__((ext_vector_type(4))) unsigned int piece_u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int piece_u32x2;

template <typename T>
struct Piece;
template <>
struct Piece<__bf16> {
    static constexpr int UNITS = 1, EACH = 8;  // instructions that move it, channels of one
    piece_u32x4 raw[1];
    __device__ inline float get(int e) const { return __uint_as_float(e & 1 ? raw[0][e >> 1] & 0xffff0000u : raw[0][e >> 1] << 16); }
    __device__ inline void set(const float (&v)[8]) {
        typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
        bf16x8 y;
#pragma unroll
        for (int e = 0; e < 8; e++) y[e] = (__bf16)v[e];
        raw[0] = __builtin_bit_cast(piece_u32x4, y);
    }
};
template <>
struct Piece<float> {
    static constexpr int UNITS = 2, EACH = 4;
    piece_u32x4 raw[2];
    __device__ inline float get(int e) const { return __uint_as_float(raw[e >> 2][e & 3]); }
    __device__ inline void set(const float (&v)[8]) {
#pragma unroll
        for (int e = 0; e < 8; e++) raw[e >> 2][e & 3] = __float_as_uint(v[e]);
    }
};

// NT: past the caches, for tensors that they do not hold until the next pass
template <bool NT>
__device__ __attribute__((always_inline)) inline piece_u32x4 load16(const void* p) {
    return NT ? __builtin_nontemporal_load((const piece_u32x4*)p) : *(const piece_u32x4*)p;
}
template <bool NT>
__device__ __attribute__((always_inline)) inline void store16(void* p, piece_u32x4 v) {
    if (NT) __builtin_nontemporal_store(v, (piece_u32x4*)p);
    else *(piece_u32x4*)p = v;
}

}  // namespace skiparse

// Eight channels of a row as they lie in memory, bf16 or float32: what a lane moves at once in the passes over rows.
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
    piece_u32x4 raw[2];
    __device__ inline float get(int e) const { return __uint_as_float(raw[e >> 2][e & 3]); }
    __device__ inline void set(const float (&v)[8]) {
#pragma unroll
        for (int e = 0; e < 8; e++) raw[e >> 2][e & 3] = __float_as_uint(v[e]);
    }
};

// `at`: in elements
template <typename T>
__device__ inline Piece<T> load_piece(const void* from, size_t at) {
    Piece<T> p;
    const piece_u32x4* const q = (const piece_u32x4*)((const T*)from + at);
#pragma unroll
    for (unsigned i = 0; i < sizeof(p.raw) / 16; i++) p.raw[i] = q[i];
    return p;
}
template <typename T>
__device__ inline void store_piece(void* to, size_t at, const Piece<T>& p) {
    piece_u32x4* const q = (piece_u32x4*)((T*)to + at);
#pragma unroll
    for (unsigned i = 0; i < sizeof(p.raw) / 16; i++) q[i] = p.raw[i];
}

}  // namespace skiparse

// Format of an 8-bit activation checkpoint: blocks of 32 consecutive channels of a row, one E4M3 code a value and one exponent byte a block.
//     a = largest finite |x| of the block,  e = smallest integer with a <= 448 * 2^e,  code = rne(x * 2^-e),  byte = e + 127
// Beyond 248 * 2^120 (3.30e38) a finite x rounds to 2^128, which is infinity in both types: as any rounding to fewer bits next to the largest number.
// A power of two as scale costs no precision (a float's rounding error is relative), makes the scaling exact in both directions and takes a byte where a
// float would take four; a block is what four lanes of an accumulator hold of a row (linear.hip), so that a product's epilogue can write one.
// Blocks of nothing but zeros have byte 127.  A value that is not finite gets a NaN code and does not enter the maximum.  The last block of a row whose length is
// no multiple of 32 is shorter.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace skiparse {

constexpr uint32_t CKPT_BLOCK = 32;

typedef __attribute__((ext_vector_type(2))) float ckpt_f32x2;

// |x| as the bits of its float, 0 if it is not finite: comparable as integers
__device__ inline uint32_t ckpt_size(float x) {
    const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
}
// 448 = 1.75 * 2^8: a larger mantissa needs the next power of two
__host__ __device__ inline uint32_t ckpt_byte(uint32_t a) {
    const int e = (int)((a + 0x1fffffu) >> 23) - 8;
    return a == 0u ? 127u : e > 0 ? (uint32_t)e : 0u;
}
// 2^(127 - byte); byte <= 247
__device__ inline float ckpt_down(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
// 2^(byte - 127); 255 stands for NaN
__device__ inline float ckpt_up(uint32_t byte) { return __uint_as_float(byte == 0u ? 0x00400000u : byte == 255u ? 0x7fc00000u : byte << 23); }

__device__ inline float ckpt_scaled(float x, float down) { return ckpt_size(x) != 0u || x == 0.f ? x * down : __uint_as_float(0x7fc00000u); }
// four codes of values that are scaled, and finite or NaN
__device__ inline uint32_t ckpt_codes_of(float a, float b, float c, float d) {
    int u = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    u = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, u, true);
    return (uint32_t)u;
}
__device__ inline uint32_t ckpt_codes(float a, float b, float c, float d, float down) {
    return ckpt_codes_of(ckpt_scaled(a, down), ckpt_scaled(b, down), ckpt_scaled(c, down), ckpt_scaled(d, down));
}
__device__ inline void ckpt_values(uint32_t codes, float up, float (&v)[4]) {
    const ckpt_f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    v[0] = lo[0] * up;
    v[1] = lo[1] * up;
    v[2] = hi[0] * up;
    v[3] = hi[1] * up;
}

}  // namespace skiparse

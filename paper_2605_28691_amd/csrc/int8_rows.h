// Rows in 8-bit integers: one code a value and one float32 scale a row.
//     m = largest |v| of the row, at least 2^-118,  code = rne(v * (127 / m)),  scale = m / 127        value = code * scale
// All in float32.  127 / m is finite and scale no denormal number then.  A row of zeros has scale 1.  A row that holds a value that is not finite has codes 0 and scale NaN, so that
// whatever is made of it is not a number either.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace skiparse {

constexpr uint32_t INT8_LEAST = 0x04800000u;  // 2^-118
constexpr uint32_t INT8_INFINITE = 0x7f800000u;

// |v| as the bits of its float: comparable as integers, with infinity above all numbers and NaN above infinity
__device__ inline uint32_t int8_size(float v) { return __float_as_uint(v) & 0x7fffffffu; }

struct Int8Row {
    float up;       // 127 / m; 0 where all codes are 0
    float scale;
    // top: the largest int8_size of the row; by: what the scale is multiplied by
    __device__ inline Int8Row(uint32_t top, float by) {
        const float m = __uint_as_float(top < INT8_LEAST ? INT8_LEAST : top);
        const bool finite = top < INT8_INFINITE;
        up = finite ? 127.f / m : 0.f;
        scale = !finite ? __uint_as_float(0x7fc00000u) : top == 0u ? 1.f : m / 127.f * by;
    }
    // Four codes.  |v| up <= 127 (1 + 2^-22), so 1.5 * 2^23 + v up has its last bit at 1: the sum rounds to the nearest, and its low byte is the code.  The product is rounded
    // first, as the definition has it: no fused multiply-add.
    __device__ inline uint32_t codes(float a, float b, float c, float d) const {
#pragma clang fp contract(off)
        if (up == 0.f) return 0u;
        constexpr float MAGIC = 12582912.f;
        const float x = a * up, y = b * up, z = c * up, w = d * up;
        const uint32_t i = __float_as_uint(x + MAGIC), j = __float_as_uint(y + MAGIC), k = __float_as_uint(z + MAGIC), l = __float_as_uint(w + MAGIC);
        return __builtin_amdgcn_perm(__builtin_amdgcn_perm(l, k, 0x0c0c0400u), __builtin_amdgcn_perm(j, i, 0x0c0c0400u), 0x05040100u);
    }
};

}  // namespace skiparse

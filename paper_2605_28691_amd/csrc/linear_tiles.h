// The products of the linear layer on the matrix cores, bf16 or in 8-bit integers, and their way out: what linear.hip and linear_int8.hip make their kernels of.
#pragma once
#include <type_traits>
#include <utility>

#include "checkpoint.h"
#include "kernels.h"
#include "lds_layout.h"
#include "linear_act.h"
#include "linear_plan.h"

namespace skiparse {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) int i32x4;

#define LDS_PTR(T) __attribute__((address_space(3))) T*

constexpr uint32_t LIN_KT = 64;           // of k a step
constexpr uint32_t LIN_OUTSIDE = ~0u;     // an offset outside every buffer
constexpr uint32_t LIN_RECORDS = 0xfffffff0u;

// Where 16-byte chunk c of row r of an operand in one piece lies: at c ^ row_swizzle(r).  A read of 16 bytes a lane is served 16 lanes at a time, 0-3, 12-15 and 20-27, then 4-11,
// 16-19 and 28-31, and the same of the upper half: of a fragment rows 0-3 and 12-15 of one chunk with rows 4-11 of its neighbour, or the other way round; these touch every bank
// once.  (With the attention's swizzle, for 32 rows of a chunk, half of the reads' clocks were conflicts.)
__host__ __device__ constexpr uint32_t row_swizzle(uint32_t r) { return r >> 1 & 7u; }

// One operand's side of a workgroup's tile: ROWS of m (or n).
//   !T: a step, 64 of k, in one piece: rows of 128 bytes, whole lines of the caches (64 bytes of a line at a time, 8192^3 took 900 us instead of 846)
//    T: halves of 32 rows of k, COLS columns each, which are free and filled again one after the other
template <int ROWS, bool T, int NW>
struct Side {
    static constexpr uint32_t COLS = ROWS < 128 ? 64 : 128, LANES = COLS / 8;  // of a row of k in LDS: columns, lanes that fetch it
    static constexpr int INSTR = ROWS * (T ? 64 : 128) / 1024 / NW;  // direct loads of a wavefront and piece, 1 KiB each
    static constexpr int BYTES = ROWS * (T ? 64 : 128);
    uint32_t off[INSTR];   // of the lane's chunk from the piece's base
    uint32_t kofs[INSTR];  // !T: where in the step's k it lies
    // row_off: byte offset of row r of the tile from the base (!T), row_bytes: of a row of k (T)
    template <typename F>
    __device__ __attribute__((always_inline)) inline void init(uint32_t wave, uint32_t lane, uint32_t row_bytes, F row_off) {
#pragma unroll
        for (int i = 0; i < INSTR; i++) {
            const uint32_t n = wave * INSTR + i;  // of the tile's
            if (!T) {
                const uint32_t r = n * 8u + lane / 8u;
                kofs[i] = ((lane % 8u) ^ row_swizzle(r)) * 8u;
                off[i] = row_off(r) + kofs[i] * 2u;
            } else {
                constexpr uint32_t PER = 64 / LANES;  // rows at once
                const uint32_t part = n / (32u / PER), r = n % (32u / PER) * PER + lane / LANES;
                kofs[i] = 0u;
                off[i] = r * row_bytes + part * (COLS * 2u) + ((lane % LANES) ^ lds_swizzle<COLS>(r)) * 16u;
            }
        }
    }
    __device__ __attribute__((always_inline)) inline void issue(int i, const char* base, uint32_t records, uint32_t k_left, char* buf, uint32_t wave) const {
#if defined(__HIP_DEVICE_COMPILE__)  // the host pass does not know the buffer's type, and would drop the kernel without a word
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, records, 0x27000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (LDS_PTR(void))(buf + (wave * INSTR + i) * 1024u), 16, T || kofs[i] < k_left ? off[i] : LIN_OUTSIDE, 0, 0, 0);
#endif
    }
};

// Fragment of 16 rows from `row0` (a multiple of 16) and 32 of k, the step's half `half`: lane l has row l % 16, k = 8 (l / 16) ...  T: `buf` is the half.
template <bool T, uint32_t COLS>
__device__ __attribute__((always_inline)) inline bf16x8 read_fragment(const char* buf, uint32_t row0, uint32_t half, uint32_t lane) {
    const uint32_t li = lane & 15u, g = lane >> 4;
    if (!T) return *(const bf16x8*)(buf + (row0 + li) * 128u + ((4u * half + g) ^ row_swizzle(li)) * 16u);
    const char* const part = buf + row0 / COLS * (COLS * 64u);
    bf16x4 v[2];
#pragma unroll
    for (uint32_t sec = 0; sec < 2; sec++) {
        const uint32_t r = 8u * g + 4u * sec + (li >> 2);
        const uint32_t c = row0 % COLS / 8u + ((li & 3u) >> 1);
        const char* const at = part + r * (COLS * 2u) + ((c ^ lds_swizzle<COLS>(r)) * 16u) + 8u * (li & 1u);
        v[sec] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(LDS_PTR(char))at);
    }
    return __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
}

// Exchange of the odd rows of 16 lanes of `a` with the even ones of `b` (v_permlane16_swap; its own inverse).
__device__ __attribute__((always_inline)) inline void swap_rows(uint32_t& a, uint32_t& b) {
    const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    const uint32_t x = r[0], y = r[1];
    a = x;
    b = y;
}

// What becomes of a whole sum of 8-bit products: the same operations in every kernel, so that a row's bits do not depend on which one has it.
__device__ __attribute__((always_inline)) inline float int8_value(int sum, float x_scale, float w_scale, float bias) {
#pragma clang fp contract(off)
    return fmaf((float)sum * x_scale, w_scale, bias);
}
// A sum is below 2^31, so from scales of 2^97 on its product with a row's could leave float32's range where that with the channel's scale as well does not.  Rows of 2^64 and more have theirs times 2^-32, the
// channels' times 2^32 then: powers of two, so no rounding changes.  A channel's that leaves the range by that is kept at its end, since a sum of 0 is 0 times it; all others are infinite either way.
__device__ __attribute__((always_inline)) inline bool int8_far(float x_scale) { return fabsf(x_scale) >= 0x1p64f; }
__device__ __attribute__((always_inline)) inline float int8_value_far(int sum, float x_scale, float w_scale, float bias) {
    const bool far = int8_far(x_scale);
    float up = w_scale * 0x1p32f;
    if (__builtin_isinf(up) && !__builtin_isinf(w_scale)) up = copysignf(3.4028234663852886e38f, w_scale);
    return int8_value(sum, far ? x_scale * 0x1p-32f : x_scale, far ? up : w_scale, bias);
}
__device__ __attribute__((always_inline)) inline float int8_plus(float z, float residual) {
#pragma clang fp contract(off)
    return z + residual;
}

// Scales and bias of a wavefront's share of a product in 8-bit integers: lane l holds those of its rows l and 64 + l, and of its channels.
template <int FM, int FN, bool INT8>
struct Scales {
    __device__ __attribute__((always_inline)) inline Scales(const LinearArgs&, uint32_t, uint32_t, uint32_t) {}
};
template <int FM, int FN>
struct Scales<FM, FN, true> {
    static constexpr int ROWS = (FM + 3) / 4, COLS = (FN + 3) / 4;
    float x[ROWS], w[COLS], bias[COLS];
    __device__ __attribute__((always_inline)) inline Scales(const LinearArgs& a, uint32_t m0, uint32_t n0, uint32_t lane) {
#pragma unroll
        for (int r = 0; r < ROWS; r++) {
            uint32_t m = m0 + 64u * r + lane;
            m = m < a.M ? m : a.M - 1u;
            if (a.order != 0) m = a.order == 1 ? source_row<TO_SPARSE>(a.rows, m, 0u) : source_row<TO_ORIGINAL>(a.rows, m, 0u);
            x[r] = a.x_scales[m];
        }
#pragma unroll
        for (int r = 0; r < COLS; r++) {
            uint32_t n = n0 + 64u * r + lane;
            n = n < a.N ? n : a.N - 1u;  // channels behind the last are not stored
            w[r] = a.w_scales[n];
            bias[r] = a.e.bias != nullptr ? (float)((const __bf16*)a.e.bias)[n] : 0.f;
        }
    }
    // of row 16 i + lane % 16
    __device__ __attribute__((always_inline)) inline float row(int i, uint32_t lane) const { return __shfl(x[i / 4], (i % 4) * 16 + (int)(lane & 15u)); }
    // of the lane's channels of block j, as they lie in the accumulators
    struct Channels {
        f32x4 w[FN], bias[FN];
    };
    __device__ __attribute__((always_inline)) inline Channels channels(uint32_t lane) const {
        Channels c;
#pragma unroll
        for (int j = 0; j < FN; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const int from = (j % 4) * 16 + 4 * (int)(lane >> 4) + e;
                c.w[j][e] = __shfl(w[j / 4], from);
                c.bias[j][e] = __shfl(bias[j / 4], from);
            }
        return c;
    }
    // sums of the lane's row -> z, in their place
    __device__ __attribute__((always_inline)) inline static void values(f32x4 (&z)[FN], float x_scale, const Channels& c) {
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(int8_far(x_scale)) != 0, 0)) {
            values<true>(z, x_scale, c);
            return;
        }
        values<false>(z, x_scale, c);
    }
    template <bool FAR>
    __device__ __attribute__((always_inline)) inline static void values(f32x4 (&z)[FN], float x_scale, const Channels& c) {
#pragma unroll
        for (int j = 0; j < FN; j++) {
            const i32x4 s = __builtin_bit_cast(i32x4, z[j]);
#pragma unroll
            for (int e = 0; e < 4; e++) z[j][e] = FAR ? int8_value_far(s[e], x_scale, c.w[j][e], c.bias[j][e]) : int8_value(s[e], x_scale, c.w[j][e], c.bias[j][e]);
        }
    }
};

// The way out, a row of 16 by 16 FN channels of C at a time.  In the accumulators of two neighbouring blocks lane l has row l % 16 and channels 4 (l / 16) .. + 3 of each; after
// swap_rows() 8 channels in a row of one of them, block l / 16 % 2, from 8 (l / 32): so that memory is moved 16 bytes a lane and 64 of a row at once.  The one wavefront that a
// SIMD has issues an instruction in five clocks, so it is their number that costs: addresses are offsets in buffers, which drop what lies behind the last row, and a channel behind
// the last one has an offset behind every buffer.  (32,760 x 1536 -> 1536, when it was chosen: through LDS in whole rows 137 us, this way with 64-bit addresses and tests 134; now 116,
// 106 without any epilogue.)
template <int FN, int FORM, bool EXTRAS>
struct Out {
    typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
    typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
    static constexpr int PAIRS = FN / 2;
    static constexpr bool INT8 = FORM == LINEAR_INT8, FWD = FORM == LINEAR_FWD, KEEPS = FWD && EXTRAS, ACTS = (FWD || INT8) && EXTRAS, ADDS = FORM == LINEAR_DX || ACTS;  // what may have been asked for
    static constexpr uint32_t OUTSIDE = 0x80000000u;  // 128 rows are less: N < 2^23; no sum with a row's offset passes 2^32
    uint32_t n0, row0, rows;   // the wavefront's first channel and row; rows from there on, at most 128
    uint32_t at[PAIRS];        // bytes, in bf16, from the wavefront's first row to the lane's 8 channels of row l % 16
    __device__ __attribute__((always_inline)) inline Out(const LinearArgs& a, uint32_t m, uint32_t n, uint32_t lane) {
        n0 = n;
        row0 = m;
        rows = m >= a.M ? 0u : a.M - m < 128u ? a.M - m : 128u;
#pragma unroll
        for (int p = 0; p < PAIRS; p++) {
            const uint32_t g = lane >> 4, c = n + 32u * p + 16u * (g & 1u) + 8u * (g >> 1);
            at[p] = c < a.N ? ((lane & 15u) * a.N + c) * 2u : OUTSIDE;
        }
    }
    // bias of the lane's channels of block j, as they lie in the accumulators
    __device__ __attribute__((always_inline)) inline static f32x4 bias(const LinearArgs& a, uint32_t n0, int j, uint32_t lane) {
        f32x4 b = {0.f, 0.f, 0.f, 0.f};
        const uint32_t n = n0 + 16u * j + 4u * (lane >> 4);
        if (FWD && a.e.bias != nullptr && n < a.N) {
            const bf16x4 x = *(const bf16x4*)((const __bf16*)a.e.bias + n);
#pragma unroll
            for (int e = 0; e < 4; e++) b[e] = (float)x[e];
        }
        return b;
    }
    // what is to be added to rows 16 i .., on its way before their results leave
    struct Residual {
        u32x4 x[PAIRS];
    };
    __device__ __attribute__((always_inline)) inline Residual residual(const LinearArgs& a, uint32_t i) const {
        Residual r;
#pragma unroll
        for (int p = 0; p < PAIRS; p++) r.x[p] = u32x4{0u, 0u, 0u, 0u};
#if defined(__HIP_DEVICE_COMPILE__)
        if (ADDS && a.e.residual != nullptr) {
            const auto from = __builtin_amdgcn_make_buffer_rsrc((char*)a.e.residual + (size_t)row0 * a.N * 2u, 0, rows * a.N * 2u, 0x27000);
#pragma unroll
            for (int p = 0; p < PAIRS; p++) r.x[p] = __builtin_amdgcn_raw_buffer_load_b128(from, at[p] + i * 32u * a.N, 0, 0);
        }
#endif
        return r;
    }
    __device__ __attribute__((always_inline)) inline static uint32_t pack(float x, float y) {
        typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
        const bf16x2 b = {(__bf16)x, (__bf16)y};
        return __builtin_bit_cast(uint32_t, b);
    }
    // rows 16 i .. in bf16 to a tensor like C
    __device__ __attribute__((always_inline)) inline void store(const LinearArgs& a, void* tensor, uint32_t i, const f32x4 (&z)[FN]) const {
#if defined(__HIP_DEVICE_COMPILE__)
        const auto to = __builtin_amdgcn_make_buffer_rsrc((char*)tensor + (size_t)row0 * a.N * 2u, 0, rows * a.N * 2u, 0x27000);
#pragma unroll
        for (int p = 0; p < PAIRS; p++) {
            const f32x4 &x = z[2 * p], &y = z[2 * p + 1];
            uint32_t x0 = pack(x[0], x[1]), x1 = pack(x[2], x[3]), y0 = pack(y[0], y[1]), y1 = pack(y[2], y[3]);
            swap_rows(x0, y0);
            swap_rows(x1, y1);
            __builtin_amdgcn_raw_buffer_store_b128(u32x4{x0, x1, y0, y1}, to, at[p] + i * 32u * a.N, 0, 0);
        }
#endif
    }
    // the same as blocks of a checkpoint; z is changed where it is not finite or lies behind the last channel
    __device__ __attribute__((always_inline)) inline void store8(const LinearArgs& a, uint32_t i, f32x4 (&z)[FN], uint32_t lane) const {
#if defined(__HIP_DEVICE_COMPILE__)
        const auto to = __builtin_amdgcn_make_buffer_rsrc((char*)a.e.pre + (size_t)row0 * a.N, 0, rows * a.N, 0x27000);
        const uint32_t blocks = (a.N + CKPT_BLOCK - 1u) / CKPT_BLOCK;
        const auto scales = __builtin_amdgcn_make_buffer_rsrc((char*)a.e.pre_scales + (size_t)row0 * blocks, 0, rows * blocks, 0x27000);
        if (n0 + 16u * FN > a.N) {
#pragma unroll
            for (int j = 0; j < FN; j++)
                if (n0 + 16u * j + 4u * (lane >> 4) >= a.N) z[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int p = 0; p < PAIRS; p++) {
            const f32x4 &x = z[2 * p], &y = z[2 * p + 1];
            float top = ckpt_top(x, y);
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(top == INFINITY) != 0, 0)) {  // rare, and the same for the wavefront
                f32x4 u = x, v = y;
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    u[e] = __builtin_isinf(u[e]) ? NAN : u[e];
                    v[e] = __builtin_isinf(v[e]) ? NAN : v[e];
                }
                z[2 * p] = u;
                z[2 * p + 1] = v;
                top = ckpt_top(u, v);
            }
            const uint32_t byte = ckpt_byte(__float_as_uint(top));
            const float down = ckpt_down(byte);
            uint32_t cx = ckpt_codes_of(x[0] * down, x[1] * down, x[2] * down, x[3] * down), cy = ckpt_codes_of(y[0] * down, y[1] * down, y[2] * down, y[3] * down);
            swap_rows(cx, cy);
            __builtin_amdgcn_raw_buffer_store_b64(u32x2{cx, cy}, to, (at[p] >> 1) + i * 16u * a.N, 0, 0);
            const uint32_t block = n0 / CKPT_BLOCK + p;
            __builtin_amdgcn_raw_buffer_store_b8((unsigned char)byte, scales, lane < 16u && block < blocks ? (16u * i + lane) * blocks + block : OUTSIDE, 0, 0);
        }
#endif
    }
    // the largest |value| of a row's block, not counting what is no number: lanes l, l + 16, l + 32, l + 48 hold it
    __device__ __attribute__((always_inline)) inline static float ckpt_top(const f32x4& x, const f32x4& y) {
        auto max3 = [](float u, float v, float w) __attribute__((always_inline)) { return fmaxf(fmaxf(u, v), w); };
        const float m = max3(max3(fabsf(x[0]), fabsf(x[1]), 0.f), max3(fabsf(x[2]), fabsf(x[3]), fabsf(y[0])), max3(fabsf(y[1]), fabsf(y[2]), fabsf(y[3])));
        uint32_t u = __float_as_uint(m), v = u;
        swap_rows(u, v);
        const float h = fmaxf(__uint_as_float(u), __uint_as_float(v));
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(h), __float_as_uint(h), false, false);
        const uint32_t r0 = r[0], r1 = r[1];
        return fmaxf(__uint_as_float(r0), __uint_as_float(r1));
    }
    // rows 16 i ..: act(z) + residual, z kept
    __device__ __attribute__((always_inline)) inline void row(const LinearArgs& a, uint32_t i, f32x4 (&z)[FN], const Residual& r, uint32_t lane) const {
        const LinearEpilogue& e = a.e;
        if (KEEPS && e.pre_scales != nullptr) {
            f32x4 kept[FN];
#pragma unroll
            for (int j = 0; j < FN; j++) kept[j] = z[j];
            store8(a, i, kept, lane);
        } else if (KEEPS && e.pre != nullptr) store(a, e.pre, i, z);
        if (ACTS && e.act == ACT_GELU_TANH) {
#pragma unroll
            for (int j = 0; j < FN; j++)
#pragma unroll
                for (int x = 0; x < 4; x++) z[j][x] = act_value(ACT_GELU_TANH, z[j][x]);
        } else if (ACTS && e.act == ACT_SILU) {
#pragma unroll
            for (int j = 0; j < FN; j++)
#pragma unroll
                for (int x = 0; x < 4; x++) z[j][x] = act_value(ACT_SILU, z[j][x]);
        }
        if (ADDS && e.residual != nullptr) {
#pragma unroll
            for (int p = 0; p < PAIRS; p++) {
                uint32_t x0 = r.x[p][0], x1 = r.x[p][1], y0 = r.x[p][2], y1 = r.x[p][3];
                swap_rows(x0, y0);
                swap_rows(x1, y1);
                const uint32_t v[2][2] = {{x0, x1}, {y0, y1}};
#pragma unroll
                for (int b = 0; b < 2; b++)
#pragma unroll
                    for (int x = 0; x < 4; x++) {
                        const float add = __uint_as_float(x & 1 ? v[b][x >> 1] & 0xffff0000u : v[b][x >> 1] << 16);
                        z[2 * p + b][x] = INT8 ? int8_plus(z[2 * p + b][x], add) : z[2 * p + b][x] + add;
                    }
            }
        }
        store(a, e.out, i, z);
    }
};

// Accumulators from their registers.  In asm as the products are, so that none is read before the wait behind the last of these: the compiler, which does not know of it, would
// take all of them at once, and put some aside in memory in front of the wait.
__device__ __attribute__((always_inline)) inline f32x4 take(const f32x4& acc) {
    float a = acc[0], b = acc[1], c = acc[2], d = acc[3], w, x, y, z;
    asm volatile("v_accvgpr_read_b32 %0, %4\n\tv_accvgpr_read_b32 %1, %5\n\tv_accvgpr_read_b32 %2, %6\n\tv_accvgpr_read_b32 %3, %7"
                 : "=&v"(w), "=&v"(x), "=&v"(y), "=&v"(z) : "a"(a), "a"(b), "a"(c), "a"(d));
    return f32x4{w, x, y, z};
}

// Accumulators by their registers' names, four for block R / 4: of the products in 8-bit integers, whose walk over three buffers has several ways out, where the compiler would move them about.  It does not know
// that they hold anything.  acc_own() overwrites all of them as far as it can tell, so nothing of its own is in one there; it stands round the walk, in it every 16 products, and on the way out in front of every
// 16 rows.  And the build looks through what was made of these kernels (accumulators.py), and fails if any other instruction of theirs names an accumulation register.  (All of them as clobbers of every
// statement cost a wait state each: 32,760 x 1536 -> 8960 with GELU 551 -> 561 us.)
#define ACC10(t) "a" #t "0", "a" #t "1", "a" #t "2", "a" #t "3", "a" #t "4", "a" #t "5", "a" #t "6", "a" #t "7", "a" #t "8", "a" #t "9"
#define ACC16 ACC10(), "a10", "a11", "a12", "a13", "a14", "a15"
#define ACC64 ACC10(), ACC10(1), ACC10(2), ACC10(3), ACC10(4), ACC10(5), "a60", "a61", "a62", "a63"
#define ACC256 ACC10(), ACC10(1), ACC10(2), ACC10(3), ACC10(4), ACC10(5), ACC10(6), ACC10(7), ACC10(8), ACC10(9), ACC10(10), ACC10(11), ACC10(12), ACC10(13), ACC10(14), ACC10(15), ACC10(16), ACC10(17), \
    ACC10(18), ACC10(19), ACC10(20), ACC10(21), ACC10(22), ACC10(23), ACC10(24), "a250", "a251", "a252", "a253", "a254", "a255"
template <int REGISTERS>
__device__ __attribute__((always_inline)) inline void acc_own() {
    static_assert(REGISTERS == 16 || REGISTERS == 64 || REGISTERS == 256, "a tile's");
    if constexpr (REGISTERS == 16) asm volatile("" ::: ACC16);
    else if constexpr (REGISTERS == 64) asm volatile("" ::: ACC64);
    else asm volatile("" ::: ACC256);
}
template <int R>
__device__ __attribute__((always_inline)) inline void acc_clear() {
    asm volatile("v_accvgpr_write_b32 a[%0], 0\n\tv_accvgpr_write_b32 a[%1], 0\n\tv_accvgpr_write_b32 a[%2], 0\n\tv_accvgpr_write_b32 a[%3], 0" ::"n"(R), "n"(R + 1), "n"(R + 2), "n"(R + 3));
}
template <int R>
__device__ __attribute__((always_inline)) inline void acc_product(const bf16x8& q, const bf16x8& p) {
    asm volatile("v_mfma_i32_16x16x64_i8 a[%0:%1], %2, %3, a[%0:%1]" ::"n"(R), "n"(R + 3), "v"(q), "v"(p));
}
template <int R>
__device__ __attribute__((always_inline)) inline f32x4 acc_take() {
    float w, x, y, z;
    asm volatile("v_accvgpr_read_b32 %0, a[%4]\n\tv_accvgpr_read_b32 %1, a[%5]\n\tv_accvgpr_read_b32 %2, a[%6]\n\tv_accvgpr_read_b32 %3, a[%7]"
                 : "=&v"(w), "=&v"(x), "=&v"(y), "=&v"(z) : "n"(R), "n"(R + 1), "n"(R + 2), "n"(R + 3));
    return f32x4{w, x, y, z};
}

template <int N>
using Int = std::integral_constant<int, N>;
// f(Int<0>) ... f(Int<N - 1>), written out (the loop of 64 products with what stands between them is too much for the unroller)
template <int... I, typename F>
__device__ __attribute__((always_inline)) inline void each(std::integer_sequence<int, I...>, F f) {
    (f(Int<I>{}), ...);
}
template <int N, typename F>
__device__ __attribute__((always_inline)) inline void each(F f) {
    each(std::make_integer_sequence<int, N>{}, f);
}

template <int BM, int BN, int FORM, bool EXTRAS>
__global__ __launch_bounds__(256, 65536 / (BM * BN) < 4 ? 1 : 65536 / (BM * BN) == 4 ? 2 : 4) void linear_kernel(LinearArgs a, TileMap tiles) {
    constexpr bool INT8 = FORM == LINEAR_INT8, PT = FORM == LINEAR_DW, QT = FORM == LINEAR_DX || FORM == LINEAR_DW;
    constexpr int NW = 4, FM = BM / 32, FN = BN / 32;  // wavefronts 2 x 2; blocks of 16 that each has
    using SP = Side<BM, PT, NW>;
    using SQ = Side<BN, QT, NW>;
    // separate arrays: the compiler must be able to tell that what is being filled is not what is being read.  [buffer][half]; what is in one piece has the first only
    __shared__ __attribute__((aligned(1024))) char p00[SP::BYTES], p01[PT ? SP::BYTES : 16], p10[SP::BYTES], p11[PT ? SP::BYTES : 16];
    __shared__ __attribute__((aligned(1024))) char q00[SQ::BYTES], q01[QT ? SQ::BYTES : 16], q10[SQ::BYTES], q11[QT ? SQ::BYTES : 16];
    __shared__ __attribute__((aligned(1024))) char p20[INT8 ? SP::BYTES : 16];  // a third one, below
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = wave & 1u, wn = wave >> 1;
    uint32_t tm, tn, k0, k1, slot;
    tiles.at(blockIdx.x, a.K, tm, tn, k0, k1, slot);
    const uint32_t m0 = tm * BM, n0 = tn * BN;
    const uint32_t ldp = (PT ? a.M : a.K) * 2u, ldq = (QT ? a.N : a.K) * 2u;  // bytes
    const bool mapped = !PT && !QT && a.order != 0;
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
    // bytes of a buffer that begins with row k: what a transposed operand still has; 0 behind the end
    auto records = [&](bool t, uint32_t k, uint32_t ld, uint32_t col0) __attribute__((always_inline)) -> uint32_t {
        if (k >= k1) return 0u;
        if (!t) return LIN_RECORDS;
        const uint64_t left = (uint64_t)(k1 - k) * ld - col0 * 2u;
        return left < LIN_RECORDS ? (uint32_t)left : LIN_RECORDS;
    };
    struct Step {
        const char *p, *q;
        uint32_t rp, rq, left;
    };
    auto step_at = [&](uint32_t k) __attribute__((always_inline)) -> Step {
        return {p0 + (PT ? (size_t)k * ldp : (size_t)k * 2u), q0 + (QT ? (size_t)k * ldq : (size_t)k * 2u), records(PT, k, ldp, m0), records(QT, k, ldq, n0), k < k1 ? k1 - k : 0u};
    };
    const Scales<FM, FN, INT8> scales(a, m0 + wm * (FM * 16u), n0 + wn * (FN * 16u), lane);  // on their way before the walk begins
    f32x4 acc[INT8 ? 1 : FM][INT8 ? 1 : FN];  // sums begin with the bias; those of a part, and whole numbers, with 0
    constexpr int ACCS = FM * FN * 4;
    if constexpr (INT8) {
        acc_own<ACCS>();
        each<FM * FN>([&](auto G) __attribute__((always_inline)) { acc_clear<4 * decltype(G)::value>(); });
        acc_own<ACCS>();
    } else
#pragma unroll
    for (int j = 0; j < FN; j++) {
        const f32x4 b = slot == ~0u ? Out<FN, FORM, EXTRAS>::bias(a, n0 + wn * (FN * 16u), j, lane) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < FM; i++) acc[i][j] = b;
    }
    struct Frags {
        bf16x8 p[FM], q[FN];
    };
    struct Half {
        char *p, *q;
        uint32_t n;
    };
    // fragment i in the order of use: the first of P, all of Q, the others of P
    auto fragment = [&](Frags& f, const Half& from, int i) __attribute__((always_inline)) {
        if (i == 0) f.p[0] = read_fragment<PT, SP::COLS>(from.p, (wm * FM) * 16u, from.n, lane);
        else if (i <= FN) f.q[i - 1] = read_fragment<QT, SQ::COLS>(from.q, (wn * FN + i - 1) * 16u, from.n, lane);
        else f.p[i - FN] = read_fragment<PT, SP::COLS>(from.p, (wm * FM + i - FN) * 16u, from.n, lane);
    };
    // Loads of a step's first part (the first halves of transposed operands) and of its second (operands in one piece, the second halves).
    constexpr int LOADS_A = (PT ? SP::INSTR : 0) + (QT ? SQ::INSTR : 0), WHOLE = (PT ? 0 : SP::INSTR) + (QT ? 0 : SQ::INSTR), LOADS_B = WHOLE + LOADS_A;
    auto load_a = [&](const Step& s, const Half& to, int i) __attribute__((always_inline)) {
        if (PT && i < SP::INSTR) sp.issue(i, s.p, s.rp, s.left, to.p, wave);
        else if (QT) sq.issue(i - (PT ? SP::INSTR : 0), s.q, s.rq, s.left, to.q, wave);
    };
    auto load_b = [&](const Step& whole, const Half& first, const Step& s, const Half& second, int i) __attribute__((always_inline)) {
        if (i >= WHOLE) load_a(s, second, i - WHOLE);
        else if (!PT && i < SP::INSTR) sp.issue(i, whole.p, whole.rp, whole.left, first.p, wave);
        else if (!QT) sq.issue(i - (PT ? 0 : SP::INSTR), whole.q, whole.rq, whole.left, first.q, wave);
    };
    // 32 of k: the products of `f`; between them the fragments of what comes next are read, and `load`s are sent off
    constexpr int MF = FM * FN, RD = FM + FN;
    auto part = [&](auto LOADC, const Frags& f, Frags& next, const Half& from, auto load) __attribute__((always_inline)) {
        constexpr int LOADS = decltype(LOADC)::value;
        each<MF>([&](auto G) __attribute__((always_inline)) {
            constexpr int g = decltype(G)::value;
            if constexpr (INT8) {
                if constexpr (g % 16 == 0) acc_own<ACCS>();
                acc_product<4 * g>(f.q[g % FN], f.p[g / FN]);
            } else asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc[g / FN][g % FN]) : "v"(f.q[g % FN]), "v"(f.p[g / FN]));
            // number i of n stands behind product i * MF / n
            constexpr int first = (g * RD + MF - 1) / MF, last = ((g + 1) * RD + MF - 1) / MF;
            each<last - first>([&](auto I) __attribute__((always_inline)) { fragment(next, from, first + decltype(I)::value); });
            constexpr int lf = (g * LOADS + MF - 1) / MF, ll = ((g + 1) * LOADS + MF - 1) / MF;
            each<ll - lf>([&](auto I) __attribute__((always_inline)) { load(lf + decltype(I)::value); });
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    // What this wavefront has read is in registers, and all but its last N loads have landed: behind the barrier that holds for the workgroup.
    auto meet = [&](auto NC) __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(decltype(NC)::value) : "memory");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
    };
    Frags f0, f1;
    // A step of 64, tile t at k: halves c0 and c1, of which c0 is in f0; the next tile's first half is n0.  A half is free once it is in registers, and is filled with its part
    // of tile t + 2 at once: what comes in halves 3/2 steps before it is read, what comes in one piece a step before.
    auto step = [&](uint32_t k, const Half& c0, const Half& c1, const Half& n0) __attribute__((always_inline)) {
        const Step s0 = step_at(k + 2u * LIN_KT), s1 = step_at(k + 2u * LIN_KT + LIN_KT / 2u);
        part(Int<LOADS_A>{}, f0, f1, c1, [&](int i) __attribute__((always_inline)) { load_a(s0, c0, i); });
        meet(Int<2 * LOADS_A>{});
        part(Int<LOADS_B>{}, f1, f0, n0, [&](int i) __attribute__((always_inline)) { load_b(s0, c0, s1, c1, i); });
        if (LOADS_A) meet(Int<LOADS_A + LOADS_B>{});
    };
    if constexpr (INT8) {
        // A step takes half the time that it takes in the other forms, less than memory needs to answer.  P, the activations, which come from memory (the weights are in the caches), has three buffers: step t asks for
        // P of t + 2 in its first half, while P of t is still read, and for Q of t + 2 in its second, into the buffer just read; between the halves all but the loads just sent have landed, the next step's, P's of
        // which had a step and Q's half of one.  32,760 x 1536 -> 1536 90.6 us with two buffers of both, 84.3 with the third.  P asked for yet half a step sooner, no wait for it until the step after the next:
        // 80,640 x 5120 -> 20,480 6165 -> 6614 us, since workgroups that share rows drift apart and read them again.
        auto step8 = [&](uint32_t k, char* cp, char* cq, char* np, char* nq, char* fp) __attribute__((always_inline)) {
            const Step s2 = step_at(k + 2u * LIN_KT);
            part(Int<SP::INSTR>{}, f0, f1, Half{cp, cq, 1}, [&](int i) __attribute__((always_inline)) { sp.issue(i, s2.p, s2.rp, s2.left, fp, wave); });
            meet(Int<SP::INSTR>{});
            part(Int<SQ::INSTR>{}, f1, f0, Half{np, nq, 0}, [&](int i) __attribute__((always_inline)) { sq.issue(i, s2.q, s2.rq, s2.left, cq, wave); });
        };
        auto fill_p = [&](uint32_t k, char* to) __attribute__((always_inline)) {
            const Step at = step_at(k);
#pragma unroll
            for (int i = 0; i < SP::INSTR; i++) sp.issue(i, at.p, at.rp, at.left, to, wave);
        };
        auto fill_q = [&](uint32_t k, char* to) __attribute__((always_inline)) {
            const Step at = step_at(k);
#pragma unroll
            for (int i = 0; i < SQ::INSTR; i++) sq.issue(i, at.q, at.rq, at.left, to, wave);
        };
        fill_p(k0, p00);
        fill_q(k0, q00);
        fill_p(k0 + LIN_KT, p10);
        fill_q(k0 + LIN_KT, q10);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(SP::INSTR + SQ::INSTR) : "memory");
        __builtin_amdgcn_s_barrier();
#pragma unroll
        for (int i = 0; i < RD; i++) fragment(f0, Half{p00, q00, 0}, i);
        // the wait behind the last products: see below
        auto pair = [&](uint32_t k, char* a, char* b, char* c) __attribute__((always_inline)) {
            step8(k, a, q00, b, q10, c);
            step8(k + LIN_KT, b, q10, c, q00, a);
            asm volatile("s_nop 15" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        };
        uint32_t k = k0;
        for (;;) {
            pair(k, p00, p10, p20);
            if ((k += 2u * LIN_KT) >= k1) break;
            pair(k, p20, p00, p10);
            if ((k += 2u * LIN_KT) >= k1) break;
            pair(k, p10, p20, p00);
            if ((k += 2u * LIN_KT) >= k1) break;
        }
    } else {
        const Half h00 = {p00, q00, 0}, h01 = {PT ? p01 : p00, QT ? q01 : q00, 1}, h10 = {p10, q10, 0}, h11 = {PT ? p11 : p10, QT ? q11 : q10, 1};
        auto fill = [&](uint32_t k, const Half& first, const Half& second) __attribute__((always_inline)) {
            const Step s0 = step_at(k), s1 = step_at(k + LIN_KT / 2u);
#pragma unroll
            for (int i = 0; i < LOADS_A; i++) load_a(s0, first, i);
#pragma unroll
            for (int i = 0; i < LOADS_B; i++) load_b(s0, first, s1, second, i);
        };
        fill(k0, h00, h01);
        fill(k0 + LIN_KT, h10, h11);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS_A + LOADS_B) : "memory");
        __builtin_amdgcn_s_barrier();
#pragma unroll
        for (int i = 0; i < RD; i++) fragment(f0, h00, i);
        if (LOADS_A) meet(Int<LOADS_A + LOADS_B>{});
        uint32_t k = k0;  // below k1
        do {              // a second step behind the end adds zeros
            step(k, h00, h01, h10);
            step(k + LIN_KT, h10, h11, h00);
            // The products are written as asm, with their accumulators pinned to accumulation registers: left to choose, the compiler moved 200 of them in and out a step.  It does not
            // see their latency then (4 passes, so 7 clocks until a result may be read): the last ones are waited for here, in front of all that may follow.
            asm volatile("s_nop 15" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            k += 2u * LIN_KT;
        } while (k < k1);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // loads behind the end still write (zeros) to LDS
    __builtin_amdgcn_sched_barrier(0);
    if (slot != ~0u) {  // a part: sums as they lie in the registers, for linear_join_kernel
        f32x4* const to = (f32x4*)a.partial + ((size_t)slot * 4u + wave) * (FM * FN * 64u) + lane;
        if constexpr (INT8) {
            acc_own<ACCS>();
            each<FM * FN>([&](auto G) __attribute__((always_inline)) { to[decltype(G)::value * 64] = acc_take<4 * decltype(G)::value>(); });
            return;
        }
#pragma unroll
        for (int i = 0; i < FM; i++)
#pragma unroll
            for (int j = 0; j < FN; j++) to[(i * FN + j) * 64] = take(acc[i][j]);
        return;
    }
    uint32_t own = lane;
    asm volatile("" : "+v"(own));  // formed here: else what follows from it is kept in registers through the whole walk
    const Out<FN, FORM, EXTRAS> out(a, m0 + wm * (FM * 16u), n0 + wn * (FN * 16u), own);
    typename Out<FN, FORM, EXTRAS>::Residual r = out.residual(a, 0);
    const auto channels = [&]() __attribute__((always_inline)) {
        if constexpr (INT8) return scales.channels(own);
        else return 0;
    }();
    each<FM>([&](auto I) __attribute__((always_inline)) {
        constexpr int i = decltype(I)::value;
        const typename Out<FN, FORM, EXTRAS>::Residual now = r;
        if (i + 1 < FM) r = out.residual(a, i + 1);
        f32x4 z[FN];
        if constexpr (INT8) {
            acc_own<ACCS>();
            each<FN>([&](auto J) __attribute__((always_inline)) { z[decltype(J)::value] = acc_take<4 * (i * FN + decltype(J)::value)>(); });
            scales.values(z, scales.row(i, own), channels);
        } else {
#pragma unroll
            for (int j = 0; j < FN; j++) z[j] = take(acc[i][j]);
        }
        out.row(a, i, z, now, own);
        __builtin_amdgcn_sched_barrier(0);
    });
}

// Adds up the parts of a tile, in order, and finishes 16 rows of a wavefront's share.
template <int BM, int BN, int FORM, bool EXTRAS>
__global__ __launch_bounds__(64) void linear_join_kernel(LinearArgs a, TileMap tiles) {
    constexpr int FM = BM / 32, FN = BN / 32;
    constexpr uint32_t UNITS = 4 * FM;  // of a tile
    const uint32_t lane = threadIdx.x, r = blockIdx.x / UNITS, unit = blockIdx.x % UNITS, wave = unit / FM, i = unit % FM;
    uint32_t tm, tn;
    tiles.tile(tiles.whole + r, tm, tn);
    const f32x4* from = (const f32x4*)a.partial + ((size_t)r * tiles.parts * 4u + wave) * (FM * FN * 64u) + i * (FN * 64u) + lane;
    const Out<FN, FORM, EXTRAS> out(a, tm * BM + (wave & 1u) * (FM * 16u), tn * BN + (wave >> 1) * (FN * 16u), lane);
    const typename Out<FN, FORM, EXTRAS>::Residual res = out.residual(a, i);
    f32x4 acc[FN];
    if constexpr (FORM == LINEAR_INT8) {
        const Scales<1, FN, true> scales(a, out.row0 + 16u * i, out.n0, lane);
        i32x4 sums[FN];
#pragma unroll
        for (int j = 0; j < FN; j++) sums[j] = __builtin_bit_cast(i32x4, from[j * 64]);
        for (uint32_t p = 1; p < tiles.parts; p++) {
            from += 4 * FM * FN * 64;
#pragma unroll
            for (int j = 0; j < FN; j++) sums[j] += __builtin_bit_cast(i32x4, from[j * 64]);
        }
        const float x_scale = scales.row(0, lane);
        const typename Scales<1, FN, true>::Channels channels = scales.channels(lane);
#pragma unroll
        for (int j = 0; j < FN; j++) acc[j] = __builtin_bit_cast(f32x4, sums[j]);
        scales.values(acc, x_scale, channels);
        out.row(a, i, acc, res, lane);
        return;
    }
#pragma unroll
    for (int j = 0; j < FN; j++) acc[j] = out.bias(a, out.n0, j, lane) + from[j * 64];
    for (uint32_t p = 1; p < tiles.parts; p++) {
        from += 4 * FM * FN * 64;
#pragma unroll
        for (int j = 0; j < FN; j++) acc[j] += from[j * 64];
    }
    out.row(a, i, acc, res, lane);
}

// EXTRAS: an activation, a residual, or values to be kept
template <int SHAPE, int FORM, bool EXTRAS>
static hipError_t launch_tiles(const LinearArgs& a, const LinearPlan& p, hipStream_t stream) {
    constexpr int BM = LINEAR_TILE[SHAPE].m, BN = LINEAR_TILE[SHAPE].n;
    const uint64_t blocks = (uint64_t)p.whole + (uint64_t)p.rest * p.parts;
    if (!fits_grid(blocks, 256u)) return hipErrorInvalidConfiguration;
    const TileMap tiles = make_tile_map(p);
    linear_kernel<BM, BN, FORM, EXTRAS><<<(uint32_t)blocks, 256, 0, stream>>>(a, tiles);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.rest == 0u) return e;
    linear_join_kernel<BM, BN, FORM, EXTRAS><<<p.rest * (4u * BM / 32u), 64, 0, stream>>>(a, tiles);
    return hipGetLastError();
}

// the largest |x| of four, not counting what is not finite, as the bits of its float
__device__ inline uint32_t ckpt_largest(const f32x4& x) {
    uint32_t m = 0u;
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const uint32_t s = ckpt_size(x[e]);
        m = s > m ? s : m;
    }
    return m;
}

// x w^T for a few more rows, up to 16 FM: bound by reading w, which a workgroup does for 16 FN channels.  Its wavefronts take every fourth step of 64 of k, so that together they read
// 512 bytes in a row, each through steps of its own in LDS (no barriers), FEW_DEEP of them on their way; their sums are added up, in order, at the end.  5 rows, 5120 -> 5120: 52 MB, 12.5 us (19.3 in tiles of
// 64 x 64, cut in six).
// KEPT: z is kept as a checkpoint, of whose blocks of 32 channels a workgroup has one, two blocks of its own.  A channel's sum is the same in every form, so that what is kept changes no bit
// of the result.  (us with a checkpoint written, so / in tiles, whose order of the sums is another: 5120 -> 5120, 2 rows 14.5 / 22.2, 16 rows 18.2 / 22.1, 32 rows 20.7 / 22.6; 1536 -> 8960, 16 rows
// 13.5 / 20.4; 8960 -> 1536, 2 rows 16.1 / 19.4, 16 rows 20.0 / 19.3, 32 rows 25.1 / 19.6; with two halves of four wavefronts, 16 channels each, 18.1, 24.4 and 32.7.)
constexpr int FEW_WAVES = 4, FEW_DEEP = 4;
template <int FM, int FN, bool KEPT, int FORM = LINEAR_FWD>
__global__ __launch_bounds__(64 * FEW_WAVES) void linear_few_kernel(LinearArgs a) {
    constexpr bool INT8 = FORM == LINEAR_INT8;
    static_assert(!(INT8 && KEPT), "a product of codes keeps nothing");
    using SP = Side<16 * FM, false, 1>;
    using SQ = Side<16 * FN, false, 1>;
    constexpr int SIZE = SP::BYTES + SQ::BYTES, LOADS = SP::INSTR + SQ::INSTR;  // of a step
    static_assert(SP::BYTES == FM * 2048 && SP::INSTR == 2 * FM, "rows of 128 bytes");
    // separate arrays for the same reason as above
    __shared__ __attribute__((aligned(1024))) char s0[FEW_WAVES * SIZE], s1[FEW_WAVES * SIZE], s2[FEW_WAVES * SIZE], s3[FEW_WAVES * SIZE];
    __shared__ __attribute__((aligned(1024))) f32x4 sums[FEW_WAVES][FM * FN][64];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t n0 = blockIdx.x * (16u * FN), ld = a.K * 2u;
    SP sp;
    SQ sq;
    sp.init(0u, lane, ld, [&](uint32_t r) __attribute__((always_inline)) -> uint32_t {
        const uint32_t m = r < a.M ? r : a.M - 1u;
        return (a.order == 0 ? m : a.order == 1 ? source_row<TO_SPARSE>(a.rows, m, 0u) : source_row<TO_ORIGINAL>(a.rows, m, 0u)) * ld;
    });
    sq.init(0u, lane, ld, [&](uint32_t r) __attribute__((always_inline)) -> uint32_t {
        const uint32_t last = a.N - 1u - n0;
        return (r < last ? r : last) * ld;
    });
#pragma unroll
    for (uint32_t i = 0; i < SP::INSTR; i++)
        if (i * 8u + lane / 8u >= a.M) sp.kofs[i] = LIN_OUTSIDE;  // rows behind the last: zeros
    const char *const p0 = (const char*)a.p, *const q0 = (const char*)a.q + (size_t)n0 * ld;
    auto fill = [&](uint32_t k, char* all) __attribute__((always_inline)) {  // behind the end: zeros
        char* const to = all + wave * SIZE;
        const uint32_t left = k < a.K ? a.K - k : 0u;
#pragma unroll
        for (int i = 0; i < SQ::INSTR; i++) sq.issue(i, q0 + (size_t)k * 2u, LIN_RECORDS, left, to, 0u);
#pragma unroll
        for (int i = 0; i < SP::INSTR; i++) sp.issue(i, p0 + (size_t)k * 2u, LIN_RECORDS, left, to + SQ::BYTES, 0u);
    };
    f32x4 acc[FM * FN];
#pragma unroll
    for (int i = 0; i < FM * FN; i++) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    constexpr uint32_t STRIDE = FEW_WAVES * LIN_KT;
    auto step = [&](uint32_t k, char* all) __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((FEW_DEEP - 1) * LOADS) : "memory");
        const char* const from = all + wave * SIZE;
        bf16x8 q[2][FN], p[2][FM];
#pragma unroll
        for (uint32_t h = 0; h < 2; h++) {
#pragma unroll
            for (int j = 0; j < FN; j++) q[h][j] = read_fragment<false, SQ::COLS>(from, 16u * j, h, lane);
#pragma unroll
            for (int i = 0; i < FM; i++) p[h][i] = read_fragment<false, SP::COLS>(from + SQ::BYTES, 16u * i, h, lane);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the step is in registers, and may be filled again
        __builtin_amdgcn_sched_barrier(0);
        fill(k + FEW_DEEP * STRIDE, all);
#pragma unroll
        for (uint32_t h = 0; h < 2; h++)
#pragma unroll
            for (int i = 0; i < FM * FN; i++) {
                if constexpr (INT8)
                    acc[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, q[h][i % FN]), __builtin_bit_cast(i32x4, p[h][i / FN]), __builtin_bit_cast(i32x4, acc[i]), 0, 0, 0));
                else acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[h][i % FN], p[h][i / FN], acc[i], 0, 0, 0);
            }
    };
    uint32_t k = wave * LIN_KT;
    fill(k, s0);
    fill(k + STRIDE, s1);
    fill(k + 2u * STRIDE, s2);
    fill(k + 3u * STRIDE, s3);
    for (; k < a.K; k += FEW_DEEP * STRIDE) {
        step(k, s0);
        step(k + STRIDE, s1);
        step(k + 2u * STRIDE, s2);
        step(k + 3u * STRIDE, s3);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < FM * FN; i++) sums[wave][i][lane] = acc[i];
    __syncthreads();
    // wavefront i finishes block i: lane l has row l % 16 and channels 4 (l / 16) .. + 3
    static_assert(FM * FN <= FEW_WAVES, "a block a wavefront");
    const uint32_t m = wave / FN * 16u + (lane & 15u), n = n0 + wave % FN * 16u + 4u * (lane >> 4);
    if (wave >= (uint32_t)(FM * FN)) return;
    const LinearEpilogue& e = a.e;
    const size_t at = (size_t)m * a.N + n;
    auto add = [&](f32x4& z, const void* t, size_t from) __attribute__((always_inline)) {
        const bf16x4 x = *(const bf16x4*)((const __bf16*)t + from);
#pragma unroll
        for (int c = 0; c < 4; c++) z[c] = INT8 ? int8_plus(z[c], (float)x[c]) : z[c] + (float)x[c];
    };
    auto sum = [&](uint32_t b, uint32_t c) __attribute__((always_inline)) -> f32x4 {  // of block b, the lane's channels from c
        f32x4 z = sums[0][b][lane];
        if constexpr (INT8) {
            i32x4 s = __builtin_bit_cast(i32x4, z);
#pragma unroll
            for (int w = 1; w < FEW_WAVES; w++) s += __builtin_bit_cast(i32x4, sums[w][b][lane]);
            if (m >= a.M || c >= a.N) return f32x4{0.f, 0.f, 0.f, 0.f};
            const float x_scale = a.x_scales[a.order == 0 ? m : a.order == 1 ? source_row<TO_SPARSE>(a.rows, m, 0u) : source_row<TO_ORIGINAL>(a.rows, m, 0u)];
            const f32x4 w_scale = *(const f32x4*)(a.w_scales + c);
            f32x4 bias = {0.f, 0.f, 0.f, 0.f};
            if (e.bias != nullptr) add(bias, e.bias, c);
#pragma unroll
            for (int i = 0; i < 4; i++) z[i] = int8_value_far(s[i], x_scale, w_scale[i], bias[i]);
            return z;
        }
#pragma unroll
        for (int w = 1; w < FEW_WAVES; w++) z += sums[w][b][lane];
        if (e.bias != nullptr && c < a.N) add(z, e.bias, c);
        return z;
    };
    f32x4 z = sum(wave, n);
    if (KEPT) {
        static_assert(!KEPT || FN * 16 == CKPT_BLOCK, "a block of a checkpoint: two wavefronts' channels");
        // the other's sums are formed here as well, in the same order: lanes l, l + 16, l + 32, l + 48 have a row's block then
        const f32x4 other = sum(wave ^ 1u, n ^ 16u);
        uint32_t top = n < a.N ? ckpt_largest(z) : 0u;
        const uint32_t o = (n ^ 16u) < a.N ? ckpt_largest(other) : 0u;
        top = o > top ? o : top;
#pragma unroll
        for (int off = 16; off <= 32; off <<= 1) {
            const uint32_t far = (uint32_t)__shfl_xor((int)top, off);
            top = far > top ? far : top;
        }
        const uint32_t byte = ckpt_byte(top);
        if (m < a.M && n < a.N) *(uint32_t*)((unsigned char*)e.pre + at) = ckpt_codes(z[0], z[1], z[2], z[3], ckpt_down(byte));
        if (m < a.M && (n & 16u) == 0u && lane < 16u) ((unsigned char*)e.pre_scales)[(size_t)m * ((a.N + CKPT_BLOCK - 1u) / CKPT_BLOCK) + blockIdx.x] = (unsigned char)byte;
    }
    if (m >= a.M || n >= a.N) return;
    auto store = [&](void* t) __attribute__((always_inline)) {
        bf16x4 x;
#pragma unroll
        for (int c = 0; c < 4; c++) x[c] = (__bf16)z[c];
        *(bf16x4*)((__bf16*)t + at) = x;
    };
    if (!KEPT && e.pre != nullptr) store(e.pre);
#pragma unroll
    for (int c = 0; c < 4; c++) z[c] = act_value(e.act, z[c]);
    if (e.residual != nullptr) add(z, e.residual, at);
    store(e.out);
}

}  // namespace skiparse

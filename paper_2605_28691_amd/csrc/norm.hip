// Root-mean-square norm of rows, with the residual's addition in front of it and, if asked for, its result in 8-bit integers; rows in 8-bit integers without a norm; and the
// norm's gradients.  All sums in float32.
//     h = x + residual,  r = 1 / sqrt(mean(h^2) + eps),  y = h r w          int8: codes and scale of h w (int8_rows.h), the scale times r: r is the same for a row and changes no code
//     g = dy w,  u = h r,  dx = r (g - u mean(g u)) + dx_add,  dw = sum over the rows of dy u
// Bound by HBM bandwidth: every tensor is moved once, a row stays in registers between its sum and its result (norm_shape.h: which lanes have it).  Of the norm's codes the largest value and the sum of squares
// come from one pass over these registers: codes do not need r.  80,640 x 5120 in bf16: with residual and sum, into the sparse layout, 565 us (3.3 GB, 5.85 TB/s; a copy of 2 GiB reaches 4.9, permute.hip 6.5), in 8-bit
// integers 200 us (1.24 GB, 6.2); 32,760 x 1536 with residual in codes 58 us (5.2).
#include "int8_rows.h"
#include "kernels.h"
#include "norm_shape.h"
#include "row_pieces.h"

namespace skiparse {

// Which row, and which channels of it, a lane has: pieces of 8, CH of them.  SPAN_LANES: several rows a wavefront, `lanes` lanes each; SPAN_WAVE: a row a wavefront; SPAN_GROUP: a row a workgroup.
template <typename T, int SPAN, int CH>
struct Place {
    uint32_t first, step, cols;  // the lane's first channel, from a piece to the next, the row's channels
    uint32_t half;               // from a unit of a piece to the next
    __device__ __attribute__((always_inline)) inline Place(uint32_t lanes, uint32_t n) {
        const uint32_t lane = threadIdx.x & 63u, in_row = SPAN == SPAN_LANES ? lane & (lanes - 1u) : lane;
        first = in_row * Piece<T>::EACH + (SPAN == SPAN_GROUP ? (threadIdx.x >> 6) * 512u : 0u);
        step = SPAN == SPAN_GROUP ? blockDim.x * 8u : 512u;
        half = SPAN == SPAN_LANES ? lanes * 4u : 256u;
        cols = n;
    }
    // rows that a workgroup has at once, and which of them is the lane's
    static __device__ inline uint32_t rows(uint32_t lanes) { return SPAN == SPAN_LANES ? blockDim.x / lanes : SPAN == SPAN_WAVE ? blockDim.x / 64u : 1u; }
    static __device__ inline uint32_t row(uint32_t lanes) {
        if (SPAN == SPAN_LANES) return threadIdx.x / lanes;
        return SPAN == SPAN_WAVE ? (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0u;
    }
    // first channel of unit u of piece i; false: behind the row's end
    __device__ __attribute__((always_inline)) inline bool at(int i, int u, uint32_t& c) const {
        c = first + i * step + u * half;
        return c < cols;
    }
    // piece i of the row that begins with element `row`; zeros behind its end, and for lanes without a row
    template <bool NT>
    __device__ __attribute__((always_inline)) inline Piece<T> load_one(const void* from, size_t row, bool on, int i) const {
        Piece<T> p;
#pragma unroll
        for (int u = 0; u < Piece<T>::UNITS; u++) {
            uint32_t c;
            p.raw[u] = piece_u32x4{0u, 0u, 0u, 0u};
            if (at(i, u, c) && on) p.raw[u] = load16<NT>((const T*)from + row + c);
        }
        return p;
    }
    template <bool NT>
    __device__ __attribute__((always_inline)) inline void load(const void* from, size_t row, bool on, Piece<T> (&p)[CH]) const {
#pragma unroll
        for (int i = 0; i < CH; i++) p[i] = load_one<NT>(from, row, on, i);
    }
    template <bool NT>
    __device__ __attribute__((always_inline)) inline void store(void* to, size_t row, bool on, int i, const float (&v)[8]) const {
        Piece<T> p;
        p.set(v);
#pragma unroll
        for (int u = 0; u < Piece<T>::UNITS; u++) {
            uint32_t c;
            if (at(i, u, c) && on) store16<NT>((T*)to + row + c, p.raw[u]);
        }
    }
};

struct Plus {
    template <typename S>
    __device__ static inline S of(S a, S b) { return a + b; }
};
struct Largest {
    __device__ static inline uint32_t of(uint32_t a, uint32_t b) { return a > b ? a : b; }
};

// The lanes of a row, of `lanes` neighbours, as one value in each of them, a + b for the pairs 1, 2, 4 .. apart.  Within rows of 16 lanes as DPP operands: where quads agree, the lanes of a mirrored half
// row are as good as those 4 apart, and so on.
template <int CONTROL>
__device__ __attribute__((always_inline)) inline uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CONTROL, 0xf, 0xf, true); }
template <typename OP, typename S, int N>
__device__ __attribute__((always_inline)) inline void across(S (&v)[N], uint32_t lanes) {
    static_assert(sizeof(S) == 4, "a register");
    auto bits = [](S x) __attribute__((always_inline)) -> uint32_t { return __builtin_bit_cast(uint32_t, x); };
    auto value = [](uint32_t x) __attribute__((always_inline)) -> S { return __builtin_bit_cast(S, x); };
#define EACH for (int i = 0; i < N; i++)
    if (lanes >= 2u)
#pragma unroll
        EACH v[i] = OP::of(v[i], value(dpp<0xb1>(bits(v[i]))));  // quad_perm 1 0 3 2
    if (lanes >= 4u)
#pragma unroll
        EACH v[i] = OP::of(v[i], value(dpp<0x4e>(bits(v[i]))));  // quad_perm 2 3 0 1
    if (lanes >= 8u)
#pragma unroll
        EACH v[i] = OP::of(v[i], value(dpp<0x141>(bits(v[i]))));  // row_half_mirror
    if (lanes >= 16u)
#pragma unroll
        EACH v[i] = OP::of(v[i], value(dpp<0x140>(bits(v[i]))));  // row_mirror
    if (lanes >= 32u)
#pragma unroll
        EACH {
            const auto r = __builtin_amdgcn_permlane16_swap(bits(v[i]), bits(v[i]), false, false);
            v[i] = OP::of(value(r[0]), value(r[1]));
        }
    if (lanes >= 64u)
#pragma unroll
        EACH {
            const auto r = __builtin_amdgcn_permlane32_swap(bits(v[i]), bits(v[i]), false, false);
            v[i] = OP::of(value(r[0]), value(r[1]));
        }
#undef EACH
}

// Sums of a row: of each 512 channels over their lanes, then these one after the other.  So they are the same whichever shape has the row, and a row's bits depend on nothing but the row.
// v[k][i]: of the lane's channels in its piece i.  all: a place for the 512s of a workgroup's row (SPAN_GROUP); each call until a barrier takes another.
template <int SPAN, int CH, int N>
__device__ __attribute__((always_inline)) inline void row_sums(float (&v)[N][CH], float (&sum)[N], uint32_t lanes, uint32_t chunks, float (*all)[N]) {
#pragma unroll
    for (int k = 0; k < N; k++) across<Plus>(v[k], SPAN == SPAN_LANES ? lanes : 64u);
    if (SPAN != SPAN_GROUP) {
#pragma unroll
        for (int k = 0; k < N; k++) {
            sum[k] = v[k][0];
#pragma unroll
            for (int i = 1; i < CH; i++) sum[k] += v[k][i];
        }
        return;
    }
    const uint32_t waves = blockDim.x >> 6, wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63u) == 0u) {
#pragma unroll
        for (int i = 0; i < CH; i++)
#pragma unroll
            for (int k = 0; k < N; k++) all[i * waves + wave][k] = v[k][i];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; k++) sum[k] = all[0][k];
    for (uint32_t c = 1; c < chunks; c++)
#pragma unroll
        for (int k = 0; k < N; k++) sum[k] += all[c][k];
}
template <int SPAN>
__device__ __attribute__((always_inline)) inline uint32_t row_largest(uint32_t v, uint32_t lanes, uint32_t* all) {
    uint32_t top[1] = {v};
    across<Largest>(top, SPAN == SPAN_LANES ? lanes : 64u);
    if (SPAN != SPAN_GROUP) return top[0];
    if ((threadIdx.x & 63u) == 0u) all[threadIdx.x >> 6] = top[0];
    __syncthreads();
    for (uint32_t w = 0; w < blockDim.x >> 6; w++) top[0] = Largest::of(top[0], all[w]);
    return top[0];
}

// Squares of values beyond 2^63 or so are infinite in float32, and those below 2^-63 lose digits: a row whose sum says so is summed once more, with its values times a power of two that keeps
// every square that counts in range (values below 2^128 times 2^-80; values below 2^-42, of which squares below 2^-126 do not count beside eps, times 2^70).
__device__ inline bool out_of_range(float squares, float per_n, float eps) { return !(squares <= 1e38f) || squares * per_n + eps < 1e-30f; }
__device__ inline float into_range(float squares) { return squares <= 1.f ? 0x1p70f : 0x1p-80f; }
// 1 / sqrt(mean + eps), of values times `by` if that is not 1
__device__ inline float inverse_size(float squares, float per_n, float eps, float by = 1.f) { return 1.f / sqrtf(squares * per_n + eps * by * by); }

__device__ inline float uniform(float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); }

__device__ inline uint32_t source_of(int order, const RowArgs& rows, uint32_t row) {
    return order == 1 ? source_row<TO_SPARSE>(rows, row, 0u) : order == 2 ? source_row<TO_ORIGINAL>(rows, row, 0u) : row;
}

// What a row's sums and largest value need of LDS.
template <int SPAN, int CH>
struct RowPlaces {
    float sums[SPAN == SPAN_GROUP ? NORM_WAVES * CH : 1][1], again[SPAN == SPAN_GROUP ? NORM_WAVES * CH : 1][1];
    uint32_t tops[SPAN == SPAN_GROUP ? NORM_WAVES : 1];
};

// A row, of whose tensors the lane's pieces are in x and other (residual).
template <typename T, int KIND, int SPAN, int CH, bool NT>
__device__ __attribute__((always_inline)) inline void norm_row(const NormArgs& a, const Place<T, SPAN, CH>& at, uint32_t lanes, uint32_t row, size_t in, bool on, const Piece<T> (&x)[CH], Piece<T> (&other)[CH],
                                                               RowPlaces<SPAN, CH>& lds) {
    const bool adds = KIND != ROWS_QUANTIZED && a.residual != nullptr;
    const size_t to = (size_t)row * a.cols;
    float h[CH][8];
    float squares[1][CH];
#pragma unroll
    for (int i = 0; i < CH; i++) {
#pragma unroll
        for (int e = 0; e < 8; e++) h[i][e] = x[i].get(e);
        if (KIND == ROWS_QUANTIZED) continue;
        if (adds) {
#pragma unroll
            for (int e = 0; e < 8; e++) h[i][e] += other[i].get(e);
            if (a.sum != nullptr) at.template store<NT>(a.sum, in, on, i, h[i]);
        }
        squares[0][i] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; e++) squares[0][i] = fmaf(h[i][e], h[i][e], squares[0][i]);
    }
    const bool weighs = KIND != ROWS_QUANTIZED && a.weight != nullptr;
    if (weighs) at.template load<false>(a.weight, 0, true, other);
    float r = 1.f;
    if (KIND != ROWS_QUANTIZED) {
        float sum[1];
        row_sums<SPAN, CH, 1>(squares, sum, lanes, a.chunks, lds.sums);
        r = inverse_size(sum[0], a.per_n, a.eps);
        const bool bad = on && out_of_range(sum[0], a.per_n, a.eps);
        if (__builtin_expect(SPAN == SPAN_GROUP ? bad : __builtin_amdgcn_ballot_w64(bad) != 0, 0)) {  // all lanes of a wavefront go
            const float by = into_range(sum[0]);
#pragma unroll
            for (int i = 0; i < CH; i++) {
                squares[0][i] = 0.f;
#pragma unroll
                for (int e = 0; e < 8; e++) squares[0][i] = fmaf(h[i][e] * by, h[i][e] * by, squares[0][i]);
            }
            row_sums<SPAN, CH, 1>(squares, sum, lanes, a.chunks, lds.again);
            if (bad) r = by * inverse_size(sum[0], a.per_n, a.eps, by);
        }
    }
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < CH; i++) {
        if (KIND == ROWS_NORM) {
#pragma unroll
            for (int e = 0; e < 8; e++) h[i][e] *= r;
        }
        if (weighs) {
#pragma unroll
            for (int e = 0; e < 8; e++) h[i][e] *= other[i].get(e);
        }
        if (KIND == ROWS_NORM) {
            at.template store<NT>(a.out, to, on, i, h[i]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++) top = Largest::of(top, int8_size(h[i][e]));
        }
    }
    if (KIND == ROWS_NORM) return;
    const Int8Row q(row_largest<SPAN>(top, lanes, lds.tops), r);
#pragma unroll
    for (int i = 0; i < CH; i++) {
        uint32_t codes[2], c;
        codes[0] = q.codes(h[i][0], h[i][1], h[i][2], h[i][3]);
        codes[1] = q.codes(h[i][4], h[i][5], h[i][6], h[i][7]);
        char* const out = (char*)a.out + to;
        if (Piece<T>::UNITS == 1) {
            if (at.at(i, 0, c) && on) *(piece_u32x2*)(out + c) = piece_u32x2{codes[0], codes[1]};
        } else {
#pragma unroll
            for (int u = 0; u < 2; u++)
                if (at.at(i, u, c) && on) *(uint32_t*)(out + c) = codes[u];
        }
    }
    if (on && at.first == 0u) a.scales[row] = q.scale;
}

template <typename T, int KIND, int SPAN, int CH, bool NT>
__global__ __launch_bounds__(SPAN == SPAN_GROUP ? 64 * NORM_WAVES : 256) void norm_rows_kernel(NormArgs a, uint32_t lanes) {
    __shared__ RowPlaces<SPAN, CH> lds;
    const Place<T, SPAN, CH> at(lanes, a.cols);
    const uint32_t row = a.first + blockIdx.x * at.rows(lanes) + at.row(lanes);
    const bool on = row < a.n_rows;
    if (SPAN == SPAN_WAVE && !on) return;
    const size_t in = on ? (size_t)source_of(a.order, a.rows, row) * a.cols : 0;
    Piece<T> x[CH], other[CH];
    at.template load<NT>(a.x, in, on, x);
    if (KIND != ROWS_QUANTIZED && a.residual != nullptr) at.template load<NT>(a.residual, in, on, other);
    norm_row<T, KIND, SPAN, CH, NT>(a, at, lanes, row, in, on, x, other, lds);
}

// The same for rows of a part of a wavefront without a residual, past the caches: the lanes have two rows, the second on its way while the first is worked on (norm_turns()).
template <typename T, int KIND>
__global__ __launch_bounds__(256) void norm_two_rows_kernel(NormArgs a, uint32_t lanes) {
    __shared__ RowPlaces<SPAN_LANES, 1> lds;
    const Place<T, SPAN_LANES, 1> at(lanes, a.cols);
    const uint32_t row = a.first + blockIdx.x * (2u * at.rows(lanes)) + at.row(lanes), second = row + at.rows(lanes);
    const bool on = row < a.n_rows, more = second < a.n_rows;
    const size_t in = on ? (size_t)source_of(a.order, a.rows, row) * a.cols : 0, next = more ? (size_t)source_of(a.order, a.rows, second) * a.cols : 0;
    Piece<T> x[1], y[1], other[1];
    at.template load<true>(a.x, in, on, x);
    at.template load<true>(a.x, next, more, y);
    norm_row<T, KIND, SPAN_LANES, 1, true>(a, at, lanes, row, in, on, x, other, lds);
    norm_row<T, KIND, SPAN_LANES, 1, true>(a, at, lanes, second, next, more, y, other, lds);
}

template <typename T, int KIND, bool NT>
static hipError_t launch_rows_t(NormArgs a, hipStream_t stream) {
    const uint32_t read = sizeof(T) * (a.residual ? 2u : 1u);
    const NormShape s = norm_shape(a.n_rows, a.cols, read);
    const bool two = norm_turns(s.span, read, NT) == 2u;
    const uint32_t per = (s.span == SPAN_LANES ? s.threads / s.lanes : s.span == SPAN_WAVE ? s.threads / 64u : 1u) * (two ? 2u : 1u);
    const uint64_t at_once = ((1ull << 31) / s.threads) * per;  // rows of a launch: a grid has less than 2^32 threads
    for (uint64_t first = 0; first < a.n_rows; first += at_once) {
        a.first = (uint32_t)first;
        const uint32_t n = (uint32_t)(a.n_rows - first < at_once ? a.n_rows - first : at_once), blocks = (n + per - 1u) / per;
        if (two) {
            if constexpr (NT && sizeof(T) == 2) norm_two_rows_kernel<T, KIND><<<blocks, s.threads, 0, stream>>>(a, s.lanes);
        } else if (s.span == SPAN_LANES) {
            if constexpr (!(NT && sizeof(T) == 2 && KIND == ROWS_QUANTIZED)) norm_rows_kernel<T, KIND, SPAN_LANES, 1, NT><<<blocks, s.threads, 0, stream>>>(a, s.lanes);
        }
#define ROWS(SPAN, CH) \
    else if (s.span == SPAN && s.ch == CH) norm_rows_kernel<T, KIND, SPAN, CH, NT><<<blocks, s.threads, 0, stream>>>(a, 64u);
        ROWS(SPAN_WAVE, 1)
        ROWS(SPAN_WAVE, 2)
        ROWS(SPAN_WAVE, 3)
        ROWS(SPAN_GROUP, 1)
        ROWS(SPAN_GROUP, 2)
        ROWS(SPAN_GROUP, 4)
#undef ROWS
        else return hipErrorInvalidValue;
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, int KIND>
static hipError_t launch_rows_of(const NormArgs& a, hipStream_t stream) {
    const uint64_t n = (uint64_t)a.n_rows * a.cols, e = sizeof(T);
    const uint64_t moved = n * (e + (a.residual ? e : 0u) + (a.sum ? e : 0u) + (KIND == ROWS_NORM ? e : 1u));
    return moved >= NORM_PAST_CACHES ? launch_rows_t<T, KIND, true>(a, stream) : launch_rows_t<T, KIND, false>(a, stream);
}

template <typename T>
static hipError_t launch_rows_as(const NormArgs& a, hipStream_t stream) {
    switch (a.kind) {
        case ROWS_NORM: return launch_rows_of<T, ROWS_NORM>(a, stream);
        case ROWS_NORM_QUANTIZED: return launch_rows_of<T, ROWS_NORM_QUANTIZED>(a, stream);
        default: return launch_rows_of<T, ROWS_QUANTIZED>(a, stream);
    }
}

hipError_t launch_norm_rows(const NormArgs& all, hipStream_t stream) {
    NormArgs a = all;
    a.per_n = 1.f / (float)a.cols;
    a.chunks = (a.cols + 511u) / 512u;
    return a.f32 ? launch_rows_as<float>(a, stream) : launch_rows_as<__bf16>(a, stream);
}

// ---- gradients

// dx and the weights' gradient in one pass over dy and h: 32,760 x 1536 with dx_add 75 us, and 4.4 for the parts' sums (403 MB: 5.1 TB/s), 80,640 x 5120 637 (5.2 TB/s), 6426 x 1000 float32 15.9 + 4.0 (77 MB: what
// is in flight with 1604 wavefronts; 17.6 + 3.9 with 1024).
// A workgroup takes a contiguous part of the rows, and has the sums of its part for the weights' gradient in registers: each lane those of its channels.  The next row is on its way while one is
// worked on.  LEAN, for rows so long that the registers do not hold all that: no next row, weights and dx_add are read where they are used.
template <typename T, int SPAN, int CH, bool NT>
__global__ __launch_bounds__(SPAN == SPAN_GROUP ? 64 * NORM_WAVES : NORM_BWD_THREADS) void norm_bwd_kernel(NormBwdArgs a, uint32_t lanes) {
    constexpr bool LEAN = SPAN == SPAN_GROUP && CH * (int)sizeof(T) >= 8;
    constexpr int CHUNKS = SPAN == SPAN_GROUP ? NORM_WAVES * CH : 1;
    __shared__ float sums[2][CHUNKS][2];  // of rows by turns: one barrier a row is enough
    __shared__ float again[CHUNKS][2];
    constexpr bool STAGED = SPAN == SPAN_GROUP && CH == 4;  // the sums for the weights' gradient in LDS: 8 floats a piece are too much as well
    __shared__ __attribute__((aligned(16))) float dws[STAGED ? 64 * NORM_WAVES * CH * 8 : SPAN == SPAN_GROUP ? 4 : NORM_BWD_THREADS / 64 * CH * 512];
    const Place<T, SPAN, CH> at(lanes, a.cols);
    const uint32_t first = (uint32_t)((uint64_t)blockIdx.x * a.n_rows / gridDim.x), end = (uint32_t)((uint64_t)(blockIdx.x + 1u) * a.n_rows / gridDim.x);
    const uint32_t stride = at.rows(lanes), own = at.row(lanes);
    Piece<T> w[CH];
    auto weight = [&](int i) __attribute__((always_inline)) {
        const float ones[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
        if (a.weight != nullptr) w[i] = at.template load_one<false>(a.weight, 0, true, i);
        else w[i].set(ones);
    };
    if (!LEAN) {
#pragma unroll
        for (int i = 0; i < CH; i++) weight(i);
    }
    float dw[STAGED ? 1 : CH][8] = {};
    piece_u32x4* const staged = (piece_u32x4*)dws + threadIdx.x;  // a lane's own
    if (STAGED) {
#pragma unroll
        for (int i = 0; i < 2 * CH; i++) staged[i * (64 * NORM_WAVES)] = piece_u32x4{0u, 0u, 0u, 0u};
    }
    Piece<T> hc[CH], yc[CH], ac[CH], hn[CH], yn[CH], an[CH];
    const bool adds = a.dx != nullptr && a.dx_add != nullptr;
    auto load = [&](uint32_t row, Piece<T> (&h)[CH], Piece<T> (&y)[CH], Piece<T> (&add)[CH]) __attribute__((always_inline)) {
        const bool on = row < end;
        const size_t in = on ? (size_t)source_of(a.order, a.rows, row) * a.cols : 0, to = (size_t)row * a.cols;
        at.template load<NT>(a.h, to, on, h);
        at.template load<NT>(a.dy, in, on, y);
        if (adds && !LEAN) at.template load<NT>(a.dx_add, to, on, add);
    };
    if (!LEAN) load(first + own, hn, yn, an);
    uint32_t turn = 0u;
    // every lane goes through every round: rows are exchanged within wavefronts
    for (uint32_t base = first; base < end; base += stride) {
        const uint32_t row = base + own;
        const bool on = row < end;
        if (SPAN == SPAN_WAVE && !on) break;
        if (LEAN) {
            load(row, hc, yc, ac);
        } else {
#pragma unroll
            for (int i = 0; i < CH; i++) {
                hc[i] = hn[i];
                yc[i] = yn[i];
                ac[i] = an[i];
            }
            load(row + stride, hn, yn, an);
        }
        float parts[2][CH], sum[2];
#pragma unroll
        for (int i = 0; i < CH; i++) {
            parts[0][i] = parts[1][i] = 0.f;
            if (LEAN) weight(i);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float h = hc[i].get(e);
                parts[0][i] = fmaf(h, h, parts[0][i]);
                parts[1][i] = fmaf(yc[i].get(e) * w[i].get(e), h, parts[1][i]);
            }
        }
        row_sums<SPAN, CH, 2>(parts, sum, lanes, a.chunks, sums[turn & 1u]);
        turn++;
        float r = inverse_size(sum[0], a.per_n, a.eps), mean = sum[1] * a.per_n * r;
        // g h may be beyond float32's range where g u is not: g times 2^-80 then
        const bool far = out_of_range(sum[0], a.per_n, a.eps), high = !(fabsf(sum[1]) <= 3.4028234663852886e38f), bad = on && (far || high);
        if (__builtin_expect(SPAN == SPAN_GROUP ? bad : __builtin_amdgcn_ballot_w64(bad) != 0, 0)) {
            float by = far ? into_range(sum[0]) : 1.f, down = high ? 0x1p-80f : 1.f;
            if (SPAN == SPAN_GROUP) {  // the workgroup's: not in vector registers
                by = uniform(by);
                down = uniform(down);
            }
#pragma unroll
            for (int i = 0; i < CH; i++) {
                parts[0][i] = parts[1][i] = 0.f;
                if (LEAN) weight(i);
#pragma unroll
                for (int u = 0; u < (CH > 1 ? Piece<T>::UNITS : 0); u++) asm volatile("" : "+v"(hc[i].raw[u]), "+v"(yc[i].raw[u]));  // formed here once more, not kept for rows that need none of it
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const float h = hc[i].get(e) * by;
                    parts[0][i] = fmaf(h, h, parts[0][i]);
                    parts[1][i] = fmaf(yc[i].get(e) * w[i].get(e) * down, h, parts[1][i]);
                }
            }
            if (SPAN == SPAN_GROUP) __syncthreads();  // the last such row's have been read
            row_sums<SPAN, CH, 2>(parts, sum, lanes, a.chunks, again);
            if (bad) {
                const float s = inverse_size(sum[0], a.per_n, a.eps, by);
                r = by * s;
                mean = sum[1] * a.per_n * s;
                mean *= 1.f / down;
            }
        }
        if (LEAN) {
            // taken from the registers as they came once more, not kept as floats from above
#pragma unroll
            for (int i = 0; i < CH; i++)
#pragma unroll
                for (int u = 0; u < Piece<T>::UNITS; u++) asm volatile("" : "+v"(hc[i].raw[u]), "+v"(yc[i].raw[u]));
        }
#pragma unroll
        for (int i = 0; i < CH; i++) {
            if (LEAN) {
                __builtin_amdgcn_sched_barrier(0);  // a piece after the other
                weight(i);
                if (adds) ac[i] = at.template load_one<NT>(a.dx_add, (size_t)row * a.cols, on, i);
            }
            float g[8];
            Piece<float> d;
            if (STAGED) {
#pragma unroll
                for (int q = 0; q < 2; q++) d.raw[q] = staged[(2 * i + q) * (64 * NORM_WAVES)];
            } else d.set(dw[i]);
            float(&sum_dw)[8] = dw[STAGED ? 0 : i];
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float u = hc[i].get(e) * r, y = yc[i].get(e);
                sum_dw[e] = on ? fmaf(y, u, d.get(e)) : d.get(e);
                g[e] = r * (y * w[i].get(e) - u * mean);
                if (adds) g[e] += ac[i].get(e);
            }
            if (STAGED) {
                d.set(sum_dw);
#pragma unroll
                for (int q = 0; q < 2; q++) staged[(2 * i + q) * (64 * NORM_WAVES)] = d.raw[q];
            }
            if (a.dx != nullptr) at.template store<NT>(a.dx, (size_t)row * a.cols, on, i, g);
        }
    }
    if (a.dw == nullptr) return;
    auto out = [&](int i, const float (&s)[8]) __attribute__((always_inline)) {
        Piece<float> p;
        p.set(s);
#pragma unroll
        for (int q = 0; q < 2; q++) {
            uint32_t c;
            if (!at.at(i, Piece<T>::UNITS == 2 ? q : 0, c)) continue;
            store16<false>(a.parts + (size_t)blockIdx.x * a.cols + c + (Piece<T>::UNITS == 2 ? 0u : 4u * q), p.raw[q]);
        }
    };
    if (SPAN == SPAN_GROUP) {
#pragma unroll
        for (int i = 0; i < CH; i++) {
            if (STAGED) {
                Piece<float> d;
#pragma unroll
                for (int q = 0; q < 2; q++) d.raw[q] = staged[(2 * i + q) * (64 * NORM_WAVES)];
#pragma unroll
                for (int e = 0; e < 8; e++) dw[0][e] = d.get(e);
            }
            out(i, dw[STAGED ? 0 : i]);
        }
        return;
    }
    // the wavefronts' sums, and those of the rows that a wavefront has at once, in order
    if constexpr (SPAN != SPAN_GROUP) {
        const uint32_t wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
        piece_u32x4* const mine = (piece_u32x4*)dws + (threadIdx.x & 63u);
#pragma unroll
        for (int i = 0; i < CH; i++) {
            if (SPAN == SPAN_LANES) {
                for (uint32_t off = 32u; off >= lanes; off >>= 1)
#pragma unroll
                    for (int e = 0; e < 8; e++) dw[i][e] += __shfl_xor(dw[i][e], (int)off);
            }
            Piece<float> p;
            p.set(dw[i]);
#pragma unroll
            for (int q = 0; q < 2; q++) mine[((wave * CH + i) * 2u + q) * 64u] = p.raw[q];
        }
        __syncthreads();
        if (wave != 0u || (SPAN == SPAN_LANES && threadIdx.x >= lanes)) return;
#pragma unroll
        for (int i = 0; i < CH; i++) {
            for (uint32_t v = 1; v < waves; v++) {
                Piece<float> p;
#pragma unroll
                for (int q = 0; q < 2; q++) p.raw[q] = mine[((v * CH + i) * 2u + q) * 64u];
#pragma unroll
                for (int e = 0; e < 8; e++) dw[i][e] += p.get(e);
            }
            out(i, dw[i]);
        }
    }
}

// The parts' sums, 32 channels a workgroup, 32 parts at a time, in an order that depends on nothing.
template <typename T>
__global__ __launch_bounds__(1024) void norm_dw_kernel(const float* __restrict__ part, T* __restrict__ dw, uint32_t parts, uint32_t cols) {
    __shared__ float sums[32][33];
    const uint32_t lane = threadIdx.x & 31u, ty = threadIdx.x >> 5, n = blockIdx.x * 32u + lane;
    float s = 0.f;
    if (n < cols) {
#pragma unroll 8
        for (uint32_t p = ty; p < parts; p += 32u) s += part[(size_t)p * cols + n];
    }
    sums[ty][lane] = s;
    __syncthreads();
    // channel `ty`, over the lanes
    s = sums[lane][ty];
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) s += __shfl_xor(s, off);
    if (lane == 0u && blockIdx.x * 32u + ty < cols) dw[blockIdx.x * 32u + ty] = (T)s;
}

uint32_t norm_bwd_parts(uint32_t rows, uint32_t cols) { return norm_bwd_shape(rows, cols).parts; }

template <typename T, bool NT>
static hipError_t launch_bwd_t(const NormBwdArgs& a, hipStream_t stream) {
    const NormBwdShape s = norm_bwd_shape(a.n_rows, a.cols);
    if (s.span == SPAN_LANES) norm_bwd_kernel<T, SPAN_LANES, 1, NT><<<s.parts, s.threads, 0, stream>>>(a, s.lanes);
#define ROWS(SPAN, CH) \
    else if (s.span == SPAN && s.ch == CH) norm_bwd_kernel<T, SPAN, CH, NT><<<s.parts, s.threads, 0, stream>>>(a, 64u);
    ROWS(SPAN_WAVE, 1)
    ROWS(SPAN_WAVE, 2)
    ROWS(SPAN_GROUP, 1)
    ROWS(SPAN_GROUP, 2)
    ROWS(SPAN_GROUP, 4)
#undef ROWS
    else return hipErrorInvalidValue;
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.dw == nullptr) return e;
    norm_dw_kernel<T><<<(a.cols + 31u) / 32u, 1024, 0, stream>>>(a.parts, (T*)a.dw, s.parts, a.cols);
    return hipGetLastError();
}

hipError_t launch_norm_bwd(const NormBwdArgs& all, hipStream_t stream) {
    NormBwdArgs a = all;
    a.per_n = 1.f / (float)a.cols;
    a.chunks = (a.cols + 511u) / 512u;
    const uint64_t moved = (uint64_t)a.n_rows * a.cols * (a.f32 ? 4u : 2u) * (2u + (a.dx ? 1u : 0u) + (a.dx && a.dx_add ? 1u : 0u));
    if (moved >= NORM_PAST_CACHES) return a.f32 ? launch_bwd_t<float, true>(a, stream) : launch_bwd_t<__bf16, true>(a, stream);
    return a.f32 ? launch_bwd_t<float, false>(a, stream) : launch_bwd_t<__bf16, false>(a, stream);
}

}  // namespace skiparse

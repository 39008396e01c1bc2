// Rotary positions on the token grid: pair i of a head's channels is turned by the angle of its token's place along the pair's axis,
//     y0 = m (x0 cos - x1 sin),   y1 = m (x0 sin + x1 cos),   angle = place * f_i
// rt / 2 pairs for t, then rh / 2 for h, rw / 2 for w; the channels behind R = rt + rh + rw are copied.  The gradient is the transposed map, sin -> -sin.
//
// Bound by HBM bandwidth: q and k are read and written once, and the row move into or out of the sparse layout (Algorithm 1) that stands next to the rotation in a
// chain of sparse blocks is folded in.  Cosines and sines come from a table [T][rt/2], [H][rh/2], [W][rw/2] that stays in the caches; angles are formed in 64 bits
// when it is made, so that far positions cost nothing here.
//
// A wavefront has CH = head_dim / 8 lanes a head and as many heads at once as fit; a lane's place in the head, and with it its cosines, is the same in all
// rounds, so one look-up serves them.  Fewer heads than fit: several tokens a wavefront.  The pairs of the half layout lie R / 2 channels apart, in another
// lane's chunk: the wavefront passes its chunks through LDS, and reads whole chunks there where R / 2 is some of them (channel by channel 824 us instead of 649 in an earlier
// state, 80,640 tokens x 40 heads).  3.3 GB, q and k of that size into the sparse layout, take 587 us (5.6 TB/s; a plain copy 4.9).
#include "kernels.h"

namespace skiparse {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;

constexpr int ROPE_WAVES = 4;
// Rounds of a wavefront that are loaded at once, and wavefronts that are left where it takes more of them, so that one look-up of the cosines serves all (us, q and k of 80,640
// tokens x 40 heads into the sparse layout / half layout in place / 32,760 x 12 half layout; 4 rounds a look-up 595 / 614 / 84.3, as many as leave 16,384 wavefronts, 3 at
// once 599 / 594 / 75.1, 4 598 / 593 / 75.5, 5 587 / 582 / 75.4).
constexpr int ROPE_ITERS = 5;
constexpr uint64_t ROPE_MIN_WAVES = 16384;
// Tensors beyond this pass by the caches: what is smaller is still there when the next kernel reads it (us, cached / past: 110 MB moved 21.4 / 27.9, 400 MB 79.0 / 70.3, 1.6 GB 634 / 596).
constexpr uint64_t ROPE_CACHED_BYTES = 128ull << 20;
constexpr uint64_t ROPE_AT_ONCE = 1ull << 23;  // workgroups of a launch: a grid has less than 2^32 threads

struct RopeDev {
    const void* x[2];
    void* y[2];
    const f32x2* table;
    RowArgs rows;            // source row of a destination row
    Div32 n_tok, hw, w;      // tokens of a grid, of a frame, of a line
    Div32 parts;             // wavefronts a token (or group of tokens)
    uint32_t n_rows, heads, ch, per_wave;  // per_wave: heads at once
    uint32_t tokens;         // tokens a wavefront
    uint32_t rounds;         // rounds of one tensor over its heads; those of the second follow
    uint32_t total_rounds, rounds_per_wave;
    uint32_t R, head_dim;
    uint32_t end_t, end_h;   // pairs below end_t turn with t, below end_h with h
    uint32_t n_t, n_h, n_w;  // pairs of an axis
    uint32_t off_t, off_h, off_w;  // where an axis begins in the table, places before the grid's first left out, minus its first pair
    float sign;
    uint32_t first;          // workgroup that a launch begins with
};

template <typename T>
struct Chunk;
template <>
struct Chunk<__bf16> {
    static constexpr int N = 1;  // 16-byte pieces of 8 channels
    __device__ static inline float get(const u32x4 (&p)[1], int e) { return __uint_as_float(e & 1 ? p[0][e >> 1] & 0xffff0000u : p[0][e >> 1] << 16); }
    __device__ static inline void put(u32x4 (&p)[1], const float (&v)[8], uint32_t turned) {
        typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const bf16x2 b = {(__bf16)v[2 * e], (__bf16)v[2 * e + 1]};
            const uint32_t u = __builtin_bit_cast(uint32_t, b);
            const uint32_t mask = (turned >> (2 * e) & 1u ? 0xffffu : 0u) | (turned >> (2 * e + 1) & 1u ? 0xffff0000u : 0u);
            p[0][e] = (u & mask) | (p[0][e] & ~mask);
        }
    }
    __device__ static inline float at(const char* row, uint32_t c) { return __uint_as_float((uint32_t)((const unsigned short*)row)[c] << 16); }
};
template <>
struct Chunk<float> {
    static constexpr int N = 2;
    __device__ static inline float get(const u32x4 (&p)[2], int e) { return __uint_as_float(p[e >> 2][e & 3]); }
    __device__ static inline void put(u32x4 (&p)[2], const float (&v)[8], uint32_t turned) {
#pragma unroll
        for (int e = 0; e < 8; e++)
            if (turned >> e & 1u) p[e >> 2][e & 3] = __float_as_uint(v[e]);
    }
    __device__ static inline float at(const char* row, uint32_t c) { return ((const float*)row)[c]; }
};

// MAP: which way rows go; a move within the sparse layout (ROPE_STAY) and within the original order have source row = destination row.
enum RopeMap : int { ROPE_SAME = 0, ROPE_TO_SPARSE = 1, ROPE_TO_ORIGINAL = 2, ROPE_STAY = 3 };

// How a head's pairs lie: next to each other, R / 2 apart by whole chunks, R / 2 apart anyhow.
enum RopePairs : int { PAIRS_NEXT = 0, PAIRS_CHUNKS = 1, PAIRS_APART = 2 };

template <typename T, int MAP, int PAIRS, bool NT>
__global__ __launch_bounds__(64 * ROPE_WAVES) void rope_kernel(RopeDev a) {
    using C = Chunk<T>;
    constexpr bool HALF = PAIRS != PAIRS_NEXT;
    __shared__ __attribute__((aligned(16))) char stage_all[HALF ? ROPE_WAVES * 64 * 16 * C::N : 16];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t id = (a.first + blockIdx.x) * ROPE_WAVES + wave;
    const uint32_t group = a.parts.div(id), part = id - group * a.parts.d;
    const uint32_t row0 = group * a.tokens;
    if (row0 >= a.n_rows) return;  // a whole wavefront
    const uint32_t sub = lane / a.ch, c = lane - sub * a.ch;  // head (and token) of the wavefront's, chunk of the head
    const uint32_t tk = a.tokens > 1u ? sub / a.heads : 0u, head0 = a.tokens > 1u ? sub - tk * a.heads : sub;
    const uint32_t row = row0 + tk;
    const bool lane_on = sub < a.per_wave && tk < a.tokens && row < a.n_rows;

    // source row, and the token's place in the original order
    uint32_t src = row, n = row;
    if (lane_on) {
        if (MAP == ROPE_TO_SPARSE || MAP == ROPE_STAY) n = source_row<TO_SPARSE>(a.rows, row, 0u);
        if (MAP == ROPE_TO_SPARSE) src = n;
        if (MAP == ROPE_TO_ORIGINAL) src = source_row<TO_ORIGINAL>(a.rows, row, 0u);
    }
    const uint64_t row_len = (uint64_t)a.heads * a.head_dim;
    u32x4 p[ROPE_ITERS][C::N];
    // where the lane's chunk of round r lies in its token's row; false: none of the wavefront's
    auto place = [&](uint32_t r, uint32_t& second, uint64_t& at) __attribute__((always_inline)) -> bool {
        second = r >= a.rounds ? 1u : 0u;
        const uint32_t head = head0 + (r - second * a.rounds) * a.per_wave;
        at = (uint64_t)head * a.head_dim + c * 8u;
        return lane_on && r < a.total_rounds && head < a.heads;
    };
    // all loads of ROPE_ITERS rounds at once
    auto load = [&](uint32_t first) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < ROPE_ITERS; i++) {
            uint32_t second;
            uint64_t at;
            if (!place(first + i, second, at)) continue;
            const u32x4* from = (const u32x4*)((const T*)a.x[second] + (uint64_t)src * row_len + at);
#pragma unroll
            for (int j = 0; j < C::N; j++) p[i][j] = NT ? __builtin_nontemporal_load(from + j) : from[j];
        }
    };
    const uint32_t first = part * a.rounds_per_wave, end = first + a.rounds_per_wave < a.total_rounds ? first + a.rounds_per_wave : a.total_rounds;
    load(first);
    // the cosines and sines of the lane's channels
    const uint32_t in_grid = n - a.n_tok.div(n) * a.n_tok.d;
    const uint32_t t = a.hw.div(in_grid), in_frame = in_grid - t * a.hw.d, h = a.w.div(in_frame), w = in_frame - h * a.w.d;
    constexpr int NP = HALF ? 8 : 4;
    float cs[NP], sn[NP];
    const uint32_t half = a.R >> 1;
    uint32_t turned = 0u;  // bit e: channel e of the chunk is turned
#pragma unroll
    for (int e = 0; e < NP; e++) {
        const uint32_t ch = HALF ? c * 8u + e : c * 8u + 2 * e;
        const bool in = ch < a.R;
        if (in) turned |= HALF ? 1u << e : 3u << (2 * e);
        uint32_t i = HALF ? (ch < half ? ch : ch - half) : ch >> 1;
        if (!in) i = 0u;
        const uint32_t k = i < a.end_t ? a.off_t + t * a.n_t + i : i < a.end_h ? a.off_h + h * a.n_h + i : a.off_w + w * a.n_w + i;
        cs[e] = 1.f;
        sn[e] = 0.f;
        if (lane_on) {
            const f32x2 v = a.table[k];
            cs[e] = v[0];
            sn[e] = (HALF && ch < half ? -a.sign : a.sign) * v[1];
        }
    }
    char* const stage = HALF ? stage_all + wave * (64 * 16 * C::N) : nullptr;
    for (uint32_t r0 = first;;) {
#pragma unroll
        for (int i = 0; i < ROPE_ITERS; i++) {
            const uint32_t r = r0 + i;
            if (r >= end) break;  // a whole wavefront
            uint32_t second;
            uint64_t at;
            const bool on = place(r, second, at);
            float v[8];
            if (HALF) {
                // other lanes may have read the region last; the wavefront's LDS accesses take effect in order
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int j = 0; j < C::N; j++) *(u32x4*)(stage + lane * (16 * C::N) + 16 * j) = p[i][j];
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
                const char* const head = stage + (lane - c) * (16 * C::N);
                if (PAIRS == PAIRS_CHUNKS) {
                    const uint32_t hc = half >> 3, oc = !lane_on || c >= 2u * hc ? c : c < hc ? c + hc : c - hc;
                    u32x4 o[C::N];
#pragma unroll
                    for (int j = 0; j < C::N; j++) o[j] = *(const u32x4*)(head + oc * (16 * C::N) + 16 * j);
#pragma unroll
                    for (int e = 0; e < 8; e++) v[e] = C::get(p[i], e) * cs[e] + C::get(o, e) * sn[e];
                } else {
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        const uint32_t ch = c * 8u + e, other = !lane_on || ch >= a.R ? ch : ch < half ? ch + half : ch - half;
                        v[e] = C::get(p[i], e) * cs[e] + C::at(head, other) * sn[e];
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const float x0 = C::get(p[i], 2 * e), x1 = C::get(p[i], 2 * e + 1);
                    v[2 * e] = x0 * cs[e] - x1 * sn[e];
                    v[2 * e + 1] = x0 * sn[e] + x1 * cs[e];
                }
            }
            C::put(p[i], v, turned);
            if (on) {
                u32x4* to = (u32x4*)((T*)a.y[second] + (uint64_t)row * row_len + at);
#pragma unroll
                for (int j = 0; j < C::N; j++) {
                    if (NT) __builtin_nontemporal_store(p[i][j], to + j);
                    else to[j] = p[i][j];
                }
            }
        }
        r0 += ROPE_ITERS;
        if (r0 >= end) break;
        load(r0);
    }
}

template <typename T, int PAIRS, bool NT>
static hipError_t launch_rope_t(const RopeDev& d, int map, uint32_t blocks, hipStream_t stream) {
    switch (map) {
        case ROPE_SAME: rope_kernel<T, ROPE_SAME, PAIRS, NT><<<blocks, 64 * ROPE_WAVES, 0, stream>>>(d); break;
        case ROPE_TO_SPARSE: rope_kernel<T, ROPE_TO_SPARSE, PAIRS, NT><<<blocks, 64 * ROPE_WAVES, 0, stream>>>(d); break;
        case ROPE_TO_ORIGINAL: rope_kernel<T, ROPE_TO_ORIGINAL, PAIRS, NT><<<blocks, 64 * ROPE_WAVES, 0, stream>>>(d); break;
        default: rope_kernel<T, ROPE_STAY, PAIRS, NT><<<blocks, 64 * ROPE_WAVES, 0, stream>>>(d); break;
    }
    return hipGetLastError();
}
template <typename T>
static hipError_t launch_rope_t(const RopeDev& d, int map, int pairs, bool nt, uint32_t blocks, hipStream_t stream) {
    if (pairs == PAIRS_NEXT) return nt ? launch_rope_t<T, PAIRS_NEXT, true>(d, map, blocks, stream) : launch_rope_t<T, PAIRS_NEXT, false>(d, map, blocks, stream);
    if (pairs == PAIRS_CHUNKS) return nt ? launch_rope_t<T, PAIRS_CHUNKS, true>(d, map, blocks, stream) : launch_rope_t<T, PAIRS_CHUNKS, false>(d, map, blocks, stream);
    return launch_rope_t<T, PAIRS_APART, false>(d, map, blocks, stream);
}

hipError_t launch_rope(const RopeArgs& r, hipStream_t stream) {
    RopeDev d = {};
    d.x[0] = r.q;
    d.x[1] = r.k;
    d.y[0] = r.q_out;
    d.y[1] = r.k_out;
    d.table = (const f32x2*)r.table;
    const uint32_t T = (uint32_t)r.T, H = (uint32_t)r.H, W = (uint32_t)r.W;
    d.rows = r.order == ROPE_TO_ORIGINAL ? make_row_args<TO_ORIGINAL>(r.g, (uint32_t)r.B) : make_row_args<TO_SPARSE>(r.g, (uint32_t)r.B);
    d.n_tok = make_div32(T * H * W);
    d.hw = make_div32(H * W);
    d.w = make_div32(W);
    d.n_rows = (uint32_t)r.B * T * H * W;
    d.heads = (uint32_t)r.heads;
    d.head_dim = (uint32_t)r.head_dim;
    d.ch = d.head_dim / 8u;
    d.per_wave = 64u / d.ch;
    d.tokens = 1u;
    if (d.heads < d.per_wave) {
        d.tokens = d.per_wave / d.heads;
        d.per_wave = d.tokens * d.heads;
    }
    d.rounds = d.tokens > 1u ? 1u : (d.heads + d.per_wave - 1u) / d.per_wave;
    d.total_rounds = d.rounds * (r.k ? 2u : 1u);
    // a look-up of the cosines serves as many rounds as leave ROPE_MIN_WAVES wavefronts
    const uint64_t groups = ((uint64_t)d.n_rows + d.tokens - 1u) / d.tokens;
    const uint32_t fours = (d.total_rounds + ROPE_ITERS - 1u) / ROPE_ITERS;
    uint64_t per = groups * fours / ROPE_MIN_WAVES;
    per = per < 1u ? 1u : per < fours ? per : fours;
    d.rounds_per_wave = (uint32_t)per * ROPE_ITERS;
    const uint32_t parts = (d.total_rounds + d.rounds_per_wave - 1u) / d.rounds_per_wave;
    d.parts = make_div32(parts);
    d.R = (uint32_t)(r.rt + r.rh + r.rw);
    d.n_t = (uint32_t)r.rt / 2u;
    d.n_h = (uint32_t)r.rh / 2u;
    d.n_w = (uint32_t)r.rw / 2u;
    d.end_t = d.n_t;
    d.end_h = d.n_t + d.n_h;
    // an axis begins with place t0 of its table; minus its first pair, since i counts the pairs of all axes (modulo 2^32)
    d.off_t = (uint32_t)r.t0 * d.n_t;
    d.off_h = (uint32_t)r.len_t * d.n_t + (uint32_t)r.h0 * d.n_h - d.end_t;
    d.off_w = (uint32_t)r.len_t * d.n_t + (uint32_t)r.len_h * d.n_h + (uint32_t)r.w0 * d.n_w - d.end_h;
    d.sign = r.inverse ? -1.f : 1.f;
    const uint64_t blocks = (groups * parts + ROPE_WAVES - 1u) / ROPE_WAVES;
    const int pairs = !r.half ? PAIRS_NEXT : d.R % 16u == 0 ? PAIRS_CHUNKS : PAIRS_APART;
    const uint64_t bytes = (uint64_t)d.n_rows * d.heads * d.head_dim * (r.f32 ? 4u : 2u) * (r.k ? 2u : 1u);
    const bool nt = bytes > ROPE_CACHED_BYTES;
    static_assert(ROPE_AT_ONCE * 64 * ROPE_WAVES < 1ull << 32, "a grid");
    for (uint64_t first = 0; first < blocks; first += ROPE_AT_ONCE) {
        d.first = (uint32_t)first;
        const uint32_t n = (uint32_t)(blocks - first < ROPE_AT_ONCE ? blocks - first : ROPE_AT_ONCE);
        const hipError_t e = r.f32 ? launch_rope_t<float>(d, r.order, pairs, nt, n, stream) : launch_rope_t<__bf16>(d, r.order, pairs, nt, n, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// ---- the table

// Frequency of pair j of an axis of r channels, in turns (2 pi) a place.
__device__ inline double rope_turns(const RopeAxis& x, const RopeScaling& s, uint32_t j) {
    const double r = (double)x.r;
    double base = s.theta;
    if (s.kind == ROPE_NTK && x.r > 2) base *= pow(x.factor, r / (r - 2.0));
    double f = pow(base, -2.0 * (double)j / r) * 0.15915494309189533577;  // 1 / (2 pi)
    if (s.kind == ROPE_LINEAR) f /= x.factor;
    if (s.kind == ROPE_YARN) {
        // by how often the pair turns within the trained length: often -> as it is, seldom -> stretched, linear in between (YaRN, "NTK-by-parts")
        const double turns = (double)x.trained * f;
        double g = (turns - s.slow) / (s.fast - s.slow);
        g = g < 0.0 ? 0.0 : g > 1.0 ? 1.0 : g;
        f = f * g + f / x.factor * (1.0 - g);
    }
    return f;
}

constexpr uint32_t ROPE_TABLE_THREADS = 256;
constexpr uint32_t ROPE_TABLE_BLOCKS = 1024;  // at most, of an axis: a workgroup forms its axis' frequencies anew, which takes as long as some thousand entries

// One launch a table.  Angles are reduced in 64 bits to an eighth of a turn either way and the quadrant; sine and cosine of what is left are taken in 32 by their series, whose
// first terms left out are 2e-9 and 1e-10 at the eighth.  Bound by the arithmetic: 131,072 x 64 pairs, 67 MB, 15.5 us (with the library's functions and eight entries a thread 22).
__global__ __launch_bounds__(ROPE_TABLE_THREADS) void rope_table_kernel(f32x2* table, RopeAxis t, RopeAxis h, RopeAxis w, RopeScaling s) {
    __shared__ double freq[ROPE_MAX_PAIRS];
    const RopeAxis x = blockIdx.x < t.blocks ? t : blockIdx.x < t.blocks + h.blocks ? h : w;
    const uint32_t block = blockIdx.x - (blockIdx.x < t.blocks ? 0u : blockIdx.x < t.blocks + h.blocks ? t.blocks : t.blocks + h.blocks);
    const uint32_t pairs = x.r / 2u;
    for (uint32_t j = threadIdx.x; j < pairs; j += ROPE_TABLE_THREADS) freq[j] = rope_turns(x, s, j);
    __syncthreads();
    const uint32_t n = x.len * pairs;  // below 2^31
    for (uint32_t i = block * ROPE_TABLE_THREADS + threadIdx.x; i < n; i += x.blocks * ROPE_TABLE_THREADS) {
        const uint32_t place = x.pairs.div(i), j = i - place * pairs;
        const double turns = (double)place * freq[j], q = rint(turns * 4.0);
        const float g = (float)((turns - q * 0.25) * 6.283185307179586477), g2 = g * g;
        const float sn = g * fmaf(g2, fmaf(g2, fmaf(g2, fmaf(g2, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
        const float cs = fmaf(g2, fmaf(g2, fmaf(g2, fmaf(g2, fmaf(g2, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
        const int quadrant = (int)(uint32_t)(long long)q & 3;
        const float c0 = quadrant & 1 ? sn : cs, s0 = quadrant & 1 ? cs : sn;
        const float c1 = quadrant == 1 || quadrant == 2 ? -c0 : c0, s1 = quadrant >= 2 ? -s0 : s0;
        table[x.first + i] = f32x2{c1 * s.attention, s1 * s.attention};
    }
}

hipError_t launch_rope_table(float* table, RopeAxis t, RopeAxis h, RopeAxis w, const RopeScaling& s, hipStream_t stream) {
    uint32_t first = 0;
    uint64_t blocks = 0;
    for (RopeAxis* x : {&t, &h, &w}) {
        const uint32_t n = x->len * (x->r / 2u);
        x->first = first;
        x->blocks = (n + ROPE_TABLE_THREADS - 1u) / ROPE_TABLE_THREADS;
        if (x->blocks > ROPE_TABLE_BLOCKS) x->blocks = ROPE_TABLE_BLOCKS;
        x->pairs = make_div32(x->r ? x->r / 2u : 1u);
        first += n;
        blocks += x->blocks;
    }
    if (!fits_grid(blocks, ROPE_TABLE_THREADS)) return hipErrorInvalidConfiguration;
    rope_table_kernel<<<(uint32_t)blocks, ROPE_TABLE_THREADS, 0, stream>>>((f32x2*)table, t, h, w, s);
    return hipGetLastError();
}

}  // namespace skiparse

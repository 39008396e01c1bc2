// Products of the linear layer on the matrix cores, bf16 in and out, float32 sums: C[m][n] = sum_k P(m, k) Q(n, k), and its epilogue
//     z = C + bias (kept, if asked for, in bf16 or as an 8-bit checkpoint),  out = act(z) + residual
// Three forms:  out = x w^T (neither operand transposed),  dx = dz w (Q = w given as [k][n]),  dw = dz^T x (both given as [k][..]).
//
//   * The MFMA takes Q's rows as its A operand and P's as B, so that a lane's accumulators are 16 channels of ONE row of C: bias, residual and the blocks of a
//     checkpoint are its own.
//   * Tiles go from memory straight into LDS (buffer_load_dwordx4 ... lds), 64 of k a step, double buffered.  Operands with k along the row are laid out in rows of
//     128 bytes and read 16 bytes at a time; transposed ones in rows of 256 and read with ds_read_b64_tr_b16; swizzles as in lds_layout.h.
//   * Ends: a 16-byte piece behind the end of k is given an offset outside the buffer and reads as zero; transposed operands end with the buffer; rows
//     past the last read the last one, columns past the last whatever lies there, and neither is stored.
#include <type_traits>

#include "checkpoint.h"
#include "kernels.h"
#include "lds_layout.h"
#include "linear_act.h"

namespace skiparse {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;

#define LDS_PTR(T) __attribute__((address_space(3))) T*

constexpr uint32_t LIN_KT = 64;           // of k a step
constexpr uint32_t LIN_OUTSIDE = ~0u;     // an offset outside every buffer
constexpr uint32_t LIN_RECORDS = 0xfffffff0u;

// One operand's side of a workgroup's tile: ROWS of m (or n) by 64 of k.
template <int ROWS, bool T, int NW>
struct Side {
    static constexpr int INSTR = ROWS * 128 / 1024 / NW;  // direct loads of a wavefront and step, 1 KiB each
    static constexpr int BYTES = ROWS * 128;
    uint32_t off[INSTR];  // of the lane's piece from the step's base
    uint32_t kofs[INSTR]; // !T: where in the step's k it lies
    // row_off: byte offset of row r of the tile from the base (!T), row_bytes: of a row of k (T)
    template <typename F>
    __device__ __attribute__((always_inline)) inline void init(uint32_t wave, uint32_t lane, uint32_t row_bytes, F row_off) {
#pragma unroll
        for (int i = 0; i < INSTR; i++) {
            const uint32_t n = wave * INSTR + i;  // of the tile's
            if (!T) {
                const uint32_t r = n * 8u + lane / 8u;
                kofs[i] = ((lane % 8u) ^ lds_swizzle<64>(r)) * 8u;
                off[i] = row_off(r) + kofs[i] * 2u;
            } else {
                const uint32_t part = n / 16u, r = n % 16u * 4u + lane / 16u;  // 128 columns a part
                kofs[i] = 0u;
                off[i] = r * row_bytes + part * 256u + ((lane % 16u) ^ lds_swizzle<128>(r)) * 16u;
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

// Fragment of 32 rows from `row0` (a multiple of 32) and 16 of k: lane l has row l % 32, k = 16 ks + 8 (l / 32) ...
template <bool T>
__device__ __attribute__((always_inline)) inline bf16x8 read_fragment(const char* buf, uint32_t row0, uint32_t ks, uint32_t lane) {
    const uint32_t h = lane >> 5;
    if (!T) {
        const uint32_t r = lane & 31u;
        return *(const bf16x8*)(buf + (row0 + r) * 128u + ((2u * ks + h) ^ lds_swizzle<64>(r)) * 16u);
    }
    const uint32_t li = lane & 15u, group = lane >> 4 & 1u;
    const char* const part = buf + row0 / 128u * 16384u;
    bf16x4 v[2];
#pragma unroll
    for (uint32_t sec = 0; sec < 2; sec++) {
        const uint32_t r = 16u * ks + 8u * h + 4u * sec + (li >> 2);
        const uint32_t c = row0 % 128u / 8u + group * 2u + ((li & 3u) >> 1);
        const char* const at = part + r * 256u + ((c ^ lds_swizzle<128>(r)) * 16u) + 8u * (li & 1u);
        v[sec] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(LDS_PTR(char))at);
    }
    return __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
}

// Workgroup -> tile.  Workgroup id % 8 is the XCD; each XCD has a contiguous range of an order in which TILE_GROUP tiles of m are walked together along n, so that the 32
// tiles that it works on at once share operands in its L2.
constexpr uint32_t TILE_GROUP = 8;
struct TileMap {
    Div32 group;   // tiles of a group: TILE_GROUP * tiles_n
    Div32 size, last;  // tiles of m in a group, in the last one
    uint32_t tiles_m, total, per_xcd;
    __device__ inline void at(uint32_t id, uint32_t& tm, uint32_t& tn) const {
        const uint32_t xcd = id & 7u, rest = total & 7u;  // the first `rest` XCDs have one tile more
        const uint32_t lin = xcd * per_xcd + (xcd < rest ? xcd : rest) + (id >> 3);
        const uint32_t g = group.div(lin), in = lin - g * group.d, first = g * TILE_GROUP;
        const bool full = first + TILE_GROUP <= tiles_m;
        const uint32_t n = full ? size.div(in) : last.div(in);
        tn = n;
        tm = first + in - n * (full ? size.d : last.d);
    }
};
static TileMap make_tile_map(uint32_t tiles_m, uint32_t tiles_n) {
    const uint32_t rest = tiles_m % TILE_GROUP;
    return {make_div32(TILE_GROUP * tiles_n), make_div32(TILE_GROUP), make_div32(rest ? rest : 1u), tiles_m, tiles_m * tiles_n, tiles_m * tiles_n / 8u};
}

// The way out: 32 rows by 32 FN channels of C at a time, a wavefront's own.  The sums are laid down in LDS as they are (float32: a residual is added before the one
// rounding) and picked up 8 channels of a row a lane, so that everything in memory is moved in 16-byte pieces of whole rows, and a checkpoint's blocks are four
// neighbouring lanes.
template <int FN>
struct Out {
    static constexpr uint32_t LPR = FN * 4, RPI = 64 / LPR;  // lanes a row, rows at once
    uint32_t n;      // the lane's channels n .. n + 7
    bool in;
    float bias[8];
    __device__ __attribute__((always_inline)) inline Out(const LinearArgs& a, uint32_t n0, uint32_t lane) {
        n = n0 + lane % LPR * 8u;
        in = n < a.N;
#pragma unroll
        for (int e = 0; e < 8; e++) bias[e] = 0.f;
        if (a.e.bias != nullptr && in) {
            const bf16x8 b = *(const bf16x8*)((const __bf16*)a.e.bias + n);
#pragma unroll
            for (int e = 0; e < 8; e++) bias[e] = (float)b[e];
        }
    }
    // 16-byte piece c of row r lies at c ^ (r % 16): 8 lanes that write (8 rows) or read (a row) touch different banks
    __device__ __attribute__((always_inline)) inline static uint32_t place(uint32_t r, uint32_t c) { return r * (FN * 128u) + ((c ^ (r & (FN == 4 ? 15u : 7u))) * 16u); }
    __device__ __attribute__((always_inline)) inline void lay_down(char* stage, const f32x16 (&acc)[FN], uint32_t lane) const {
        const uint32_t r = lane & 31u, h = lane >> 5;
        // the wavefront's LDS accesses take effect in order; the fences keep the compiler from exchanging them
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < FN; j++)
#pragma unroll
            for (int g = 0; g < 4; g++)
                *(f32x4*)(stage + place(r, j * 8u + g * 2u + h)) = f32x4{acc[j][4 * g], acc[j][4 * g + 1], acc[j][4 * g + 2], acc[j][4 * g + 3]};
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    __device__ __attribute__((always_inline)) inline void rows(const char* stage, const LinearArgs& a, uint32_t m0, uint32_t lane) const {
#pragma unroll
        for (uint32_t it = 0; it < 32u / RPI; it++) {
            const uint32_t r = it * RPI + lane / LPR, c = lane % LPR * 2u;
            const f32x4 x = *(const f32x4*)(stage + place(r, c)), y = *(const f32x4*)(stage + place(r, c + 1u));
            const float z[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
            finish(a, m0 + r, z);
        }
    }
    // row m, the lane's channels: act(z + bias) + residual; z + bias kept
    __device__ __attribute__((always_inline)) inline void finish(const LinearArgs& a, uint32_t m, const float (&sum)[8]) const {
        typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
        const LinearEpilogue& e = a.e;
        const bool here = in && m < a.M;
        const size_t at = (size_t)m * a.N + n;
        float z[8];
#pragma unroll
        for (int i = 0; i < 8; i++) z[i] = sum[i] + bias[i];
        if (e.pre_scales != nullptr) {
            uint32_t top = 0u;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const uint32_t s = in ? ckpt_size(z[i]) : 0u;
                top = s > top ? s : top;
            }
#pragma unroll
            for (int off = 1; off <= 2; off <<= 1) {
                const uint32_t o = (uint32_t)__shfl_xor((int)top, off);
                top = o > top ? o : top;
            }
            const uint32_t byte = ckpt_byte(top);
            const float down = ckpt_down(byte);
            if (here) {
                *(u32x2*)((char*)e.pre + at) = u32x2{ckpt_codes(z[0], z[1], z[2], z[3], down), ckpt_codes(z[4], z[5], z[6], z[7], down)};
                if (n % CKPT_BLOCK == 0u) ((unsigned char*)e.pre_scales)[(size_t)m * ((a.N + CKPT_BLOCK - 1u) / CKPT_BLOCK) + n / CKPT_BLOCK] = (unsigned char)byte;
            }
        }
        if (!here) return;
        if (e.pre != nullptr && e.pre_scales == nullptr) {
            bf16x8 o;
#pragma unroll
            for (int i = 0; i < 8; i++) o[i] = (__bf16)z[i];
            *(bf16x8*)((__bf16*)e.pre + at) = o;
        }
        if (e.act != ACT_NONE) {
#pragma unroll
            for (int i = 0; i < 8; i++) z[i] = act_value(e.act, z[i]);
        }
        if (e.residual != nullptr) {
            const bf16x8 r = *(const bf16x8*)((const __bf16*)e.residual + at);
#pragma unroll
            for (int i = 0; i < 8; i++) z[i] += (float)r[i];
        }
        bf16x8 o;
#pragma unroll
        for (int i = 0; i < 8; i++) o[i] = (__bf16)z[i];
        *(bf16x8*)((__bf16*)e.out + at) = o;
    }
};

template <int BM, int BN, int FORM>
__global__ __launch_bounds__(256, BM * BN == 256 * 256 ? 1 : 2) void linear_kernel(LinearArgs a, TileMap tiles) {
    constexpr bool PT = FORM == LINEAR_DW, QT = FORM != LINEAR_FWD;
    constexpr int NW = 4, FM = BM / 64, FN = BN / 64;  // wavefronts 2 x 2; blocks of 32 that each has
    using SP = Side<BM, PT, NW>;
    using SQ = Side<BN, QT, NW>;
    // separate arrays: the compiler must be able to tell that the tile being filled is not the tile being read
    __shared__ __attribute__((aligned(1024))) char pbuf0[SP::BYTES];
    __shared__ __attribute__((aligned(1024))) char pbuf1[SP::BYTES];
    __shared__ __attribute__((aligned(1024))) char qbuf0[SQ::BYTES];
    __shared__ __attribute__((aligned(1024))) char qbuf1[SQ::BYTES];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = wave & 1u, wn = wave >> 1;
    uint32_t tm, tn;
    tiles.at(blockIdx.x, tm, tn);
    const uint32_t m0 = tm * BM, n0 = tn * BN;
    const uint32_t ldp = (PT ? a.M : a.K) * 2u, ldq = (QT ? a.N : a.K) * 2u;  // bytes
    const bool mapped = FORM == LINEAR_FWD && a.order != 0;
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
        if (k >= a.K) return 0u;
        if (!t) return LIN_RECORDS;
        const uint64_t left = (uint64_t)(a.K - k) * ld - col0 * 2u;
        return left < LIN_RECORDS ? (uint32_t)left : LIN_RECORDS;
    };
    constexpr int LOADS = SP::INSTR + SQ::INSTR;
    struct Step {
        const char *p, *q;
        uint32_t rp, rq, left;
    };
    auto step_at = [&](uint32_t k) __attribute__((always_inline)) -> Step {
        return {p0 + (PT ? (size_t)k * ldp : (size_t)k * 2u), q0 + (QT ? (size_t)k * ldq : (size_t)k * 2u), records(PT, k, ldp, m0), records(QT, k, ldq, n0), k < a.K ? a.K - k : 0u};
    };
    auto load = [&](const Step& s, char* pb, char* qb, int i) __attribute__((always_inline)) {
        if (i < SP::INSTR) sp.issue(i, s.p, s.rp, s.left, pb, wave);
        else sq.issue(i - SP::INSTR, s.q, s.rq, s.left, qb, wave);
    };
    f32x16 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; i++)
#pragma unroll
        for (int j = 0; j < FN; j++)
#pragma unroll
            for (int r = 0; r < 16; r++) acc[i][j][r] = 0.f;
    struct Frags {
        bf16x8 p[FM], q[FN];
    };
    // fragment n in the order of use: the first of P, all of Q, the others of P
    auto fragment = [&](Frags& f, const char* pb, const char* qb, uint32_t ks, int n) __attribute__((always_inline)) {
        if (n == 0) f.p[0] = read_fragment<PT>(pb, (wm * FM) * 32u, ks, lane);
        else if (n <= FN) f.q[n - 1] = read_fragment<QT>(qb, (wn * FN + n - 1) * 32u, ks, lane);
        else f.p[n - FN] = read_fragment<PT>(pb, (wm * FM + n - FN) * 32u, ks, lane);
    };
    // 16 of k: the products of `f`, and between them the reads of what comes next and, with LOAD, a whole step's loads
    constexpr int MF = FM * FN, RD = FM + FN;
    auto sixteen = [&](auto LOADC, const Frags& f, Frags& next, const char* pb, const char* qb, uint32_t ks, const Step& s, char* pl, char* ql) __attribute__((always_inline)) {
        constexpr bool LOAD = decltype(LOADC)::value;
#pragma unroll
        for (int g = 0; g < MF; g++) {
            acc[g / FN][g % FN] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.q[g % FN], f.p[g / FN], acc[g / FN][g % FN], 0, 0, 0);
#pragma unroll
            for (int n = 0; n < RD; n++)
                if (n * MF / RD == g) fragment(next, pb, qb, ks, n);
            if (LOAD) {
#pragma unroll
                for (int i = 0; i < LOADS; i++)
                    if (i * MF / LOADS == g) load(s, pl, ql, i);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    using No = std::integral_constant<bool, false>;
    using Yes = std::integral_constant<bool, true>;
    Frags f0, f1;
    // A step of 64 on the tile in (pc, qc), whose first fragments are in f0.  Its last 16 of k are worked on behind the barrier, from registers: (pc, qc) is free then for the
    // tile after the next, and the next one, in (pn, qn), has landed.
    auto step = [&](uint32_t k, char* pc, char* qc, char* pn, char* qn) __attribute__((always_inline)) {
        const Step s = step_at(k + 2u * LIN_KT);
        sixteen(No{}, f0, f1, pc, qc, 1, s, pc, qc);
        sixteen(No{}, f1, f0, pc, qc, 2, s, pc, qc);
        sixteen(No{}, f0, f1, pc, qc, 3, s, pc, qc);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        sixteen(Yes{}, f1, f0, pn, qn, 0, s, pc, qc);
    };
    const Step first = step_at(0), second = step_at(LIN_KT);
#pragma unroll
    for (int i = 0; i < LOADS; i++) load(first, pbuf0, qbuf0, i);
#pragma unroll
    for (int i = 0; i < LOADS; i++) load(second, pbuf1, qbuf1, i);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");
    __builtin_amdgcn_s_barrier();
#pragma unroll
    for (int n = 0; n < RD; n++) fragment(f0, pbuf0, qbuf0, 0, n);
    for (uint32_t k = 0; k < a.K; k += 2u * LIN_KT) {  // a second step behind the end adds zeros
        step(k, pbuf0, qbuf0, pbuf1, qbuf1);
        step(k + LIN_KT, pbuf1, qbuf1, pbuf0, qbuf0);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // loads behind the end still write (zeros) to LDS
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    // the epilogue, 32 rows of the wavefront at a time, through LDS
    char* const stage = wave == 0u ? pbuf0 : wave == 1u ? pbuf1 : wave == 2u ? qbuf0 : qbuf1;
    Out<FN> out(a, n0 + wn * (FN * 32u), lane);
#pragma unroll
    for (int i = 0; i < FM; i++) {
        out.lay_down(stage, acc[i], lane);
        out.rows(stage, a, m0 + (wm * FM + i) * 32u, lane);
        __builtin_amdgcn_sched_barrier(0);
    }
}

template <int FORM>
static hipError_t launch_form(const LinearArgs& a, hipStream_t stream) {
    constexpr int BM = 256, BN = 256;
    const uint32_t tiles_m = (a.M + BM - 1u) / BM, tiles_n = (a.N + BN - 1u) / BN;
    if (!fits_grid((uint64_t)tiles_m * tiles_n, 256u)) return hipErrorInvalidConfiguration;
    linear_kernel<BM, BN, FORM><<<tiles_m * tiles_n, 256, 0, stream>>>(a, make_tile_map(tiles_m, tiles_n));
    return hipGetLastError();
}

hipError_t launch_linear(int form, const LinearArgs& a, hipStream_t stream) {
    switch (form) {
        case LINEAR_FWD: return launch_form<LINEAR_FWD>(a, stream);
        case LINEAR_DX: return launch_form<LINEAR_DX>(a, stream);
        default: return launch_form<LINEAR_DW>(a, stream);
    }
}

}  // namespace skiparse

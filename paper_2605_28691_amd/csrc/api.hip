// C ABI of the library: argument validation and dispatch.  Everything is checked before the first HIP call, so the
// error paths run on a host without a GPU.
#include "../../include/skiparse.h"

#include <stdint.h>

#include <initializer_list>
#include <mutex>

#include "kernels.h"
#include "linear_plan.h"

using namespace skiparse;

// Scratch of skiparse_attn_bwd_static (the backward pass for callers that cannot allocate): the delta array, one float per
// (subsequence, head, position).  Every GPU the library runs on holds its own copy at its own address until the process ends.
// In host code this name is only a stand-in for the symbol: the device address is looked up once per device (static_scratch())
// and that pointer, never the name, is what the kernels get.
constexpr size_t STATIC_SCRATCH_BYTES = (size_t)SKIPARSE_STATIC_SCRATCH_BYTES;
static __device__ __align__(256) unsigned char scratch[STATIC_SCRATCH_BYTES];

namespace {

thread_local int g_last_hip_error = 0;

constexpr int MAX_DEVICES = 64;
void* g_scratch_ptr[MAX_DEVICES] = {};  // device address of `scratch` on each device, filled on the first call there
std::mutex g_scratch_mutex;

int elem_size(int dtype) {
    switch (dtype) {
        case SKIPARSE_BF16: return 2;
        case SKIPARSE_FP32: return 4;
        case SKIPARSE_FP8_E4M3: return 1;
        default: return 0;
    }
}

bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
bool misaligned_float(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }  // written one at a time: as those of any rows of a larger tensor lie

// [a, a + a_bytes) and [b, b + b_bytes) share at least one byte
bool overlap2(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + b_bytes && y < x + a_bytes;
}
bool overlap(const void* a, const void* b, size_t bytes) { return overlap2(a, bytes, b, bytes); }

struct Shape {
    size_t n_tok;     // T*H*W
    size_t n_sub;     // n_tok / s^2
    size_t row_elems; // heads*head_dim
    size_t elems;     // B*n_tok*row_elems
};

// Checks everything that does not involve pointers.  Returns SKIPARSE_OK and fills `sh`, or an error code.
int check_shape(int B, int heads, int T, int H, int W, int head_dim, int s, int pattern, Shape* sh, bool allow_pad = false) {
    if (B < 1 || heads < 1 || T < 1 || H < 1 || W < 1 || head_dim < 1 || s < 1) return SKIPARSE_EINVAL;
    if (pattern != SKIPARSE_TOKEN && pattern != SKIPARSE_GROUP) return SKIPARSE_EINVAL;
    if (s > 1024) return SKIPARSE_ESHAPE;
    const int unit = pattern == SKIPARSE_TOKEN ? s : s * s;
    if (!allow_pad && (H % unit != 0 || W % unit != 0)) return SKIPARSE_ESHAPE;
    const uint64_t n_tok = (uint64_t)T * (uint64_t)H * (uint64_t)W;
    const uint64_t rows = n_tok * (uint64_t)B;
    if (rows >= (1ull << 31)) return SKIPARSE_ESHAPE;  // row numbers are 32-bit in the kernels
    // in the any-resolution mode the subsequences are those of the grid padded to multiples of s*s
    const uint64_t Hp = allow_pad ? ((uint64_t)H + s * s - 1) / (s * s) * (s * s) : (uint64_t)H;
    const uint64_t Wp = allow_pad ? ((uint64_t)W + s * s - 1) / (s * s) * (s * s) : (uint64_t)W;
    if ((uint64_t)T * Hp * Wp >= (1ull << 31)) return SKIPARSE_ESHAPE;
    const uint64_t n_sub = (uint64_t)T * Hp * Wp / ((uint64_t)s * s);
    uint64_t dmax = Wp / (uint64_t)s > (uint64_t)s ? Wp / (uint64_t)s : (uint64_t)s;
    if (allow_pad && Hp > dmax) dmax = Hp;
    if (n_sub * dmax >= (1ull << 32)) return SKIPARSE_ESHAPE;  // range of the multiply-high divisions
    const uint64_t row_elems = (uint64_t)heads * (uint64_t)head_dim;
    if (row_elems >= (1ull << 31) || rows * row_elems >= (1ull << 40)) return SKIPARSE_ESHAPE;
    sh->n_tok = (size_t)n_tok;
    sh->n_sub = (size_t)n_sub;
    sh->row_elems = (size_t)row_elems;
    sh->elems = (size_t)(rows * row_elems);
    return SKIPARSE_OK;
}

// The same where rows keep their places, and no index map bounds the grid.
int check_rows(int B, int heads, int T, int H, int W, int head_dim, Shape* sh) {
    if (B < 1 || heads < 1 || T < 1 || H < 1 || W < 1 || head_dim < 1) return SKIPARSE_EINVAL;
    const uint64_t frame = (uint64_t)H * (uint64_t)W;
    if (frame >= (1ull << 31)) return SKIPARSE_ESHAPE;
    const uint64_t n_tok = frame * (uint64_t)T;
    if (n_tok >= (1ull << 31)) return SKIPARSE_ESHAPE;
    const uint64_t rows = n_tok * (uint64_t)B, row_elems = (uint64_t)heads * (uint64_t)head_dim;
    if (rows >= (1ull << 31) || row_elems >= (1ull << 31) || rows * row_elems >= (1ull << 40)) return SKIPARSE_ESHAPE;
    sh->n_tok = sh->n_sub = (size_t)n_tok;
    sh->row_elems = (size_t)row_elems;
    sh->elems = (size_t)(rows * row_elems);
    return SKIPARSE_OK;
}

GridMap make_gridmap(int T, int H, int W, int s, int pattern, bool pad = false) {
    return skiparse::make_gridmap(T, H, W, s, pattern == SKIPARSE_GROUP, pad);
}

int finish(hipError_t e) {
    if (e == hipSuccess) return SKIPARSE_OK;
    g_last_hip_error = (int)e;
    return SKIPARSE_EHIP;
}

// Device address of the static scratch on the CURRENT device: looked up once per device, with that device current, and kept.
int static_scratch(void** ptr) {
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return finish(e);
    if (dev < 0 || dev >= MAX_DEVICES) return SKIPARSE_EUNSUPPORTED;
    std::lock_guard<std::mutex> lock(g_scratch_mutex);
    if (g_scratch_ptr[dev] == nullptr) {
        void* p = nullptr;
        e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
        if (e != hipSuccess) return finish(e);
        if (p == nullptr) return finish(hipErrorInvalidSymbol);
        g_scratch_ptr[dev] = p;
    }
    *ptr = g_scratch_ptr[dev];
    return SKIPARSE_OK;
}

int permute_common(const void* src, void* dst, int B, int heads, int T, int H, int W, int head_dim, int s, int pattern,
                   int dtype, void* stream, int to_sparse) {
    if (!src || !dst) return SKIPARSE_EINVAL;
    const int esz = elem_size(dtype);
    if (esz == 0) return SKIPARSE_EINVAL;
    Shape sh;
    const int rc = check_shape(B, heads, T, H, W, head_dim, s, pattern, &sh);
    if (rc != SKIPARSE_OK) return rc;
    if (misaligned(src) || misaligned(dst)) return SKIPARSE_EINVAL;
    const size_t row_bytes = sh.row_elems * (size_t)esz;
    if (row_bytes % 16 != 0) return SKIPARSE_EUNSUPPORTED;
    if (overlap(src, dst, sh.elems * (size_t)esz)) return SKIPARSE_EINVAL;
    const GridMap g = make_gridmap(T, H, W, s, pattern);
    return finish(launch_permute(src, dst, B, g, row_bytes, to_sparse, (hipStream_t)stream));
}

// The attention kernels address rows with 32-bit byte offsets inside one batch element: one batch element must stay below
// 4 GiB (tokens per batch element, row length W and bytes per token row are kept below 2^24 as well).
int check_attn_ranges(const Shape& sh, int W, int elem_bytes) {
    const uint64_t row_bytes = (uint64_t)sh.row_elems * (uint64_t)elem_bytes;
    if (sh.n_tok >= (1u << 24) || (uint64_t)W >= (1u << 24) || row_bytes >= (1u << 24)) return SKIPARSE_ESHAPE;
    if ((uint64_t)sh.n_tok * row_bytes >= (1ull << 32)) return SKIPARSE_ESHAPE;
    return SKIPARSE_OK;
}

int check_attn_ptrs(const void* q, const void* k, const void* v, const void* out, size_t bytes) {
    if (!q || !k || !v || !out) return SKIPARSE_EINVAL;
    if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(out)) return SKIPARSE_EINVAL;
    if (overlap(out, q, bytes) || overlap(out, k, bytes) || overlap(out, v, bytes)) return SKIPARSE_EINVAL;
    return SKIPARSE_OK;
}

size_t align256(size_t x) { return (x + 255u) & ~(size_t)255u; }

}  // namespace

extern "C" {

int skiparse_permute(const void* src, void* dst, int B, int heads, int T, int H, int W, int head_dim, int s, int pattern,
                     int dtype, void* stream) {
    return permute_common(src, dst, B, heads, T, H, W, head_dim, s, pattern, dtype, stream, 1);
}

int skiparse_unpermute(const void* src, void* dst, int B, int heads, int T, int H, int W, int head_dim, int s, int pattern,
                       int dtype, void* stream) {
    return permute_common(src, dst, B, heads, T, H, W, head_dim, s, pattern, dtype, stream, 0);
}

// Local halves of the pattern switch under Sparse Sequence Parallelism (Sec. 3.3; Alg. 1, sparse_sequence_parallel): shared checks.
static int ssp_common(const void* src, void* dst, int b, int heads, int T, int H, int W, int head_dim, int s, int group_size, int dtype,
                      void* stream, bool pack) {
    if (!src || !dst) return SKIPARSE_EINVAL;
    const int esz = elem_size(dtype);
    if (esz == 0) return SKIPARSE_EINVAL;
    if (b < 1 || s < 1 || s > 1024 || group_size < 1) return SKIPARSE_EINVAL;
    if ((s * s) % group_size != 0) return SKIPARSE_ESHAPE;  // whole subsequences per rank
    const int G = s * s / group_size;
    if ((int64_t)G * b > (int64_t)1 << 24) return SKIPARSE_ESHAPE;
    Shape full;  // the full grid must admit both patterns: H and W multiples of s*s
    int rc = check_shape(b, heads, T, H, W, head_dim, s, SKIPARSE_GROUP, &full);
    if (rc != SKIPARSE_OK) return rc;
    // a rank's shard: G*b batch elements on the reduced grid (T, H/s, W/s), split token-wise once more
    Shape sh;
    rc = check_shape(G * b, heads, T, H / s, W / s, head_dim, s, SKIPARSE_TOKEN, &sh);
    if (rc != SKIPARSE_OK) return rc;
    if (misaligned(src) || misaligned(dst)) return SKIPARSE_EINVAL;
    const size_t row_bytes = sh.row_elems * (size_t)esz;
    if (row_bytes % 16 != 0) return SKIPARSE_EUNSUPPORTED;
    if (overlap(src, dst, sh.elems * (size_t)esz)) return SKIPARSE_EINVAL;
    const GridMap g = make_gridmap(T, H / s, W / s, s, SKIPARSE_TOKEN);
    if (pack) return finish(launch_permute(src, dst, G * b, g, row_bytes, 1, (hipStream_t)stream));
    return finish(launch_permute(src, dst, G * b, g, row_bytes, 0, (hipStream_t)stream, s == 1 ? 0 : G));
}

int skiparse_ssp_pack(const void* x, void* send, int b, int heads, int T, int H, int W, int head_dim, int s, int group_size, int dtype,
                      void* stream) {
    return ssp_common(x, send, b, heads, T, H, W, head_dim, s, group_size, dtype, stream, true);
}

int skiparse_ssp_unpack(const void* recv, void* y, int b, int heads, int T, int H, int W, int head_dim, int s, int group_size, int dtype,
                        void* stream) {
    return ssp_common(recv, y, b, heads, T, H, W, head_dim, s, group_size, dtype, stream, false);
}

int skiparse_switch_pattern(const void* src, void* dst, int B, int heads, int T, int H, int W, int head_dim, int s,
                            int from_pattern, int dtype, void* stream) {
    if (!src || !dst) return SKIPARSE_EINVAL;
    const int esz = elem_size(dtype);
    if (esz == 0) return SKIPARSE_EINVAL;
    if (from_pattern != SKIPARSE_TOKEN && from_pattern != SKIPARSE_GROUP) return SKIPARSE_EINVAL;
    Shape sh;
    const int rc = check_shape(B, heads, T, H, W, head_dim, s, SKIPARSE_GROUP, &sh);  // both patterns must fit: multiples of s*s
    if (rc != SKIPARSE_OK) return rc;
    if (misaligned(src) || misaligned(dst)) return SKIPARSE_EINVAL;
    const size_t row_bytes = sh.row_elems * (size_t)esz;
    if (row_bytes % 16 != 0) return SKIPARSE_EUNSUPPORTED;
    if (overlap(src, dst, sh.elems * (size_t)esz)) return SKIPARSE_EINVAL;
    if (s == 1) return finish(launch_permute(src, dst, B, make_gridmap(T, H, W, 1, SKIPARSE_TOKEN), row_bytes, 1, (hipStream_t)stream));
    const int to_pattern = from_pattern == SKIPARSE_TOKEN ? SKIPARSE_GROUP : SKIPARSE_TOKEN;
    const GridMap g_to = make_gridmap(T, H, W, s, to_pattern);
    return finish(launch_switch(src, dst, B, g_to, row_bytes, (hipStream_t)stream));
}

int dense_attn_fwd(const void* q, const void* k, const void* v, void* out, int B, int heads, int T, int H, int W,
                   int head_dim, float scale, int dtype, void* stream) {
    Shape sh;
    int rc = check_shape(B, heads, T, H, W, head_dim, 1, SKIPARSE_TOKEN, &sh);
    if (rc != SKIPARSE_OK) return rc;
    if (elem_size(dtype) == 0) return SKIPARSE_EINVAL;
    if (dtype != SKIPARSE_BF16 || (head_dim != 64 && head_dim != 128)) return SKIPARSE_EUNSUPPORTED;
    rc = check_attn_ranges(sh, W, 2);
    if (rc != SKIPARSE_OK) return rc;
    rc = check_attn_ptrs(q, k, v, out, sh.elems * 2);
    if (rc != SKIPARSE_OK) return rc;
    AttnArgs a;
    a.q = q; a.k = k; a.v = v; a.out = out;
    a.B = B; a.heads = heads; a.head_dim = head_dim;
    a.scale = scale > 0.f ? scale : 1.0f / sqrtf((float)head_dim);
    a.g = make_dense_gridmap(sh.n_tok);
    a.pad = false;
    a.out_kind = OUT_AS_INPUT;
    a.lse = nullptr;
    return finish(launch_attn_bf16(a, (hipStream_t)stream));
}

size_t skiparse_workspace_bytes(int B, int heads, int T, int H, int W, int head_dim, int s, int dtype, unsigned flags) {
    Shape sh;
    if (check_shape(B, heads, T, H, W, head_dim, s, SKIPARSE_TOKEN, &sh) != SKIPARSE_OK) return 0;
    if (dtype != SKIPARSE_BF16 || (flags & SKIPARSE_FUSED)) return 0;
    return 4 * align256(sh.elems * 2);
}

int skiparse_attn_fwd(const void* q, const void* k, const void* v, void* out, int B, int heads, int T, int H, int W,
                      int head_dim, int s, int pattern, float scale, int dtype, unsigned flags, void* workspace,
                      size_t workspace_bytes, void* stream) {
    if (flags & ~(unsigned)(SKIPARSE_FUSED | SKIPARSE_PAD)) return SKIPARSE_EINVAL;
    const bool pad = (flags & SKIPARSE_PAD) != 0 && s > 1;
    Shape sh;
    int rc = check_shape(B, heads, T, H, W, head_dim, s, pattern, &sh, pad);
    if (rc != SKIPARSE_OK) return rc;
    if (elem_size(dtype) == 0) return SKIPARSE_EINVAL;
    if (pad && !(flags & SKIPARSE_FUSED)) return SKIPARSE_EUNSUPPORTED;  // only the fused kernel has the any-resolution walk
    if (dtype != SKIPARSE_BF16 || (head_dim != 64 && head_dim != 128)) return SKIPARSE_EUNSUPPORTED;
    const size_t bytes = sh.elems * 2;
    rc = check_attn_ranges(sh, W, 2);
    if (rc != SKIPARSE_OK) return rc;
    rc = check_attn_ptrs(q, k, v, out, bytes);
    if (rc != SKIPARSE_OK) return rc;
    AttnArgs a;
    a.B = B; a.heads = heads; a.head_dim = head_dim;
    a.scale = scale > 0.f ? scale : 1.0f / sqrtf((float)head_dim);
    a.out_kind = OUT_AS_INPUT;
    a.lse = nullptr;
    hipStream_t st = (hipStream_t)stream;
    if (flags & SKIPARSE_FUSED) {
        a.q = q; a.k = k; a.v = v; a.out = out;
        a.g = make_gridmap(T, H, W, s, pattern, pad);
        a.pad = pad;
        return finish(launch_attn_bf16(a, st));
    }
    const size_t need = 4 * align256(bytes);
    if (!workspace || workspace_bytes < need || misaligned(workspace)) return SKIPARSE_EWORKSPACE;
    if (overlap2(workspace, need, q, bytes) || overlap2(workspace, need, k, bytes) || overlap2(workspace, need, v, bytes) ||
        overlap2(workspace, need, out, bytes))
        return SKIPARSE_EINVAL;
    char* w = (char*)workspace;
    void* qp = w;
    void* kp = w + align256(bytes);
    void* vp = w + 2 * align256(bytes);
    void* op = w + 3 * align256(bytes);
    const GridMap g = make_gridmap(T, H, W, s, pattern);
    const size_t row_bytes = sh.row_elems * 2;
    hipError_t e;
    if ((e = launch_permute(q, qp, B, g, row_bytes, 1, st)) != hipSuccess) return finish(e);
    if ((e = launch_permute(k, kp, B, g, row_bytes, 1, st)) != hipSuccess) return finish(e);
    if ((e = launch_permute(v, vp, B, g, row_bytes, 1, st)) != hipSuccess) return finish(e);
    a.q = qp; a.k = kp; a.v = vp; a.out = op;
    a.B = B * s * s;  // the subsequences are the batch of the inner attention (Alg. 1: "(p q b)")
    a.g = make_dense_gridmap(sh.n_sub);
    a.pad = false;
    if ((e = launch_attn_bf16(a, st)) != hipSuccess) return finish(e);
    return finish(launch_permute(op, out, B, g, row_bytes, 0, st));
}

int skiparse_attn_fwd_sparse(const void* q, const void* k, const void* v, void* out, int B, int heads, int T, int H, int W,
                             int head_dim, int s, int pattern, int out_layout, float scale, int dtype, void* stream) {
    if (out_layout != SKIPARSE_OUT_SAME && out_layout != SKIPARSE_OUT_OTHER && out_layout != SKIPARSE_OUT_ORIGINAL)
        return SKIPARSE_EINVAL;
    Shape sh;
    // the other pattern's layout exists only when both patterns do: multiples of s*s
    int rc = check_shape(B, heads, T, H, W, head_dim, s, out_layout == SKIPARSE_OUT_OTHER ? SKIPARSE_GROUP : pattern, &sh);
    if (rc != SKIPARSE_OK) return rc;
    if (pattern != SKIPARSE_TOKEN && pattern != SKIPARSE_GROUP) return SKIPARSE_EINVAL;
    if (elem_size(dtype) == 0) return SKIPARSE_EINVAL;
    if (dtype != SKIPARSE_BF16 || (head_dim != 64 && head_dim != 128)) return SKIPARSE_EUNSUPPORTED;
    rc = check_attn_ranges(sh, W, 2);
    if (rc != SKIPARSE_OK) return rc;
    rc = check_attn_ptrs(q, k, v, out, sh.elems * 2);
    if (rc != SKIPARSE_OK) return rc;
    AttnArgs a;
    a.q = q; a.k = k; a.v = v; a.out = out;
    a.B = B * s * s;  // the subsequences are the batch of the attention (Alg. 1: "(p q b)")
    a.heads = heads; a.head_dim = head_dim;
    a.scale = scale > 0.f ? scale : 1.0f / sqrtf((float)head_dim);
    a.g = make_dense_gridmap(sh.n_sub);
    a.pad = false;
    // with s = 1 every layout is the original one
    a.out_kind = (out_layout == SKIPARSE_OUT_SAME || s == 1) ? OUT_AS_INPUT : out_layout == SKIPARSE_OUT_ORIGINAL ? OUT_ORIGINAL : OUT_OTHER_PATTERN;
    a.out_B = B;
    a.lse = nullptr;
    a.g_in = make_gridmap(T, H, W, s, pattern);
    return finish(launch_attn_bf16(a, (hipStream_t)stream));
}

// floats in the log-sum-exp / delta arrays: one per (subsequence, head, position); positions run over the padded grid in the
// any-resolution mode (sh.n_sub is then the padded count)
static size_t lse_elems(int B, int heads, int s, const Shape& sh) { return (size_t)s * s * B * heads * sh.n_sub; }

size_t skiparse_lse_bytes(int B, int heads, int T, int H, int W, int head_dim, int s, int pattern, unsigned flags) {
    if (flags & ~(unsigned)SKIPARSE_PAD) return 0;
    Shape sh;
    if (check_shape(B, heads, T, H, W, head_dim, s, pattern, &sh, (flags & SKIPARSE_PAD) != 0 && s > 1) != SKIPARSE_OK) return 0;
    return lse_elems(B, heads, s, sh) * sizeof(float);
}

int skiparse_attn_fwd_lse(const void* q, const void* k, const void* v, void* out, float* lse, int B, int heads, int T, int H, int W,
                          int head_dim, int s, int pattern, float scale, int dtype, unsigned flags, void* stream) {
    if (flags & ~(unsigned)SKIPARSE_PAD) return SKIPARSE_EINVAL;
    const bool pad = (flags & SKIPARSE_PAD) != 0 && s > 1;
    Shape sh;
    int rc = check_shape(B, heads, T, H, W, head_dim, s, pattern, &sh, pad);
    if (rc != SKIPARSE_OK) return rc;
    if (elem_size(dtype) == 0) return SKIPARSE_EINVAL;
    if (dtype != SKIPARSE_BF16 || (head_dim != 64 && head_dim != 128)) return SKIPARSE_EUNSUPPORTED;
    const size_t bytes = sh.elems * 2, lse_bytes = lse_elems(B, heads, s, sh) * sizeof(float);
    rc = check_attn_ranges(sh, W, 2);
    if (rc != SKIPARSE_OK) return rc;
    rc = check_attn_ptrs(q, k, v, out, bytes);
    if (rc != SKIPARSE_OK) return rc;
    if (!lse || ((uintptr_t)lse & 3u)) return SKIPARSE_EINVAL;
    if (overlap2(lse, lse_bytes, q, bytes) || overlap2(lse, lse_bytes, k, bytes) || overlap2(lse, lse_bytes, v, bytes) ||
        overlap2(lse, lse_bytes, out, bytes))
        return SKIPARSE_EINVAL;
    AttnArgs a;
    a.q = q; a.k = k; a.v = v; a.out = out;
    a.B = B; a.heads = heads; a.head_dim = head_dim;
    a.scale = scale > 0.f ? scale : 1.0f / sqrtf((float)head_dim);
    a.g = make_gridmap(T, H, W, s, pattern, pad);
    a.pad = pad;
    a.out_kind = OUT_AS_INPUT;
    a.lse = lse;
    return finish(launch_attn_bf16(a, (hipStream_t)stream));
}

// Whether the backward passes dQ along workgroups where it has the workspace for it, and what they share there.
static bool bwd_chain(int B, int heads, int head_dim, const GridMap& g, bool pad, BwdChain* w) {
    const UnitSizes u = unit_sizes(g, pad, (uint64_t)B * (uint32_t)heads);
    if (!bwd_chain(head_dim, u)) return false;
    *w = make_bwd_chain((uint32_t)B * (g.mode == MODE_DENSE ? 1u : (uint32_t)(g.s * g.s)) * (uint32_t)heads, u.n_max);
    return true;
}

size_t skiparse_bwd_workspace_bytes(int B, int heads, int T, int H, int W, int head_dim, int s, int pattern, unsigned flags) {
    return align256(skiparse_lse_bytes(B, heads, T, H, W, head_dim, s, pattern, flags));
}

size_t skiparse_bwd_walk_workspace_bytes(int B, int heads, int T, int H, int W, int head_dim, int s, int pattern, unsigned flags) {
    const size_t delta = skiparse_bwd_workspace_bytes(B, heads, T, H, W, head_dim, s, pattern, flags);
    if (delta == 0) return 0;
    BwdChain w;
    const bool pad = (flags & SKIPARSE_PAD) != 0 && s > 1;
    return delta + (bwd_chain(B, heads, head_dim, make_gridmap(T, H, W, s, pattern, pad), pad, &w) ? w.bytes(head_dim) : 0);
}

// Shared by skiparse_attn_bwd (caller's workspace) and skiparse_attn_bwd_static (workspace == nullptr: the library's static scratch,
// whose device address is looked up after the arguments have been validated).
static int attn_bwd_common(const void* q, const void* k, const void* v, const void* out, const void* dout, const float* lse, void* dq,
                           void* dk, void* dv, int B, int heads, int T, int H, int W, int head_dim, int s, int pattern, float scale,
                           int dtype, unsigned flags, void* workspace, size_t workspace_bytes, bool use_static, void* stream) {
    if (flags & ~(unsigned)SKIPARSE_PAD) return SKIPARSE_EINVAL;
    const bool pad = (flags & SKIPARSE_PAD) != 0 && s > 1;
    Shape sh;
    int rc = check_shape(B, heads, T, H, W, head_dim, s, pattern, &sh, pad);
    if (rc != SKIPARSE_OK) return rc;
    if (elem_size(dtype) == 0) return SKIPARSE_EINVAL;
    if (dtype != SKIPARSE_BF16 || (head_dim != 64 && head_dim != 128)) return SKIPARSE_EUNSUPPORTED;
    const size_t bytes = sh.elems * 2, lse_bytes = lse_elems(B, heads, s, sh) * sizeof(float);
    rc = check_attn_ranges(sh, W, 2);
    if (rc != SKIPARSE_OK) return rc;
    const void* ins[5] = {q, k, v, out, dout};
    void* outs[3] = {dq, dk, dv};
    for (const void* x : ins)
        if (!x || misaligned(x)) return SKIPARSE_EINVAL;
    for (void* y : outs)
        if (!y || misaligned(y)) return SKIPARSE_EINVAL;
    if (!lse || ((uintptr_t)lse & 3u)) return SKIPARSE_EINVAL;
    const size_t need = align256(lse_bytes);
    if (use_static) {
        if (need > STATIC_SCRATCH_BYTES) return SKIPARSE_EWORKSPACE;  // the problem is larger than the static scratch
        rc = static_scratch(&workspace);
        if (rc != SKIPARSE_OK) return rc;
    } else if (!workspace || workspace_bytes < need || misaligned(workspace)) {
        return SKIPARSE_EWORKSPACE;
    }
    // no gradient may alias an input, another gradient, the log-sum-exp or the workspace
    for (int i = 0; i < 3; i++) {
        for (const void* x : ins)
            if (overlap(outs[i], x, bytes)) return SKIPARSE_EINVAL;
        for (int j = i + 1; j < 3; j++)
            if (overlap(outs[i], outs[j], bytes)) return SKIPARSE_EINVAL;
        if (overlap2(outs[i], bytes, lse, lse_bytes)) return SKIPARSE_EINVAL;
    }
    // whether an argument lies in the first n bytes of the workspace
    auto holds_argument = [&](size_t n) {
        for (const void* x : ins)
            if (overlap2(workspace, n, x, bytes)) return true;
        for (const void* y : outs)
            if (overlap2(workspace, n, y, bytes)) return true;
        return overlap2(workspace, n, lse, lse_bytes);
    };
    if (holds_argument(need)) return SKIPARSE_EINVAL;
    const GridMap g = make_gridmap(T, H, W, s, pattern, pad);
    BwdChain chain;
    bool chained = !use_static && bwd_chain(B, heads, head_dim, g, pad, &chain);
    if (chained) {
        // the call does without the rest: a workspace that is the front of a buffer whose rest holds tensors of the call is no error
        const size_t all = need + chain.bytes(head_dim);
        chained = workspace_bytes >= all && !holds_argument(all);
        chain.place((char*)workspace + need);
    }
    BwdArgs a;
    a.q = q; a.k = k; a.v = v; a.out = out; a.dout = dout; a.lse = lse;
    a.delta = (float*)workspace;
    a.dq = dq; a.dk = dk; a.dv = dv;
    a.B = B; a.heads = heads; a.head_dim = head_dim;
    a.scale = scale > 0.f ? scale : 1.0f / sqrtf((float)head_dim);
    a.pad = pad;
    a.g = g;
    return finish(chained ? launch_attn_bwd_chain(a, chain, (hipStream_t)stream) : launch_attn_bwd_bf16(a, (hipStream_t)stream));
}

int skiparse_attn_bwd(const void* q, const void* k, const void* v, const void* out, const void* dout, const float* lse, void* dq,
                      void* dk, void* dv, int B, int heads, int T, int H, int W, int head_dim, int s, int pattern, float scale,
                      int dtype, unsigned flags, void* workspace, size_t workspace_bytes, void* stream) {
    return attn_bwd_common(q, k, v, out, dout, lse, dq, dk, dv, B, heads, T, H, W, head_dim, s, pattern, scale, dtype, flags, workspace,
                           workspace_bytes, false, stream);
}

size_t skiparse_static_scratch_bytes(void) { return STATIC_SCRATCH_BYTES; }

int skiparse_attn_bwd_static(const void* q, const void* k, const void* v, const void* out, const void* dout, const float* lse, void* dq,
                             void* dk, void* dv, int B, int heads, int T, int H, int W, int head_dim, int s, int pattern, float scale,
                             int dtype, unsigned flags, void* stream) {
    return attn_bwd_common(q, k, v, out, dout, lse, dq, dk, dv, B, heads, T, H, W, head_dim, s, pattern, scale, dtype, flags, nullptr, 0,
                           true, stream);
}

// elements of a tensor in the sparse layout over the (possibly padded) grid: s*s*B subsequences of sh.n_sub positions
static size_t sparse_elems(int B, int s, const Shape& sh) { return (size_t)s * s * B * sh.n_sub * sh.row_elems; }

int skiparse_quantize_fp8_ex(const void* x_bf16, void* x8, float* scales, int B, int heads, int T, int H, int W, int head_dim,
                             int s, int pattern, unsigned flags, void* stream) {
    if (flags & ~(unsigned)SKIPARSE_PAD) return SKIPARSE_EINVAL;
    const bool pad = (flags & SKIPARSE_PAD) != 0 && s > 1;
    Shape sh;
    const int rc = check_shape(B, heads, T, H, W, head_dim, s, pattern, &sh, pad);
    if (rc != SKIPARSE_OK) return rc;
    if (!x_bf16 || !x8 || !scales) return SKIPARSE_EINVAL;
    if (misaligned(x_bf16) || misaligned(x8) || (reinterpret_cast<uintptr_t>(scales) & 3u)) return SKIPARSE_EINVAL;
    if (head_dim != 64 && head_dim != 128) return SKIPARSE_EUNSUPPORTED;
    if (overlap2(x_bf16, sh.elems * 2, x8, sparse_elems(B, s, sh))) return SKIPARSE_EINVAL;
    const GridMap g = make_gridmap(T, H, W, s, pattern, pad);
    return finish(launch_quantize_fp8(x_bf16, x8, scales, B, heads, head_dim, g, pad, (hipStream_t)stream));
}

int skiparse_quantize_fp8(const void* x_bf16, void* x8, float* scales, int B, int heads, int T, int H, int W, int head_dim,
                          int s, int pattern, void* stream) {
    return skiparse_quantize_fp8_ex(x_bf16, x8, scales, B, heads, T, H, W, head_dim, s, pattern, 0u, stream);
}

int skiparse_attn_fwd_fp8_ex(const void* q8, const void* k8, const void* v8, const float* sq, const float* sk, const float* sv,
                             void* out_bf16, int B, int heads, int T, int H, int W, int head_dim, int s, int pattern,
                             float scale, unsigned flags, void* stream) {
    if (flags & ~(unsigned)SKIPARSE_PAD) return SKIPARSE_EINVAL;
    const bool pad = (flags & SKIPARSE_PAD) != 0 && s > 1;
    Shape sh;
    int rc = check_shape(B, heads, T, H, W, head_dim, s, pattern, &sh, pad);
    if (rc != SKIPARSE_OK) return rc;
    if (!q8 || !k8 || !v8 || !sq || !sk || !sv || !out_bf16) return SKIPARSE_EINVAL;
    if (misaligned(q8) || misaligned(k8) || misaligned(v8) || misaligned(out_bf16)) return SKIPARSE_EINVAL;
    if (head_dim != 64 && head_dim != 128) return SKIPARSE_EUNSUPPORTED;
    rc = check_attn_ranges(sh, W, 2);
    if (rc != SKIPARSE_OK) return rc;
    // the quantised tensors are addressed with 32-bit byte offsets inside one subsequence
    if ((uint64_t)sh.n_sub * sh.row_elems >= (1ull << 32)) return SKIPARSE_ESHAPE;
    const size_t in_bytes = sparse_elems(B, s, sh), out_bytes = sh.elems * 2;
    if (overlap2(out_bf16, out_bytes, q8, in_bytes) || overlap2(out_bf16, out_bytes, k8, in_bytes) ||
        overlap2(out_bf16, out_bytes, v8, in_bytes))
        return SKIPARSE_EINVAL;
    // one float per (subsequence, head, 128 positions); the kernel reads them while it writes out
    const size_t scale_bytes = (size_t)s * s * B * heads * ((sh.n_sub + 127) / 128) * sizeof(float);
    for (const float* sc : {sq, sk, sv})
        if ((reinterpret_cast<uintptr_t>(sc) & 3u) || overlap2(out_bf16, out_bytes, sc, scale_bytes)) return SKIPARSE_EINVAL;
    Fp8AttnArgs a;
    a.q8 = q8; a.k8 = k8; a.v8 = v8; a.sq = sq; a.sk = sk; a.sv = sv; a.out = out_bf16;
    a.B = B; a.heads = heads; a.head_dim = head_dim;
    a.scale = scale > 0.f ? scale : 1.0f / sqrtf((float)head_dim);
    a.n_blk = (uint32_t)((sh.n_sub + 127) / 128);
    a.pad = pad;
    a.g = make_gridmap(T, H, W, s, pattern, pad);
    return finish(launch_attn_fp8(a, (hipStream_t)stream));
}

int skiparse_attn_fwd_fp8(const void* q8, const void* k8, const void* v8, const float* sq, const float* sk, const float* sv,
                          void* out_bf16, int B, int heads, int T, int H, int W, int head_dim, int s, int pattern,
                          float scale, void* stream) {
    return skiparse_attn_fwd_fp8_ex(q8, k8, v8, sq, sk, sv, out_bf16, B, heads, T, H, W, head_dim, s, pattern, scale, 0u, stream);
}

// ---- rotary positions

static bool valid_order(int order, bool stay) { return order >= SKIPARSE_ORDER_SAME && order <= (stay ? SKIPARSE_ORDER_STAY_SPARSE : SKIPARSE_ORDER_TO_ORIGINAL); }

// Pairs of the table, 0 on bad arguments.  Places times pairs of an axis, and all pairs, stay below 2^31.
static uint64_t rope_pairs(int T, int H, int W, int rt, int rh, int rw) {
    if (T < 1 || H < 1 || W < 1) return 0;
    uint64_t n = 0;
    const int r[3] = {rt, rh, rw}, len[3] = {T, H, W};
    for (int i = 0; i < 3; i++) {
        if (r[i] < 0 || r[i] % 2 != 0 || (uint32_t)r[i] / 2u > ROPE_MAX_PAIRS) return 0;
        n += (uint64_t)len[i] * (uint32_t)(r[i] / 2);
    }
    return n < (1ull << 31) ? n : 0;
}

size_t skiparse_rope_table_bytes(int T, int H, int W, int rt, int rh, int rw) { return (size_t)rope_pairs(T, H, W, rt, rh, rw) * 2 * sizeof(float); }

int skiparse_rope_table(float* table, int T, int H, int W, int rt, int rh, int rw, float theta, int scaling, float factor_t, float factor_h, float factor_w,
                        int trained_t, int trained_h, int trained_w, float fast, float slow, float attention, void* stream) {
    return skiparse_rope_table_ex(table, T, H, W, rt, rh, rw, theta, scaling, factor_t, factor_h, factor_w, trained_t, trained_h, trained_w, fast, slow, attention, stream);
}

int skiparse_rope_table_ex(float* table, int T, int H, int W, int rt, int rh, int rw, double theta, int scaling, double factor_t, double factor_h, double factor_w,
                           int trained_t, int trained_h, int trained_w, double fast, double slow, double attention, void* stream) {
    if (!table || misaligned(table)) return SKIPARSE_EINVAL;
    if (T < 1 || H < 1 || W < 1 || rt < 0 || rh < 0 || rw < 0 || (rt | rh | rw) % 2 != 0 || (rt | rh | rw) == 0) return SKIPARSE_EINVAL;
    if (rt > 2 * (int)ROPE_MAX_PAIRS || rh > 2 * (int)ROPE_MAX_PAIRS || rw > 2 * (int)ROPE_MAX_PAIRS) return SKIPARSE_EUNSUPPORTED;
    if (rope_pairs(T, H, W, rt, rh, rw) == 0) return SKIPARSE_ESHAPE;
    if (scaling < SKIPARSE_ROPE_PLAIN || scaling > SKIPARSE_ROPE_YARN) return SKIPARSE_EINVAL;
    const double limit = 3.0e38;  // not finite, or not a number: refused
    if (!(theta > 0. && theta < limit) || !(attention > -limit && attention < limit)) return SKIPARSE_EINVAL;
    const double factor[3] = {factor_t, factor_h, factor_w};
    const int trained[3] = {trained_t, trained_h, trained_w}, r[3] = {rt, rh, rw}, len[3] = {T, H, W};
    RopeAxis axis[3] = {};
    for (int i = 0; i < 3; i++) {
        axis[i].len = (uint32_t)len[i];
        axis[i].r = (uint32_t)r[i];
        axis[i].factor = factor[i];
        axis[i].trained = (uint32_t)trained[i];
        if (scaling == SKIPARSE_ROPE_PLAIN || r[i] == 0) continue;
        if (!(factor[i] >= 1. && factor[i] < limit)) return SKIPARSE_EINVAL;
        if (scaling == SKIPARSE_ROPE_YARN && trained[i] < 1) return SKIPARSE_EINVAL;
    }
    if (scaling == SKIPARSE_ROPE_YARN && !(fast > slow && fast < limit && slow > -limit)) return SKIPARSE_EINVAL;
    const RopeScaling sc = {scaling, theta, fast, slow, (float)attention};  // the last one multiplies what is stored in 32 bits
    return finish(launch_rope_table(table, axis[0], axis[1], axis[2], sc, (hipStream_t)stream));
}

int skiparse_rope(const void* q, const void* k, void* q_out, void* k_out, const float* table, int B, int heads, int T, int H, int W, int head_dim, int rt, int rh,
                  int rw, int len_t, int len_h, int len_w, int t0, int h0, int w0, int s, int pattern, int order, int layout, int inverse, int dtype, void* stream) {
    if (!q || !q_out || !table || !k != !k_out) return SKIPARSE_EINVAL;
    if (!valid_order(order, true)) return SKIPARSE_EINVAL;
    if ((layout != SKIPARSE_ROPE_INTERLEAVED && layout != SKIPARSE_ROPE_HALF) || (inverse != 0 && inverse != 1)) return SKIPARSE_EINVAL;
    const int esz = elem_size(dtype);
    if (esz == 0) return SKIPARSE_EINVAL;
    Shape sh;
    const bool moved = order != SKIPARSE_ORDER_SAME && s != 1;
    const int rc = moved ? check_shape(B, heads, T, H, W, head_dim, s, pattern, &sh) : check_rows(B, heads, T, H, W, head_dim, &sh);
    if (rc != SKIPARSE_OK) return rc;
    if (misaligned(q) || misaligned(q_out) || misaligned(table) || (k && (misaligned(k) || misaligned(k_out)))) return SKIPARSE_EINVAL;
    if (dtype == SKIPARSE_FP8_E4M3 || head_dim % 8 != 0 || head_dim > 512) return SKIPARSE_EUNSUPPORTED;
    if (rt < 0 || rh < 0 || rw < 0 || (rt | rh | rw) % 2 != 0 || rt > head_dim || rh > head_dim || rw > head_dim) return SKIPARSE_EINVAL;
    if (rt + rh + rw == 0 || rt + rh + rw > head_dim) return SKIPARSE_EINVAL;
    const uint64_t pairs = rope_pairs(len_t, len_h, len_w, rt, rh, rw);
    if (pairs == 0) return SKIPARSE_EINVAL;
    if (t0 < 0 || h0 < 0 || w0 < 0) return SKIPARSE_EINVAL;
    if ((rt && (int64_t)t0 + T > len_t) || (rh && (int64_t)h0 + H > len_h) || (rw && (int64_t)w0 + W > len_w)) return SKIPARSE_ESHAPE;
    const size_t bytes = sh.elems * (size_t)esz, table_bytes = (size_t)pairs * 8;
    const bool in_place = !moved || order == SKIPARSE_ORDER_STAY_SPARSE;  // a row's place is read and written by one wavefront
    if (overlap(q_out, q, bytes) && !(in_place && q_out == q)) return SKIPARSE_EINVAL;
    if (overlap2(q_out, bytes, table, table_bytes)) return SKIPARSE_EINVAL;
    if (k) {
        if (overlap(k_out, k, bytes) && !(in_place && k_out == k)) return SKIPARSE_EINVAL;
        if (overlap(q_out, k, bytes) || overlap(k_out, q, bytes) || overlap(q_out, k_out, bytes) || overlap2(k_out, bytes, table, table_bytes)) return SKIPARSE_EINVAL;
    }
    RopeArgs a;
    a.q = q; a.k = k; a.q_out = q_out; a.k_out = k_out; a.table = table;
    a.B = B; a.heads = heads; a.T = T; a.H = H; a.W = W; a.head_dim = head_dim;
    a.rt = rt; a.rh = rh; a.rw = rw;
    a.len_t = len_t; a.len_h = len_h;
    a.t0 = t0; a.h0 = h0; a.w0 = w0;
    a.order = moved ? order : SKIPARSE_ORDER_SAME;  // with s = 1 every layout is the original one
    a.half = layout == SKIPARSE_ROPE_HALF;
    a.inverse = inverse != 0;
    a.f32 = dtype == SKIPARSE_FP32;
    a.g = moved ? make_gridmap(T, H, W, s, pattern) : make_dense_gridmap(sh.n_tok);
    return finish(launch_rope(a, (hipStream_t)stream));
}

// ---- 8-bit activation checkpoints

static size_t checkpoint_scales(size_t rows, size_t cols) { return rows * ((cols + 31) / 32); }

static int checkpoint_common(const void* x, const void* codes, const void* scales, int rows, int cols, int dtype) {
    if (!x || !codes || !scales || rows < 1 || cols < 1) return SKIPARSE_EINVAL;
    const int esz = elem_size(dtype);
    if (esz == 0 || misaligned(x) || misaligned(codes)) return SKIPARSE_EINVAL;
    if (dtype == SKIPARSE_FP8_E4M3 || cols % 8 != 0) return SKIPARSE_EUNSUPPORTED;
    const size_t n = (size_t)rows * (size_t)cols, m = checkpoint_scales((size_t)rows, (size_t)cols);
    if (n >= (1ull << 36)) return SKIPARSE_ESHAPE;
    if (overlap2(x, n * esz, codes, n) || overlap2(x, n * esz, scales, m) || overlap2(codes, n, scales, m)) return SKIPARSE_EINVAL;
    return SKIPARSE_OK;
}

int skiparse_checkpoint_save(const void* x, void* codes, void* scales, int rows, int cols, int dtype, void* stream) {
    const int rc = checkpoint_common(x, codes, scales, rows, cols, dtype);
    if (rc != SKIPARSE_OK) return rc;
    return finish(launch_checkpoint_save(x, codes, scales, (uint32_t)rows, (uint32_t)cols, dtype == SKIPARSE_FP32, (hipStream_t)stream));
}

int skiparse_checkpoint_load(const void* codes, const void* scales, void* out, int rows, int cols, int dtype, void* stream) {
    const int rc = checkpoint_common(out, codes, scales, rows, cols, dtype);
    if (rc != SKIPARSE_OK) return rc;
    return finish(launch_checkpoint_load(codes, scales, out, (uint32_t)rows, (uint32_t)cols, dtype == SKIPARSE_FP32, (hipStream_t)stream));
}

// ---- linear layer

// Sizes, enums and the row map that both directions share; `moved`: rows change places.
static int linear_common(int B, int T, int H, int W, int in_features, int out_features, int s, int pattern, int order, int act, int dtype, bool* moved, size_t* rows) {
    if (!valid_order(order, false) || act < SKIPARSE_ACT_NONE || act > SKIPARSE_ACT_SILU || elem_size(dtype) == 0) return SKIPARSE_EINVAL;
    *moved = order != SKIPARSE_ORDER_SAME && s != 1;
    Shape sh;
    for (int features : {in_features, out_features}) {
        const int rc = *moved ? check_shape(B, 1, T, H, W, features, s, pattern, &sh) : check_rows(B, 1, T, H, W, features, &sh);
        if (rc != SKIPARSE_OK) return rc;
        if (features >= (1 << 23)) return SKIPARSE_ESHAPE;
    }
    if ((uint64_t)in_features * (uint64_t)out_features >= (1ull << 40)) return SKIPARSE_ESHAPE;
    if (dtype != SKIPARSE_BF16 || in_features % 8 != 0 || out_features % 8 != 0) return SKIPARSE_EUNSUPPORTED;
    *rows = (size_t)B * sh.n_tok;
    return SKIPARSE_OK;
}

struct Span {
    const void* at;
    size_t bytes;
};
// Whether the buffer `x`, which is written, shares a byte with one of the others; null spans are not there.
static bool touches(Span x, std::initializer_list<Span> others) {
    for (const Span& o : others)
        if (x.at && o.at && overlap2(x.at, x.bytes, o.at, o.bytes)) return true;
    return false;
}

size_t skiparse_linear_workspace_bytes(int rows, int in_features, int out_features) {
    if (rows < 1 || in_features < 1 || out_features < 1) return 0;
    return linear_workspace(LINEAR_FWD, (uint32_t)rows, (uint32_t)out_features, (uint32_t)in_features);
}

int skiparse_linear_fwd(const void* x, const void* w, const void* bias, const void* residual, void* out, void* pre, void* pre_scales, int B, int T, int H, int W,
                        int in_features, int out_features, int s, int pattern, int order, int act, int dtype, void* workspace, size_t workspace_bytes,
                        void* stream) {
    if (!x || !w || !out || (pre_scales && !pre)) return SKIPARSE_EINVAL;
    bool moved;
    size_t rows;
    const int rc = linear_common(B, T, H, W, in_features, out_features, s, pattern, order, act, dtype, &moved, &rows);
    if (rc != SKIPARSE_OK) return rc;
    for (const void* p : {x, w, bias, residual, (const void*)out, (const void*)pre})
        if (p && misaligned(p)) return SKIPARSE_EINVAL;
    const size_t K = (size_t)in_features, N = (size_t)out_features;
    if (!linear_fits(rows, N)) return SKIPARSE_ESHAPE;
    if (moved && rows * K * 2 >= (1ull << 32) - 64) return SKIPARSE_ESHAPE;  // rows that move are addressed with 32-bit byte offsets
    const Span sx = {x, rows * K * 2}, sw = {w, N * K * 2}, sb = {bias, N * 2}, so = {out, rows * N * 2};
    const Span sp = {pre, rows * N * (pre_scales ? 1 : 2)}, ss = {pre_scales, checkpoint_scales(rows, N)}, sr = {residual, rows * N * 2};
    if (touches(so, {sx, sw, sb, sp, ss}) || (residual && residual != out && overlap2(out, so.bytes, residual, sr.bytes))) return SKIPARSE_EINVAL;
    if (touches(sp, {sx, sw, sb, ss, sr}) || touches(ss, {sx, sw, sb, sr})) return SKIPARSE_EINVAL;
    const size_t need = linear_workspace(LINEAR_FWD, (uint32_t)rows, (uint32_t)N, (uint32_t)K);
    if (need && (!workspace || workspace_bytes < need || misaligned(workspace))) return SKIPARSE_EWORKSPACE;
    if (touches({need ? workspace : nullptr, need}, {sx, sw, sb, sr, so, sp, ss})) return SKIPARSE_EINVAL;
    LinearArgs a = {};
    a.p = x; a.q = w;
    a.M = (uint32_t)rows; a.N = (uint32_t)N; a.K = (uint32_t)K;
    a.e = {bias, residual, out, pre, pre_scales, act};
    a.partial = (float*)workspace;
    a.order = moved ? order : SKIPARSE_ORDER_SAME;
    if (moved) {
        const GridMap g = make_gridmap(T, H, W, s, pattern);
        a.rows = order == SKIPARSE_ORDER_TO_SPARSE ? make_row_args<TO_SPARSE>(g, (uint32_t)B) : make_row_args<TO_ORIGINAL>(g, (uint32_t)B);
    }
    return finish(launch_linear(LINEAR_FWD, a, (hipStream_t)stream));
}

// What a backward call keeps in its workspace, one after the other.
struct LinearBwdSpace {
    size_t dz, x, db, parts, total;
};
static LinearBwdSpace linear_bwd_space(size_t rows, size_t K, size_t N, bool dz, bool x, bool db, bool dx, bool dw) {
    LinearBwdSpace l;
    l.dz = dz ? align256(rows * N * 2) : 0;
    l.x = x ? align256(rows * K * 2) : 0;
    l.db = db ? align256((size_t)linear_rows_parts((uint32_t)rows, (uint32_t)N) * N * sizeof(float)) : 0;
    const size_t px = dx ? linear_workspace(LINEAR_DX, (uint32_t)rows, (uint32_t)K, (uint32_t)N) : 0, pw = dw ? linear_workspace(LINEAR_DW, (uint32_t)N, (uint32_t)K, (uint32_t)rows) : 0;
    l.parts = px > pw ? px : pw;  // one product after the other
    l.total = l.dz + l.x + l.db + l.parts;
    return l;
}

size_t skiparse_linear_bwd_workspace_bytes(int rows, int in_features, int out_features, int order, int act, int x_checkpoint) {
    if (rows < 1 || in_features < 1 || out_features < 1 || !valid_order(order, false) || act < SKIPARSE_ACT_NONE || act > SKIPARSE_ACT_SILU) return 0;
    return linear_bwd_space((size_t)rows, (size_t)in_features, (size_t)out_features, order != SKIPARSE_ORDER_SAME || act != SKIPARSE_ACT_NONE, x_checkpoint != 0, true, true, true).total;
}

int skiparse_linear_bwd(const void* dy, const void* x, const void* x_scales, const void* w, const void* pre, const void* pre_scales, const void* dx_add, void* dx,
                        void* dw, void* db, int B, int T, int H, int W, int in_features, int out_features, int s, int pattern, int order, int act, int dtype,
                        void* workspace, size_t workspace_bytes, void* stream) {
    if (!dy || (!dx && !dw && !db) || (dx && !w) || (dw && !x) || (x_scales && !x) || (pre_scales && !pre) || (dx_add && !dx)) return SKIPARSE_EINVAL;
    bool moved;
    size_t rows;
    const int rc = linear_common(B, T, H, W, in_features, out_features, s, pattern, order, act, dtype, &moved, &rows);
    if (rc != SKIPARSE_OK) return rc;
    if (act != SKIPARSE_ACT_NONE && !pre) return SKIPARSE_EINVAL;
    for (const void* p : {dy, x, w, pre, dx_add, (const void*)dx, (const void*)dw, (const void*)db})
        if (p && misaligned(p)) return SKIPARSE_EINVAL;
    if (act == SKIPARSE_ACT_NONE) pre = pre_scales = nullptr;
    if (!dw) x = x_scales = nullptr;
    if (!dx) w = nullptr;
    const size_t K = (size_t)in_features, N = (size_t)out_features;
    if ((dx && !linear_fits(rows, K)) || (dw && !linear_fits(N, K))) return SKIPARSE_ESHAPE;  // before the first launch: a call that is refused has written nothing
    const LinearBwdSpace l = linear_bwd_space(rows, K, N, (dx || dw) && (moved || act != SKIPARSE_ACT_NONE), x_scales != nullptr, db != nullptr, dx != nullptr, dw != nullptr);
    if (l.total && (!workspace || workspace_bytes < l.total || misaligned(workspace))) return SKIPARSE_EWORKSPACE;
    const Span sy = {dy, rows * N * 2}, sx = {x, rows * K * (x_scales ? 1 : 2)}, sxs = {x_scales, checkpoint_scales(rows, K)}, sw = {w, N * K * 2};
    const Span sp = {pre, rows * N * (pre_scales ? 1 : 2)}, sps = {pre_scales, checkpoint_scales(rows, N)}, sa = {dx_add, rows * K * 2};
    const Span gx = {dx, rows * K * 2}, gw = {dw, N * K * 2}, gb = {db, N * 2}, ws = {l.total ? workspace : nullptr, l.total};
    if (touches(gx, {sy, sx, sxs, sw, sp, sps, gw, gb, ws}) || (dx_add && dx_add != dx && overlap(dx, dx_add, gx.bytes))) return SKIPARSE_EINVAL;
    if (touches(gw, {sy, sx, sxs, sw, sp, sps, sa, gb, ws}) || touches(gb, {sy, sx, sxs, sw, sp, sps, sa, ws})) return SKIPARSE_EINVAL;
    if (touches(ws, {sy, sx, sxs, sw, sp, sps, sa})) return SKIPARSE_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    char* const at = (char*)workspace;
    hipError_t e;
    const void* dz = dy;
    float* const partial = (float*)(at + l.dz + l.x + l.db);
    if (l.dz || db) {
        LinearRowsArgs r = {};
        r.dy = dy; r.pre = pre; r.pre_scales = pre_scales;
        r.dz = l.dz ? at : nullptr;
        r.db_part = db ? (float*)(at + l.dz + l.x) : nullptr;
        r.db = db;
        r.M = (uint32_t)rows; r.N = (uint32_t)N;
        r.act = act;
        if (moved) {  // row of the input -> row of the output that was made of it
            const GridMap g = make_gridmap(T, H, W, s, pattern);
            const bool back = order == SKIPARSE_ORDER_TO_SPARSE;
            r.order = back ? SKIPARSE_ORDER_TO_ORIGINAL : SKIPARSE_ORDER_TO_SPARSE;
            r.rows = back ? make_row_args<TO_ORIGINAL>(g, (uint32_t)B) : make_row_args<TO_SPARSE>(g, (uint32_t)B);
        }
        if ((e = launch_linear_rows(r, st)) != hipSuccess) return finish(e);
        if (l.dz) dz = at;
    }
    if (x_scales) {
        if ((e = launch_checkpoint_load(x, x_scales, at + l.dz, (uint32_t)rows, (uint32_t)K, false, st)) != hipSuccess) return finish(e);
        x = at + l.dz;
    }
    if (dx) {
        LinearArgs a = {};
        a.p = dz; a.q = w;
        a.M = (uint32_t)rows; a.N = (uint32_t)K; a.K = (uint32_t)N;
        a.e = {nullptr, dx_add, dx, nullptr, nullptr, ACT_NONE};
        a.partial = partial;
        if ((e = launch_linear(LINEAR_DX, a, st)) != hipSuccess) return finish(e);
    }
    if (dw) {
        LinearArgs a = {};
        a.p = dz; a.q = x;
        a.M = (uint32_t)N; a.N = (uint32_t)K; a.K = (uint32_t)rows;
        a.e = {nullptr, nullptr, dw, nullptr, nullptr, ACT_NONE};
        a.partial = partial;
        if ((e = launch_linear(LINEAR_DW, a, st)) != hipSuccess) return finish(e);
    }
    return SKIPARSE_OK;
}

// ---- root-mean-square norm, rows in 8-bit integers

// Sizes, enums and the row map; `moved`: rows change places.
static int rows_common(int B, int T, int H, int W, int cols, int s, int pattern, int order, int dtype, bool* moved, size_t* rows) {
    if (!valid_order(order, false) || elem_size(dtype) == 0) return SKIPARSE_EINVAL;
    *moved = order != SKIPARSE_ORDER_SAME && s != 1;
    Shape sh;
    const int rc = *moved ? check_shape(B, 1, T, H, W, cols, s, pattern, &sh) : check_rows(B, 1, T, H, W, cols, &sh);
    if (rc != SKIPARSE_OK) return rc;
    if (dtype == SKIPARSE_FP8_E4M3 || cols % 8 != 0 || (uint32_t)cols > NORM_MAX_COLS) return SKIPARSE_EUNSUPPORTED;
    *rows = (size_t)B * sh.n_tok;
    return SKIPARSE_OK;
}
// Which row of the source a row of the destination takes, where rows move from the original order to the sparse layout or back.
static RowArgs row_args(int B, int T, int H, int W, int s, int pattern, bool to_sparse) {
    const GridMap g = make_gridmap(T, H, W, s, pattern);
    return to_sparse ? make_row_args<TO_SPARSE>(g, (uint32_t)B) : make_row_args<TO_ORIGINAL>(g, (uint32_t)B);
}
// no denormal number, and so far from the largest that it can be added to a mean of squares
static bool valid_eps(float eps) { return eps >= 0x1p-126f && eps <= 0x1p100f; }

int skiparse_rmsnorm_fwd(const void* x, const void* residual, const void* weight, void* sum, void* out, float* out_scales, int B, int T, int H, int W, int cols,
                         float eps, int s, int pattern, int order, int dtype, void* stream) {
    if (!x || !out || (sum && !residual) || !valid_eps(eps)) return SKIPARSE_EINVAL;
    bool moved;
    size_t rows;
    const int rc = rows_common(B, T, H, W, cols, s, pattern, order, dtype, &moved, &rows);
    if (rc != SKIPARSE_OK) return rc;
    for (const void* p : {x, residual, weight, (const void*)sum, (const void*)out})
        if (p && misaligned(p)) return SKIPARSE_EINVAL;
    if (misaligned_float(out_scales)) return SKIPARSE_EINVAL;
    const size_t bytes = rows * cols * elem_size(dtype);
    const Span sx = {x, bytes}, sr = {residual, bytes}, sw = {weight, (size_t)cols * elem_size(dtype)}, ss = {sum, bytes};
    const Span so = {out, out_scales ? rows * cols : bytes}, sc = {out_scales, rows * sizeof(float)};
    if (touches(so, {sr, sw, ss, sc}) || touches(sc, {sx, sr, sw, ss}) || touches(ss, {sw})) return SKIPARSE_EINVAL;
    if (touches(so, {sx}) && (out != x || moved || out_scales)) return SKIPARSE_EINVAL;
    if ((touches(ss, {sx}) && sum != x) || (touches(ss, {sr}) && sum != residual)) return SKIPARSE_EINVAL;
    NormArgs a = {};
    a.x = x; a.residual = residual; a.weight = weight; a.sum = sum; a.out = out; a.scales = out_scales;
    a.n_rows = (uint32_t)rows; a.cols = (uint32_t)cols;
    a.eps = eps;
    a.kind = out_scales ? ROWS_NORM_QUANTIZED : ROWS_NORM;
    a.f32 = dtype == SKIPARSE_FP32;
    a.order = moved ? order : SKIPARSE_ORDER_SAME;
    if (moved) a.rows = row_args(B, T, H, W, s, pattern, order == SKIPARSE_ORDER_TO_SPARSE);
    return finish(launch_norm_rows(a, (hipStream_t)stream));
}

int skiparse_quantize_int8(const void* x, void* codes, float* scales, int B, int T, int H, int W, int cols, int s, int pattern, int order, int dtype, void* stream) {
    if (!x || !codes || !scales) return SKIPARSE_EINVAL;
    bool moved;
    size_t rows;
    const int rc = rows_common(B, T, H, W, cols, s, pattern, order, dtype, &moved, &rows);
    if (rc != SKIPARSE_OK) return rc;
    if (misaligned(x) || misaligned(codes) || misaligned_float(scales)) return SKIPARSE_EINVAL;
    const Span sx = {x, rows * cols * elem_size(dtype)}, so = {codes, rows * cols}, sc = {scales, rows * sizeof(float)};
    if (touches(so, {sx, sc}) || touches(sc, {sx})) return SKIPARSE_EINVAL;
    NormArgs a = {};
    a.x = x; a.out = codes; a.scales = scales;
    a.n_rows = (uint32_t)rows; a.cols = (uint32_t)cols;
    a.kind = ROWS_QUANTIZED;
    a.f32 = dtype == SKIPARSE_FP32;
    a.order = moved ? order : SKIPARSE_ORDER_SAME;
    if (moved) a.rows = row_args(B, T, H, W, s, pattern, order == SKIPARSE_ORDER_TO_SPARSE);
    return finish(launch_norm_rows(a, (hipStream_t)stream));
}

size_t skiparse_rmsnorm_bwd_workspace_bytes(int rows, int cols) {
    if (rows < 1 || cols < 1 || (uint32_t)cols > NORM_MAX_COLS) return 0;
    return (size_t)norm_bwd_parts((uint32_t)rows, (uint32_t)cols) * (size_t)cols * sizeof(float);
}

int skiparse_rmsnorm_bwd(const void* dy, const void* h, const void* weight, const void* dx_add, void* dx, void* dw, int B, int T, int H, int W, int cols, float eps,
                         int s, int pattern, int order, int dtype, void* workspace, size_t workspace_bytes, void* stream) {
    if (!dy || !h || (!dx && !dw) || (dx_add && !dx) || !valid_eps(eps)) return SKIPARSE_EINVAL;
    bool moved;
    size_t rows;
    const int rc = rows_common(B, T, H, W, cols, s, pattern, order, dtype, &moved, &rows);
    if (rc != SKIPARSE_OK) return rc;
    for (const void* p : {dy, h, weight, dx_add, (const void*)dx, (const void*)dw})
        if (p && misaligned(p)) return SKIPARSE_EINVAL;
    const size_t need = dw ? skiparse_rmsnorm_bwd_workspace_bytes((int)rows, cols) : 0;
    if (need && (!workspace || workspace_bytes < need || misaligned(workspace))) return SKIPARSE_EWORKSPACE;
    const size_t bytes = rows * cols * elem_size(dtype), wbytes = (size_t)cols * elem_size(dtype);
    const Span sy = {dy, bytes}, sh = {h, bytes}, sw = {weight, wbytes}, sa = {dx_add, bytes}, gx = {dx, bytes}, gw = {dw, wbytes}, ws = {need ? workspace : nullptr, need};
    if (touches(gx, {sy, sh, sw, gw, ws}) || touches(gw, {sy, sh, sw, sa, ws}) || touches(ws, {sy, sh, sw, sa})) return SKIPARSE_EINVAL;
    if (touches(gx, {sa}) && dx_add != dx) return SKIPARSE_EINVAL;
    NormBwdArgs a = {};
    a.dy = dy; a.h = h; a.weight = weight; a.dx_add = dx_add; a.dx = dx; a.dw = dw;
    a.parts = (float*)workspace;
    a.n_rows = (uint32_t)rows; a.cols = (uint32_t)cols;
    a.eps = eps;
    a.f32 = dtype == SKIPARSE_FP32;
    if (moved) {  // row of x -> row of the result that was made of it
        const bool back = order == SKIPARSE_ORDER_TO_SPARSE;
        a.order = back ? SKIPARSE_ORDER_TO_ORIGINAL : SKIPARSE_ORDER_TO_SPARSE;
        a.rows = row_args(B, T, H, W, s, pattern, !back);
    }
    return finish(launch_norm_bwd(a, (hipStream_t)stream));
}

// ---- linear layer in 8-bit integers

constexpr int INT8_MAX_FEATURES = 131056;  // 2^14 a product: 2^31 / 2^14 of them could leave 32 bits

size_t skiparse_linear_fwd_int8_workspace_bytes(int rows, int in_features, int out_features) {
    if (rows < 1 || in_features < 1 || out_features < 1) return 0;
    return linear_int8_workspace((uint32_t)rows, (uint32_t)out_features, (uint32_t)in_features);
}

int skiparse_linear_fwd_int8(const void* x, const float* x_scales, const void* w, const float* w_scales, const void* bias, const void* residual, void* out, int B, int T, int H,
                             int W, int in_features, int out_features, int s, int pattern, int order, int act, void* workspace, size_t workspace_bytes, void* stream) {
    if (!x || !x_scales || !w || !w_scales || !out) return SKIPARSE_EINVAL;
    bool moved;
    size_t rows;
    const int rc = linear_common(B, T, H, W, in_features, out_features, s, pattern, order, act, SKIPARSE_BF16, &moved, &rows);
    if (rc != SKIPARSE_OK) return rc;
    if (in_features % 16 != 0) return SKIPARSE_EUNSUPPORTED;
    if (in_features > INT8_MAX_FEATURES) return SKIPARSE_ESHAPE;
    for (const void* p : {x, (const void*)x_scales, w, (const void*)w_scales, bias, residual, (const void*)out})
        if (p && misaligned(p)) return SKIPARSE_EINVAL;
    const size_t K = (size_t)in_features, N = (size_t)out_features;
    if (!linear_fits(rows, N)) return SKIPARSE_ESHAPE;
    if (moved && rows * K >= (1ull << 32) - 64) return SKIPARSE_ESHAPE;  // rows that move are addressed with 32-bit byte offsets
    const Span sx = {x, rows * K}, sxs = {x_scales, rows * sizeof(float)}, sw = {w, N * K}, sws = {w_scales, N * sizeof(float)}, sb = {bias, N * 2}, sr = {residual, rows * N * 2};
    const Span so = {out, rows * N * 2};
    if (touches(so, {sx, sxs, sw, sws, sb}) || (residual != out && touches(so, {sr}))) return SKIPARSE_EINVAL;
    const size_t need = linear_int8_workspace((uint32_t)rows, (uint32_t)N, (uint32_t)K);
    if (need && (!workspace || workspace_bytes < need || misaligned(workspace))) return SKIPARSE_EWORKSPACE;
    if (touches({need ? workspace : nullptr, need}, {sx, sxs, sw, sws, sb, sr, so})) return SKIPARSE_EINVAL;
    LinearArgs a = {};
    a.p = x; a.q = w; a.x_scales = x_scales; a.w_scales = w_scales;
    a.M = (uint32_t)rows; a.N = (uint32_t)N; a.K = (uint32_t)K / 2u;
    a.e = {bias, residual, out, nullptr, nullptr, act};
    a.partial = (float*)workspace;
    a.order = moved ? order : SKIPARSE_ORDER_SAME;
    if (moved) a.rows = row_args(B, T, H, W, s, pattern, order == SKIPARSE_ORDER_TO_SPARSE);
    return finish(launch_linear_int8(a, (hipStream_t)stream));
}

const char* skiparse_strerror(int code) {
    switch (code) {
        case SKIPARSE_OK: return "ok";
        case SKIPARSE_EINVAL: return "invalid argument (null or misaligned pointer, non-positive size, unknown enum, overlapping buffers)";
        case SKIPARSE_ESHAPE: return "grid not divisible as the pattern requires, or sizes out of range";
        case SKIPARSE_EUNSUPPORTED: return "no kernel for this head_dim / element type";
        case SKIPARSE_EWORKSPACE: return "workspace missing, misaligned or too small (or, for the static-scratch entry point, the problem exceeds the scratch)";
        case SKIPARSE_EHIP: return "kernel launch failed (see skiparse_last_hip_error)";
        default: return "unknown error code";
    }
}

int skiparse_last_hip_error(void) { return g_last_hip_error; }

}  // extern "C"

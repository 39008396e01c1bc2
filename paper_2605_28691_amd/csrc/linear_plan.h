// How a product of the linear layer is cut into workgroups.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "index_map.h"

namespace skiparse {

// Tiles of C that workgroups take; LINEAR_SHAPES of them.
enum LinearShape : int { T256 = 0, T128 = 1, T64 = 2, T128X256 = 3, LINEAR_SHAPES = 4 };
struct LinearTile {
    uint32_t m, n;    // rows and channels of a tile
    uint32_t per_cu;  // workgroups that a CU holds
    float fixed;      // us of a workgroup outside its walk over k
    float few;        // us a step of 64 of k with few workgroups on the chip,
    float step[4];    // and with 1, 2, .. on every CU (the clock falls as the chip fills)
};
constexpr uint32_t LINEAR_CUS = 256;
constexpr uint32_t LINEAR_STEP = 64, LINEAR_STEPS = 2 * LINEAR_STEP;  // k is walked in pairs of steps
constexpr uint32_t LINEAR_MAX_PARTS = 16;
constexpr uint64_t LINEAR_GRID = 1ull << 24;  // a launch has fewer workgroups of 256: a grid, fewer than 2^32 threads
// Fitted to products of 28 sizes (1 to 32,760 rows, 256 to 20,480 channels, the three forms), each with every tile and several numbers of parts: over the last 36 of them what the
// rule takes is 1 % slower than the best in the mean, 9 % at most (profiles/linear_tiles.txt; without an epilogue, which the rule does not see, nor whether operands are transposed).  For example, us, 256 / 128 / 64 / 128 x 256, uncut: 8190 x 1536 -> 1536 36 / 43 / 60 / 48, dx of
// 6426 x 1000 -> 4008 82 / 71 / 120 / 53 (408 tiles of 128 are 80 % of a round of two a CU, 204 of 128 x 256 of a round of one; 256 x 128 64), 1000 x 2048 -> 2048
// 40 / 17 / 18 / 25; cut best: 3840 x 5120 -> 5120 155 / 173 / 285 / 184.
constexpr LinearTile LINEAR_TILE[LINEAR_SHAPES] = {
    {256, 256, 1, 7.6f, 0.945f, {1.3f}}, {128, 128, 2, 2.58f, 0.308f, {0.57f, 0.88f}}, {64, 64, 4, 1.45f, 0.241f, {0.302f, 0.39f, 0.61f, 0.883f}}, {128, 256, 1, 4.29f, 0.587f, {0.809f}}};
constexpr float LINEAR_JOIN = 3.2f, LINEAR_JOIN_BYTE = 2.3e-7f;  // us of the launch that joins parts, and of a byte that goes through memory

// us a step with `units` workgroups running, at most a full round
inline float linear_step(const LinearTile& t, uint64_t units) {
    if (units <= LINEAR_CUS) return t.few + (t.step[0] - t.few) * (float)units / (float)LINEAR_CUS;
    return t.step[(units - 1u) / LINEAR_CUS];
}

// Tiles in the order of their numbers: `whole` of them are one workgroup each, every other one `parts` workgroups of `per` of k.  Their sums are joined by a second launch.
struct LinearPlan {
    int shape;
    uint32_t tiles_m, tiles_n, whole, rest, parts, per;
    size_t workspace() const { return parts > 1 ? (size_t)rest * parts * LINEAR_TILE[shape].m * LINEAR_TILE[shape].n * 4u : 0u; }
};

// Whether a result of M x N can be written by one launch: by the largest tiles, uncut, if at all.
inline bool linear_fits(uint64_t M, uint64_t N) { return ((M + 255u) / 256u) * ((N + 255u) / 256u) < LINEAR_GRID; }

// Rows of a part of the pass in front of the backward's products, 256 channels a workgroup.  Small problems need the workgroups, large ones' parts would cost traffic: 4 bytes written
// and read of every 32 rows' 64 and more; beyond that as many as fit one launch.
inline uint32_t linear_rows_per_part(uint32_t M, uint32_t N) {
    uint32_t per = M < 32768u ? 32u : 128u;
    while (((uint64_t)M + per - 1u) / per * (((uint64_t)N + 255u) / 256u) >= LINEAR_GRID) per *= 2u;
    return per;
}
inline uint32_t linear_rows_parts(uint32_t M, uint32_t N) {
    const uint32_t per = linear_rows_per_part(M, N);
    return (uint32_t)(((uint64_t)M + per - 1u) / per);
}

// The last round of workgroups over the CUs is seldom full: its tiles are cut along k, into as many parts as make it shortest.
inline LinearPlan plan_linear(uint32_t M, uint32_t N, uint32_t K) {
    LinearPlan best = {};
    float best_cost = 0.f;
    for (int shape = 0; shape < LINEAR_SHAPES; shape++) {
        const LinearTile& t = LINEAR_TILE[shape];
        const uint64_t tiles_m = ((uint64_t)M + t.m - 1u) / t.m, tiles_n = ((uint64_t)N + t.n - 1u) / t.n, tiles = tiles_m * tiles_n;
        const uint64_t slots = (uint64_t)LINEAR_CUS * t.per_cu, rounds = tiles / slots, rest = tiles - rounds * slots;
        const uint32_t pairs = (uint32_t)(((uint64_t)K + LINEAR_STEPS - 1u) / LINEAR_STEPS);
        const float full = t.step[t.per_cu - 1u];
        for (uint32_t parts = 1; parts <= LINEAR_MAX_PARTS && parts <= pairs; parts++) {
            if (rest == 0 && parts > 1) break;
            const uint32_t per = (pairs + parts - 1u) / parts;
            if (parts > 1 && (uint64_t)(parts - 1u) * per >= pairs) continue;  // the last part would be empty
            const uint64_t units = rest * parts, again = units / slots, left = units - again * slots;
            if (tiles - rest + units >= LINEAR_GRID) break;
            float cost = (float)rounds * (t.fixed + 2.f * (float)pairs * full) + (float)again * (t.fixed + 2.f * (float)per * full);
            if (left) cost += t.fixed + 2.f * (float)per * linear_step(t, left);
            if (parts > 1) cost += LINEAR_JOIN + LINEAR_JOIN_BYTE * (float)(units * t.m * t.n * 4u);
            if (best_cost == 0.f || cost < best_cost) {
                best_cost = cost;
                best = {shape, (uint32_t)tiles_m, (uint32_t)tiles_n, (uint32_t)(parts > 1 ? tiles - rest : tiles), (uint32_t)(parts > 1 ? rest : 0), parts, per * LINEAR_STEPS};
            }
        }
    }
    return best;
}

// Whether x w^T with M rows goes to the kernels for few rows, which read w once, whatever is kept.  (us, these / tiles: 5120 -> 5120, 5 rows 12.5 / 19.3, 16 rows 14.4 / 19.4,
// 32 rows 17.8 / 19.7; 1536 -> 8960, 16 rows 8.4 / 12.8, 32 rows 11.3 / 12.9; 13,824 -> 5120, 16 rows 32.1 / 37.0, 32 rows 39.5 / 37.1; 64 -> 11,200, 16 rows 5.9 / 5.9, 32 rows
// 6.9 / 5.9.)
inline bool linear_few(uint32_t M, uint32_t K) { return M <= 16u || (M <= 32u && K >= 512u); }

// One row: channels of a wavefront, as many as leave 2048 wavefronts.
inline uint32_t row_channels(uint32_t N) { return N >= 8192u ? 4u : N >= 4096u ? 2u : 1u; }

// More: blocks of 16 channels of a workgroup.  Two halve what is read of x; one leaves more workgroups, and with up to 16 rows a CU has two of them (68 KB of LDS each; 104
// with up to 32), of which one can begin while the other ends.  (us, two / one: 5120 -> 5120, 2 rows 12.2 / 13.9, 16 rows 14.4 / 17.0; 5120 -> 13,824, 16 rows 30.4 / 32.9;
// 1536 -> 8960, 2 rows 9.4 / 8.1, 16 rows 9.7 / 8.4, 17 rows 11.0 / 11.8; 8960 -> 1536, 16 rows 11.9 / 8.7.)
inline uint32_t few_blocks(uint32_t M, uint32_t N, uint32_t K) { return N >= 4096u && (K >= 4096u || M > 16u) ? 2u : 1u; }

// Workgroup -> tile.  Workgroup id % 8 is the XCD; each XCD has a contiguous range of an order in which TILE_GROUP tiles of m are walked together along n, so that the 32
// tiles that it works on at once share operands in its L2.
constexpr uint32_t TILE_GROUP = 4;
struct TileMap {
    Div32 group;       // tiles of a group: TILE_GROUP * tiles_n
    Div32 size, last;  // tiles of m in a group, in the last one
    Div32 rest;        // tiles that are cut along k
    uint32_t tiles_m, whole, parts, per;
    static __host__ __device__ inline uint32_t of_xcd(uint32_t id, uint32_t total) {
        const uint32_t xcd = id & 7u, over = total & 7u;  // the first `over` XCDs have one more
        return xcd * (total >> 3) + (xcd < over ? xcd : over) + (id >> 3);
    }
    // tile number `lin`
    __host__ __device__ inline void tile(uint32_t lin, uint32_t& tm, uint32_t& tn) const {
        const uint32_t g = group.div(lin), in = lin - g * group.d, first = g * TILE_GROUP;
        const bool full = first + TILE_GROUP <= tiles_m;
        tn = full ? size.div(in) : last.div(in);
        tm = first + in - tn * (full ? size.d : last.d);
    }
    // workgroup `id`: its tile, its range of k, and for a part its number among the parts, else ~0
    __host__ __device__ inline void at(uint32_t id, uint32_t K, uint32_t& tm, uint32_t& tn, uint32_t& k0, uint32_t& k1, uint32_t& slot) const {
        k0 = 0u;
        k1 = K;
        slot = ~0u;
        if (id < whole) {
            tile(of_xcd(id, whole), tm, tn);
            return;
        }
        const uint32_t lin = of_xcd(id - whole, rest.d * parts);  // neighbours: tiles that walk the same k
        const uint32_t part = rest.div(lin), r = lin - part * rest.d;
        tile(whole + r, tm, tn);
        k0 = part * per;
        k1 = K - k0 < per ? K : k0 + per;
        slot = r * parts + part;
    }
};
inline TileMap make_tile_map(const LinearPlan& p) {
    const uint32_t over = p.tiles_m % TILE_GROUP;
    return {make_div32(TILE_GROUP * p.tiles_n), make_div32(TILE_GROUP), make_div32(over ? over : 1u), make_div32(p.rest ? p.rest : 1u), p.tiles_m, p.whole, p.parts, p.per};
}

}  // namespace skiparse

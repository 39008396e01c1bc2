// How a product of the linear layer is cut into workgroups.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace skiparse {

// Tiles of C that workgroups take; LINEAR_SHAPES of them.
enum LinearShape : int { T256 = 0, T128 = 1, T64 = 2, LINEAR_SHAPES = 3 };
struct LinearTile {
    uint32_t m, n;      // rows and channels of a tile
    uint32_t per_cu;    // workgroups that a CU holds
    float fixed;        // us of a workgroup outside its walk over k
    float step, last;   // us a step of 64 of k with all CUs busy, and with few
};
constexpr uint32_t LINEAR_CUS = 256;
constexpr uint32_t LINEAR_STEP = 64, LINEAR_STEPS = 2 * LINEAR_STEP;  // k is walked in pairs of steps
constexpr uint32_t LINEAR_MAX_PARTS = 16;
constexpr LinearTile LINEAR_TILE[LINEAR_SHAPES] = {{256, 256, 1, 7.f, 1.4f, 1.0f}, {128, 128, 2, 4.f, 0.9f, 0.5f}, {64, 64, 4, 3.f, 0.6f, 0.3f}};
constexpr float LINEAR_JOIN = 4.f, LINEAR_JOIN_BYTES = 2.0e-7f;  // us of the launch that joins parts, and of a byte that goes through memory

// Tiles in the order of their numbers: `whole` of them are one workgroup each, every other one `parts` workgroups of `per` of k.  Their sums are joined by a second launch.
struct LinearPlan {
    int shape;
    uint32_t tiles_m, tiles_n, whole, rest, parts, per;
    size_t workspace() const { return parts > 1 ? (size_t)rest * parts * LINEAR_TILE[shape].m * LINEAR_TILE[shape].n * 4u : 0u; }
};

// The last round of workgroups over the CUs is seldom full: its tiles are cut along k, into as many parts as make it shortest.
inline LinearPlan plan_linear(uint32_t M, uint32_t N, uint32_t K) {
    LinearPlan best = {};
    float best_cost = 0.f;
    for (int shape = 0; shape < LINEAR_SHAPES; shape++) {
        const LinearTile& t = LINEAR_TILE[shape];
        const uint64_t tiles_m = ((uint64_t)M + t.m - 1u) / t.m, tiles_n = ((uint64_t)N + t.n - 1u) / t.n, tiles = tiles_m * tiles_n;
        const uint64_t slots = (uint64_t)LINEAR_CUS * t.per_cu, rounds = tiles / slots, rest = tiles - rounds * slots;
        const uint32_t pairs = (uint32_t)(((uint64_t)K + LINEAR_STEPS - 1u) / LINEAR_STEPS);
        const float walk = 2.f * (float)pairs, full = (float)rounds * (t.fixed + walk * t.step);
        for (uint32_t parts = 1; parts <= LINEAR_MAX_PARTS && parts <= pairs; parts++) {
            if (rest == 0 && parts > 1) break;
            const uint32_t per = (pairs + parts - 1u) / parts;
            if (parts > 1 && (uint64_t)(parts - 1u) * per >= pairs) continue;  // the last part would be empty
            const uint64_t units = rest * parts, again = (units + slots - 1u) / slots;
            const uint64_t running = units < slots ? units : slots;
            const float step = t.last + (t.step - t.last) * (float)running / (float)slots;
            float cost = full + (float)again * (t.fixed + 2.f * (float)per * step);
            if (parts > 1) cost += LINEAR_JOIN + LINEAR_JOIN_BYTES * (float)(units * t.m * t.n * 4u);
            if (best_cost == 0.f || cost < best_cost) {
                best_cost = cost;
                best = {shape, (uint32_t)tiles_m, (uint32_t)tiles_n, (uint32_t)(parts > 1 ? tiles - rest : tiles), (uint32_t)(parts > 1 ? rest : 0), parts, per * LINEAR_STEPS};
            }
        }
    }
    return best;
}

}  // namespace skiparse

// Cuts products of the linear layer into workgroups (paper_2605_28691_amd/csrc/linear_plan.h) on the host.  Reads M N K, one product a line; prints, for each, the tile's rows and channels, whole
// tiles, cut tiles, parts, bytes of workspace, and "ok" where every place of C and k is some workgroup's once and every part has a slot of its own.  Built and run by
// tests/test_linear_plan.py.
#include <cstdio>
#include <map>
#include <set>
#include <utility>

#include "../paper_2605_28691_amd/csrc/linear_plan.h"

using namespace skiparse;

int main() {
    unsigned M, N, K;
    while (scanf("%u %u %u", &M, &N, &K) == 3) {
        const LinearPlan p = plan_linear(M, N, K);
        const LinearTile& t = LINEAR_TILE[p.shape];
        const TileMap map = make_tile_map(p);
        const unsigned blocks = p.whole + p.rest * p.parts, tiles = p.tiles_m * p.tiles_n;
        const char* bad = nullptr;
        if ((uint64_t)p.tiles_m * t.m < M || (uint64_t)p.tiles_n * t.n < N || p.whole + p.rest != tiles) bad = "tiles";
        std::map<std::pair<unsigned, unsigned>, std::map<unsigned, unsigned>> walked;  // tile -> ranges of k
        std::set<unsigned> slots;
        for (unsigned id = 0; id < blocks && !bad; id++) {
            uint32_t tm, tn, k0, k1, slot;
            map.at(id, K, tm, tn, k0, k1, slot);
            if (tm >= p.tiles_m || tn >= p.tiles_n) bad = "outside";
            if (k0 >= k1 || k1 > K || k0 % LINEAR_STEPS != 0) bad = "range of k";
            if (!walked[{tm, tn}].emplace(k0, k1).second) bad = "twice";
            if (id < p.whole ? slot != ~0u : slot >= p.rest * p.parts || !slots.insert(slot).second) bad = "slot";
            if (id >= p.whole && !bad) {  // the join reads tile `whole + slot / parts`, and its parts in order
                uint32_t jm, jn;
                map.tile(p.whole + slot / p.parts, jm, jn);
                if (jm != tm || jn != tn || k0 != slot % p.parts * p.per) bad = "join";
            }
        }
        if (!bad && walked.size() != tiles) bad = "missing tile";
        for (const auto& w : walked) {
            unsigned at = 0;
            for (const auto& r : w.second) {
                if (r.first != at) bad = "gap";
                at = r.second;
            }
            if (at != K) bad = "end of k";
        }
        printf("%u %u %u %u %u %zu %s\n", t.m, t.n, p.whole, p.rest, p.parts, p.workspace(), bad ? bad : "ok");
    }
}

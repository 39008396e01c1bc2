// Plans of the products in 8-bit integers (paper_2605_28691_amd/csrc/linear_plan.h) on the host.  Reads M, N and codes of a row, one product a line; prints which kernel for few rows it takes (0: none, 1: one row, else
// 2 + blocks of 16 channels + 2 for over 16 rows) and, without and with an activation, tile and parts, and "ok" where the parts are every tile's k once.  Built and run by tests/test_linear8_plan.py.
#include <cstdio>
#include <map>
#include <set>
#include <utility>

#include "../paper_2605_28691_amd/csrc/linear_plan.h"

using namespace skiparse;

int main() {
    unsigned M, N, codes;
    while (scanf("%u %u %u", &M, &N, &codes) == 3) {
        const unsigned K = codes / 2;
        printf("%u", !linear_few8(M, N, codes) ? 0u : M == 1u ? 1u : few_blocks8(M, N, codes) + (M > 16u ? 2u : 0u) + 2u);
        for (int act = 0; act < 2; act++) {
            const LinearPlan p = plan_linear8(M, N, K, act != 0);
            const TileMap map = make_tile_map(p);
            const unsigned blocks = p.whole + p.rest * p.parts, tiles = p.tiles_m * p.tiles_n;
            bool ok = blocks > 0 && blocks < LINEAR_GRID && p.whole + p.rest == tiles && (uint64_t)p.tiles_m * LINEAR_TILE[p.shape].m >= M && (uint64_t)p.tiles_n * LINEAR_TILE[p.shape].n >= N;
            std::map<std::pair<unsigned, unsigned>, std::map<unsigned, unsigned>> walked;
            std::set<unsigned> slots;
            for (unsigned id = 0; ok && id < blocks; id++) {
                uint32_t tm, tn, k0, k1, slot;
                map.at(id, K, tm, tn, k0, k1, slot);
                ok = tm < p.tiles_m && tn < p.tiles_n && k0 < k1 && k1 <= K && k0 % LINEAR_STEPS == 0 && walked[{tm, tn}].emplace(k0, k1).second;
                if (id >= p.whole) ok = ok && slot < p.rest * p.parts && slots.insert(slot).second;
            }
            for (const auto& w : walked) {
                unsigned at = 0;
                for (const auto& r : w.second) {
                    ok = ok && r.first == at;
                    at = r.second;
                }
                ok = ok && at == K;
            }
            printf(" %u %u %u %s", LINEAR_TILE8[p.shape].m, LINEAR_TILE8[p.shape].n, p.parts, ok && walked.size() == tiles ? "ok" : "bad");
        }
        printf("\n");
    }
}

// How the passes over rows (norm.hip) are cut: which lanes have a row, and how many pieces of 8 channels each of them.
#pragma once
#include <stdint.h>

namespace skiparse {

constexpr uint32_t NORM_WAVES = 16;          // of a workgroup that has a row, at most
constexpr uint32_t NORM_BWD_THREADS = 256;   // of one whose wavefronts have a row each

// threads of a workgroup that has a row, at most, with `ch` pieces a lane
constexpr uint32_t norm_group_threads(int ch) { return ch >= 8 ? 32u * NORM_WAVES : 64u * NORM_WAVES; }

enum NormSpan : int { SPAN_LANES = 0, SPAN_WAVE = 1, SPAN_GROUP = 2 };  // a row: of a part of a wavefront, of one, of a workgroup
struct NormShape {
    int span, ch;            // pieces of a lane
    uint32_t lanes, threads; // of a row (SPAN_LANES); of a workgroup
};

inline uint32_t norm_lanes(uint32_t pieces) {
    uint32_t lanes = 1u;
    while (lanes < pieces) lanes *= 2u;
    return lanes;
}

inline NormShape norm_shape(uint32_t rows, uint32_t cols) {
    const uint32_t pieces = (cols + 7u) / 8u;
    if (pieces <= 32u) return {SPAN_LANES, 1, norm_lanes(pieces), 256u};
    const uint32_t per_lane = (pieces + 63u) / 64u;
    if (rows >= 2048u && per_lane <= 10u) {
        for (int ch : {1, 2, 3, 4, 6, 8, 10})
            if ((uint32_t)ch >= per_lane) return {SPAN_WAVE, ch, 64u, 256u};
    }
    const uint32_t most = rows >= 2048u ? 8u : 1u;
    for (int ch : {1, 2, 4, 8}) {
        const uint32_t waves = (per_lane + (uint32_t)ch - 1u) / (uint32_t)ch;
        if (waves <= NORM_WAVES && (uint32_t)ch >= most) return {SPAN_GROUP, ch, 64u, 64u * waves};
    }
    return {SPAN_GROUP, 4, 64u, 64u * NORM_WAVES};
}

struct NormBwdShape {
    int span, ch;
    uint32_t lanes, threads, parts;
};
inline NormBwdShape norm_bwd_shape(uint32_t rows, uint32_t cols) {
    const uint32_t pieces = (cols + 7u) / 8u, per_lane = (pieces + 63u) / 64u;
    NormBwdShape s;
    uint32_t at_once = 1u;  // rows of a workgroup
    if (pieces <= 32u) {
        s = {SPAN_LANES, 1, norm_lanes(pieces), NORM_BWD_THREADS, 0u};
        at_once = NORM_BWD_THREADS / s.lanes;
    } else if (per_lane <= 4u) {
        s = {SPAN_WAVE, (int)per_lane, 64u, NORM_BWD_THREADS, 0u};
        at_once = NORM_BWD_THREADS / 64u;
    } else {
        const uint32_t ch = per_lane <= 48u ? 3u : 4u;
        s = {SPAN_GROUP, (int)ch, 64u, 64u * ((per_lane + ch - 1u) / ch), 0u};
    }
    const uint32_t rounds = (rows + at_once - 1u) / at_once;
    s.parts = rounds < 1024u ? rounds : 1024u;
    return s;
}

}  // namespace skiparse

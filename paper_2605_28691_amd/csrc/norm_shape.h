// How the passes over rows (norm.hip) are cut: which lanes have a row, and how many pieces of 8 channels each of them.
#pragma once
#include <stdint.h>

namespace skiparse {

constexpr uint32_t NORM_WAVES = 16;          // of a workgroup that has a row, at most
constexpr uint32_t NORM_BWD_THREADS = 256;   // of one whose wavefronts have a row each

// Bytes that a call moves, from which on nothing of them is worth a place in the caches.  (us, past them / through them: 80,640 x 5120 with residual 542 / 558, 32,760 x 1536 in codes 62.5 / 68.9, their gradients 633 / 660
// and 82.9 / 88.2; 3840 x 5120 in codes, 98 MB, 33.2 / 30.7.)
constexpr uint64_t NORM_PAST_CACHES = 256ull << 20;

enum NormSpan : int { SPAN_LANES = 0, SPAN_WAVE = 1, SPAN_GROUP = 2 };  // a row: of a part of a wavefront, of one, of a workgroup
struct NormShape {
    int span, ch;            // pieces of a lane
    uint32_t lanes, threads; // of a row (SPAN_LANES); of a workgroup
};

// Rows that lanes have at once, `read` bytes of a channel: two where a part of a wavefront has a row and a lane no more than 16 bytes of it on their way, in calls past the caches.  (us, one / two: 3,225,600 rows of
// 128 channels in bf16 285 / 270, quantised 224 / 207; with residual, 800,000 x 256, 268 / 283; 2,000,000 x 64 in float32 170 / 175; rows of a wavefront, 131,040 x 1536 with residual 264 / 284; through the caches,
// 393,120 x 128, 42.6 / 43.4.)
constexpr uint32_t norm_turns(int span, uint32_t read, bool past_caches) { return past_caches && span == SPAN_LANES && read <= 2u ? 2u : 1u; }

inline uint32_t norm_lanes(uint32_t pieces) {
    uint32_t lanes = 1u;
    while (lanes < pieces) lanes *= 2u;
    return lanes;
}

// `read`: bytes that are read for a channel.  What counts is that enough of them are on their way: 16 workgroups of few wavefronts a CU, or fewer of more; with rows of more than 3 pieces a lane the wavefronts of
// a workgroup share one, two pieces a lane where a channel has 2 bytes, one otherwise.  (us, rows of a wavefront / of a workgroup with 1, 2, 4 pieces a lane: 80,640 x 5120 with residual 579 / 535 / 562 / 564,
// quantised 225 / 308 / 217 / 225; 32,760 x 1536 with residual, quantised 57.3 / 59.8 / 58.6 / 58.3; 6426 x 4008 float32 with residual - / 75.8 / 78.8 / 82.7; one row of 5120 4.9 / 2.6 / 2.9 / 3.6,
// 256 rows 8.7 / 5.3 / 5.6 / 6.2.)
inline NormShape norm_shape(uint32_t rows, uint32_t cols, uint32_t read) {
    const uint32_t pieces = (cols + 7u) / 8u, per_lane = (pieces + 63u) / 64u;
    if (pieces <= 32u) return {SPAN_LANES, 1, norm_lanes(pieces), 256u};
    if (per_lane == 1u || (rows >= 1024u && per_lane <= 3u)) return {SPAN_WAVE, (int)per_lane, 64u, 256u};
    for (int ch : {rows >= 1024u && read <= 2u ? 2 : 1, 2}) {
        const uint32_t waves = (per_lane + (uint32_t)ch - 1u) / (uint32_t)ch;
        if (waves <= NORM_WAVES) return {SPAN_GROUP, ch, 64u, 64u * waves};
    }
    return {SPAN_GROUP, 4, 64u, 64u * ((per_lane + 3u) / 4u)};
}

struct NormBwdShape {
    int span, ch;
    uint32_t lanes, threads, parts;
};
// Parts: enough wavefronts for the chip, and no more, since a part's sums are written and read once more; few rows in few parts.  (us, 256 / 512 / 768 / 1024 parts: 32,760 x 1536, 3 wavefronts a row, 119 / 85 / 83 / 82;
// 3840 x 5120, 10 wavefronts, 38 / 41 / 41 / 44; 390 x 1536 7.4 / 8.3 / 8.3 / 8.3; 80,640 x 1024, a wavefront a row and 4 in a workgroup, 128 / 136 / 138 / 143.)  Narrow rows' parts cost little: twice as many, and
// of fewer rows (as the others / so: 3,225,600 x 128 496 / 485, 393,120 x 128 67.5 / 63.0, 64,260 x 128 19.2 / 17.2, 20,000 x 256 in float32 24.9 / 20.7; four times as many 505, 65.8, 21.4, 22.2).
// Rounds of a part, 8 / 4: a wavefront a row, 16,000 x 512 18.7 / 17.8, 16,000 x 1000 28.5 / 26.7.  Rows of more than 16,384 channels in float32 do
// not fit the registers with all that the pass keeps: 4000 x 32,768 507 us, floor 420 (bf16 245, 210).
inline NormBwdShape norm_bwd_shape(uint32_t rows, uint32_t cols) {
    const uint32_t pieces = (cols + 7u) / 8u, per_lane = (pieces + 63u) / 64u;
    NormBwdShape s;
    uint32_t at_once = 1u;  // rows of a workgroup
    if (pieces <= 32u) {
        s = {SPAN_LANES, 1, norm_lanes(pieces), NORM_BWD_THREADS, 0u};
        at_once = NORM_BWD_THREADS / s.lanes;
    } else if (per_lane <= 2u) {
        s = {SPAN_WAVE, (int)per_lane, 64u, NORM_BWD_THREADS, 0u};
        at_once = NORM_BWD_THREADS / 64u;
    } else {
        const uint32_t ch = per_lane <= 16u ? 1u : per_lane <= 32u ? 2u : 4u;
        s = {SPAN_GROUP, (int)ch, 64u, 64u * ((per_lane + ch - 1u) / ch), 0u};
    }
    const uint32_t rounds = (rows + at_once - 1u) / at_once, waves = s.threads / 64u;
    const bool narrow = s.span == SPAN_LANES;
    const uint32_t each = rounds / (narrow ? 2u : s.span == SPAN_WAVE ? 4u : 8u), most = (narrow ? 512u : 256u) * ((7u + waves) / waves), few = each > 256u ? each : 256u;
    s.parts = most < few ? most : few;
    if (s.parts > rounds) s.parts = rounds;
    return s;
}

}  // namespace skiparse

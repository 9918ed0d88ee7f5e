// How a call of attention to an encoder's states is cut into launches: by its sizes and the compute units
// `cus` alone, on the host.
#pragma once
#include <algorithm>
#include <cstdint>

#include "ts3_cross.h"

namespace ts3 {

// B samples, HK shared heads each, with R rows (points and the head's sharers) of S states.
struct CrossSize {
    int64_t B, HK, R, S;
    bool lengths;
    int64_t pairs() const { return B * HK; }
};

constexpr int64_t CROSS_ROWS_MAX = (int64_t(1) << 31) - 1024;
constexpr int64_t CROSS_WGS_MAX = int64_t(1) << 24;  // of 256 threads: fewer than 2^32 of them

// Whether there is a launch: the most workgroups are those of four waves, 128 rows or states each.
inline bool cross_fits(const CrossSize &c) {
    return c.R <= CROSS_ROWS_MAX && c.S <= CROSS_ROWS_MAX && c.pairs() <= CROSS_WGS_MAX &&
           c.pairs() * ((c.R + 127) / 128) < CROSS_WGS_MAX && c.pairs() * ((c.S + 127) / 128) < CROSS_WGS_MAX;
}

// A loop of tiles in `splits` parts of `per`.
struct CrossCut {
    int64_t splits, per;
};
// Splits `tiles` of a loop so that the workgroups (of `blocks` blocks per sample and shared head) become
// about `target`, each of two tiles at least.
inline CrossCut cross_cut(const CrossSize &c, int64_t blocks, int64_t tiles, int64_t target) {
    const int64_t wgs = c.pairs() * blocks;
    const int64_t s = std::max<int64_t>(1, std::min(target / std::max<int64_t>(wgs, 1), tiles / 2));
    const int64_t per = std::max<int64_t>(1, (tiles + s - 1) / s);
    return {std::max<int64_t>(1, (tiles + per - 1) / per), per};
}

// Workgroups per sample and shared head of the kernels that hold all states in LDS, one per compute unit at a time; 0
// where these do not fit, or where the rows are too few.
template <typename All> int64_t cross_all(const CrossSize &c, int64_t cus) {
    if (!All::FITS || c.S == 0 || All::bytes(c.S) > All::LDS) return 0;
    // Each workgroup's blocks of 32 rows: four a wave at least, or filling LDS and uneven ends cost more than it saves.
    // 2,048 samples and heads of 32 against 512 states, here and in the four-wave kernels: 256 rows each forward 139 and
    // 92 us, 512 170 and 139, 1,024 281 and 267, 2,048 500 and 520.  So a grid has less than 2^30 threads, too.
    const int64_t blocks = (c.R + 31) / 32, per = std::max<int64_t>(1, cus / c.pairs());
    if (blocks < 4 * All::W * per || blocks * c.pairs() < 4 * All::W * cus) return 0;
    // Of the units' rounds, seven tenths at least, which the four-wave kernels' smaller workgroups fill: 32,768 rows each
    // of 512 states, heads of 32, here and there: 264 samples and heads (0.52 of two rounds) forward 1,472 and 1,032 us,
    // the gradient 4,051 and 3,317, 136 (0.53) 709 and 539, 1,951 and 1,773, 160 (0.63) 699 and 629, 2,028 and 1,963,
    // 192 (0.75) 722 and 754, 2,203 and 2,217, 256 870 and 996, 2,817 and 2,991.
    const int64_t wgs = c.pairs() * per, rounds = (wgs + cus - 1) / cus;
    return 10 * wgs < 7 * rounds * cus ? 0 : per;
}

// CROSS_ONE: a workgroup is a wave of 32 rows; CROSS_FOUR: four waves; CROSS_ALL: all states in LDS.
enum CrossKind { CROSS_ONE, CROSS_FOUR, CROSS_ALL };
enum CrossJoin { CROSS_WHOLE, CROSS_JOIN_FEW, CROSS_JOIN };
struct CrossPlan {
    CrossKind kind;
    int64_t blocks;  // workgroups per sample and shared head, before the split
    CrossCut cut;
    CrossJoin join;
};

template <int P, int DP> CrossPlan cross_forward_plan(const CrossSize &c, int64_t cus) {
    // A wave of its own for a row or a few (float32 heads of 128 would not fit its registers).
    const bool one = DP * P <= 192 && c.R <= 32;
    if (!one)
        if (const int64_t per = cross_all<CrossAll<P, DP, 16>>(c, cus); per > 0) return {CROSS_ALL, per, {1, per}, CROSS_WHOLE};
    const int64_t W = one ? 1 : 4, TK = one ? cross_tile<P, DP, 1>() : cross_tile<P, DP, 4>();
    const int64_t blocks = (c.R + 32 * W - 1) / (32 * W);
    // As many workgroups as fit: 30,000 rows of width 32 against 2,782 states 67 us with two a unit, 37 with four.
    // With lengths, twice as many for few rows: those of long samples take as long as their own loops (4 samples
    // of up to 100,003 states, two heads of 64: 40 against 37 us; of 128 wide, 32 states a tile, 66 against 71).
    const int64_t units = one ? c.lengths && DP < 128 ? 16 : 8 : DP * P <= 32 ? 4 : 2;
    const CrossCut cut = cross_cut(c, blocks, (c.S + TK - 1) / TK, units * cus);
    // 12,496 rows of width 80 in two parts: 67 us in all with a workgroup a row, 45 with lanes
    const bool few = cut.splits <= 16 && (c.pairs() * c.R * (DP / 4) + 255) / 256 >= cus;
    return {one ? CROSS_ONE : CROSS_FOUR, blocks, cut, cut.splits == 1 ? CROSS_WHOLE : few ? CROSS_JOIN_FEW : CROSS_JOIN};
}

struct CrossBackwardPlan {
    CrossKind kind;             // of dq
    int64_t qblocks, vblocks;   // workgroups per sample and shared head, before the split
    CrossCut q, v;
};
template <int P, int DP> CrossBackwardPlan cross_backward_plan(const CrossSize &c, int64_t cus) {
    constexpr int T = P == 1 && DP < 128 ? 64 : 32;
    CrossBackwardPlan p{CROSS_FOUR, (c.R + 127) / 128, (c.S + 127) / 128, {}, {}};
    p.q = cross_cut(c, p.qblocks, (c.S + T - 1) / T, 2 * cus);
    if (const int64_t per = cross_all<CrossAll<P, DP, CROSS_DQ_WAVES<DP * P>>>(c, cus); per > 0) {
        p.kind = CROSS_ALL;
        p.qblocks = per;
        p.q = {1, per};
    }
    p.v = cross_cut(c, p.vblocks, (c.R + T - 1) / T, (DP * P <= 48 ? 3 : 2) * cus);
    return p;
}

}  // namespace ts3

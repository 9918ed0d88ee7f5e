// How a call of the gated feed-forward is cut: by its sizes and the compute units `cus` alone, on the
// host.
#pragma once
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "ts3_gated.h"

namespace ts3 {

// Splits of the hidden units over workgroups, for a call of n points in nb blocks that leaves
// compute units idle.  S splits take chunks / S steps of t us (what one workgroup alone on its
// compute unit takes: 0.5 us and 5 ns per channel, 18 in float32), and write and read S sums of
// n CP floats at 1.9 TB/s together: the sum of both is least at S = sqrt(chunks t / sums).
inline int gated_splits(int64_t n, int64_t nb, int nchunk, int P, int CP, int cus) {
    const double t = 0.5 + (P == 1 ? 0.005 : 0.018) * CP, sums = (double)n * CP * 4 / 1.9e6;
    const int64_t best = (int64_t)std::ceil(std::sqrt(nchunk * t / sums));
    const int64_t s = std::max<int64_t>(1, std::min(std::min<int64_t>(best, nchunk), cus / std::max<int64_t>(nb, 1)));
    const int per = (int)((nchunk + s - 1) / s);
    return (nchunk + per - 1) / per;
}

// The forward's HW, for `wgs` workgroups of `per` chunks: one workgroup per compute unit or none takes
// two waves per SIMD on the same points.  At C = 256, F = 1024 in bfloat16, with one wave in brackets:
// 20,000 points 48 us (52.5), 32,768 58 (59); 32,769, on one wave, 62.6.  Of few points in short
// splits it loses: 4,096 in six splits 28.3 us (26.6), in float32 at C = 128, F = 512 25.2 (23.4).
template <int P, int CP> int gated_halves(int64_t wgs, int per, int cus) {
    return GatedShape<P, CP>::OCC == 2 && per > 1 && wgs <= cus ? 2 : 1;
}

// Waves of the weight gradients' workgroups: eight where they cover the hidden units with no more
// than an eighth of their products on units that do not exist.
template <int P, int CP> int gated_dw_waves(int nchunk) {
    if constexpr (GatedDwWide<P, CP>::USE8) {
        constexpr int HB = GatedDw<P, CP, 8>::HB;
        const int F = nchunk * 32, covered = (F + HB - 1) / HB * HB;
        if (8 * (covered - F) <= covered) return 8;
    }
    return 4;
}

// Splits of the points for the weight gradients: at most eight waves per compute unit in all.  A
// split costs its sums, 3 F C floats written and read at 2.5 TB/s together, and saves
// steps of KP points (0.6 us each, 0.8 in float32), so few points take fewer: of 3,000 at C =
// 256, F = 1024 in bfloat16, 21 splits took 34 us with their sums, 7 take 22.
template <int P, int CP> int gated_point_splits(int nchunk, int64_t points, int cus) {
    using Dw = GatedDw<P, CP, 4>;
    const int W = gated_dw_waves<P, CP>(nchunk), HB = Dw::HB / 4 * W;
    const int nhb = (nchunk * 32 + HB - 1) / HB;
    const int64_t most = std::max<int64_t>(1, (int64_t)(8 / W) * cus / (3 * nhb));
    const double steps = (double)points / Dw::KP * (P == 1 ? 0.6 : 0.8), sums = 3.0 * nchunk * 32 * CP * 4 / 2.5e6;
    return (int)std::min<int64_t>(most, std::max<int64_t>(1, (int64_t)std::ceil(std::sqrt(steps / sums))));
}

}  // namespace ts3

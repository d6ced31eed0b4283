// How rows of a layer norm are dealt to lanes and workgroups.  Plain C++ (no device code), shared by the launcher and host-side tests.
#pragma once

#include <stdint.h>

#include "tile_walk.hpp"

namespace sv {

// n / d for 0 <= n < 2^31 by a product and shifts: with 2^(s-1) < d <= 2^s and M = floor(2^(31+s) / d) + 1, M d exceeds 2^(31+s) by at most d <=
// 2^s, so n M / 2^(31+s) exceeds n / d by less than 1 / d.  (A division proper is some twenty-five instructions, and rows of 112 features have
// not much more arithmetic than that: 93 600 rows 13.8 us.)
struct NormDivisor {
    uint32_t extent, mul, shift;
    static NormDivisor of(int32_t d)
    {
        uint32_t s = 0;
        while (((int64_t)1 << s) < d) ++s;
        return NormDivisor{(uint32_t)d, (uint32_t)((((uint64_t)1 << (31 + s)) / (uint32_t)d) + 1), s};
    }
    SV_HOST_DEVICE uint32_t quotient(uint32_t n) const { return (uint32_t)(((uint64_t)n * mul >> 31) >> shift); }
};

// A row is held by `lanes` lanes, `vecs` 16-byte pieces each: lanes <= 64 lie in one wave (64 / lanes rows of a wave side by side),
// 128 and more in two waves and more of a workgroup of 256, or in all of a workgroup of 512 or 1024.
struct NormForm {
    int lanes, vecs;
};

constexpr int kNormMostWidth = 8192;         // features of the widest row: 1 024 pieces of bf16, 2 048 of fp32

// The form for rows of `pieces` 16-byte pieces; lanes == 0: none.  Forwards a row stays in one wave while it fits six pieces per lane (2 240
// features of bf16, 32 760 rows: 64 x 5 48 us, 128 x 3 54); backwards, where a lane also keeps the sums of its features' gradients, three
// (64 x 5 101 us, 128 x 3 96, 256 x 2 122; 1 504 features: 64 x 3 88, 128 x 2 104), and four over two waves (4 096: 128 x 4 92, 256 x 2 99).
inline NormForm norm_form(int pieces, bool backward)
{
    if (pieces <= 0 || pieces > kNormMostWidth / 4) return NormForm{0, 0};
    for (int lanes = 4; lanes <= 64; lanes *= 2)
        if (pieces <= lanes) return NormForm{lanes, 1};
    if (pieces <= 64 * (backward ? 3 : 6)) return NormForm{64, (pieces + 63) / 64};
    if (pieces <= 128 * 4) return NormForm{128, (pieces + 127) / 128};
    if (pieces <= 256 * 3) return NormForm{256, 3};
    return NormForm{pieces <= 1024 ? 512 : 1024, 2};
}

inline int norm_threads(const NormForm &f) { return f.lanes > 256 ? f.lanes : 256; }
inline int norm_rows_per_step(const NormForm &f) { return norm_threads(f) / f.lanes; }

// Workgroups of one group of rows (rows that share a row of parameters): `most` for all groups together, none without a row.
inline int norm_workgroups(const NormForm &f, int64_t rows, int64_t groups, int most)
{
    const int per = norm_rows_per_step(f);
    const int64_t steps = (rows + per - 1) / per;
    int64_t n = most / groups;
    if (n > steps) n = steps;
    return n < 1 ? 1 : (int)n;
}

// Workgroups of all groups together, if there are not more groups.  Backwards each leaves a partial sum of 2 d floats, which are added up
// after: fewer than forwards, and fewer still for wide rows (147 MB of bf16 rows, us with 1 024 / 512 / 256: 64 features of 32 heads 97 / 96 / ., 1 024
// 99 / 86 / 97, 2 240 104 / 96 / 120, 8 192 129 / 107 / 97).
constexpr int kNormForwardWgs = 2048, kNormMostBackwardWgs = 512;
inline int norm_backward_wgs(int d) { return d < 4096 ? kNormMostBackwardWgs : 256; }

}  // namespace sv

// How rows of a layer norm are dealt to lanes and workgroups.  Plain C++ (no device code), shared by the launcher and host-side tests.
#pragma once

#include <stdint.h>

namespace sv {

// A row is held by `lanes` lanes, `vecs` 16-byte pieces each: lanes <= 64 lie in one wave (64 / lanes rows of a wave side by side),
// 256, 512 or 1024 are a whole workgroup.
struct NormForm {
    int lanes, vecs;
};

constexpr int kNormMostWidth = 8192;         // features of the widest row: 1 024 pieces of bf16, 2 048 of fp32

// The form for rows of `pieces` 16-byte pieces; lanes == 0: none.
inline NormForm norm_form(int pieces)
{
    if (pieces <= 0 || pieces > kNormMostWidth / 4) return NormForm{0, 0};
    for (int lanes = 4; lanes <= 64; lanes *= 2)
        if (pieces <= lanes) return NormForm{lanes, 1};
    if (pieces <= 64 * 6) return NormForm{64, (pieces + 63) / 64};
    return NormForm{pieces <= 512 ? 256 : pieces <= 1024 ? 512 : 1024, 2};
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

constexpr int kNormForwardWgs = 2048;        // all groups together, if there are not more groups
constexpr int kNormBackwardWgs = 1024;

}  // namespace sv

// What every entry point that takes token tensors checks of their descriptors before it launches anything.
#pragma once

#include <stdint.h>

#include <type_traits>

#include "../../include/sv_linattn.h"
#include "common.hpp"

namespace sv {

struct Shape {
    int B, H, N, d, BH;
    TokStrides st;
    bool bf16;
    int elem_bytes;
    bool host_epochs_only = false;   // the workspace is the library's own static array (see next_epoch)
};

inline bool head_dim_ok(int d) { return d == 32 || d == 64 || d == 112 || d == 128; }

// Calls f(std::integral_constant<int, D>) for the supported head dimension d.
template <typename F> void with_head_dim(int d, F &&f)
{
    switch (d) {
    case 32: f(std::integral_constant<int, 32>{}); break;
    case 64: f(std::integral_constant<int, 64>{}); break;
    case 112: f(std::integral_constant<int, 112>{}); break;
    default: f(std::integral_constant<int, 128>{}); break;
    }
}

// A launch's lanes are counted in 32 bits.
inline bool grid_ok(int64_t workgroups, int threads) { return workgroups < ((int64_t)1 << 32) / threads; }

inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// `any_width`: rows of any width (the caller checks it), not a head dimension of the attention kernels.  `most_heads`: bound of B*H, by
// default the grid's y limit.
inline sv_status check_desc(const sv_tensor_desc *t, Shape *s, bool any_width = false, int64_t most_heads = 65535)
{
    if (!t) return SV_ERR_NULL;
    if (t->dtype != SV_BF16 && t->dtype != SV_F32) return SV_ERR_UNSUPPORTED;
    if (!any_width && !head_dim_ok(t->d)) return SV_ERR_UNSUPPORTED;
    if (t->B <= 0 || t->H <= 0 || t->N <= 0) return SV_ERR_SHAPE;
    if ((int64_t)t->B * t->H > most_heads) return SV_ERR_SHAPE;
    if (t->stride_n < t->d || t->stride_b < 0 || t->stride_h < 0) return SV_ERR_SHAPE;
    if (t->B > 1 && t->stride_b == 0) return SV_ERR_SHAPE;
    if (t->H > 1 && t->stride_h == 0) return SV_ERR_SHAPE;
    s->B = t->B; s->H = t->H; s->N = t->N; s->d = t->d; s->BH = t->B * t->H;
    s->st = TokStrides{t->stride_b, t->stride_h, t->stride_n};
    s->bf16 = t->dtype == SV_BF16;
    s->elem_bytes = s->bf16 ? 2 : 4;
    const int64_t per16 = 16 / s->elem_bytes;
    if (t->stride_n % per16 || t->stride_b % per16 || t->stride_h % per16) return SV_ERR_ALIGN;
    // No two (b, h, n) rows may share memory (O rows would overwrite each other): taken in order of
    // ascending stride, every axis with more than one index must step over all that the axes below it span.
    struct Axis { int64_t stride, extent; } ax[3] = {{t->stride_b, t->B}, {t->stride_h, t->H}, {t->stride_n, t->N}};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 3; ++j)
            if (ax[j].stride < ax[i].stride) { const Axis x = ax[i]; ax[i] = ax[j]; ax[j] = x; }
    int64_t span = t->d;                             // elements covered by the axes handled so far
    for (const Axis &a : ax) {
        if (a.extent <= 1) continue;
        if (a.stride < span) return SV_ERR_SHAPE;
        if (a.stride > INT64_MAX / a.extent) return SV_ERR_SHAPE;
        span = a.stride * a.extent;
    }
    return SV_OK;
}

constexpr int64_t kMostHeads = 1 << 24;        // batches times heads of the operators that deal rows, not heads, to the grid
constexpr int kMostRowWidth = 8192;            // features of their widest row
constexpr int kMostTokens = INT32_MAX - 4096;  // of the operators that count a little past the last token

// A tensor of rows of any width that is whole 16-byte pieces.
inline sv_status check_rows(const sv_tensor_desc *t, Shape *s)
{
    const sv_status rc = check_desc(t, s, true, kMostHeads);
    if (rc != SV_OK) return rc;
    const int per = 16 / s->elem_bytes;
    if (s->d <= 0 || s->d % per || s->d > kMostRowWidth) return SV_ERR_UNSUPPORTED;
    return (int64_t)s->BH * s->N >= (int64_t)1 << 31 ? SV_ERR_SHAPE : SV_OK;
}
inline bool same_shape(const Shape &x, const Shape &y) { return x.B == y.B && x.H == y.H && x.N == y.N && x.d == y.d && x.bf16 == y.bf16; }
inline bool same_rows(const Shape &x, const Shape &y) { return x.st.b == y.st.b && x.st.h == y.st.h && x.st.n == y.st.n; }

// Is every row a run of whole 128-byte lines (given a tensor that begins with one)?
inline bool lines_whole(const Shape &s)
{
    const int64_t line = 128 / s.elem_bytes;
    return s.d % line == 0 && s.st.n % line == 0 && (s.H == 1 || s.st.h % line == 0) && (s.B == 1 || s.st.b % line == 0);
}

inline bool overlaps(const void *a, const void *b, size_t bytes)
{
    const auto pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    return a && b && pa < pb + bytes && pb < pa + bytes;
}
template <size_t N> bool all_aligned(const void *const (&p)[N])
{
    for (const void *x : p)
        if (!aligned16(x)) return false;
    return true;
}

inline sv_status launched() { return hipGetLastError() == hipSuccess ? SV_OK : SV_ERR_LAUNCH; }

}  // namespace sv

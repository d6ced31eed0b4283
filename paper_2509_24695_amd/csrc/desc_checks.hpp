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

}  // namespace sv

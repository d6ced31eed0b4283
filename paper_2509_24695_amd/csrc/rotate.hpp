// The three-axis rotation on its own: y = R x over the pairs of token rows.
//
// A copy with four multiplications per pair: bound by memory.  A thread owns 16 bytes of one token's rows (four pairs of bf16, two of fp32),
// works the token's place out and fetches its angles once, and then runs over the heads, first of q, then of k, whose rows all take the
// same angles.  Sixteen heads at a time (32 760 tokens of 20 heads of 112, views of one projection's output, 587 MB: 122 us, 4.8 TB/s; four at a
// time 132).  Heads that share no cache lines are written past the caches (with buffers that change from call to call 3 519 tokens of 3 x 16 heads of
// 128 in fp32 63.4 us, 5.2 TB/s, without the hint 65.9; 32 760 tokens of 32 heads of 64 104.3 and 106.6); heads that do, do without (133 with it).
#pragma once

#include "common.hpp"

namespace sv {

struct RotateArgs {
    const void *x[2];
    void *y[2];                    // q and k; tensors == 1: q alone
    TokStrides sx, sy;             // elements
    int B, H, N, tensors;
    int frames, rows, cols, n_t, n_h, n_w;
    const float *cs_t, *cs_h, *cs_w;
    const int32_t *positions;      // [B][N][3] or NULL
    float sign;                    // of the sines
    int head_group;                // heads that a workgroup runs over
    int own_lines;                 // heads of y share no cache lines: written past the caches
};

template <typename T, int D> struct RotateShape {
    static constexpr int kVec = 16 / (int)sizeof(T), kCols = D / kVec, kTokens = kThreads / kCols;
};

// Two features turned by one angle, in fp32, rounded once.
__device__ __forceinline__ u32x4 rotate16(u32x4 v, const f32x2 (&cs)[4], uint16_t)
{
#pragma unroll
    for (int p = 0; p < 4; ++p) v[p] = rope_rotate_pair(v[p], cs[p].x, cs[p].y);
    return v;
}
__device__ __forceinline__ u32x4 rotate16(u32x4 v, const f32x2 (&cs)[2], float)
{
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const float a = __uint_as_float(v[2 * p]), b = __uint_as_float(v[2 * p + 1]);
        v[2 * p] = __float_as_uint(a * cs[p].x - b * cs[p].y);
        v[2 * p + 1] = __float_as_uint(a * cs[p].y + b * cs[p].x);
    }
    return v;
}

template <typename T, int D> __global__ __launch_bounds__(kThreads) void rotate_rows(RotateArgs a)
{
    using W = RotateShape<T, D>;
    constexpr int kPairs = W::kVec / 2, kAhead = 16;              // heads whose rows are on their way together
    const int groups = (a.H + a.head_group - 1) / a.head_group, tiles = (a.N + W::kTokens - 1) / W::kTokens;
    const int h0 = (int)(blockIdx.x % groups) * a.head_group, h1 = h0 + a.head_group < a.H ? h0 + a.head_group : a.H;
    const int b = (int)(blockIdx.x / groups / tiles);
    const int64_t n = (int64_t)(blockIdx.x / groups % tiles) * W::kTokens + threadIdx.x / W::kCols;
    const int col = threadIdx.x % W::kCols;
    if (threadIdx.x >= W::kTokens * W::kCols || n >= a.N) return;
    int f, r, c;
    if (a.positions) {
        const int32_t *p = a.positions + ((int64_t)b * a.N + n) * 3;
        f = p[0], r = p[1], c = p[2];
        if (f < 0 || f >= a.frames || r < 0 || r >= a.rows || c < 0 || c >= a.cols) return;
    } else {
        const uint32_t t = (uint32_t)n, line = t / (uint32_t)a.cols;
        c = (int)(t - line * (uint32_t)a.cols);
        f = (int)(line / (uint32_t)a.rows);
        r = (int)(line - (uint32_t)f * (uint32_t)a.rows);
    }
    f32x2 cs[kPairs];
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
        const int p = col * kPairs + j, q = p - a.n_t, w = q - a.n_h;
        const float *at = q < 0 ? a.cs_t + ((int64_t)f * a.n_t + p) * 2 : w < 0 ? a.cs_h + ((int64_t)r * a.n_h + q) * 2 : a.cs_w + ((int64_t)c * a.n_w + w) * 2;
        cs[j] = *reinterpret_cast<const f32x2 *>(at);
        cs[j].y *= a.sign;
    }
    for (int which = 0; which < a.tensors; ++which) {
        const T *x = static_cast<const T *>(a.x[which]) + b * a.sx.b + n * a.sx.n + col * W::kVec;
        T *y = static_cast<T *>(a.y[which]) + b * a.sy.b + n * a.sy.n + col * W::kVec;
        for (int h = h0; h < h1; h += kAhead) {
            u32x4 v[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (h + i < h1) v[i] = *reinterpret_cast<const u32x4 *>(x + (h + i) * a.sx.h);
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (h + i < h1) store16(y + (h + i) * a.sy.h, rotate16(v[i], cs, T{}), a.own_lines);
        }
    }
}

}  // namespace sv

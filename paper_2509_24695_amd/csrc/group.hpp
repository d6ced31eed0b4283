// Group norm of channels-last rows with an activation, and its backward pass.  Over the N rows of a (b, h) and the d / G channels of a group:
//
//   mean = sum x / count,  rstd = 1 / sqrt(sum (x - mean)^2 / count + eps),  xh = (x - mean) rstd,  a = w xh + b,  y = a or silu(a)
//   da = dy or dy silu'(a),  t = w da,  dx = rstd (t - sum t / count - xh sum (t xh) / count),  dw = sum da xh,  db = sum da
//
// Bound by memory: two passes over the rows (the second finds what the cache behind the L2s still holds).  A thread keeps the same eight (fp32: four)
// channels for all of its rows, so groups need not be whole pieces: sums are kept by channel, and group_fold adds up a group's channels and chunks.
// Forwards the sums of x and x^2 are fp64, in which products of tensor values are exact: no cancellation shows for any mean that
// fp32 rows can have.
#pragma once

#include "activation.hpp"
#include "common.hpp"
#include "group_plan.hpp"
#include "piece.hpp"

namespace sv {

struct GroupArgs {
    const void *x, *dy;
    void *y;                               // backward: dx
    TokStrides sx, sdy, sy;
    const float *weight, *bias;            // [d] or NULL
    double *sums;                          // [BH][chunks][2][d]: of x and x^2 (backward fp32, of da and da xh)
    float *level, *scale;                  // [BH][G]: mean and rstd; backward: sum t / count and sum (t xh) / count
    float *mean, *rstd;                    // [BH][G]: outputs, or backward inputs
    float *dw, *db;
    int H, N, d, G, width;                 // width: channels of a group
    int64_t BH;
    int across, tiles, chunks;             // of this launch
    int64_t rows;
    int sum_chunks;                        // of the launch that wrote `sums`
    int whole_lines;
    float eps;
};

// A workgroup's tile and chunk, and its threads' channels and first row.
template <typename T> struct GroupPlace {
    int bh, chunk, tile, col, line, down, c;
    int64_t first, last;
    bool mine;
    __device__ __forceinline__ explicit GroupPlace(const GroupArgs &a)
    {
        uint32_t id = blockIdx.x;
        tile = (int)(id % (uint32_t)a.tiles);
        id /= (uint32_t)a.tiles;
        chunk = (int)(id % (uint32_t)a.chunks);
        bh = (int)(id / (uint32_t)a.chunks);
        col = (int)threadIdx.x % a.across;
        line = (int)threadIdx.x / a.across;
        down = kGroupThreads / a.across;
        c = (tile * a.across + col) * Piece<T>::kN;
        mine = c < a.d;
        first = (int64_t)chunk * a.rows;
        last = first + a.rows < a.N ? first + a.rows : a.N;
    }
    __device__ __forceinline__ const T *at(const GroupArgs &a, const void *p, const TokStrides &s) const
    {
        return static_cast<const T *>(p) + bh / a.H * s.b + bh % a.H * s.h + c;
    }
};

// What a thread's channels have of their groups.
template <int N> __device__ __forceinline__ void by_channel(const GroupArgs &a, const float *p, int bh, int c, float (&x)[N])
{
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = p[(int64_t)bh * a.G + (c + e) / a.width];
}
template <int N> __device__ __forceinline__ void of_channel(const float *p, int c, float otherwise, float (&x)[N])
{
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = p ? p[c + e] : otherwise;
}

// Walks a thread's rows, kGroupAhead at a time, the next ones on their way: f(row, pieces of x and (BOTH) dy).
template <typename T, bool BOTH, typename F> __device__ __forceinline__ void group_walk(const GroupArgs &a, const GroupPlace<T> &at, F &&f)
{
    const T *x = at.at(a, a.x, a.sx), *dy = BOTH ? at.at(a, a.dy, a.sdy) : nullptr;
    u32x4 nx[kGroupAhead] = {}, ndy[kGroupAhead] = {};
    auto request = [&](int64_t row) {
#pragma unroll
        for (int i = 0; i < kGroupAhead; ++i) {
            const int64_t r = row + i * at.down;
            if (r < at.last) {
                nx[i] = *reinterpret_cast<const u32x4 *>(x + r * a.sx.n);
                if (BOTH) ndy[i] = *reinterpret_cast<const u32x4 *>(dy + r * a.sdy.n);
            }
        }
    };
    request(at.first + at.line);
    for (int64_t row = at.first + at.line; row < at.last; row += kGroupAhead * at.down) {
        u32x4 vx[kGroupAhead], vdy[kGroupAhead];
#pragma unroll
        for (int i = 0; i < kGroupAhead; ++i) {
            vx[i] = nx[i];
            vdy[i] = ndy[i];
        }
        request(row + kGroupAhead * at.down);
#pragma unroll
        for (int i = 0; i < kGroupAhead; ++i)
            if (row + i * at.down < at.last) f(row + i * at.down, vx[i], vdy[i]);
    }
}

// Sums of a workgroup's lines, two numbers (of type S) a channel, into its place of `sums`.
template <typename T, typename S, int N> __device__ __forceinline__ void group_store_sums(const GroupArgs &a, const GroupPlace<T> &at, const S (&p)[N], const S (&q)[N])
{
    __shared__ S lines[kGroupThreads * N];
    S *out = reinterpret_cast<S *>(a.sums) + ((int64_t)at.bh * a.chunks + at.chunk) * 2 * a.d;
    const int width = a.across * N;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < N; ++e) lines[at.line * width + at.col * N + e] = which ? q[e] : p[e];
        __syncthreads();
        for (int k = threadIdx.x; k < width; k += kGroupThreads) {
            S s = lines[k];
            for (int r = 1; r < at.down; ++r) s += lines[r * width + k];
            const int c = at.tile * width + k;
            if (c < a.d) out[which * a.d + c] = s;
        }
    }
}

template <typename T> __global__ __launch_bounds__(kGroupThreads) void group_sums(GroupArgs a)
{
    constexpr int kN = Piece<T>::kN;
    const GroupPlace<T> at(a);
    double s[kN], q[kN];
#pragma unroll
    for (int e = 0; e < kN; ++e) s[e] = q[e] = 0.;
    if (at.mine)
        group_walk<T, false>(a, at, [&](int64_t, u32x4 vx, u32x4) {
            float x[kN];
            Piece<T>::open(vx, x);
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                const double v = x[e];
                s[e] += v;
                q[e] = __builtin_fma(v, v, q[e]);
            }
        });
    group_store_sums<T, double, kN>(a, at, s, q);
}

// A wave's sums.
__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int m = 1; m < 64; m *= 2) x += __shfl_xor(x, m, 64);
    return x;
}

// mean and rstd of each group: a wave adds up the chunks and channels of one.
__global__ __launch_bounds__(kGroupThreads) void group_fold(GroupArgs a)
{
    const int64_t id = (int64_t)blockIdx.x * (kGroupThreads / 64) + threadIdx.x / 64;
    if (id >= a.BH * a.G) return;
    const int64_t bh = id / a.G;
    const int group = (int)(id % a.G), lane = threadIdx.x % 64;
    const double *p = a.sums + bh * a.sum_chunks * 2 * a.d + group * a.width;
    double s = 0., q = 0.;
    const int count = a.sum_chunks * a.width;
#pragma unroll 4
    for (int k = lane; k < count; k += 64) {
        const double *at = p + (int64_t)(k / a.width) * 2 * a.d + k % a.width;
        s += at[0];
        q += at[a.d];
    }
    s = wave_sum(s);
    q = wave_sum(q);
    if (lane) return;
    const double over = 1. / ((double)a.N * a.width), mean = s * over, var = __builtin_fma(-mean, mean, q * over);
    const float m = (float)mean, r = (float)(1. / __builtin_sqrt((var > 0. || var != var ? var : 0.) + a.eps));
    a.level[id] = m;
    a.scale[id] = r;
    if (a.mean) {
        a.mean[id] = m;
        a.rstd[id] = r;
    }
}

template <typename T, bool SILU> __global__ __launch_bounds__(kGroupThreads) void group_apply(GroupArgs a)
{
    constexpr int kN = Piece<T>::kN;
    const GroupPlace<T> at(a);
    if (!at.mine) return;
    float mean[kN], rstd[kN], w[kN], b[kN];
    by_channel<kN>(a, a.level, at.bh, at.c, mean);
    by_channel<kN>(a, a.scale, at.bh, at.c, rstd);
    of_channel<kN>(a.weight, at.c, 1.f, w);
    of_channel<kN>(a.bias, at.c, 0.f, b);
    T *y = const_cast<T *>(at.at(a, a.y, a.sy));
    group_walk<T, false>(a, at, [&](int64_t row, u32x4 vx, u32x4) {
        float x[kN];
        Piece<T>::open(vx, x);
#pragma unroll
        for (int e = 0; e < kN; ++e) {
            x[e] = __builtin_fmaf((x[e] - mean[e]) * rstd[e], w[e], b[e]);
            if (SILU) x[e] = silu(x[e]);
        }
        store16(y + row * a.sy.n, Piece<T>::close(x), a.whole_lines);
    });
}

// xh and da of a thread's channels of one row.
template <typename T, bool SILU, int N>
__device__ __forceinline__ void group_terms(u32x4 vx, u32x4 vdy, const float (&mean)[N], const float (&rstd)[N], const float (&w)[N], const float (&b)[N], float (&xh)[N],
                                            float (&da)[N])
{
    Piece<T>::open(vx, xh);
    Piece<T>::open(vdy, da);
#pragma unroll
    for (int e = 0; e < N; ++e) {
        xh[e] = (xh[e] - mean[e]) * rstd[e];
        if (SILU) {
            const float y = __builtin_fmaf(xh[e], w[e], b[e]);
            da[e] *= silu_slope(y, sigmoid(y));
        }
    }
}

// Sums of da and da xh by channel.
template <typename T, bool SILU> __global__ __launch_bounds__(kGroupThreads) void group_back_sums(GroupArgs a)
{
    constexpr int kN = Piece<T>::kN;
    const GroupPlace<T> at(a);
    float p[kN], q[kN];
#pragma unroll
    for (int e = 0; e < kN; ++e) p[e] = q[e] = 0.f;
    if (at.mine) {
        float mean[kN], rstd[kN], w[kN], b[kN];
        by_channel<kN>(a, a.mean, at.bh, at.c, mean);
        by_channel<kN>(a, a.rstd, at.bh, at.c, rstd);
        of_channel<kN>(a.weight, at.c, 1.f, w);
        of_channel<kN>(a.bias, at.c, 0.f, b);
        group_walk<T, true>(a, at, [&](int64_t, u32x4 vx, u32x4 vdy) {
            float xh[kN], da[kN];
            group_terms<T, SILU, kN>(vx, vdy, mean, rstd, w, b, xh, da);
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                p[e] += da[e];
                q[e] = __builtin_fmaf(da[e], xh[e], q[e]);
            }
        });
    }
    group_store_sums<T, float, kN>(a, at, p, q);
}

// Of each group sum t / count and sum (t xh) / count (a wave each, in fp64); behind these db and dw of each channel.
__global__ __launch_bounds__(kGroupThreads) void group_back_fold(GroupArgs a)
{
    const float *sums = reinterpret_cast<const float *>(a.sums);
    const int64_t waves = a.BH * a.G, blocks = (waves + kGroupThreads / 64 - 1) / (kGroupThreads / 64);
    if ((int64_t)blockIdx.x < blocks) {
        const int64_t id = (int64_t)blockIdx.x * (kGroupThreads / 64) + threadIdx.x / 64;
        if (id >= waves) return;
        const int64_t bh = id / a.G;
        const int group = (int)(id % a.G), lane = threadIdx.x % 64, count = a.sum_chunks * a.width;
        double s = 0., q = 0.;
#pragma unroll 4
        for (int k = lane; k < count; k += 64) {
            const int c = group * a.width + k % a.width;
            const float *at = sums + (bh * a.sum_chunks + k / a.width) * 2 * a.d + c;
            const double w = a.weight ? a.weight[c] : 1.f;
            s = __builtin_fma(w, (double)at[0], s);
            q = __builtin_fma(w, (double)at[a.d], q);
        }
        s = wave_sum(s);
        q = wave_sum(q);
        const double over = 1. / ((double)a.N * a.width);
        if (lane == 0) {
            a.level[id] = (float)(s * over);
            a.scale[id] = (float)(q * over);
        }
        return;
    }
    // sixteen channels of either sum, sixteen runs of the chunks each, added up in order
    __shared__ float runs[16][16];
    const int64_t k = ((int64_t)blockIdx.x - blocks) * 16 + threadIdx.x % 16, parts = a.BH * a.sum_chunks;
    const int run = threadIdx.x / 16;
    float s = 0.f;
    if (k < 2 * a.d)
#pragma unroll 4
        for (int64_t i = run; i < parts; i += 16) s += sums[i * 2 * a.d + k];
    runs[run][threadIdx.x % 16] = s;
    __syncthreads();
    if (run || k >= 2 * a.d) return;
#pragma unroll
    for (int r = 1; r < 16; ++r) s += runs[r][threadIdx.x];
    float *out = k < a.d ? a.db : a.dw;
    if (out) out[k < a.d ? k : k - a.d] = s;
}

template <typename T, bool SILU> __global__ __launch_bounds__(kGroupThreads) void group_back_apply(GroupArgs a)
{
    constexpr int kN = Piece<T>::kN;
    const GroupPlace<T> at(a);
    if (!at.mine) return;
    float mean[kN], rstd[kN], w[kN], b[kN], level[kN], along[kN];
    by_channel<kN>(a, a.mean, at.bh, at.c, mean);
    by_channel<kN>(a, a.rstd, at.bh, at.c, rstd);
    by_channel<kN>(a, a.level, at.bh, at.c, level);
    by_channel<kN>(a, a.scale, at.bh, at.c, along);
    of_channel<kN>(a.weight, at.c, 1.f, w);
    of_channel<kN>(a.bias, at.c, 0.f, b);
    T *dx = const_cast<T *>(at.at(a, a.y, a.sy));
    group_walk<T, true>(a, at, [&](int64_t row, u32x4 vx, u32x4 vdy) {
        float xh[kN], da[kN];
        group_terms<T, SILU, kN>(vx, vdy, mean, rstd, w, b, xh, da);
#pragma unroll
        for (int e = 0; e < kN; ++e) da[e] = rstd[e] * (w[e] * da[e] - level[e] - xh[e] * along[e]);
        store16(dx + row * a.sy.n, Piece<T>::close(da), a.whole_lines);
    });
}

}  // namespace sv

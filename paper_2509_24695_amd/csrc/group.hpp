// Group norm of channels-last rows with an activation, and its backward pass.  Over the N rows of a (b, h) and the d / G channels of a group:
//
//   mean = sum x / count,  rstd = 1 / sqrt(sum (x - mean)^2 / count + eps),  xh = (x - mean) rstd,  a = w xh + b,  y = a or silu(a)
//   da = dy or dy silu'(a),  t = w da,  dx = rstd (t - sum t / count - xh sum (t xh) / count),  dw = sum da xh,  db = sum da
//
// Bound by memory, twice over: a pass for the sums and one for the rows (a copy is as slow out of the cache behind the L2s as out of memory).  21 frames of
// 1 560 rows of 2 240 channels in 32 groups bf16 86 us, 32 for the sums (4.6 TB/s) and 54 for the rows (5.4 TB/s; a reading and a copying pass 80); backwards 14 040 rows
// 62 us, 26 for the sums (4.8 TB/s), 5 for the fold and 32 (5.9 TB/s).  A thread keeps the same eight (fp32: four)
// channels for all of its rows, so groups need not be whole pieces: sums are kept by channel, and group_fold adds up a group's channels and chunks.
// Forwards the sums are of x - x0 and its square in fp64, x0 the group's first number.  As one of the group's `count` numbers x0 is at most sqrt(count)
// deviations from the mean, so the variance loses at most count fp64 roundings to cancellation however far from zero the rows lie (without x0, rows
// of 1e6 with a deviation of 0.1 had an rstd that was 0.6 % off).
#pragma once

#include "activation.hpp"
#include "common.hpp"
#include "group_plan.hpp"
#include "norm_plan.hpp"
#include "piece.hpp"

namespace sv {

struct GroupArgs {
    const void *x, *dy;
    void *y;                               // backward: dx
    TokStrides sx, sdy, sy;
    const float *weight, *bias;            // [d] or NULL
    double *sums;                          // [BH][chunks][2][d]: of x - x0 and its square (backward fp32, of da and da xh)
    double *pairs;                         // [BH][chunks][tiles][per_tile][2]: the same by group (backward of t and t xh); NULL: groups are narrow
    int per_tile, sum_tiles, tile_width;   // groups and channels of a tile of the launch that writes them
    float *level, *scale;                  // [BH][G]: x0, then mean, and rstd; backward: sum t / count and sum (t xh) / count
    float *mean, *rstd;                    // [BH][G]: outputs, or backward inputs
    float *dw, *db;
    int H, N, d, G, width;                 // width: channels of a group
    int64_t BH;
    int across, tiles, chunks, lines;      // of this launch
    int64_t folds;                         // workgroups of group_back_fold for groups
    int64_t rows;
    int sum_chunks;                        // of the launch that wrote `sums`
    int whole_lines;
    NormDivisor width_div;
    float eps;
};

template <typename T> using GroupSums = Piece<T>;
template <typename T> using GroupApply = Piece<T>;
template <typename T> using GroupBack = Quad<T>;

// A workgroup's tile and chunk, and its threads' channels and first row.
template <typename T, typename P> struct GroupPlace {
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
        c = (tile * a.across + col) * P::kN;
        mine = c < a.d && line < down;
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

// Walks a thread's rows, kAhead at a time, the next ones on their way: f(row, pieces of x and (BOTH) dy).  Two of both, which leave room for more waves (backwards, 14 040
// rows of 2 240 channels 68.1 us on buffers in turn; four 71, one 72; 21 frames of 1 560 rows 134, 136 and 160).
template <typename T, typename P, bool BOTH, typename F> __device__ __forceinline__ void group_walk(const GroupArgs &a, const GroupPlace<T, P> &at, F &&f)
{
    typedef typename P::V V;
    constexpr int kAhead = BOTH ? kGroupAhead / 2 : kGroupAhead;
    const T *x = at.at(a, a.x, a.sx), *dy = BOTH ? at.at(a, a.dy, a.sdy) : nullptr;
    V nx[kAhead], ndy[kAhead];
    // past the last row the last one is read again: no branch stands between the loads
    auto request = [&](int64_t row) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t r = row + i * at.down < at.last ? row + i * at.down : at.last - 1;
            nx[i] = *reinterpret_cast<const V *>(x + r * a.sx.n);
            if (BOTH) ndy[i] = *reinterpret_cast<const V *>(dy + r * a.sdy.n);
        }
    };
    request(at.first + at.line);
    int64_t row = at.first + at.line;
    for (; row + (kAhead - 1) * at.down < at.last; row += kAhead * at.down) {
        V vx[kAhead], vdy[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            vx[i] = nx[i];
            if (BOTH) vdy[i] = ndy[i];
        }
        request(row + kAhead * at.down);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) f(row + i * at.down, vx[i], vdy[i]);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (row + i * at.down < at.last) f(row + i * at.down, nx[i], ndy[i]);
}

// Sums over a workgroup's lines of two numbers (of type S) a channel: into its place of `sums`, and (PAIRS) by group into its place of `pairs`, there
// times the channel's weight if `weigh`.
template <bool SUMS, bool PAIRS, typename T, typename P, typename S, int N>
__device__ __forceinline__ void group_store_sums(const GroupArgs &a, const GroupPlace<T, P> &at, const S (&p)[N], const S (&q)[N], bool weigh)
{
    __shared__ S lines[kGroupThreads * N];
    __shared__ double channels[2][32 * N];
    const int64_t part = (int64_t)at.bh * a.chunks + at.chunk;
    S *out = reinterpret_cast<S *>(a.sums) + part * 2 * a.d;
    const int width = a.across * N, c0 = at.tile * width;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (at.line < at.down) lines[at.line * width + at.col * N + e] = which ? q[e] : p[e];
        __syncthreads();
        for (int k = threadIdx.x; k < width; k += kGroupThreads) {
            S s = lines[k];
            for (int r = 1; r < at.down; ++r) s += lines[r * width + k];
            const int c = c0 + k;
            if (SUMS && c < a.d) out[which * a.d + c] = s;
            if (PAIRS) channels[which][k] = c < a.d ? (weigh ? (double)a.weight[c] : 1.) * (double)s : 0.;
        }
    }
    if constexpr (PAIRS) {
        __syncthreads();
        const int lane = threadIdx.x % 64, first = c0 / a.width, end = c0 + width < a.d ? c0 + width : a.d;
        for (int g = first + (int)threadIdx.x / 64; g * a.width < end; g += kGroupThreads / 64) {
            const int from = g * a.width > c0 ? g * a.width - c0 : 0, to = (g + 1) * a.width < end ? (g + 1) * a.width - c0 : end - c0;
            double s = 0., t = 0.;
            for (int k = from + lane; k < to; k += 64) {
                s += channels[0][k];
                t += channels[1][k];
            }
#pragma unroll
            for (int m = 1; m < 64; m *= 2) {
                s += __shfl_xor(s, m, 64);
                t += __shfl_xor(t, m, 64);
            }
            double *pair = a.pairs + ((part * a.tiles + at.tile) * a.per_tile + g - first) * 2;
            if (lane == 0) {
                pair[0] = s;
                pair[1] = t;
            }
        }
    }
}

template <typename T, bool WIDE> __global__ __launch_bounds__(kGroupThreads) void group_sums(GroupArgs a)
{
    using P = GroupSums<T>;
    typedef typename P::V V;
    constexpr int kN = P::kN;
    const GroupPlace<T, P> at(a);
    double s[kN], q[kN];
#pragma unroll
    for (int e = 0; e < kN; ++e) s[e] = q[e] = 0.;
    if (at.mine) {
        float from[kN];
        const T *row = at.at(a, a.x, a.sx) - at.c;
#pragma unroll
        for (int e = 0; e < kN; ++e) {
            const float first = Elem<T>::load(row + a.width_div.quotient(at.c + e) * a.width);
            from[e] = __builtin_isfinite(first) ? first : 0.f;        // (an infinity's mean is that infinity)
        }
        group_walk<T, P, false>(a, at, [&](int64_t, V vx, V) {
            float x[kN];
            P::open(vx, x);
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                const double v = (double)x[e] - from[e];
                s[e] += v;
                q[e] = __builtin_fma(v, v, q[e]);
            }
        });
        // x0 for the next launch, which may write into the rows
        if (at.chunk == 0 && at.line == 0)
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                const int g = (int)a.width_div.quotient(at.c + e);
                if (at.c + e == g * a.width) a.level[(int64_t)at.bh * a.G + g] = from[e];
            }
    }
    group_store_sums<!WIDE, WIDE>(a, at, s, q, false);
}

// A workgroup's sums of one number or two, for all of its threads (`lds`: as many for each wave).
template <int THREADS, typename... Q> __device__ __forceinline__ void group_total(double *lds, Q &...q)
{
    constexpr int kNumbers = sizeof...(q);
#pragma unroll
    for (int m = 1; m < 64; m *= 2) ((q += __shfl_xor(q, m, 64)), ...);
    __syncthreads();
    double *own = lds + threadIdx.x / 64 * kNumbers;
    if (threadIdx.x % 64 == 0) ((*own++ = q), ...);
    __syncthreads();
    const double *at = lds;
    ((q = *at++), ...);
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) ((q += *at++), ...);
}

// A group's two sums over its chunks and channels: f(channel, address of the first sum).
template <typename S, typename F> __device__ __forceinline__ void group_gather(const GroupArgs &a, int64_t bh, int group, F &&f)
{
    const uint32_t count = (uint32_t)a.sum_chunks * a.width;
    const S *p = reinterpret_cast<const S *>(a.sums) + bh * a.sum_chunks * 2 * a.d;
    constexpr int kAt = 8;
    for (uint32_t k0 = threadIdx.x; k0 < count; k0 += kAt * kGroupThreads) {
        S s[kAt], q[kAt];
        int c[kAt];
#pragma unroll
        for (int i = 0; i < kAt; ++i) {
            const uint32_t k = k0 + i * kGroupThreads < count ? k0 + i * kGroupThreads : k0, chunk = a.width_div.quotient(k);
            c[i] = group * a.width + (int)(k - chunk * a.width);
            const S *at = p + (int64_t)chunk * 2 * a.d + c[i];
            s[i] = at[0];
            q[i] = at[a.d];
        }
#pragma unroll
        for (int i = 0; i < kAt; ++i)
            if (k0 + i * kGroupThreads < count) f(c[i], s[i], q[i]);
    }
}

// A group's two sums out of the pairs of its chunks and tiles.
__device__ __forceinline__ void group_gather_pairs(const GroupArgs &a, int64_t bh, int group, int first, int threads, double &s, double &q)
{
    const int t0 = group * a.width / a.tile_width, t1 = ((group + 1) * a.width - 1) / a.tile_width, n = t1 - t0 + 1, count = a.sum_chunks * n;
    const double *p = a.pairs + bh * a.sum_chunks * a.sum_tiles * a.per_tile * 2;
#pragma unroll 4
    for (int k = first; k < count; k += threads) {
        const int chunk = k / n, t = t0 + k - chunk * n;
        const double *pair = p + (((int64_t)chunk * a.sum_tiles + t) * a.per_tile + group - t * a.tile_width / a.width) * 2;
        s += pair[0];
        q += pair[1];
    }
}

// rstd from a group's sum of squares of deviations
__device__ __forceinline__ float group_scale(double squares, double over, float eps)
{
    const double var = squares * over;
    return (float)(1. / __builtin_sqrt((var > 0. || var != var ? var : 0.) + eps));
}

// mean and rstd of each group: a workgroup adds up the chunks and channels of one.
__global__ __launch_bounds__(kGroupThreads) void group_fold(GroupArgs a)
{
    __shared__ double lds[2 * kGroupThreads / 64];
    const int64_t id = blockIdx.x, bh = id / a.G;
    double s = 0., q = 0.;
    if (a.pairs) group_gather_pairs(a, bh, (int)(id - bh * a.G), threadIdx.x, kGroupThreads, s, q);
    else
        group_gather<double>(a, bh, (int)(id - bh * a.G), [&](int, double x, double xx) {
            s += x;
            q += xx;
        });
    group_total<kGroupThreads>(lds, s, q);
    if (threadIdx.x) return;
    const double over = 1. / ((double)a.N * a.width), past = s * over;
    const float m = (float)(a.level[id] + past), r = group_scale(__builtin_fma(-past, s, q), over, a.eps);
    a.level[id] = m;
    a.scale[id] = r;
    if (a.mean) {
        a.mean[id] = m;
        a.rstd[id] = r;
    }
}

// FOLD: a workgroup adds up the pairs of its tile's groups by itself, a wave a group (a launch less: 21 frames of 1 560 rows of 2 240 channels 90 -> 84 us).
template <typename T, bool SILU, bool FOLD> __global__ __launch_bounds__(kGroupThreads) void group_apply(GroupArgs a)
{
    using P = GroupApply<T>;
    typedef typename P::V V;
    constexpr int kN = P::kN;
    const GroupPlace<T, P> at(a);
    float mean[kN], rstd[kN], w[kN], b[kN];
    if constexpr (FOLD) {
        __shared__ float stats[2][32 * kN / kWideGroup + 2];
        const int width = a.across * kN, c0 = at.tile * width, first = c0 / a.width, end = c0 + width < a.d ? c0 + width : a.d, lane = threadIdx.x % 64;
        for (int g = first + (int)threadIdx.x / 64; g * a.width < end; g += kGroupThreads / 64) {
            double s = 0., q = 0.;
            group_gather_pairs(a, at.bh, g, lane, 64, s, q);
#pragma unroll
            for (int m = 1; m < 64; m *= 2) {
                s += __shfl_xor(s, m, 64);
                q += __shfl_xor(q, m, 64);
            }
            const double over = 1. / ((double)a.N * a.width), past = s * over;
            const float m = (float)(a.level[(int64_t)at.bh * a.G + g] + past), r = group_scale(__builtin_fma(-past, s, q), over, a.eps);
            if (lane == 0) {
                stats[0][g - first] = m;
                stats[1][g - first] = r;
                if (a.mean && at.chunk == 0 && g * a.width >= c0) {
                    a.mean[(int64_t)at.bh * a.G + g] = m;
                    a.rstd[(int64_t)at.bh * a.G + g] = r;
                }
            }
        }
        __syncthreads();
        if (!at.mine) return;
#pragma unroll
        for (int e = 0; e < kN; ++e) {
            const int g = (at.c + e) / a.width - first;
            mean[e] = stats[0][g];
            rstd[e] = stats[1][g];
        }
    } else {
        if (!at.mine) return;
        by_channel<kN>(a, a.level, at.bh, at.c, mean);
        by_channel<kN>(a, a.scale, at.bh, at.c, rstd);
    }
    of_channel<kN>(a.weight, at.c, 1.f, w);
    of_channel<kN>(a.bias, at.c, 0.f, b);
    T *y = const_cast<T *>(at.at(a, a.y, a.sy));
    group_walk<T, P, false>(a, at, [&](int64_t row, V vx, V) {
        float x[kN];
        P::open(vx, x);
#pragma unroll
        for (int e = 0; e < kN; ++e) {
            x[e] = __builtin_fmaf((x[e] - mean[e]) * rstd[e], w[e], b[e]);
            if (SILU) x[e] = silu(x[e]);
        }
        store16(y + row * a.sy.n, P::close(x), a.whole_lines);
    });
}

// xh and da of a thread's channels of one row.
template <typename P, bool SILU, int N>
__device__ __forceinline__ void group_terms(typename P::V vx, typename P::V vdy, const float (&mean)[N], const float (&rstd)[N], const float (&w)[N], const float (&b)[N], float (&xh)[N],
                                            float (&da)[N])
{
    P::open(vx, xh);
    P::open(vdy, da);
#pragma unroll
    for (int e = 0; e < N; ++e) {
        xh[e] = (xh[e] - mean[e]) * rstd[e];
        if (SILU) {
            const float y = __builtin_fmaf(xh[e], w[e], b[e]);
            da[e] *= silu_slope(y, sigmoid(y));
        }
    }
}

// Sums of da and da xh, by channel (SUMS) and, for wide groups, by group.
template <typename T, bool SILU, bool SUMS, bool WIDE> __global__ __launch_bounds__(kGroupThreads) void group_back_sums(GroupArgs a)
{
    using P = GroupBack<T>;
    typedef typename P::V V;
    constexpr int kN = P::kN;
    const GroupPlace<T, P> at(a);
    float p[kN], q[kN];
#pragma unroll
    for (int e = 0; e < kN; ++e) p[e] = q[e] = 0.f;
    if (at.mine) {
        float mean[kN], rstd[kN], w[kN], b[kN];
        by_channel<kN>(a, a.mean, at.bh, at.c, mean);
        by_channel<kN>(a, a.rstd, at.bh, at.c, rstd);
        of_channel<kN>(a.weight, at.c, 1.f, w);
        of_channel<kN>(a.bias, at.c, 0.f, b);
        group_walk<T, P, true>(a, at, [&](int64_t, V vx, V vdy) {
            float xh[kN], da[kN];
            group_terms<P, SILU, kN>(vx, vdy, mean, rstd, w, b, xh, da);
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                p[e] += da[e];
                q[e] = __builtin_fmaf(da[e], xh[e], q[e]);
            }
        });
    }
    group_store_sums<SUMS, WIDE>(a, at, p, q, a.weight != nullptr);
}

// Of each group sum t / count and sum (t xh) / count (a workgroup each, in fp64); behind these db and dw of each channel.
__global__ __launch_bounds__(kGroupThreads) void group_back_fold(GroupArgs a)
{
    const float *sums = reinterpret_cast<const float *>(a.sums);
    const int64_t blocks = a.folds;
    if ((int64_t)blockIdx.x < blocks) {
        __shared__ double lds[2 * kGroupThreads / 64];
        const int64_t id = blockIdx.x, bh = id / a.G;
        double s = 0., q = 0.;
        if (a.pairs) group_gather_pairs(a, bh, (int)(id - bh * a.G), threadIdx.x, kGroupThreads, s, q);
        else
            group_gather<float>(a, bh, (int)(id - bh * a.G), [&](int c, float p, float px) {
                const double w = a.weight ? a.weight[c] : 1.f;
                s = __builtin_fma(w, (double)p, s);
                q = __builtin_fma(w, (double)px, q);
            });
        group_total<kGroupThreads>(lds, s, q);
        const double over = 1. / ((double)a.N * a.width);
        if (threadIdx.x == 0) {
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
    using P = GroupBack<T>;
    typedef typename P::V V;
    constexpr int kN = P::kN;
    const GroupPlace<T, P> at(a);
    if (!at.mine) return;
    float mean[kN], rstd[kN], w[kN], b[kN], level[kN], along[kN];
    by_channel<kN>(a, a.mean, at.bh, at.c, mean);
    by_channel<kN>(a, a.rstd, at.bh, at.c, rstd);
    by_channel<kN>(a, a.level, at.bh, at.c, level);
    by_channel<kN>(a, a.scale, at.bh, at.c, along);
    of_channel<kN>(a.weight, at.c, 1.f, w);
    of_channel<kN>(a.bias, at.c, 0.f, b);
    T *dx = const_cast<T *>(at.at(a, a.y, a.sy));
    group_walk<T, P, true>(a, at, [&](int64_t row, V vx, V vdy) {
        float xh[kN], da[kN];
        group_terms<P, SILU, kN>(vx, vdy, mean, rstd, w, b, xh, da);
#pragma unroll
        for (int e = 0; e < kN; ++e) da[e] = rstd[e] * (w[e] * da[e] - level[e] - xh[e] * along[e]);
        store16(dx + row * a.sy.n, P::close(da), a.whole_lines);
    });
}

}  // namespace sv

// Group norm of groups that one workgroup holds in registers: read once, one launch (a second one backwards, for the
// parameters' gradients).  A thread has the same channels in all of its rows.  Three batches of 901 rows of 320 channels in 32 groups fp32: 8.7 us, in three launches
// 12.6; 84 frames of 64 rows of 320 channels 30.  Bound by its own run through a launch: loads, two joins of 1 024 threads, stores.  Groups of twice the size (64 words a thread) lose: 21 frames of
// 1 560 x 2 240 took 100 us, as nothing overlaps the arithmetic of the one workgroup on a compute unit.
#pragma once

#include "group.hpp"

namespace sv {

// A thread's unit of a row as words, and its numbers.
template <typename T, int UNIT> struct Unit;
template <> struct Unit<uint16_t, 16> : Piece<uint16_t> {};
template <> struct Unit<float, 16> : Piece<float> {};
template <> struct Unit<float, 4> {
    typedef uint32_t V;
    static constexpr int kN = 1;
    static __device__ __forceinline__ void open(uint32_t v, float (&x)[1]) { x[0] = __uint_as_float(v); }
    static __device__ __forceinline__ uint32_t close(const float (&x)[1]) { return __float_as_uint(x[0]); }
};
template <> struct Unit<uint16_t, 4> {
    typedef uint32_t V;
    static constexpr int kN = 2;
    static __device__ __forceinline__ void open(uint32_t v, float (&x)[2])
    {
        x[0] = bf16_lo(v);
        x[1] = bf16_hi(v);
    }
    static __device__ __forceinline__ uint32_t close(const float (&x)[2]) { return pack_bf16x2(x[0], x[1]); }
};
template <> struct Unit<uint16_t, 2> {
    typedef uint16_t V;
    static constexpr int kN = 1;
    static __device__ __forceinline__ void open(uint16_t v, float (&x)[1]) { x[0] = bf16_bits_to_f32(v); }
    static __device__ __forceinline__ uint16_t close(const float (&x)[1]) { return f32_to_bf16_bits(x[0]); }
};

// The group of a workgroup (neighbouring groups, whose rows share lines, on one die) and a thread's channels and first row.
template <typename T, typename P> struct HeldPlace {
    int64_t id, bh;
    int group, line, c;
    bool mine;
    int all, rows;                         // of all lines, and of the thread: one more or not
    __device__ __forceinline__ HeldPlace(const GroupArgs &a)
        : id(held_task(blockIdx.x, gridDim.x)), bh(id / a.G), group((int)(id - bh * a.G)), line((int)threadIdx.x / a.across),
          c(group * a.width + ((int)threadIdx.x - line * a.across) * P::kN), mine(line < a.lines && line < a.N)
    {
        all = a.N / a.lines;
        rows = mine ? all + (line < a.N - all * a.lines) : 0;
        line = mine ? line : 0;
        c = mine ? c : group * a.width;
    }
    __device__ __forceinline__ const T *at(const GroupArgs &a, const void *p, const TokStrides &s) const
    {
        return static_cast<const T *>(p) + bh / a.H * s.b + bh % a.H * s.h + c;
    }
};
// A thread's units.  All lines have `all` rows; one more, which only the first lines have, is the thread's first again where there is none.
template <typename T, typename V, int ROWS> __device__ __forceinline__ void held_load(const T *p, int64_t stride, int lines, int line, int all, int count, V (&v)[ROWS])
{
    const T *first = p + line * stride, *at = first;
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
        if (i <= all) {
            v[i] = *reinterpret_cast<const V *>(i < count ? at : first);
            at += lines * stride;
        }
}
// The words as they were loaded: what was made of them in one pass over them is made again in the next, and takes no registers in between.
template <typename V, int ROWS> __device__ __forceinline__ void held_again(V (&v)[ROWS])
{
#pragma unroll
    for (int i = 0; i < ROWS; ++i) asm volatile("" : "+v"(v[i]));
}
// The same for a row of a pass that ends before the next.  (Without it the compiler gathers all rows' numbers into one long vector, which spills.)
template <typename P, int N> __device__ __forceinline__ void held_open(typename P::V v, float (&x)[N])
{
    asm volatile("" : "+v"(v));
    P::open(v, x);
}
template <typename V> __device__ __forceinline__ void held_store(void *p, V v, bool past_caches)
{
    if constexpr (sizeof(V) == 16) store16(p, v, past_caches);
    else *static_cast<V *>(p) = v;
}

template <typename T, int UNIT, int ROWS, bool SILU> __global__ __launch_bounds__(kHeldThreads) void group_held(GroupArgs a)
{
    using P = Unit<T, UNIT>;
    constexpr int kN = P::kN;
    __shared__ double lds[2 * kHeldThreads / 64];
    const HeldPlace<T, P> at(a);
    if (at.bh >= a.BH) return;
    typename P::V v[ROWS];
    held_load(at.at(a, a.x, a.sx), a.sx.n, a.lines, at.line, at.all, at.rows, v);
    float w[kN], b[kN];
    of_channel<kN>(a.weight, at.c, 1.f, w);
    of_channel<kN>(a.bias, at.c, 0.f, b);
    // Every number is added up in fp64, and so is the square of what is left of the fp64 mean: neither overflows for any fp32 rows, and constant groups
    // have a variance of zero.
    double s = 0., q = 0.;
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
        if (i < at.rows) {
            float x[kN];
            held_open<P>(v[i], x);
#pragma unroll
            for (int e = 0; e < kN; ++e) s += x[e];
        }
    group_total<kHeldThreads>(lds, s);
    const double over = 1. / ((double)a.N * a.width), exact = s * over;
    const float mean = (float)exact;
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
        if (i < at.rows) {
            float x[kN];
            held_open<P>(v[i], x);
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                const double left = x[e] - exact;
                q = __builtin_fma(left, left, q);
            }
        }
    group_total<kHeldThreads>(lds, q);
    const float rstd = group_scale(q, over, a.eps);
    if (a.mean && threadIdx.x == 0) {
        a.mean[at.id] = mean;
        a.rstd[at.id] = rstd;
    }
    if (!at.mine) return;
    T *y = const_cast<T *>(at.at(a, a.y, a.sy)) + at.line * a.sy.n;
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
        if (i <= at.all) {
            float x[kN];
            held_open<P>(v[i], x);
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                x[e] = __builtin_fmaf((x[e] - mean) * rstd, w[e], b[e]);
                if (SILU) x[e] = silu(x[e]);
            }
            if (i < at.rows) held_store(y, P::close(x), a.whole_lines);
            y += a.lines * a.sy.n;
        }
}

// PARAMS: the channels' sums of da and da xh over the (b, h) as well, [BH][2][d] in `sums`.
template <typename T, int UNIT, int ROWS, bool SILU, bool PARAMS> __global__ __launch_bounds__(kHeldThreads) void group_held_back(GroupArgs a)
{
    using P = Unit<T, UNIT>;
    constexpr int kN = P::kN;
    __shared__ double lds[2 * kHeldThreads / 64];
    const HeldPlace<T, P> at(a);
    if (at.bh >= a.BH) return;
    typename P::V vx[ROWS], vdy[ROWS];
    held_load(at.at(a, a.x, a.sx), a.sx.n, a.lines, at.line, at.all, at.rows, vx);
    held_load(at.at(a, a.dy, a.sdy), a.sdy.n, a.lines, at.line, at.all, at.rows, vdy);
    const float m = a.mean[at.id], r = a.rstd[at.id];
    float w[kN], b[kN], mean[kN], rstd[kN], p[kN], px[kN];
    of_channel<kN>(a.weight, at.c, 1.f, w);
    of_channel<kN>(a.bias, at.c, 0.f, b);
#pragma unroll
    for (int e = 0; e < kN; ++e) {
        mean[e] = m;
        rstd[e] = r;
        p[e] = px[e] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
        if (i < at.rows) {
            float xh[kN], da[kN];
            group_terms<P, SILU, kN>(vx[i], vdy[i], mean, rstd, w, b, xh, da);
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                p[e] += da[e];
                px[e] = __builtin_fmaf(da[e], xh[e], px[e]);
            }
        }
    double s = 0., q = 0.;
#pragma unroll
    for (int e = 0; e < kN; ++e) {
        s = __builtin_fma((double)w[e], (double)p[e], s);
        q = __builtin_fma((double)w[e], (double)px[e], q);
    }
    group_total<kHeldThreads>(lds, s, q);
    const double over = 1. / ((double)a.N * a.width);
    const float level = (float)(s * over), along = (float)(q * over);
    if (at.mine) {
        held_again(vx);
        held_again(vdy);
        T *dx = const_cast<T *>(at.at(a, a.y, a.sy)) + at.line * a.sy.n;
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
            if (i <= at.all) {
                float xh[kN], da[kN];
                group_terms<P, SILU, kN>(vx[i], vdy[i], mean, rstd, w, b, xh, da);
#pragma unroll
                for (int e = 0; e < kN; ++e) da[e] = r * (w[e] * da[e] - level - xh[e] * along);
                if (i < at.rows) held_store(dx, P::close(da), a.whole_lines);
                dx += a.lines * a.sy.n;
            }
    }
    if constexpr (PARAMS) {
        __shared__ float lines[kHeldThreads * kN];
        float *out = reinterpret_cast<float *>(a.sums) + at.bh * 2 * a.d + at.group * a.width;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
            if (at.mine)
#pragma unroll
                for (int e = 0; e < kN; ++e) lines[at.line * a.width + (at.c - at.group * a.width) + e] = which ? px[e] : p[e];
            __syncthreads();
            // (as many threads as a row has numbers add up their lines in order)
            for (int k = threadIdx.x; k < a.width; k += kHeldThreads) {
                float t = lines[k];
                for (int l = 1; l < a.lines && l < a.N; ++l) t += lines[l * a.width + k];
                out[which * a.d + k] = t;
            }
        }
    }
}

}  // namespace sv

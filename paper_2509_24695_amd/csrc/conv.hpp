// Short causal convolution of each channel along tokens, and its backward pass.
//
//   a_t = bias + sum_j W[j] x_{t-(K-1)+j},  y = a or silu(a);   da = dy or dy silu'(a)
//   dx_t = sum_j W[j] da_{t+(K-1)-j},  dW[j] = sum da_t x_{t-(K-1)+j},  db = sum da_t
//
// A thread owns a piece of the channels, whose taps it keeps in registers, and walks a run of tokens with the last K-1 of them in registers too, so
// that a token is read once (and K-1 more times at the runs' edges, out of the caches).  Forwards bound by memory: 32 760 tokens of 2 240 channels bf16
// 58 us (294 MB, 5.0 TB/s; a copy 56).  Backwards a thread has four channels of either type (with eight, 256 registers and one wave on a SIMD, the call
// below took 174 us), and the vector unit is as busy as the memory: some 30 instructions a value, 62 of the kernel's 80 us for 2 x 20 heads of
// 14 040 and 9 360 tokens of 112 (315 MB, 3.9 TB/s), and 5 us for the fold of the partial sums.  Neighbouring runs
// on one die, which fetches what they share once (it is 19 % of the reads forwards), lose: 59.3 and 87 us.
#pragma once

#include "activation.hpp"
#include "common.hpp"
#include "conv_plan.hpp"
#include "piece.hpp"
#include "sequences.hpp"

namespace sv {

struct ConvArgs {
    const void *x, *dy;
    void *y;                           // backward: dx
    TokStrides sx, sdy, sy;
    const float *weight, *bias;
    const int32_t *lengths;            // or NULL; tokens: slots
    const void *cache_in, *dcache_out;
    void *cache_out;                   // backward: dcache_in
    float *partial;
    int B, H, N, d, run, runs;         // runs of a sequence (backward: workgroups along one)
    int across, n_slots;
    int silu, whole_lines;
    NormDivisor pieces, head_pieces, run_div;
};

template <typename T> using ConvForward = Piece<T>;
template <typename T> using ConvBackward = Quad<T>;

// A thread's channels: head, feature, and place among all channels.
template <typename P> struct ConvPlace {
    int h, i, c;
    __device__ __forceinline__ ConvPlace(const ConvArgs &a, uint32_t piece)
    {
        h = (int)a.head_pieces.quotient(piece);
        i = (int)(piece - (uint32_t)h * a.head_pieces.extent) * P::kN;
        c = h * a.d + i;
    }
};

template <int N> __device__ __forceinline__ void load_floats(const float *p, float (&x)[N])
{
#pragma unroll
    for (int q = 0; q < N / 4; ++q) {
        const f32x4 v = *reinterpret_cast<const f32x4 *>(p + 4 * q);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * q + e] = v[e];
    }
}

// Taps and bias of a piece.
template <typename P, int K> struct ConvWeights {
    static constexpr int kN = P::kN;
    float w[K][kN], b[kN];
    __device__ __forceinline__ ConvWeights(const ConvArgs &a, int c)
    {
        const int64_t channels = (int64_t)a.H * a.d;
#pragma unroll
        for (int j = 0; j < K; ++j) load_floats<kN>(a.weight + j * channels + c, w[j]);
        if (a.bias) load_floats<kN>(a.bias + c, b);
        else
#pragma unroll
            for (int e = 0; e < kN; ++e) b[e] = 0.f;
    }
    // a_t from the K - 1 tokens before t and t itself
    __device__ __forceinline__ float mix(const float (&before)[K - 1][kN], const float (&now)[kN], int e) const
    {
        float s = b[e];
#pragma unroll
        for (int j = 0; j < K - 1; ++j) s = __builtin_fmaf(w[j][e], before[j][e], s);
        return __builtin_fmaf(w[K - 1][e], now[e], s);
    }
};

// Row m of the cache and the tokens one after the other (m = 0: the cache's first); nothing where there is neither.
template <typename T, typename P, int K>
__device__ __forceinline__ typename P::V conv_row(const ConvArgs &a, const T *x, const void *cache, int64_t cache_at, int64_t m, int length)
{
    typedef typename P::V V;
    if (m < K - 1) return cache ? *reinterpret_cast<const V *>(static_cast<const T *>(cache) + cache_at + m * a.d) : V{};
    const int64_t t = m - (K - 1);
    return t < length ? *reinterpret_cast<const V *>(x + t * a.sx.n) : V{};
}

// The rows of a run that come next, AHEAD at a time.  Past the last the last one is read again: no branch stands between a group's
// loads.
template <typename T, typename P, int AHEAD> struct ConvRows {
    typedef typename P::V V;
    const T *at, *end;
    int64_t stride;
    int left;
    V next[AHEAD];
    __device__ __forceinline__ ConvRows(const T *x, int64_t stride, int first, int last)
        : at(x + first * stride), end(x + (last - 1) * stride), stride(stride), left(last - first) {}
    __device__ __forceinline__ void request()
    {
        if (left >= AHEAD) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) next[i] = *reinterpret_cast<const V *>(at + i * stride);
        } else {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) next[i] = *reinterpret_cast<const V *>(i < left ? at + i * stride : end);
        }
        at += AHEAD * stride;
        left -= AHEAD;
    }
    __device__ __forceinline__ void take(V (&v)[AHEAD]) const
    {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) v[i] = next[i];
    }
};

template <int K, int N> __device__ __forceinline__ void conv_shift(float (&w)[K][N], const float (&now)[N])
{
#pragma unroll
    for (int j = 0; j + 1 < K; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) w[j][e] = w[j + 1][e];
#pragma unroll
    for (int e = 0; e < N; ++e) w[K - 1][e] = now[e];
}

template <typename T, int K, bool SILU> __global__ __launch_bounds__(kConvThreads) void conv_rows(ConvArgs a)
{
    using P = ConvForward<T>;
    typedef typename P::V V;
    constexpr int kN = P::kN, kAhead = 4;
    const uint32_t id = blockIdx.x * kConvThreads + threadIdx.x, all = a.pieces.quotient(id), piece = id - all * a.pieces.extent;
    const uint32_t b = a.run_div.quotient(all), run = all - b * a.run_div.extent;
    if ((int)b >= a.B) return;
    const int length = held_length(a.lengths, (int)b, a.N);
    const int first = (int)run * a.run, last = first + a.run < length ? first + a.run : length;
    if (first >= length && run > 0) return;
    const ConvPlace<P> at(a, piece);
    const T *x = static_cast<const T *>(a.x) + b * a.sx.b + at.h * a.sx.h + at.i;
    T *y = static_cast<T *>(a.y) + b * a.sy.b + at.h * a.sy.h + at.i;
    const int64_t cache_at = ((int64_t)b * a.H + at.h) * (K - 1) * a.d + at.i;
    if (first < last) {
        ConvRows<T, P, kAhead> rows(x, a.sx.n, first, last);
        rows.request();
        float before[K - 1][kN];
#pragma unroll
        for (int j = 0; j < K - 1; ++j) P::open(conv_row<T, P, K>(a, x, a.cache_in, cache_at, first + j, length), before[j]);
        const ConvWeights<P, K> w(a, at.c);
        T *to = y + first * a.sy.n;
        for (int t = first; t < last; t += kAhead) {
            V v[kAhead];
            rows.take(v);
            rows.request();
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                float now[kN], out[kN];
                P::open(v[i], now);
#pragma unroll
                for (int e = 0; e < kN; ++e) {
                    out[e] = w.mix(before, now, e);
                    if (SILU) out[e] = silu(out[e]);
                }
                if (t + i < last) store16(to + i * a.sy.n, P::close(out), a.whole_lines);
                conv_shift(before, now);
            }
            to += kAhead * a.sy.n;
        }
    }
    // the run that read the old cache writes the new one, which may be the same memory
    if (run == 0 && a.cache_out) {
        V rows[K - 1];
#pragma unroll
        for (int r = 0; r < K - 1; ++r) rows[r] = conv_row<T, P, K>(a, x, a.cache_in, cache_at, (int64_t)length + r, length);
#pragma unroll
        for (int r = 0; r < K - 1; ++r) *reinterpret_cast<V *>(static_cast<T *>(a.cache_out) + cache_at + (int64_t)r * a.d) = rows[r];
    }
}

// One token of each row of a batch: a workgroup has `across` pieces of one row.
template <typename T, int K, bool SILU> __global__ __launch_bounds__(kConvThreads) void conv_token(ConvArgs a)
{
    using P = ConvForward<T>;
    typedef typename P::V V;
    constexpr int kN = P::kN;
    const int b = (int)(blockIdx.x / a.runs);
    const uint32_t piece = blockIdx.x % a.runs * a.across + threadIdx.x;
    const int slot = a.lengths ? a.lengths[b] : b;
    if (slot < 0 || slot >= a.n_slots) return;
    const bool mine = threadIdx.x < (unsigned)a.across && piece < a.pieces.extent;
    const ConvPlace<P> at(a, mine ? piece : 0);
    const int64_t cache_at = ((int64_t)slot * a.H + at.h) * (K - 1) * a.d + at.i;
    const T *x = static_cast<const T *>(a.x) + b * a.sx.b + at.h * a.sx.h + at.i;
    V rows[K];
#pragma unroll
    for (int j = 0; j < K; ++j) rows[j] = conv_row<T, P, K>(a, x, a.cache_in, cache_at, j, 1);
    const ConvWeights<P, K> w(a, at.c);
    if (slot_taken(a.lengths, b, slot) || !mine) return;
    float before[K - 1][kN], now[kN], out[kN];
#pragma unroll
    for (int j = 0; j < K - 1; ++j) P::open(rows[j], before[j]);
    P::open(rows[K - 1], now);
#pragma unroll
    for (int e = 0; e < kN; ++e) {
        out[e] = w.mix(before, now, e);
        if (SILU) out[e] = silu(out[e]);
    }
    *reinterpret_cast<V *>(static_cast<T *>(a.y) + b * a.sy.b + at.h * a.sy.h + at.i) = P::close(out);
#pragma unroll
    for (int r = 0; r < K - 1; ++r) *reinterpret_cast<V *>(static_cast<T *>(a.cache_out) + cache_at + (int64_t)r * a.d) = rows[r + 1];
}

// dx of a run of tokens (of the cache too, for a sequence's first run), and the workgroup's part of dW and db.  With da_t known for the last
// K tokens, row m of cache and tokens together gets sum_j W[j] da_{m-j}; so a run goes on for K - 1 tokens of the next.
template <typename T, int K, bool SILU, bool PARAMS> __global__ __launch_bounds__(kConvThreads) void conv_rows_backward(ConvArgs a)
{
    using P = ConvBackward<T>;
    typedef typename P::V V;
    constexpr int kN = P::kN, kAhead = 4;
    const uint32_t tiles = (a.pieces.extent + a.across - 1) / a.across, tile = blockIdx.x % tiles, rest = blockIdx.x / tiles;
    const int block = (int)(rest % a.runs), b = (int)(rest / a.runs), down = kConvThreads / a.across;
    const int col = (int)threadIdx.x % a.across, line = (int)threadIdx.x / a.across;
    const uint32_t piece = tile * a.across + col;
    const bool mine = piece < a.pieces.extent && line < down;
    const int length = held_length(a.lengths, b, a.N);
    const int64_t begin = ((int64_t)block * down + line) * a.run;      // past the last token of a short sequence: nothing
    const int first = begin < length ? (int)begin : length, last = first + a.run < length ? first + a.run : length;
    const ConvPlace<P> at(a, mine ? piece : 0);
    float dw[K][kN], db[kN];
#pragma unroll
    for (int e = 0; e < kN; ++e) {
        db[e] = 0.f;
#pragma unroll
        for (int j = 0; j < K; ++j) dw[j][e] = 0.f;
    }
    const int64_t cache_at = ((int64_t)b * a.H + at.h) * (K - 1) * a.d + at.i;
    const T *dcache_out = a.dcache_out ? static_cast<const T *>(a.dcache_out) + cache_at : nullptr;
    T *dcache_in = a.cache_out ? static_cast<T *>(a.cache_out) + cache_at : nullptr;
    if (mine && first < last) {
        const T *x = static_cast<const T *>(a.x) + b * a.sx.b + at.h * a.sx.h + at.i;
        const T *dy = static_cast<const T *>(a.dy) + b * a.sdy.b + at.h * a.sdy.h + at.i;
        T *dx = static_cast<T *>(a.y) + b * a.sy.b + at.h * a.sy.h + at.i;
        const int end = last + K - 1, live = end < length ? end : length;      // rows [first, end) of da, tokens up to `live`
        ConvRows<T, P, kAhead> xs(x, a.sx.n, first, live), dys(dy, a.sdy.n, first, live);
        xs.request();
        dys.request();
        float before[K - 1][kN], da[K][kN];
#pragma unroll
        for (int j = 0; j < K - 1; ++j) P::open(conv_row<T, P, K>(a, x, a.cache_in, cache_at, first + j, length), before[j]);
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int e = 0; e < kN; ++e) da[j][e] = 0.f;
        const ConvWeights<P, K> w(a, at.c);
        T *to = dx + (int64_t)(first - (K - 1)) * a.sy.n;              // of the row that da_t is the last to reach
        // rows t .. t + kAhead - 1; `inside`: all of them are tokens of this run
        auto group = [&](int t, auto inside) {
            V vx[kAhead], vdy[kAhead];
            xs.take(vx);
            dys.take(vdy);
            xs.request();
            dys.request();
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int m = t + i;                                  // da_m is the newest that row m gets
                float now[kN], g[kN], out[kN];
                P::open(vx[i], now);
                P::open(vdy[i], g);
#pragma unroll
                for (int e = 0; e < kN; ++e) {
                    if (SILU) {
                        const float y = w.mix(before, now, e);
                        g[e] *= silu_slope(y, sigmoid(y));
                    }
                    if (!inside()) g[e] = m < live ? g[e] : 0.f;
                }
                // (not with a factor of zero for the next run's tokens: they may be no numbers)
                if (PARAMS && (inside() || m < last)) {
#pragma unroll
                    for (int e = 0; e < kN; ++e) {
#pragma unroll
                        for (int j = 0; j < K - 1; ++j) dw[j][e] = __builtin_fmaf(g[e], before[j][e], dw[j][e]);
                        dw[K - 1][e] = __builtin_fmaf(g[e], now[e], dw[K - 1][e]);
                        db[e] += g[e];
                    }
                }
                conv_shift(da, g);
                conv_shift(before, now);
#pragma unroll
                for (int e = 0; e < kN; ++e) {
                    out[e] = w.w[0][e] * da[K - 1][e];
#pragma unroll
                    for (int j = 1; j < K; ++j) out[e] = __builtin_fmaf(w.w[j][e], da[K - 1 - j][e], out[e]);
                }
                if (!inside() && dcache_out && m >= length && m < end) {
                    float more[kN];
                    P::open(*reinterpret_cast<const V *>(dcache_out + (m - length) * a.d), more);
#pragma unroll
                    for (int e = 0; e < kN; ++e) out[e] += more[e];
                }
                if ((inside() || m < end) && (i >= K - 1 || m - first >= K - 1)) store16(to + i * a.sy.n, P::close(out), a.whole_lines);
                else if (dcache_in && m < K - 1) *reinterpret_cast<V *>(dcache_in + m * a.d) = P::close(out);       // (m < end: K - 1 at least)
            }
            to += kAhead * a.sy.n;
        };
        int t = first;
        for (; t + kAhead <= last; t += kAhead) group(t, std::true_type{});
        for (; t < end; t += kAhead) group(t, std::false_type{});
    } else if (mine && length == 0 && begin == 0 && dcache_in) {
        // no tokens: the cache was handed through
        V rows[K - 1];
#pragma unroll
        for (int r = 0; r < K - 1; ++r) rows[r] = dcache_out ? *reinterpret_cast<const V *>(dcache_out + r * a.d) : V{};
#pragma unroll
        for (int r = 0; r < K - 1; ++r) *reinterpret_cast<V *>(dcache_in + r * a.d) = rows[r];
    }
    if constexpr (PARAMS) {
        // lanes with the same channels are added up in order of their runs
        __shared__ float sums[kConvThreads * kN];
        const int64_t channels = (int64_t)a.H * a.d;
        float *partial = a.partial + rest * channels * (K + 1);
        const int width = a.across * kN;
#pragma unroll
        for (int j = 0; j <= K; ++j) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kN; ++e)
                if (line < down) sums[(line * kN + e) * a.across + col] = j < K ? dw[j < K ? j : 0][e] : db[e];
            __syncthreads();
            for (int q = threadIdx.x; q < width; q += kConvThreads) {
                float s = sums[q];
                for (int r = 1; r < down; ++r) s += sums[r * width + q];
                const uint32_t p = tile * a.across + q % a.across;
                if (p < a.pieces.extent) partial[j * channels + ConvPlace<P>(a, p).c + q / a.across] = s;
            }
        }
    }
}

// Partial sums [parts][floats], added up in sixteen runs and these in order; the first `split` numbers go to one place, the rest to another.
struct FoldArgs {
    const float *partial;
    int64_t parts, floats, split;
    float *first, *second;             // either may be NULL
};
__global__ __launch_bounds__(256) void fold_parts(FoldArgs a)
{
    constexpr int kRuns = 16, kQuads = 16;
    __shared__ f32x4 runs[kRuns][kQuads];
    const int64_t quads = a.floats / 4, q = (int64_t)blockIdx.x * kQuads + threadIdx.x % kQuads;
    const int run = threadIdx.x / kQuads;
    const f32x4 *p = reinterpret_cast<const f32x4 *>(a.partial);
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if (q < quads) {
#pragma unroll 8
        for (int64_t w = run; w < a.parts; w += kRuns) s += p[w * quads + q];
    }
    runs[run][threadIdx.x % kQuads] = s;
    __syncthreads();
    if (run == 0 && q < quads) {
#pragma unroll
        for (int r = 1; r < kRuns; ++r) s += runs[r][threadIdx.x];
        float *out = q * 4 < a.split ? a.first : a.second;
        if (out) *reinterpret_cast<f32x4 *>(out + (q * 4 < a.split ? q * 4 : q * 4 - a.split)) = s;
    }
}

}  // namespace sv

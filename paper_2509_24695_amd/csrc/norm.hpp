// Layer norm over the rows of a token tensor, and its backward pass.
//
//   mean = sum x / d,   rstd = 1 / sqrt(sum (x - mean)^2 / d + eps),   xh = (x - mean) rstd,   y = w xh + b
//   dx = rstd (t - sum t / d - xh sum (t xh) / d)  with t = w dy,   dw = sum over rows of dy xh,   db = sum over rows of dy
//
// Bound by memory: a row is read once into registers (16 bytes per lane and piece), its sums go across the lanes that hold it, and it is
// written from there, while the next one is on its way (two and four rows at a time gained nothing).  A lane keeps the same features for all
// rows that its workgroup walks, so the parameters stay in registers too, and the backward pass adds up dw and db of its features there: a
// workgroup leaves one partial sum of each, norm_fold adds these up in order.  32 760 rows of 2 240 features, with buffers that change from
// call to call: bf16 forwards 55 us (294 MB, 5.4 TB/s), backwards 88 (441 MB, 5.0 TB/s, the fold of 9 MB of partial sums included), fp32 111 (587 MB, 5.3
// TB/s) and 157 (881 MB, 5.6 TB/s).
#pragma once

#include "common.hpp"
#include "norm_plan.hpp"
#include "piece.hpp"

namespace sv {

// An axis of the rows' index, fastest first; strides in elements of the tensors and of the statistics.
struct NormAxis {
    NormDivisor extent;
    int64_t a, b, c, stat;
};
struct NormArgs {
    const void *x, *dy;            // dy: backward only
    void *y;                       // backward: dx
    const float *weight, *bias;    // [groups][d] or NULL
    float *mean, *rstd;            // forward: written, may be NULL
    float *partial;                // [groups][workgroups][2][d]
    float *dw, *db;
    NormAxis axis[3];              // a: x, b: y (forward) or dy, c: dx
    int64_t group_a, group_b, group_c, group_stat;     // strides of the groups
    int64_t rows;                  // of a group
    int d, groups, workgroups;     // workgroups of a group
    int whole_lines;               // rows are whole 128-byte lines: written past the caches
    float eps;
};

// Sum over the LANES lanes that hold a row; every one of them gets it, added in the same order.
template <int LANES> __device__ __forceinline__ float row_sum(float x, float *lds)
{
    constexpr int kIn = LANES > 64 ? 64 : LANES;
    if constexpr (kIn >= 16) x = row16_sum(x);
    else {
        x = dpp_add<0xb1>(x);
        x = dpp_add<0x4e>(x);
        if constexpr (kIn == 8) x = dpp_add<0x141>(x);
    }
#pragma unroll
    for (int m = 16; m < kIn; m *= 2) x += __shfl_xor(x, m, 64);
    if constexpr (LANES > 64) {
        constexpr int kWaves = LANES / 64;
        lds_barrier();                                                // the last sum has been read
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
        lds_barrier();
        const float *mine = lds + threadIdx.x / LANES * kWaves;
        x = mine[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) x += mine[w];
    }
    return x;
}

// The rows that a lane's workgroup walks: rows first, first + step, ... of its group.
template <int LANES> struct NormWalk {
    static constexpr int kThreadsOf = LANES > 256 ? LANES : 256, kRows = kThreadsOf / LANES;
    int group, slot, lane;
    int64_t row, step;
    __device__ __forceinline__ explicit NormWalk(const NormArgs &a)
        : group((int)(blockIdx.x / a.workgroups)), slot((int)(blockIdx.x % a.workgroups)), lane((int)threadIdx.x % LANES),
          row((int64_t)slot * kRows + threadIdx.x / LANES), step((int64_t)a.workgroups * kRows) {}
};
struct NormPlace {
    int64_t a, b, c, stat;
    __device__ __forceinline__ NormPlace(const NormArgs &g, int group, int64_t row)
        : a(group * g.group_a), b(group * g.group_b), c(group * g.group_c), stat(group * g.group_stat)
    {
        uint32_t r = (uint32_t)row;                                   // the host keeps rows below 2^31
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const uint32_t q = i < 2 ? g.axis[i].extent.quotient(r) : 0u, k = r - q * g.axis[i].extent.extent;
            a += k * g.axis[i].a;
            b += k * g.axis[i].b;
            c += k * g.axis[i].c;
            stat += k * g.axis[i].stat;
            r = q;
        }
    }
};

// (d == 0: nothing, zeros)
template <typename T, int LANES, int VECS> __device__ __forceinline__ void load_row(const void *base, int64_t at, int lane, int d, u32x4 (&v)[VECS])
{
    const T *p = static_cast<const T *>(base) + at;
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
        const int f = (lane + i * LANES) * Piece<T>::kN;
        v[i] = f < d ? *reinterpret_cast<const u32x4 *>(p + f) : u32x4{0u, 0u, 0u, 0u};
    }
}

// A lane's part of a row of parameters, or `otherwise` where there is none.
template <typename T, int LANES, int VECS>
__device__ __forceinline__ void load_parameters(const float *p, int group, int lane, int d, float otherwise, float (&w)[VECS][Piece<T>::kN])
{
#pragma unroll
    for (int i = 0; i < VECS; ++i)
#pragma unroll
        for (int q = 0; q < Piece<T>::kN / 4; ++q) {
            const int f = (lane + i * LANES) * Piece<T>::kN + 4 * q;
            const f32x4 x = p && f < d ? *reinterpret_cast<const f32x4 *>(p + (int64_t)group * d + f) : f32x4{otherwise, otherwise, otherwise, otherwise};
#pragma unroll
            for (int e = 0; e < 4; ++e) w[i][4 * q + e] = x[e];
        }
}

template <typename T, int LANES, int VECS> __global__ __launch_bounds__((NormWalk<LANES>::kThreadsOf)) void norm_rows(NormArgs a)
{
    constexpr int kN = Piece<T>::kN;
    __shared__ float lds[16];
    NormWalk<LANES> walk(a);
    const int64_t first = walk.row - threadIdx.x / LANES;             // whole workgroups stay together: row_sum has barriers
    float w[VECS][kN], b[VECS][kN];
    load_parameters<T, LANES, VECS>(a.weight, walk.group, walk.lane, a.d, 1.f, w);
    load_parameters<T, LANES, VECS>(a.bias, walk.group, walk.lane, a.d, 0.f, b);
    const float over = 1.f / (float)a.d;
    const int64_t last = a.rows - 1;
    u32x4 next[VECS];
    // (nothing of a row past the last, which another workgroup may be writing where Y is X)
    auto request = [&](int64_t row) {
        load_row<T, LANES, VECS>(a.x, NormPlace(a, walk.group, row < last ? row : last).a, walk.lane, row <= last ? a.d : 0, next);
    };
    request(walk.row);
    for (int64_t at = first; at < a.rows; at += walk.step) {
        const int64_t row = at + threadIdx.x / LANES;
        u32x4 v[VECS];
#pragma unroll
        for (int i = 0; i < VECS; ++i) v[i] = next[i];
        if (at + walk.step < a.rows) request(row + walk.step);
        float sum = 0.f, x[VECS][kN];
#pragma unroll
        for (int i = 0; i < VECS; ++i) {
            Piece<T>::open(v[i], x[i]);
#pragma unroll
            for (int e = 0; e < kN; ++e) sum += x[i][e];
        }
        const float mean = row_sum<LANES>(sum, lds) * over;
        float var = 0.f;
#pragma unroll
        for (int i = 0; i < VECS; ++i) {
            const bool in = (walk.lane + i * LANES) * kN < a.d;
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                x[i][e] = in ? x[i][e] - mean : 0.f;
                var = __builtin_fmaf(x[i][e], x[i][e], var);
            }
        }
        const float rstd = 1.f / sqrtf(row_sum<LANES>(var, lds) * over + a.eps);
        if (row > last) continue;
        const NormPlace place(a, walk.group, row);
        T *y = static_cast<T *>(a.y) + place.b;
#pragma unroll
        for (int i = 0; i < VECS; ++i) {
            const int f = (walk.lane + i * LANES) * kN;
#pragma unroll
            for (int e = 0; e < kN; ++e) x[i][e] = __builtin_fmaf(x[i][e] * rstd, w[i][e], b[i][e]);
            if (f < a.d) store16(y + f, Piece<T>::close(x[i]), a.whole_lines);
        }
        if (a.mean && walk.lane == 0) {
            a.mean[place.stat] = mean;
            a.rstd[place.stat] = rstd;
        }
    }
}

// dx of the rows, and the workgroup's part of dw and db.
template <typename T, int LANES, int VECS, bool PARAMS> __global__ __launch_bounds__((NormWalk<LANES>::kThreadsOf)) void norm_rows_backward(NormArgs a)
{
    constexpr int kN = Piece<T>::kN, kRows = NormWalk<LANES>::kRows;
    __shared__ float lds[16];
    NormWalk<LANES> walk(a);
    const int64_t first = walk.row - threadIdx.x / LANES;
    float w[VECS][kN], dw[VECS][kN], db[VECS][kN];
    load_parameters<T, LANES, VECS>(a.weight, walk.group, walk.lane, a.d, 1.f, w);
#pragma unroll
    for (int i = 0; i < VECS; ++i)
#pragma unroll
        for (int e = 0; e < kN; ++e) dw[i][e] = db[i][e] = 0.f;
    const float over = 1.f / (float)a.d;
    const int64_t last = a.rows - 1;
    u32x4 nx[VECS], ndy[VECS];
    float nmean, nrstd;
    auto request = [&](int64_t row) {
        const NormPlace p(a, walk.group, row < last ? row : last);
        // a row past the last is one of zeros: the last row's gradient times nothing would be NaN where that gradient is infinite, and dX may
        // already have taken its place
        const int d = row <= last ? a.d : 0;
        load_row<T, LANES, VECS>(a.x, p.a, walk.lane, d, nx);
        load_row<T, LANES, VECS>(a.dy, p.b, walk.lane, d, ndy);
        nmean = a.mean[p.stat];
        nrstd = a.rstd[p.stat];
    };
    request(walk.row);
    for (int64_t at = first; at < a.rows; at += walk.step) {
        const int64_t row = at + threadIdx.x / LANES;
        u32x4 vx[VECS], vdy[VECS];
#pragma unroll
        for (int i = 0; i < VECS; ++i) {
            vx[i] = nx[i];
            vdy[i] = ndy[i];
        }
        const float mean = nmean, rstd = nrstd;
        if (at + walk.step < a.rows) request(row + walk.step);
        const bool live = row <= last;
        float level = 0.f, along = 0.f;
#pragma unroll
        for (int i = 0; i < VECS; ++i) {
            float x[kN], g[kN];
            Piece<T>::open(vx[i], x);
            Piece<T>::open(vdy[i], g);
            const bool in = live && (walk.lane + i * LANES) * kN < a.d;
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                const float xh = in ? (x[e] - mean) * rstd : 0.f, t = w[i][e] * g[e];
                level += t;
                along = __builtin_fmaf(t, xh, along);
                if (PARAMS) {
                    dw[i][e] = __builtin_fmaf(g[e], xh, dw[i][e]);
                    db[i][e] += g[e];
                }
            }
        }
        level = row_sum<LANES>(level, lds) * over;
        along = row_sum<LANES>(along, lds) * over;
        if (!live) continue;
        T *dx = static_cast<T *>(a.y) + NormPlace(a, walk.group, row).c;
#pragma unroll
        for (int i = 0; i < VECS; ++i) {
            const int f = (walk.lane + i * LANES) * kN;
            float x[kN], g[kN];
            Piece<T>::open(vx[i], x);
            Piece<T>::open(vdy[i], g);
#pragma unroll
            for (int e = 0; e < kN; ++e) x[e] = rstd * (w[i][e] * g[e] - level - (x[e] - mean) * rstd * along);
            if (f < a.d) store16(dx + f, Piece<T>::close(x), a.whole_lines);
        }
    }
    if constexpr (PARAMS) {
        float *out = a.partial + (int64_t)blockIdx.x * 2 * a.d;
        // lanes of the workgroup that hold the same features are added up in order of their rows
        if constexpr (kRows == 1) {
#pragma unroll
            for (int i = 0; i < VECS; ++i) {
                const int f = (walk.lane + i * LANES) * kN;
#pragma unroll
                for (int e = 0; e < kN; ++e)
                    if (f < a.d) {
                        out[f + e] = dw[i][e];
                        out[a.d + f + e] = db[i][e];
                    }
            }
        } else {
            __shared__ float sums[kRows][LANES * kN + 1];
#pragma unroll
            for (int which = 0; which < 2; ++which)
#pragma unroll
                for (int i = 0; i < VECS; ++i) {
                    __syncthreads();
#pragma unroll
                    for (int e = 0; e < kN; ++e) sums[threadIdx.x / LANES][walk.lane * kN + e] = which ? db[i][e] : dw[i][e];
                    __syncthreads();
                    for (int c = threadIdx.x; c < LANES * kN; c += NormWalk<LANES>::kThreadsOf) {
                        float s = sums[0][c];
#pragma unroll 4
                        for (int r = 1; r < kRows; ++r) s += sums[r][c];
                        const int f = i * LANES * kN + c;
                        if (f < a.d) out[which * a.d + f] = s;
                    }
                }
        }
    }
}

// dw and db of each group: the workgroups' partial sums, added up in sixteen runs and these in order.
__global__ __launch_bounds__(256) void norm_fold(NormArgs a)
{
    constexpr int kRuns = 16, kQuads = 16;
    __shared__ f32x4 runs[kRuns][kQuads];
    const int quads = a.d / 4 * 2, tiles = (quads + kQuads - 1) / kQuads;
    const int group = (int)(blockIdx.x / tiles), q = (int)(blockIdx.x % tiles) * kQuads + (int)(threadIdx.x % kQuads), run = threadIdx.x / kQuads;
    const f32x4 *p = reinterpret_cast<const f32x4 *>(a.partial) + (int64_t)group * a.workgroups * quads;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if (q < quads) {
#pragma unroll 8
        for (int w = run; w < a.workgroups; w += kRuns) s += p[(int64_t)w * quads + q];
    }
    runs[run][threadIdx.x % kQuads] = s;
    __syncthreads();
    if (run == 0 && q < quads) {
#pragma unroll
        for (int r = 1; r < kRuns; ++r) s += runs[r][threadIdx.x];
        const int half = a.d / 4, which = q >= half, f = (q - which * half) * 4;
        float *out = which ? a.db : a.dw;
        if (out) *reinterpret_cast<f32x4 *>(out + (int64_t)group * a.d + f) = s;
    }
}

}  // namespace sv

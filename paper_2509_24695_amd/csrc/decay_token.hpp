// One token of decayed linear attention for each row of a batch, whose states lie in a pool:
//
//   S' = l S + k v^T,   o = scale S'^T q
//
// A call moves the states, 2 d^2 fp32 per row and head, and next to nothing else: a workgroup takes the columns of one head's state
// (all, or a quarter where there are few heads), each thread a column group of four of every R-th row, all of its loads in flight at once.
// 187 rows of 16 heads of 128, 395 MB, with pools that change from call to call: 79 us, 5.0 TB/s (60 on one pair of pools, part of which
// the 256 MB cache then holds).  States that go to another pool are written past the caches (82.5 us without the hint); states that are written in
// place are not (86 us, on one pool 61 with the hint and 59 without).
//
// Row b looks through the slots of the rows before it: 4 b bytes for each of its heads.  256 rows of 16 heads of 128 87 us, without slots 86; 16 384 of 16
// heads of 64 1 871 and 1 581; 16 384 of 2 heads of 32, whose states are as many bytes as that, 124 and 45.
#pragma once

#include "common.hpp"

namespace sv {

struct TokenArgs {
    const void *q, *k, *v;
    void *o;
    int64_t sb, sh, ob, oh;        // element strides of rows and heads
    const float *log_decay;
    const int32_t *slots;          // [B] or NULL: row b has state b
    int n_slots, B, H;
    float scale;
    const float *s_in;
    float *s_out;                  // [n_slots][H][d][d]; may be s_in
};
// Up to this many heads of all rows a workgroup takes a quarter of one (us with quarters / whole heads: 20 of 112 4.1 / 4.6, 32 of 128 3.8 / 4.6, 256
// of 128 5.6 / 6.5; 5 120 of 112 192 / 107, whose workgroups are then many and short).
constexpr int kFewTokenHeads = 256;

// SPLIT: workgroups per head.  Threads: kGroups column groups x kRows rows.
template <int D, int SPLIT> struct TokenShape {
    static constexpr int kGroups = D / 4 / SPLIT, kRows = 256 / kGroups < 32 ? 256 / kGroups / 8 * 8 : 32;
    static constexpr int kTokThreads = kGroups * kRows, kSteps = (D + kRows - 1) / kRows;
    static_assert(kGroups * 4 * SPLIT == D, "whole column groups");
};

template <typename T, int D, int SPLIT> __global__ __launch_bounds__(256) void decay_token(TokenArgs a)
{
    using W = TokenShape<D, SPLIT>;
    __shared__ float qs[D], ks[D];
    __shared__ f32x4 sums[W::kRows][W::kGroups];
    const int part = blockIdx.x % SPLIT, h = blockIdx.x / SPLIT % a.H, b = blockIdx.x / SPLIT / a.H;
    const int slot = a.slots ? a.slots[b] : b;
    if (slot < 0 || slot >= a.n_slots) return;
    const int group = threadIdx.x % W::kGroups, row0 = threadIdx.x / W::kGroups, c = (part * W::kGroups + group) * 4;
    const int64_t at = ((int64_t)slot * a.H + h) * D * D;
    f32x4 s[W::kSteps];
#pragma unroll
    for (int i = 0; i < W::kSteps; ++i) {
        const int row = row0 + i * W::kRows;
        s[i] = row < D ? *reinterpret_cast<const f32x4 *>(a.s_in + at + row * D + c) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const T *q = static_cast<const T *>(a.q) + b * a.sb + h * a.sh, *k = static_cast<const T *>(a.k) + b * a.sb + h * a.sh;
    const T *v = static_cast<const T *>(a.v) + b * a.sb + h * a.sh;
    if (threadIdx.x < D) {
        qs[threadIdx.x] = Elem<T>::load(q + threadIdx.x);
        ks[threadIdx.x] = Elem<T>::load(k + threadIdx.x);
    }
    float vv[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) vv[e] = Elem<T>::load(v + c + e);
    // a slot that an earlier row has already is left to that row
    bool taken = false;
    if (a.slots)
        for (int r = threadIdx.x; r < b; r += W::kTokThreads) taken |= a.slots[r] == slot;
    if (__syncthreads_or(taken)) return;
    const float grown = expf(a.log_decay[h]), l = grown > 3.40282347e38f ? 3.40282347e38f : grown;       // a state of nothing stays one
    const bool elsewhere = a.s_out != a.s_in;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < W::kSteps; ++i) {
        const int row = row0 + i * W::kRows;
        if (row < D) {
            const float kk = ks[row], qq = qs[row];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[i][e] = __builtin_fmaf(kk, vv[e], l * s[i][e]);
                sum[e] = __builtin_fmaf(qq, s[i][e], sum[e]);
            }
            store16(a.s_out + at + row * D + c, s[i], elsewhere);
        }
    }
    sums[row0][group] = sum;
    __syncthreads();
    if (threadIdx.x < W::kGroups * 4) {
        const float *p = reinterpret_cast<const float *>(&sums[0][0]) + threadIdx.x;
        float o = 0.f;
#pragma unroll 8
        for (int r = 0; r < W::kRows; ++r) o += p[r * W::kGroups * 4];
        Elem<T>::store(static_cast<T *>(a.o) + b * a.ob + h * a.oh + part * W::kGroups * 4 + threadIdx.x, a.scale * o);
    }
}

}  // namespace sv

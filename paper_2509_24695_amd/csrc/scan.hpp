// Selective state space scan: per channel c and state number i
//
//   D_t = softplus(dt_t + dt_bias),  h_t[i] = exp(D_t A[i]) h_{t-1}[i] + D_t u_t B_t[i],  y_t = (sum_i C_t[i] h_t[i] + skip u_t) silu(z_t)
//
// A lane owns a channel and holds its n states; B_t and C_t are the same for all lanes of a wave and come through the scalar cache.  Bound
// by the vector unit: an exponential and four other instructions for each state, with softplus and the gate beside them.  A long sequence
// is cut into segments that are walked side by side: scan_sums finds what each segment adds to a state of nothing and its sum of steps,
// scan_states turns these into the states the segments begin from (what a segment keeps of its state is exp(A sum D)), and scan_walk
// walks from there.  32 760 tokens of 2 240 channels, n = 16, with a gate, bf16: 491 us (590 MB); under the profiler, whose clock is lower, the sums 219, the states 28, the walk 297
// (an exponential costs 2.2 instructions, the walk 117 instructions a value and token: at the rate that the vector unit reaches, 36 T a second, 182 and 280 us).  Decays that are
// kept instead of worked out twice would be 64 bytes a value.
#pragma once

#include "activation.hpp"
#include "common.hpp"
#include "scan_plan.hpp"
#include "sequences.hpp"

namespace sv {

struct ScanArgs {
    const void *u, *dt, *z, *bm, *cm, *dy;
    void *y;
    TokStrides su, sz, sbc, sy;              // sy: y, or dy
    const float *A, *dt_bias, *skip;
    const int32_t *lengths;
    const float *s_in, *ds_out;
    float *s_out;
    float *states, *grads, *steps;           // [B][segments][n][C], the same, [B][segments][C]
    float *marks, *mark_steps;               // [B][runs][n][C], [B][runs][C]: local states before each run of tokens
    float *shared, *params;                  // [B][blocks][N][2][n]; [B][segments][n + 2][C]
    void *du, *ddt, *dz, *db, *dc;
    float *ds_in, *dA, *ddt_bias, *dskip;
    int B, H, N, d, G, channels, group_channels, group_blocks, blocks;
    int segments, per_segment, runs;
};

// Where a wave's lanes work: a block of 64 channels of one group.  Lanes past the group's last channel double it and store nothing.
struct ScanPlace {
    int b, segment, group, block, channel, length, first, last;
    bool mine;
    int64_t u, z, y;                         // elements of token 0
    __device__ __forceinline__ ScanPlace(const ScanArgs &a, uint32_t id)
    {
        block = (int)(id % (uint32_t)a.blocks);
        id /= (uint32_t)a.blocks;
        segment = (int)(id % (uint32_t)a.segments);
        b = (int)(id / (uint32_t)a.segments);
        group = block / a.group_blocks;
        int c = (block - group * a.group_blocks) * kScanWave + (int)threadIdx.x % kScanWave;
        mine = c < a.group_channels;
        c = mine ? c : a.group_channels - 1;
        channel = group * a.group_channels + c;
        const int h = channel / a.d, i = channel - h * a.d;
        u = b * a.su.b + h * a.su.h + i;
        z = b * a.sz.b + h * a.sz.h + i;
        y = b * a.sy.b + h * a.sy.h + i;
        length = held_length(a.lengths, b, a.N);
        first = segment * a.per_segment;
        const int64_t end = (int64_t)first + a.per_segment;
        last = end < length ? (int)end : length;
    }
    __device__ __forceinline__ int64_t slot(const ScanArgs &a) const { return (int64_t)b * a.segments + segment; }
};

// n numbers that are the same for all lanes, out of the scalar cache.  Scalar loads come back in any order, so a wait for one waits for all:
// arrive() makes it in front of the request for the next token's numbers, which then are on their way for a whole token.
template <typename T, int n> struct Scalars;
template <int n> struct Scalars<float, n> {
    uint32_t w[n];
    __device__ __forceinline__ void load(const void *base, int64_t at)
    {
        const auto *p = (const __attribute__((address_space(4))) uint32_t *)(reinterpret_cast<uintptr_t>(base) + at * 4);
#pragma unroll
        for (int i = 0; i < n; ++i) w[i] = p[i];
    }
    __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(w[i]); }
    __device__ __forceinline__ void arrive()
    {
#pragma unroll
        for (int i = 0; i < n; ++i) asm volatile("" : "+s"(w[i]));
    }
};
template <int n> struct Scalars<uint16_t, n> {
    uint32_t w[n / 2];
    __device__ __forceinline__ void load(const void *base, int64_t at)
    {
        const auto *p = (const __attribute__((address_space(4))) uint32_t *)(reinterpret_cast<uintptr_t>(base) + at * 2);
#pragma unroll
        for (int i = 0; i < n / 2; ++i) w[i] = p[i];
    }
    __device__ __forceinline__ float operator[](int i) const { return i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]); }
    __device__ __forceinline__ void arrive()
    {
#pragma unroll
        for (int i = 0; i < n / 2; ++i) asm volatile("" : "+s"(w[i]));
    }
};

// A channel's A, times log2(e): exp(D A) = 2^(D A2).
template <int n> __device__ __forceinline__ void load_rates(const ScanArgs &a, int channel, float (&A2)[n])
{
#pragma unroll
    for (int q = 0; q < n / 4; ++q) {
        const f32x4 v = *reinterpret_cast<const f32x4 *>(a.A + (int64_t)channel * n + 4 * q);
#pragma unroll
        for (int e = 0; e < 4; ++e) A2[4 * q + e] = v[e] * kLog2E;
    }
}
// A state as it lies in S_in: a channel's n numbers side by side.
template <int n> __device__ __forceinline__ void load_state(const float *p, int64_t row, float (&h)[n])
{
#pragma unroll
    for (int q = 0; q < n / 4; ++q) {
        const f32x4 v = p ? *reinterpret_cast<const f32x4 *>(p + row * n + 4 * q) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 4; ++e) h[4 * q + e] = v[e];
    }
}
template <int n> __device__ __forceinline__ void store_state(float *p, int64_t row, const float (&h)[n])
{
#pragma unroll
    for (int q = 0; q < n / 4; ++q) *reinterpret_cast<f32x4 *>(p + row * n + 4 * q) = f32x4{h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]};
}
// What a run of tokens whose steps sum to `steps` makes of a state number s, with what the run adds: exp(A steps) s + add.  The exponential may be far outside of
// fp32's range where its product with s is not (a state of 1e-30 that grows, one of 1e30 that decays, one of nothing that stays so): what its exponent has
// past 125 goes into that of s.
__device__ __forceinline__ float carried(float A2, float steps, float s, float add)
{
    const float x = __builtin_amdgcn_fmed3f(A2 * steps, -1000.f, 1000.f), past = __builtin_rintf(x - __builtin_amdgcn_fmed3f(x, -125.f, 125.f));
    return __builtin_fmaf(__builtin_amdgcn_exp2f(x - past), __builtin_amdgcn_ldexpf(s, (int)past), add);
}
// Has a lane of the wave a state number that grows (A > 0)?
template <int n> __device__ __forceinline__ bool wave_grows(const float (&A2)[n])
{
    bool grows = false;
#pragma unroll
    for (int i = 0; i < n; ++i) grows |= A2[i] > 0.f;
    return __any(grows);
}

// Numbers of AHEAD tokens on their way, as they lie in memory (a conversion here would wait for them).  Past the last token the last one
// is read again: no branch stands between the loads.
template <typename T, int AHEAD> struct Ahead {
    T raw[AHEAD];
    __device__ __forceinline__ void request(const void *base, int64_t at, int64_t stride, int t, int last)
    {
        const T *p = static_cast<const T *>(base) + at;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) raw[i] = p[(t + i < last ? t + i : last - 1) * stride];
    }
    __device__ __forceinline__ float operator[](int i) const { return Elem<T>::load(&raw[i]); }
};

// Tokens whose numbers are on their way: eight in the backward sums, of which two waves run on a SIMD (2 x 4 680 tokens of 2 240 channels 151 us, with four 186; the
// forward walk gains nothing).
constexpr int kScanAhead = 4, kScanBackAhead = 8;

// What the tokens of a segment add to a state of nothing, and the sum of their steps.  MARKS: the local state before each run too.  GRADS: and what
// they add to the gradient of the state that the segment begins from, sum_t C_t y'_t times the decays up to t (for A <= 0: the product of the decays then stays in
// range but for what is less than 2^-126 of C_t y'_t).
template <typename T, int n, bool MARKS, bool GRADS, bool GATE> __device__ __forceinline__ void scan_sum(const ScanArgs &a, const ScanPlace &at)
{
    constexpr int kAhead = MARKS ? kScanBackAhead : kScanAhead;
    float A2[n], h[n], along[n], g[n], steps = 0.f;
    load_rates<n>(a, at.channel, A2);
    const float bias = a.dt_bias ? a.dt_bias[at.channel] : 0.f;
#pragma unroll
    for (int i = 0; i < n; ++i) {
        h[i] = g[i] = 0.f;
        along[i] = 1.f;
    }
    const int64_t bc = at.b * a.sbc.b + at.group * a.sbc.h;
    Ahead<T, kAhead> u, dt, dy, z;
    auto request = [&](int t) {
        u.request(a.u, at.u, a.su.n, t, at.last);
        dt.request(a.dt, at.u, a.su.n, t, at.last);
        if (GRADS) dy.request(a.dy, at.y, a.sy.n, t, at.last);
        if (GRADS && GATE) z.request(a.z, at.z, a.sz.n, t, at.last);
    };
    request(at.first);
    Scalars<T, n> nB, nC;
    auto request_scalars = [&](int t) {
        nB.load(a.bm, bc + t * a.sbc.n);
        if (GRADS) nC.load(a.cm, bc + t * a.sbc.n);
    };
    request_scalars(at.first);
    auto token = [&](int t, float ut, float dtt, float v, float zt) {
        Scalars<T, n> B = nB, C = nC;
        B.arrive();
        if (GRADS) C.arrive();
        request_scalars(t + 1 < at.last ? t + 1 : t);
        __builtin_amdgcn_sched_barrier(0);                            // not behind the arithmetic
        const float D = softplus(dtt + bias), x = D * ut;
        steps += D;
        if (GRADS && GATE) v *= silu(zt);
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float decay = __builtin_amdgcn_exp2f(D * A2[i]);
            h[i] = __builtin_fmaf(decay, h[i], x * B[i]);
            if (GRADS) {
                along[i] *= decay;
                g[i] = __builtin_fmaf(along[i], C[i] * v, g[i]);
            }
        }
    };
    auto mark = [&](int t) {
        if (!MARKS || t == at.first || t >= at.last || !at.mine) return;
        const int64_t mark = (int64_t)at.b * a.runs + t / kScanRun;
#pragma unroll
        for (int i = 0; i < n; ++i) a.marks[(mark * n + i) * a.channels + at.channel] = h[i];
        a.mark_steps[mark * a.channels + at.channel] = steps;
    };
    int t = at.first;
    for (; t + kAhead <= at.last; t += kAhead) {
        const Ahead<T, kAhead> u0 = u, dt0 = dt, dy0 = dy, z0 = z;
        request(t + kAhead);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (k % kScanRun == 0) mark(t + k);
            token(t + k, u0[k], dt0[k], GRADS ? dy0[k] : 0.f, GRADS && GATE ? z0[k] : 0.f);
        }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
        if (k % kScanRun == 0) mark(t + k);
        if (t + k < at.last) token(t + k, u[k], dt[k], GRADS ? dy[k] : 0.f, GRADS && GATE ? z[k] : 0.f);
    }
    if (!at.mine) return;
#pragma unroll
    for (int i = 0; i < n; ++i) {
        a.states[(at.slot(a) * n + i) * a.channels + at.channel] = h[i];
        if (GRADS) a.grads[(at.slot(a) * n + i) * a.channels + at.channel] = g[i];
    }
    a.steps[at.slot(a) * a.channels + at.channel] = steps;
}

template <typename T, int n> __global__ __launch_bounds__(kScanWave) void scan_sums(ScanArgs a)
{
    // (the last segment's sum is not needed)
    const uint32_t per_b = (uint32_t)a.blocks * (a.segments - 1), b = blockIdx.x / per_b;
    const ScanPlace at(a, b * (uint32_t)a.blocks * a.segments + (blockIdx.x - b * per_b));
    if (at.first >= at.length) return;
    scan_sum<T, n, false, false, false>(a, at);
}

// The states that the segments begin from, in place of what the segments before add; backwards (BACK) the gradients that arrive at their ends.
// A workgroup is 64 state numbers of one sequence by RUNS runs of SPAN segments: every thread fetches its run at once and adds it up, the runs are
// joined through LDS, and the thread goes over its run again.  (One after the other, 32 segments fetched at a time, 498 segments of 3 200 numbers took
// 33 us and 117 of 35 840 15.5.)
template <int n, int RUNS, int SPAN, bool BACK> __device__ __forceinline__ void scan_state(const ScanArgs &a, int block)
{
    __shared__ float sums[RUNS][64], ends[RUNS][64];
    const int tiles = (a.channels * n + 63) / 64, b = block / tiles, lane = threadIdx.x % 64, run = threadIdx.x / 64;
    const int last = a.channels * n - 1, mine = (block - b * tiles) * 64 + lane, at = mine < last ? mine : last;
    const int i = at / a.channels, c = at - i * a.channels;
    const float A2 = a.A[(int64_t)c * n + i] * kLog2E;
    const float *from = BACK ? a.ds_out : a.s_in;
    const int64_t stride = (int64_t)n * a.channels;
    float *slots = (BACK ? a.grads : a.states) + (int64_t)b * a.segments * stride;
    const float *steps = a.steps + (int64_t)b * a.segments * a.channels;
    const int length = held_length(a.lengths, b, a.N), used = length ? (length - 1) / a.per_segment + 1 : 1;
    float add[SPAN], sum[SPAN], total = 0.f, s = 0.f;
    auto segment = [&](int k) { return BACK ? used - 1 - run * SPAN - k : run * SPAN + k; };
#pragma unroll
    for (int k = 0; k < SPAN; ++k) {
        int seg = segment(k);                                         // the walk's last segment hands nothing on: any other is read in its place
        if (BACK) seg = seg > 0 ? seg : used - 1;
        else seg = seg + 1 < used ? seg : 0;
        add[k] = (slots + seg * stride)[at];
        sum[k] = (steps + (int64_t)seg * a.channels)[c];
    }
#pragma unroll
    for (int k = 0; k < SPAN; ++k)
        if (run * SPAN + k + 1 < used) {
            s = carried(A2, sum[k], s, add[k]);
            total += sum[k];
        }
    sums[run][lane] = total;
    ends[run][lane] = s;
    __syncthreads();
    s = from ? from[((int64_t)b * a.channels + c) * n + i] : 0.f;
    for (int r = 0; r < run; ++r) s = carried(A2, sums[r][lane], s, ends[r][lane]);
#pragma unroll
    for (int k = 0; k < SPAN; ++k)
        if (run * SPAN + k < used) {
            if (mine <= last) (slots + segment(k) * stride)[at] = s;
            s = carried(A2, sum[k], s, add[k]);
        }
}
template <int n, int RUNS, int SPAN> __global__ __launch_bounds__(64 * RUNS) void scan_states(ScanArgs a)
{
    scan_state<n, RUNS, SPAN, false>(a, (int)blockIdx.x);
}

template <typename T, int n, bool GATE> __global__ __launch_bounds__(kScanWave) void scan_walk(ScanArgs a)
{
    const ScanPlace at(a, blockIdx.x);
    if (at.first >= at.length && at.segment > 0) return;
    float A2[n], h[n];
    load_rates<n>(a, at.channel, A2);
    const float bias = a.dt_bias ? a.dt_bias[at.channel] : 0.f, skip = a.skip ? a.skip[at.channel] : 0.f;
    if (a.segments == 1) load_state<n>(a.s_in, (int64_t)at.b * a.channels + at.channel, h);
    else
#pragma unroll
        for (int i = 0; i < n; ++i) h[i] = a.states[(at.slot(a) * n + i) * a.channels + at.channel];
    const int64_t bc = at.b * a.sbc.b + at.group * a.sbc.h;
    T *y = static_cast<T *>(a.y) + at.y;
    Ahead<T, kScanAhead> u, dt, z;
    auto request = [&](int t) {
        u.request(a.u, at.u, a.su.n, t, at.last);
        dt.request(a.dt, at.u, a.su.n, t, at.last);
        if (GATE) z.request(a.z, at.z, a.sz.n, t, at.last);
    };
    Scalars<T, n> nB, nC;
    auto request_scalars = [&](int t) {
        nB.load(a.bm, bc + t * a.sbc.n);
        nC.load(a.cm, bc + t * a.sbc.n);
        __builtin_amdgcn_sched_barrier(0);                            // not behind the arithmetic
    };
    if (at.first < at.last) {
        request(at.first);
        request_scalars(at.first);
    }
    auto token = [&](int t, float ut, float dtt, float zt) {
        Scalars<T, n> B = nB, C = nC;
        B.arrive();
        C.arrive();
        request_scalars(t + 1 < at.last ? t + 1 : t);
        const float D = softplus(dtt + bias), x = D * ut;
        float out = skip * ut;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            h[i] = __builtin_fmaf(__builtin_amdgcn_exp2f(D * A2[i]), h[i], x * B[i]);
            out = __builtin_fmaf(C[i], h[i], out);
        }
        if (GATE) out *= silu(zt);
        if (at.mine) Elem<T>::store(y + t * a.sy.n, out);
    };
    int t = at.first;
    for (; t + kScanAhead <= at.last; t += kScanAhead) {
        const Ahead<T, kScanAhead> u0 = u, dt0 = dt, z0 = z;
        request(t + kScanAhead);
#pragma unroll
        for (int k = 0; k < kScanAhead; ++k) token(t + k, u0[k], dt0[k], GATE ? z0[k] : 0.f);
    }
#pragma unroll
    for (int k = 0; k < kScanAhead; ++k)
        if (t + k < at.last) token(t + k, u[k], dt[k], GATE ? z[k] : 0.f);
    if (a.s_out && at.mine && at.last == at.length) store_state<n>(a.s_out, (int64_t)at.b * a.channels + at.channel, h);
}

}  // namespace sv

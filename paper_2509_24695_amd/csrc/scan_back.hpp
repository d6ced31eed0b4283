// The selective scan's backward pass.  With y' = dy silu(z) and g_t = C_t y'_t + exp(D_{t+1} A) g_{t+1}, token by token from the end:
//
//   dC = sum_c y' h_t,  dB = sum_c g D u,  e = sum_i g B,  p = g exp(D A) h_{t-1},  dD = sum_i A p + u e,  du = D e + skip y',
//   ddt = dD sigmoid(dt + bias),  dz = dy (sum_i C h_t + skip u) silu'(z),  dA = sum_t D p,  dskip = sum_t y' u
//
// Cut into segments like the forward pass, with gradients handed on from segment to segment the same way from the end.  The states are
// needed from the last to the first: scan_back_sums leaves the local state before every run of four tokens, a wave adds what the
// segment's first state has become by then, walks the run forwards with its states in registers, and then backwards.  The sums over channels (dB, dC)
// go through the wave by exchanges that halve the number of values a lane holds with every step: 2 n values cost little more than 2 n additions.
//
// Bound by the vector unit: some 390 instructions a token and channel in scan_back_walk.  Runs of four tokens, with their decays (and what the segment begins
// from) in LDS, 20 KB a wave, keep a wave below 256 registers, so that two run on a SIMD (one alone reaches half of its rate).  The next run's numbers and mark
// are on their way during a run's first token, which comes last.  2 x 4 680 tokens of 2 240 channels, n = 16, bf16: 467 to 475 us, sums 151, states 12, walk 323 to 334, fold 12;
// with decays worked out again and marks fetched when they were needed the walk took 358, with runs of eight tokens and one wave 545.
#pragma once

#include "scan.hpp"

namespace sv {

// A segment's two sums can be had in one walk forwards, with the decays and the softplus of both worked out once; the gradients' is then of the decays multiplied up.
// It pays with a gate (2 x 4 680 tokens of 2 240 channels bf16 146 us, in a walk each 170; fp32 170 and 181) and at n = 8 (83 and 91 without a gate);
// without one, n = 16, a walk each is as fast or faster (bf16 145 and 141, fp32, whose B and C take all scalar registers, 176 and 146).  Where a state grows the
// product would leave fp32's range before the sum does: a wave with an A > 0 takes a walk each.
template <int n, bool GATE> constexpr bool kSumsTogether = GATE || n == 8;

// g = C dy of a segment's tokens from its last on, carried to before its first: what the segment adds to the gradient of the state it began from.
template <typename T, int n, bool GATE> __device__ __forceinline__ void scan_sum_back(const ScanArgs &a, const ScanPlace &at)
{
    float A2[n], g[n];
    load_rates<n>(a, at.channel, A2);
    const float bias = a.dt_bias ? a.dt_bias[at.channel] : 0.f;
#pragma unroll
    for (int i = 0; i < n; ++i) g[i] = 0.f;
    const int64_t bc = at.b * a.sbc.b + at.group * a.sbc.h;
    // tokens from the last: token k of the walk is last - 1 - k
    Ahead<T, kScanBackAhead> dy, dt, z;
    const int count = at.last - at.first;
    auto request = [&](int k) {
        const int64_t top = at.last - 1;
        dy.request(a.dy, at.y + top * a.sy.n, -a.sy.n, k, count);
        dt.request(a.dt, at.u + top * a.su.n, -a.su.n, k, count);
        if (GATE) z.request(a.z, at.z + top * a.sz.n, -a.sz.n, k, count);
    };
    request(0);
    Scalars<T, n> next;
    next.load(a.cm, bc + (at.last - 1) * a.sbc.n);
    auto token = [&](int k, float v, float dtt, float zt) {
        Scalars<T, n> C = next;
        C.arrive();
        next.load(a.cm, bc + (at.last - 1 - (k + 1 < count ? k + 1 : k)) * a.sbc.n);
        __builtin_amdgcn_sched_barrier(0);                            // not behind the arithmetic
        const float D = softplus(dtt + bias);
        if (GATE) v *= silu(zt);
#pragma unroll
        for (int i = 0; i < n; ++i) g[i] = __builtin_amdgcn_exp2f(D * A2[i]) * __builtin_fmaf(C[i], v, g[i]);
    };
    int k0 = 0;
    for (; k0 + kScanBackAhead <= count; k0 += kScanBackAhead) {
        const Ahead<T, kScanBackAhead> dy0 = dy, dt0 = dt, z0 = z;
        request(k0 + kScanBackAhead);
#pragma unroll
        for (int k = 0; k < kScanBackAhead; ++k) token(k0 + k, dy0[k], dt0[k], GATE ? z0[k] : 0.f);
    }
#pragma unroll
    for (int k = 0; k < kScanBackAhead; ++k)
        if (k0 + k < count) token(k0 + k, dy[k], dt[k], GATE ? z[k] : 0.f);
    if (!at.mine) return;
#pragma unroll
    for (int i = 0; i < n; ++i) a.grads[(at.slot(a) * n + i) * a.channels + at.channel] = g[i];
}

template <typename T, int n, bool GATE> __global__ __launch_bounds__(kScanWave) void scan_back_sums(ScanArgs a)
{
    if constexpr (kSumsTogether<n, GATE>) {
        const ScanPlace at(a, blockIdx.x);
        if (at.first >= at.length) return;
        float A2[n];
        load_rates<n>(a, at.channel, A2);
        if (!wave_grows(A2)) {
            scan_sum<T, n, true, true, GATE>(a, at);
        } else {
            scan_sum<T, n, true, false, false>(a, at);
            if (at.segment > 0) scan_sum_back<T, n, GATE>(a, at);
        }
    } else {
        const uint32_t half = gridDim.x / 2;
        const bool back = blockIdx.x >= half;
        const ScanPlace at(a, back ? blockIdx.x - half : blockIdx.x);
        if (at.first >= at.length) return;
        if (!back) scan_sum<T, n, true, false, false>(a, at);
        else if (at.segment > 0) scan_sum_back<T, n, GATE>(a, at);
    }
}
// A sequence of one segment: the marks alone.
template <typename T, int n> __global__ __launch_bounds__(kScanWave) void scan_back_marks(ScanArgs a)
{
    const ScanPlace at(a, blockIdx.x);
    if (at.first < at.length) scan_sum<T, n, true, false, false>(a, at);
}

template <int n, int RUNS, int SPAN> __global__ __launch_bounds__(64 * RUNS) void scan_back_states(ScanArgs a)
{
    const int half = (int)gridDim.x / 2;
    if ((int)blockIdx.x < half) scan_state<n, RUNS, SPAN, false>(a, (int)blockIdx.x);
    else scan_state<n, RUNS, SPAN, true>(a, (int)blockIdx.x - half);
}

// Sums over the wave of 2 n values, n of either kind, by exchanges: two lanes keep one of two values each and get the other's share of it.
// both(): the first exchange, between the halves of the wave, of value i of either kind.
__device__ __forceinline__ float wave_both(float first, float second)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(first), __float_as_uint(second), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}
// The rest: v[i] as wave_both left value i.  A lane ends with the sum of value wave_value<n>(lane), in v[0].
template <int n> __device__ __forceinline__ void wave_sums(float (&v)[n])
{
    static_assert(n == 8 || n == 16, "two or four lanes a value at the end");
    const int lane = threadIdx.x % kScanWave;
#pragma unroll
    for (int i = 0; i < n / 2; ++i) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[i]), __float_as_uint(v[i + n / 2]), false, false);
        v[i] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    auto step = [&](auto ctrl, int bit, float keep_low, float keep_high) {
        const bool high = lane & bit;
        const float own = high ? keep_high : keep_low, other = high ? keep_low : keep_high;
        return own + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, other), ctrl(), 0xf, 0xf, true));
    };
#pragma unroll
    for (int i = 0; i < n / 4; ++i) v[i] = step(std::integral_constant<int, 0x128>{}, 8, v[i], v[i + n / 4]);      // row_ror 8
#pragma unroll
    for (int i = 0; i < n / 8; ++i) v[i] = step(std::integral_constant<int, 0x141>{}, 4, v[i], v[i + n / 8]);      // row_half_mirror
    if constexpr (n == 16) v[0] = step(std::integral_constant<int, 0x4e>{}, 2, v[0], v[1]);                        // quad_perm 2,3,0,1
    else v[0] = dpp_add<0x4e>(v[0]);
    v[0] = dpp_add<0xb1>(v[0]);
}
// (the kind is the wave's half: values of the second kind follow those of the first)
template <int n> __device__ __forceinline__ int wave_value(int lane)
{
    int i = (lane >> 5 & 1) * n + (lane >> 4 & 1) * (n / 2) + (lane >> 3 & 1) * (n / 4) + (lane >> 2 & 1) * (n / 8);
    if (n == 16) i += lane >> 1 & 1;
    return i;
}

template <typename T, int n, bool GATE> __global__ __launch_bounds__(kScanWave, 2) void scan_back_walk(ScanArgs a)
{
    __shared__ f32x4 decays[kScanRun][n / 4][kScanWave], begins[n / 4][kScanWave];
    const ScanPlace at(a, blockIdx.x);
    const int lane = threadIdx.x;
    auto store_params = [&](const float (&dA)[n], float dbias, float dskip) {
        int channel = at.channel;                                     // (the address is worked out here: kept since the start it would take registers)
        asm volatile("" : "+v"(channel));
        float *params = a.params + at.slot(a) * (n + 2) * a.channels + channel;
#pragma unroll
        for (int i = 0; i < n; ++i) params[(int64_t)i * a.channels] = dA[i];
        params[(int64_t)n * a.channels] = dbias;
        params[(int64_t)(n + 1) * a.channels] = dskip;
    };
    if (at.first >= at.length && at.segment > 0) {
        const float none[n] = {};
        if (at.mine) store_params(none, 0.f, 0.f);
        return;
    }
    float A2[n], begin[n], g[n], dA[n], dbias = 0.f, dskip = 0.f;
    load_rates<n>(a, at.channel, A2);
    const bool grows = wave_grows(A2);
    const float bias = a.dt_bias ? a.dt_bias[at.channel] : 0.f, skip = a.skip ? a.skip[at.channel] : 0.f;
    if (a.segments == 1) {
        load_state<n>(a.s_in, (int64_t)at.b * a.channels + at.channel, begin);
        load_state<n>(a.ds_out, (int64_t)at.b * a.channels + at.channel, g);
    } else {
#pragma unroll
        for (int i = 0; i < n; ++i) {
            begin[i] = a.states[(at.slot(a) * n + i) * a.channels + at.channel];
            g[i] = a.grads[(at.slot(a) * n + i) * a.channels + at.channel];
        }
    }
#pragma unroll
    for (int q = 0; q < n / 4; ++q) begins[q][lane] = f32x4{begin[4 * q], begin[4 * q + 1], begin[4 * q + 2], begin[4 * q + 3]};
#pragma unroll
    for (int i = 0; i < n; ++i) dA[i] = 0.f;
    const int64_t bc = at.b * a.sbc.b + at.group * a.sbc.h;
    float *shared = a.shared + ((int64_t)at.b * a.blocks + at.block) * a.N * 2 * n + wave_value<n>(lane);
    const bool sums_mine = lane % (64 / (2 * n)) == 0;
    const int runs = (at.last - at.first + kScanRun - 1) / kScanRun;
    Ahead<T, kScanRun> u, dt, z, dy;
    auto request = [&](int t) {
        u.request(a.u, at.u, a.su.n, t, at.last);
        dt.request(a.dt, at.u, a.su.n, t, at.last);
        dy.request(a.dy, at.y, a.sy.n, t, at.last);
        if (GATE) z.request(a.z, at.z, a.sz.n, t, at.last);
    };
    // B and C of the token that comes after the present one: a run's tokens forwards, then backwards, then those of the run before
    Scalars<T, n> nB, nC;
    auto request_scalars = [&](int t) {
        nB.load(a.bm, bc + t * a.sbc.n);
        nC.load(a.cm, bc + t * a.sbc.n);
        __builtin_amdgcn_sched_barrier(0);                            // not behind the arithmetic
    };
    float mark[n], mark_steps;
    auto request_mark = [&](int t0) {
        const int64_t m = (int64_t)at.b * a.runs + t0 / kScanRun;
        mark_steps = a.mark_steps[m * a.channels + at.channel];
#pragma unroll
        for (int i = 0; i < n; ++i) mark[i] = a.marks[(m * n + i) * a.channels + at.channel];
    };
    auto run = [&](int t0, int count, auto whole) {
        const Ahead<T, kScanRun> u0 = u, dt0 = dt, z0 = z, dy0 = dy;
        const bool more = t0 > at.first;
        float h[kScanRun + 1][n], D[kScanRun], slope[kScanRun], raw[kScanRun];
        if (more && !grows) {
            // carried() for exponents below zero, in two halves: each has what fp32 can have beside the largest state
            const float half = 0.5f * mark_steps;
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const float part = __builtin_amdgcn_exp2f(A2[i] * half);
                h[0][i] = __builtin_fmaf(part, part * begins[i / 4][lane][i % 4], mark[i]);
            }
        } else if (more) {
#pragma unroll
            for (int i = 0; i < n; ++i) h[0][i] = carried(A2[i], mark_steps, begins[i / 4][lane][i % 4], mark[i]);
        } else {
#pragma unroll
            for (int i = 0; i < n; ++i) h[0][i] = begins[i / 4][lane][i % 4];
        }
#pragma unroll
        for (int k = 0; k < kScanRun; ++k) {
            if (!whole() && k >= count) break;
            Scalars<T, n> B = nB, C = nC;
            B.arrive();
            C.arrive();
            request_scalars(t0 + (k + 1 < count ? k + 1 : k));
            D[k] = softplus(dt0[k] + bias, slope[k]);
            const float x = D[k] * u0[k];
            raw[k] = skip * u0[k];
#pragma unroll
            for (int q = 0; q < n / 4; ++q) {
                f32x4 decay;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 4 * q + e;
                    decay[e] = __builtin_amdgcn_exp2f(D[k] * A2[i]);
                    h[k + 1][i] = __builtin_fmaf(decay[e], h[k][i], x * B[i]);
                    if (GATE) raw[k] = __builtin_fmaf(C[i], h[k + 1][i], raw[k]);
                }
                decays[k][q][lane] = decay;
            }
        }
#pragma unroll
        for (int k = kScanRun - 1; k >= 0; --k) {
            if (k == 0 && more) {                                     // (the later tokens' states are no longer needed: their registers do)
                request(t0 - kScanRun);
                if (t0 - kScanRun > at.first) request_mark(t0 - kScanRun);
            }
            if (!whole() && k >= count) continue;
            const int t = t0 + k;
            Scalars<T, n> B = nB, C = nC;
            B.arrive();
            C.arrive();
            request_scalars(k > 0 ? t - 1 : more ? t - kScanRun : t);
            float v = dy0[k];
            if (GATE) {
                const float s = sigmoid(z0[k]);
                if (at.mine) Elem<T>::store(static_cast<T *>(a.dz) + at.z + t * a.sz.n, v * raw[k] * silu_slope(z0[k], s));
                v *= z0[k] * s;
            }
            // lanes that double a channel add nothing to the sums over channels
            v = at.mine ? v : 0.f;
            const float x = at.mine ? D[k] * u0[k] : 0.f;
            float sums[n], e = 0.f, along = 0.f;
            f32x4 decay[n / 4];
#pragma unroll
            for (int q = 0; q < n / 4; ++q) decay[q] = decays[k][q][lane];
#pragma unroll
            for (int i = 0; i < n; ++i) {
                g[i] = __builtin_fmaf(C[i], v, g[i]);
                sums[i] = wave_both(g[i] * x, v * h[k + 1][i]);
                e = __builtin_fmaf(g[i], B[i], e);
                g[i] *= decay[i / 4][i % 4];
                const float p = g[i] * h[k][i];
                dA[i] = __builtin_fmaf(D[k], p, dA[i]);
                along = __builtin_fmaf(A2[i], p, along);
            }
            const float ddt = __builtin_fmaf(along, 1.f / kLog2E, u0[k] * e) * slope[k];
            dbias += ddt;
            dskip = __builtin_fmaf(v, u0[k], dskip);
            if (at.mine) {
                Elem<T>::store(static_cast<T *>(a.du) + at.u + t * a.su.n, __builtin_fmaf(D[k], e, skip * v));
                Elem<T>::store(static_cast<T *>(a.ddt) + at.u + t * a.su.n, ddt);
            }
            wave_sums<n>(sums);
            if (sums_mine) shared[(int64_t)t * 2 * n] = sums[0];
        }
    };
    if (runs) {
        int t0 = at.first + (runs - 1) * kScanRun;
        if (t0 > at.first) request_mark(t0);
        request(t0);
        request_scalars(t0);
        run(t0, at.last - t0, std::false_type{});
        for (t0 -= kScanRun; t0 >= at.first; t0 -= kScanRun) run(t0, kScanRun, std::true_type{});
    }
    if (!at.mine) return;
    store_params(dA, dbias, dskip);
    if (a.ds_in && at.segment == 0) {
        int channel = at.channel;
        asm volatile("" : "+v"(channel));
        store_state<n>(a.ds_in, (int64_t)at.b * a.channels + channel, g);
    }
}

// dB and dC: the blocks' sums over their channels, added up in order and rounded.  Behind these workgroups (`shared` of them) dA, ddt_bias and dskip:
// the segments' sums, added up in order.
template <typename T, int n> __global__ __launch_bounds__(256) void scan_back_fold(ScanArgs a, uint32_t shared)
{
    if (blockIdx.x < shared) {
        const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, per = (int64_t)a.N * 2 * n;
        const int64_t bg = id / per, at = id - bg * per;
        if (bg >= (int64_t)a.B * a.G) return;
        const int b = (int)(bg / a.G), group = (int)(bg % a.G), t = (int)(at / (2 * n)), i = (int)(at % (2 * n));
        if (t >= held_length(a.lengths, b, a.N)) return;
        const float *p = a.shared + ((int64_t)b * a.blocks + group * a.group_blocks) * per + at;
        float s = 0.f;
#pragma unroll 8
        for (int k = 0; k < a.group_blocks; ++k) s += p[k * per];
        T *out = static_cast<T *>(i < n ? a.db : a.dc) + b * a.sbc.b + group * a.sbc.h + t * a.sbc.n;
        Elem<T>::store(out + i % n, s);
        return;
    }
    const int64_t id = (int64_t)(blockIdx.x - shared) * 256 + threadIdx.x, per = (int64_t)a.channels * (n + 2);
    if (id >= per) return;
    const int i = (int)(id / a.channels), c = (int)(id % a.channels);
    float s = 0.f;
    const int64_t parts = (int64_t)a.B * a.segments;
#pragma unroll 8
    for (int64_t k = 0; k < parts; ++k) s += a.params[k * per + id];
    if (i < n) {
        if (a.dA) a.dA[(int64_t)c * n + i] = s;
    } else if (float *out = i == n ? a.ddt_bias : a.dskip) {
        out[c] = s;
    }
}

}  // namespace sv

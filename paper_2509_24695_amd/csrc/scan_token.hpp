// One token of the selective scan for each row of a batch, whose states lie in a pool.  A call moves the states, 2 n fp32 numbers a channel,
// and little else: four lanes (two at n = 8) hold a channel, four numbers of its state each, all of their loads in flight at once.
#pragma once

#include "scan.hpp"

namespace sv {

struct ScanTokenArgs {
    const void *u, *dt, *z, *bm, *cm;
    void *y;
    TokStrides su, sz, sbc, sy;
    const float *A, *dt_bias, *skip;
    const int32_t *slots;
    const float *s_in;
    float *s_out;
    int n_slots, d, channels, group_channels, tiles;
};

// UNITS: groups of 64 channels (128 at n = 8) that a workgroup has: one where there are few, two where the loads of one do not fill the memory's latency (187
// rows of 2 240 channels 12.9 us, with one 14.4, with four 13.8).
template <typename T, int n, bool GATE, int UNITS> __global__ __launch_bounds__(256) void scan_token(ScanTokenArgs a)
{
    constexpr int kLanes = n / 4, kChannels = 256 / kLanes;
    const int b = (int)(blockIdx.x / a.tiles), slot = a.slots ? a.slots[b] : b;
    if (slot < 0 || slot >= a.n_slots) return;
    const int part = threadIdx.x % kLanes, first = (int)(blockIdx.x % a.tiles) * (UNITS * kChannels) + (int)threadIdx.x / kLanes;
    f32x4 s[UNITS], A[UNITS];
    T Bt[UNITS][4], Ct[UNITS][4], ut[UNITS], dtt[UNITS], zt[UNITS];
    float bias[UNITS], skip[UNITS];
    int64_t state[UNITS], y[UNITS];
#pragma unroll
    for (int k = 0; k < UNITS; ++k) {
        const int at = first + k * kChannels, c = at < a.channels ? at : a.channels - 1, h = c / a.d, i = c - h * a.d, group = c / a.group_channels;
        state[k] = ((int64_t)slot * a.channels + c) * n + 4 * part;
        y[k] = b * a.sy.b + h * a.sy.h + i;
        s[k] = *reinterpret_cast<const f32x4 *>(a.s_in + state[k]);
        A[k] = *reinterpret_cast<const f32x4 *>(a.A + (int64_t)c * n + 4 * part);
        const int64_t bc = b * a.sbc.b + group * a.sbc.h + 4 * part;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            Bt[k][e] = static_cast<const T *>(a.bm)[bc + e];
            Ct[k][e] = static_cast<const T *>(a.cm)[bc + e];
        }
        ut[k] = static_cast<const T *>(a.u)[b * a.su.b + h * a.su.h + i];
        dtt[k] = static_cast<const T *>(a.dt)[b * a.su.b + h * a.su.h + i];
        if (GATE) zt[k] = static_cast<const T *>(a.z)[b * a.sz.b + h * a.sz.h + i];
        bias[k] = a.dt_bias ? a.dt_bias[c] : 0.f;
        skip[k] = a.skip ? a.skip[c] : 0.f;
    }
    if (slot_taken(a.slots, b, slot)) return;
#pragma unroll
    for (int k = 0; k < UNITS; ++k) {
        const float u = Elem<T>::load(&ut[k]), D = softplus(Elem<T>::load(&dtt[k]) + bias[k]), x = D * u;
        float out = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            s[k][e] = __builtin_fmaf(__builtin_amdgcn_exp2f(D * (A[k][e] * kLog2E)), s[k][e], x * Elem<T>::load(&Bt[k][e]));
            out = __builtin_fmaf(Elem<T>::load(&Ct[k][e]), s[k][e], out);
        }
        out = dpp_add<0xb1>(out);                                     // quad_perm 1,0,3,2
        if (kLanes == 4) out = dpp_add<0x4e>(out);                    // quad_perm 2,3,0,1
        if (first + k * kChannels < a.channels) {
            store16(a.s_out + state[k], s[k], a.s_out != a.s_in);
            if (part == 0) {
                out = __builtin_fmaf(skip[k], u, out);
                if (GATE) out *= silu(Elem<T>::load(&zt[k]));
                Elem<T>::store(static_cast<T *>(a.y) + y[k], out);
            }
        }
    }
}

}  // namespace sv

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

template <typename T, int n, bool GATE> __global__ __launch_bounds__(256) void scan_token(ScanTokenArgs a)
{
    constexpr int kLanes = n / 4;
    const int b = (int)(blockIdx.x / a.tiles), slot = a.slots ? a.slots[b] : b;
    if (slot < 0 || slot >= a.n_slots) return;
    const int part = threadIdx.x % kLanes, mine_at = (int)(blockIdx.x % a.tiles) * (int)(blockDim.x / kLanes) + (int)threadIdx.x / kLanes;
    const bool mine = mine_at < a.channels;
    const int c = mine ? mine_at : a.channels - 1, h = c / a.d, i = c - h * a.d, group = c / a.group_channels;
    const int64_t state = ((int64_t)slot * a.channels + c) * n + 4 * part, rate = (int64_t)c * n + 4 * part;
    f32x4 s = *reinterpret_cast<const f32x4 *>(a.s_in + state);
    const f32x4 A = *reinterpret_cast<const f32x4 *>(a.A + rate);
    const int64_t bc = b * a.sbc.b + group * a.sbc.h + 4 * part;
    float B[4], C[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        B[e] = Elem<T>::load(static_cast<const T *>(a.bm) + bc + e);
        C[e] = Elem<T>::load(static_cast<const T *>(a.cm) + bc + e);
    }
    const float u = Elem<T>::load(static_cast<const T *>(a.u) + b * a.su.b + h * a.su.h + i);
    const float dt = Elem<T>::load(static_cast<const T *>(a.dt) + b * a.su.b + h * a.su.h + i) + (a.dt_bias ? a.dt_bias[c] : 0.f);
    const float z = GATE ? Elem<T>::load(static_cast<const T *>(a.z) + b * a.sz.b + h * a.sz.h + i) : 0.f;
    const float skip = a.skip ? a.skip[c] : 0.f;
    if (slot_taken(a.slots, b, slot)) return;
    const float D = softplus(dt), x = D * u;
    float out = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        s[e] = __builtin_fmaf(__builtin_amdgcn_exp2f(D * (A[e] * kLog2E)), s[e], x * B[e]);
        out = __builtin_fmaf(C[e], s[e], out);
    }
    out = dpp_add<0xb1>(out);                                         // quad_perm 1,0,3,2
    if (kLanes == 4) out = dpp_add<0x4e>(out);                        // quad_perm 2,3,0,1
    if (!mine) return;
    *reinterpret_cast<f32x4 *>(a.s_out + state) = s;
    if (part) return;
    out = __builtin_fmaf(skip, u, out);
    if (GATE) out *= silu(z);
    Elem<T>::store(static_cast<T *>(a.y) + b * a.sy.b + h * a.sy.h + i, out);
}

}  // namespace sv

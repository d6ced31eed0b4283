// C ABI of the selective scan (include/sv_scan.h): argument checks and launches.
#include "../../include/sv_scan.h"

#include "desc_checks.hpp"
#include "scan.hpp"
#include "scan_back.hpp"
#include "scan_token.hpp"

namespace {

using namespace sv;

bool state_ok(int n) { return n == 8 || n == 16; }

// Checks u, z (if there is one), bc and y, which agree in B, N and dtype; u, z and y in H and d too; and what is shared among their groups.
sv_status check_tensors(const sv_tensor_desc *u, const void *Z, const sv_tensor_desc *z, const sv_tensor_desc *bc, const sv_tensor_desc *y, Shape *su,
                        Shape *sz, Shape *sbc, Shape *sy)
{
    sv_status rc = check_rows(u, su);
    if (rc != SV_OK) return rc;
    rc = check_rows(y, sy);
    if (rc != SV_OK) return rc;
    if (!same_shape(*su, *sy)) return SV_ERR_SHAPE;
    *sz = *su;
    if (Z) {
        rc = check_rows(z, sz);
        if (rc != SV_OK) return rc;
        if (!same_shape(*su, *sz)) return SV_ERR_SHAPE;
    }
    if (!bc) return SV_ERR_NULL;
    if (!state_ok(bc->d)) return SV_ERR_UNSUPPORTED;
    rc = check_rows(bc, sbc);
    if (rc != SV_OK) return rc;
    if (sbc->B != su->B || sbc->N != su->N || sbc->bf16 != su->bf16 || su->H % sbc->H) return SV_ERR_SHAPE;
    if ((int64_t)su->H * su->d >= (int64_t)1 << 27 || su->N > kMostTokens) return SV_ERR_SHAPE;
    return SV_OK;
}

size_t state_bytes(const Shape &u, int64_t entries, int n) { return (size_t)entries * u.H * u.d * n * sizeof(float); }

ScanArgs scan_args(const Shape &u, const Shape &z, const Shape &bc, const Shape &y, const ScanPlan &plan)
{
    ScanArgs a{};
    a.su = u.st; a.sz = z.st; a.sbc = bc.st; a.sy = y.st;
    a.B = u.B; a.H = u.H; a.N = u.N; a.d = u.d; a.G = bc.H;
    a.channels = u.H * u.d;
    a.group_channels = a.channels / a.G;
    a.group_blocks = (a.group_channels + kScanWave - 1) / kScanWave;
    a.blocks = plan.blocks;
    a.segments = plan.segments;
    a.per_segment = plan.per_segment;
    a.runs = (u.N + kScanRun - 1) / kScanRun;
    return a;
}

// Calls f(element, n, gate) with their constants.
template <typename F> void with_scan(bool bf16, int n, bool gate, F &&f)
{
    auto gated = [&](auto t, auto k) {
        if (gate) f(t, k, std::true_type{});
        else f(t, k, std::false_type{});
    };
    auto sized = [&](auto t) {
        if (n == 8) gated(t, std::integral_constant<int, 8>{});
        else gated(t, std::integral_constant<int, 16>{});
    };
    if (bf16) sized(uint16_t{});
    else sized(float{});
}

// Calls f(runs, span) with the form of scan_states for this many segments.
template <typename F> void with_span(int segments, F &&f)
{
    const std::integral_constant<int, 4> four;
    const std::integral_constant<int, 16> sixteen;
    if (segments <= 16) f(four, four);
    else if (segments <= 32) f(four, std::integral_constant<int, 8>{});
    else if (segments <= 64) f(sixteen, four);
    else if (segments <= 128) f(sixteen, std::integral_constant<int, 8>{});
    else if (segments <= 256) f(sixteen, sixteen);
    else f(sixteen, std::integral_constant<int, 32>{});
}
static_assert(kScanMostSegments <= 16 * 32, "segments of a sequence");

bool sizes_ok(int32_t B, int32_t H, int32_t N, int32_t d, int32_t n)
{
    return B > 0 && H > 0 && N > 0 && d > 0 && d % 4 == 0 && d <= kMostRowWidth && state_ok(n) && (int64_t)B * H <= kMostHeads;
}

}  // namespace

extern "C" size_t sv_selective_scan_workspace_bytes(int32_t B, int32_t H, int32_t n_tokens, int32_t d, int32_t n)
{
    if (!sizes_ok(B, H, n_tokens, d, n)) return 0;
    const int64_t channels = (int64_t)H * d;
    return (size_t)scan_slots(B, n_tokens, channels, kScanForwardWaves) * channels * (n + 1) * sizeof(float);
}

extern "C" size_t sv_selective_scan_backward_workspace_bytes(int32_t B, int32_t H, int32_t n_tokens, int32_t d, int32_t G, int32_t n)
{
    if (!sizes_ok(B, H, n_tokens, d, n) || G <= 0 || H % G) return 0;
    const int64_t channels = (int64_t)H * d;
    return (size_t)scan_backward_space(B, G, channels, n_tokens, n, scan_slots(B, n_tokens, channels, kScanBackwardWaves)).total * sizeof(float);
}

extern "C" sv_status sv_selective_scan(const void *U, const void *DT, const sv_tensor_desc *u, const void *Z, const sv_tensor_desc *z, const void *Bm,
                                       const void *Cm, const sv_tensor_desc *bc, const float *A, const float *dt_bias, const float *skip,
                                       const int32_t *lengths, const float *S_in, float *S_out, void *Y, const sv_tensor_desc *y, void *workspace,
                                       size_t workspace_bytes, void *stream)
{
    if (!U || !DT || !Bm || !Cm || !A || !Y || !workspace) return SV_ERR_NULL;
    Shape su, sz, sbc, sy;
    const sv_status rc = check_tensors(u, Z, z, bc, y, &su, &sz, &sbc, &sy);
    if (rc != SV_OK) return rc;
    if (!all_aligned({U, DT, Z, Bm, Cm, A, S_in, S_out, Y, workspace}) || !aligned4(dt_bias) || !aligned4(skip) || !aligned4(lengths)) return SV_ERR_ALIGN;
    const int n = sbc.d;
    if (Y == U || Y == DT || Y == Z || Y == Bm || Y == Cm || (S_in != S_out && overlaps(S_in, S_out, state_bytes(su, su.B, n)))) return SV_ERR_SHAPE;
    const ScanPlan plan = scan_plan(su.B, sbc.H, su.H / sbc.H * su.d, su.N, kScanForwardWaves);
    ScanArgs a = scan_args(su, sz, sbc, sy, plan);
    const int64_t states = (int64_t)a.B * a.segments * a.channels * n, waves = (int64_t)a.B * a.segments * a.blocks;
    if (a.segments > 1 && workspace_bytes < (size_t)(states + states / n) * sizeof(float)) return SV_ERR_WORKSPACE;
    const int64_t scan = (int64_t)a.B * (((int64_t)a.channels * n + 63) / 64);
    if (!grid_ok(waves, kScanWave) || (a.segments > 1 && !grid_ok(scan, 1024))) return SV_ERR_SHAPE;
    a.u = U; a.dt = DT; a.z = Z; a.bm = Bm; a.cm = Cm; a.y = Y;
    a.A = A; a.dt_bias = dt_bias; a.skip = skip; a.lengths = lengths;
    a.s_in = S_in; a.s_out = S_out;
    a.states = static_cast<float *>(workspace);
    a.steps = a.states + states;
    const auto hs = static_cast<hipStream_t>(stream);
    sv_status done = SV_OK;
    with_scan(su.bf16, n, Z != nullptr, [&](auto t, auto k, auto gate) {
        if (a.segments > 1) {
            scan_sums<decltype(t), k()><<<(unsigned)(waves / a.segments * (a.segments - 1)), kScanWave, 0, hs>>>(a);
            if ((done = launched()) != SV_OK) return;
            with_span(a.segments, [&](auto runs, auto span) { scan_states<k(), runs(), span()><<<(unsigned)scan, 64 * runs(), 0, hs>>>(a); });
            if ((done = launched()) != SV_OK) return;
        }
        scan_walk<decltype(t), k(), gate()><<<(unsigned)waves, kScanWave, 0, hs>>>(a);
        done = launched();
    });
    return done;
}

extern "C" sv_status sv_selective_scan_token(const void *U, const void *DT, const sv_tensor_desc *u, const void *Z, const sv_tensor_desc *z, const void *Bm,
                                             const void *Cm, const sv_tensor_desc *bc, const float *A, const float *dt_bias, const float *skip,
                                             const int32_t *slots, int32_t n_slots, const float *S_in, float *S_out, void *Y,
                                             const sv_tensor_desc *y, void *stream)
{
    if (!U || !DT || !Bm || !Cm || !A || !Y || !S_in || !S_out) return SV_ERR_NULL;
    Shape su, sz, sbc, sy;
    const sv_status rc = check_tensors(u, Z, z, bc, y, &su, &sz, &sbc, &sy);
    if (rc != SV_OK) return rc;
    if (su.N != 1 || n_slots <= 0 || (!slots && n_slots < su.B)) return SV_ERR_SHAPE;
    if (!all_aligned({U, DT, Z, Bm, Cm, A, S_in, S_out, Y}) || !aligned4(dt_bias) || !aligned4(skip) || !aligned4(slots)) return SV_ERR_ALIGN;
    const int n = sbc.d;
    if (Y == U || Y == DT || Y == Z || Y == Bm || Y == Cm || (S_in != S_out && overlaps(S_in, S_out, state_bytes(su, n_slots, n)))) return SV_ERR_SHAPE;
    ScanTokenArgs a{U, DT, Z, Bm, Cm, Y, su.st, sz.st, sbc.st, sy.st, A, dt_bias, skip, slots, S_in, S_out, n_slots, su.d, su.H * su.d,
                    su.H / sbc.H * su.d, 0};
    constexpr int kTokenThreads = 256, kFewTokens = 2048;             // workgroups of one unit
    const int per = kTokenThreads / (n / 4);
    const bool few = (int64_t)su.B * ((a.channels + per - 1) / per) <= kFewTokens;
    a.tiles = few ? (a.channels + per - 1) / per : (a.channels + 2 * per - 1) / (2 * per);
    if (!grid_ok((int64_t)su.B * a.tiles, kTokenThreads)) return SV_ERR_SHAPE;
    const unsigned grid = (unsigned)((int64_t)su.B * a.tiles);
    const auto hs = static_cast<hipStream_t>(stream);
    with_scan(su.bf16, n, Z != nullptr, [&](auto t, auto k, auto gate) {
        if (few) scan_token<decltype(t), k(), gate(), 1><<<grid, kTokenThreads, 0, hs>>>(a);
        else scan_token<decltype(t), k(), gate(), 2><<<grid, kTokenThreads, 0, hs>>>(a);
    });
    return launched();
}

extern "C" sv_status sv_selective_scan_backward(const void *U, const void *DT, const sv_tensor_desc *u, const void *Z, const sv_tensor_desc *z,
                                                const void *Bm, const void *Cm, const sv_tensor_desc *bc, const void *dY, const sv_tensor_desc *dy,
                                                const float *A, const float *dt_bias, const float *skip, const int32_t *lengths, const float *S_in,
                                                const float *dS_out, void *dU, void *dDT, void *dZ, void *dB, void *dC, float *dS_in, float *dA,
                                                float *ddt_bias, float *dskip, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!U || !DT || !Bm || !Cm || !A || !dY || !dU || !dDT || !dB || !dC || (Z && !dZ) || !workspace) return SV_ERR_NULL;
    Shape su, sz, sbc, sy;
    const sv_status rc = check_tensors(u, Z, z, bc, dy, &su, &sz, &sbc, &sy);
    if (rc != SV_OK) return rc;
    if (!all_aligned({U, DT, Z, Bm, Cm, dY, A, S_in, dS_out, dU, dDT, dZ, dB, dC, dS_in, dA, workspace}) || !aligned4(dt_bias) || !aligned4(skip) ||
        !aligned4(lengths) || !aligned4(ddt_bias) || !aligned4(dskip))
        return SV_ERR_ALIGN;
    const int n = sbc.d;
    const void *in[] = {U, DT, Z, Bm, Cm, dY, A, dt_bias, skip, S_in}, *out[] = {dU, dDT, Z ? dZ : nullptr, dB, dC, dA, ddt_bias, dskip, dS_in};
    for (size_t i = 0; i < sizeof(out) / sizeof(*out); ++i) {
        for (const void *p : in)
            if (out[i] && out[i] == p) return SV_ERR_SHAPE;
        for (size_t j = 0; j < i; ++j)
            if (out[i] && out[i] == out[j]) return SV_ERR_SHAPE;
    }
    const size_t held = state_bytes(su, su.B, n);
    if ((dS_in != dS_out && overlaps(dS_in, dS_out, held)) || overlaps(dS_in, S_in, held)) return SV_ERR_SHAPE;
    const ScanPlan plan = scan_plan(su.B, sbc.H, su.H / sbc.H * su.d, su.N, kScanBackwardWaves);
    ScanArgs a = scan_args(su, sz, sbc, sy, plan);
    const ScanBackwardSpace space = scan_backward_space(a.B, a.G, a.channels, a.N, n, (int64_t)a.B * a.segments);
    if (workspace_bytes < (size_t)space.total * sizeof(float)) return SV_ERR_WORKSPACE;
    const int64_t waves = (int64_t)a.B * a.segments * a.blocks, states = 2 * (int64_t)a.B * (((int64_t)a.channels * n + 63) / 64);
    const int64_t shared = ((int64_t)a.B * a.G * a.N * 2 * n + 255) / 256, params = dA || ddt_bias || dskip ? ((int64_t)a.channels * (n + 2) + 255) / 256 : 0;
    if (!grid_ok(2 * waves, kScanWave) || (a.segments > 1 && !grid_ok(states, 1024)) || !grid_ok(shared + params, 256)) return SV_ERR_SHAPE;
    a.u = U; a.dt = DT; a.z = Z; a.bm = Bm; a.cm = Cm; a.dy = dY;
    a.A = A; a.dt_bias = dt_bias; a.skip = skip; a.lengths = lengths;
    a.s_in = S_in; a.ds_out = dS_out;
    a.du = dU; a.ddt = dDT; a.dz = dZ; a.db = dB; a.dc = dC;
    a.ds_in = dS_in; a.dA = dA; a.ddt_bias = ddt_bias; a.dskip = dskip;
    float *p = static_cast<float *>(workspace);
    a.states = p; p += space.forward;
    a.grads = p; p += space.backward;
    a.steps = p; p += space.steps;
    a.marks = p; p += space.marks;
    a.mark_steps = p; p += space.mark_steps;
    a.shared = p; p += space.shared;
    a.params = p;
    const auto hs = static_cast<hipStream_t>(stream);
    sv_status done = SV_OK;
    with_scan(su.bf16, n, Z != nullptr, [&](auto t, auto k, auto gate) {
        using T = decltype(t);
        if (a.segments > 1) scan_back_sums<T, k(), gate()><<<(unsigned)(kSumsTogether<k(), gate()> ? waves : 2 * waves), kScanWave, 0, hs>>>(a);
        else scan_back_marks<T, k()><<<(unsigned)waves, kScanWave, 0, hs>>>(a);
        if ((done = launched()) != SV_OK) return;
        if (a.segments > 1) {
            with_span(a.segments, [&](auto runs, auto span) { scan_back_states<k(), runs(), span()><<<(unsigned)states, 64 * runs(), 0, hs>>>(a); });
            if ((done = launched()) != SV_OK) return;
        }
        scan_back_walk<T, k(), gate()><<<(unsigned)waves, kScanWave, 0, hs>>>(a);
        if ((done = launched()) != SV_OK) return;
        scan_back_fold<T, k()><<<(unsigned)(shared + params), 256, 0, hs>>>(a, (uint32_t)shared);
        done = launched();
    });
    return done;
}

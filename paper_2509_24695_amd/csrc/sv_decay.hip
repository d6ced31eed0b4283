// C ABI of decayed causal linear attention (include/sv_decay.h): argument checks and launches.
#include "../../include/sv_decay.h"

#include <math.h>

#include "decay_token.hpp"
#include "decay_walk.hpp"
#include "desc_checks.hpp"
#include "layout_rules.hpp"

namespace {

using namespace sv;

constexpr int kBackwardWalks = 3;              // dq, dv and dk, in one launch

// Checks `qkv` and `o`, which must agree in everything but their strides.
sv_status check_pair(const sv_tensor_desc *qkv, const sv_tensor_desc *o, Shape *x, Shape *y)
{
    sv_status rc = check_desc(qkv, x, false, kMostHeads);
    if (rc != SV_OK) return rc;
    rc = check_desc(o, y, false, kMostHeads);
    if (rc != SV_OK) return rc;
    if (qkv->B != o->B || qkv->H != o->H || qkv->N != o->N || qkv->d != o->d || qkv->dtype != o->dtype) return SV_ERR_SHAPE;
    for (const Shape *s : {x, y})
        if (s->st.n > (((int64_t)1 << 31) - 1) / (64 * s->elem_bytes)) return SV_ERR_UNSUPPORTED;
    return SV_OK;
}

DecayPlan plan_of(int64_t BH, int n_tokens, int d, bool bf16, int walks) { return decay_plan(BH, n_tokens, d, bf16 ? kDecayChunkBf16 : kDecayChunkF32, walks); }

size_t slots_bytes(int64_t BH, int n_tokens, int d, int walks)
{
    return (size_t)decay_slots(BH, n_tokens, d, walks) * d * d * sizeof(float);
}

bool sizes_ok(int32_t B, int32_t H, int32_t N, int32_t d)
{
    return B > 0 && H > 0 && N > 0 && head_dim_ok(d) && (int64_t)B * H <= kMostHeads;
}

// Sums, scan and walk: `sums` holds the problems whose states the walks of `walks` begin from (the same slots).
template <typename T, int D> sv_status run_walk(WalkArgs sums, const WalkArgs &walks, hipStream_t stream)
{
    using W = WalkShape<T, D>;
    const int64_t BH = (int64_t)walks.B * walks.H;
    // (the sums are fewer; a scan has D * D / 4 lanes a head and problem, and is there only where heads are few)
    if (!grid_ok(walks.problems * BH * walks.segments + 64, W::kWalkThreads)) return SV_ERR_SHAPE;
    if (walks.segments > 1) {
        decay_sums<T, D><<<decay_grid(sums.problems * BH * (walks.segments - 1), walks.together), W::kWalkThreads, 0, stream>>>(sums);
        if (launched() != SV_OK) return SV_ERR_LAUNCH;
        decay_scan<T, D><<<(unsigned)(sums.problems * BH * ((D * D / 4 + 255) / 256)), 256, 0, stream>>>(sums);
        if (launched() != SV_OK) return SV_ERR_LAUNCH;
    }
    const unsigned grid = decay_grid(walks.problems * BH * walks.segments, walks.together);
    if (decay_past_caches(BH, walks.N, D, (int)sizeof(T), walks.problems, walks.together > 1))
        decay_walk<T, D, true><<<grid, W::kWalkThreads, 0, stream>>>(walks);
    else
        decay_walk<T, D, false><<<grid, W::kWalkThreads, 0, stream>>>(walks);
    return launched();
}

sv_status run_walk(bool bf16, int d, const WalkArgs &sums, const WalkArgs &walks, void *stream)
{
    sv_status rc = SV_OK;
    const auto hs = static_cast<hipStream_t>(stream);
    with_head_dim(d, [&](auto D) { rc = bf16 ? run_walk<uint16_t, D()>(sums, walks, hs) : run_walk<float, D()>(sums, walks, hs); });
    return rc;
}

WalkArgs walk_args(const Shape &s, const float *log_decay, const int32_t *lengths, const DecayPlan &plan, int problems)
{
    WalkArgs a{};
    a.log_decay = log_decay;
    a.lengths = lengths;
    a.B = s.B;
    a.H = s.H;
    a.N = s.N;
    a.segments = plan.segments;
    a.per_segment = plan.per_segment;
    a.problems = problems;
    // four neighbouring heads that share lines on one die (20 heads of 32 760 tokens of 112 247 us, dealt singly 249; backward of 2 x 20 heads of
    // 14 040 446 and 454)
    a.together = TokenLayout{s.BH, s.H, s.d, s.elem_bytes, s.st.h, s.st.n}.shares_lines() ? 4 : 1;
    return a;
}

}  // namespace

extern "C" size_t sv_decay_linattn_workspace_bytes(int32_t B, int32_t H, int32_t n_tokens, int32_t d)
{
    return sizes_ok(B, H, n_tokens, d) ? slots_bytes((int64_t)B * H, n_tokens, d, 1) : 0;
}

extern "C" size_t sv_decay_linattn_backward_workspace_bytes(int32_t B, int32_t H, int32_t n_tokens, int32_t d)
{
    return sizes_ok(B, H, n_tokens, d) ? 2 * slots_bytes((int64_t)B * H, n_tokens, d, kBackwardWalks) : 0;
}

extern "C" sv_status sv_decay_linattn(const void *Q, const void *K, const void *V, const sv_tensor_desc *qkv, const float *log_decay,
                                      const int32_t *lengths, float scale, const float *S_in, float *S_out, void *O, const sv_tensor_desc *o,
                                      void *workspace, size_t workspace_bytes, void *stream)
{
    if (!Q || !K || !V || !O || !log_decay || !workspace) return SV_ERR_NULL;
    Shape x, y;
    const sv_status rc = check_pair(qkv, o, &x, &y);
    if (rc != SV_OK) return rc;
    if (!all_aligned({Q, K, V, O, S_in, S_out, workspace}) || !aligned4(log_decay) || !aligned4(lengths)) return SV_ERR_ALIGN;
    if (!isfinite(scale)) return SV_ERR_RANGE;
    const size_t states = (size_t)x.BH * x.d * x.d * sizeof(float);
    if (O == Q || O == K || O == V || (S_in != S_out && overlaps(S_in, S_out, states))) return SV_ERR_SHAPE;
    if (workspace_bytes < slots_bytes(x.BH, x.N, x.d, 1)) return SV_ERR_WORKSPACE;
    WalkArgs a = walk_args(x, log_decay, lengths, plan_of(x.BH, x.N, x.d, x.bf16, 1), 1);
    a.p[0] = WalkProblem{Q, K, V, O, x.st, x.st, x.st, y.st, S_in, S_out, static_cast<float *>(workspace), scale, scale, 1.f, 0, 0, 1};
    return run_walk(x.bf16, x.d, a, a, stream);
}

extern "C" sv_status sv_decay_linattn_backward(const void *Q, const void *K, const void *V, const sv_tensor_desc *qkv, const void *dO,
                                               const sv_tensor_desc *o, const float *log_decay, const int32_t *lengths, float scale,
                                               const float *S_in, const float *dS_out, void *dQ, void *dK, void *dV, float *dS_in,
                                               void *workspace, size_t workspace_bytes, void *stream)
{
    if (!Q || !K || !V || !dO || !log_decay || !dQ || !dK || !dV || !workspace) return SV_ERR_NULL;
    Shape x, y;
    const sv_status rc = check_pair(qkv, o, &x, &y);
    if (rc != SV_OK) return rc;
    if (!all_aligned({Q, K, V, dO, S_in, dS_out, dQ, dK, dV, dS_in, workspace}) || !aligned4(log_decay) || !aligned4(lengths)) return SV_ERR_ALIGN;
    if (!isfinite(scale)) return SV_ERR_RANGE;
    const size_t states = (size_t)x.BH * x.d * x.d * sizeof(float);
    for (const void *out : {dQ, dK, dV})
        if (out == Q || out == K || out == V || out == dO) return SV_ERR_SHAPE;
    if (dQ == dK || dQ == dV || dK == dV || overlaps(dS_in, dS_out, states) || overlaps(dS_in, S_in, states)) return SV_ERR_SHAPE;
    const size_t half = slots_bytes(x.BH, x.N, x.d, kBackwardWalks);
    if (workspace_bytes < 2 * half) return SV_ERR_WORKSPACE;
    float *states_fwd = static_cast<float *>(workspace), *states_back = states_fwd + half / sizeof(float);
    const DecayPlan plan = plan_of(x.BH, x.N, x.d, x.bf16, kBackwardWalks);
    WalkArgs sums = walk_args(x, log_decay, lengths, plan, 2), walks = walk_args(x, log_decay, lengths, plan, kBackwardWalks);
    sums.p[0] = WalkProblem{nullptr, K, V, nullptr, x.st, x.st, x.st, y.st, S_in, nullptr, states_fwd, 0.f, 0.f, 1.f, 0, 0, 0};
    sums.p[1] = WalkProblem{nullptr, Q, dO, nullptr, x.st, x.st, y.st, y.st, dS_out, nullptr, states_back, 0.f, 0.f, scale, 1, 0, 1};
    walks.p[0] = WalkProblem{dO, V, K, dQ, y.st, x.st, x.st, x.st, S_in, nullptr, states_fwd, scale, scale, 1.f, 0, 1, 0};
    walks.p[1] = WalkProblem{K, Q, dO, dV, x.st, x.st, y.st, x.st, dS_out, dS_in, states_back, 1.f, scale, scale, 1, 0, 1};
    walks.p[2] = WalkProblem{V, dO, Q, dK, x.st, y.st, x.st, x.st, dS_out, nullptr, states_back, 1.f, scale, scale, 1, 1, 0};
    return run_walk(x.bf16, x.d, sums, walks, stream);
}

extern "C" sv_status sv_decay_linattn_token(const void *Q, const void *K, const void *V, const sv_tensor_desc *qkv, const float *log_decay,
                                            const int32_t *slots, int32_t n_slots, float scale, const float *S_in, float *S_out, void *O,
                                            const sv_tensor_desc *o, void *stream)
{
    if (!Q || !K || !V || !O || !log_decay || !S_in || !S_out) return SV_ERR_NULL;
    Shape x, y;
    const sv_status rc = check_pair(qkv, o, &x, &y);
    if (rc != SV_OK) return rc;
    if (x.N != 1 || n_slots <= 0 || (!slots && n_slots < x.B)) return SV_ERR_SHAPE;
    if (!all_aligned({Q, K, V, O, S_in, S_out}) || !aligned4(log_decay) || !aligned4(slots)) return SV_ERR_ALIGN;
    if (!isfinite(scale)) return SV_ERR_RANGE;
    const size_t states = (size_t)n_slots * x.H * x.d * x.d * sizeof(float);
    if (O == Q || O == K || O == V || (S_in != S_out && overlaps(S_in, S_out, states))) return SV_ERR_SHAPE;
    if (!grid_ok(x.BH, 256)) return SV_ERR_SHAPE;
    TokenArgs a{Q, K, V, O, x.st.b, x.st.h, y.st.b, y.st.h, log_decay, slots, n_slots, x.B, x.H, scale, S_in, S_out};
    const auto hs = static_cast<hipStream_t>(stream);
    with_head_dim(x.d, [&](auto D) {
        auto go = [&](auto t, auto split) {
            using T = decltype(t);
            constexpr int kSplit = split();
            decay_token<T, D(), kSplit><<<(unsigned)((int64_t)x.BH * kSplit), TokenShape<D(), kSplit>::kTokThreads, 0, hs>>>(a);
        };
        const bool few = x.BH <= kFewTokenHeads;
        auto pick = [&](auto t) {
            if (few) go(t, std::integral_constant<int, 4>{});
            else go(t, std::integral_constant<int, 1>{});
        };
        if (x.bf16) pick(uint16_t{});
        else pick(float{});
    });
    return launched();
}

// C ABI of layer norm (include/sv_norm.h): argument checks and launches.
#include "../../include/sv_norm.h"

#include <math.h>

#include "desc_checks.hpp"
#include "norm.hpp"

namespace {

using namespace sv;

constexpr int64_t kMostHeads = 1 << 24;

sv_status check_rows(const sv_tensor_desc *t, Shape *s)
{
    const sv_status rc = check_desc(t, s, true, kMostHeads);
    if (rc != SV_OK) return rc;
    const int per = 16 / s->elem_bytes;
    if (s->d <= 0 || s->d % per || s->d > kNormMostWidth) return SV_ERR_UNSUPPORTED;
    return (int64_t)s->BH * s->N >= (int64_t)1 << 31 ? SV_ERR_SHAPE : SV_OK;
}

bool same_shape(const Shape &x, const Shape &y) { return x.B == y.B && x.H == y.H && x.N == y.N && x.d == y.d && x.bf16 == y.bf16; }
bool same_rows(const Shape &x, const Shape &y) { return x.st.b == y.st.b && x.st.h == y.st.h && x.st.n == y.st.n; }

// The rows of x's shape as groups (heads with parameters of their own, or one) of rows, walked in the order in which x lies in memory.
void set_rows(NormArgs &g, const Shape &x, const Shape &b, const Shape &c, int groups)
{
    NormAxis ax[3] = {{NormDivisor::of(x.N), x.st.n, b.st.n, c.st.n, 1},
                      {NormDivisor::of(x.H), x.st.h, b.st.h, c.st.h, x.N},
                      {NormDivisor::of(x.B), x.st.b, b.st.b, c.st.b, (int64_t)x.H * x.N}};
    if (groups > 1) {
        g.group_a = ax[1].a; g.group_b = ax[1].b; g.group_c = ax[1].c; g.group_stat = ax[1].stat;
        ax[1].extent = NormDivisor::of(1);
    }
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 3; ++j)
            if (ax[j].extent.extent > 1 && (ax[i].extent.extent == 1 || ax[j].a < ax[i].a)) { const NormAxis t = ax[i]; ax[i] = ax[j]; ax[j] = t; }
    for (int i = 0; i < 3; ++i) g.axis[i] = ax[i];
    g.groups = groups;
    g.rows = (int64_t)x.BH * x.N / groups;
    g.d = x.d;
}

// Is every row a run of whole 128-byte lines (given a tensor that begins with one)?
bool lines_whole(const Shape &s)
{
    const int64_t line = 128 / s.elem_bytes;
    return s.d % line == 0 && s.st.n % line == 0 && (s.H == 1 || s.st.h % line == 0) && (s.B == 1 || s.st.b % line == 0);
}

sv_status launched() { return hipGetLastError() == hipSuccess ? SV_OK : SV_ERR_LAUNCH; }

// Calls f(lanes, vecs) with the constants of a form.
template <typename F> void with_form(const NormForm &form, F &&f)
{
    auto is = [&](auto lanes, auto vecs) {
        if (form.lanes == lanes() && form.vecs == vecs()) f(lanes, vecs);
    };
    auto one = [&](auto lanes) { is(lanes, std::integral_constant<int, 1>{}); };
    auto two = [&](auto lanes) { is(lanes, std::integral_constant<int, 2>{}); };
    auto three = [&](auto lanes) { is(lanes, std::integral_constant<int, 3>{}); };
    auto four = [&](auto lanes) { is(lanes, std::integral_constant<int, 4>{}); };
    one(std::integral_constant<int, 4>{});
    one(std::integral_constant<int, 8>{});
    one(std::integral_constant<int, 16>{});
    one(std::integral_constant<int, 32>{});
    const std::integral_constant<int, 64> wave;
    one(wave), two(wave), three(wave), four(wave);
    is(wave, std::integral_constant<int, 5>{});
    is(wave, std::integral_constant<int, 6>{});
    const std::integral_constant<int, 128> waves;
    two(waves), three(waves), four(waves);
    three(std::integral_constant<int, 256>{});
    two(std::integral_constant<int, 512>{});
    two(std::integral_constant<int, 1024>{});
}

size_t partial_bytes(int64_t groups, int workgroups, int d) { return (size_t)groups * workgroups * 2 * d * sizeof(float); }

}  // namespace

extern "C" sv_status sv_layernorm(const void *X, const sv_tensor_desc *x, const float *weight, const float *bias, int32_t weight_heads, float eps,
                                  void *Y, const sv_tensor_desc *y, float *mean, float *rstd, void *stream)
{
    if (!X || !Y || (mean == nullptr) != (rstd == nullptr)) return SV_ERR_NULL;
    Shape in, out;
    sv_status rc = check_rows(x, &in);
    if (rc != SV_OK) return rc;
    rc = check_rows(y, &out);
    if (rc != SV_OK) return rc;
    if (!same_shape(in, out) || (weight_heads != 1 && weight_heads != in.H)) return SV_ERR_SHAPE;
    if (!aligned16(X) || !aligned16(Y) || !aligned16(weight) || !aligned16(bias) || !aligned16(mean) || !aligned16(rstd)) return SV_ERR_ALIGN;
    if (!isfinite(eps) || eps < 0.f) return SV_ERR_RANGE;
    if ((Y == X && !same_rows(in, out)) || (mean && mean == rstd)) return SV_ERR_SHAPE;
    NormArgs a{};
    a.x = X; a.y = Y; a.weight = weight; a.bias = bias; a.mean = mean; a.rstd = rstd; a.eps = eps;
    set_rows(a, in, out, out, weight_heads);
    const NormForm form = norm_form(in.d * in.elem_bytes / 16, false);
    a.whole_lines = lines_whole(out);
    a.workgroups = norm_workgroups(form, a.rows, a.groups, kNormForwardWgs);
    if (!grid_ok((int64_t)a.groups * a.workgroups, norm_threads(form))) return SV_ERR_SHAPE;
    const unsigned grid = (unsigned)((int64_t)a.groups * a.workgroups);
    const auto hs = static_cast<hipStream_t>(stream);
    with_form(form, [&](auto lanes, auto vecs) {
        if constexpr (lanes() != 128 || vecs() == 4) {                // forwards, narrower rows lie in one wave
            if constexpr (lanes() <= 512)                             // bf16 rows have no more pieces
                if (in.bf16) norm_rows<uint16_t, lanes(), vecs()><<<grid, NormWalk<lanes()>::kThreadsOf, 0, hs>>>(a);
            if (!in.bf16) norm_rows<float, lanes(), vecs()><<<grid, NormWalk<lanes()>::kThreadsOf, 0, hs>>>(a);
        }
    });
    return launched();
}

extern "C" size_t sv_layernorm_backward_workspace_bytes(int32_t B, int32_t H, int32_t n_tokens, int32_t d)
{
    if (B <= 0 || H <= 0 || n_tokens <= 0 || d <= 0 || d % 4 || d > kNormMostWidth || (int64_t)B * H > kMostHeads) return 0;
    // at most this many partial sums, whatever the type and the number of parameter rows
    const int64_t most = H > kNormMostBackwardWgs ? H : kNormMostBackwardWgs;
    return partial_bytes(1, (int)most, d);
}

extern "C" sv_status sv_layernorm_backward(const void *X, const sv_tensor_desc *x, const void *dY, const sv_tensor_desc *dy, const float *weight,
                                           int32_t weight_heads, const float *mean, const float *rstd, void *dX, const sv_tensor_desc *dx,
                                           float *dweight, float *dbias, void *workspace, size_t workspace_bytes, void *stream)
{
    const bool params = dweight || dbias;
    if (!X || !dY || !dX || !mean || !rstd || (params && !workspace)) return SV_ERR_NULL;
    Shape in, grad, out;
    sv_status rc = check_rows(x, &in);
    if (rc != SV_OK) return rc;
    rc = check_rows(dy, &grad);
    if (rc != SV_OK) return rc;
    rc = check_rows(dx, &out);
    if (rc != SV_OK) return rc;
    if (!same_shape(in, grad) || !same_shape(in, out) || (weight_heads != 1 && weight_heads != in.H)) return SV_ERR_SHAPE;
    for (const void *p : {X, dY, static_cast<const void *>(dX), static_cast<const void *>(weight), static_cast<const void *>(mean), static_cast<const void *>(rstd),
                          static_cast<const void *>(dweight), static_cast<const void *>(dbias), static_cast<const void *>(workspace)})
        if (!aligned16(p)) return SV_ERR_ALIGN;
    if (dX == X || (dX == dY && !same_rows(grad, out)) || (dweight && dweight == dbias) || (params && (dweight == weight || dbias == weight) && weight)) return SV_ERR_SHAPE;
    NormArgs a{};
    a.x = X; a.dy = dY; a.y = dX; a.weight = weight;
    a.mean = const_cast<float *>(mean); a.rstd = const_cast<float *>(rstd);
    a.dw = dweight; a.db = dbias;
    set_rows(a, in, grad, out, weight_heads);
    const NormForm form = norm_form(in.d * in.elem_bytes / 16, true);
    a.whole_lines = lines_whole(out);
    a.workgroups = norm_workgroups(form, a.rows, a.groups, norm_backward_wgs(in.d));
    if (params && workspace_bytes < partial_bytes(a.groups, a.workgroups, in.d)) return SV_ERR_WORKSPACE;
    a.partial = static_cast<float *>(workspace);
    const int64_t tiles = (in.d / 4 * 2 + 15) / 16;
    if (!grid_ok((int64_t)a.groups * a.workgroups, norm_threads(form)) || (params && !grid_ok(a.groups * tiles, 256))) return SV_ERR_SHAPE;
    const unsigned grid = (unsigned)((int64_t)a.groups * a.workgroups);
    const auto hs = static_cast<hipStream_t>(stream);
    with_form(form, [&](auto lanes, auto vecs) {
        auto go = [&](auto t, auto p) {
            norm_rows_backward<decltype(t), lanes(), vecs(), p()><<<grid, NormWalk<lanes()>::kThreadsOf, 0, hs>>>(a);
        };
        auto pick = [&](auto t) {
            if (params) go(t, std::true_type{});
            else go(t, std::false_type{});
        };
        if constexpr (lanes() != 64 || vecs() <= 3) {                 // backwards, wider rows lie in more lanes
            if constexpr (lanes() <= 512)
                if (in.bf16) pick(uint16_t{});
            if (!in.bf16) pick(float{});
        }
    });
    if (launched() != SV_OK) return SV_ERR_LAUNCH;
    if (params) {
        norm_fold<<<(unsigned)(a.groups * tiles), 256, 0, hs>>>(a);
        return launched();
    }
    return SV_OK;
}

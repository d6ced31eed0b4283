// C ABI of group norm (include/sv_norm.h): argument checks and launches.
#include "../../include/sv_norm.h"

#include <math.h>

#include "desc_checks.hpp"
#include "group.hpp"
#include "group_held.hpp"

namespace {

using namespace sv;

sv_status check_hidden(const sv_tensor_desc *t, int groups, Shape *s)
{
    const sv_status rc = check_rows(t, s);
    if (rc != SV_OK) return rc;
    return groups <= 0 || s->d % groups ? SV_ERR_SHAPE : SV_OK;
}

bool sizes_ok(int32_t B, int32_t H, int32_t N, int32_t d, int32_t groups)
{
    return B > 0 && H > 0 && N > 0 && d > 0 && d % 4 == 0 && d <= kMostRowWidth && groups > 0 && d % groups == 0 && (int64_t)B * H <= kMostHeads;
}

int64_t lines(int64_t bytes) { return (bytes + 255) / 256 * 256; }

GroupArgs group_args(const Shape &x, int groups, void *workspace)
{
    GroupArgs a{};
    a.sx = x.st;
    a.H = x.H; a.N = x.N; a.d = x.d; a.G = groups; a.width = x.d / groups;
    a.width_div = NormDivisor::of(a.width);
    a.BH = x.BH;
    a.level = static_cast<float *>(workspace);
    a.scale = a.level + a.BH * groups;
    a.sums = reinterpret_cast<double *>(static_cast<char *>(workspace) + lines(2 * a.BH * groups * (int64_t)sizeof(float)));
    return a;
}
// Where the sums of wide groups go: `pairs`, as many as group_slots has channels for.
void pair_args(GroupArgs &a, const GroupCut &c, int channels, double *pairs)
{
    a.tile_width = c.across * channels;
    a.sum_tiles = (int)c.tiles;
    a.per_tile = group_pairs(a.tile_width, a.width);
    a.pairs = a.width >= kWideGroup ? pairs : nullptr;
}
// The workgroups of a launch; 0: more than a launch has.
unsigned cut_args(GroupArgs &a, const GroupCut &c)
{
    a.across = c.across;
    a.tiles = (int)c.tiles;
    a.chunks = (int)c.chunks;
    a.rows = c.rows;
    const int64_t grid = a.BH * c.tiles * c.chunks;
    return grid_ok(grid, kGroupThreads) ? (unsigned)grid : 0;
}

template <typename F> void with_group(bool bf16, int silu, F &&f)
{
    auto act = [&](auto t) {
        if (silu) f(t, std::true_type{});
        else f(t, std::false_type{});
    };
    if (bf16) act(uint16_t{});
    else act(float{});
}

// Calls f(element, unit, rows) with the constants of a form of at most `most` words a thread: the rows it has room for are a quarter of `most`, half
// of it or all (in units of 16 bytes a quarter of that).
template <int MOST, typename F> void with_held(bool bf16, const HeldForm &form, F &&f)
{
    auto sized = [&](auto t, auto unit) {
        constexpr int kMost = unit() == 16 ? MOST / 4 : MOST;
        if (form.unit != unit()) return;
        if (form.rows <= kMost / 4) f(t, unit, std::integral_constant<int, kMost / 4>{});
        else if (form.rows <= kMost / 2) f(t, unit, std::integral_constant<int, kMost / 2>{});
        else f(t, unit, std::integral_constant<int, kMost>{});
    };
    const std::integral_constant<int, 2> two;
    const std::integral_constant<int, 4> four;
    const std::integral_constant<int, 16> sixteen;
    if (bf16) sized(uint16_t{}, two), sized(uint16_t{}, four), sized(uint16_t{}, sixteen);
    else sized(float{}, four), sized(float{}, sixteen);
}
// Gives a launch the form; its workgroups.
unsigned held_args(GroupArgs &a, const HeldForm &form, int elem_bytes)
{
    a.across = form.across;
    a.lines = form.lines;
    a.whole_lines = a.whole_lines && a.width * elem_bytes % 128 == 0;
    return (unsigned)held_grid(a.BH * a.G);
}

size_t workspace_bytes_of(int32_t B, int32_t H, int32_t N, int32_t d, int32_t groups, size_t number)
{
    if (!sizes_ok(B, H, N, d, groups)) return 0;
    const int64_t BH = (int64_t)B * H;
    return (size_t)lines(2 * BH * groups * (int64_t)sizeof(float)) + (size_t)group_slots(BH, N, d) * 2 * number;
}

}  // namespace

extern "C" size_t sv_groupnorm_workspace_bytes(int32_t B, int32_t H, int32_t n_tokens, int32_t d, int32_t groups)
{
    return workspace_bytes_of(B, H, n_tokens, d, groups, sizeof(double));
}

extern "C" size_t sv_groupnorm_backward_workspace_bytes(int32_t B, int32_t H, int32_t n_tokens, int32_t d, int32_t groups)
{
    return workspace_bytes_of(B, H, n_tokens, d, groups, 2 * sizeof(float));
}

extern "C" sv_status sv_groupnorm(const void *X, const sv_tensor_desc *x, const float *weight, const float *bias, int32_t groups, float eps, int32_t silu,
                                  void *Y, const sv_tensor_desc *y, float *mean, float *rstd, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!X || !Y || !workspace || (mean == nullptr) != (rstd == nullptr)) return SV_ERR_NULL;
    Shape in, out;
    sv_status rc = check_hidden(x, groups, &in);
    if (rc != SV_OK) return rc;
    rc = check_hidden(y, groups, &out);
    if (rc != SV_OK) return rc;
    if (!same_shape(in, out)) return SV_ERR_SHAPE;
    if (!all_aligned({X, Y, weight, bias, mean, rstd, workspace})) return SV_ERR_ALIGN;
    if (!isfinite(eps) || eps < 0.f || silu < 0 || silu > 1) return SV_ERR_RANGE;
    if ((Y == X && !same_rows(in, out)) || (mean && mean == rstd)) return SV_ERR_SHAPE;
    GroupArgs a = group_args(in, groups, workspace);
    const int pieces = in.d * in.elem_bytes / 16;
    const GroupCut sums = group_cut(a.BH, a.N, pieces, kGroupSumWgs), rows = group_cut(a.BH, a.N, pieces, kGroupApplyWgs);
    if (workspace_bytes < (size_t)(reinterpret_cast<char *>(a.sums) - static_cast<char *>(workspace)) + (size_t)a.BH * sums.chunks * 2 * a.d * sizeof(double))
        return SV_ERR_WORKSPACE;
    a.x = X; a.y = Y; a.sy = out.st;
    a.weight = weight; a.bias = bias; a.mean = mean; a.rstd = rstd; a.eps = eps;
    a.whole_lines = lines_whole(out);
    const auto hs = static_cast<hipStream_t>(stream);
    if (const HeldForm held = held_form(a.N, (int64_t)a.width * in.elem_bytes, kHeldForwardWords, a.BH * a.G); held.unit) {
        const unsigned grid = held_args(a, held, in.elem_bytes);
        with_held<kHeldForwardWords>(in.bf16, held, [&](auto t, auto unit, auto rows) {
            if (silu) group_held<decltype(t), unit(), rows(), true><<<grid, kHeldThreads, 0, hs>>>(a);
            else group_held<decltype(t), unit(), rows(), false><<<grid, kHeldThreads, 0, hs>>>(a);
        });
        return launched();
    }
    pair_args(a, sums, 16 / in.elem_bytes, a.sums);
    GroupArgs b = a;
    const unsigned sum_grid = cut_args(a, sums), row_grid = cut_args(b, rows);
    const int64_t fold = a.BH * a.G;
    if (!sum_grid || !row_grid || !grid_ok(fold, kGroupThreads)) return SV_ERR_SHAPE;
    a.sum_chunks = b.sum_chunks = (int)sums.chunks;
    auto sum = [&](auto t, auto wide) { group_sums<decltype(t), wide()><<<sum_grid, kGroupThreads, 0, hs>>>(a); };
    auto sum_of = [&](auto t) {
        if (a.pairs) sum(t, std::true_type{});
        else sum(t, std::false_type{});
    };
    if (in.bf16) sum_of(uint16_t{});
    else sum_of(float{});
    if (launched() != SV_OK) return SV_ERR_LAUNCH;
    if (a.pairs && sums.chunks * ((a.width - 1) / a.tile_width + 2) <= kFoldedPairs) {
        with_group(in.bf16, silu, [&](auto t, auto s) { group_apply<decltype(t), s(), true><<<row_grid, kGroupThreads, 0, hs>>>(b); });
        return launched();
    }
    group_fold<<<(unsigned)fold, kGroupThreads, 0, hs>>>(a);
    if (launched() != SV_OK) return SV_ERR_LAUNCH;
    with_group(in.bf16, silu, [&](auto t, auto s) { group_apply<decltype(t), s(), false><<<row_grid, kGroupThreads, 0, hs>>>(b); });
    return launched();
}

extern "C" sv_status sv_groupnorm_backward(const void *X, const sv_tensor_desc *x, const void *dY, const sv_tensor_desc *dy, const float *weight,
                                           const float *bias, int32_t groups, int32_t silu, const float *mean, const float *rstd, void *dX,
                                           const sv_tensor_desc *dx, float *dweight, float *dbias, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!X || !dY || !mean || !rstd || !dX || !workspace) return SV_ERR_NULL;
    Shape in, grad, out;
    sv_status rc = check_hidden(x, groups, &in);
    if (rc != SV_OK) return rc;
    rc = check_hidden(dy, groups, &grad);
    if (rc != SV_OK) return rc;
    rc = check_hidden(dx, groups, &out);
    if (rc != SV_OK) return rc;
    if (!same_shape(in, grad) || !same_shape(in, out)) return SV_ERR_SHAPE;
    if (!all_aligned({X, dY, weight, bias, mean, rstd, dX, dweight, dbias, workspace})) return SV_ERR_ALIGN;
    if (silu < 0 || silu > 1) return SV_ERR_RANGE;
    if (dX == X || (dX == dY && !same_rows(grad, out)) || (dweight && (dweight == dbias || dweight == weight)) || (dbias && dbias == bias)) return SV_ERR_SHAPE;
    GroupArgs a = group_args(in, groups, workspace);
    const int pieces = in.d / 4;
    const GroupCut sums = group_cut(a.BH, a.N, pieces, kGroupSumWgs), rows = group_cut(a.BH, a.N, pieces, kGroupApplyWgs);
    if (workspace_bytes < (size_t)(reinterpret_cast<char *>(a.sums) - static_cast<char *>(workspace)) + (size_t)a.BH * sums.chunks * 2 * a.d * 2 * sizeof(float))
        return SV_ERR_WORKSPACE;
    a.x = X; a.dy = dY; a.y = dX; a.sdy = grad.st; a.sy = out.st;
    a.weight = weight; a.bias = bias; a.dw = dweight; a.db = dbias;
    a.mean = const_cast<float *>(mean); a.rstd = const_cast<float *>(rstd);
    a.whole_lines = lines_whole(out);
    const auto hs = static_cast<hipStream_t>(stream);
    const bool params = dweight || dbias;
    const int64_t param_folds = params ? (2 * a.d + 15) / 16 : 0;
    if (const HeldForm held = held_form(a.N, (int64_t)a.width * in.elem_bytes, kHeldBackwardWords, a.BH * a.G); held.unit) {
        const unsigned grid = held_args(a, held, in.elem_bytes);
        with_held<kHeldBackwardWords>(in.bf16, held, [&](auto t, auto unit, auto rows) {
            auto go = [&](auto act, auto p) { group_held_back<decltype(t), unit(), rows(), act(), p()><<<grid, kHeldThreads, 0, hs>>>(a); };
            auto with = [&](auto act) {
                if (params) go(act, std::true_type{});
                else go(act, std::false_type{});
            };
            if (silu) with(std::true_type{});
            else with(std::false_type{});
        });
        if (launched() != SV_OK) return SV_ERR_LAUNCH;
        if (!params) return SV_OK;
        a.sum_chunks = 1;
        group_back_fold<<<(unsigned)param_folds, kGroupThreads, 0, hs>>>(a);
        return launched();
    }
    a.folds = a.BH * a.G;
    // (the first half of the sums' place is the channels', the second the groups')
    pair_args(a, sums, 4, a.sums + a.BH * sums.chunks * a.d);
    GroupArgs b = a;
    const unsigned sum_grid = cut_args(a, sums), row_grid = cut_args(b, rows);
    const int64_t fold = a.folds + param_folds;
    if (!sum_grid || !row_grid || !grid_ok(fold, kGroupThreads)) return SV_ERR_SHAPE;
    a.sum_chunks = b.sum_chunks = (int)sums.chunks;
    with_group(in.bf16, silu, [&](auto t, auto s) {
        auto go = [&](auto by_channel, auto wide) { group_back_sums<decltype(t), s(), by_channel(), wide()><<<sum_grid, kGroupThreads, 0, hs>>>(a); };
        if (!a.pairs) go(std::true_type{}, std::false_type{});
        else if (params) go(std::true_type{}, std::true_type{});
        else go(std::false_type{}, std::true_type{});
    });
    if (launched() != SV_OK) return SV_ERR_LAUNCH;
    group_back_fold<<<(unsigned)fold, kGroupThreads, 0, hs>>>(a);
    if (launched() != SV_OK) return SV_ERR_LAUNCH;
    with_group(in.bf16, silu, [&](auto t, auto s) { group_back_apply<decltype(t), s()><<<row_grid, kGroupThreads, 0, hs>>>(b); });
    return launched();
}

// C ABI of the short causal convolution (include/sv_conv.h): argument checks and launches.
#include "../../include/sv_conv.h"

#include "conv.hpp"
#include "desc_checks.hpp"

namespace {

using namespace sv;

constexpr int64_t kMostThreads = (int64_t)1 << 31;     // what NormDivisor divides

// Checks two descriptors that must agree in everything but their strides.
sv_status check_two(const sv_tensor_desc *x, const sv_tensor_desc *y, Shape *a, Shape *b)
{
    sv_status rc = check_rows(x, a);
    if (rc != SV_OK) return rc;
    rc = check_rows(y, b);
    if (rc != SV_OK) return rc;
    return same_shape(*a, *b) ? SV_OK : SV_ERR_SHAPE;
}

// `bytes`: of the channels that a thread has.
ConvArgs conv_args(const Shape &x, const float *weight, const float *bias, int silu, int bytes)
{
    ConvArgs a{};
    a.weight = weight; a.bias = bias;
    a.sx = x.st;
    a.B = x.B; a.H = x.H; a.N = x.N; a.d = x.d;
    a.silu = silu;
    const int per_head = x.d * x.elem_bytes / bytes;
    a.head_pieces = NormDivisor::of(per_head);
    a.pieces = NormDivisor::of(per_head * x.H);
    return a;
}

// What the kernels count in 32 bits: channels, and tokens a little past the last.
bool counts_ok(const Shape &x) { return (int64_t)x.H * x.d < (int64_t)1 << 28 && x.N <= kMostTokens; }

size_t cache_bytes(const Shape &x, int64_t entries, int taps) { return (size_t)entries * x.H * (taps - 1) * x.d * x.elem_bytes; }

// Calls f(element, taps, silu) with their constants.
template <typename F> void with_conv(bool bf16, int taps, int silu, F &&f)
{
    auto act = [&](auto t, auto k) {
        if (silu) f(t, k, std::true_type{});
        else f(t, k, std::false_type{});
    };
    auto tap = [&](auto t) {
        if (taps == 2) act(t, std::integral_constant<int, 2>{});
        else if (taps == 3) act(t, std::integral_constant<int, 3>{});
        else act(t, std::integral_constant<int, 4>{});
    };
    if (bf16) tap(uint16_t{});
    else tap(float{});
}

}  // namespace

extern "C" sv_status sv_causal_conv(const void *X, const sv_tensor_desc *x, const float *weight, const float *bias, int32_t taps, int32_t silu,
                                    const int32_t *lengths, const void *cache_in, void *cache_out, void *Y, const sv_tensor_desc *y, void *stream)
{
    if (!X || !weight || !Y) return SV_ERR_NULL;
    Shape in, out;
    const sv_status rc = check_two(x, y, &in, &out);
    if (rc != SV_OK) return rc;
    if (taps < 2 || taps > 4) return SV_ERR_UNSUPPORTED;
    if (silu < 0 || silu > 1) return SV_ERR_RANGE;
    if (!all_aligned({X, weight, bias, cache_in, cache_out, Y}) || !aligned4(lengths)) return SV_ERR_ALIGN;
    if (Y == X || (cache_in != cache_out && overlaps(cache_in, cache_out, cache_bytes(in, in.B, taps))) || cache_out == X || cache_out == Y) return SV_ERR_SHAPE;
    if (!counts_ok(in)) return SV_ERR_SHAPE;
    ConvArgs a = conv_args(in, weight, bias, silu, 16);
    a.x = X; a.y = Y; a.sy = out.st;
    a.lengths = lengths; a.cache_in = cache_in; a.cache_out = cache_out;
    a.whole_lines = lines_whole(out);
    a.run = conv_run((int64_t)in.B * in.N, (int)a.pieces.extent);
    a.runs = (int)(((int64_t)in.N + a.run - 1) / a.run);
    a.run_div = NormDivisor::of(a.runs);
    const int64_t threads = (int64_t)in.B * a.runs * a.pieces.extent;
    if (threads > kMostThreads - kConvThreads) return SV_ERR_SHAPE;
    const unsigned grid = (unsigned)((threads + kConvThreads - 1) / kConvThreads);
    const auto hs = static_cast<hipStream_t>(stream);
    with_conv(in.bf16, taps, silu, [&](auto t, auto k, auto s) { conv_rows<decltype(t), k(), s()><<<grid, kConvThreads, 0, hs>>>(a); });
    return launched();
}

extern "C" sv_status sv_causal_conv_token(const void *X, const sv_tensor_desc *x, const float *weight, const float *bias, int32_t taps, int32_t silu,
                                          const int32_t *slots, int32_t n_slots, const void *cache_in, void *cache_out, void *Y,
                                          const sv_tensor_desc *y, void *stream)
{
    if (!X || !weight || !Y || !cache_in || !cache_out) return SV_ERR_NULL;
    Shape in, out;
    const sv_status rc = check_two(x, y, &in, &out);
    if (rc != SV_OK) return rc;
    if (taps < 2 || taps > 4) return SV_ERR_UNSUPPORTED;
    if (silu < 0 || silu > 1) return SV_ERR_RANGE;
    if (in.N != 1 || n_slots <= 0 || (!slots && n_slots < in.B)) return SV_ERR_SHAPE;
    if (!all_aligned({X, weight, bias, cache_in, cache_out, Y}) || !aligned4(slots)) return SV_ERR_ALIGN;
    if (Y == X || (cache_in != cache_out && overlaps(cache_in, cache_out, cache_bytes(in, n_slots, taps))) || cache_out == X || cache_out == Y) return SV_ERR_SHAPE;
    if (!counts_ok(in)) return SV_ERR_SHAPE;
    ConvArgs a = conv_args(in, weight, bias, silu, 16);
    a.x = X; a.y = Y; a.sy = out.st;
    a.lengths = slots; a.n_slots = n_slots;
    a.cache_in = cache_in; a.cache_out = cache_out;
    const int pieces = (int)a.pieces.extent;
    a.runs = (pieces + kConvThreads - 1) / kConvThreads;              // workgroups of a row
    a.across = (pieces + a.runs - 1) / a.runs;
    const int threads = (a.across + 63) / 64 * 64;
    if (!grid_ok((int64_t)in.B * a.runs, threads)) return SV_ERR_SHAPE;
    const auto hs = static_cast<hipStream_t>(stream);
    with_conv(in.bf16, taps, silu, [&](auto t, auto k, auto s) { conv_token<decltype(t), k(), s()><<<(unsigned)(in.B * a.runs), threads, 0, hs>>>(a); });
    return launched();
}

extern "C" size_t sv_causal_conv_backward_workspace_bytes(int32_t B, int32_t H, int32_t n_tokens, int32_t d)
{
    if (B <= 0 || H <= 0 || n_tokens <= 0 || d <= 0 || d % 4 || d > kMostRowWidth || (int64_t)B * H > kMostHeads) return 0;
    return conv_workspace_floats(B, n_tokens, (int64_t)H * d) * sizeof(float);
}

extern "C" sv_status sv_causal_conv_backward(const void *X, const sv_tensor_desc *x, const void *dY, const sv_tensor_desc *dy, const float *weight,
                                             const float *bias, int32_t taps, int32_t silu, const int32_t *lengths, const void *cache_in,
                                             const void *dcache_out, void *dX, const sv_tensor_desc *dx, void *dcache_in, float *dweight,
                                             float *dbias, void *workspace, size_t workspace_bytes, void *stream)
{
    const bool params = dweight || dbias;
    if (!X || !dY || !weight || !dX || (params && !workspace)) return SV_ERR_NULL;
    Shape in, grad, out;
    sv_status rc = check_two(x, dy, &in, &grad);
    if (rc != SV_OK) return rc;
    rc = check_two(x, dx, &in, &out);
    if (rc != SV_OK) return rc;
    if (taps < 2 || taps > 4) return SV_ERR_UNSUPPORTED;
    if (silu < 0 || silu > 1) return SV_ERR_RANGE;
    if (!all_aligned({X, dY, weight, bias, cache_in, dcache_out, dX, dcache_in, dweight, dbias, workspace}) || !aligned4(lengths)) return SV_ERR_ALIGN;
    const size_t caches = cache_bytes(in, in.B, taps);
    if (dX == X || dX == dY || overlaps(dcache_in, dcache_out, caches) || overlaps(dcache_in, cache_in, caches) || dcache_in == X || dcache_in == dY ||
        dcache_in == dX || (dweight && (dweight == dbias || dweight == weight)) || (dbias && dbias == bias))
        return SV_ERR_SHAPE;
    if (!counts_ok(in)) return SV_ERR_SHAPE;
    ConvArgs a = conv_args(in, weight, bias, silu, 4 * in.elem_bytes);
    const ConvCut cut = conv_cut(in.B, in.N, a.pieces.extent);
    const int64_t channels = (int64_t)in.H * in.d, floats = channels * (taps + 1);
    if (params && workspace_bytes < (size_t)conv_partial_floats(in.B, cut.blocks, channels, taps) * sizeof(float)) return SV_ERR_WORKSPACE;
    const int64_t groups = in.B * cut.blocks * cut.tiles, fold = (floats / 4 + 15) / 16;
    if (!grid_ok(groups, kConvThreads) || groups >= (int64_t)1 << 31 || !grid_ok(fold, 256)) return SV_ERR_SHAPE;
    a.x = X; a.dy = dY; a.y = dX; a.sdy = grad.st; a.sy = out.st;
    a.lengths = lengths; a.cache_in = cache_in; a.dcache_out = dcache_out; a.cache_out = dcache_in;
    a.partial = static_cast<float *>(workspace);
    a.whole_lines = lines_whole(out);
    a.run = cut.run; a.runs = (int)cut.blocks; a.across = cut.across;
    const auto hs = static_cast<hipStream_t>(stream);
    with_conv(in.bf16, taps, silu, [&](auto t, auto k, auto s) {
        if (params) conv_rows_backward<decltype(t), k(), s(), true><<<(unsigned)groups, kConvThreads, 0, hs>>>(a);
        else conv_rows_backward<decltype(t), k(), s(), false><<<(unsigned)groups, kConvThreads, 0, hs>>>(a);
    });
    if (launched() != SV_OK) return SV_ERR_LAUNCH;
    if (!params) return SV_OK;
    const FoldArgs f{a.partial, in.B * cut.blocks, floats, channels * taps, dweight, dbias};
    fold_parts<<<(unsigned)fold, 256, 0, hs>>>(f);
    return launched();
}

// How a short causal convolution's tokens are dealt to threads.  Plain C++ (no device code), shared by the launchers and host-side tests.
#pragma once

#include <stdint.h>

#include "norm_plan.hpp"

namespace sv {

// Forwards a thread owns one 16-byte piece of the channels and walks a run of tokens; threads are numbered pieces first, then runs.  Sixteen tokens where that
// makes 1 024 threads a compute unit (32 760 tokens of 2 240 channels bf16 58.6 us, runs of 8 60.2, of 32 62.5), fewer in smaller calls.
constexpr int kConvThreads = 256;
inline int conv_run(int64_t BN, int pieces)
{
    for (int run = 16; run > 4; run /= 2)
        if (BN * pieces / run >= (int64_t)256 * 1024) return run;
    return 4;
}

// Backwards a workgroup is `across` pieces (at most 32, as many in every tile) by `down` runs of tokens, so that one partial sum of the parameters' gradients is left for all
// of its runs.  Runs as long as 2 048 workgroups allow (2 x 20 heads of up to 14 040 tokens of 112 80 us, with 1 024 88, with 4 096 86), of eight tokens at least (2 799 x 3
// tokens of 672 channels fp32 17 us, with four 26).
struct ConvCut {
    int across, down, run;             // run: tokens of a thread
    int64_t tiles, blocks;             // workgroups across the channels; workgroups along one sequence
};
constexpr int kConvLeastRun = 8, kConvMostRun = 64;
constexpr int64_t kConvBackwardWgs = 2048;
inline ConvCut conv_cut(int64_t B, int64_t N, int64_t pieces)
{
    ConvCut c{};
    c.tiles = (pieces + 31) / 32;
    c.across = (int)((pieces + c.tiles - 1) / c.tiles);
    c.down = kConvThreads / c.across;
    c.run = kConvLeastRun;
    while (c.run < kConvMostRun && B * ((N + (int64_t)c.down * c.run - 1) / ((int64_t)c.down * c.run)) * c.tiles > kConvBackwardWgs) c.run *= 2;
    c.blocks = (N + (int64_t)c.down * c.run - 1) / ((int64_t)c.down * c.run);
    return c;
}
// Partial sums of a call; and of the largest call with no more batches, tokens and channels: with more than kConvBackwardWgs workgroups runs are as long as they
// get, with fewer these leave at most as many sums of 256 channels.
inline int64_t conv_partial_floats(int64_t B, int64_t blocks, int64_t channels, int taps) { return B * blocks * channels * (taps + 1); }
inline int64_t conv_workspace_floats(int64_t B, int64_t N, int64_t channels)
{
    const int64_t shortest = B * ((N + 31) / 32) * channels, longest = B * ((N + 511) / 512) * channels;
    const int64_t most = longest > kConvBackwardWgs * 256 ? longest : kConvBackwardWgs * 256;
    return 5 * (shortest < most ? shortest : most);
}

}  // namespace sv

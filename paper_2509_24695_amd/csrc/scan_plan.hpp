// How a selective scan is cut up: waves of channels, segments of tokens.  Plain C++ (no device code), shared by the launchers and host-side
// tests.
#pragma once

#include <stdint.h>

namespace sv {

constexpr int kScanWave = 64;               // channels of a wave
constexpr int kScanRun = 4;                 // tokens whose states the backward pass holds at once: segments are multiples of it
constexpr int kScanShortest = 8;            // tokens of a segment, where there is more than one (64 tokens of 2 240 channels 16 us, with 32 33; backwards 33 and 70)

// A sequence is walked by `segments` waves per channel block, `per_segment` tokens each (the last fewer).
struct ScanPlan {
    int blocks;                             // waves across the channels of all groups
    int segments, per_segment;
};

// As many waves as run at once, forwards four on a SIMD, backwards two; forwards twice as many where segments are long enough for it (a state
// that is handed on costs 16 bytes of traffic a number): 32 760 tokens of 2 240 channels without a gate 490 us, with four 545; 8 190 tokens 181 and 168.
// Not where the sequences alone fill them by more than half: a first cut brings the sums with it (64, 100 and 117 sequences of 512 tokens of 2 240 channels
// 406, 504 and 508 us, in three, two and two segments 481, 673 and 771; of 1 560 tokens 1 223, 1 526 and 1 533, cut 1 347, 1 918 and 2 209).
constexpr int kScanMostSegments = 512, kScanLongSegment = 128;
constexpr int64_t kScanForwardWaves = 4096, kScanBackwardWaves = 2048;

inline int64_t scan_longest_chain(int64_t n_tokens)
{
    const int64_t shortest = (n_tokens + kScanShortest - 1) / kScanShortest;
    return shortest < kScanMostSegments ? shortest : kScanMostSegments;
}
inline int64_t scan_most_segments(int64_t B, int64_t n_tokens, int64_t blocks, int64_t waves)
{
    int64_t s = waves / (B * blocks), more = waves == kScanForwardWaves && s > 1 ? 2 * waves / (B * blocks) : 0;
    if (more > n_tokens / kScanLongSegment) more = n_tokens / kScanLongSegment;
    if (s < more) s = more;
    const int64_t longest = scan_longest_chain(n_tokens);
    return s < 1 ? 1 : s < longest ? s : longest;
}
inline ScanPlan scan_plan(int64_t B, int groups, int group_channels, int n_tokens, int64_t waves)
{
    ScanPlan p{};
    p.blocks = groups * ((group_channels + kScanWave - 1) / kScanWave);
    const int64_t s = scan_most_segments(B, n_tokens, p.blocks, waves);
    int64_t per = (n_tokens + s - 1) / s;
    if (s > 1 && per < kScanShortest) per = kScanShortest;
    per = (per + kScanRun - 1) / kScanRun * kScanRun;
    p.per_segment = (int)per;
    p.segments = (int)((n_tokens + per - 1) / per);
    return p;
}

// Segments of all sequences together in the largest call with no more batches and tokens and the same channels.
inline int64_t scan_slots(int64_t B, int64_t n_tokens, int64_t channels, int64_t waves)
{
    const int64_t blocks = (channels + kScanWave - 1) / kScanWave;
    const int64_t most = B * scan_longest_chain(n_tokens), full = 2 * waves / blocks > B ? 2 * waves / blocks : B;
    return most < full ? most : full;
}

// Floats of the backward pass's workspace, part by part.
struct ScanBackwardSpace {
    int64_t forward, backward, steps, marks, mark_steps, shared, params, total;
};
inline ScanBackwardSpace scan_backward_space(int64_t B, int64_t groups, int64_t channels, int64_t n_tokens, int n, int64_t slots)
{
    const int64_t runs = (n_tokens + kScanRun - 1) / kScanRun, blocks = groups * ((channels / groups + kScanWave - 1) / kScanWave);
    auto lines = [](int64_t floats) { return (floats + 63) / 64 * 64; };
    ScanBackwardSpace s{};
    s.forward = s.backward = lines(slots * channels * n);
    s.steps = lines(slots * channels);
    s.marks = lines(B * runs * channels * n);
    s.mark_steps = lines(B * runs * channels);
    s.shared = lines(B * blocks * n_tokens * 2 * n);
    s.params = lines(slots * channels * (n + 2));
    s.total = s.forward + s.backward + s.steps + s.marks + s.mark_steps + s.shared + s.params;
    return s;
}

}  // namespace sv

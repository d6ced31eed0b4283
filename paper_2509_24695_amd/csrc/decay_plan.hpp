// How a decayed linear-attention call is cut up: chunks of tokens, segments of chunks, workgroups.  Plain C++ (no device code), shared by
// the launcher, the kernels and host-side tests.
#pragma once

#include <stdint.h>

#include "tile_walk.hpp"

namespace sv {

constexpr int kMaxDecaySegments = 128;      // what decay_scan walks one after the other
constexpr int kDecayChunkBf16 = 64, kDecayChunkF32 = 32;

// A head's sequence of `chunks` chunks is walked by `segments` workgroups, `per_segment` chunks each (the last fewer).
struct DecayPlan {
    int chunks, segments, per_segment;
};

// As many workgroups as run at once, in all `walks` of a launch together: the walk is bound by what a wave waits for (its own products, LDS,
// the other waves), so a second round or fewer waves cost more than the partial states of shorter segments (32 heads, 4 680 tokens, us with
// half as many / these / one and a half times: d = 64 41.3 / 37.9 / 45.1, d = 128 74.8 / 71.1 / 81.8; d = 32, 128 heads of 4 096: 56.4 / 45.2 /
// 49.8; backward, all three walks with the forward call's number each: d = 64 72.7 against 64).  No segment is a single chunk.
inline DecayPlan decay_plan(int64_t BH, int n_tokens, int d, int chunk, int walks)
{
    DecayPlan p;
    p.chunks = (int)(((int64_t)n_tokens + chunk - 1) / chunk);
    const int64_t workgroups = (d <= 64 ? 1024 : 512) / walks;
    const int64_t wanted = workgroups / BH < 1 ? 1 : workgroups / BH;
    int64_t segments = wanted > kMaxDecaySegments ? kMaxDecaySegments : wanted;
    if (segments > (p.chunks + 1) / 2) segments = (p.chunks + 1) / 2;
    if (segments < 1) segments = 1;
    p.per_segment = (int)((p.chunks + segments - 1) / segments);
    p.segments = (p.chunks + p.per_segment - 1) / p.per_segment;
    return p;
}

// The chunks of one sequence of `length` tokens: whole ones at its end, so that every chunk's last row is a token and only the first
// chunk begins with `lead` rows of nothing.
struct DecayWalk {
    int chunks, lead;
    SV_HOST_DEVICE DecayWalk(int length, int chunk) : chunks((int)(((int64_t)length + chunk - 1) / chunk)), lead((int)((int64_t)chunks * chunk - length)) {}
};

// A launch's tasks are neighbouring heads one after the other.  Workgroup ids go round the dies; a die takes `together` neighbouring tasks at a
// time (heads whose rows share cache lines when tokens lie outside heads).
constexpr int kDecayDies = 8;
SV_HOST_DEVICE inline int decay_task(int id, int together)
{
    const int die = id % kDecayDies, turn = id / kDecayDies;
    return (turn / together * kDecayDies + die) * together + turn % together;
}
inline unsigned decay_grid(int64_t tasks, int together)
{
    const int64_t round = (int64_t)kDecayDies * together;
    return (unsigned)((tasks + round - 1) / round * round);
}

}  // namespace sv

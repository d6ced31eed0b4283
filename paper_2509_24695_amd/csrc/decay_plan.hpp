// How a decayed linear-attention call is cut up: chunks of tokens, segments of chunks, workgroups.  Plain C++ (no device code), shared by
// the launcher, the kernels and host-side tests.
#pragma once

#include <stdint.h>

#include <initializer_list>

#include "tile_walk.hpp"

namespace sv {

constexpr int kMaxDecaySegments = 128;      // what decay_scan walks one after the other
constexpr int kDecayChunkBf16 = 64, kDecayChunkF32 = 32;

// A head's sequence of `chunks` chunks is walked by `segments` workgroups, `per_segment` chunks each (the last fewer).
struct DecayPlan {
    int chunks, segments, per_segment;
};

// What a plan takes, in ns.  A chunk is a step that waits mostly for itself (products, LDS, the other waves), so a second workgroup on a compute
// unit costs `beside` of the first one's time, up to `resident` of them; what is beyond them waits its turn.  More than one segment costs two more
// launches (6 us), a third of a walk step for each chunk that is not in the last segment (decay_sums; three walks share two such problems), and
// the state's d x d numbers written, scanned and read again (8 bytes each at 4 TB/s: 2 ns per 1 000).
struct DecayCost {
    int step, resident;
    double beside;
};
inline DecayCost decay_cost(int d, bool bf16)
{
    if (d <= 32) return {bf16 ? 2200 : 2300, 4, 0.15};
    if (d <= 64) return {bf16 ? 2450 : 3900, 4, 0.35};
    return {bf16 ? 3450 : 6450, 2, 0.73};
}

constexpr int kDecayUnits = 256;            // compute units
constexpr double kDecayLaunches = 6000, kDecaySumsStep = 0.33, kDecayStateNs = 0.002;

inline double decay_time(const DecayCost &cost, int64_t BH, int segments, int per_segment, int d, int walks)
{
    const auto steps = [&](int64_t workgroups) {
        const int64_t on_a_unit = (workgroups + kDecayUnits - 1) / kDecayUnits;
        const auto load = [&](int64_t n) { return n ? 1 + cost.beside * (double)(n - 1) : 0; };
        return (double)per_segment * cost.step * ((double)(on_a_unit / cost.resident) * load(cost.resident) + load(on_a_unit % cost.resident));
    };
    const double walk = steps(BH * walks * segments);
    if (segments == 1) return walk;
    const int64_t states = BH * (walks > 1 ? 2 : 1);
    return kDecayLaunches + walk + kDecaySumsStep * steps(states * (segments - 1)) + kDecayStateNs * (double)states * segments * d * d;
}

// States that the segments of all heads together begin from: no more than this, where there are fewer heads (eight workgroups of a walk on a compute
// unit, four at d > 64; twice the figure, or none, gains nothing, half of it costs up to 33 %).  A call with fewer batches, heads or tokens
// needs no more than one with more.  (With as many heads or more a call is one segment and touches none of them.)
inline int64_t decay_slots(int64_t BH, int n_tokens, int d, int walks)
{
    const int64_t most = (d <= 64 ? 2048 : 1024) / walks, chunks = ((int64_t)n_tokens + kDecayChunkF32 - 1) / kDecayChunkF32;
    const int64_t slots = BH * (chunks < kMaxDecaySegments ? chunks : kMaxDecaySegments);
    return BH >= most ? BH : slots < most ? slots : most;
}

// The cut that takes least by decay_time.  Its figures were fitted to the times of 178 calls (both directions and types, d of 32 to 128, 2 to 224
// heads, 100 to 75 600 tokens) each cut into one to 128 segments, with kernels that took the scores in one piece and the sums to their
// end: 1.6 % longer than the best cut of each, at most 13 %, where "as many workgroups as run at once, segments of two chunks or more" took
// 12 %, at most 87 %.  On the present kernels, 157 calls (2 to 224 heads, 100 to 32 760 tokens, memories of one token to a thousand): 1.4 % longer than the
// best cut, at most 16 % (backward, d = 32, 224 heads of 2 400 tokens 100 us, one segment 86); 39 of them with memories of 10 000 tokens: 0.8
// %, at most 9 %.
inline DecayPlan decay_plan(int64_t BH, int n_tokens, int d, int chunk, int walks)
{
    const int chunks = (int)(((int64_t)n_tokens + chunk - 1) / chunk);
    const DecayCost cost = decay_cost(d, chunk == kDecayChunkBf16);
    DecayPlan best{chunks, 1, chunks};
    double least = decay_time(cost, BH, 1, chunks, d, walks);
    const int64_t slots = decay_slots(BH, n_tokens, d, walks);
    for (int segments : {2, 3, 4, 5, 6, 8, 10, 12, 14, 16, 20, 24, 28, 32, 40, 48, 56, 64, 80, 96, 112, kMaxDecaySegments}) {
        const int per_segment = (chunks + segments - 1) / segments;
        if (per_segment == best.per_segment) continue;
        const int used = (chunks + per_segment - 1) / per_segment;
        if (BH * used > slots) break;
        const double time = decay_time(cost, BH, used, per_segment, d, walks);
        if (time < least) {
            least = time;
            best = {chunks, used, per_segment};
        }
        if (per_segment == 1) break;
    }
    return best;
}

// The memory side's cache.  A prompt whose k and v do not fit there reads its tokens past the caches in the walk, as nothing of them is met again (us
// so / else: 64 heads of 75 600 tokens of 64 656 / 688, 16 of 128 420 / 432, 20 of 112, heads outside tokens, 482 / 488); a smaller one finds there
// what the sums have read (32 heads of 4 680 tokens of 128 79.0 / 71.5, of 64 44.5 / 38.0, 7 x 8 of up to 1 501 of 128 52.1 / 49.0), and heads that
// share lines find each other's (views of one projection's output, 20 heads of 75 600 tokens of 112 561 / 531, 40 of 32 760 473 / 459).
constexpr int64_t kLastCacheBytes = (int64_t)256 << 20;
inline bool decay_past_caches(int64_t BH, int n_tokens, int d, int elem_bytes, int walks, bool shares_lines)
{
    return walks == 1 && !shares_lines && 2 * BH * n_tokens * d * elem_bytes > kLastCacheBytes;
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

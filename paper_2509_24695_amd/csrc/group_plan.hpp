// How the rows of a group norm are dealt to workgroups.  Plain C++ (no device code), shared by the launchers and host-side tests.
#pragma once

#include <stdint.h>

#include "tile_walk.hpp"

namespace sv {

// A workgroup is `across` pieces (at most 32, as many in every tile) by `down` rows, and walks a chunk of the rows of one (b, h).
constexpr int kGroupThreads = 256, kGroupAhead = 4;
struct GroupCut {
    int across, down;
    int64_t tiles, chunks;             // workgroups across the channels; chunks of the N rows
    int64_t rows;                      // of a chunk, a multiple of `down`
};
// As many chunks as give `most` workgroups, of at least kGroupAhead rows a thread.
inline GroupCut group_cut(int64_t BH, int64_t N, int64_t pieces, int64_t most)
{
    GroupCut c{};
    c.tiles = (pieces + 31) / 32;
    c.across = (int)((pieces + c.tiles - 1) / c.tiles);
    c.down = kGroupThreads / c.across;
    const int64_t step = (int64_t)c.down * kGroupAhead, steps = (N + step - 1) / step;
    int64_t chunks = most / (BH * c.tiles);
    chunks = chunks > steps ? steps : chunks < 1 ? 1 : chunks;
    c.rows = (steps + chunks - 1) / chunks * step;
    c.chunks = (N + c.rows - 1) / c.rows;
    return c;
}
// (21 frames of 1 560 rows of 2 240 channels: sums with 1 024 workgroups at most 30.6 us, 1 280 33, 4 096 34; rows with 4 096 53, 2 048 55, 8 192 52; backwards, 14 040 rows,
// with 4 096 32, 8 192 35)
constexpr int64_t kGroupSumWgs = 1024, kGroupApplyWgs = 4096;

// Sums of wide groups are kept by group: a chunk and tile leave two numbers for each group that the tile touches, at most this many groups.
// Those of narrow ones are kept by channel, and so are those that become the parameters' gradients.
constexpr int kWideGroup = 32;
inline int group_pairs(int64_t tile_channels, int64_t width) { return (int)((tile_channels - 1) / width) + 2; }

// With this many pairs a group at most the workgroups of the next launch add them up themselves.
constexpr int64_t kFoldedPairs = 128;

// Chunks times channels of all (b, h) together in the largest call with no more batches, heads and rows and the same d: with one chunk each
// these are BH d, with more there are at most kGroupSumWgs workgroups of 32 pieces of at most eight channels; and a chunk has at least 32 rows.
inline int64_t group_slots(int64_t BH, int64_t N, int64_t d)
{
    const int64_t most = BH * d > kGroupSumWgs * 256 ? BH * d : kGroupSumWgs * 256, all = BH * ((N + 31) / 32) * d;
    return all < most ? all : most;
}

// A group whose rows fit the registers of one workgroup is read once, by one launch: units of 16, 4 or 2 bytes (the largest that a group's part of a
// row is whole units of), a thread the same unit of every row that it has, `most` words of it at most.
constexpr int kHeldThreads = 1024;
struct HeldForm {
    int unit, across, lines, rows;     // bytes; units of a row; rows side by side; rows of a thread; unit == 0: does not fit
};
inline HeldForm held_form(int64_t N, int64_t width_bytes, int most)
{
    HeldForm f{};
    const int unit = width_bytes % 16 == 0 ? 16 : width_bytes % 4 == 0 ? 4 : 2, words = unit == 16 ? 4 : 1;
    if (width_bytes / unit > kHeldThreads) return f;
    f.across = (int)(width_bytes / unit);
    f.lines = kHeldThreads / f.across;
    const int64_t rows = (N + f.lines - 1) / f.lines;
    if (rows * words > most) return f;
    f.unit = unit;
    f.rows = (int)rows;
    return f;
}
// Workgroup ids go round the dies (one L2 each); a die takes a run of neighbouring groups, whose parts of a row share lines (901 x 3 rows of 32 groups of ten channels
// fp32 9.6 us, dealt singly 11.0, with the sums of the time).  For ids below 8 ceil(groups / 8); a task past the last group is none.
constexpr int kGroupDies = 8;
inline int64_t held_grid(int64_t groups) { return (groups + kGroupDies - 1) / kGroupDies * kGroupDies; }
SV_HOST_DEVICE inline uint32_t held_task(uint32_t id, uint32_t grid) { return id % kGroupDies * (grid / kGroupDies) + id / kGroupDies; }

constexpr int kHeldForwardWords = 32, kHeldBackwardWords = 16;      // (a thread of 1 024 has 128 registers)

// The form of a whole call: more groups than a launch has workgroups (lanes are counted in 32 bits) are streamed like those that do not fit.
inline HeldForm held_form(int64_t N, int64_t width_bytes, int most, int64_t groups)
{
    return held_grid(groups) * kHeldThreads < (int64_t)1 << 32 ? held_form(N, width_bytes, most) : HeldForm{};
}

}  // namespace sv

// The cuts of group norms and short convolutions: every row is walked once, and what a call needs fits the workspace of every larger call.
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "../paper_2509_24695_amd/csrc/conv_plan.hpp"
#include "../paper_2509_24695_amd/csrc/group_plan.hpp"

using namespace sv;

#define CHECK(x)                                                             \
    if (!(x)) {                                                              \
        std::printf("line %d: %s (BH %ld N %ld d %d)\n", __LINE__, #x, BH, N, d); \
        std::exit(1);                                                        \
    }

int main()
{
    for (long BH : {1L, 2L, 7L, 21L, 64L, 5000L, 1L << 20})
        for (long N : {1L, 2L, 7L, 31L, 32L, 33L, 100L, 511L, 513L, 1560L, 4681L, 32760L, 75600L, 1L << 20, (1L << 31) - 1})
            for (int d : {8, 16, 40, 64, 112, 256, 264, 320, 2240, 4104, 8192})
                for (int per : {4, 8}) {
                    if (BH * N >= 1L << 31) continue;
                    const long pieces = d / per;
                    for (long most : {kGroupSumWgs, kGroupApplyWgs}) {
                        const GroupCut c = group_cut(BH, N, pieces, most);
                        CHECK(c.across <= 32 && c.across * c.down <= kGroupThreads && c.across * (c.down + 1) > kGroupThreads && c.tiles * c.across >= pieces && (c.tiles - 1) * c.across < pieces);
                        CHECK(c.chunks >= 1 && c.chunks * c.rows >= N && (c.chunks - 1) * c.rows < N && c.rows % c.down == 0);
                        CHECK(c.chunks == 1 || BH * c.tiles * c.chunks <= most);
                        for (int width : {32, 40, 70, 256, d})
                            if (width >= kWideGroup && width <= d) CHECK(2 * c.tiles * group_pairs(c.across * per, width) <= d);
                        if (most == kGroupSumWgs) CHECK(BH * c.chunks * d <= group_slots(BH, N, d));
                    }
                    CHECK(group_slots(BH, N, d) <= group_slots(BH + 1, N, d) && group_slots(BH, N, d) <= group_slots(BH, N + 1, d));
                    for (int width : {1, 2, 3, 10, 70, 256, d})
                        for (int most : {kHeldForwardWords, kHeldBackwardWords}) {
                            const int bytes = width * (per == 8 ? 2 : 4);
                            const HeldForm f = held_form(N, bytes, most);
                            if (!f.unit) continue;
                            CHECK((f.unit == 2 || f.unit == 4 || f.unit == 16) && f.across * f.unit == bytes && f.across * f.lines <= kHeldThreads && f.lines >= 1);
                            CHECK((long)f.lines * f.rows >= N && f.rows * (f.unit == 16 ? 4 : 1) <= most && (per == 8 || f.unit != 2));
                        }
                    for (long H : {1L, 3L, 20L}) {
                        const ConvCut c = conv_cut(BH, N, H * pieces);
                        CHECK(c.across <= 32 && c.across * c.down <= kConvThreads && c.across * (c.down + 1) > kConvThreads && c.tiles * c.across >= H * pieces);
                        CHECK(c.blocks * c.down * c.run >= N && (c.blocks - 1) * c.down * c.run < N && c.run >= kConvLeastRun && c.run <= kConvMostRun);
                        CHECK(conv_partial_floats(BH, c.blocks, H * d, 4) <= conv_workspace_floats(BH, N, H * d));
                        CHECK(conv_workspace_floats(BH, N, H * d) <= conv_workspace_floats(BH + 1, N, H * d));
                        CHECK(conv_workspace_floats(BH, N, H * d) <= conv_workspace_floats(BH, N + 1, H * d));
                        CHECK(conv_workspace_floats(BH, N, H * d) <= conv_workspace_floats(BH, N, (H + 1) * d));
                        const int run = conv_run(BH * N, (int)(H * pieces));
                        CHECK(run >= 4 && run <= 32);
                    }
                }
    return 0;
}

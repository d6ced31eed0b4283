// Which group norms a workgroup holds: those whose rows fit its registers, and no more groups than a launch has workgroups of them.
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "../paper_2509_24695_amd/csrc/group_plan.hpp"

using namespace sv;

#define CHECK(x)                                                      \
    if (!(x)) {                                                       \
        std::printf("line %d: %s (groups %ld)\n", __LINE__, #x, groups); \
        std::exit(1);                                                 \
    }

int main()
{
    const long most = (1L << 32) / kHeldThreads;
    for (long groups : {1L, 7L, 8L, 9L, 96L, 1L << 20, most - 8, most - 7, most - 1, most, most + 1, 6400000L, 1L << 24, 1L << 30})
        for (int words : {kHeldForwardWords, kHeldBackwardWords}) {
            const HeldForm f = held_form(1, 20, words, groups);
            CHECK((f.unit != 0) == (held_grid(groups) < most));
            CHECK(!f.unit || held_grid(groups) * (long)kHeldThreads < 1L << 32);
            CHECK(held_form(1 << 20, 20, words, groups).unit == 0);   // rows that do not fit
        }
    return 0;
}

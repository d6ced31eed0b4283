// Prints how csrc/decay_plan.hpp cuts calls up: for each "BH tokens d bf16 walks shares_lines" segments, chunks per segment, and whether the walk's tokens pass
// the caches by.
#include "../paper_2509_24695_amd/csrc/decay_plan.hpp"

#include <cstdio>
#include <cstdlib>

int main(int argc, char **argv)
{
    for (int i = 1; i + 5 < argc; i += 6) {
        const long long BH = std::atoll(argv[i]);
        const int n = std::atoi(argv[i + 1]), d = std::atoi(argv[i + 2]), bf16 = std::atoi(argv[i + 3]), walks = std::atoi(argv[i + 4]);
        const sv::DecayPlan p = sv::decay_plan(BH, n, d, bf16 ? sv::kDecayChunkBf16 : sv::kDecayChunkF32, walks);
        std::printf("%d %d %d\n", p.segments, p.per_segment, (int)sv::decay_past_caches(BH, n, d, bf16 ? 2 : 4, walks, std::atoi(argv[i + 5]) != 0));
    }
}

// Reads calls (B groups group_channels tokens) and prints how they are cut, forwards and backwards: segments and tokens of a segment.
#include <cstdio>

#include "../paper_2509_24695_amd/csrc/scan_plan.hpp"

int main()
{
    long B;
    int G, channels, N;
    while (std::scanf("%ld %d %d %d", &B, &G, &channels, &N) == 4) {
        const sv::ScanPlan f = sv::scan_plan(B, G, channels, N, sv::kScanForwardWaves), b = sv::scan_plan(B, G, channels, N, sv::kScanBackwardWaves);
        std::printf("%d %d %d %d\n", f.segments, f.per_segment, b.segments, b.per_segment);
    }
    return 0;
}

// The cuts of selective scans: segments cover the tokens, begin at whole runs, and fit the workspace of every larger call.
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "../paper_2509_24695_amd/csrc/scan_plan.hpp"

using namespace sv;

#define CHECK(x)                                                                    \
    if (!(x)) {                                                                     \
        std::printf("line %d: %s (B %ld G %d K %d N %d)\n", __LINE__, #x, B, G, K, N); \
        std::exit(1);                                                               \
    }

int main()
{
    for (long B : {1L, 2L, 7L, 64L, 5000L})
        for (int G : {1, 2, 5, 20})
            for (int K : {4, 32, 64, 72, 448, 2240, 8192})
                for (int N : {1, 2, 7, 8, 9, 31, 32, 33, 63, 64, 65, 100, 511, 4680, 4681, 32760, 75600, 1 << 20, (1 << 30) + 3})
                    for (long waves : {kScanForwardWaves, kScanBackwardWaves}) {
                        if (B * N > (1L << 31)) continue;
                        const ScanPlan p = scan_plan(B, G, K, N, waves);
                        CHECK(p.blocks == G * ((K + 63) / 64));
                        CHECK(p.segments >= 1 && p.segments <= kScanMostSegments);
                        CHECK(p.per_segment % kScanRun == 0);
                        CHECK((int64_t)p.per_segment * p.segments >= N && (int64_t)p.per_segment * (p.segments - 1) < N);
                        CHECK(p.segments == 1 || p.per_segment >= kScanShortest);
                        CHECK(B * p.segments <= scan_slots(B, N, (int64_t)G * K, waves));
                        CHECK(scan_slots(B, N, (int64_t)G * K, waves) <= scan_slots(B + 1, N, (int64_t)G * K, waves));
                        CHECK(scan_slots(B, N, (int64_t)G * K, waves) <= scan_slots(B, N + 1, (int64_t)G * K, waves));
                        CHECK(p.segments == 1 || B * p.segments * p.blocks <= waves || (B * p.segments * p.blocks <= 2 * waves && p.per_segment >= kScanLongSegment));
                    }
    return 0;
}

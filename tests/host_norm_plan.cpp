// csrc/norm_plan.hpp on the CPU: every width has lanes for all of its pieces, and no group of rows is left without a workgroup.
#include "../paper_2509_24695_amd/csrc/norm_plan.hpp"

#include <cstdio>
#include <initializer_list>

using namespace sv;

int main()
{
    for (int pieces = 1; pieces <= kNormMostWidth / 4; ++pieces) {
        const NormForm f = norm_form(pieces);
        const bool known = f.lanes == 4 || f.lanes == 8 || f.lanes == 16 || f.lanes == 32 || (f.lanes == 64 && f.vecs <= 6) ||
                           ((f.lanes == 256 || f.lanes == 512 || f.lanes == 1024) && f.vecs == 2);
        if (!known || f.lanes * f.vecs < pieces || norm_threads(f) % f.lanes || norm_threads(f) > 1024) {
            std::printf("FAIL %d pieces: %d lanes x %d\n", pieces, f.lanes, f.vecs);
            return 1;
        }
        if (pieces <= kNormMostWidth / 8 && f.lanes * f.vecs > kNormMostWidth / 8) {
            std::printf("FAIL bf16 %d pieces: %d lanes x %d\n", pieces, f.lanes, f.vecs);
            return 1;
        }
        for (long long rows : {1ll, 2ll, 63ll, 64ll, 65ll, 100000ll, (1ll << 31) - 1})
            for (long long groups : {1ll, 2ll, 20ll, 3000ll, 1ll << 24}) {
                const int n = norm_workgroups(f, rows, groups, kNormBackwardWgs);
                const long long steps = (rows + norm_rows_per_step(f) - 1) / norm_rows_per_step(f);
                if (n < 1 || n > steps || (n > 1 && n * groups > kNormBackwardWgs)) {
                    std::printf("FAIL %lld rows, %lld groups: %d workgroups\n", rows, groups, n);
                    return 1;
                }
            }
    }
    if (norm_form(0).lanes || norm_form(kNormMostWidth / 4 + 1).lanes) return 1;
    std::printf("OK\n");
    return 0;
}

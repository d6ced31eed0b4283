// csrc/norm_plan.hpp on the CPU: every width has lanes for all of its pieces, and no group of rows is left without a workgroup.
#include "../paper_2509_24695_amd/csrc/norm_plan.hpp"

#include <cstdio>
#include <initializer_list>

using namespace sv;

int main()
{
    for (int both = 2; both < 2 * (kNormMostWidth / 4 + 1); ++both) {
        const int pieces = both / 2;
        const bool backward = both % 2;
        const NormForm f = norm_form(pieces, backward);
        const bool known = f.lanes == 4 || f.lanes == 8 || f.lanes == 16 || f.lanes == 32 || (f.lanes == 64 && f.vecs <= (backward ? 3 : 6)) ||
                           (f.lanes == 128 && f.vecs >= 2 && f.vecs <= 4) || (f.lanes == 256 && f.vecs == 3) || ((f.lanes == 512 || f.lanes == 1024) && f.vecs == 2);
        if (!known || f.lanes * f.vecs < pieces || norm_threads(f) % f.lanes || norm_threads(f) > 1024) {
            std::printf("FAIL %d pieces: %d lanes x %d\n", pieces, f.lanes, f.vecs);
            return 1;
        }
        if (pieces <= kNormMostWidth / 8 && f.lanes > 512) {
            std::printf("FAIL bf16 %d pieces: %d lanes x %d\n", pieces, f.lanes, f.vecs);
            return 1;
        }
        for (long long rows : {1ll, 2ll, 63ll, 64ll, 65ll, 100000ll, (1ll << 31) - 1})
            for (long long groups : {1ll, 2ll, 20ll, 3000ll, 1ll << 24}) {
                const int n = norm_workgroups(f, rows, groups, kNormMostBackwardWgs);
                const long long steps = (rows + norm_rows_per_step(f) - 1) / norm_rows_per_step(f);
                if (n < 1 || n > steps || (n > 1 && n * groups > kNormMostBackwardWgs)) {
                    std::printf("FAIL %lld rows, %lld groups: %d workgroups\n", rows, groups, n);
                    return 1;
                }
            }
    }
    if (norm_form(0, false).lanes || norm_form(kNormMostWidth / 4 + 1, true).lanes) return 1;
    for (int d = 4; d <= kNormMostWidth; d += 4)
        if (norm_backward_wgs(d) > kNormMostBackwardWgs) return 1;
    for (long long d : {1ll, 2ll, 3ll, 5ll, 7ll, 20ll, 64ll, 112ll, 4680ll, 32760ll, 65537ll, (1ll << 30) - 1, 1ll << 30, (1ll << 30) + 1, (1ll << 31) - 1}) {
        const NormDivisor q = NormDivisor::of((int32_t)d);
        auto right = [&](long long n) { return n < 0 || n >= 1ll << 31 || q.quotient((uint32_t)n) == n / d; };
        for (long long k = 0; k < 20000; ++k)                        // around multiples of d, where a quotient goes wrong first, and all over
            for (long long n : {k, (1ll << 31) - 1 - k, k * d, k * d - 1, ((1ll << 31) / d - k) * d, ((1ll << 31) / d - k) * d - 1, k * 107374ll})
                if (!right(n)) {
                    std::printf("FAIL %lld / %lld\n", n, d);
                    return 1;
                }
    }
    std::printf("OK\n");
    return 0;
}

// csrc/decay_plan.hpp on the CPU: every chunk belongs to one segment, segments stay within their bound, a walk's chunks hold its tokens, and
// the tasks of a launch are dealt to workgroups one to one.
#include "../paper_2509_24695_amd/csrc/decay_plan.hpp"

#include <climits>
#include <cstdio>
#include <initializer_list>
#include <vector>

using namespace sv;

static int fail(const char *what, long long a, long long b)
{
    std::printf("FAIL %s %lld %lld\n", what, a, b);
    return 1;
}

int main()
{
    const int lengths[] = {1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 1000, 4680, 32760, 75600, 1 << 20, INT_MAX};
    const long long heads[] = {1, 2, 3, 20, 40, 64, 255, 256, 257, 511, 512, 513, 4096, 1 << 24};
    for (int chunk : {32, 64})
        for (int d : {32, 64, 112, 128})
            for (int walks : {1, 3})
                for (int n : lengths)
                    for (long long BH : heads) {
                        const DecayPlan p = decay_plan(BH, n, d, chunk, walks);
                        if (p.chunks != (int)(((long long)n + chunk - 1) / chunk)) return fail("chunks", n, BH);
                        if (p.segments < 1 || p.segments > kMaxDecaySegments || p.per_segment < 1) return fail("segments", n, BH);
                        if ((long long)p.segments * p.per_segment < p.chunks) return fail("chunks left over", n, BH);
                        if ((long long)(p.segments - 1) * p.per_segment >= p.chunks) return fail("empty segment", n, BH);
                        if (p.segments > 1 && (long long)p.per_segment * chunk > (1ll << 30) + chunk) return fail("tokens of a segment", n, BH);
                        const long long slots = decay_slots(BH, n, d, walks);
                        if (BH * p.segments > slots || slots > (BH > 2048 ? BH : 2048)) return fail("slots", n, BH);
                        if (decay_slots(BH + 1, n, d, walks) < slots || (n < INT_MAX && decay_slots(BH, n + 1, d, walks) < slots)) return fail("slots of a larger call", n, BH);
                    }
    for (int chunk : {32, 64})
        for (int n : lengths) {
            const DecayWalk w(n, chunk);
            if (w.lead < 0 || w.lead >= chunk || (long long)w.chunks * chunk - w.lead != n) return fail("lead", n, chunk);
        }
    const DecayWalk none(0, 64);
    if (none.chunks != 0 || none.lead != 0) return fail("no tokens", none.chunks, none.lead);
    for (int together : {1, 2, 4, 5})
        for (int tasks : {1, 7, 8, 9, 40, 41, 513}) {
            std::vector<int> seen(tasks, 0);
            const unsigned grid = decay_grid(tasks, together);
            for (unsigned id = 0; id < grid; ++id) {
                const int t = decay_task((int)id, together);
                if (t < 0) return fail("task", t, id);
                if (t < tasks) ++seen[t];
            }
            for (int s : seen)
                if (s != 1) return fail("dealt", tasks, together);
        }
    std::printf("OK\n");
    return 0;
}

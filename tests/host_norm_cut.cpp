// Prints how csrc/norm_plan.hpp deals rows out: for each "pieces rows backward width" lanes, 16-byte pieces per lane, rows per step and workgroups.
#include "../paper_2509_24695_amd/csrc/norm_plan.hpp"

#include <cstdio>
#include <cstdlib>

int main(int argc, char **argv)
{
    for (int i = 1; i + 3 < argc; i += 4) {
        const int pieces = std::atoi(argv[i]), rows = std::atoi(argv[i + 1]), backward = std::atoi(argv[i + 2]), d = std::atoi(argv[i + 3]);
        const sv::NormForm f = sv::norm_form(pieces, backward);
        std::printf("%d %d %d %d\n", f.lanes, f.vecs, sv::norm_rows_per_step(f),
                    sv::norm_workgroups(f, rows, 1, backward ? sv::norm_backward_wgs(d) : sv::kNormForwardWgs));
    }
}

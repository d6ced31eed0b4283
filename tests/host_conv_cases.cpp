// Reads calls (B, pieces of a token forwards and backwards, tokens) and prints the tokens of a run, forwards and backwards.
#include <cstdio>

#include "../paper_2509_24695_amd/csrc/conv_plan.hpp"

int main()
{
    long B, N;
    int forward, backward;
    while (std::scanf("%ld %d %d %ld", &B, &forward, &backward, &N) == 4) std::printf("%d %d\n", sv::conv_run(B * N, forward), sv::conv_cut(B, N, backward).run);
    return 0;
}

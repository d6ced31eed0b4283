// The sequences of a padded batch and the rows of a server's batch.
#pragma once

#include "common.hpp"

namespace sv {

// Tokens of sequence b.
__device__ __forceinline__ int held_length(const int32_t *lengths, int b, int N)
{
    if (!lengths) return N;
    const int n = lengths[b];
    return n < 0 ? 0 : n > N ? N : n;
}

// Has an earlier row of the batch the same slot?  For all threads of a workgroup.
__device__ __forceinline__ bool slot_taken(const int32_t *slots, int b, int slot)
{
    bool taken = false;
    if (slots)
        for (int r = threadIdx.x; r < b; r += blockDim.x) taken |= slots[r] == slot;
    return __syncthreads_or(taken);
}

}  // namespace sv

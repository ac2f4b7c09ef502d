// The order in which a group of warps goes through its ring of slots in shared memory (rcd_norm.cuh).
#pragma once

#include <cstdint>

#include <cuda_runtime.h>

namespace rcd {

// Where a group is in its ring.  A wait that ran out leaves its slot's barrier in the phase of a copy that has not arrived: an order for the next
// row would arrive there a second time in that phase, and the barrier's parity says no more which copy is meant.  So whoever
// has waited in vain orders nothing from then on.
struct RingTurn {
    int slot = 0;
    uint32_t parity = 0;
    bool live = true;
    __host__ __device__ void waited(bool came) { live = live && came; }
    __host__ __device__ bool may_order() const { return live; }
    __host__ __device__ void next(int stages)
    {
        if (++slot == stages) { slot = 0; parity ^= 1; }
    }
};

}  // namespace rcd

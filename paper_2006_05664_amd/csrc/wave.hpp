// Lanes of a wave that exchange values through LDS.
#pragma once

namespace {

// Between the writes of some lanes and the reads of others, and before the next writes.  A wave's accesses to the LDS take effect in the order of the code; this keeps the
// compiler from changing that order, as it might where it can tell one lane's addresses apart.  No instruction comes of it.
__device__ __forceinline__ void exchange()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

}  // namespace

// What kernels of several units need of a wave.
#pragma once
#include <hip/hip_runtime.h>

namespace rnnt {

// What lanes of a wave wrote to LDS is there for the others
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// An address that all lanes have alike, in scalar registers
template <class T> __device__ __forceinline__ const T *uniform(const T *p)
{
    const unsigned long long u = reinterpret_cast<unsigned long long>(p);
    const unsigned lo = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)u), hi = (unsigned)__builtin_amdgcn_readfirstlane((int)(u >> 32));
    return reinterpret_cast<const T *>((unsigned long long)hi << 32 | lo);
}

}  // namespace rnnt

// soma_wave.hpp -- exchange between the lanes of a wave.
#pragma once

#include <hip/hip_runtime.h>

namespace soma {

// Orders a wave's LDS accesses before its later ones, of other lanes' words too (they are
// carried out in order; this keeps the compiler from moving them, or from taking a load
// from the lane's own store).
__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

}  // namespace soma

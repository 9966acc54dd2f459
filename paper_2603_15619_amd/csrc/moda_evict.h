// Shared by the kernels that choose the rows of an eviction (moda_evict.hip, moda_evict_long.hip).
#pragma once
#include <type_traits>

#include "moda_launch.h"

namespace moda {

// A row's rank: orders as the weight does; -0 as 0, a NaN below everything.  Recent rows take 0xffffffff, above everything.
__device__ __forceinline__ unsigned weight_key(float w) {
  const unsigned u = __builtin_bit_cast(unsigned, w + 0.f);
  return w != w ? 0u : u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}

// The choice for long caches, several launches; index and workspace as for the short ones.
size_t evict_long_workspace_bytes(long long groups, int T, int n);
bool evict_long_grid_ok(long long groups, int T);
hipError_t launch_evict_choose_long(const EvictParams& p, void* workspace, hipStream_t stream);

}  // namespace moda

// Device helpers shared by the kernels that serve from the paged cache.
#pragma once

#include "kamera_cache.h"
#include "kamera_device.h"

namespace kamera {

// Memory that no kernel writes while this one runs, at a wave-uniform address:
// a scalar load.
template <typename T>
__device__ __forceinline__ T uniform_load(const T* p) {
  return *(const __attribute__((address_space(4))) T*)(uintptr_t)p;
}

// p[i], or `other` where the optional array is not there.  The load is made either
// way (from `there`, an array that is), so that several of these leave together: a
// branch around each would cost a memory latency a piece.
__device__ __forceinline__ int load_or(const int32_t* p, int64_t i, int other, const int32_t* there) {
  const bool has = p != nullptr;
  const int x = uniform_load((has ? p : there) + (has ? i : 0));
  return has ? x : other;
}

}  // namespace kamera

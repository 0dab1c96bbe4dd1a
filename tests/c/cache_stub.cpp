// Stand-ins for the GPU launches of the paged-cache entry points, for CPU-only
// builds of the host layer (kamera_cache.cpp) under the sanitizers: each reads
// every byte of the parameters it was handed.

#include <atomic>

#include "kamera_cache.h"

std::atomic<long> g_cache_launches{0};
std::atomic<int> g_cache_fail{0};

namespace kamera {

template <typename T>
static hipError_t take(const T& p) {
  volatile long sink = 0;
  for (size_t k = 0; k < sizeof(p); ++k) sink += reinterpret_cast<const unsigned char*>(&p)[k];
  g_cache_launches.fetch_add(1);
  return static_cast<hipError_t>(g_cache_fail.load());
}

hipError_t launch_page_tables(const TablesParams& p, hipStream_t) { return take(p); }
hipError_t launch_append(const AppendParams& p, hipStream_t) { return take(p); }
hipError_t launch_select(const SelectParams& p, hipStream_t) { return take(p); }
hipError_t launch_attend(const AttendParams& p, hipStream_t) { return take(p); }

}  // namespace kamera

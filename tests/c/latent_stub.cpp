// Stand-ins for the GPU launches of the latent-cache entry points, for CPU-only
// builds of the host layer (kamera_latent.cpp) under the sanitizers: each reads
// every byte of the parameters it was handed, and checks what the kernels assume.

#include <atomic>
#include <cstdio>
#include <cstdlib>

#include "kamera_latent.h"

std::atomic<long> g_latent_launches{0};
std::atomic<int> g_latent_fail{0};

namespace kamera {

template <typename T>
static hipError_t take(const T& p, bool ok) {
  volatile long sink = 0;
  for (size_t k = 0; k < sizeof(p); ++k) sink += reinterpret_cast<const unsigned char*>(&p)[k];
  if (!ok) {
    fprintf(stderr, "parameters out of the kernels' range\n");
    abort();
  }
  g_latent_launches.fetch_add(1);
  return static_cast<hipError_t>(g_latent_fail.load());
}

hipError_t launch_rotate(const RotateParams& p, hipStream_t) {
  return take(p, p.n_tasks > 0 && p.block_tokens >= 1 && p.block_tokens <= kRotateTokens &&
                     (int64_t)p.n_blocks * p.block_tokens >= p.n_tokens);
}
hipError_t launch_project(const ProjectParams& p, hipStream_t) {
  return take(p, p.n_tasks > 0 && (int64_t)p.per_xcd * 8 >= p.n_tasks && p.n_in % 64 == 0);
}
static bool mla(const MlaParams& p) {
  return p.n_tasks > 0 && p.n_parts >= 0 && (p.n_parts == 0 || (p.part_o != nullptr && p.prefix != nullptr && p.min_units > 0)) &&
         (int64_t)p.n_row_blocks * p.rows_block >= (int64_t)p.n_queries * p.group;
}
hipError_t launch_attend_latent(const MlaParams& p, hipStream_t) {
  return take(p, mla(p) && p.rows_block == 16 * p.row_waves && (p.dim == 256 || p.dim == 512));
}
hipError_t launch_attend_expanded(const MlaParams& p, hipStream_t) {
  return take(p, mla(p) && p.rows_block == 128 && (p.dim == 64 || p.dim == 128));
}

}  // namespace kamera

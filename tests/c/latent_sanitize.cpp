// Drives the latent-cache entry points' host layer with randomised argument
// structs: valid ones with up to three 32- or 64-bit words overwritten by
// boundary values.  A call launches exactly when its validation passed and there is
// work.

#include <atomic>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <thread>
#include <vector>

#include "kamera.h"

extern std::atomic<long> g_latent_launches;
extern std::atomic<int> g_latent_fail;

namespace {

std::atomic<int> failures{0};
#define CHECK(c)                                                \
  do {                                                          \
    if (!(c)) {                                                 \
      failures.fetch_add(1);                                    \
      fprintf(stderr, "line %d: %s (%s)\n", __LINE__, #c, kamera_last_error()); \
    }                                                           \
  } while (0)

template <typename T>
T* at(uintptr_t p) { return reinterpret_cast<T*>(p); }

void set(int64_t* s, std::initializer_list<int64_t> v) {
  for (int64_t x : v) *s++ = x;
}

kamera_append_rotated_args rotate() {
  kamera_append_rotated_args a;
  memset(&a, 0, sizeof(a));
  a.n_chunks = 2; a.n_layers = 3; a.n_tokens = 40; a.n_k_heads = 4; a.k_dim = 128; a.n_v_heads = 4; a.v_dim = 128;
  a.n_q_heads = 8; a.page_size = 16; a.pt_stride = 4; a.n_pool_pages = 10;
  a.rope.theta = 1e4; a.rope.rope_dim = 64; a.rope.n_sections = 1;
  a.scaling.kind = KAMERA_SCALING_PAIRS; a.scaling.factor = 4; a.scaling.original_tokens = 4096; a.scaling.low_turns = 1;
  a.scaling.high_turns = 32;
  a.page_table = at<int32_t>(0x10000); a.k = at<void>(0x20000000); a.v = at<void>(0x21000000); a.q = at<void>(0x22000000);
  a.q_out = at<void>(0x23000000); a.k_cache = at<void>(0x30000000); a.v_cache = at<void>(0x31000000);
  set(a.k_stride, {61440, 20480, 512, 128}); set(a.v_stride, {61440, 20480, 512, 128});
  set(a.q_stride, {122880, 40960, 1024, 128}); set(a.q_out_stride, {61440, 20480, 512, 64});
  set(a.k_cache_stride, {81920, 8192, 512, 128}); set(a.v_cache_stride, {81920, 8192, 512, 128});
  return a;
}

kamera_project_args project() {
  kamera_project_args a;
  memset(&a, 0, sizeof(a));
  a.n_rows = 100; a.n_heads = 16; a.n_in = 128; a.n_out = 512;
  a.x = at<void>(0x20000000); a.w = at<void>(0x21000000); a.out = at<void>(0x22000000);
  set(a.x_stride, {2048, 128}); set(a.w_stride, {65536, 512, 1}); set(a.out_stride, {8192, 512});
  return a;
}

kamera_expand_args expand() {
  kamera_expand_args a;
  memset(&a, 0, sizeof(a));
  a.n_requests = 3; a.n_heads = 16; a.n_in = 512; a.n_out = 256; a.n_keys = 1000; a.page_size = 16; a.pt_stride = 64;
  a.n_pool_pages = 200; a.kv_tokens = at<int32_t>(0x10000); a.page_table = at<int32_t>(0x11000);
  a.cache = at<void>(0x20000000); a.w = at<void>(0x21000000); a.out = at<void>(0x22000000);
  set(a.cache_stride, {9216, 576}); set(a.w_stride, {131072, 1, 512}); set(a.out_stride, {4096, 256});
  return a;
}

template <typename A>
A attend() {
  A a;
  memset(&a, 0, sizeof(a));
  a.n_requests = 2; a.n_heads = 16; a.rope_dim = 64; a.n_queries = 4; a.n_keys = 4096; a.page_size = 16; a.pt_stride = 256;
  a.n_pool_pages = 600; a.causal = 1; a.scale = 0.1f; a.kv_tokens = at<int32_t>(0x10000); a.page_table = at<int32_t>(0x11000);
  a.q = at<void>(0x20000000); a.out = at<void>(0x21000000); a.workspace = at<void>(0x60000000); a.workspace_bytes = 1 << 30;
  return a;
}

kamera_attend_latent_args latent() {
  auto a = attend<kamera_attend_latent_args>();
  a.latent_dim = 512; a.cache = at<void>(0x30000000);
  set(a.q_stride, {9216, 576}); set(a.out_stride, {8192, 512}); set(a.cache_stride, {9216, 576});
  return a;
}

kamera_attend_expanded_args expanded() {
  auto a = attend<kamera_attend_expanded_args>();
  a.head_dim = 128; a.rope_cache = at<void>(0x30000000); a.k = at<void>(0x40000000); a.v = at<void>(0x48000000);
  set(a.q_stride, {3200, 192}); set(a.out_stride, {2048, 128}); set(a.rope_cache_stride, {9216, 576});
  set(a.k_stride, {2048, 128}); set(a.v_stride, {2048, 128});
  return a;
}

template <typename A>
void spoil(A& a, std::mt19937_64& rng) {
  static const int64_t words[] = {0, 1, -1, 2, 16, 63, 64, 65, 127, 128, 129, 1024, 4096, 1 << 20, INT32_MAX, INT32_MIN,
                                  (int64_t)1 << 31, (int64_t)1 << 32, (int64_t)1 << 40, INT64_MAX, INT64_MIN,
                                  0x20000000, 0x21000000, 0x30000000, 0x60000000};
  const int n = (int)(rng() % 4);
  for (int i = 0; i < n; ++i) {
    const int64_t w = words[rng() % (sizeof(words) / sizeof(words[0]))];
    if (rng() & 1) {
      const int32_t x = (int32_t)w;
      memcpy(reinterpret_cast<char*>(&a) + 4 * (rng() % (sizeof(A) / 4)), &x, 4);
    } else {
      memcpy(reinterpret_cast<char*>(&a) + 8 * (rng() % (sizeof(A) / 8)), &w, 8);
    }
  }
}

template <typename A>
void drive(int which, A (*make)(), int (*call)(const A*, void*), std::mt19937_64& rng, int n, bool count) {
  for (int i = 0; i < n; ++i) {
    A a = make();
    spoil(a, rng);
    const long before = g_latent_launches.load();
    const int rc = kamera_validate_latent(which, &a), got = call(&a, nullptr);
    CHECK(rc == got);
    CHECK((rc == KAMERA_OK) == (kamera_last_error()[0] == '\0'));
    if (count) {
      const long made = g_latent_launches.load() - before;
      CHECK(made == 0 || (made == 1 && rc == KAMERA_OK));
    }
  }
}

template <typename A>
void workspaces(int which, A (*make)(), int64_t (*bytes)(const A*), std::mt19937_64& rng, int n) {
  for (int i = 0; i < n; ++i) {
    A a = make();
    spoil(a, rng);
    const int64_t w = bytes(&a);
    // a call that passes has enough workspace
    if (kamera_validate_latent(which, &a) == KAMERA_OK) CHECK(w >= 0 && (w == 0 || w <= a.workspace_bytes));
  }
}

void all(uint64_t seed, int n, bool count) {
  std::mt19937_64 rng(seed);
  drive<kamera_append_rotated_args>(0, rotate, kamera_append_rotated, rng, n, count);
  drive<kamera_project_args>(1, project, kamera_project_heads, rng, n, count);
  drive<kamera_expand_args>(2, expand, kamera_expand_latent, rng, n, count);
  drive<kamera_attend_latent_args>(3, latent, kamera_attend_latent, rng, n, count);
  drive<kamera_attend_expanded_args>(4, expanded, kamera_attend_expanded, rng, n, count);
  workspaces<kamera_attend_latent_args>(3, latent, kamera_attend_latent_workspace, rng, n);
  workspaces<kamera_attend_expanded_args>(4, expanded, kamera_attend_expanded_workspace, rng, n);
}

}  // namespace

int main() {
  all(1, 40000, true);
  g_latent_fail.store(1);
  const kamera_attend_latent_args a = latent();
  CHECK(kamera_attend_latent(&a, nullptr) == KAMERA_ERR_HIP);
  g_latent_fail.store(0);
  std::vector<std::thread> ts;
  for (int t = 0; t < 8; ++t) ts.emplace_back(all, 100 + t, 2000, false);
  for (auto& t : ts) t.join();
  if (failures.load()) return 1;
  printf("ok\n");
  return 0;
}

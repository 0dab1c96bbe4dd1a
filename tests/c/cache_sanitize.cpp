// Drives the paged-cache entry points' host layer with randomised argument
// structs: valid ones with up to three 32- or 64-bit words overwritten by
// boundary values.  A call launches exactly when its validation passed.

#include <atomic>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <thread>
#include <vector>

#include "kamera.h"

extern std::atomic<long> g_cache_launches;
extern std::atomic<int> g_cache_fail;

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

kamera_page_tables_args tables() {
  kamera_page_tables_args a;
  memset(&a, 0, sizeof(a));
  a.n_requests = 4; a.page_size = 16; a.pt_stride = 8; a.n_pool_pages = 100; a.n_free = 20; a.n_slots = 64;
  a.tokens_before = at<int32_t>(0x10000); a.tokens_after = at<int32_t>(0x11000); a.free_pages = at<int32_t>(0x12000);
  a.free_end = at<int32_t>(0x13000); a.page_table = at<int32_t>(0x14000); a.token_base = at<int32_t>(0x15000);
  a.slots = at<int64_t>(0x16000);
  return a;
}

kamera_append_args append() {
  kamera_append_args a;
  memset(&a, 0, sizeof(a));
  a.n_chunks = 2; a.n_layers = 3; a.n_heads = 4; a.head_dim = 128; a.n_tokens = 40; a.page_size = 16;
  a.pt_stride = 4; a.n_pool_pages = 10;
  a.page_table = at<int32_t>(0x10000); a.k = at<void>(0x20000000); a.v = at<void>(0x21000000);
  a.k_cache = at<void>(0x30000000); a.v_cache = at<void>(0x31000000);
  a.k_scale = at<float>(0x32000000); a.v_scale = at<float>(0x33000000);
  for (int64_t* s : {a.k_stride, a.v_stride}) { s[0] = 61440; s[1] = 20480; s[2] = 512; s[3] = 128; }
  for (int64_t* s : {a.k_cache_stride, a.v_cache_stride}) { s[0] = 81920; s[1] = 8192; s[2] = 128; s[3] = 2048; }
  for (int64_t* s : {a.k_scale_stride, a.v_scale_stride}) { s[0] = 40; s[1] = 4; s[2] = 1; }
  return a;
}

kamera_select_args select() {
  kamera_select_args a;
  memset(&a, 0, sizeof(a));
  a.n_requests = 3; a.n_q_heads = 8; a.n_kv_heads = 2; a.head_dim = 128; a.n_keys = 1000; a.page_size = 16;
  a.pt_stride = 64; a.n_pool_pages = 200; a.n_keep = 8; a.n_first = 1; a.n_last = 1;
  a.kv_tokens = at<int32_t>(0x10000); a.page_table = at<int32_t>(0x11000); a.q = at<void>(0x20000000);
  a.k_sum = at<int8_t>(0x30000000); a.k_sum_scale = at<float>(0x31000000); a.sel = at<int32_t>(0x32000000);
  a.sel_count = at<int32_t>(0x33000000);
  a.q_stride[0] = 1024; a.q_stride[1] = 128; a.k_sum_stride[0] = 256; a.k_sum_stride[1] = 128;
  a.k_sum_scale_stride[0] = 2; a.k_sum_scale_stride[1] = 1;
  return a;
}

kamera_attend_args attend() {
  kamera_attend_args a;
  memset(&a, 0, sizeof(a));
  a.n_requests = 2; a.n_q_heads = 16; a.n_kv_heads = 2; a.head_dim = 128; a.n_queries = 4; a.n_keys = 4096;
  a.page_size = 16; a.pt_stride = 256; a.n_pool_pages = 600; a.cache_type = KAMERA_CACHE_E4M3; a.causal = 1;
  a.scale = 0.1f;
  a.kv_tokens = at<int32_t>(0x10000); a.page_table = at<int32_t>(0x11000); a.q = at<void>(0x20000000);
  a.out = at<void>(0x21000000); a.k_cache = at<void>(0x30000000); a.v_cache = at<void>(0x40000000);
  a.k_scale = at<float>(0x50000000); a.v_scale = at<float>(0x51000000); a.workspace = at<void>(0x60000000);
  a.workspace_bytes = 1 << 30;
  for (int64_t* s : {a.q_stride, a.out_stride}) { s[0] = 2048; s[1] = 128; }
  for (int64_t* s : {a.k_cache_stride, a.v_cache_stride}) { s[0] = 4096; s[1] = 128; s[2] = 2048; }
  for (int64_t* s : {a.k_scale_stride, a.v_scale_stride}) { s[0] = 2; s[1] = 1; }
  return a;
}

template <typename T>
void spoil(T& a, std::mt19937_64& rng) {
  static const int32_t w32[] = {0, 1, -1, 2, 15, 16, 17, 64, 127, 128, 129, 512, 8192, 8193, 32768, 1 << 20, 1 << 30,
                                INT32_MAX, INT32_MIN, 0x7fc00000};
  static const int64_t w64[] = {0, 1, -1, 8, 16, 4096, (int64_t)1 << 31, (int64_t)1 << 32, (int64_t)1 << 50,
                                (int64_t)1 << 62, INT64_MAX, INT64_MIN, 0x20000000};
  unsigned char* b = reinterpret_cast<unsigned char*>(&a);
  for (int k = (int)(rng() % 4); k > 0; --k) {
    if (rng() % 2) {
      const int32_t v = w32[rng() % (sizeof(w32) / 4)];
      memcpy(b + 4 * (rng() % (sizeof(T) / 4)), &v, 4);
    } else {
      const int64_t v = w64[rng() % (sizeof(w64) / 8)];
      memcpy(b + 8 * (rng() % (sizeof(T) / 8)), &v, 8);
    }
  }
}

template <typename T>
void drive(int which, T (*make)(), int (*call)(const T*, void*), std::mt19937_64& rng, int n, bool count) {
  T good = make();
  CHECK(call(&good, nullptr) == KAMERA_OK);
  for (int i = 0; i < n; ++i) {
    T a = make();
    spoil(a, rng);
    const int rc = kamera_validate_cache(which, &a);
    CHECK((rc == KAMERA_OK) == (kamera_last_error()[0] == '\0'));
    const long before = g_cache_launches.load();
    const int got = call(&a, nullptr);
    CHECK(got == rc);
    if (count) CHECK(g_cache_launches.load() - before <= (rc == KAMERA_OK ? 1 : 0));
  }
}

int64_t workspace_of(const kamera_attend_args& a) { return kamera_attend_workspace(&a); }

void all(uint64_t seed, int n, bool count) {
  std::mt19937_64 rng(seed);
  drive<kamera_page_tables_args>(0, tables, kamera_page_tables, rng, n, count);
  drive<kamera_append_args>(1, append, kamera_append_paged8, rng, n, count);
  drive<kamera_select_args>(2, select, kamera_select_pages, rng, n, count);
  drive<kamera_attend_args>(3, attend, kamera_attend_paged, rng, n, count);
  for (int i = 0; i < n; ++i) {
    kamera_attend_args a = attend();
    spoil(a, rng);
    const int64_t w = workspace_of(a);
    // a call that passes has enough workspace
    if (kamera_validate_cache(3, &a) == KAMERA_OK) CHECK(w >= 0 && (w == 0 || w <= a.workspace_bytes));
  }
}

}  // namespace

int main() {
  all(1, 40000, true);
  g_cache_fail.store(1);
  kamera_attend_args a = attend();
  CHECK(kamera_attend_paged(&a, nullptr) == KAMERA_ERR_HIP);
  g_cache_fail.store(0);
  std::vector<std::thread> ts;
  for (int t = 0; t < 8; ++t) ts.emplace_back(all, 100 + t, 2000, false);
  for (auto& t : ts) t.join();
  if (failures.load()) return 1;
  printf("ok\n");
  return 0;
}

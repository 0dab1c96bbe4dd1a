// What the host layer hands the kernels: launches that keep their parameters.

#include <cstdio>
#include <cstring>

#include "kamera.h"
#include "kamera_cache.h"

namespace kamera {

static SelectParams g_select;

hipError_t launch_page_tables(const TablesParams&, hipStream_t) { return hipSuccess; }
hipError_t launch_append(const AppendParams&, hipStream_t) { return hipSuccess; }
hipError_t launch_select(const SelectParams& p, hipStream_t) { g_select = p; return hipSuccess; }
hipError_t launch_attend(const AttendParams&, hipStream_t) { return hipSuccess; }

}  // namespace kamera

namespace {

int failures = 0;
#define CHECK(c)                                                  \
  do {                                                            \
    if (!(c)) {                                                   \
      ++failures;                                                 \
      fprintf(stderr, "line %d: %s (%s)\n", __LINE__, #c, kamera_last_error()); \
    }                                                             \
  } while (0)

template <typename T>
T* at(uintptr_t p) { return reinterpret_cast<T*>(p); }

// The selection looks up the first max_pages entries of a row: no more than the keys need.
void select_entries() {
  for (const int keys : {0, 1, 16, 17, 64}) {
    kamera_select_args a;
    memset(&a, 0, sizeof(a));
    a.n_requests = 3; a.n_q_heads = 8; a.n_kv_heads = 2; a.head_dim = 128; a.n_keys = keys; a.page_size = 16;
    a.pt_stride = (keys + 15) / 16; a.n_pool_pages = 200; a.n_keep = 2; a.n_first = 1; a.n_last = 1;
    a.kv_tokens = at<int32_t>(0x10000); a.page_table = at<int32_t>(0x11000); a.q = at<void>(0x20000000);
    a.k_sum = at<int8_t>(0x30000000); a.k_sum_scale = at<float>(0x31000000); a.sel = at<int32_t>(0x32000000);
    a.sel_count = at<int32_t>(0x33000000);
    a.q_stride[0] = 1024; a.q_stride[1] = 128; a.k_sum_stride[0] = 256; a.k_sum_stride[1] = 128;
    a.k_sum_scale_stride[0] = 2; a.k_sum_scale_stride[1] = 1;
    CHECK(kamera_select_pages(&a, nullptr) == KAMERA_OK);
    CHECK(kamera::g_select.max_pages <= a.pt_stride);
  }
}

}  // namespace

int main() {
  select_entries();
  if (failures) return 1;
  printf("ok\n");
  return 0;
}

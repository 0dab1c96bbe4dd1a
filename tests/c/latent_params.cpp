// The tile that the host layer picks for a product: latent_params project|expand
// requests rows heads in out prints its rows.  Launches keep their parameters.

#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "kamera.h"
#include "kamera_latent.h"

namespace kamera {

static ProjectParams g_project;

hipError_t launch_rotate(const RotateParams&, hipStream_t) { return hipSuccess; }
hipError_t launch_project(const ProjectParams& p, hipStream_t) { g_project = p; return hipSuccess; }
hipError_t launch_attend_latent(const MlaParams&, hipStream_t) { return hipSuccess; }
hipError_t launch_attend_expanded(const MlaParams&, hipStream_t) { return hipSuccess; }

}  // namespace kamera

namespace {

template <typename T>
T* at(uintptr_t p) { return reinterpret_cast<T*>(p); }

// What both calls have: dense W and results at places far from each other, never looked at.
template <typename A>
void product(A& a, int heads, int in, int out) {
  a.n_heads = heads; a.n_in = in; a.n_out = out;
  a.w = at<void>(0x2000000000); a.out = at<void>(0x3000000000);
  a.w_stride[0] = (int64_t)in * out; a.w_stride[1] = out; a.w_stride[2] = 1;
  a.out_stride[0] = (int64_t)heads * out; a.out_stride[1] = out;
}

}  // namespace

int main(int argc, char** argv) {
  if (argc != 7) return 2;
  const int requests = atoi(argv[2]), rows = atoi(argv[3]), heads = atoi(argv[4]), in = atoi(argv[5]), out = atoi(argv[6]);
  int rc;
  if (strcmp(argv[1], "project") == 0) {
    kamera_project_args a;
    memset(&a, 0, sizeof(a));
    product(a, heads, in, out);
    a.n_rows = rows; a.x = at<void>(0x1000000000);
    a.x_stride[0] = (int64_t)heads * in; a.x_stride[1] = in;
    rc = kamera_project_heads(&a, nullptr);
  } else {
    kamera_expand_args a;
    memset(&a, 0, sizeof(a));
    product(a, heads, in, out);
    a.n_requests = requests; a.n_keys = rows; a.page_size = 16; a.pt_stride = (rows + 15) / 16; a.n_pool_pages = 1000;
    a.kv_tokens = at<int32_t>(0x10000); a.page_table = at<int32_t>(0x20000); a.cache = at<void>(0x1000000000);
    a.cache_stride[0] = 16 * 576; a.cache_stride[1] = 576;
    rc = kamera_expand_latent(&a, nullptr);
  }
  if (rc != KAMERA_OK) {
    fprintf(stderr, "%s\n", kamera_last_error());
    return 1;
  }
  printf("%d\n", kamera::g_project.tile_rows);
  return 0;
}

// kamera_page_tables: pages and token slots for requests that grow, in one
// launch.
//
// With a_r = ceil(before_r / P), b_r = ceil(after_r / P), the pages of request
// r start at place free_begin + sum_{s<r} (b_s - a_s) of the free list and its
// new tokens at sum_{s<r} (after_s - before_s) of the packed batch.  Every
// workgroup takes both prefix sums over all requests for itself (they are a few
// KiB, and a second launch or a wait between workgroups would cost more than
// the whole call), keeps them in LDS, and then writes its share of the outputs:
// the owner of an entry is found by bisection of the sums (64 requests by a token
// each: 5.9 us, 256 requests by 0.8 million tokens: 7.9 us of kernel, a chain of
// loads).  No workgroup reads
// what another writes: entries of new pages are taken from the free list, of
// older ones from the table.

#include <algorithm>

#include "kamera_cache.h"
#include "kamera_device.h"

namespace kamera {

namespace {

constexpr int kTabThreads = 256;

// Exclusive sum of x over the workgroup's threads; `total` is the sum of all.
__device__ __forceinline__ int block_scan(int x, int* s_wave, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int incl = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(incl, d);
    if (lane >= d) incl += y;
  }
  if (lane == 63) s_wave[wave] = incl;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kTabThreads / 64; ++w) {
    if (w < wave) before += s_wave[w];
    total += s_wave[w];
  }
  __syncthreads();
  return before + incl - x;
}

// The r in [0, n) with sums[r] <= i < sums[r + 1] (sums ascending, i < sums[n]).
__device__ __forceinline__ int owner(const int* sums, int n, int i) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] <= i) lo = mid; else hi = mid;
  }
  return lo;
}

}  // namespace

__global__ __launch_bounds__(kTabThreads) void tables_kernel(TablesParams) {
  const TablesParams& p = kernel_params<TablesParams>();
  extern __shared__ int s_sums[];                  // pages [n + 1], tokens [n + 1], tokens before [n]
  __shared__ int s_wave[kTabThreads / 64];
  const int n = p.n_requests, tid = threadIdx.x;
  int* s_pages = s_sums;
  int* s_tokens = s_sums + n + 1;
  int* s_before = s_sums + 2 * (n + 1);
  const int per = (n + kTabThreads - 1) / kTabThreads;
  const int r0 = min(n, tid * per), r1 = min(n, r0 + per);
  const int cap = p.pt_stride * p.page_size;       // < 2^31
  const int begin = p.free_begin != nullptr ? p.free_begin[0] : 0;
  int pages = 0, tokens = 0;
  uint32_t flags = 0;
  for (int r = r0; r < r1; ++r) {
    int b = p.tokens_before != nullptr ? max(p.tokens_before[r], 0) : 0;
    int a = max(p.tokens_after[r], 0);
    if (a > cap) flags |= KAMERA_STATUS_BAD_LENGTH;
    a = min(a, cap);
    b = min(b, a);                                 // a request that shrinks stays where it is
    const int need = (int)(fast_div((uint32_t)a + p.page_size - 1, p.fd_page) -
                           fast_div((uint32_t)b + p.page_size - 1, p.fd_page));
    s_before[r] = b;
    s_pages[r] = need;
    s_tokens[r] = a - b;
    pages += need;
    tokens += a - b;
  }
  int total_pages, total_tokens;
  int page_at = block_scan(pages, s_wave, total_pages);
  int token_at = block_scan(tokens, s_wave, total_tokens);
  for (int r = r0; r < r1; ++r) {
    const int need = s_pages[r], grown = s_tokens[r];
    s_pages[r] = page_at;
    s_tokens[r] = token_at;
    page_at += need;
    token_at += grown;
  }
  if (tid == 0) {
    s_pages[n] = total_pages;
    s_tokens[n] = total_tokens;
  }
  __syncthreads();

  const int first = min(max(begin, 0), p.n_free);
  const int left = p.n_free - first;
  // page number k of the new ones, or -1
  auto new_page = [&](int k) -> int {
    if (k >= left) {
      flags |= KAMERA_STATUS_NO_PAGE;
      return -1;
    }
    const int pg = p.free_pages[first + k];
    if (pg < 0 || pg >= p.n_pool_pages) {
      flags |= KAMERA_STATUS_BAD_PAGE;
      return -1;
    }
    return pg;
  };

  const int64_t stride = (int64_t)gridDim.x * kTabThreads;
  const int64_t self = (int64_t)blockIdx.x * kTabThreads + tid;
  for (int64_t r = self; r <= n; r += stride) p.token_base[r] = s_tokens[r];
  if (self == 0) p.free_end[0] = first + min(total_pages, left);
  for (int64_t k = self; k < total_pages; k += stride) {
    const int r = owner(s_pages, n, (int)k);
    const int held = (int)fast_div((uint32_t)s_before[r] + p.page_size - 1, p.fd_page);
    p.page_table[(int64_t)r * p.pt_stride + held + ((int)k - s_pages[r])] = new_page((int)k);
  }
  if (p.slots != nullptr) {
    // four neighbouring tokens a thread: one bisection, then a walk
    for (int64_t i0 = self * 4; i0 < p.n_slots; i0 += stride * 4) {
      int r = i0 < total_tokens ? owner(s_tokens, n, (int)i0) : n;
      int last_k = -1, pg = -1;
      int64_t slot[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int64_t i = i0 + e;
        slot[e] = -1;
        if (i < total_tokens) {
          while (i >= s_tokens[r + 1]) {
            ++r;
            last_k = -1;
          }
          const int b = s_before[r];
          const uint32_t tok = (uint32_t)(b + ((int)i - s_tokens[r]));
          const int k = (int)fast_div(tok, p.fd_page);
          if (k != last_k) {
            const int held = (int)fast_div((uint32_t)b + p.page_size - 1, p.fd_page);
            if (k < held) {
              pg = p.page_table[(int64_t)r * p.pt_stride + k];
              if (pg < 0 || pg >= p.n_pool_pages) {
                flags |= KAMERA_STATUS_BAD_PAGE;
                pg = -1;
              }
            } else {
              pg = new_page(s_pages[r] + k - held);
            }
            last_k = k;
          }
          if (pg >= 0) slot[e] = (int64_t)pg * p.page_size + (tok - (uint32_t)k * p.page_size);
        }
      }
      if (i0 + 4 <= p.n_slots && p.slots_aligned) {
        reinterpret_cast<longlong2*>(p.slots + i0)[0] = make_longlong2(slot[0], slot[1]);
        reinterpret_cast<longlong2*>(p.slots + i0)[1] = make_longlong2(slot[2], slot[3]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (i0 + e < p.n_slots) p.slots[i0 + e] = slot[e];
      }
    }
  }
  if (flags != 0 && p.status != nullptr) atomicOr(p.status, flags);
}

hipError_t launch_page_tables(const TablesParams& p, hipStream_t s) {
  const size_t lds = (3 * (size_t)p.n_requests + 2) * sizeof(int);
  static std::atomic<bool> done[kMaxDevices];
  if (lds > 60 * 1024) {
    const hipError_t e = ensure_lds_limit((const void*)tables_kernel,
                                          (int)((3 * (size_t)KAMERA_MAX_REQUESTS + 2) * sizeof(int)), done);
    if (e != hipSuccess) return e;
  }
  // Four slots a thread.  Every workgroup repeats the sums: one a CU where these are
  // long, four where a thread has one request at most.
  const int64_t items = p.slots != nullptr ? (p.n_slots + 3) / 4 : 0;
  const int64_t want = std::max<int64_t>(items, p.n_requests + 1), most = p.n_requests <= kTabThreads ? 1024 : 256;
  const int grid = (int)std::min<int64_t>((want + kTabThreads - 1) / kTabThreads, most);
  hipLaunchKernelGGL(tables_kernel, dim3(grid), dim3(kTabThreads), lds, s, p);
  return hipGetLastError();
}

}  // namespace kamera

// kamera_select_pages: the pages a query needs most, by an integer score.
//
// One workgroup of 16 waves per (request, KV head).  The group's query rows
// become int8 with one power-of-two scale; a page's score is the largest of
// the group's int8 products with the page's key sum, times the page's scale.
// |product| <= 127 * 127 * 128 < 2^24, so the fp32 score is exact and the
// selection one answer.
//
// Scores: 16x16x64 int8 MFMA with the query rows as A and 16 pages as B, so a
// lane holds 4 rows of one page and the maximum over the rows is 3 in-lane
// steps and 2 across the wave.  Keys (scores as ordered 32-bit patterns) stay in
// LDS.  The n_keep-th largest key is found two bits a pass, 16 passes of counts
// by ballots (no atomics: the scores of a request share their leading bits, and
// histogram bins would be hit by whole waves at once).  Then one ordered pass
// writes the indices: above the threshold, and the first of those equal to it.
// Bound by the latency of the page-table and sum loads (128 bytes a page) and of
// the 16 passes.

#include "kamera_cache.h"
#include "kamera_device.h"

namespace kamera {

namespace {

constexpr int kSelThreads = 1024;
constexpr int kSelWaves = kSelThreads / 64;
constexpr uint32_t kAlways = 0xffffffffu;          // above the key of +infinity
constexpr uint32_t kNever = 0x007fffffu;           // the key of -infinity

typedef int i32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}

__device__ __forceinline__ int wave_max(int x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x = max(x, __shfl_xor(x, d));
  return x;
}

}  // namespace

// D columns; RT tiles of 16 query rows (group <= 16 * RT).
template <int D, int RT>
__global__ __launch_bounds__(kSelThreads) void select_kernel(SelectParams) {
  const SelectParams& p = kernel_params<SelectParams>();
  extern __shared__ uint32_t s_key[];              // [max_pages]
  __shared__ __attribute__((aligned(16))) int8_t s_q[RT * 16 * D];
  __shared__ int s_wave[kSelWaves];
  __shared__ int s_cnt[2][3][kSelWaves];
  __shared__ int s_run[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = blockIdx.x / p.n_kv_heads, h = blockIdx.x % p.n_kv_heads;
  int kv = min(max(p.kv_tokens[r], 0), p.n_keys);
  const int n = (kv + p.page_size - 1) / p.page_size;
  int32_t* sel = p.sel + ((int64_t)r * p.n_kv_heads + h) * p.n_keep;
  const int keep = p.n_keep;
  if (n <= keep) {                                 // every page
    for (int j = tid; j < keep; j += kSelThreads) sel[j] = j < n ? j : -1;
    if (tid == 0) p.sel_count[(int64_t)r * p.n_kv_heads + h] = n;
    return;
  }

  // the group's queries in 8 bits
  const uint16_t* q = p.q + r * p.q_s[0] + (int64_t)h * p.group * p.q_s[1];
  int amax = 0;
  for (int i = tid; i < p.group * D; i += kSelThreads) {
    const int b = q[(i / D) * p.q_s[1] + i % D] & 0x7fff;
    if (b < 0x7f80) amax = max(amax, b);
  }
  amax = wave_max(amax);
  if (lane == 0) s_wave[wave] = amax;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSelWaves; ++w) amax = max(amax, s_wave[w]);
  // 127 = (1 + 0x7e / 2^7) * 2^6
  int f = (amax >> 7) - 127 - 6 + ((amax & 0x7f) > 0x7e ? 1 : 0);
  f = f < kMinExp ? kMinExp : f;
  const float down = __uint_as_float((uint32_t)(127 - f) << 23);
  for (int i = tid; i < RT * 16 * D; i += kSelThreads) {
    const int row = i / D;
    int8_t v = 0;
    if (row < p.group) {
      const uint32_t b = q[row * p.q_s[1] + i % D];
      if ((b & 0x7fff) < 0x7f80) v = (int8_t)(int)rintf(bf_lo(b) * down);
    }
    s_q[i] = v;
  }
  __syncthreads();

  const int c16 = lane & 15, g = lane >> 4;
  i32x4 qa[RT][D / 64];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int k = 0; k < D / 64; ++k)
      qa[t][k] = *reinterpret_cast<const i32x4*>(s_q + (t * 16 + c16) * D + k * 64 + g * 16);

  const int32_t* table = p.page_table + (int64_t)r * p.pt_stride;
  const int8_t* sums = p.k_sum + h * p.k_sum_s[1];
  const float* scales = p.k_sum_scale + h * p.k_sum_scale_s[1];
  constexpr int U = 4;                             // page tiles in flight a wave
  for (int t0 = wave * 16; t0 < n; t0 += kSelWaves * 16 * U) {
    int page[U];
    i32x4 b[U][D / 64];
    float sc[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = t0 + u * kSelWaves * 16 + c16;
      page[u] = j < n ? table[j] : -1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool in = page[u] >= 0 && page[u] < p.n_pool_pages;
      const int pg = in ? page[u] : 0;
#pragma unroll
      for (int k = 0; k < D / 64; ++k)
        b[u][k] = *reinterpret_cast<const i32x4*>(sums + pg * p.k_sum_s[0] + k * 64 + g * 16);
      sc[u] = scales[pg * p.k_sum_scale_s[0]];
      const int j = t0 + u * kSelWaves * 16 + c16;
      if (!in && j < n && g == 0 && p.status != nullptr) atomicOr(p.status, KAMERA_STATUS_BAD_PAGE);
      page[u] = in ? pg : -1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      int best = INT32_MIN;
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        i32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < D / 64; ++k) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(qa[t][k], b[u][k], acc, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (t * 16 + 4 * g + i < p.group) best = max(best, acc[i]);
      }
      best = max(best, __shfl_xor(best, 16));
      best = max(best, __shfl_xor(best, 32));
      const int j = t0 + u * kSelWaves * 16 + c16;
      if (g == 0 && j < n) {
        uint32_t key = page[u] >= 0 ? ordered((float)best * sc[u]) : kNever;
        if (j < p.n_first || j >= n - p.n_last) key = kAlways;
        s_key[j] = key;
      }
    }
  }
  __syncthreads();

  // The largest T with at least `keep` keys >= T, two bits a pass.
  uint32_t T = 0;
  int turn = 0;
  for (int bit = 30; bit >= 0; bit -= 2, turn ^= 1) {
    const uint32_t a1 = T | (1u << bit), a2 = T | (2u << bit), a3 = T | (3u << bit);
    int n1 = 0, n2 = 0, n3 = 0;
    for (int j0 = wave * 64; j0 < n; j0 += kSelThreads) {
      const uint32_t key = j0 + lane < n ? s_key[j0 + lane] : 0u;
      n1 += __popcll(__ballot(key >= a1));
      n2 += __popcll(__ballot(key >= a2));
      n3 += __popcll(__ballot(key >= a3));
    }
    if (lane == 0) {
      s_cnt[turn][0][wave] = n1;
      s_cnt[turn][1][wave] = n2;
      s_cnt[turn][2][wave] = n3;
    }
    __syncthreads();
    n1 = n2 = n3 = 0;
#pragma unroll
    for (int w = 0; w < kSelWaves; ++w) {
      n1 += s_cnt[turn][0][w];
      n2 += s_cnt[turn][1][w];
      n3 += s_cnt[turn][2][w];
    }
    T = n3 >= keep ? a3 : (n2 >= keep ? a2 : (n1 >= keep ? a1 : T));
  }

  // Ordered output.  Each wave takes a contiguous run of 64-key groups, so two
  // counts a wave order the whole.
  const int groups = (n + 63) / 64, per = (groups + kSelWaves - 1) / kSelWaves;
  const int g0 = min(groups, wave * per), g1 = min(groups, g0 + per);
  int above = 0, equal = 0;
  for (int k = g0; k < g1; ++k) {
    const bool there = k * 64 + lane < n;
    const uint32_t key = there ? s_key[k * 64 + lane] : 0u;
    above += __popcll(__ballot(there && key > T));
    equal += __popcll(__ballot(there && key == T));
  }
  __syncthreads();                                 // s_cnt of the last pass is read
  if (lane == 0) {
    s_cnt[0][0][wave] = above;
    s_cnt[0][1][wave] = equal;
  }
  __syncthreads();
  int above_at = 0, equal_at = 0, above_all = 0;
  for (int w = 0; w < kSelWaves; ++w) {
    if (w < wave) {
      above_at += s_cnt[0][0][w];
      equal_at += s_cnt[0][1][w];
    }
    above_all += s_cnt[0][0][w];
  }
  const int ties = keep - above_all;               // of those equal to T, the first
  const uint64_t below = (1ull << lane) - 1;
  for (int k = g0; k < g1; ++k) {
    const int j = k * 64 + lane;
    const bool there = j < n;
    const uint32_t key = there ? s_key[j] : 0u;
    const uint64_t gt = __ballot(there && key > T), eq = __ballot(there && key == T);
    const int e_rank = equal_at + __popcll(eq & below);
    const int place = above_at + __popcll(gt & below) + min(e_rank, ties);
    if (there && (key > T || (key == T && e_rank < ties))) sel[place] = j;
    above_at += __popcll(gt);
    equal_at += __popcll(eq);
  }
  if (tid == 0) p.sel_count[(int64_t)r * p.n_kv_heads + h] = keep;
}

namespace {

template <int D, int RT>
hipError_t launch_one(const SelectParams& p, hipStream_t s) {
  static std::atomic<bool> done[kMaxDevices];
  const size_t lds = (size_t)p.max_pages * sizeof(uint32_t);
  if (lds > 32 * 1024) {
    const hipError_t e = ensure_lds_limit((const void*)select_kernel<D, RT>,
                                          KAMERA_MAX_SELECT_PAGES * (int)sizeof(uint32_t), done);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((select_kernel<D, RT>), dim3((uint32_t)p.n_requests * p.n_kv_heads), dim3(kSelThreads), lds, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_select(const SelectParams& p, hipStream_t s) {
  if (p.head_dim == 128) return p.group <= 16 ? launch_one<128, 1>(p, s) : launch_one<128, 4>(p, s);
  return p.group <= 16 ? launch_one<64, 1>(p, s) : launch_one<64, 4>(p, s);
}

}  // namespace kamera

// kamera_select_pages: the pages a query needs most, by an integer score.
//
// A workgroup of 16 waves per (request, KV head) selects; it also scores the pages
// itself where these are few or the workgroups many, and otherwise 256-page pieces
// are scored by workgroups of their own before (the keys in between in a
// workspace): a CU takes in about 25 bytes of key sums a cycle, 2 ns a page (one
// request of 8 KV heads, one kernel / two: 1000 pages 11.8 / 12.2 us, 2048 pages
// 14.1 / 12.4, 8192 pages 29.0 / 13.8; 32 requests, 4096 pages: 50.1 / 54.4).  The group's query rows become int8 with one power-of-two scale; a page's score is the largest of
// the group's int8 products with the page's key sum, times the page's scale.
// |product| <= 127 * 127 * 128 < 2^24, so the fp32 score is exact and the
// selection one answer.
//
// Scores: 16x16x64 int8 MFMA with the query rows as A and 16 pages as B, so a
// lane holds 4 rows of one page and the maximum over the rows is 3 in-lane
// steps and 2 across the wave.  The B operand wants neighbouring lanes on
// different pages; loaded like that each lane is a memory access of its own (13
// cycles a page and CU), so four neighbouring lanes take 64 bytes of one page and
// 1 KB of LDS a wave turns them round.
//
// Selection: keys (scores as ordered 32-bit patterns) in registers.  A histogram of
// 1024 bins, even in the score's value, finds the bin of the n_keep-th largest; the
// pages of that bin are ranked among each other.  Where a bin holds over 64 pages (ties,
// or one score far from the rest) the n_keep-th largest key is found two bits a pass
// by ballots instead (always so: 13 us in place of 8 for 64 of 4096 pages).  The
// indices are then written in order.
// Bound by the latency of the page-table and sum loads (128 bytes a page) and of
// the steps of the selection.

#include "kamera_cache_device.h"

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

__device__ __forceinline__ float unordered(uint32_t u) {
  return __uint_as_float(u ^ ((u >> 31) ? 0x80000000u : 0xffffffffu));
}

__device__ __forceinline__ int lane_of(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

// Pages of request r.
__device__ __forceinline__ int pages_of(const SelectParams& p, int r) {
  return (min(max(uniform_load(p.kv_tokens + r), 0), p.n_keys) + p.page_size - 1) / p.page_size;
}

__device__ __forceinline__ int wave_max(int x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x = max(x, __shfl_xor(x, d));
  return x;
}

// Keys of pages [first, end) of a request with n pages in all, by the workgroup's
// WAVES waves; put(j, key) takes them.  D columns; RT tiles of 16 query rows
// (group <= 16 * RT).  s_q: RT * 16 * D bytes, s_turn: 64 chunks a wave.
template <int D, int RT, int WAVES, typename Put>
__device__ __forceinline__ void score_pages(const SelectParams& p, int r, int h, int first, int end_most, int& n,
                                            int8_t* s_q, i32x4* s_turn, int* s_wave, const Put& put) {
  constexpr int kThreads = WAVES * 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c16 = lane & 15, g = lane >> 4;
  const int32_t* table = p.page_table + (int64_t)r * p.pt_stride;

  // table entries, a turn ahead of their use; those past the request's pages are
  // not used, so its length is not waited for.  Lane i looks up page i / 4 of a tile.
  constexpr int U = RT == 1 && WAVES == 16 ? 8 : 4, kTurn = WAVES * 16 * U;
  int ahead[U];
  auto look_up = [&](int t0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = t0 + u * 16 + (lane >> 2);
      ahead[u] = j < end_most ? table[j] : 0;
    }
  };
  look_up(first + wave * 16 * U);

  // the group's queries in 8 bits
  const uint16_t* q = p.q + r * p.q_s[0] + (int64_t)h * p.group * p.q_s[1];
  constexpr int QN = RT * 16 * D / kThreads;
  uint32_t qv[QN];
  int amax = 0;
#pragma unroll
  for (int k = 0; k < QN; ++k) {
    const int i = tid + k * kThreads;
    qv[k] = i < p.group * D ? q[(i / D) * p.q_s[1] + i % D] : 0;
    if ((qv[k] & 0x7fff) >= 0x7f80) qv[k] = 0;     // what is not finite
    amax = max(amax, (int)(qv[k] & 0x7fff));
  }
  n = pages_of(p, r);
  const int end = min(end_most, n);
  if (n <= p.n_keep || first >= end) return;
  amax = wave_max(amax);
  if (lane == 0) s_wave[wave] = amax;
  __syncthreads();
  amax = wave_max(s_wave[c16 & (WAVES - 1)]);
  // 127 = (1 + 0x7e / 2^7) * 2^6
  int f = (amax >> 7) - 127 - 6 + ((amax & 0x7f) > 0x7e ? 1 : 0);
  f = f < kMinExp ? kMinExp : f;
  const float down = __uint_as_float((uint32_t)(127 - f) << 23);
#pragma unroll
  for (int k = 0; k < QN; ++k) s_q[tid + k * kThreads] = (int8_t)(int)rintf(bf_lo(qv[k]) * down);
  __syncthreads();

  i32x4 qa[RT][D / 64];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int k = 0; k < D / 64; ++k)
      qa[t][k] = *reinterpret_cast<const i32x4*>(s_q + (t * 16 + c16) * D + k * 64 + g * 16);

  // U tiles of 16 pages in flight a wave
  const int8_t* sums = p.k_sum + h * p.k_sum_s[1] + (lane & 3) * 16;
  const float* scales = p.k_sum_scale + h * p.k_sum_scale_s[1];
  i32x4* turn = s_turn + wave * 64;
  for (int t0 = first + wave * 16 * U; t0 < end; t0 += kTurn) {
    i32x4 b[U][D / 64];
    float sc[U];
    uint32_t in = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool ok = ahead[u] >= 0 && ahead[u] < p.n_pool_pages;
      in |= ok || t0 + u * 16 + (lane >> 2) >= end ? 1u << u : 0u;
      const int pg = ok ? ahead[u] : 0;
#pragma unroll
      for (int k = 0; k < D / 64; ++k) b[u][k] = *reinterpret_cast<const i32x4*>(sums + pg * p.k_sum_s[0] + k * 64);
      sc[u] = scales[pg * p.k_sum_scale_s[0]];
    }
    look_up(t0 + kTurn);
    if (in != (1u << U) - 1 && p.status != nullptr) atomicOr(p.status, KAMERA_STATUS_BAD_PAGE);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      i32x4 bt[D / 64];
#pragma unroll
      for (int k = 0; k < D / 64; ++k) {
        // chunk c of page i at 4 i + (c ^ i / 4): 16 lanes that read one chunk of 16 pages hit all banks
        turn[(lane & ~3) + ((lane & 3) ^ (lane >> 4))] = b[u][k];
        __builtin_amdgcn_wave_barrier();           // one wave's LDS accesses are in order
        bt[k] = turn[c16 * 4 + (g ^ (c16 >> 2))];
        __builtin_amdgcn_wave_barrier();
      }
      int best = INT32_MIN;
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        i32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < D / 64; ++k) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(qa[t][k], bt[k], acc, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (t * 16 + 4 * g + i < p.group) best = max(best, acc[i]);
      }
      best = max(best, __shfl_xor(best, 16));
      best = max(best, __shfl_xor(best, 32));
      // page c16's maximum is in lane c16, its scale in lane 4 c16
      best = __shfl(best, lane >> 2);
      const int j = t0 + u * 16 + (lane >> 2);
      if ((lane & 3) == 0 && j < end) {
        // one that is not a number would pass for another key: a page always taken, or none
        const float score = (float)best * sc[u] + 0.0f;   // -0 becomes 0, which it ties with
        uint32_t key = ((in >> u) & 1) && score == score ? ordered(score) : kNever;
        if (j < p.n_first || j >= n - p.n_last) key = kAlways;
        put(j, key);
      }
    }
  }
}

constexpr int kPiece = 256, kPieceWaves = 4;

// For bits[k], a bit for each of the pages k * 1024 + wave * 64 + lane: how many bits
// of all waves come before this wave's in each k.  All threads; one barrier.
template <int KPT>
__device__ __forceinline__ void places(const uint64_t (&bits)[KPT], int* s_run, int (&before)[KPT]) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int k = 0; k < KPT; ++k)
    if (lane == 0) s_run[k * kSelWaves + wave] = __popcll(bits[k]);
  __syncthreads();
  constexpr int kPer = KPT * kSelWaves / 64;       // counts a lane
  int run[kPer], sum = 0;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    run[e] = sum;
    sum += s_run[lane * kPer + e];
  }
  int incl = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(incl, d);
    if (lane >= d) incl += y;
  }
#pragma unroll
  for (int k = 0; k < KPT; ++k) {
    const int grp = k * kSelWaves + wave;
    int x = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e)
      if (grp % kPer == e) x = lane_of(run[e] + incl - sum, grp / kPer);
    before[k] = x;
  }
}

}  // namespace

// The keys of one 256-page piece of a (request, KV head) into the workspace.
template <int D, int RT>
__global__ __launch_bounds__(kPieceWaves * 64) void score_kernel(SelectParams) {
  const SelectParams& p = kernel_params<SelectParams>();
  __shared__ __attribute__((aligned(16))) int8_t s_q[RT * 16 * D];
  __shared__ i32x4 s_turn[kPieceWaves * 64];
  __shared__ int s_wave[kPieceWaves];
  // the heads of a piece run at the same time: their sums lie together
  uint32_t w = blockIdx.x, d;
  d = w / p.n_kv_heads;
  const int h = (int)(w - d * p.n_kv_heads);
  w = d;
  d = w / p.n_pieces;
  const int piece = (int)(w - d * p.n_pieces), r = (int)d;
  uint32_t* keys = p.keys + ((int64_t)r * p.n_kv_heads + h) * p.max_pages;
  int n;
  score_pages<D, RT, kPieceWaves>(p, r, h, piece * kPiece, min(p.max_pages, (piece + 1) * kPiece), n, s_q, s_turn, s_wave,
                                  [&](int j, uint32_t key) { keys[j] = key; });
}

// Selection; at most KPT * 1024 pages.  SCORE: the workgroup makes the keys itself
// (D, RT as in score_pages).
template <int D, int RT, int KPT, bool SCORE>
__global__ __launch_bounds__(kSelThreads) void select_kernel(SelectParams) {
  const SelectParams& p = kernel_params<SelectParams>();
  extern __shared__ uint32_t s_key[];              // [max_pages] (SCORE)
  __shared__ __attribute__((aligned(16))) int8_t s_q[SCORE ? RT * 16 * D : 16];
  __shared__ i32x4 s_turn[SCORE ? kSelWaves * 64 : 1];
  __shared__ int s_wave[kSelWaves];
  __shared__ int s_cnt[3][3];
  __shared__ int s_run[KPT * kSelWaves];
  __shared__ int s_bin[1024];
  __shared__ uint32_t s_edge[2][kSelWaves];
  __shared__ int s_found[4];                       // bin, how many of it, its pages, listed so far
  __shared__ uint32_t s_list[64];
  __shared__ int s_list_page[64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = blockIdx.x / p.n_kv_heads, h = blockIdx.x % p.n_kv_heads;
  int n;
  uint32_t key[KPT];                               // of pages k * 1024 + tid; 0: none
  if (SCORE) {
    score_pages<D, RT, kSelWaves>(p, r, h, 0, p.max_pages, n, s_q, s_turn, s_wave,
                                  [&](int j, uint32_t k) { s_key[j] = k; });
  } else {
    const uint32_t* keys = p.keys + (int64_t)blockIdx.x * p.max_pages;
#pragma unroll
    for (int k = 0; k < KPT; ++k) key[k] = k * kSelThreads + tid < p.max_pages ? keys[k * kSelThreads + tid] : 0u;
    n = pages_of(p, r);
  }
  int32_t* sel = p.sel + (int64_t)blockIdx.x * p.n_keep;
  const int keep = p.n_keep;
  if (n <= keep) {                                 // every page
    for (int j = tid; j < keep; j += kSelThreads) sel[j] = j < n ? j : -1;
    if (tid == 0) p.sel_count[blockIdx.x] = n;
    return;
  }
  // Bins, even in value between the least and the largest score; the pages that are
  // always taken stay out (first and last ones are distinct: n > keep).
  const int want = keep - p.n_first - p.n_last;
  uint32_t lo = 0xffffffffu, hi = 0;
  if (SCORE) __syncthreads();
#pragma unroll
  for (int k = 0; k < KPT; ++k) {
    if (SCORE) key[k] = k * kSelThreads + tid < n ? s_key[k * kSelThreads + tid] : 0u;
    if (k * kSelThreads + tid >= n) key[k] = 0u;   // past the request's pages
    if (key[k] > kNever && key[k] != kAlways) {
      lo = min(lo, key[k]);
      hi = max(hi, key[k]);
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    lo = min(lo, (uint32_t)__shfl_xor((int)lo, d));
    hi = max(hi, (uint32_t)__shfl_xor((int)hi, d));
  }
  if (lane == 0) {
    s_edge[0][wave] = lo;
    s_edge[1][wave] = hi;
  }
  s_bin[tid] = 0;
  if (tid == 0) s_found[3] = 0;
  __syncthreads();
  lo = s_edge[0][lane & 15];
  hi = s_edge[1][lane & 15];
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) {
    lo = min(lo, (uint32_t)__shfl_xor((int)lo, d));
    hi = max(hi, (uint32_t)__shfl_xor((int)hi, d));
  }
  const float flo = unordered(lo), width = unordered(hi) - flo;
  const float per = width > 0.f && width < INFINITY ? 1023.0f / width : 0.f;
  // every step of this is monotone: a higher bin holds higher scores only
  auto bin_of = [&](uint32_t x) { return x > kNever ? min((int)((unordered(x) - flo) * per), 1023) : 0; };
#pragma unroll
  for (int k = 0; k < KPT; ++k)
    if (key[k] != 0u && key[k] != kAlways) atomicAdd(&s_bin[bin_of(key[k])], 1);
  __syncthreads();
  {
    // sums from the top bin down: thread t has bin 1023 - t
    const int count = s_bin[1023 - tid];
    int incl = count;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(incl, d);
      if (lane >= d) incl += y;
    }
    if (lane == 63) s_wave[wave] = incl;
    __syncthreads();
    int upto = lane < wave ? s_wave[lane & 15] : 0;
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) upto += __shfl_xor(upto, d);
    incl += lane_of(upto, 0);
    if (incl >= want && incl - count < want) {     // one thread, where want > 0
      s_found[0] = 1023 - tid;
      s_found[1] = want - (incl - count);
      s_found[2] = count;
    }
    if (want == 0 && tid == 0) {
      s_found[0] = 1024;
      s_found[1] = s_found[2] = 0;
    }
  }
  __syncthreads();
  const int bin = s_found[0], need = s_found[1];
  uint64_t taken[KPT];                             // this wave's pages, a bit a lane
  if (s_found[2] <= 64) {
    int own = -1;                                  // place in the list, of key[own_k]
#pragma unroll
    for (int k = 0; k < KPT; ++k)
      if (key[k] != 0u && key[k] != kAlways && bin_of(key[k]) == bin) {
        own = atomicAdd(&s_found[3], 1);
        s_list[own] = key[k];
        s_list_page[own] = k * kSelThreads + tid;
      }
    __syncthreads();
    const int listed = s_found[2];
#pragma unroll
    for (int k = 0; k < KPT; ++k) {
      bool take = key[k] == kAlways;
      if (key[k] != 0u && !take) {
        const int b = bin_of(key[k]);
        take = b > bin;
        if (b == bin) {
          int rank = 0;
          for (int e = 0; e < listed; ++e)
            rank += s_list[e] > key[k] || (s_list[e] == key[k] && s_list_page[e] < k * kSelThreads + tid) ? 1 : 0;
          take = rank < need;
        }
      }
      taken[k] = __ballot(take);
    }
  } else {
    // The largest T with at least `keep` keys >= T, two bits a pass, or the first T
    // met with exactly that many: no smaller key can be taken then either.
    if (tid < 9) s_cnt[tid / 3][tid % 3] = 0;
    __syncthreads();
    uint32_t T = 0;
    int set = 0;
    for (int bit = 30; bit >= 0; bit -= 2) {
      const uint32_t a1 = T | (1u << bit), a2 = T | (2u << bit), a3 = T | (3u << bit);
      int n1 = 0, n2 = 0, n3 = 0;
#pragma unroll
      for (int k = 0; k < KPT; ++k)
        if (k * kSelThreads < n) {
          n1 += __popcll(__ballot(key[k] >= a1));
          n2 += __popcll(__ballot(key[k] >= a2));
          n3 += __popcll(__ballot(key[k] >= a3));
        }
      if (lane < 3) atomicAdd(&s_cnt[set][lane], lane == 0 ? n1 : (lane == 1 ? n2 : n3));
      __syncthreads();
      n1 = s_cnt[set][0];
      n2 = s_cnt[set][1];
      n3 = s_cnt[set][2];
      // three sets of counts: this pass's are read while the next one's are added to,
      // and the third is cleared
      const int clear = set == 0 ? 2 : set - 1;
      if (tid < 3) s_cnt[clear][tid] = 0;
      set = set == 2 ? 0 : set + 1;
      const int at = n3 >= keep ? n3 : (n2 >= keep ? n2 : n1);
      T = n3 >= keep ? a3 : (n2 >= keep ? a2 : (n1 >= keep ? a1 : T));
      if (at == keep) break;
    }
    // of those equal to T, the first
    uint64_t eq[KPT];
    int above = 0;
#pragma unroll
    for (int k = 0; k < KPT; ++k) {
      taken[k] = __ballot(key[k] > T);
      eq[k] = __ballot(key[k] != 0u && key[k] == T);
      above += __popcll(taken[k]);
    }
    if (lane == 0) s_wave[wave] = above;
    int before[KPT];
    places<KPT>(eq, s_run, before);                // a barrier in here
    int ties = keep;
#pragma unroll
    for (int w = 0; w < kSelWaves; ++w) ties -= s_wave[w];
#pragma unroll
    for (int k = 0; k < KPT; ++k) {
      const bool level = (eq[k] >> lane) & 1;
      const int rank = before[k] + __popcll(eq[k] & ((1ull << lane) - 1));
      taken[k] |= __ballot(level && rank < ties);
    }
    __syncthreads();                               // s_run is used again
  }

  int before[KPT];
  places<KPT>(taken, s_run, before);
#pragma unroll
  for (int k = 0; k < KPT; ++k)
    if ((taken[k] >> lane) & 1) sel[before[k] + __popcll(taken[k] & ((1ull << lane) - 1))] = k * kSelThreads + tid;
  if (tid == 0) p.sel_count[blockIdx.x] = keep;
}

namespace {

template <int D, int RT, int KPT, bool SCORE>
hipError_t launch_one(const SelectParams& p, hipStream_t s) {
  static std::atomic<bool> done[kMaxDevices];
  const size_t lds = SCORE ? (size_t)p.max_pages * sizeof(uint32_t) : 0;
  if (SCORE && KPT > 8) {
    const hipError_t e = ensure_lds_limit((const void*)select_kernel<D, RT, KPT, SCORE>,
                                          KAMERA_MAX_SELECT_PAGES * (int)sizeof(uint32_t), done);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((select_kernel<D, RT, KPT, SCORE>), dim3((uint32_t)p.n_requests * p.n_kv_heads), dim3(kSelThreads),
                     lds, s, p);
  return hipGetLastError();
}

template <int D, int RT>
hipError_t launch_rt(const SelectParams& p, hipStream_t s) {
  const bool small = p.max_pages <= 8 * kSelThreads;
  if (p.n_pieces == 0) return small ? launch_one<D, RT, 8, true>(p, s) : launch_one<D, RT, 32, true>(p, s);
  hipLaunchKernelGGL((score_kernel<D, RT>), dim3((uint32_t)p.n_requests * p.n_pieces * p.n_kv_heads),
                     dim3(kPieceWaves * 64), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return small ? launch_one<64, 1, 8, false>(p, s) : launch_one<64, 1, 32, false>(p, s);
}

}  // namespace

hipError_t launch_select(const SelectParams& p, hipStream_t s) {
  if (p.head_dim == 128) return p.group <= 16 ? launch_rt<128, 1>(p, s) : launch_rt<128, 4>(p, s);
  return p.group <= 16 ? launch_rt<64, 1>(p, s) : launch_rt<64, 4>(p, s);
}

}  // namespace kamera

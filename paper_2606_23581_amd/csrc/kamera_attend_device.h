// Device code shared by the attention kernels: cache formats, page look-up and
// the bookkeeping of which keys a row sees.
#pragma once

#include "kamera_cache_device.h"

namespace kamera {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// v_exp_f32 and v_log_f32: 2^x and log2 x, about 1 ulp
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Two neighbouring bytes of w (the low or the high half) as bf16 times a power
// of two: exact.
template <bool HI>
__device__ __forceinline__ uint32_t e4m3_to_bf16x2(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
}

// The larger of two, NaN if one is: v_maximum3_f32 for two of these, with none of
// the quieting that fmaxf needs.
__device__ __forceinline__ float max2(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// The largest / sum over the lanes l, l ^ 32 and (groups of 16) l ^ 16, l ^ 32.
__device__ __forceinline__ float max_x32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_x16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_x32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float sum_x16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Not a finite number among the elements of w (four e4m3 bytes / two bf16): the
// top bit of each such element.
template <int FMT>
__device__ __forceinline__ uint32_t nonfinite(uint32_t w) {
  if (FMT == KAMERA_CACHE_E4M3) return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
  return ((w & 0x7fff7fffu) + 0x00800080u) & 0x80008000u;
}

// w with these elements zero.
template <int FMT>
__device__ __forceinline__ uint32_t finite_only(uint32_t w) {
  const uint32_t top = nonfinite<FMT>(w);
  const uint32_t all = FMT == KAMERA_CACHE_E4M3 ? (top >> 7) * 0xffu : (top >> 15) * 0xffffu;
  return w & ~all;
}

// a + the sum of a pair of bf16 values, in fp32.
__device__ __forceinline__ float add_pair(uint32_t pair, float a) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3f803f80u), a,
                                         false);
}

// A row's weights are p as the product with V takes them, rounded to bf16, over
// the sum of these, so that they add up to one; lse is taken from the sum of p
// itself, kept beside it where a call asks for lse.  bf16 because the matrix
// instructions take both operands in one type, and V's is bf16 (products in fp32
// have a sixteenth of the rate): with it an output is off by 0.0023 of its size
// (root of the mean square), of which rounding the output alone makes 0.0017.
__device__ __forceinline__ float row_lse(float m, float l_exact) {
  return l_exact == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l_exact)) * 0.69314718055994530942f;
}

// A request of the batch as every wave of a workgroup sees it.
struct Request {
  int n;                             // query tokens
  int kv;                            // cached tokens
  int64_t row0;                      // row of query 0 in q and out
};

__device__ __forceinline__ Request request_of(const AttendParams& p, int r) {
  // all three at once, without a branch between them
  const int n = load_or(p.q_tokens, r, p.n_queries, p.kv_tokens);
  const int kv = load_or(p.kv_tokens, r, 0, p.kv_tokens);
  const int base = load_or(p.q_base, r, 0, p.kv_tokens);
  Request q;
  q.n = min(max(n, 0), p.n_queries);
  q.kv = min(max(kv, 0), p.n_keys);
  q.row0 = p.q_base != nullptr ? (int64_t)base : (int64_t)r * p.n_queries;
  return q;
}

// Query i sees the keys [first, last].
__device__ __forceinline__ int last_key(const AttendParams& p, const Request& q, int i) {
  return p.causal ? q.kv - q.n + i : q.kv - 1;
}
__device__ __forceinline__ int first_key(const AttendParams& p, int last) {
  return p.window > 0 ? max(0, last - p.window + 1) : 0;
}

// 16-token parts of pages, one a lane: where each is in the pool and in the
// request, and its scales.  A wave looks up 64 parts at once and then takes them
// lane by lane as wave-uniform values, so that no look-up stands between two
// steps of the walk.
struct Parts {
  uint64_t k, v;                     // address of its first K and V row, readable also where ok is clear
  int pos;                           // first token of the request
  float ks, vs;
  uint64_t ok;                       // lanes whose part is in the pool
};

// The walk over a request's keys: part n is tokens [16 n, 16 n + 16), or with
// selected pages the n-th part of those.  Parts outside [begin, end) are not
// looked up: what lies before a window may have left the pool.
struct Walk {
  const int32_t* table;
  const int32_t* sel;
  int begin, end;
};

template <int FMT>
__device__ __forceinline__ Parts fetch_parts(const AttendParams& p, const Walk& w, int n, int h) {
  Parts a;
  const int k = (int)fast_div((uint32_t)n, p.fd_page16);
  const int in_page = (n - k * (p.page_size >> 4)) * 16;
  a.pos = n * 16;
  int idx = k;
  int page = -1;
  const bool look = n >= w.begin && n < w.end;
  if (look) {
    if (w.sel != nullptr) {
      idx = w.sel[k];
      a.pos = (int)((uint32_t)idx * (uint32_t)p.page_size) + in_page;
    }
    if (idx >= 0 && idx < p.pt_pages) page = w.table[idx];
  }
  const bool ok = page >= 0 && page < p.n_pool_pages;
  a.ok = __ballot(ok);
  if (look && !ok && p.status != nullptr) atomicOr(p.status, KAMERA_STATUS_BAD_PAGE);
  const int64_t pg = ok ? page : 0, at = look ? in_page : 0;
  a.k = (uint64_t)p.k + pg * p.k_s[0] + at * p.k_s[1] + h * p.k_s[2];
  a.v = (uint64_t)p.v + pg * p.v_s[0] + at * p.v_s[1] + h * p.v_s[2];
  a.ks = a.vs = 1.0f;
  if (FMT == KAMERA_CACHE_E4M3) {
    a.ks = p.k_scale[pg * p.k_scale_s[0] + h * p.k_scale_s[1]];
    a.vs = p.v_scale[pg * p.v_scale_s[0] + h * p.v_scale_s[1]];
  }
  return a;
}

__device__ __forceinline__ int lane_int(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }
// An address that was a number is said to be global memory: a generic (flat) load
// would count as an LDS access too, and every wait for LDS then wait for it.
typedef const __attribute__((address_space(1))) uint8_t* GlobalBytes;
template <typename T>
__device__ __forceinline__ T load_global(GlobalBytes p) {
  return *reinterpret_cast<const __attribute__((address_space(1))) T*>(p);
}
__device__ __forceinline__ GlobalBytes lane_address(uint64_t x, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x, lane);
  const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)(x >> 32), lane);
  return (GlobalBytes)(((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ float lane_float(float x, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane));
}

// A value that is not finite must reach the rows that see its token, and no
// others: 0 * NaN is NaN, so a product over a tile that some row does not see
// whole takes such values as 0, and this adds them to those rows' results in
// memory afterwards (v itself: any positive weight of it is the same).  It runs
// only where the workgroup met one.  Parts [first, end) in groups of `group`, the
// tiles of the caller; all_lo, all_hi: the keys that every row of the block sees.
// Called by all threads after their results are stored.
template <int D, int FMT>
__device__ __forceinline__ void add_nonfinite(const AttendParams& p, const Request& rq, const Walk& w, int first,
                                              int end, int group, int all_lo, int all_hi, int h, int r, int row_first,
                                              int row_end, int split) {
  constexpr int kEl = FMT == KAMERA_CACHE_BF16 ? 2 : 1;
  __threadfence();
  __syncthreads();
  const int col = threadIdx.x % D, sub = threadIdx.x / D, subs = kThreads / D;
  for (int g0 = first; g0 < end; g0 += group) {
    const int lane = threadIdx.x & 63;
    const Parts a = fetch_parts<KAMERA_CACHE_BF16>(p, w, lane < group ? g0 + lane : -1, h);   // no scales needed
    bool partial = false;
    for (int u = 0; u < group; ++u) {
      const int pos = lane_int(a.pos, u);
      partial = partial || ((a.ok >> u) & 1) == 0 || pos + 15 > all_hi || pos < all_lo;
    }
    if (!partial) continue;
    for (int u = 0; u < group; ++u) {
      if (((a.ok >> u) & 1) == 0) continue;
      const int pos = lane_int(a.pos, u);
      const GlobalBytes vb = lane_address(a.v, u) + col * kEl;
      for (int t = 0; t < 16 && pos + t < rq.kv; ++t) {
        float v;
        if (FMT == KAMERA_CACHE_BF16) {
          const uint32_t x = load_global<uint16_t>(vb + t * p.v_s[1]);
          if ((x & 0x7f80u) != 0x7f80u) continue;
          v = bf_lo(x);
        } else {
          const uint32_t x = vb[t * p.v_s[1]];
          if ((x & 0x7fu) != 0x7fu) continue;
          v = __uint_as_float(0x7fc00000u);
        }
        for (int row = row_first + sub; row < row_end; row += subs) {
          const int i = (int)fast_div((uint32_t)row, p.fd_group);
          const int last = last_key(p, rq, i);
          if (pos + t > last || pos + t < first_key(p, last)) continue;
          if (p.n_splits > 1) {
            float* o = p.part_o + ((((int64_t)r * p.n_kv_heads + h) * p.rows_max + row) * p.n_splits + split) * D + col;
            *o += v;
          } else {
            uint16_t* o =
                p.out + (rq.row0 + i) * p.out_s[0] + ((int64_t)h * p.group + (row - i * p.group)) * p.out_s[1] + col;
            *o = (uint16_t)pack_bf16x2(bf_lo(*o) + v, 0.f);
          }
        }
      }
    }
  }
}

}  // namespace kamera

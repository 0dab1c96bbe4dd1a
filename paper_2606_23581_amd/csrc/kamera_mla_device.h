// Device code shared by the two forms of attention over a latent cache: which keys a
// block of rows sees, how the work is divided among workgroups, and page look-up.
#pragma once

#include "kamera_latent.h"
#include "kamera_lds_device.h"

namespace kamera {

constexpr float kLow = -3.402823466e38f;           // running maximum of a row that saw no key
constexpr float kSlack = 8.0f;                     // by how much (in powers of 2) a score may pass the running maximum

// v_exp_f32: 2^x, about 1 ulp
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Memory that no kernel writes while this one runs, at a wave-uniform address: a scalar
// load.
template <typename T>
__device__ __forceinline__ T uniform_load(const T* p) {
  return *(const __attribute__((address_space(4))) T*)(uintptr_t)p;
}

// First row of a request's in q and out, or of its expanded keys.
__device__ __forceinline__ int64_t first_row(const int32_t* base, int r, int most) {
  return base != nullptr ? (int64_t)uniform_load(base + r) : (int64_t)r * most;
}

// The larger of two, NaN if one is.
__device__ __forceinline__ float max2(float a, float b) { return __builtin_elementwise_maximum(a, b); }

__device__ __forceinline__ float max_x32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_x32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// a + the sum of a pair of bf16 values, in fp32.
__device__ __forceinline__ float add_pair(uint32_t pair, float a) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3f803f80u), a,
                                         false);
}

// A row's weights are p as the product with the values takes them, rounded to bf16
// (the matrix instructions take both operands in one type, and the values' is bf16),
// over the sum of these, so that they add up to one; lse is taken from the sum of p
// itself.
__device__ __forceinline__ float row_lse(float m, float l_exact) {
  return l_exact == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l_exact)) * 0.69314718055994530942f;
}

// A block of rows of one request: task = (request, head, row block), the block last.
// Row i * group + g of a (request, head) is query i, head g of the group.
struct Block {
  int r, h, rb;
  int n, kv;                         // query tokens, cached tokens
  int row_first, row_end;            // rows of the (request, head); none where row_first >= row_end
  int lo, hi;                        // keys that some row sees ...
  int all_lo, all_hi;                // ... and that every row sees
};

__device__ __forceinline__ int mla_last_key(const MlaParams& p, int n, int kv, int i) {
  return p.causal ? kv - n + i : kv - 1;
}
__device__ __forceinline__ int mla_first_key(const MlaParams& p, int last) {
  return p.window > 0 ? max(0, last - p.window + 1) : 0;
}

// UNIFORM: the task is the same for the whole wave, and its lengths are scalar loads.
template <bool UNIFORM = true>
__device__ __forceinline__ Block block_of(const MlaParams& p, uint32_t task) {
  Block b;
  uint32_t d = fast_div(task, p.fd_blocks);
  b.rb = (int)(task - d * p.n_row_blocks);
  const uint32_t r = fast_div(d, p.fd_heads);
  b.h = (int)(d - r * p.task_heads);
  b.r = (int)r;
  // both at once, without a branch between them
  const int32_t* q_tokens = p.q_tokens != nullptr ? p.q_tokens : p.kv_tokens;
  const int n = UNIFORM ? uniform_load(q_tokens + r) : q_tokens[r];
  const int kv = UNIFORM ? uniform_load(p.kv_tokens + r) : p.kv_tokens[r];
  b.n = p.q_tokens != nullptr ? min(max(n, 0), p.n_queries) : p.n_queries;
  b.kv = min(max(kv, 0), p.n_keys);
  const int rows = b.n * p.group;
  b.row_first = b.rb * p.rows_block;
  b.row_end = min(rows, b.row_first + p.rows_block);
  b.lo = b.all_lo = 0;
  b.hi = b.all_hi = -1;
  if (b.row_first >= b.row_end) return b;
  const int first = mla_last_key(p, b.n, b.kv, (int)fast_div((uint32_t)b.row_first, p.fd_group));
  const int last = mla_last_key(p, b.n, b.kv, (int)fast_div((uint32_t)b.row_end - 1, p.fd_group));
  b.hi = min(last, b.kv - 1);
  b.all_hi = min(first, b.kv - 1);
  b.lo = mla_first_key(p, first);
  b.all_lo = mla_first_key(p, last);
  return b;
}

// Units of UNIT keys that a block walks: those from lo / UNIT on.  A block that sees
// no key has one all the same, so that its rows are written.
template <int UNIT>
__device__ __forceinline__ int units_of(const Block& b) {
  if (b.row_first >= b.row_end) return 0;
  return b.hi < b.lo ? 1 : b.hi / UNIT - b.lo / UNIT + 1;
}

// What a workgroup does: units [u0, u1) of consecutive tasks, from task `task` on, of
// which `skip` units belong to workgroups before it.
struct Share {
  uint32_t task;
  int skip;
  int units;
};

// The tasks' units, divided evenly: workgroup w takes the w-th range of `per` units.
// Every wave adds up all tasks' units, some a lane (a few loads and shuffles, no
// barrier); the first workgroup leaves the sums, and each its first task, for the kernel
// that joins the parts.
template <int UNIT>
__device__ __forceinline__ Share divide(const MlaParams& p, uint32_t w) {
  const int lane = threadIdx.x & 63, each = (p.n_tasks + 63) / 64;
  const int t0 = min(lane * each, p.n_tasks), t1 = min(t0 + each, p.n_tasks);
  int sum = 0;
  for (int t = t0; t < t1; ++t) sum += units_of<UNIT>(block_of<false>(p, t));
  int x = sum;                                     // inclusive sums over the lanes
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_up(x, d);
    x += lane >= d ? y : 0;
  }
  const int total = __builtin_amdgcn_readlane(x, 63);
  const int per = max((total + p.n_parts - 1) / p.n_parts, p.min_units);
  const int64_t begin = (int64_t)w * per;
  int at = x - sum, task = p.n_tasks, skip = 0;    // units before this lane's tasks
  const bool mine = begin >= at && begin < x, first = w == 0 && threadIdx.x < 64;
  if (mine || first) {
    for (int t = t0; t < t1; ++t) {
      const int u = each == 1 ? sum : units_of<UNIT>(block_of<false>(p, t));
      if (first) p.prefix[t] = at;
      if (begin >= at && begin < at + u) {
        task = t;
        skip = (int)(begin - at);
      }
      at += u;
    }
  }
  const uint64_t found = __ballot(mine);
  const int from = found != 0 ? __builtin_ctzll(found) : 0;
  Share s;
  s.task = (uint32_t)__builtin_amdgcn_readlane(task, from);
  s.skip = __builtin_amdgcn_readlane(skip, from);
  s.units = begin >= total ? 0 : (int)min((int64_t)per, total - begin);
  if (first && lane == 0) {
    p.prefix[p.n_tasks] = total;
    p.prefix[p.n_tasks + 1] = per;
  }
  if (threadIdx.x == 0) p.prefix[p.n_tasks + 2 + w] = (int)s.task;
  return s;
}

// 16-token parts of a request's pages, one a lane: address of the part's first row and
// which lanes' are in the pool.  Parts outside [begin, end) are not looked up: what
// lies before a window may have left the pool.
struct PoolParts {
  uint64_t at;                       // readable also where ok is clear
  uint64_t ok;
};

__device__ __forceinline__ PoolParts fetch_pool_parts(const MlaParams& p, int r, int n, int begin, int end) {
  PoolParts a;
  const bool look = n >= begin && n < end;
  int page = -1;
  const int k = (int)fast_div((uint32_t)(look ? n : 0), p.fd_page16);
  const int in_page = (n - k * (p.page_size >> 4)) * 16;
  if (look) page = p.page_table[(int64_t)r * p.pt_stride + k];
  const bool ok = page >= 0 && page < p.n_pool_pages;
  a.ok = __ballot(ok);
  if (look && !ok && p.status != nullptr) atomicOr(p.status, KAMERA_STATUS_BAD_PAGE);
  a.at = (uint64_t)p.pool + (ok ? page * p.pool_s[0] + in_page * p.pool_s[1] : 0);
  return a;
}

__device__ __forceinline__ uint64_t lane_u64(uint64_t x, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x, lane);
  const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)(x >> 32), lane);
  return ((uint64_t)hi << 32) | lo;
}

// A row of zeros: where a key that no row of a block may see would be loaded.
static __device__ __attribute__((aligned(16))) uint32_t g_zero_row[(512 + kRopeCols) / 2];

// The keys [pos, pos + n) hold some that a row of the block sees and another does not.
__device__ __forceinline__ bool mixed(const Block& b, int pos, int n) {
  return min(pos + n - 1, b.hi) > b.all_hi || max(pos, b.lo) < b.all_lo;
}

// A 16-byte chunk of LDS with what is not finite zero; whether there was any.
__device__ __forceinline__ bool clean_chunk(uint32_t at) {
  __attribute__((address_space(3))) u32x4* c = (__attribute__((address_space(3))) u32x4*)(uintptr_t)at;
  u32x4 w = *c;
  uint32_t odd = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t top = ((w[k] & 0x7fff7fffu) + 0x00800080u) & 0x80008000u;
    odd |= top;
    w[k] &= ~((top >> 15) * 0xffffu);
  }
  if (odd != 0) *c = w;
  return odd != 0;
}

// A value that is not finite must reach the rows that see its key, and no others:
// 0 * NaN is NaN, so the product over keys that some rows see and others do not leaves
// such values out, and this adds them to those rows' results in memory afterwards (v
// itself: any positive weight of it is the same).  It runs only where the workgroup met
// one.  Keys [from, to) in steps of `step`; value_at(key): its row of values, or null
// where its page is outside the pool.  Called by all threads after their results are
// stored; a column is one thread's.
template <typename F>
__device__ __forceinline__ void add_nonfinite(const MlaParams& p, const Block& b, int from, int to, int step, int cols,
                                              bool direct, int64_t part, int64_t row0, F value_at) {
  __threadfence();
  __syncthreads();
  for (int pos = from; pos < to; pos += step) {
    if (!mixed(b, pos, step)) continue;
    for (int key = max(pos, b.lo); key <= min(pos + step - 1, b.hi); ++key) {
      const uint16_t* v = value_at(key);
      if (v == nullptr) continue;
      for (int c = threadIdx.x; c < cols; c += blockDim.x) {
        const uint32_t x = v[c];
        if ((x & 0x7f80u) != 0x7f80u) continue;
        for (int row = b.row_first; row < b.row_end; ++row) {
          const int i = (int)fast_div((uint32_t)row, p.fd_group), last = mla_last_key(p, b.n, b.kv, i);
          if (key > last || key < mla_first_key(p, last)) continue;
          if (direct) {
            uint16_t* o = p.out + (row0 + i) * p.out_s[0] + ((int64_t)b.h * p.group + row - i * p.group) * p.out_s[1] + c;
            *o = (uint16_t)pack_bf16x2(bf_lo(*o) + bf_lo(x), 0.f);
          } else {
            p.part_o[(part + row - b.row_first) * cols + c] += bf_lo(x);
          }
        }
      }
    }
  }
}

}  // namespace kamera

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

__device__ __forceinline__ Block block_from(const MlaParams& p, int r, int h, int rb, int n, int kv) {
  Block b;
  b.r = r;
  b.h = h;
  b.rb = rb;
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

// The block of a task that is the same for the whole wave.
__device__ __forceinline__ Block block_of(const MlaParams& p, uint32_t task) {
  const uint32_t d = fast_div(task, p.fd_blocks), r = fast_div(d, p.fd_heads);
  // both lengths at once, without a branch between them
  const int n = uniform_load((p.q_tokens != nullptr ? p.q_tokens : p.kv_tokens) + r), kv = uniform_load(p.kv_tokens + r);
  return block_from(p, (int)r, (int)(d - r * p.task_heads), (int)(task - d * p.n_row_blocks), n, kv);
}

// Units of `unit` keys that a block walks: those from lo / unit on.  A block that sees
// no key has one all the same, so that its rows are written.
__device__ __forceinline__ int units_of(const Block& b, int unit) {
  if (b.row_first >= b.row_end) return 0;
  return b.hi < b.lo ? 1 : b.hi / unit - b.lo / unit + 1;
}

// What a block costs, in units: p.fixed of them, in which nothing is walked, for taking it
// up and storing its results, and its own.  Without the first, workgroups with many short
// blocks end last.
__device__ __forceinline__ int cost_of(const MlaParams& p, const Block& b, int unit) {
  const int u = units_of(b, unit);
  return u > 0 ? u + p.fixed : 0;
}

// What a workgroup does: costs `units` of consecutive tasks, from task `task` on, of which
// `skip` belong to workgroups before it.
struct Share {
  uint32_t task;
  int skip;
  int units;
  int begin;                         // cost before its range
};

// The units [from, to) of a task that a workgroup walks, of its `total`.
struct Segment {
  int from, to, total;
  __device__ __forceinline__ bool whole() const { return from == 0 && to == total; }
};

// The next task's part of a share; false where there is nothing to walk in it.
__device__ __forceinline__ bool take_segment(const MlaParams& p, const Block& b, int unit, uint32_t task, const Share& share,
                                             int& units, int skip, Segment& s) {
  s.total = units_of(b, unit);
  if (s.total == 0) return false;
  if (p.n_parts > 0 && skip == 0 && threadIdx.x == 0) p.prefix[task] = share.begin + share.units - units;
  const int take = min(s.total + p.fixed - skip, units);
  units -= take;
  s.from = max(skip - p.fixed, 0);
  s.to = max(skip + take - p.fixed, 0);
  return s.from < s.to;
}

// Inclusive sums over the lanes.
__device__ __forceinline__ int lane_sums(int x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_up(x, d);
    x += lane >= d ? y : 0;
  }
  return x;
}

// The tasks' costs, divided evenly: workgroup w takes the w-th range of `per` units.
// Every wave adds up all requests' costs: so many lanes a request as it has row blocks,
// a request's heads alike.
template <int UNIT>
__device__ __forceinline__ Share divide(const MlaParams& p, uint32_t w) {
  const int lane = threadIdx.x & 63, width = p.lanes, slot = lane & (width - 1), each = 64 / width;
  // cost of one head of the lane's request in this pass, the same in all its lanes
  auto units_in = [&](int pass) {
    const int r = pass * each + lane / width;
    int s = 0;
    if (r < p.n_requests) {
      const int n = (p.q_tokens != nullptr ? p.q_tokens : p.kv_tokens)[r], kv = p.kv_tokens[r];
      for (int rb = slot; rb < p.n_row_blocks; rb += width) s += cost_of(p, block_from(p, r, 0, rb, n, kv), UNIT);
    }
    for (int d = 1; d < width; d *= 2) s += __shfl_xor(s, d);
    return s;
  };
  const int passes = (p.n_requests + each - 1) / each;
  int total = 0, one = 0, sums = 0;
  for (int i = 0; i < passes; ++i) {
    one = units_in(i);
    sums = lane_sums(slot == 0 ? one * p.task_heads : 0);
    total += __builtin_amdgcn_readlane(sums, 63);
  }
  const int per = max((total + p.n_parts - 1) / p.n_parts, p.min_units);
  const int64_t begin = (int64_t)w * per;
  Share s;
  s.task = p.n_tasks;
  s.skip = 0;
  s.units = begin >= total ? 0 : (int)min((int64_t)per, total - begin);
  if (w == 0 && threadIdx.x == 0) p.prefix[p.n_tasks] = per;
  if (s.units > 0) {
    // the request, its head, its row block
    int at = 0, r = 0, rest = 0, head_units = 1;
    for (int i = 0; i < passes; ++i) {
      if (passes > 1) {
        one = units_in(i);
        sums = lane_sums(slot == 0 ? one * p.task_heads : 0);
      }
      const int mine = slot == 0 ? one * p.task_heads : 0;
      const uint64_t found = __ballot(begin >= at + sums - mine && begin < at + sums);
      if (found != 0) {
        const int from = __builtin_ctzll(found);
        r = i * each + from / width;
        rest = (int)(begin - at) - __builtin_amdgcn_readlane(sums - mine, from);
        head_units = __builtin_amdgcn_readlane(one, from);
        break;
      }
      at += __builtin_amdgcn_readlane(sums, 63);
    }
    const int h = rest / head_units;
    rest -= h * head_units;
    const int n = uniform_load((p.q_tokens != nullptr ? p.q_tokens : p.kv_tokens) + r), kv = uniform_load(p.kv_tokens + r);
    for (int rb0 = 0; rb0 < p.n_row_blocks; rb0 += 64) {
      const int u = rb0 + lane < p.n_row_blocks ? cost_of(p, block_from(p, r, h, rb0 + lane, n, kv), UNIT) : 0;
      const int x = lane_sums(u);
      const uint64_t found = __ballot(rest >= x - u && rest < x);
      if (found != 0) {
        const int from = __builtin_ctzll(found);
        s.task = ((uint32_t)r * p.task_heads + h) * p.n_row_blocks + rb0 + from;
        s.skip = rest - __builtin_amdgcn_readlane(x - u, from);
        break;
      }
      rest -= __builtin_amdgcn_readlane(x, 63);
    }
    s.task = __builtin_amdgcn_readfirstlane(s.task);
    s.skip = __builtin_amdgcn_readfirstlane(s.skip);
  }
  // for the kernel that joins the parts: the task that each range begins in (and, from
  // take_segment, the cost before each task)
  if (threadIdx.x == 0) p.prefix[p.n_tasks + 1 + w] = (int)s.task;
  s.begin = (int)begin;
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
// itself: any positive weight of it is the same; with a weight of 0 an infinity stays one
// here and is NaN in the product and the join, not finite in either).  It runs only where
// the workgroup met one.  Keys [from, to) in steps of `step`; value_at(key): its row of values, or null
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

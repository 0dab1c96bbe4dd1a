// kamera_attend_paged, few query rows: attention over the paged cache where
// reading the cache is the work (decode, a few speculated tokens).
//
// Rows.  The query rows that share a KV head -- every query token's `group`
// heads -- are one matrix of rows (token, head), taken 16 at a time as the N
// side of the 16x16x32 bf16 MFMA, NR such tiles a workgroup (one, or two of an
// 8-bit cache), so a key is fetched and converted once for all of them.
//
// A step of a wave is 32 tokens, two 16-token parts that each lie in one page.
//   S^T = K Q^T: K's rows are the A operand; a lane takes 16 bytes of one
//     token's row at a time, which is 16 columns of e4m3 or 8 of bf16.  Which
//     columns make up a K-step of the product is free, so Q is loaded in the
//     order that these loads give.  Lane l gets the scores of row l % 16 for
//     tokens 4 (l / 16) + i of each part.
//   O^T = V^T P^T: P goes in as the B operand straight from those registers,
//     when the product's inner index is read as (part, token): lane group g holds
//     tokens 4g .. 4g+3 of part 0, then of part 1.  V^T as the A operand needs
//     the same 8 tokens of one column in a lane: it loads VC = D / 16
//     neighbouring columns of each of its 8 tokens, pairs tokens with v_perm,
//     and feeds product b the columns c * VC + b, c = l % 16.  Nothing passes
//     through LDS, and each row is read in whole 64- to 256-byte runs.
// e4m3 becomes bf16 with the page's power-of-two scale inside the conversion
// (v_cvt_scalef32_pk_bf16_fp8, exact).
//
// Softmax: scores in powers of two (scale * log2 e folded in), fp32.  A row's
// running maximum moves only when a score passes it by more than 8, so p <= 2^8
// and the sums stay far inside fp32, while most steps skip the rescaling; the
// row sum stays per lane until the end.
//
// Bound by HBM: 64 ragged requests of 8 x 8 heads over up to 8192 keys in 8 bits
// 137 us, 4.9 TB/s; 16 requests of 32 heads over 4096-key windows in bf16 183 us, 5.4
// TB/s.  The next step's loads are in flight while a step is computed; the four
// waves of a workgroup take steps in turn and join in LDS; with few rows the keys
// are split over workgroups too, and attend_join_kernel joins (65536 keys of one
// request: 24.0 us of reading, 5.6 TB/s, and 4.4 us of joining).

#include <algorithm>

#include "kamera_attend_device.h"

namespace kamera {

namespace {

constexpr int kAttThreads = 256;
constexpr int kAttWaves = kAttThreads / 64;
constexpr float kLow = -3.402823466e38f;           // running maximum of a row that saw no key
constexpr float kSlack = 8.0f;

template <int D, int FMT>
struct Tile {
  static constexpr int kEl = FMT == KAMERA_CACHE_BF16 ? 2 : 1;   // bytes an element
  static constexpr int kLoads = D * kEl / 64;      // 16-byte loads of a K row by its 4 lanes
  static constexpr int kSteps = D / 32;            // K-steps of the score product
  static constexpr int VC = D / 16;                // V columns a lane
  static constexpr int kVW = VC * kEl / 4;         // dwords of a V load (1, 2 or 4)
};

// The loads of one step: two parts of 16 tokens.
template <int D, int FMT>
struct Step {
  u32x4 k[2][Tile<D, FMT>::kLoads];
  uint32_t v[2][4][Tile<D, FMT>::kVW];
  float ks[2], vs[2];
  int pos[2];
  uint32_t ok;                                     // bit u: part u is in the pool
};

// Parts `lane` and `lane + 1` of a batch.
template <int D, int FMT>
__device__ __forceinline__ void load_step(const AttendParams& p, const Parts& a, int lane, uint32_t k_lane, uint32_t v_lane,
                                          Step<D, FMT>& s) {
  using T = Tile<D, FMT>;
  s.ok = (uint32_t)(a.ok >> lane) & 3u;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    s.pos[u] = lane_int(a.pos, lane + u);
    const GlobalBytes kb = lane_address(a.k, lane + u);
    const GlobalBytes vb = lane_address(a.v, lane + u);
#pragma unroll
    for (int i = 0; i < T::kLoads; ++i) s.k[u][i] = load_global<u32x4>(kb + k_lane + i * 64);
    const uint32_t vt = (uint32_t)p.v_s[1];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const GlobalBytes at = vb + v_lane + j * vt;
      if (T::kVW == 1) s.v[u][j][0] = load_global<uint32_t>(at);
      else if (T::kVW == 2) {
        const u32x2 w = load_global<u32x2>(at);
        s.v[u][j][0] = w.x;
        s.v[u][j][T::kVW > 1 ? 1 : 0] = w.y;
      } else {
        const u32x4 w = load_global<u32x4>(at);
#pragma unroll
        for (int e = 0; e < T::kVW; ++e) s.v[u][j][e] = u4_get(w, e);
      }
    }
  }
  // after the loads: these wait for the look-up's scales
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    s.ks[u] = lane_float(a.ks, lane + u);
    s.vs[u] = lane_float(a.vs, lane + u);
  }
}

// The A operand of K-step ks for part u.
template <int D, int FMT>
__device__ __forceinline__ bf16x8 k_frag(const Step<D, FMT>& s, int u, int ks) {
  if (FMT == KAMERA_CACHE_BF16) return __builtin_bit_cast(bf16x8, s.k[u][FMT == KAMERA_CACHE_BF16 ? ks : 0]);
  const u32x4 w = s.k[u][FMT == KAMERA_CACHE_BF16 ? 0 : ks >> 1];
  const uint32_t a = (ks & 1) ? w.z : w.x, b = (ks & 1) ? w.w : w.y;
  u32x4 f;
  f.x = e4m3_to_bf16x2<false>(a, s.ks[u]);
  f.y = e4m3_to_bf16x2<true>(a, s.ks[u]);
  f.z = e4m3_to_bf16x2<false>(b, s.ks[u]);
  f.w = e4m3_to_bf16x2<true>(b, s.ks[u]);
  return __builtin_bit_cast(bf16x8, f);
}

// The A operand of column b (of VC): token pairs of both parts.
template <int D, int FMT>
__device__ __forceinline__ bf16x8 v_frag(const Step<D, FMT>& s, int b) {
  u32x4 f;
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      uint32_t r;
      if (FMT == KAMERA_CACHE_BF16) {
        const uint32_t w0 = s.v[u][2 * t][b >> 1], w1 = s.v[u][2 * t + 1][b >> 1];
        r = __builtin_amdgcn_perm(w1, w0, (b & 1) ? 0x07060302u : 0x05040100u);
      } else {
        // bytes (w0.0, w1.0, w0.1, w1.1) or (w0.2, w1.2, w0.3, w1.3): two columns' pairs
        const uint32_t w0 = s.v[u][2 * t][b >> 2], w1 = s.v[u][2 * t + 1][b >> 2];
        const uint32_t x = __builtin_amdgcn_perm(w1, w0, (b & 2) ? 0x07030602u : 0x05010400u);
        r = (b & 1) ? e4m3_to_bf16x2<true>(x, s.vs[u]) : e4m3_to_bf16x2<false>(x, s.vs[u]);
      }
      if (u == 0 && t == 0) f.x = r;
      if (u == 0 && t == 1) f.y = r;
      if (u == 1 && t == 0) f.z = r;
      if (u == 1 && t == 1) f.w = r;
    }
  return __builtin_bit_cast(bf16x8, f);
}

// Zero the V rows of this lane's tokens outside [lo, hi], and what is not finite
// in the others (the result says whether there was any; see add_nonfinite).
// A part that is not there has been read from the pool's first page: its scale,
// which may be no number, goes too.
template <int D, int FMT>
__device__ __forceinline__ bool clear_unseen(Step<D, FMT>& s, int g, int lo, int hi) {
  uint32_t odd = 0;
#pragma unroll
  for (int u = 0; u < 2; ++u) s.vs[u] = (s.ok >> u) & 1 ? s.vs[u] : 1.0f;
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int pos = s.pos[u] + 4 * g + j;
      const bool keep = ((s.ok >> u) & 1) && pos >= lo && pos <= hi;
#pragma unroll
      for (int e = 0; e < Tile<D, FMT>::kVW; ++e) {
        const uint32_t w = keep ? s.v[u][j][e] : 0u;
        odd |= nonfinite<FMT>(w);
        s.v[u][j][e] = finite_only<FMT>(w);
      }
    }
  return odd != 0;
}

}  // namespace

template <int D, int FMT, int NR>
__global__ __launch_bounds__(kAttThreads, 2) void attend_rows_kernel(AttendParams) {
  using T = Tile<D, FMT>;
  const AttendParams& p = kernel_params<AttendParams>();
  constexpr int kPad = 4;
  __shared__ float s_o[kAttWaves][16][D + kPad];
  __shared__ float s_ml[kAttWaves][NR * 16][3];
  __shared__ int s_odd[kAttWaves];                 // a value that is not finite was taken as 0

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c16 = lane & 15, g = lane >> 4;
  uint32_t w = blockIdx.x, d;
  d = fast_div(w, p.fd_splits);
  const int split = (int)(w - d * p.n_splits);
  w = d;
  d = fast_div(w, p.fd_blocks);
  const int rb = (int)(w - d * p.n_row_blocks);
  w = d;
  d = fast_div(w, p.fd_heads);
  const int h = (int)(w - d * p.n_kv_heads), r = (int)d;

  const Request rq = request_of(p, r);
  const int rows = rq.n * p.group;                 // rows of this KV head
  const int row_first = rb * NR * 16, row_end = min(rows, row_first + NR * 16);
  if (row_first >= rows) return;
  const int i_first = (int)fast_div((uint32_t)row_first, p.fd_group);
  const int i_last = (int)fast_div((uint32_t)row_end - 1, p.fd_group);

  // keys that some row of the block sees, and those that every row sees
  Walk walk;
  walk.table = p.page_table + (int64_t)r * p.pt_stride;
  walk.sel = nullptr;
  const int hi = min(last_key(p, rq, i_last), rq.kv - 1), all_hi = last_key(p, rq, i_first);
  const int lo = first_key(p, last_key(p, rq, i_first)), all_lo = first_key(p, last_key(p, rq, i_last));
  walk.begin = lo >> 4;
  walk.end = (hi >> 4) + 1;
  if (p.sel != nullptr) {
    const int64_t at = (int64_t)r * p.n_kv_heads + h;
    walk.sel = p.sel + at * p.sel_stride;
    walk.begin = 0;
    walk.end = min(max(uniform_load(p.sel_count + at), 0), p.sel_stride) * (p.page_size >> 4);
  }
  const int step0 = walk.begin >> 1, step1 = (walk.end + 1) >> 1;
  const int n_steps = max(step1 - step0, 0);
  const int per = (n_steps + p.n_splits - 1) / p.n_splits;
  const int s_begin = step0 + split * per, s_end = min(step1, s_begin + per);

  f32x4 o[NR][T::VC];
  float m[NR], l[NR], lx[NR];
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    m[t] = kLow;
    l[t] = lx[t] = 0.f;
#pragma unroll
    for (int b = 0; b < T::VC; ++b) o[t][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const uint32_t k_lane = (uint32_t)(c16 * p.k_s[1]) + g * 16;
  const uint32_t v_lane = (uint32_t)(4 * g * p.v_s[1]) + c16 * T::VC * T::kEl;

  // The wave's steps s_begin + wave + 4 j, looked up 32 at a time: lane i has part
  // i % 2 of step i / 2 of the batch.  The look-up of a batch is issued a batch ahead.
  const int first = s_begin + wave, n_own = s_end > first ? (s_end - first + kAttWaves - 1) / kAttWaves : 0;
  auto batch = [&](int j) {
    return fetch_parts<FMT>(p, walk, j < n_own ? 2 * (first + (j + (lane >> 1)) * kAttWaves) + (lane & 1) : -1, h);
  };
  Step<D, FMT> cur, nxt;
  bool odd = false;
  Parts parts = batch(0), ahead = parts;

  // Q rows as B operands, in the column order of the K loads; rows past the end are zero
  bf16x8 qf[NR][T::kSteps];
  int row_hi[NR], row_lo[NR];
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    const int row = row_first + t * 16 + c16;
    const int i = (int)fast_div((uint32_t)row, p.fd_group), hq = row - i * p.group;
    const bool there = row < row_end;
    row_hi[t] = there ? min(last_key(p, rq, i), rq.kv - 1) : -1;
    row_lo[t] = there ? first_key(p, last_key(p, rq, i)) : 0;
    const uint16_t* src = p.q + (rq.row0 + i) * p.q_s[0] + ((int64_t)h * p.group + hq) * p.q_s[1];
#pragma unroll
    for (int ks = 0; ks < T::kSteps; ++ks) {
      const int col = FMT == KAMERA_CACHE_BF16 ? (g + 4 * ks) * 8 : (g + 4 * (ks >> 1)) * 16 + (ks & 1) * 8;
      u32x4 x = {0u, 0u, 0u, 0u};
      if (there) x = *reinterpret_cast<const u32x4*>(src + col) ^ p.q_sign;
      qf[t][ks] = __builtin_bit_cast(bf16x8, x);
    }
  }

  if (n_own > 0) load_step<D, FMT>(p, parts, 0, k_lane, v_lane, cur);
  if (n_own > 32) ahead = batch(32);
  for (int j = 0; j < n_own; ++j) {
    if (j + 1 < n_own) {
      if (((j + 1) & 31) == 0) {
        parts = ahead;
        ahead = batch(j + 33);
      }
      load_step<D, FMT>(p, parts, 2 * ((j + 1) & 31), k_lane, v_lane, nxt);
    }

    // a step that some row does not see whole
    const bool partial = cur.ok != 3u || max(cur.pos[0], cur.pos[1]) + 15 > all_hi || min(cur.pos[0], cur.pos[1]) < all_lo;
    if (partial) odd |= clear_unseen<D, FMT>(cur, g, lo, hi);

    f32x4 sc[NR][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int t = 0; t < NR; ++t) sc[t][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < T::kSteps; ++ks) {
        const bf16x8 a = k_frag<D, FMT>(cur, u, ks);
#pragma unroll
        for (int t = 0; t < NR; ++t) sc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[t][ks], sc[t][u], 0, 0, 0);
      }
    }

    bf16x8 pf[NR];
#pragma unroll
    for (int t = 0; t < NR; ++t) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[u * 4 + i] = sc[t][u][i];
      if (partial) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int pos = cur.pos[u] + 4 * g + i;
            const bool seen = ((cur.ok >> u) & 1) && pos >= row_lo[t] && pos <= row_hi[t];
            x[u * 4 + i] = seen ? x[u * 4 + i] : -INFINITY;
          }
      }
      float top = max2(max2(max2(x[0], x[1]), max2(x[2], x[3])), max2(max2(x[4], x[5]), max2(x[6], x[7]))) * p.scale2;
      if (__ballot(top > m[t] + kSlack) != 0) {
        top = max_x32(max_x16(top));
        const float m_new = fmaxf(m[t], top);
        const float down = exp2_fast(m[t] - m_new);
        m[t] = m_new;
        l[t] *= down;
        lx[t] *= down;
#pragma unroll
        for (int b = 0; b < T::VC; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[t][b][i] *= down;
      }
      u32x4 pk;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = exp2_fast(__builtin_fmaf(x[i], p.scale2, -m[t]));
      if (p.lse != nullptr) lx[t] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
      pk.x = pack_bf16x2(x[0], x[1]);
      pk.y = pack_bf16x2(x[2], x[3]);
      pk.z = pack_bf16x2(x[4], x[5]);
      pk.w = pack_bf16x2(x[6], x[7]);
      l[t] = add_pair(pk.w, add_pair(pk.z, add_pair(pk.y, add_pair(pk.x, l[t]))));
      pf[t] = __builtin_bit_cast(bf16x8, pk);
    }

#pragma unroll
    for (int b = 0; b < T::VC; ++b) {
      const bf16x8 a = v_frag<D, FMT>(cur, b);
#pragma unroll
      for (int t = 0; t < NR; ++t) o[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pf[t], o[t][b], 0, 0, 0);
    }
    cur = nxt;
  }

  // join the four waves
  odd = __ballot(odd) != 0;
  if (lane == 0) s_odd[wave] = odd;
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    l[t] = sum_x32(sum_x16(l[t]));
    lx[t] = sum_x32(sum_x16(lx[t]));
    if (g == 0) {
      s_ml[wave][t * 16 + c16][0] = m[t];
      s_ml[wave][t * 16 + c16][1] = l[t];
      s_ml[wave][t * 16 + c16][2] = lx[t];
    }
  }
  __syncthreads();
  const int row_t = threadIdx.x >> 4, col = (threadIdx.x & 15) * T::VC;   // output: 16 rows x 16 threads
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    float top = kLow;
#pragma unroll
    for (int k = 0; k < kAttWaves; ++k) top = fmaxf(top, s_ml[k][t * 16 + c16][0]);
    const float down = exp2_fast(m[t] - top);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int b = 0; b < T::VC; ++b) s_o[wave][c16][(4 * g + i) * T::VC + b] = o[t][b][i] * down;
    __syncthreads();
    const int row = row_first + t * 16 + row_t;
    if (row < row_end) {
      float mm = kLow, ll = 0.f, lxx = 0.f;
#pragma unroll
      for (int k = 0; k < kAttWaves; ++k) mm = fmaxf(mm, s_ml[k][t * 16 + row_t][0]);
#pragma unroll
      for (int k = 0; k < kAttWaves; ++k) {
        const float f = exp2_fast(s_ml[k][t * 16 + row_t][0] - mm);
        ll += s_ml[k][t * 16 + row_t][1] * f;
        lxx += s_ml[k][t * 16 + row_t][2] * f;
      }
      float a[T::VC];
#pragma unroll
      for (int b = 0; b < T::VC; ++b)
        a[b] = (s_o[0][row_t][col + b] + s_o[1][row_t][col + b]) + (s_o[2][row_t][col + b] + s_o[3][row_t][col + b]);
      if (p.n_splits > 1) {
        const int64_t at = (((int64_t)r * p.n_kv_heads + h) * p.rows_max + row) * p.n_splits + split;
#pragma unroll
        for (int b = 0; b < T::VC; b += 4)
          *reinterpret_cast<f32x4*>(p.part_o + at * D + col + b) = f32x4{a[b], a[b + 1], a[b + 2], a[b + 3]};
        if ((threadIdx.x & 15) == 0) *reinterpret_cast<f32x4*>(p.part_ml + at * 4) = f32x4{mm, ll, lxx, 0.f};
      } else {
        const int i = (int)fast_div((uint32_t)row, p.fd_group);
        const int64_t hq = (int64_t)h * p.group + (row - i * p.group);
        const float inv = ll == 0.f ? 0.f : 1.0f / ll;
        uint16_t* dst = p.out + (rq.row0 + i) * p.out_s[0] + hq * p.out_s[1] + col;
#pragma unroll
        for (int b = 0; b < T::VC; b += 4)
          *reinterpret_cast<u32x2*>(dst + b) =
              u32x2{pack_bf16x2(a[b] * inv, a[b + 1] * inv), pack_bf16x2(a[b + 2] * inv, a[b + 3] * inv)};
        if (p.lse != nullptr && (threadIdx.x & 15) == 0)
          p.lse[(rq.row0 + i) * p.lse_s[0] + hq * p.lse_s[1]] = row_lse(mm, lxx);
      }
    }
    __syncthreads();
  }
  if (s_odd[0] | s_odd[1] | s_odd[2] | s_odd[3])
    add_nonfinite<D, FMT>(p, rq, walk, 2 * s_begin, 2 * s_end, 2, all_lo, all_hi, h, r, row_first, row_end, split);
}

// Joins the parts of each row: with M the largest of the parts' maxima m_s,
// out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s.  A thread takes four columns
// of every WAYS-th part, eight parts at a time with all their loads in flight; the
// ways of a row meet in LDS.  Up to 8 parts one way a row and several rows a
// workgroup (a workgroup a row took 88 us for 16384 rows of 2 parts), else 8 ways.
template <int D, int WAYS>
__global__ __launch_bounds__(kAttThreads) void attend_join_kernel(AttendParams) {
  const AttendParams& p = kernel_params<AttendParams>();
  constexpr int kCols = D / 4, kRows = kAttThreads / (kCols * WAYS), kChunk = 8;
  static_assert(WAYS == 1 || kRows == 1 || D == 64, "");
  __shared__ f32x4 s_o[WAYS > 1 ? kRows * WAYS : 1][kCols];
  __shared__ float s_ml[WAYS > 1 ? kRows * WAYS : 1][3];
  const int tid = threadIdx.x, col = tid % kCols, way = tid / kCols % WAYS, slot = tid / kCols;
  const uint32_t task = blockIdx.x * kRows + tid / (kCols * WAYS);
  if (WAYS == 1 && task >= (uint32_t)p.n_join) return;
  uint32_t w = min(task, (uint32_t)p.n_join - 1), d;
  d = fast_div(w, p.fd_rows);
  const int row = (int)(w - d * p.rows_max);
  w = d;
  d = fast_div(w, p.fd_heads);
  const int h = (int)(w - d * p.n_kv_heads), r = (int)d;
  const int i = (int)fast_div((uint32_t)row, p.fd_group);
  int n = p.n_queries;
  if (p.q_tokens != nullptr) n = min(max(p.q_tokens[r], 0), p.n_queries);
  const int64_t row0 = p.q_base != nullptr ? (int64_t)p.q_base[r] : (int64_t)r * p.n_queries;
  const int64_t at = (((int64_t)r * p.n_kv_heads + h) * p.rows_max + row) * p.n_splits;

  float top = kLow, l = 0.f, lx = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = way; s0 < p.n_splits; s0 += kChunk * WAYS) {
    f32x4 ml[kChunk], o[kChunk];
#pragma unroll
    for (int k = 0; k < kChunk; ++k) {
      const int s = min(s0 + k * WAYS, p.n_splits - 1);     // one past the end is read again and left out
      ml[k] = *reinterpret_cast<const f32x4*>(p.part_ml + (at + s) * 4);
      o[k] = *reinterpret_cast<const f32x4*>(p.part_o + (at + s) * D + col * 4);
    }
    float m = top;
#pragma unroll
    for (int k = 0; k < kChunk; ++k) m = fmaxf(m, ml[k].x);
    const float down = exp2_fast(top - m);
    top = m;
    l *= down;
    lx *= down;
    acc *= down;
#pragma unroll
    for (int k = 0; k < kChunk; ++k)
      if (s0 + k * WAYS < p.n_splits) {
        const float f = exp2_fast(ml[k].x - top);
        l += ml[k].y * f;
        lx += ml[k].z * f;
        acc += o[k] * f;
      }
  }
  if (WAYS > 1) {
    s_o[WAYS > 1 ? slot : 0][col] = acc;
    if (col == 0) {
      s_ml[WAYS > 1 ? slot : 0][0] = top;
      s_ml[WAYS > 1 ? slot : 0][1] = l;
      s_ml[WAYS > 1 ? slot : 0][2] = lx;
    }
    __syncthreads();
    if (way != 0) return;
    const float own = top;
#pragma unroll
    for (int k = 1; k < WAYS; ++k) top = fmaxf(top, s_ml[WAYS > 1 ? slot + k : 0][0]);
    const float down = exp2_fast(own - top);
    l *= down;
    lx *= down;
    acc *= down;
#pragma unroll
    for (int k = 1; k < WAYS; ++k) {
      const float f = exp2_fast(s_ml[WAYS > 1 ? slot + k : 0][0] - top);
      l += s_ml[WAYS > 1 ? slot + k : 0][1] * f;
      lx += s_ml[WAYS > 1 ? slot + k : 0][2] * f;
      acc += s_o[WAYS > 1 ? slot + k : 0][col] * f;
    }
  }
  if (i >= n || task >= (uint32_t)p.n_join) return;   // a row that no request has (its parts were not written)
  const int64_t hq = (int64_t)h * p.group + (row - i * p.group);
  acc *= l == 0.f ? 0.f : 1.0f / l;
  *reinterpret_cast<u32x2*>(p.out + (row0 + i) * p.out_s[0] + hq * p.out_s[1] + 4 * col) =
      u32x2{pack_bf16x2(acc.x, acc.y), pack_bf16x2(acc.z, acc.w)};
  if (col == 0 && p.lse != nullptr) p.lse[(row0 + i) * p.lse_s[0] + hq * p.lse_s[1]] = row_lse(top, lx);
}

namespace {

template <int D, int FMT, int NR>
hipError_t launch_rows(const AttendParams& p, hipStream_t s) {
  hipLaunchKernelGGL((attend_rows_kernel<D, FMT, NR>), dim3((uint32_t)p.n_tasks), dim3(kAttThreads), 0, s, p);
  return hipGetLastError();
}

template <int D>
hipError_t launch_few(const AttendParams& p, hipStream_t s) {
  if (p.cache_type == KAMERA_CACHE_BF16) return launch_rows<D, KAMERA_CACHE_BF16, 1>(p, s);
  return p.row_tiles == 1 ? launch_rows<D, KAMERA_CACHE_E4M3, 1>(p, s) : launch_rows<D, KAMERA_CACHE_E4M3, 2>(p, s);
}

template <int D>
hipError_t launch_join(const AttendParams& p, hipStream_t s) {
  const int ways = p.n_splits <= 8 ? 1 : 8, rows = kAttThreads / (D / 4 * ways);
  const dim3 grid((uint32_t)((p.n_join + rows - 1) / rows)), block(kAttThreads);
  if (ways == 1) hipLaunchKernelGGL((attend_join_kernel<D, 1>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((attend_join_kernel<D, 8>), grid, block, 0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend(const AttendParams& p, hipStream_t s) {
  const hipError_t e =
      p.tiles ? launch_attend_tiles(p, s) : (p.head_dim == 128 ? launch_few<128>(p, s) : launch_few<64>(p, s));
  if (e != hipSuccess || p.n_splits == 1) return e;
  return p.head_dim == 128 ? launch_join<128>(p, s) : launch_join<64>(p, s);
}

}  // namespace kamera

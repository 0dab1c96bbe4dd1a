// kamera_attend_paged, many query rows: attention over the paged cache where the
// matrix products are the work (prompt chunks).
//
// Rows as in the few-rows kernel: (query token, head of the group) of one KV
// head.  A wave takes 32 rows, a workgroup four waves, all over the
// same 64-token tiles of K and V, which the workgroup stages in LDS as bf16: K as
// [token][D], V transposed, [D][token].  e4m3 becomes bf16 on the way, once for
// all rows.
//
//   S^T = K Q^T and O^T = V^T P^T with 32x32x16 bf16 MFMAs, K and V^T the A
//   operands.  In S^T lane l holds row l % 32 and tokens 8 (i / 4) + 4 (l / 32) +
//   i % 4; these registers are P^T's B operand as they are when the inner index
//   of the second product runs over the tokens in that order, so V^T is stored
//   with the 4-token runs 0 1 2 3 of each 16 as 0 2 1 3.  A row's scores lie in
//   two lanes: its maximum takes one exchange.
//
// LDS: 16-byte chunks are exchanged by an exclusive-or with bits of the row
// number, so that the 16 lanes that read a chunk together (16 rows, one column)
// and those that write transposed columns spread over all banks.  Two buffers:
// the loads of the next tile are issued before a tile is computed and stored
// after it, with one barrier a tile.
//
// Softmax as in the few-rows kernel.
//
// Bound by the softmax's vector instructions beside the matrix pipe: 64 keys cost a
// wave 1024 cycles of MFMA and about as many of exponentials, maxima and
// conversions, which two waves a SIMD (two workgroups a CU) overlap in part.  1024
// queries of 8 x 8 heads over 16384 keys in 8 bits: 500 us, 1065 TFLOP/s, matrix pipe
// busy 46%.  64 rows a wave, one wave a SIMD: 522 against 755
// TFLOP/s in an earlier form, for want of a second wave to overlap with.

#include <algorithm>
#include <type_traits>

#include "kamera_attend_device.h"

namespace kamera {

namespace {

constexpr int kTileThreads = 256;
constexpr int kTileKeys = 64;
constexpr int kMfma = 0x8, kDsRead = 0x100;   // instruction groups of the scheduler
constexpr float kLow = -3.402823466e38f;
constexpr float kSlack = 8.0f;

// Place of 16-byte chunk `c` of row `r`: K rows of 16 or 8 chunks (the exchange
// repeats every 16 rows), V^T rows of 8.
template <int CHUNKS>
__device__ __forceinline__ uint32_t k_chunk(uint32_t r, uint32_t c) {
  return CHUNKS == 16 ? r * 16 + (c ^ (r & 15)) : r * 8 + (c ^ ((r >> 1) & 7));
}
__device__ __forceinline__ uint32_t v_chunk(uint32_t r, uint32_t c) { return r * 8 + (c ^ (((r >> 1) ^ (r >> 4)) & 7)); }

template <int D, int FMT>
struct Stage {                                     // a thread's share of a tile
  static constexpr int kEl = FMT == KAMERA_CACHE_BF16 ? 2 : 1;
  static constexpr int kRowLoads = D * kEl / 16;   // 16-byte loads of a K row
  static constexpr int KN = kTileKeys * kRowLoads / kTileThreads;
  static constexpr int VC = D / 16;                // V columns a thread, of 4 tokens
  static constexpr int VW = VC * kEl / 4;          // dwords of them in one token
  u32x4 k[KN];
  uint32_t v[4][VW];
  float ks[KN], vs;
};

// Tile number `tile` % 16 of a batch of looked-up parts.  k_off, v_off: this
// thread's place in a 16-token part.
template <int D, int FMT>
__device__ __forceinline__ void load_tile(const Parts& a, int tile, int wave, uint32_t k_off, uint32_t v_off,
                                          int64_t v_token, Stage<D, FMT>& s, uint32_t& bad) {
  using S = Stage<D, FMT>;
  const int lane0 = (tile & 15) * 4;
  bad = ~(uint32_t)(a.ok >> lane0) & 15u;
#pragma unroll
  for (int i = 0; i < S::KN; ++i) {
    // a wave's tokens of one load lie in one part
    const int u = lane0 + (wave * 64 + i * kTileThreads) / S::kRowLoads / 16;
    s.k[i] = load_global<u32x4>(lane_address(a.k, u) + k_off);
    s.ks[i] = lane_float(a.ks, u);
  }
  GlobalBytes vb = lane_address(a.v, lane0 + wave);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const GlobalBytes at = vb + v_off;
    if (S::VW == 1) s.v[j][0] = load_global<uint32_t>(at);
    else if (S::VW == 2) {
      const u32x2 x = load_global<u32x2>(at);
      s.v[j][0] = x.x;
      s.v[j][S::VW > 1 ? 1 : 0] = x.y;
    } else {
      const u32x4 x = load_global<u32x4>(at);
#pragma unroll
      for (int e = 0; e < S::VW; ++e) s.v[j][e] = u4_get(x, e);
    }
    vb += v_token;
  }
  s.vs = lane_float(a.vs, lane0 + wave);
}

// This thread's places in a buffer, in bytes.
template <int D, int FMT>
struct Places {
  using S = Stage<D, FMT>;
  uint32_t k[FMT == KAMERA_CACHE_E4M3 ? 2 : 1];    // its first K chunks; those of load i lie i * kTileThreads / kRowLoads rows on
  uint32_t v[S::VC];
};

// Registers -> LDS.  With `clear`, V rows that no row of the block sees become
// zero, and so does what is not finite in the others (the result says whether
// there was any; see add_nonfinite).  A part that is not there has been read from
// the pool's first page: its scale, which may be no number, goes too.
template <int D, int FMT>
__device__ __forceinline__ bool store_tile(Stage<D, FMT>& s, uint8_t* buf, const Places<D, FMT>& at, bool clear,
                                           uint32_t bad, int wave, int v_pos, int lo, int hi) {
  using S = Stage<D, FMT>;
#pragma unroll
  for (int i = 0; i < S::KN; ++i) {
    uint8_t* row = buf + i * (kTileThreads / S::kRowLoads) * D * 2;
    if (FMT == KAMERA_CACHE_BF16) {
      *reinterpret_cast<u32x4*>(row + at.k[0]) = s.k[i];
    } else {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t a = e ? s.k[i].z : s.k[i].x, b = e ? s.k[i].w : s.k[i].y;
        *reinterpret_cast<u32x4*>(row + at.k[FMT == KAMERA_CACHE_E4M3 ? e : 0]) =
            u32x4{e4m3_to_bf16x2<false>(a, s.ks[i]), e4m3_to_bf16x2<true>(a, s.ks[i]),
                  e4m3_to_bf16x2<false>(b, s.ks[i]), e4m3_to_bf16x2<true>(b, s.ks[i])};
      }
    }
  }
  uint32_t odd = 0;
  if (clear) {
    const bool missing = (bad >> wave) & 1;
    s.vs = missing ? 1.0f : s.vs;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool keep = !missing && v_pos + j >= lo && v_pos + j <= hi;
#pragma unroll
      for (int e = 0; e < S::VW; ++e) {
        s.v[j][e] = keep ? s.v[j][e] : 0u;
        odd |= nonfinite<FMT>(s.v[j][e]);
        s.v[j][e] = finite_only<FMT>(s.v[j][e]);
      }
    }
  }
#pragma unroll
  for (int c = 0; c < S::VC; ++c) {
    u32x2 r;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      uint32_t y;
      if (FMT == KAMERA_CACHE_BF16) {
        y = __builtin_amdgcn_perm(s.v[2 * t + 1][c >> 1], s.v[2 * t][c >> 1], (c & 1) ? 0x07060302u : 0x05040100u);
      } else {
        const uint32_t x =
            __builtin_amdgcn_perm(s.v[2 * t + 1][c >> 2], s.v[2 * t][c >> 2], (c & 2) ? 0x07030602u : 0x05010400u);
        y = (c & 1) ? e4m3_to_bf16x2<true>(x, s.vs) : e4m3_to_bf16x2<false>(x, s.vs);
      }
      if (t == 0) r.x = y; else r.y = y;
    }
    *reinterpret_cast<u32x2*>(buf + at.v[c]) = r;
  }
  return odd != 0;
}

}  // namespace

template <int D, int FMT, bool LSE>
__global__ __launch_bounds__(kTileThreads, 2) void attend_tiles_kernel(AttendParams) {
  const AttendParams& p = kernel_params<AttendParams>();
  constexpr int KC = D / 8, KS = D / 16, DT = D / 32;
  constexpr int kRows = 4 * 32;
  constexpr int kVAt = kTileKeys * D * 2;          // a buffer holds K, then V^T: bytes to V^T, and of both
  constexpr int kBuf = 2 * kVAt;
  using S = Stage<D, FMT>;
  extern __shared__ u32x4 s_buf[];
  uint8_t* const lds = reinterpret_cast<uint8_t*>(s_buf);
  __shared__ int s_odd;                            // a value that is not finite was taken as 0

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c32 = lane & 31, hf = lane >> 5;
  // The row blocks of a (request, KV head) pair are dealt into the fewest shares
  // that spread every request over all XCDs alike (one where the heads are a
  // multiple of 8: an XCD's L2 then serves all blocks of a pair).  Within an XCD all
  // pairs' late blocks, which see the most keys, come before the early ones, and the
  // order of the pairs turns by one from block to block: workgroups go to an XCD's
  // shader engines in turn, and without the turning an engine keeps its requests
  // (eight ragged requests of 4 heads: 198 us with whole pairs on an XCD, 171 us dealt
  // out, 137 us dealt out and turned).
  uint32_t w = blockIdx.x >> 3, d;
  d = fast_div(w, p.fd_shares);
  uint32_t local = w - d * p.n_shares + (d - fast_div(d, p.fd_shares) * p.n_shares);
  if (local >= (uint32_t)p.n_shares) local -= p.n_shares;
  const uint32_t share = local * 8 + (blockIdx.x & 7), pair = fast_div(share, p.fd_deal);
  w = d;
  d = fast_div(w, p.fd_splits);
  const int split = (int)(w - d * p.n_splits);
  // which of `deal` neighbouring blocks an XCD takes turns from pair to pair and split to
  // split too, or where the blocks are no multiple of `deal` the same XCDs would go without
  // (37 requests of 3 queries of 16 heads over one bf16 KV head, up to 10040 keys: one XCD
  // had all the work, 222 us, now 72)
  const int rb = (p.blocks_share - 1 - (int)d) * p.deal +
                 (int)((share - pair * p.deal + local + (uint32_t)split) & (uint32_t)(p.deal - 1));
  d = fast_div(pair, p.fd_heads);
  const int h = (int)(pair - d * p.n_kv_heads), r = (int)d;
  if (rb >= p.n_row_blocks) return;

  const Request rq = request_of(p, r);
  const int rows = rq.n * p.group;
  const int row_first = rb * kRows, row_end = min(rows, row_first + kRows);
  if (row_first >= rows) return;
  const int i_first = (int)fast_div((uint32_t)row_first, p.fd_group);
  const int i_last = (int)fast_div((uint32_t)row_end - 1, p.fd_group);
  Walk walk;
  walk.table = p.page_table + (int64_t)r * p.pt_stride;
  walk.sel = nullptr;
  // keys that some row of the block sees, and those that every row sees
  const int hi = min(last_key(p, rq, i_last), rq.kv - 1), lo = first_key(p, last_key(p, rq, i_first));
  walk.begin = lo >> 4;
  walk.end = (hi >> 4) + 1;
  const int all_hi = last_key(p, rq, i_first), all_lo = first_key(p, last_key(p, rq, i_last));
  const int tile0 = lo / kTileKeys, tile1 = (hi + kTileKeys) / kTileKeys;   // hi = -1: none
  const int per = (max(tile1 - tile0, 0) + p.n_splits - 1) / p.n_splits;
  const int t_begin = tile0 + split * per, t_end = min(tile1, t_begin + per);

  // this wave's rows; lane l has row l % 32
  const int wave_row = row_first + wave * 32, row = wave_row + c32;
  bf16x8 qf[KS];
  int row_lo = INT32_MAX;                          // sees the keys row_lo .. row_lo + row_span; none past the end
  uint32_t row_span = 0;
  {
    const int i = (int)fast_div((uint32_t)row, p.fd_group), hq = row - i * p.group;
    const bool there = row < row_end;
    const int last = last_key(p, rq, i);
    if (there && last >= 0) {
      row_lo = first_key(p, last);
      row_span = (uint32_t)(min(last, rq.kv - 1) - row_lo);
    }
    const uint16_t* src = p.q + (rq.row0 + i) * p.q_s[0] + ((int64_t)h * p.group + hq) * p.q_s[1] + hf * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      u32x4 x = {0u, 0u, 0u, 0u};
      if (there) x = *reinterpret_cast<const u32x4*>(src + ks * 16) ^ p.q_sign;
      qf[ks] = __builtin_bit_cast(bf16x8, x);
    }
  }

  f32x16 o[DT];
  float m = kLow, l = 0.f, l1 = 0.f, lx = 0.f;
#pragma unroll
  for (int b = 0; b < DT; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[b][i] = 0.f;

  // this thread's places in global memory and in LDS
  const int tid = threadIdx.x, q4 = (tid >> 4) & 3, cg = tid & 15;
  const uint32_t k_off = (uint32_t)((tid / S::kRowLoads & 15) * (uint32_t)p.k_s[1] + tid % S::kRowLoads * 16);
  const uint32_t v_off = (uint32_t)(q4 * 4 * (uint32_t)p.v_s[1] + cg * S::VC * S::kEl);
  const int64_t v_token = p.v_s[1];
  Places<D, FMT> at;
#pragma unroll
  for (int e = 0; e < (FMT == KAMERA_CACHE_E4M3 ? 2 : 1); ++e)
    at.k[e] = 16 * k_chunk<KC>(tid / S::kRowLoads, (FMT == KAMERA_CACHE_E4M3 ? 2 : 1) * (tid % S::kRowLoads) + e);
  // tokens 4 q .. 4 q + 3 of the tile: run q % 4 of 16-token group q / 4
  const uint32_t run = q4 == 1 ? 2 : (q4 == 2 ? 1 : q4);
#pragma unroll
  for (int c = 0; c < S::VC; ++c) at.v[c] = kVAt + 16 * v_chunk(cg * S::VC + c, wave * 2 + (run >> 1)) + 8 * (run & 1);
  uint32_t k_at[KS], v_at[DT][4];                  // the chunks of its MFMA operands
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) k_at[ks] = 16 * k_chunk<KC>(c32, 2 * ks + hf);
#pragma unroll
  for (int b = 0; b < DT; ++b)
#pragma unroll
    for (int s = 0; s < 4; ++s) v_at[b][s] = kVAt + 16 * v_chunk(b * 32 + c32, 2 * s + hf);

  S st;
  uint32_t bad = 0, bad_next = 0;
  auto is_partial = [&](int tile, uint32_t missing) {
    return missing != 0 || tile * kTileKeys + kTileKeys - 1 > all_hi || tile * kTileKeys < all_lo;
  };
  auto store = [&](int tile, uint32_t missing, uint8_t* buf) {
    if (store_tile<D, FMT>(st, buf, at, is_partial(tile, missing), missing, wave, tile * kTileKeys + wave * 16 + q4 * 4,
                           lo, hi))
      s_odd = 1;
  };
  if (threadIdx.x == 0) s_odd = 0;
  __syncthreads();
  // parts looked up 16 tiles at a time, a batch ahead
  auto batch = [&](int tile) { return fetch_parts<FMT>(p, walk, tile < t_end ? (tile & ~15) * 4 + lane : -1, h); };
  Parts parts = batch(t_begin), ahead = batch((t_begin & ~15) + 16);
  if (t_begin < t_end) {
    load_tile<D, FMT>(parts, t_begin, wave, k_off, v_off, v_token, st, bad);
    store(t_begin, bad, lds);
  }
  __syncthreads();

  // One tile, from buffer B; the next one goes into the other.
  auto step = [&](auto which, int tile) {
    constexpr int B = decltype(which)::value * kBuf, kOther = kBuf - B;
    if (tile + 1 < t_end) {
      if (((tile + 1) & 15) == 0) {
        parts = ahead;
        ahead = batch(tile + 17);
      }
      load_tile<D, FMT>(parts, tile + 1, wave, k_off, v_off, v_token, st, bad_next);
    }
    const bool partial = is_partial(tile, bad);

    // S^T.  The chunks of the first 32 tokens are read together and those of the
    // second one by one behind the products, so that no product waits for its own
    // read: with reads two products ahead a third of the time went into such waits.
    __builtin_amdgcn_s_setprio(1);
    f32x16 sc[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[u][i] = 0.f;
    constexpr int kAhead = FMT == KAMERA_CACHE_BF16 ? KS / 2 : KS;
    bf16x8 kf[2][KS];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) kf[u][ks] = *reinterpret_cast<const bf16x8*>(lds + k_at[ks] + (B + u * 32 * D * 2));
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[u][ks], qf[ks], sc[u], 0, 0, 0);
    __builtin_amdgcn_sched_group_barrier(kDsRead, kAhead, 0);
#pragma unroll
    for (int ks = 0; ks < 2 * KS - kAhead; ++ks) {
      __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(kMfma, kAhead, 0);
    __builtin_amdgcn_s_setprio(0);

    if (partial) {
      const int row_at = tile * kTileKeys + 4 * hf - row_lo;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t from_lo = (uint32_t)(row_at + (u * 32 + 8 * (i >> 2) + (i & 3)));
          sc[u][i] = from_lo <= row_span ? sc[u][i] : -INFINITY;
        }
      if (bad != 0) {                              // parts that are not in the pool
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 16; ++i) sc[u][i] = (bad >> (u * 2 + (i >> 3))) & 1 ? -INFINITY : sc[u][i];
      }
    }
    float top = sc[0][0];                          // the first half's are there before the second's
#pragma unroll
    for (int i = 1; i < 31; i += 2) top = max2(max2(top, sc[i >> 4][i & 15]), sc[(i + 1) >> 4][(i + 1) & 15]);
    top = max2(top, sc[1][15]);
    top *= p.scale2;
    if (__ballot(top > m + kSlack) != 0) {
      const float m_new = fmaxf(m, max_x32(top));
      const float down = exp2_fast(m - m_new);
      m = m_new;
      l *= down;
      l1 *= down;
      lx *= down;
#pragma unroll
      for (int b = 0; b < DT; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] *= down;
    }

    // P^T of the first 32 tokens, then their products with V^T between the steps of
    // the other half's exponentials.
    __builtin_amdgcn_s_setprio(1);
    bf16x8 vf[4][DT];
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int b = 0; b < DT; ++b) vf[s][b] = *reinterpret_cast<const bf16x8*>(lds + v_at[b][s] + B);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = exp2_fast(__builtin_fmaf(sc[u][i], p.scale2, -m));
      if (LSE) {
#pragma unroll
        for (int i = 0; i < 16; i += 4) lx += (x[i] + x[i + 1]) + (x[i + 2] + x[i + 3]);
      }
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const u32x4 w = {pack_bf16x2(x[8 * s], x[8 * s + 1]), pack_bf16x2(x[8 * s + 2], x[8 * s + 3]),
                         pack_bf16x2(x[8 * s + 4], x[8 * s + 5]), pack_bf16x2(x[8 * s + 6], x[8 * s + 7])};
        l = add_pair(w.y, add_pair(w.x, l));
        l1 = add_pair(w.w, add_pair(w.z, l1));
        const bf16x8 pf = __builtin_bit_cast(bf16x8, w);
#pragma unroll
        for (int b = 0; b < DT; ++b)
          o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[2 * u + s][b], pf, o[b], 0, 0, 0);
      }
    }
    asm volatile("" : "+v"(l), "+v"(l1));         // or the sums sink behind the next tile's stores
    __builtin_amdgcn_s_setprio(0);
    bad = bad_next;
    if (tile + 1 < t_end) store(tile + 1, bad, lds + kOther);
    __syncthreads();
  };
  for (int tile = t_begin; tile < t_end; tile += 2) {
    step(std::integral_constant<int, 0>{}, tile);
    if (tile + 1 < t_end) step(std::integral_constant<int, 1>{}, tile + 1);
  }

  l = sum_x32(l + l1);
  if (LSE) lx = sum_x32(lx);
  if (row < row_end) {
    if (p.n_splits > 1) {
      const int64_t part = (((int64_t)r * p.n_kv_heads + h) * p.rows_max + row) * p.n_splits + split;
#pragma unroll
      for (int b = 0; b < DT; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<f32x4*>(p.part_o + part * D + b * 32 + 2 * i + 4 * hf) =
              f32x4{o[b][i], o[b][i + 1], o[b][i + 2], o[b][i + 3]};
      if (hf == 0) *reinterpret_cast<f32x4*>(p.part_ml + part * 4) = f32x4{m, l, lx, 0.f};
    } else {
      const int i = (int)fast_div((uint32_t)row, p.fd_group);
      const int64_t hq = (int64_t)h * p.group + (row - i * p.group);
      const float inv = l == 0.f ? 0.f : 1.0f / l;
      uint16_t* dst = p.out + (rq.row0 + i) * p.out_s[0] + hq * p.out_s[1] + 4 * hf;
#pragma unroll
      for (int b = 0; b < DT; ++b)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          *reinterpret_cast<u32x2*>(dst + b * 32 + 2 * e) =
              u32x2{pack_bf16x2(o[b][e] * inv, o[b][e + 1] * inv), pack_bf16x2(o[b][e + 2] * inv, o[b][e + 3] * inv)};
      if (LSE && hf == 0) p.lse[(rq.row0 + i) * p.lse_s[0] + hq * p.lse_s[1]] = row_lse(m, lx);
    }
  }
  if (s_odd)
    add_nonfinite<D, FMT>(p, rq, walk, t_begin * 4, t_end * 4, 4, all_lo, all_hi, h, r, row_first, row_end, split);
}

namespace {

template <int D, int FMT, bool LSE>
hipError_t launch_one(const AttendParams& p, hipStream_t s) {
  static std::atomic<bool> done[kMaxDevices];
  const int lds = 4 * kTileKeys * D * 2;
  const hipError_t e = ensure_lds_limit((const void*)attend_tiles_kernel<D, FMT, LSE>, lds, done);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((attend_tiles_kernel<D, FMT, LSE>), dim3((uint32_t)p.n_tasks), dim3(kTileThreads), lds, s, p);
  return hipGetLastError();
}

template <int D, int FMT>
hipError_t launch_lse(const AttendParams& p, hipStream_t s) {
  return p.lse != nullptr ? launch_one<D, FMT, true>(p, s) : launch_one<D, FMT, false>(p, s);
}

}  // namespace

hipError_t launch_attend_tiles(const AttendParams& p, hipStream_t s) {
  if (p.cache_type == KAMERA_CACHE_E4M3)
    return p.head_dim == 128 ? launch_lse<128, KAMERA_CACHE_E4M3>(p, s) : launch_lse<64, KAMERA_CACHE_E4M3>(p, s);
  return p.head_dim == 128 ? launch_lse<128, KAMERA_CACHE_BF16>(p, s) : launch_lse<64, KAMERA_CACHE_BF16>(p, s);
}

}  // namespace kamera

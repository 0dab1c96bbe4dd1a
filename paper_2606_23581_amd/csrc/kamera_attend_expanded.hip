// kamera_attend_expanded: attention over expanded keys and values of every head, with
// the rope keys that all heads share read from the paged pool.
//
// A wave takes 32 query rows of one head, a workgroup four waves, all over the same
// 64-key tiles: K and V rows from the dense arrays, rope rows from the pool, straight
// from global memory into LDS, the next tile's while a tile is computed.
//   S^T = K Q^T + R Q_r^T and O^T = V^T P^T with 32x32x16 bf16 MFMAs, as in the latent
//   form; V's columns come by transposed reads.
//
// LDS: 16-byte chunks are exchanged by an exclusive-or with bits of the key number,
// so that 16 keys' reads of a chunk and four keys' of 64 bytes spread over all banks.
//
// Softmax in powers of two (scale * log2 e folded in), fp32.  A row's running maximum
// moves only when a score passes it by more than 8.
//
// Neither pipe is full: with two workgroups a CU (81,920 bytes of LDS each, all there is),
// two waves a SIMD, the matrix pipe is busy 45% of the time and vector instructions, four
// beside each MFMA, issue 34% of it.  What is missing is their overlap: one wave's exponentials
// and the other's products run one after the other for the most part.  1024 queries of
// 16 heads over 16384 keys: 172 us, 970 TFLOP/s; eight ragged prompts of up to 1024
// queries over up to 2048 keys, 1024 tasks of 1 to 32 tiles: 101 us, of which some 14000
// cycles a task, as much as its tiles, go to its start (lengths, pages, first loads) and its
// end, where results are stored as the products leave them, 16 bytes of each of 32 rows at a
// time.

#include "kamera_mla_device.h"

namespace kamera {

namespace {

constexpr int kExpThreads = 256;
constexpr int kTileKeys = 64;
constexpr int kAhead = 4;                          // products whose operands are read ahead

}  // namespace

template <int D>
__global__ __launch_bounds__(kExpThreads, 2) void attend_expanded_kernel(MlaParams) {
  const MlaParams& p = kernel_params<MlaParams>();
  constexpr int KS = D / 16, RS = kRopeCols / 16, DT = D / 32;
  constexpr int kRowB = D * 2, kTile = kTileKeys * kRowB, kRopeTile = kTileKeys * kRopeCols * 2;
  constexpr int kVAt = kTile, kRAt = 2 * kTile, kBuf = 2 * kTile + kRopeTile;
  constexpr int RPL = 1024 / kRowB, NL = 16 / RPL;  // keys of a wave's load; loads for its 16 keys
  extern __shared__ u32x4 s_buf[];
  const uint32_t lds = lds_offset(s_buf);

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c32 = lane & 31, hf = lane >> 5;

  // neighbouring shares, which read the same head's keys, on one XCD
  const uint32_t n_wgs = p.n_parts > 0 ? p.n_parts : p.n_tasks, per_xcd = (n_wgs + 7) / 8;
  const uint32_t wg = (uint32_t)xcd_task((int32_t)per_xcd);
  if (wg >= n_wgs) return;
  Share share;
  if (p.n_parts > 0) {
    share = divide<kTileKeys>(p, wg);
  } else {
    share.task = p.n_tasks - 1 - wg;               // late row blocks, which see the most keys, first
    share.skip = 0;
    share.units = INT32_MAX;
  }

  // this lane's pieces of the wave's 16 keys of a tile: key and chunk of load j
  const uint32_t k_stride = (uint32_t)p.k_s[0], v_stride = (uint32_t)p.v_s[0], t_stride = (uint32_t)p.pool_s[1];
  uint32_t k_off[NL], v_off[NL], r_off[2];
#pragma unroll
  for (int j = 0; j < NL; ++j) {
    const uint32_t key = RPL * j + lane / (kRowB / 16), c = lane % (kRowB / 16);
    k_off[j] = key * k_stride + ((c ^ (D == 128 ? key & 15 : (key >> 1) & 7)) << 4);
    v_off[j] = key * v_stride + ((c ^ (D == 128 ? (key & 3) << 2 : (key & 2) << 1)) << 4);
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t key = 8 * j + (lane >> 3);
    r_off[j] = key * t_stride + (((lane & 7) ^ ((key >> 1) & 7)) << 4);
  }
  // places of the operands in a buffer
  uint32_t k_at[KS], r_at[RS], v_at[DT];
#pragma unroll
  for (int s = 0; s < KS; ++s) k_at[s] = c32 * kRowB + (((2 * s + hf) ^ (D == 128 ? c32 & 15 : (c32 >> 1) & 7)) << 4);
#pragma unroll
  for (int s = 0; s < RS; ++s) r_at[s] = kRAt + c32 * (kRopeCols * 2) + (((2 * s + hf) ^ ((c32 >> 1) & 7)) << 4);
#pragma unroll
  for (int b = 0; b < DT; ++b) {
    const uint32_t i16 = lane & 15, key = 4 * hf + (i16 >> 2), c = 4 * b + 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1);
    v_at[b] = kVAt + key * kRowB + ((c ^ (D == 128 ? (key & 3) << 2 : (key & 2) << 1)) << 4) + (i16 & 1) * 8;
  }

  uint32_t task = share.task;
  int skip = share.skip, units = share.units, segment = 0;
  const uint32_t end = p.n_parts > 0 ? p.n_tasks : task + 1;
  for (; units > 0 && task < end; ++task, skip = 0) {
    const Block blk = block_of(p, task);
    Segment seg;
    if (!take_segment(p, blk, kTileKeys, task, share, units, skip, seg)) continue;
    const int take = seg.to - seg.from, tile0 = blk.lo / kTileKeys + seg.from;
    const int part_begin = blk.lo >> 4, part_end = (blk.hi >> 4) + 1;
    const int64_t key_row = first_row(p.kv_base, blk.r, p.n_keys);
    const uint64_t k_head = (uint64_t)p.k + key_row * p.k_s[0] + blk.h * p.k_s[1];
    const uint64_t v_head = (uint64_t)p.v + key_row * p.v_s[0] + blk.h * p.v_s[1];

    // parts looked up 16 tiles at a time: lane i has part i % 4 of tile i / 4 of the batch
    auto batch = [&](int it) {
      const int at = it + (lane >> 2);
      return fetch_pool_parts(p, blk.r, at < take ? (tile0 + at) * 4 + (lane & 3) : -1, part_begin, part_end);
    };
    PoolParts parts = batch(0);

    auto issue = [&](int it) {
      if (it > 0 && (it & 15) == 0) parts = batch(it);
      const int pos = (tile0 + it) * kTileKeys, first = pos + wave * 16;
      const uint32_t ok = (uint32_t)(parts.ok >> (4 * (it & 15))) & 15u;
      const uint64_t rope = lane_u64(parts.at, 4 * (it & 15) + wave);
      const uint64_t kb = k_head + first * p.k_s[0], vb = v_head + first * p.v_s[0];
      const uint32_t to = lds + (it & 1) * kBuf;
      const bool whole = ok == 15u && pos >= blk.lo && pos + kTileKeys - 1 <= blk.hi;
      if (whole) {
#pragma unroll
        for (int j = 0; j < NL; ++j) load_lds((const uint8_t*)kb, k_off[j], to + (wave * NL + j) * 1024);
#pragma unroll
        for (int j = 0; j < 2; ++j) load_lds((const uint8_t*)rope, r_off[j], to + kRAt + (wave * 2 + j) * 1024);
#pragma unroll
        for (int j = 0; j < NL; ++j) load_lds((const uint8_t*)vb, v_off[j], to + kVAt + (wave * NL + j) * 1024);
      } else {
        const bool there = (ok >> wave) & 1;
        const uint64_t zero = (uint64_t)g_zero_row;
        auto place = [&](int key, uint64_t at) { return there && key >= blk.lo && key <= blk.hi ? at : zero; };
#pragma unroll 1
        for (int j = 0; j < NL; ++j) {
          const uint32_t in_part = RPL * j + lane / (kRowB / 16), c = lane % (kRowB / 16);
          const uint32_t kc = c ^ (D == 128 ? in_part & 15 : (in_part >> 1) & 7);
          const uint32_t vc = c ^ (D == 128 ? (in_part & 3) << 2 : (in_part & 2) << 1);
          load_lds(place(first + in_part, kb + in_part * k_stride) + kc * 16, to + (wave * NL + j) * 1024);
          load_lds(place(first + in_part, vb + in_part * v_stride) + vc * 16, to + kVAt + (wave * NL + j) * 1024);
        }
#pragma unroll 1
        for (int j = 0; j < 2; ++j) {
          const uint32_t in_part = 8 * j + (lane >> 3);
          load_lds(place(first + in_part, rope + in_part * t_stride) + (((lane & 7) ^ ((in_part >> 1) & 7)) << 4),
                   to + kRAt + (wave * 2 + j) * 1024);
        }
      }
      return ok;
    };

    uint32_t ok = issue(0);

    // this wave's rows; lane l has row l % 32 (past the end the last one, whose results
    // are not stored)
    const int wave_row = blk.row_first + wave * 32, row = min(wave_row + c32, blk.row_end - 1);
    const int64_t row0 = first_row(p.q_base, blk.r, p.n_queries);
    bf16x8 qf[KS + RS];
    int row_lo = INT32_MAX;                        // sees the keys row_lo .. row_lo + row_span, or none
    uint32_t row_span = 0;
    {
      const int last = mla_last_key(p, blk.n, blk.kv, row);
      if (last >= 0 && blk.kv > 0) {
        row_lo = mla_first_key(p, last);
        row_span = (uint32_t)(min(last, blk.kv - 1) - row_lo);
      }
      const uint16_t* src = p.q + (row0 + row) * p.q_s[0] + blk.h * p.q_s[1] + hf * 8;
#pragma unroll
      for (int ks = 0; ks < KS + RS; ++ks)
        qf[ks] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(src + ks * 16) ^ p.q_sign);
    }
    f32x16 o[DT];
    float m = kLow, l = 0.f, l1 = 0.f, lx = 0.f;
    bool odd = false;                              // a value that is not finite was left out of a product
#pragma unroll
    for (int b = 0; b < DT; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[b][i] = 0.f;

    // A tile: scores, softmax and the product with the values.
    auto compute = [&](int pos, uint32_t buf, uint32_t ok) {
      f32x16 sc[2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[u][i] = 0.f;
      // operand i: keys 32 (i / N) on, inner step i % N
      constexpr int N = KS + RS;
      auto rows = [&](int i) {
        const int u = i / N, ks = i % N;
        return ks < KS ? read_chunk(buf + k_at[ks < KS ? ks : 0] + u * 32 * kRowB)
                       : read_chunk(buf + r_at[ks < KS ? 0 : ks - KS] + u * 32 * kRopeCols * 2);
      };
      __builtin_amdgcn_s_setprio(1);
      bf16x8 kf[2 * N];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) kf[i] = rows(i);
#pragma unroll
      for (int i = 0; i < 2 * N; ++i) {
        if (i + kAhead < 2 * N) kf[i + kAhead] = rows(i + kAhead);
        sc[i / N] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i], qf[i % N], sc[i / N], 0, 0, 0);
      }
      pipeline<2 * N, 1, kAhead>();
      __builtin_amdgcn_s_setprio(0);
      if (ok != 15u || pos + kTileKeys - 1 > blk.all_hi || pos < blk.all_lo) {     // some row does not see it whole
        const int at = pos + 4 * hf - row_lo;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const bool there = (ok >> (u * 2 + (i >> 3))) & 1;
            sc[u][i] = there && (uint32_t)(at + (u * 32 + 8 * (i >> 2) + (i & 3))) <= row_span ? sc[u][i] : -INFINITY;
          }
      }
      float top = sc[0][0];
#pragma unroll
      for (int i = 1; i < 31; i += 2) top = max2(max2(top, sc[i >> 4][i & 15]), sc[(i + 1) >> 4][(i + 1) & 15]);
      top = max2(top, sc[1][15]) * p.scale2;
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
      // the products with the first half's weights run beside the second half's exponentials
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        bf16x8 vf[2][DT];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int b = 0; b < DT; ++b) {
            const uint32_t at = buf + v_at[b] + (2 * u + s) * 16 * kRowB;
            vf[s][b] = join(read_columns(at), read_columns(at + 8 * kRowB));
          }
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = exp2_fast(__builtin_fmaf(sc[u][i], p.scale2, -m));
        if (p.lse != nullptr) {
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
          for (int b = 0; b < DT; ++b) o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[s][b], pf, o[b], 0, 0, 0);
        }
      }
      __builtin_amdgcn_s_setprio(0);
    };

    for (int it = 0; it < take; ++it) {
      vm_wait<0>();
      lds_barrier();                               // the tile is there, and the other buffer is free
      uint32_t ok_next = 0;
      if (it + 1 < take) ok_next = issue(it + 1);
      const int pos = (tile0 + it) * kTileKeys;
      const uint32_t buf = lds + (it & 1) * kBuf;
      if (mixed(blk, pos, kTileKeys)) {
        // what is not finite is left out of the product and added to the stored results
        for (int i = tid; i < kTile / 16; i += kExpThreads) odd |= clean_chunk(buf + kVAt + i * 16);
        lds_barrier();
      }
      if (wave_row < blk.row_end) compute(pos, buf, ok);
      ok = ok_next;
    }
    lds_barrier();                                 // the buffers are free
    int* flags = reinterpret_cast<int*>(s_buf);
    const bool any = __ballot(odd) != 0;
    if (lane == 0) flags[wave] = any;
    lds_barrier();
    const bool left_out = __builtin_amdgcn_readfirstlane(flags[0] | flags[1] | flags[2] | flags[3]) != 0;
    lds_barrier();

    l = sum_x32(l + l1);
    lx = sum_x32(lx);
    const bool direct = seg.whole();
    const int64_t part = ((int64_t)wg * 2 + (segment > 0 ? 1 : 0)) * p.rows_block, at = part + wave * 32 + c32;
    ++segment;
    if (wave_row + c32 < blk.row_end) {
      if (direct) {
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        uint16_t* dst = p.out + (row0 + row) * p.out_s[0] + blk.h * p.out_s[1] + 4 * hf;
#pragma unroll
        for (int b = 0; b < DT; ++b)
#pragma unroll
          for (int e = 0; e < 16; e += 4)
            *reinterpret_cast<u32x2*>(dst + b * 32 + 2 * e) =
                u32x2{pack_bf16x2(o[b][e] * inv, o[b][e + 1] * inv), pack_bf16x2(o[b][e + 2] * inv, o[b][e + 3] * inv)};
        if (p.lse != nullptr && hf == 0) p.lse[(row0 + row) * p.lse_s[0] + blk.h * p.lse_s[1]] = row_lse(m, lx);
      } else {
#pragma unroll
        for (int b = 0; b < DT; ++b)
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<f32x4*>(p.part_o + at * D + b * 32 + 2 * i + 4 * hf) =
                f32x4{o[b][i], o[b][i + 1], o[b][i + 2], o[b][i + 3]};
        if (hf == 0) *reinterpret_cast<f32x4*>(p.part_ml + at * 4) = f32x4{m, l, lx, 0.f};
      }
    }
    if (left_out) {
      const int from = tile0 * kTileKeys;
      add_nonfinite(p, blk, from, from + take * kTileKeys, kTileKeys, D, direct, part, row0, [&](int key) {
        const int k = (int)fast_div((uint32_t)key >> 4, p.fd_page16);
        const int page = p.page_table[(int64_t)blk.r * p.pt_stride + k];
        if (page < 0 || page >= p.n_pool_pages) return (const uint16_t*)nullptr;
        return (const uint16_t*)(v_head + key * p.v_s[0]);
      });
    }
  }
}

namespace {

template <int D>
hipError_t launch_dim(const MlaParams& p, hipStream_t s) {
  static std::atomic<bool> done[kMaxDevices];
  const int lds = 2 * kTileKeys * (2 * D + kRopeCols) * 2;
  const hipError_t e = ensure_lds_limit((const void*)attend_expanded_kernel<D>, lds, done);
  if (e != hipSuccess) return e;
  const uint32_t n = (uint32_t)(p.n_parts > 0 ? p.n_parts : p.n_tasks);
  hipLaunchKernelGGL((attend_expanded_kernel<D>), dim3((n + 7) / 8 * 8), dim3(kExpThreads), lds, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_expanded(const MlaParams& p, hipStream_t s) {
  const hipError_t e = p.dim == 128 ? launch_dim<128>(p, s) : launch_dim<64>(p, s);
  if (e != hipSuccess || p.n_parts == 0) return e;
  return launch_mla_join(p, s);
}

}  // namespace kamera

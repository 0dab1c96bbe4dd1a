// kamera_attend_latent: attention over the rows of a paged latent pool.
//
// A row is key and value at once: x = [c | r], scores <q, x>, results sum p c.  The
// rows of a request -- every query token's heads -- are one matrix, taken in blocks of
// 16 RW rows: RW waves of 16 rows each share the keys of a group, and the KW groups
// of a workgroup take 32 keys in turn.  Keys go from the pool straight into LDS and
// are read from there twice, as rows for the scores and, transposed, as columns for
// the results:
//   S^T = X Q^T and O^T = C^T P^T with 16x16x32 bf16 MFMAs.  In S^T lane l holds row
//   l % 16 and keys 4 (l / 16) + i of each 16; these registers are P^T's B operand as
//   they are when the inner index of the second product runs over the keys in that
//   order, which transposed reads give at no cost.
// 16 rows a wave and not 32, which would halve the reads of LDS for each product: the
// results of 32 rows (256 registers) and their queries (144) leave the compiler no room
// and it spills.  16 rows of 512 columns fill the 256 registers of a wave of eight: two of
// them spill there (12 bytes of scratch a lane), none in the other forms.
//
// LDS: a slot holds 32 keys.  16-byte chunks are exchanged by an exclusive-or of their
// number with a mix of bits 1 .. 3 of the key, so that eight keys' reads of 32 bytes
// spread over all banks, and so do those of a chunk of 16 keys, which the hardware takes
// as lanes 0-3, 12-15 and 20-27 (and so on): keys 0-3 and 12-15 of one chunk with keys
// 4-11 of its neighbour.  With the bits in plain order a third of the reads' cycles were
// conflicts.
//
// Softmax in powers of two (scale * log2 e folded in), fp32.  A row's running maximum
// moves only when a score passes it by more than 8.
//
// Single queries of 16 heads are bound by HBM (64 requests of up to 8192 keys: 378 MB in
// 80 us, 4.7 TB/s).  With more rows the reads of LDS bound it: a wave reads 36 KB for the
// scores of its 16 rows with 32 keys and 32 KB for their results, eight waves 550 KB, 4300
// cycles at 128 bytes a cycle (measured 1.8 us for 32 more keys), beside 2200 of products (two queries
// of 128 heads, 16 requests of up to 8192 keys: 72 us, 46 GFLOP, pipes busy 25%).  Short calls are a chain of latencies (256 keys:
// 12 us, one workgroup).

#include "kamera_mla_device.h"

namespace kamera {

namespace {

constexpr int kStepKeys = 32;

__device__ __forceinline__ uint32_t twist(uint32_t key) {
  const uint32_t b1 = (key >> 1) & 1, b2 = (key >> 2) & 1, b3 = (key >> 3) & 1;
  return (b2 ^ b3) << 2 | b1 << 1 | b3;
}

__device__ __forceinline__ float max_x16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_x16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

}  // namespace

template <int LAT, int RW>
__global__ __launch_bounds__(latent_waves(RW) * 64, latent_waves(RW) / 4) void attend_latent_kernel(MlaParams) {
  const MlaParams& p = kernel_params<MlaParams>();
  constexpr int NW = latent_waves(RW), kThr = NW * 64, KW = latent_groups(RW), NB = 4 / KW;
  constexpr int kRowB = (LAT + kRopeCols) * 2, CH = kRowB / 16, kSlot = kStepKeys * kRowB;
  constexpr int kUnit = kStepKeys * KW, KS = (LAT + kRopeCols) / 32, DT = LAT / 16;
  constexpr int LPG = CH / 8;                      // loads of a wave for 8 keys
  constexpr int LW = RW < 4 ? RW : 4;              // waves that load a step's keys (of 8, those take turns)
  constexpr int NA = 4 / LW;                       // groups of 8 keys that a wave loads
  constexpr int kAhead = NW == 4 ? 6 : 4;          // products whose operands are read ahead
  constexpr int kPad = LAT + 4;                    // floats of a row of the epilogue's tile
  static_assert(kUnit == 32 * KW && NB >= 1, "");
  extern __shared__ __attribute__((aligned(128))) u32x4 s_buf[];
  __shared__ float s_ml[NW][16][3];
  __shared__ uint32_t s_off[NW == 8 ? LPG : 1][64];
  __shared__ int s_odd;                            // a value that is not finite was left out of a product
  const uint32_t lds = lds_offset(s_buf);

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c16 = lane & 15, g = lane >> 4, wr = wave % RW, kg = wave / RW;

  Share share;
  if (p.n_parts > 0) {
    share = divide<kUnit>(p, blockIdx.x);
  } else {
    share.task = p.n_tasks - 1 - blockIdx.x;       // late row blocks, which see the most keys, first
    share.skip = 0;
    share.units = INT32_MAX;
  }

  // this lane's pieces of 8 keys that the wave loads: offset from the first one's row, and
  // in the low bits bits 0 and 2 of the chunk's number, which keys 8 .. 15 of 16 have the
  // other way round (in LDS where registers are short)
  const uint32_t t_stride = (uint32_t)p.pool_s[1];
  uint32_t off[NW == 8 ? 1 : LPG];
#pragma unroll
  for (int b = 0; b < LPG; ++b) {
    const uint32_t i = b * 64 + lane, key = i / CH, c = (i % CH) ^ twist(key);
    const uint32_t x = key * t_stride + c * 16 + (c & 1) + (c >> 1 & 2);
    if (NW == 8) s_off[NW == 8 ? b : 0][lane] = x;             // every wave writes the same
    else off[NW == 8 ? 0 : b] = x;
  }
  auto piece = [&](int b, uint32_t odd) {
    const uint32_t x = NW == 8 ? s_off[NW == 8 ? b : 0][lane] : off[NW == 8 ? 0 : b];
    return (x & ~15u) + odd * (80 - (x & 1) * 32 - (x & 2) * 64);
  };
  // places of the operands in a slot: chunk 4 s + g of key c16, and of keys 4 g ..
  // (rows and slots are multiples of 128 bytes, so that chunks are exchanged in the address)
  const uint32_t k_at = c16 * kRowB + ((g ^ twist(c16)) << 4), v_key = 4 * g + (c16 >> 2);
  const uint32_t v_at = v_key * kRowB + ((((c16 & 3) >> 1) ^ twist(v_key)) << 4) + (c16 & 1) * 8;

  uint32_t task = share.task;
  int skip = share.skip, units = share.units, segment = 0;
  const uint32_t end = p.n_parts > 0 ? p.n_tasks : task + 1;
  for (; units > 0 && task < end; ++task, skip = 0) {
    const Block blk = block_of(p, task);
    Segment seg;
    if (!take_segment(p, blk, kUnit, task, share, units, skip, seg)) continue;
    const int take = seg.to - seg.from;
    const int key0 = (blk.lo / kUnit + seg.from) * kUnit + kg * kStepKeys;   // the group's keys of the first unit
    const int part_begin = blk.lo >> 4, part_end = (blk.hi >> 4) + 1;

    // pages looked up 32 steps at a time: lane i has part i % 2 of step i / 2 of the batch
    auto batch = [&](int it) {
      const int at = it + (lane >> 1);
      return fetch_pool_parts(p, blk.r, at < take ? ((key0 + at * kUnit) >> 4) + (lane & 1) : -1, part_begin, part_end);
    };
    PoolParts parts = batch(0);
    auto slot_of = [&](int it) { return lds + (kg * NB + (NB > 1 ? it % NB : 0)) * kSlot; };

    // Step it's keys into its slot: the wave's share of them.  The result: which of its
    // two parts are in the pool.
    auto issue = [&](int it) {
      if (it > 0 && (it & 31) == 0) parts = batch(it);
      const uint32_t ok = (uint32_t)(parts.ok >> (2 * (it & 31))) & 3u;
      if (RW == 8 && ((wave >> 2) ^ it) & 1) return ok;
      const int pos = key0 + it * kUnit, first = (wr % LW) * NA * 8;       // first key that the wave loads
      if (pos > blk.hi || pos + kStepKeys <= blk.lo) return ok;            // no row sees any: not looked at
      const uint32_t to = slot_of(it) + first * kRowB;
      if (ok == 3u && pos >= blk.lo && pos + kStepKeys - 1 <= blk.hi) {
#pragma unroll
        for (int a = 0; a < NA; ++a) {
          const uint32_t odd = (first >> 3) + a & 1;
          const uint64_t base = lane_u64(parts.at, 2 * (it & 31) + ((first + 8 * a) >> 4)) + odd * (8 * (uint64_t)t_stride);
#pragma unroll
          for (int b = 0; b < LPG; ++b)
            load_lds((const uint8_t*)base, piece(b, odd), to + (a * LPG + b) * 1024);
        }
      } else {
        const uint64_t part0 = lane_u64(parts.at, 2 * (it & 31)), part1 = lane_u64(parts.at, 2 * (it & 31) + 1);
#pragma unroll 1
        for (int j = 0; j < NA * LPG; ++j) {
          const uint32_t i = j * 64 + lane, in_step = first + i / CH, c = (i % CH) ^ twist(in_step);
          const int key = pos + (int)in_step;
          const bool seen = ((ok >> (in_step >> 4)) & 1) && key >= blk.lo && key <= blk.hi;
          const uint64_t row = (in_step >> 4 ? part1 : part0) + (in_step & 15) * t_stride;
          load_lds((seen ? row : (uint64_t)g_zero_row) + c * 16, to + j * 1024);
        }
      }
      return ok;
    };
    uint32_t oks = 0;                              // two bits a slot
#pragma unroll
    for (int i = 0; i < (NB > 1 ? NB / 2 : 1); ++i)
      if (i < take) oks |= issue(i) << (2 * i);

    // this wave's rows; lane l has row l % 16 (past the end the last one, whose results
    // are not stored)
    const int wave_row = blk.row_first + wr * 16, row = min(wave_row + c16, blk.row_end - 1);
    const int64_t row0 = first_row(p.q_base, blk.r, p.n_queries);
    const int query = (int)fast_div((uint32_t)row, p.fd_group);
    bf16x8 qf[KS];
    int row_lo = INT32_MAX;                        // sees the keys row_lo .. row_lo + row_span, or none
    uint32_t row_span = 0;
    {
      const int last = mla_last_key(p, blk.n, blk.kv, query);
      if (last >= 0 && blk.kv > 0) {
        row_lo = mla_first_key(p, last);
        row_span = (uint32_t)(min(last, blk.kv - 1) - row_lo);
      }
      const uint16_t* src = p.q + (row0 + query) * p.q_s[0] + (int64_t)(row - query * p.group) * p.q_s[1] + g * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qf[ks] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(src + ks * 32) ^ p.q_sign);
    }
    f32x4 o[DT];
    float m = kLow, l = 0.f, lx = 0.f;
#pragma unroll
    for (int b = 0; b < DT; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (tid == 0) s_odd = 0;
    lds_barrier();

    // Scores and softmax of a step; the weights as the second product takes them.
    auto weigh = [&](int pos, uint32_t slot, uint32_t ok) {
      if constexpr (NW == 4) {                     // the queries in the accumulators' registers, of which there are enough
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+a"(qf[ks]));
#pragma unroll
        for (int b = 0; b < DT; ++b) asm volatile("" : "+v"(o[b]));
      }
      f32x4 sc[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) sc[u] = f32x4{0.f, 0.f, 0.f, 0.f};
      // operand i of 2 KS: inner step i / 2, keys 16 (i % 2) on; read kAhead products ahead
      auto rows = [&](int i) {
        return read_chunk(((slot + k_at) ^ ((i >> 1 & 1) << 6)) + (i >> 2) * 128 + (i & 1) * 16 * kRowB);
      };
      bf16x8 kf[2 * KS];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) kf[i] = rows(i);
#pragma unroll
      for (int i = 0; i < 2 * KS; ++i) {
        if (i + kAhead < 2 * KS) kf[i + kAhead] = rows(i + kAhead);
        sc[i & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[i], qf[i >> 1], sc[i & 1], 0, 0, 0);
      }
      pipeline<2 * KS, 1, kAhead>();

      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = sc[i >> 2][i & 3];
      if (ok != 3u || pos + kStepKeys - 1 > blk.all_hi || pos < blk.all_lo) {      // some row does not see it whole
        const int at = pos + 4 * g - row_lo;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const bool there = (ok >> (i >> 2)) & 1;
          x[i] = there && (uint32_t)(at + (16 * (i >> 2) + (i & 3))) <= row_span ? x[i] : -INFINITY;
        }
      }
      float top = max2(max2(max2(x[0], x[1]), max2(x[2], x[3])), max2(max2(x[4], x[5]), max2(x[6], x[7]))) * p.scale2;
      if (__ballot(top > m + kSlack) != 0) {
        const float m_new = fmaxf(m, max_x32(max_x16(top)));
        const float down = exp2_fast(m - m_new);
        m = m_new;
        l *= down;
        lx *= down;
#pragma unroll
        for (int b = 0; b < DT; ++b) o[b] *= down;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = exp2_fast(__builtin_fmaf(x[i], p.scale2, -m));
      if (p.lse != nullptr) lx += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
      const u32x4 w = {pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
      l = add_pair(w.w, add_pair(w.z, add_pair(w.y, add_pair(w.x, l))));
      return __builtin_bit_cast(bf16x8, w);
    };
    auto gather = [&](uint32_t slot, bf16x8 pf) {
      auto columns = [&](int b) {
        const uint32_t at = ((slot + v_at) ^ ((b & 3) << 5)) + (b >> 2) * 128;
        return join(read_columns(at), read_columns(at + 16 * kRowB));
      };
      bf16x8 vf[DT];
#pragma unroll
      for (int b = 0; b < kAhead; ++b) vf[b] = columns(b);
#pragma unroll
      for (int b = 0; b < DT; ++b) {
        if (b + kAhead < DT) vf[b + kAhead] = columns(b + kAhead);
        o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[b], pf, o[b], 0, 0, 0);
      }
      pipeline<DT, 2, kAhead>();
    };
    // The values of a group's slot without what is not finite, by its RW waves.
    auto clean = [&](uint32_t slot) {
      bool met = false;
      for (int i = wr * 64 + lane; i < kStepKeys * (LAT / 8); i += RW * 64)
        met |= clean_chunk(slot + (i / (LAT / 8)) * kRowB + (i % (LAT / 8)) * 16);
      if (met) s_odd = 1;
    };
    // a step in which the wave has work
    auto busy = [&](int pos) { return pos <= blk.hi && pos + kStepKeys > blk.lo && wave_row < blk.row_end; };

    if constexpr (NB == 1) {
      // a wave's keys are its own: no one else waits for them
      for (int it = 0; it < take; ++it) {
        const int pos = key0 + it * kUnit;
        vm_wait<0>();
        if (busy(pos)) {
          const bf16x8 pf = weigh(pos, slot_of(it), oks);
          if (mixed(blk, pos, kStepKeys)) clean(slot_of(it));
          gather(slot_of(it), pf);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (it + 1 < take) oks = issue(it + 1);
      }
    } else {
      // NB / 2 steps between barriers: their slots are read while the others are filled
      constexpr int kHalf = NB / 2;
#pragma unroll 1
      for (int it = 0; it < take; ++it) {
        if (it % kHalf == 0) {
          vm_wait<0>();
          lds_barrier();                           // the steps' keys are there, and the other slots are free
#pragma unroll
          for (int i = kHalf; i < NB; ++i) {
            const int s = (it + i) % NB;
            if (it + i < take) oks = (oks & ~(3u << (2 * s))) | (issue(it + i) << (2 * s));
          }
        }
        const int pos = key0 + it * kUnit;
        bf16x8 pf = {};
        if (busy(pos)) pf = weigh(pos, slot_of(it), (oks >> (2 * (it % NB))) & 3u);
        if (mixed(blk, pos - kg * kStepKeys, kUnit)) {             // the same for all waves
          lds_barrier();
          clean(slot_of(it));
          lds_barrier();
        }
        if (busy(pos)) gather(slot_of(it), pf);
      }
    }

    l = sum_x32(sum_x16(l));
    lx = sum_x32(sum_x16(lx));
    const bool direct = seg.whole();
    const int64_t part = ((int64_t)blockIdx.x * 2 + (segment > 0 ? 1 : 0)) * p.rows_block;
    ++segment;
    // Where a row's results belong: looked up before the waits below.
    struct Place {
      uint16_t* out;
      float* part_o;
      float* lse;
      float* part_ml;
    };
    auto place_of = [&](int out_row, int col) {
      const int i = (int)fast_div((uint32_t)out_row, p.fd_group);
      const int64_t hq = out_row - i * p.group, at = part + out_row - blk.row_first;
      Place d;
      d.out = p.out + (row0 + i) * p.out_s[0] + hq * p.out_s[1] + col;
      d.lse = p.lse != nullptr ? p.lse + (row0 + i) * p.lse_s[0] + hq * p.lse_s[1] : nullptr;
      d.part_o = p.part_o + at * LAT + col;
      d.part_ml = p.part_ml + at * 4;
      return d;
    };
    // A row's columns, [N] of four `step` apart.
    auto store = [&](const Place& d, int step, const auto& a, float mm, float ll, float lxx, bool lead) {
      constexpr int N = sizeof(a) / sizeof(f32x4);
      if (direct) {
        const float inv = ll == 0.f ? 0.f : 1.0f / ll;
#pragma unroll
        for (int n = 0; n < N; ++n)
          *reinterpret_cast<u32x2*>(d.out + n * step) =
              u32x2{pack_bf16x2(a[n].x * inv, a[n].y * inv), pack_bf16x2(a[n].z * inv, a[n].w * inv)};
        if (lead && d.lse != nullptr) *d.lse = row_lse(mm, lxx);
      } else {
#pragma unroll
        for (int n = 0; n < N; ++n) *reinterpret_cast<f32x4*>(d.part_o + n * step) = a[n];
        if (lead) *reinterpret_cast<f32x4*>(d.part_ml) = f32x4{mm, ll, lxx, 0.f};
      }
    };
    lds_barrier();                                 // the slots are free
    const bool odd = __builtin_amdgcn_readfirstlane(s_odd) != 0;   // cleared for the next task behind a barrier below
    if constexpr (KW == 1) {
      if (wave_row + c16 < blk.row_end) store(place_of(wave_row + c16, 4 * g), 16, o, m, l, lx, g == 0);
      lds_barrier();
    } else {
      // the groups' results are joined in LDS
      if (g == 0) {
        s_ml[wave][c16][0] = m;
        s_ml[wave][c16][1] = l;
        s_ml[wave][c16][2] = lx;
      }
      // kPer threads a row
      constexpr int kPer = kThr / (RW * 16);
      const int mine = tid / kPer, first = tid % kPer * 4;
      const Place place = place_of(blk.row_first + mine, first);
      float* tile = reinterpret_cast<float*>(s_buf);
#pragma unroll
      for (int b = 0; b < DT; ++b) *reinterpret_cast<f32x4*>(tile + (wave * 16 + c16) * kPad + b * 16 + 4 * g) = o[b];
      lds_barrier();
      float f[KW], mm = kLow, ll = 0.f, lxx = 0.f;
#pragma unroll
      for (int k = 0; k < KW; ++k) mm = fmaxf(mm, s_ml[k * RW + (mine >> 4)][mine & 15][0]);
#pragma unroll
      for (int k = 0; k < KW; ++k) {
        f[k] = exp2_fast(s_ml[k * RW + (mine >> 4)][mine & 15][0] - mm);
        ll += s_ml[k * RW + (mine >> 4)][mine & 15][1] * f[k];
        lxx += s_ml[k * RW + (mine >> 4)][mine & 15][2] * f[k];
      }
      constexpr int N = LAT / (4 * kPer);
      f32x4 a[N];
#pragma unroll
      for (int n = 0; n < N; ++n) a[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KW; ++k)
#pragma unroll
        for (int n = 0; n < N; ++n)
          a[n] += *reinterpret_cast<const f32x4*>(tile + (k * RW * 16 + mine) * kPad + first + n * kPer * 4) * f[k];
      if (blk.row_first + mine < blk.row_end) store(place, kPer * 4, a, mm, ll, lxx, first == 0);
      lds_barrier();
    }
    if (odd) {
      const int from = (blk.lo / kUnit + seg.from) * kUnit;
      add_nonfinite(p, blk, from, from + take * kUnit, NB == 1 ? kStepKeys : kUnit, LAT, direct, part, row0, [&](int key) {
        const int k = (int)fast_div((uint32_t)key >> 4, p.fd_page16);
        const int page = p.page_table[(int64_t)blk.r * p.pt_stride + k];
        if (page < 0 || page >= p.n_pool_pages) return (const uint16_t*)nullptr;
        return (const uint16_t*)(p.pool + page * p.pool_s[0] + (key - k * p.page_size) * p.pool_s[1]);
      });
    }
  }
}

namespace {

template <int LAT, int RW>
hipError_t launch_rows(const MlaParams& p, hipStream_t s) {
  static std::atomic<bool> done[kMaxDevices];
  const int slots = 4 * kStepKeys * (LAT + kRopeCols) * 2;
  const int tile = latent_groups(RW) > 1 ? latent_waves(RW) * 16 * (LAT + 4) * 4 : 0;
  const int lds = slots > tile ? slots : tile;
  const hipError_t e = ensure_lds_limit((const void*)attend_latent_kernel<LAT, RW>, lds, done);
  if (e != hipSuccess) return e;
  const uint32_t grid = (uint32_t)(p.n_parts > 0 ? p.n_parts : p.n_tasks);
  hipLaunchKernelGGL((attend_latent_kernel<LAT, RW>), dim3(grid), dim3(latent_waves(RW) * 64), lds, s, p);
  return hipGetLastError();
}

template <int LAT>
hipError_t launch_lat(const MlaParams& p, hipStream_t s) {
  switch (p.row_waves) {
    case 1: return launch_rows<LAT, 1>(p, s);
    case 2: return launch_rows<LAT, 2>(p, s);
    default: return launch_rows<LAT, 8>(p, s);
  }
}

}  // namespace

hipError_t launch_attend_latent(const MlaParams& p, hipStream_t s) {
  const hipError_t e = p.dim == 512 ? launch_lat<512>(p, s) : launch_lat<256>(p, s);
  if (e != hipSuccess || p.n_parts == 0) return e;
  return launch_mla_join(p, s);
}

}  // namespace kamera

// kamera_project_heads and kamera_expand_latent: rows times a matrix of its own for
// every head, of dense rows or of the rows of a paged pool.
//
// Tiles of BM rows and BN columns of one head, the inner index 64 at a time, with
// 32x32x16 bf16 MFMAs: out^T = W^T X^T, W^T's rows (the outputs' columns) the A
// operand and X's rows the B operand, so that a lane ends with four neighbouring
// columns of one row.  Both tiles go straight from global memory into LDS, the next
// step's while a step is computed.  W comes in either order: with a column's inputs
// together as X's rows, with a row's outputs together through transposed LDS reads.
//
// LDS: 16-byte chunks are exchanged by an exclusive-or with bits of the row number,
// so that the 16 lanes that read a chunk of 16 rows together, or four rows of 64
// bytes, spread over all banks.
//
// Bound by bytes where a head's matrix is narrow (8192 rows of 16 heads, 512 x 128:
// 170 MB, 26.8 us of kernel with rows in the cache, 39 us a call without), by the
// matrix pipe's supply where it is wide (16384 pool rows, 16 heads, 512 x 256: 69
// GFLOP in 84 us, 820 TFLOP/s; a library product of that shape takes 81): the pipe
// is busy a third of the time, waits for the next step's tiles the rest, and neither
// steps of 32 columns in more buffers (103 us) nor 128 x 256 tiles, two to a CU (108),
// nor workgroups that stay (94) feed it better.  A few rows are a chain of latencies
// (64 rows of 16 heads, 128 x 512: 4.2 us).

#include "kamera_latent.h"
#include "kamera_lds_device.h"

namespace kamera {

namespace {

// Place of 16-byte chunk c of row r in a tile of rows of STEP columns.
template <int STEP>
__device__ __forceinline__ uint32_t k_place(uint32_t r, uint32_t c) {
  static_assert(STEP == 64, "");
  return r * (STEP * 2) + ((c ^ ((r >> 1) & 7)) << 4);
}
// ... of a tile of rows of BN columns.
template <int BN>
__device__ __forceinline__ uint32_t n_place(uint32_t r, uint32_t c) {
  static_assert(BN >= 128, "");
  return r * (BN * 2) + ((c ^ (r & 3) << 2) << 4);
}

}  // namespace

// Waves: WM x WN, each BM / WM rows and BN / WN columns.  STEP inner columns a step; NS
// buffers, of which NS - 1 are being filled while one is read.
template <int BM, int BN, int WM, int WN, int STEP, int NS, bool WK>
__global__ __launch_bounds__(WM * WN * 64, 2) void project_kernel(ProjectParams) {
  const ProjectParams& p = kernel_params<ProjectParams>();
  constexpr int kProjThreads = WM * WN * 64;
  constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
  constexpr int kX = BM * STEP * 2, kW = BN * STEP * 2, kBuf = kX + kW, CH = STEP / 8;
  constexpr int LX = kX / 16 / kProjThreads, LW = kW / 16 / kProjThreads;   // loads a thread
  static_assert(LX >= 1 && LW >= 1 && TM >= 1 && TN >= 1, "");
  extern __shared__ u32x4 s_buf[];
  const uint32_t lds = lds_offset(s_buf);

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c32 = lane & 31, hf = lane >> 5;
  uint32_t task = (uint32_t)xcd_task(p.per_xcd);
  if (task >= (uint32_t)p.n_tasks) return;
  uint32_t d = fast_div(task, p.fd_rows);
  const uint32_t rb = task - d * p.n_row_blocks;
  task = d;
  d = fast_div(task, p.fd_cols);
  const uint32_t cb = task - d * p.n_col_blocks;
  task = d;
  d = fast_div(task, p.fd_heads);
  const int g = (int)(task - d * p.n_heads), r = (int)d;
  const int row0 = rb * BM, col0 = cb * BN;
  const int n_rows = p.paged ? min(max(p.kv_tokens[r], 0), p.n_keys) : p.n_rows;
  if (row0 >= n_rows) return;
  const int64_t first_row = p.paged && p.row_base != nullptr ? (int64_t)p.row_base[r] : (int64_t)r * p.n_keys;

  // this thread's chunks: rows tid / CH + .. of X (and of W where its inputs lie together);
  // the exchange of places is its own inverse
  uint64_t xa[LX];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < LX; ++i) {
    const int at = tid / CH + i * (kProjThreads / CH);
    const int row = min(row0 + at, n_rows - 1);
    int64_t e;
    if (p.paged) {
      const int k = (int)fast_div((uint32_t)row, p.fd_page);
      int page = p.page_table[(int64_t)r * p.pt_stride + k];
      if (page < 0 || page >= p.n_pool_pages) {
        page = 0;                                  // readable; its rows are not stored
        bad = true;
      }
      e = page * p.x_s[0] + (int64_t)(row - k * p.page_size) * p.x_s[1];
    } else {
      e = row * p.x_s[0] + g * p.x_s[1];
    }
    xa[i] = (uint64_t)(p.x + e) + k_place<STEP>(at, tid % CH) - at * (STEP * 2);
  }
  if (bad && p.status != nullptr) atomicOr(p.status, KAMERA_STATUS_BAD_PAGE);
  __shared__ int s_bad[WM * WN];
  const bool wave_bad = __ballot(bad) != 0;
  if (lane == 0) s_bad[wave] = wave_bad;
  uint64_t wa[LW];
#pragma unroll
  for (int i = 0; i < LW; ++i) {
    if (WK) {
      const int at = tid / CH + i * (kProjThreads / CH);
      const int col = min(col0 + at, p.n_out - 1);
      wa[i] = (uint64_t)(p.w + g * p.w_s[0] + col * p.w_s[2]) + k_place<STEP>(at, tid % CH) - at * (STEP * 2);
    } else {
      constexpr int kRow = BN / 8;
      const int at = tid / kRow + i * (kProjThreads / kRow);
      const int c = (int)((n_place<BN>(at, tid % kRow) - at * (BN * 2)) >> 4);
      const int col = min(col0 + 8 * c, p.n_out - 8);
      wa[i] = (uint64_t)(p.w + g * p.w_s[0] + at * p.w_s[1] + col);
    }
  }
  const uint64_t w_step = WK ? STEP * 2 : (uint64_t)(p.w_s[1] * (STEP * 2));
  auto load = [&](int buf) {
    const uint32_t at = lds + buf * kBuf + wave * 1024;
#pragma unroll
    for (int i = 0; i < LX; ++i) {
      load_lds(xa[i], at + i * (kProjThreads * 16));
      xa[i] += STEP * 2;
    }
#pragma unroll
    for (int i = 0; i < LW; ++i) {
      load_lds(wa[i], at + kX + i * (kProjThreads * 16));
      wa[i] += w_step;
    }
  };

  const int wm = wave / WN, wn = wave % WN;
  f32x16 acc[TN][TM];
#pragma unroll
  for (int a = 0; a < TN; ++a)
#pragma unroll
    for (int b = 0; b < TM; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.f;

  const int n_steps = p.n_in / STEP;
#pragma unroll
  for (int i = 0; i < NS - 1; ++i)
    if (i < n_steps) load(i);
  for (int step = 0, buf = 0; step < n_steps; ++step) {
    // the loads of the NS - 2 steps behind this one may be under way
    if (step + NS - 2 < n_steps) vm_wait<(NS - 2) * (LX + LW)>();
    else vm_wait<0>();
    lds_barrier();                                 // this step's tiles are there, and the buffer before is free
    if (step + NS - 1 < n_steps) load(buf == 0 ? NS - 1 : buf - 1);
    const uint32_t x = lds + buf * kBuf, w = x + kX;
    if (++buf == NS) buf = 0;
    // operands read a step of 16 ahead of their products
    bf16x8 xf[2][TM], wf[2][TN];
    auto read = [&](int ks) {
#pragma unroll
      for (int b = 0; b < TM; ++b) xf[ks & 1][b] = read_chunk(x + k_place<STEP>((wm * TM + b) * 32 + c32, 2 * ks + hf));
#pragma unroll
      for (int a = 0; a < TN; ++a) {
        const uint32_t col = (wn * TN + a) * 32;
        if (WK) {
          wf[ks & 1][a] = read_chunk(w + k_place<STEP>(col + c32, 2 * ks + hf));
        } else {
          const uint32_t i16 = lane & 15, k = 16 * ks + 8 * hf + (i16 >> 2);
          const uint32_t c = (col >> 3) + ((lane >> 4) & 1) * 2 + ((i16 & 3) >> 1);
          wf[ks & 1][a] = join(read_columns(w + n_place<BN>(k, c) + (i16 & 1) * 8),
                               read_columns(w + n_place<BN>(k + 4, c) + (i16 & 1) * 8));
        }
      }
    };
    read(0);
#pragma unroll
    for (int ks = 0; ks < STEP / 16; ++ks) {
      if (ks + 1 < STEP / 16) read(ks + 1);
#pragma unroll
      for (int a = 0; a < TN; ++a)
#pragma unroll
        for (int b = 0; b < TM; ++b)
          acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wf[ks & 1][a], xf[ks & 1][b], acc[a][b], 0, 0, 0);
    }
    // reads spread between the products of the step before
    constexpr int kReads = TM + (WK ? 1 : 2) * TN, kEach = (kReads + TM * TN - 1) / (TM * TN);
    __builtin_amdgcn_sched_group_barrier(kDsRead, kReads, 0);
#pragma unroll
    for (int ks = 0; ks + 1 < STEP / 16; ++ks)
#pragma unroll
      for (int i = 0; i < TM * TN; ++i) {
        __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
        __builtin_amdgcn_sched_group_barrier(kDsRead, kEach, 0);
      }
    __builtin_amdgcn_sched_group_barrier(kMfma, TM * TN, 0);
  }

  // Results through LDS, where a wave turns its own into rows: lanes of four columns of 32
  // rows would write 16 bytes of each of 32 lines at a time.
  lds_barrier();
  constexpr int kCols = TN * 32, kRowB = kCols * 2 + 16, kVec = kCols / 8, kRows = 64 / kVec;
  const uint32_t own = lds + wave * (32 * kRowB);
  const int64_t out_row0 = p.paged ? first_row : 0;
  int some_bad = 0;                                // rows that are not stored have to be looked up once more
#pragma unroll
  for (int i = 0; i < WM * WN; ++i) some_bad |= s_bad[i];
  some_bad = __builtin_amdgcn_readfirstlane(some_bad);
#pragma unroll
  for (int b = 0; b < TM; ++b) {
#pragma unroll
    for (int a = 0; a < TN; ++a)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *(__attribute__((address_space(3))) u32x2*)(uintptr_t)(own + c32 * kRowB + (a * 32 + 2 * i + 4 * hf) * 2) =
            u32x2{pack_bf16x2(acc[a][b][i], acc[a][b][i + 1]), pack_bf16x2(acc[a][b][i + 2], acc[a][b][i + 3])};
    const int col = col0 + wn * kCols + lane % kVec * 8;
#pragma unroll
    for (int j = 0; j < 32 / kRows; ++j) {
      const int in = j * kRows + lane / kVec, row = row0 + (wm * TM + b) * 32 + in;
      const u32x4 v = __builtin_bit_cast(u32x4, read_chunk(own + in * kRowB + lane % kVec * 16));
      bool there = row < n_rows && col < p.n_out;
      if (some_bad && there) {
        const int page = p.page_table[(int64_t)r * p.pt_stride + fast_div((uint32_t)row, p.fd_page)];
        there = page >= 0 && page < p.n_pool_pages;
      }
      if (there) st16(p.out + (out_row0 + row) * p.out_s[0] + g * p.out_s[1] + col, v);
    }
  }
}

namespace {

template <int BM, int BN, int WM, int WN, int STEP, int NS, bool WK>
hipError_t launch_tiles(const ProjectParams& p, hipStream_t s) {
  static std::atomic<bool> done[kMaxDevices];
  const int lds = NS * (BM + BN) * STEP * 2;
  const hipError_t e = ensure_lds_limit((const void*)project_kernel<BM, BN, WM, WN, STEP, NS, WK>, lds, done);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((project_kernel<BM, BN, WM, WN, STEP, NS, WK>), dim3((uint32_t)p.per_xcd * 8), dim3(WM * WN * 64), lds, s, p);
  return hipGetLastError();
}

template <bool WK>
hipError_t launch_order(const ProjectParams& p, hipStream_t s) {
  switch (p.tile_rows) {
    case 32: return launch_tiles<32, 128, 1, 4, 64, 3, WK>(p, s);
    case 128: return launch_tiles<128, 128, 2, 2, 64, 2, WK>(p, s);
    default: return launch_tiles<256, 256, 2, 4, 64, 2, WK>(p, s);
  }
}

}  // namespace

hipError_t launch_project(const ProjectParams& p, hipStream_t s) {
  return p.w_k ? launch_order<true>(p, s) : launch_order<false>(p, s);
}

}  // namespace kamera

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

#include "kamera_latent.h"
#include "kamera_lds_device.h"

namespace kamera {

namespace {

constexpr int kProjThreads = 256;
constexpr int kStep = 64;                          // inner columns a step

// Place of 16-byte chunk c of row r in a tile of 128-byte rows.
__device__ __forceinline__ uint32_t k_place(uint32_t r, uint32_t c) { return r * 128 + ((c ^ ((r >> 1) & 7)) << 4); }
// ... of a tile of rows of BN columns.
template <int BN>
__device__ __forceinline__ uint32_t n_place(uint32_t r, uint32_t c) {
  return r * (BN * 2) + ((c ^ (BN >= 128 ? (r & 3) << 2 : (r & 2) << 1)) << 4);
}

}  // namespace

// Waves: WM x WN, each BM / WM rows and BN / WN columns.
template <int BM, int BN, int WM, int WN, bool WK>
__global__ __launch_bounds__(kProjThreads, 2) void project_kernel(ProjectParams) {
  const ProjectParams& p = kernel_params<ProjectParams>();
  constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
  constexpr int kX = BM * 128, kW = BN * 128, kBuf = kX + kW;
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

  // this thread's chunks: rows tid / 8 + 32 i of X (and of W where its inputs lie together)
  uint64_t xa[LX];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < LX; ++i) {
    const int at = tid / 8 + i * (kProjThreads / 8);
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
    xa[i] = (uint64_t)(p.x + e) + (((tid & 7) ^ ((at >> 1) & 7)) << 4);
  }
  if (p.paged && bad && p.status != nullptr) atomicOr(p.status, KAMERA_STATUS_BAD_PAGE);
  uint64_t wa[LW];
#pragma unroll
  for (int i = 0; i < LW; ++i) {
    if (WK) {
      const int at = tid / 8 + i * (kProjThreads / 8);
      const int col = min(col0 + at, p.n_out - 1);
      wa[i] = (uint64_t)(p.w + g * p.w_s[0] + col * p.w_s[2]) + (((tid & 7) ^ ((at >> 1) & 7)) << 4);
    } else {
      constexpr int kRow = BN / 8;
      const int at = tid / kRow + i * (kProjThreads / kRow);
      const int c = (int)((n_place<BN>(at, tid % kRow) - at * (BN * 2)) >> 4);   // the exchange is its own inverse
      const int col = min(col0 + 8 * c, p.n_out - 8);
      wa[i] = (uint64_t)(p.w + g * p.w_s[0] + at * p.w_s[1] + col);
    }
  }
  const uint64_t w_step = WK ? kStep * 2 : (uint64_t)(p.w_s[1] * (kStep * 2));
  auto load = [&](int buf) {
    const uint32_t at = lds + buf * kBuf + wave * 1024;
#pragma unroll
    for (int i = 0; i < LX; ++i) {
      load_lds(xa[i], at + i * (kProjThreads * 16));
      xa[i] += kStep * 2;
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

  const int n_steps = p.n_in / kStep;
  load(0);
  for (int step = 0; step < n_steps; ++step) {
    vm_wait<0>();
    lds_barrier();                                 // this step's tiles are there, and the other buffer is free
    if (step + 1 < n_steps) load((step + 1) & 1);
    const uint32_t x = lds + (step & 1) * kBuf, w = x + kX;
#pragma unroll
    for (int ks = 0; ks < kStep / 16; ++ks) {
      bf16x8 xf[TM], wf[TN];
#pragma unroll
      for (int b = 0; b < TM; ++b) xf[b] = read_chunk(x + k_place((wm * TM + b) * 32 + c32, 2 * ks + hf));
#pragma unroll
      for (int a = 0; a < TN; ++a) {
        const uint32_t col = (wn * TN + a) * 32;
        if (WK) {
          wf[a] = read_chunk(w + k_place(col + c32, 2 * ks + hf));
        } else {
          const uint32_t i16 = lane & 15, k = 16 * ks + 8 * hf + (i16 >> 2);
          const uint32_t c = (col >> 3) + ((lane >> 4) & 1) * 2 + ((i16 & 3) >> 1);
          wf[a] = join(read_columns(w + n_place<BN>(k, c) + (i16 & 1) * 8),
                       read_columns(w + n_place<BN>(k + 4, c) + (i16 & 1) * 8));
        }
      }
#pragma unroll
      for (int a = 0; a < TN; ++a)
#pragma unroll
        for (int b = 0; b < TM; ++b) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wf[a], xf[b], acc[a][b], 0, 0, 0);
    }
  }

  const int64_t out_row0 = p.paged ? (p.row_base != nullptr ? (int64_t)p.row_base[r] : (int64_t)r * p.n_keys) : 0;
#pragma unroll
  for (int b = 0; b < TM; ++b) {
    const int row = row0 + (wm * TM + b) * 32 + c32;
    if (row >= n_rows) continue;
    if (p.paged) {
      const int page = p.page_table[(int64_t)r * p.pt_stride + fast_div((uint32_t)row, p.fd_page)];
      if (page < 0 || page >= p.n_pool_pages) continue;
    }
    uint16_t* dst = p.out + (out_row0 + row) * p.out_s[0] + g * p.out_s[1];
#pragma unroll
    for (int a = 0; a < TN; ++a)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int col = col0 + (wn * TN + a) * 32 + 2 * i + 4 * hf;
        if (col < p.n_out)
          *reinterpret_cast<u32x2*>(dst + col) =
              u32x2{pack_bf16x2(acc[a][b][i], acc[a][b][i + 1]), pack_bf16x2(acc[a][b][i + 2], acc[a][b][i + 3])};
      }
  }
}

namespace {

template <int BM, int BN, int WM, int WN, bool WK>
hipError_t launch_tiles(const ProjectParams& p, hipStream_t s) {
  static std::atomic<bool> done[kMaxDevices];
  const int lds = 2 * (BM + BN) * 128;
  const hipError_t e = ensure_lds_limit((const void*)project_kernel<BM, BN, WM, WN, WK>, lds, done);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((project_kernel<BM, BN, WM, WN, WK>), dim3((uint32_t)p.per_xcd * 8), dim3(kProjThreads), lds, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_project(const ProjectParams& p, hipStream_t s) {
  if (p.small) return p.w_k ? launch_tiles<32, 128, 1, 4, true>(p, s) : launch_tiles<32, 128, 1, 4, false>(p, s);
  return p.w_k ? launch_tiles<128, 128, 2, 2, true>(p, s) : launch_tiles<128, 128, 2, 2, false>(p, s);
}

}  // namespace kamera

// The second kernel of the attentions over a latent cache: joins the parts of rows
// whose keys were divided among workgroups.
//
// With M the largest of the parts' maxima m_s,
//   out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s.
// 32 threads take 128 columns of a row's parts: with WAYS > 1 every WAYS-th part, the
// ways meeting in LDS, else all of them, for one row or for four.  Tasks that were
// divided are found from where the workgroups' ranges begin: a grid over the ranges where
// there are fewer of them than tasks, else over the tasks.
//
// Bound by latency: a launch, four dependent loads (the task's lengths, its cost, the
// parts, their sums), and the parts once from the cache beyond the L2s, at 76 MB in
// 15.6 us (16 requests of 256 rows of 512 columns in 256 ranges), 25 MB in 10 (48 rows
// in 256 parts).

#include "kamera_mla_device.h"

namespace kamera {

// A row's running maximum, sums and four columns.
struct Sum {
  float top, l, lx;
  f32x4 acc;
  // Two such sums become one.
  __device__ __forceinline__ void add(const Sum& b) {
    const float m = fmaxf(top, b.top), f = exp2_fast(top - m), g = exp2_fast(b.top - m);
    top = m;
    l = l * f + b.l * g;
    lx = lx * f + b.lx * g;
    acc = acc * f + b.acc * g;
  }
};

// OWN: rows of a thread, 8 apart.
template <int WAYS, int OWN>
__global__ __launch_bounds__(WAYS > 1 ? WAYS * 32 : 256) void mla_join_kernel(MlaParams) {
  const MlaParams& p = kernel_params<MlaParams>();
  constexpr int kChunk = OWN > 1 ? 2 : 8;          // parts of a row that a thread has in flight
  __shared__ f32x4 s_o[WAYS > 1 ? WAYS : 1][32];
  __shared__ float s_ml[WAYS > 1 ? WAYS : 1][3];
  const int tid = threadIdx.x, col = tid & 31, way = WAYS > 1 ? tid >> 5 : 0;
  const int per = uniform_load(p.prefix + p.n_tasks);
  // the task, and the workgroups w0 .. w1 that share it
  const bool by_task = p.n_tasks < p.n_parts;
  const int task = by_task ? (int)blockIdx.x : uniform_load(p.prefix + p.n_tasks + 2 + blockIdx.x);
  if (task >= p.n_tasks) return;
  const Block blk = block_of(p, task);
  const int n_units = units_of(blk, p.unit);
  if (n_units == 0) return;
  // (the cost before it, and then p.fixed in which nothing is walked)
  const int u0 = uniform_load(p.prefix + task), w0 = (u0 + p.fixed) / per, w1 = (u0 + p.fixed + n_units - 1) / per;
  if (w0 == w1 || (!by_task && (int)blockIdx.x != w0)) return;     // one workgroup had it all, or not its first range
  const int quarters = (p.dim + 127) >> 7, cq = blockIdx.y % quarters;
  const int rr = blockIdx.y / quarters * (WAYS > 1 ? 1 : 8 * OWN) + (WAYS > 1 ? 0 : tid >> 5);
  if (blk.row_first + rr >= blk.row_end) return;   // of all threads where they meet in LDS
  const int c0 = cq * 128 + col * 4;
  const bool there = c0 < p.dim;
  // the first part is its workgroup's first segment only where that's range begins with it
  const int first_slot = w0 * per >= u0 ? 0 : 1;

  Sum sum[OWN];
#pragma unroll
  for (int n = 0; n < OWN; ++n) sum[n] = {kLow, 0.f, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
  for (int s0 = w0 + way; s0 <= w1; s0 += kChunk * WAYS) {
    f32x4 ml[OWN][kChunk], o[OWN][kChunk];
#pragma unroll
    for (int n = 0; n < OWN; ++n)
#pragma unroll
      for (int k = 0; k < kChunk; ++k) {
        // a part or row past the end is read again and left out
        const int s = min(s0 + k * WAYS, w1), row = min(rr + 8 * n, blk.row_end - blk.row_first - 1);
        const int64_t at = ((int64_t)s * 2 + (s == w0 ? first_slot : 0)) * p.rows_block + row;
        ml[n][k] = *reinterpret_cast<const f32x4*>(p.part_ml + at * 4);
        o[n][k] = *reinterpret_cast<const f32x4*>(p.part_o + at * p.dim + (there ? c0 : 0));
      }
#pragma unroll
    for (int n = 0; n < OWN; ++n) {
      float m = sum[n].top;
#pragma unroll
      for (int k = 0; k < kChunk; ++k) m = fmaxf(m, ml[n][k].x);
      const float down = exp2_fast(sum[n].top - m);
      sum[n].top = m;
      sum[n].l *= down;
      sum[n].lx *= down;
      sum[n].acc *= down;
#pragma unroll
      for (int k = 0; k < kChunk; ++k)
        if (s0 + k * WAYS <= w1) {
          const float f = exp2_fast(ml[n][k].x - m);
          sum[n].l += ml[n][k].y * f;
          sum[n].lx += ml[n][k].z * f;
          sum[n].acc += o[n][k] * f;
        }
    }
  }
  if (WAYS > 1) {
    s_o[WAYS > 1 ? way : 0][col] = sum[0].acc;
    if (col == 0) {
      s_ml[WAYS > 1 ? way : 0][0] = sum[0].top;
      s_ml[WAYS > 1 ? way : 0][1] = sum[0].l;
      s_ml[WAYS > 1 ? way : 0][2] = sum[0].lx;
    }
    __syncthreads();
    if (way != 0) return;
#pragma unroll
    for (int k = 1; k < WAYS; ++k)
      sum[0].add({s_ml[WAYS > 1 ? k : 0][0], s_ml[WAYS > 1 ? k : 0][1], s_ml[WAYS > 1 ? k : 0][2], s_o[WAYS > 1 ? k : 0][col]});
  }
  const int64_t row0 = first_row(p.q_base, blk.r, p.n_queries);
#pragma unroll
  for (int n = 0; n < OWN; ++n) {
    const int row = blk.row_first + rr + 8 * n;
    if (row >= blk.row_end) break;
    const int i = (int)fast_div((uint32_t)row, p.fd_group);
    const int64_t hq = (int64_t)blk.h * p.group + row - i * p.group;
    const f32x4 a = sum[n].acc * (sum[n].l == 0.f ? 0.f : 1.0f / sum[n].l);
    if (there)
      *reinterpret_cast<u32x2*>(p.out + (row0 + i) * p.out_s[0] + hq * p.out_s[1] + c0) =
          u32x2{pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w)};
    if (cq == 0 && col == 0 && p.lse != nullptr)
      p.lse[(row0 + i) * p.lse_s[0] + hq * p.lse_s[1]] = row_lse(sum[n].top, sum[n].lx);
  }
}

hipError_t launch_mla_join(const MlaParams& p, hipStream_t s) {
  if (p.n_parts == 1) return hipSuccess;           // no task was divided
  const int64_t most = (int64_t)p.n_queries * p.group;
  const uint32_t rows = (uint32_t)(most < p.rows_block ? most : p.rows_block), quarters = (uint32_t)(p.dim + 127) >> 7;
  const uint32_t x = (uint32_t)(p.n_tasks < p.n_parts ? p.n_tasks : p.n_parts - 1);
  // Many parts of few rows: a workgroup a row and 128 columns (256 parts of 48 rows of 512 columns, 192 workgroups: 40 us
  // with the attention, 77 with eight rows a workgroup; 768 workgroups 43.3 and 44.3, 1536 workgroups 52.3 and 39.6).
  // Else all parts by one thread, and four rows of it where ranges share few tasks (1024 tasks in 512 ranges: 14.7 us,
  // 20 one row a thread).
  if (p.n_parts >= 16 * (int64_t)p.n_tasks && x * rows * quarters <= 512)
    hipLaunchKernelGGL((mla_join_kernel<16, 1>), dim3(x, rows * quarters), dim3(512), 0, s, p);
  else if (p.n_tasks < p.n_parts)
    hipLaunchKernelGGL((mla_join_kernel<1, 1>), dim3(x, (rows + 7) / 8 * quarters), dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL((mla_join_kernel<1, 4>), dim3(x, (rows + 31) / 32 * quarters), dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace kamera

// The second kernel of the attentions over a latent cache: joins the parts of rows
// whose keys were divided among workgroups.
//
// With M the largest of the parts' maxima m_s,
//   out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s.
// 32 threads take 128 columns of a row's parts; with WAYS = 8 every eighth part, the
// ways meeting in LDS, else eight rows a workgroup.  Tasks that were divided are found
// from where the workgroups' ranges begin: a grid over the ranges where there are
// fewer of them than tasks, else over the tasks.

#include "kamera_mla_device.h"

namespace kamera {

namespace {

constexpr int kJoinThreads = 256;

}  // namespace

template <int WAYS>
__global__ __launch_bounds__(kJoinThreads) void mla_join_kernel(MlaParams) {
  const MlaParams& p = kernel_params<MlaParams>();
  constexpr int kChunk = 4, kRows = 8 / WAYS;
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
  const int rr = blockIdx.y / quarters * kRows + (WAYS > 1 ? 0 : tid >> 5);
  const int row = blk.row_first + rr;
  if (row >= blk.row_end) return;                  // of all 256 threads where they meet in LDS
  const int c0 = cq * 128 + col * 4;
  const bool there = c0 < p.dim;
  // the first part is its workgroup's first segment only where that's range begins with it
  const int first_slot = w0 * per >= u0 ? 0 : 1;

  float top = kLow, l = 0.f, lx = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = w0 + way; s0 <= w1; s0 += kChunk * WAYS) {
    f32x4 ml[kChunk], o[kChunk];
#pragma unroll
    for (int k = 0; k < kChunk; ++k) {
      const int s = min(s0 + k * WAYS, w1);        // one past the end is read again and left out
      const int64_t at = ((int64_t)s * 2 + (s == w0 ? first_slot : 0)) * p.rows_block + rr;
      ml[k] = *reinterpret_cast<const f32x4*>(p.part_ml + at * 4);
      o[k] = *reinterpret_cast<const f32x4*>(p.part_o + at * p.dim + (there ? c0 : 0));
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
      if (s0 + k * WAYS <= w1) {
        const float f = exp2_fast(ml[k].x - top);
        l += ml[k].y * f;
        lx += ml[k].z * f;
        acc += o[k] * f;
      }
  }
  if (WAYS > 1) {
    s_o[WAYS > 1 ? way : 0][col] = acc;
    if (col == 0) {
      s_ml[WAYS > 1 ? way : 0][0] = top;
      s_ml[WAYS > 1 ? way : 0][1] = l;
      s_ml[WAYS > 1 ? way : 0][2] = lx;
    }
    __syncthreads();
    if (way != 0) return;
    const float own = top;
#pragma unroll
    for (int k = 1; k < WAYS; ++k) top = fmaxf(top, s_ml[k][0]);
    const float down = exp2_fast(own - top);
    l *= down;
    lx *= down;
    acc *= down;
#pragma unroll
    for (int k = 1; k < WAYS; ++k) {
      const float f = exp2_fast(s_ml[k][0] - top);
      l += s_ml[k][1] * f;
      lx += s_ml[k][2] * f;
      acc += s_o[k][col] * f;
    }
  }
  const int64_t row0 = first_row(p.q_base, blk.r, p.n_queries);
  const int i = (int)fast_div((uint32_t)row, p.fd_group);
  const int64_t hq = (int64_t)blk.h * p.group + row - i * p.group;
  acc *= l == 0.f ? 0.f : 1.0f / l;
  if (there)
    *reinterpret_cast<u32x2*>(p.out + (row0 + i) * p.out_s[0] + hq * p.out_s[1] + c0) =
        u32x2{pack_bf16x2(acc.x, acc.y), pack_bf16x2(acc.z, acc.w)};
  if (cq == 0 && col == 0 && p.lse != nullptr) p.lse[(row0 + i) * p.lse_s[0] + hq * p.lse_s[1]] = row_lse(top, lx);
}

hipError_t launch_mla_join(const MlaParams& p, hipStream_t s) {
  if (p.n_parts == 1) return hipSuccess;           // no task was divided
  const int64_t most = (int64_t)p.n_queries * p.group;
  const uint32_t rows = (uint32_t)(most < p.rows_block ? most : p.rows_block), quarters = (uint32_t)(p.dim + 127) >> 7;
  const uint32_t x = (uint32_t)(p.n_tasks < p.n_parts ? p.n_tasks : p.n_parts - 1);
  // eight ways where a task has many parts
  if (p.n_parts >= 16 * (int64_t)p.n_tasks)
    hipLaunchKernelGGL(mla_join_kernel<8>, dim3(x, rows * quarters), dim3(kJoinThreads), 0, s, p);
  else
    hipLaunchKernelGGL(mla_join_kernel<1>, dim3(x, (rows + 7) / 8 * quarters), dim3(kJoinThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace kamera

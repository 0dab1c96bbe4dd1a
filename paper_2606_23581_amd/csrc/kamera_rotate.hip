// kamera_append_rotated: rows of new tokens into the bf16 paged pool, with their
// rotary positions applied on the way, and the rope bands of their queries.
//
// A pair (x, y) of a row at position p becomes a (x cos f p - y sin f p,
// x sin f p + y cos f p).  Bound by HBM: every row is read and written once and
// there are three multiplications for each rotated element.  What would cost more
// is the angles, in fp64 for far positions: a workgroup takes a few tokens of one
// (chunk, layer) and works their cosines and sines out once, into LDS, for the
// heads of all three planes.  6270 tokens (eight ragged prompts) of 8 x 128 columns of K and V
// and the bands of 64 query heads (257 MB): 54 us, 4.8 TB/s.  Two pieces a thread at a time,
// which leaves room for more waves (60.2 us, four 68.6), and past the caches (56.8 us
// beside 60.2).

#include "kamera_device.h"
#include "kamera_latent.h"

namespace kamera {

namespace {

constexpr int kRotThreads = 256;
constexpr int kBatch = 2;                          // pieces a thread has in flight

// Piece `it` of a head's row: its 16-byte vector, and the partner of a NeoX pair.
struct Piece {
  int vec, other;                                  // other < 0: none
  int pair;                                        // first rotated pair; < 0: a copy
};

__device__ __forceinline__ Piece piece_of(const RotateParams& p, const RotatePlane& pl, int it) {
  Piece x;
  if (it >= pl.band_items) {
    const int v = it - pl.band_items, first = p.rope.rope_dim >> 3;
    x.vec = v + (v >= pl.band_vec ? (pl.band_items > 0 ? first : 0) : 0);
    x.other = x.pair = -1;
  } else if (p.rope.pairing == KAMERA_PAIR_NEOX) {
    x.vec = pl.band_vec + it;
    x.other = x.vec + (p.rope.rope_dim >> 4);
    x.pair = it * 8;
  } else {
    x.vec = pl.band_vec + it;
    x.other = -1;
    x.pair = it * 4;
  }
  return x;
}

// Eight NeoX pairs: a holds the x, b the y.
__device__ __forceinline__ void turn_halves(u32x4& a, u32x4& b, const f32x2* cs) {
  u32x4 ra, rb;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t wa = u4_get(a, k), wb = u4_get(b, k);
    const f32x2 c0 = cs[2 * k], c1 = cs[2 * k + 1];
    const float x0 = bf_lo(wa), x1 = bf_hi(wa), y0 = bf_lo(wb), y1 = bf_hi(wb);
    ra[k] = pack_bf16x2(x0 * c0.x - y0 * c0.y, x1 * c1.x - y1 * c1.y);
    rb[k] = pack_bf16x2(x0 * c0.y + y0 * c0.x, x1 * c1.y + y1 * c1.x);
  }
  a = ra;
  b = rb;
}

// Four interleaved pairs.
__device__ __forceinline__ void turn_neighbours(u32x4& a, const f32x2* cs) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t w = u4_get(a, k);
    const float x = bf_lo(w), y = bf_hi(w);
    a[k] = pack_bf16x2(x * cs[k].x - y * cs[k].y, x * cs[k].y + y * cs[k].x);
  }
}

}  // namespace

__global__ __launch_bounds__(kRotThreads) void rotate_kernel(RotateParams) {
  const RotateParams& p = kernel_params<RotateParams>();
  __shared__ f32x2 s_cs[kRotateTokens][kMaxPairs];
  __shared__ int64_t s_page[kRotateTokens];        // page of the token, or -1
  __shared__ int s_in[kRotateTokens];              // its place in the page

  uint32_t w = blockIdx.x, d = fast_div(w, p.fd_blocks);
  const int blk = (int)(w - d * p.n_blocks);
  w = d;
  d = fast_div(w, p.fd_layers);
  const int l = (int)(w - d * p.n_layers), c = (int)d;
  const int n = p.chunk_tokens != nullptr ? min(max(p.chunk_tokens[c], 0), p.n_tokens) : p.n_tokens;
  const int first = blk * p.block_tokens, m = min(n - first, p.block_tokens);
  if (m <= 0) return;
  const int before = p.tokens_before != nullptr ? max(p.tokens_before[c], 0) : 0;
  const int64_t base = (p.row_base != nullptr ? p.row_base[c] : 0) + (int64_t)first;
  const int tid = threadIdx.x;

  const int half = p.rope.rope_dim >> 1;
  for (int e = tid; e < m * kMaxPairs; e += kRotThreads) {
    const int t = e / kMaxPairs, j = e % kMaxPairs;
    if (j >= half) continue;
    double pos;
    if (p.positions != nullptr)
      pos = p.positions[c * p.position_s[0] + (base + t) * p.position_s[1] + p.rope.coord[j] * p.position_s[2]];
    else
      pos = (double)((int64_t)before + first + t);
    float s, co;
    sincos_rev(pos, p.rope.rev_freq[j], s, co);
    s_cs[t][j] = f32x2{co * p.amplitude, s * p.amplitude};
  }
  if (tid < m) {
    const int64_t tok = (int64_t)before + first + tid;
    int64_t page = -1, k = 0;
    if (tok > INT32_MAX) {
      if (p.status != nullptr) atomicOr(p.status, KAMERA_STATUS_BAD_LENGTH);
    } else {
      k = fast_div((uint32_t)tok, p.fd_page);
      if (k >= p.pt_pages) {
        if (p.status != nullptr) atomicOr(p.status, KAMERA_STATUS_BAD_LENGTH);
      } else {
        page = p.page_table[(int64_t)c * p.pt_stride + k];
        if (page < 0 || page >= p.n_pool_pages) {
          page = -1;
          if (p.status != nullptr) atomicOr(p.status, KAMERA_STATUS_BAD_PAGE);
        }
      }
    }
    s_page[tid] = page;
    s_in[tid] = (int)(tok - k * p.page_size);
  }
  __syncthreads();

#pragma unroll
  for (int pi = 0; pi < 3; ++pi) {
    const RotatePlane& pl = p.plane[pi];
    const int total = m * pl.n_heads * pl.n_items;
    for (int e0 = tid; e0 < total; e0 += kRotThreads * kBatch) {
      u32x4 a[kBatch], b[kBatch];
      uint16_t* dst[kBatch];
      int t[kBatch];
      Piece x[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int e = e0 + u * kRotThreads;
        dst[u] = nullptr;
        if (e >= total) continue;
        const uint32_t row = fast_div((uint32_t)e, pl.fd_items);
        const uint32_t tt = fast_div(row, pl.fd_heads);
        const int h = (int)(row - tt * pl.n_heads);
        t[u] = (int)tt;
        x[u] = piece_of(p, pl, e - (int)row * pl.n_items);
        if (pi == 2) {
          dst[u] = pl.out + c * pl.out_s[0] + l * pl.out_s[1] + (base + t[u]) * pl.out_s[2] + h * pl.out_s[3];
        } else {
          if (s_page[t[u]] < 0) continue;
          dst[u] = pl.out + l * pl.out_s[0] + s_page[t[u]] * pl.out_s[1] + s_in[t[u]] * pl.out_s[2] + h * pl.out_s[3];
        }
        const uint16_t* src = pl.in + c * pl.in_s[0] + l * pl.in_s[1] + (base + t[u]) * pl.in_s[2] + h * pl.in_s[3];
        a[u] = ld16(src + 8 * x[u].vec);
        if (x[u].other >= 0) b[u] = ld16(src + 8 * x[u].other);
      }
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        if (dst[u] == nullptr) continue;
        if (x[u].other >= 0) {
          turn_halves(a[u], b[u], &s_cs[t[u]][x[u].pair]);
          st16(dst[u] + 8 * x[u].other, b[u]);
        } else if (x[u].pair >= 0) {
          turn_neighbours(a[u], &s_cs[t[u]][x[u].pair]);
        }
        st16(dst[u] + 8 * x[u].vec, a[u]);
      }
    }
  }
}

hipError_t launch_rotate(const RotateParams& p, hipStream_t s) {
  hipLaunchKernelGGL(rotate_kernel, dim3((uint32_t)p.n_tasks), dim3(kRotThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace kamera

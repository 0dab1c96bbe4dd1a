// kamera_append_paged8: bf16 rows into the 8-bit paged cache.
//
// Unit = (chunk, layer, page of the chunk, plane, head); a wave takes 16 of its
// tokens, so a unit is one, two or four waves of a 4-wave workgroup, whose units
// are neighbouring heads of the same rows.  With A the
// largest finite |x| of the page's new rows, e = min { e : A <= 448 * 2^e } is
// read off A's bf16 bits: 448 = 1.75 * 2^8, so e = exponent(A) - 8, one more
// where the fraction of A passes 1.75.  Scaling by 2^-e is exact, so one
// rounding (v_cvt_pk_fp8_f32, to nearest even) stands between the row and its
// byte, and a second one only where a later call raises the page's e and the
// byte leaves the normal range.  Any correct implementation stores the same
// bytes for the same calls.
//
// Bound by HBM: 2 bytes read and 1 written for each element.  Waves keep their
// rows in registers between the maximum and the conversion, so rows are read
// once; the page's key sums come from the converted bytes that they still hold.
// 64 chunks of 1024 tokens, 8 heads, 4 layers: 329 us, 4.95 TB/s.
// (One wave for a whole 64-token page: 1024-token chunks of 8 requests, one layer
// of 8 heads, took 20.3 us.)

#include "kamera_cache_device.h"

namespace kamera {

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  const u16x2 x = __builtin_bit_cast(u16x2, a), y = __builtin_bit_cast(u16x2, b);
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(x, y));
}

__device__ __forceinline__ int clamp_exp(int e) { return e < kMinExp ? kMinExp : (e > kMaxExp ? kMaxExp : e); }

__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Eight bf16 values times 2^-e as e4m3 bytes.
__device__ __forceinline__ u32x2 to_e4m3(u32x4 w, float inv) {
  u32x2 r = {0u, 0u};
  r.x = __builtin_amdgcn_cvt_pk_fp8_f32(bf_lo(w.x) * inv, bf_hi(w.x) * inv, r.x, false);
  r.x = __builtin_amdgcn_cvt_pk_fp8_f32(bf_lo(w.y) * inv, bf_hi(w.y) * inv, r.x, true);
  r.y = __builtin_amdgcn_cvt_pk_fp8_f32(bf_lo(w.z) * inv, bf_hi(w.z) * inv, r.y, false);
  r.y = __builtin_amdgcn_cvt_pk_fp8_f32(bf_lo(w.w) * inv, bf_hi(w.w) * inv, r.y, true);
  return r;
}

__device__ __forceinline__ void from_e4m3(u32x2 w, float (&f)[8]) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w.x, true);
  const f32x2 c = __builtin_amdgcn_cvt_pk_f32_fp8(w.y, false), d = __builtin_amdgcn_cvt_pk_f32_fp8(w.y, true);
  f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y;
  f[4] = c.x; f[5] = c.y; f[6] = d.x; f[7] = d.y;
}

}  // namespace

// D columns, SUB 16-token parts (and waves) a page.  A row takes D / 8 lanes of 8 columns.
template <int D, int SUB>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(AppendParams) {
  constexpr int LPR = D / 8;                       // lanes a row
  constexpr int TPI = 64 / LPR;                    // tokens a step of the wave
  constexpr int IT = 16 / TPI;                     // steps
  constexpr int P = SUB * 16;
  constexpr int kWaves = kAppendThreads / 64, kUnits = kWaves / SUB;
  const AppendParams& p = kernel_params<AppendParams>();
  __shared__ uint32_t s_top[kWaves];
  __shared__ float s_sum[SUB > 1 ? kWaves : 1][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int sub = wave % SUB, wave0 = wave - sub;  // this wave's part, the unit's first wave
  const uint32_t unit = blockIdx.x * kUnits + wave / SUB;
  bool live = unit < (uint32_t)p.n_units;
  if (SUB == 1 && !live) return;
  uint32_t u = live ? unit : 0u, q;
  q = fast_div(u, p.fd_heads);
  const int h = (int)(u - q * p.n_heads);
  const int pl = (int)(q & 1);
  u = q >> 1;
  q = fast_div(u, p.fd_pages);
  const int jp = (int)(u - q * p.pages);
  u = q;
  q = fast_div(u, p.fd_layers);
  const int l = (int)(u - q * p.n_layers), c = (int)q;

  const int base = load_or(p.row_base, c, 0, p.page_table);
  const int before = max(load_or(p.tokens_before, c, 0, p.page_table), 0);
  const int n = min(max(load_or(p.chunk_tokens, c, p.n_tokens, p.page_table), 0), p.n_tokens);
  const int64_t j = before / P + jp;               // page of the chunk
  const int64_t p0 = j * P;
  const int64_t lo64 = max((int64_t)before, p0) - p0, hi64 = min((int64_t)before + n, p0 + P) - p0;
  live = live && hi64 > lo64;
  if (SUB == 1 && !live) return;
  const int lo = (int)lo64, hi = (int)hi64;        // new tokens of the page: [lo, hi)
  int page = -1;
  if (live && j < p.pt_pages) page = uniform_load(p.page_table + (int64_t)c * p.pt_stride + j);
  if (live && (page < 0 || page >= p.n_pool_pages)) {
    if (lane == 0 && p.status != nullptr)
      atomicOr(p.status, j < p.pt_pages ? KAMERA_STATUS_BAD_PAGE : KAMERA_STATUS_BAD_LENGTH);
    live = false;
  }
  if (SUB == 1 && !live) return;
  // with several waves a unit, all of the workgroup's waves go on to the barriers
  if (!live) page = 0;

  const AppendPlane& pp = p.plane[pl];
  const int t_lane = sub * 16 + lane / LPR, col = (lane % LPR) * 8;
  const int64_t row0 = p0 - before + base;         // row of the page's token 0
  const uint16_t* rows = pp.rows + c * pp.rows_s[0] + l * pp.rows_s[1] + h * pp.rows_s[3] + col;
  u32x4 x[IT];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    const int t = i * TPI + t_lane;
    x[i] = u32x4{0u, 0u, 0u, 0u};
    if (live && t >= lo && t < hi) x[i] = ld16(rows + (row0 + t) * pp.rows_s[2]);
  }
#pragma unroll
  for (int i = 0; i < IT; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) top = max_u16x2(top, u4_get(x[i], k) & 0x7fff7fffu);
  uint32_t amax = max(top & 0xffffu, top >> 16);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, d));
  if (amax >= 0x7f80u) {                           // infinities or NaN: the largest of the rest
    amax = 0;
#pragma unroll
    for (int i = 0; i < IT; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t w = u4_get(x[i], k), a = w & 0x7fffu, b = (w >> 16) & 0x7fffu;
        amax = max(amax, a < 0x7f80u ? a : 0u);
        amax = max(amax, b < 0x7f80u ? b : 0u);
      }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, d));
  }
  if (SUB > 1) {
    if (lane == 0) s_top[wave] = amax;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < SUB; ++k) amax = max(amax, s_top[wave0 + k]);
  }
  int e = clamp_exp((int)(amax >> 7) - 127 - 8 + ((amax & 0x7fu) > 0x60u ? 1 : 0));

  float* scale = pp.scale + l * pp.scale_s[0] + page * pp.scale_s[1] + h * pp.scale_s[2];
  uint8_t* cache = pp.cache + l * pp.cache_s[0] + page * pp.cache_s[1] + h * pp.cache_s[3] + col;
  const bool sums = live && pl == 0 && p.k_sum != nullptr && hi == P;
  u32x2 old[IT];
#pragma unroll
  for (int i = 0; i < IT; ++i) old[i] = u32x2{0u, 0u};
  int e_old = kMinExp;
  if (live && lo > 0) e_old = clamp_exp((int)((__float_as_uint(*scale) >> 23) & 0xffu) - 127);
  if (SUB > 1) __syncthreads();                    // every wave of the unit has the old scale
  if (live && lo > 0) {                            // tokens [0, lo) are there already
    const bool lift = e > e_old;
    if (lift || sums) {
#pragma unroll
      for (int i = 0; i < IT; ++i) {
        const int t = i * TPI + t_lane;
        if (t < lo) old[i] = *reinterpret_cast<const u32x2*>(cache + t * pp.cache_s[2]);
      }
    }
    if (lift) {
      // to the new exponent: exact but where a byte leaves the normal range.
      // A step of over 126 leaves nothing of any byte.
      const float by = e - e_old > 126 ? 0.0f : pow2(e_old - e);
#pragma unroll
      for (int i = 0; i < IT; ++i) {
        const int t = i * TPI + t_lane;
        float f[8];
        from_e4m3(old[i], f);
        u32x2 r = {0u, 0u};
        r.x = __builtin_amdgcn_cvt_pk_fp8_f32(f[0] * by, f[1] * by, r.x, false);
        r.x = __builtin_amdgcn_cvt_pk_fp8_f32(f[2] * by, f[3] * by, r.x, true);
        r.y = __builtin_amdgcn_cvt_pk_fp8_f32(f[4] * by, f[5] * by, r.y, false);
        r.y = __builtin_amdgcn_cvt_pk_fp8_f32(f[6] * by, f[7] * by, r.y, true);
        old[i] = r;
        if (t < lo) *reinterpret_cast<u32x2*>(cache + t * pp.cache_s[2]) = r;
      }
    } else {
      e = e_old;
    }
  }
  const float inv = pow2(-e);
  if (live && lane == 0 && sub == 0) *scale = pow2(e);
  float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    const int t = i * TPI + t_lane;
    const u32x2 r = to_e4m3(x[i], inv);
    if (live && t >= lo && t < hi) *reinterpret_cast<u32x2*>(cache + t * pp.cache_s[2]) = r;
    if (sums) {
      float f[8];
      from_e4m3(t < lo ? old[i] : r, f);
#pragma unroll
      for (int k = 0; k < 8; ++k) sum[k] += f[k] == f[k] ? f[k] : 0.0f;
    }
  }
  if (SUB == 1 && !sums) return;
  // Multiples of 2^-9 below 64 * 448 < 2^15: every partial sum is exact in 24
  // bits, so the order does not matter.
#pragma unroll
  for (int k = 0; k < 8; ++k)
#pragma unroll
    for (int d = LPR; d < 64; d <<= 1) sum[k] += __shfl_xor(sum[k], d);
  if (SUB > 1) {
    if (lane < LPR)
#pragma unroll
      for (int k = 0; k < 8; ++k) s_sum[wave][col + k] = sum[k];
    __syncthreads();
    if (!sums || sub != 0) return;
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int w = 1; w < SUB; ++w) sum[k] += s_sum[wave + w][col + k];
  }
  float big = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) big = fmaxf(big, fabsf(sum[k]));
#pragma unroll
  for (int d = 1; d < LPR; d <<= 1) big = fmaxf(big, __shfl_xor(big, d));
  // 127 = (1 + 0x7e0000 / 2^23) * 2^6
  const uint32_t bits = __float_as_uint(big);
  const int f = clamp_exp(big > 0.f ? (int)(bits >> 23) - 127 - 6 + ((bits & 0x7fffffu) > 0x7e0000u ? 1 : 0) : kMinExp);
  const float down = pow2(-f);
  if (lane < LPR) {
    u32x2 w = {0u, 0u};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t b = (uint32_t)(int)rintf(sum[k] * down) & 0xffu;
      if (k < 4) w.x |= b << (8 * k); else w.y |= b << (8 * (k - 4));
    }
    *reinterpret_cast<u32x2*>(p.k_sum + l * p.k_sum_s[0] + page * p.k_sum_s[1] + h * p.k_sum_s[2] + col) = w;
    if (lane == 0)
      p.k_sum_scale[l * p.k_sum_scale_s[0] + page * p.k_sum_scale_s[1] + h * p.k_sum_scale_s[2]] =
          ldexpf(1.0f, e + f);
  }
}

hipError_t launch_append(const AppendParams& p, hipStream_t s) {
  const int per = append_units_wg(p.page_size);
  const dim3 grid((uint32_t)((p.n_units + per - 1) / per)), block(kAppendThreads);
#define KAMERA_APPEND(D, SUB) hipLaunchKernelGGL((append_kernel<D, SUB>), grid, block, 0, s, p)
  if (p.head_dim == 128) {
    switch (p.page_size) {
      case 16: KAMERA_APPEND(128, 1); break;
      case 32: KAMERA_APPEND(128, 2); break;
      default: KAMERA_APPEND(128, 4); break;
    }
  } else {
    switch (p.page_size) {
      case 16: KAMERA_APPEND(64, 1); break;
      case 32: KAMERA_APPEND(64, 2); break;
      default: KAMERA_APPEND(64, 4); break;
    }
  }
#undef KAMERA_APPEND
  return hipGetLastError();
}

}  // namespace kamera

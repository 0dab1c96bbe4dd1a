// What the host layers of the C ABI share: the per-thread error text, and
// extent arithmetic that cannot overflow.
#pragma once

#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include <initializer_list>

#include "kamera.h"
#include "kamera_launch.h"

namespace kamera {
namespace host {

inline thread_local char g_err[512] = "";

inline int fail(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return code;
}

inline int ok() {
  g_err[0] = '\0';
  return KAMERA_OK;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Largest work a call may describe (elements, rows or tasks): far beyond any
// device, and small enough that the host arithmetic on it cannot overflow.
constexpr int64_t kMaxWork = (int64_t)1 << 50;

// product of non-negative factors, or -1 once it exceeds kMaxWork
inline int64_t bounded_product(std::initializer_list<int64_t> factors) {
  __int128 p = 1;
  for (const int64_t f : factors) {
    if (f < 0) return -1;
    p *= f;
    if (p > kMaxWork) return -1;
  }
  return (int64_t)p;
}

// byte range [lo, hi) of an n-D strided view (element strides, elem_bytes
// each) whose innermost rows are row_elems contiguous elements; false when
// the range does not fit in the address space (the arithmetic is 128-bit)
inline bool span(const void* base, const int64_t* s, const int64_t* ext, int nd, int64_t row_elems, int elem_bytes,
                 uintptr_t& lo, uintptr_t& hi) {
  __int128 a = 0, b = 0;
  for (int k = 0; k < nd; ++k) {
    if (ext[k] <= 0) continue;
    const __int128 d = (__int128)(ext[k] - 1) * s[k];
    if (d < 0) a += d; else b += d;
  }
  const __int128 p = (__int128)reinterpret_cast<uintptr_t>(base);
  const __int128 l = p + a * elem_bytes, h = p + (b + row_elems) * elem_bytes;
  if (l < 0 || h > (__int128)UINTPTR_MAX) return false;
  lo = (uintptr_t)l;
  hi = (uintptr_t)h;
  return true;
}

inline bool overlap(uintptr_t a0, uintptr_t a1, uintptr_t b0, uintptr_t b1) { return a0 < b1 && b0 < a1; }

struct Range {
  uintptr_t lo, hi;
};

// Byte range of n elements from p.
inline Range flat(const void* p, int64_t n, int bytes) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  return {a, a + (uintptr_t)n * bytes};
}

// The same of an optional array.
inline Range flat_or(const void* p, int64_t n, int bytes) { return flat(p, p != nullptr ? n : 0, bytes); }

inline bool meet(const Range& a, const Range& b) { return a.lo < a.hi && b.lo < b.hi && overlap(a.lo, a.hi, b.lo, b.hi); }

inline bool multiples(const int64_t* s, int n, int64_t of) {
  for (int k = 0; k < n; ++k)
    if (s[k] % of != 0) return false;
  return true;
}

// `pages`: the entries of a row.
inline int check_table(const int32_t* table, int32_t pt_stride, int32_t pages, int32_t page_size, int32_t n_pool_pages,
                int64_t tokens, const char* who) {
  if (table == nullptr) return fail(KAMERA_ERR_NULL, "%s: page_table is NULL", who);
  if (n_pool_pages <= 0) return fail(KAMERA_ERR_SHAPE, "%s: n_pool_pages must be positive", who);
  if (pt_stride < 0 || pages < ceil_div(tokens, page_size))
    return fail(KAMERA_ERR_SHAPE, "%s: %d pages a row (stride %d) < %lld pages needed for %lld tokens", who, pages,
                pt_stride, (long long)ceil_div(tokens, page_size), (long long)tokens);
  return KAMERA_OK;
}

// Entries that a row of a page table has.
inline int32_t row_pages(int32_t pt_stride, int32_t pt_pages) { return pt_pages != 0 ? pt_pages : pt_stride; }

// Bytes of a table of n rows.
inline Range table_range(const int32_t* table, int64_t n, int32_t pt_stride, int32_t pages) {
  return flat(table, n > 0 && pages > 0 ? (n - 1) * pt_stride + pages : 0, 4);
}

inline int check_workspace(const void* workspace, int64_t bytes, int64_t needed, const char* who) {
  if (workspace == nullptr) return fail(KAMERA_ERR_NULL, "%s: workspace is NULL", who);
  if (bytes < needed)
    return fail(KAMERA_ERR_SHAPE, "%s: workspace of %lld bytes, %lld needed", who, (long long)bytes, (long long)needed);
  if (!aligned16(workspace)) return fail(KAMERA_ERR_ALIGN, "%s: workspace must be 16-byte aligned", who);
  return KAMERA_OK;
}

}  // namespace host
}  // namespace kamera

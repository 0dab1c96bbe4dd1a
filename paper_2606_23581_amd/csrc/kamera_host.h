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

}  // namespace host
}  // namespace kamera

// The rotary descriptor on the host: its checks, and the frequencies that the
// kernels take.
#pragma once

#include <math.h>
#include <string.h>

#include "kamera.h"
#include "kamera_host.h"
#include "kamera_launch.h"

namespace kamera {
namespace host {

constexpr double kTwoPi = 6.283185307179586476925286766559;

// ---------------------------------------------------------------------------
// RoPE descriptor
// ---------------------------------------------------------------------------

inline int check_rope(const kamera_rope& r, int32_t head_dim, const char* who) {
  if (!(r.theta > 0.0) || !isfinite(r.theta))
    return fail(KAMERA_ERR_SHAPE, "%s: rope.theta must be a finite positive number (got %g)", who, r.theta);
  if (r.rope_dim <= 0 || (r.rope_dim & 1))
    return fail(KAMERA_ERR_SHAPE, "%s: rope.rope_dim must be positive and even (got %d)", who, r.rope_dim);
  if (r.rope_dim > KAMERA_MAX_ROPE_DIM)
    return fail(KAMERA_ERR_RANGE, "%s: rope.rope_dim %d exceeds %d", who, r.rope_dim, KAMERA_MAX_ROPE_DIM);
  if (r.rope_offset < 0 || (int64_t)r.rope_offset + r.rope_dim > head_dim)
    return fail(KAMERA_ERR_SHAPE, "%s: rope band [%d, %lld) lies outside the %d-column row", who,
                r.rope_offset, (long long)r.rope_offset + r.rope_dim, head_dim);
  if (r.pairing != KAMERA_PAIR_NEOX && r.pairing != KAMERA_PAIR_INTERLEAVED)
    return fail(KAMERA_ERR_SHAPE, "%s: unknown rope.pairing %d", who, r.pairing);
  if (r.n_sections != 1 && r.n_sections != 3)
    return fail(KAMERA_ERR_SHAPE, "%s: rope.n_sections must be 1 or 3 (got %d)", who, r.n_sections);
  if (r.n_sections == 3) {
    if (r.sections[0] < 0 || r.sections[1] < 0 || r.sections[2] < 0 ||
        r.sections[0] + r.sections[1] + r.sections[2] != r.rope_dim / 2)
      return fail(KAMERA_ERR_SHAPE, "%s: sections %d/%d/%d must be >= 0 and sum to rope_dim/2 = %d", who,
                  r.sections[0], r.sections[1], r.sections[2], r.rope_dim / 2);
    if (r.section_order != KAMERA_SECTIONS_BLOCKED && r.section_order != KAMERA_SECTIONS_INTERLEAVED)
      return fail(KAMERA_ERR_SHAPE, "%s: unknown rope.section_order %d", who, r.section_order);
  }
  return KAMERA_OK;
}

// Frequencies in revolutions per position step, and the (t, h, w) coordinate
// of each pair.
inline void fill_rope(const kamera_rope& r, kamera::RopeParams& o) {
  memset(&o, 0, sizeof(o));
  const int half = r.rope_dim / 2;
  for (int j = 0; j < half; ++j) o.rev_freq[j] = pow(r.theta, -2.0 * j / (double)r.rope_dim) / kTwoPi;
  if (r.n_sections == 3) {
    if (r.section_order == KAMERA_SECTIONS_BLOCKED) {
      for (int j = 0; j < half; ++j)
        o.coord[j] = (int8_t)(j < r.sections[0] ? 0 : (j < r.sections[0] + r.sections[1] ? 1 : 2));
    } else {
      int left[3] = {r.sections[0], r.sections[1], r.sections[2]};
      int j = 0;
      while (j < half) {
        for (int s = 0; s < 3 && j < half; ++s)
          if (left[s] > 0) {
            o.coord[j++] = (int8_t)s;
            --left[s];
          }
      }
    }
  }
  o.rope_offset = r.rope_offset;
  o.rope_dim = r.rope_dim;
  o.pairing = r.pairing;
}

}  // namespace host
}  // namespace kamera

// 8-bit integers with a scale per row: q = round(x * (127 / max)), scale = max / 127, max the row's largest
// magnitude.  Symmetric, -127 .. 127, so that a product needs no correction for a zero point.
#pragma once

#include "fd_scaled.h"

namespace fd {

// Rows below this largest magnitude are zeros: 127 / max stays finite and max / 127 a normal number.
constexpr float kLeastTop = 0x1p-100f;

struct IntScale { float scale, up; };
// `top`: the bits of the row's largest magnitude.  Rows with an infinity or a NaN: scale NaN and codes 0.
// Divisions are correctly rounded, so that a scale and its codes depend on the row alone.
FD_DEVICE IntScale int_scale(uint32_t top) {
  if (top >= 0x7f800000u) return {__uint_as_float(0x7fc00000u), 0.f};
  const float t = __uint_as_float(top);
  if (t < kLeastTop) return {0.f, 0.f};
  return {t / 127.f, 127.f / t};
}
// Eight values to eight integers, nearest, ties to even; up = 0: zeros, whatever the values.
FD_DEVICE uint2 pack_ints(const float (&v)[8], float up) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int q[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) q[e] = up == 0.f ? 0 : static_cast<int>(rintf(v[4 * i + e] * up));
    w[i] = (q[0] & 255) | (q[1] & 255) << 8 | (q[2] & 255) << 16 | static_cast<uint32_t>(q[3]) << 24;
  }
  return make_uint2(w[0], w[1]);
}

}  // namespace fd

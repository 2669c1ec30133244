// Correctly rounded quotients in few operations, for the rows of a quantised cache.
#pragma once

#include <math.h>

#include "host_device.hpp"

namespace fqi {

// a / b correctly rounded from r = 1 / b correctly rounded: y = a r is next to it, a - y b
// is exact, and one more step of it gives the rounded quotient (Markstein), far from the
// ends of the range.  (The host tests check it for b = 255 and 15 over all fp32 significands,
// and for all pairs of bf16 ones.)
FQ_HOST_DEVICE float quotient(float a, float b, float r) {
  const float y = a * r;
  return fmaf(fmaf(-y, b, a), r, y);
}

// 1 / s correctly rounded from r0, within two of its last places: one step of it, for every s
// of 8 bits (checked over all of them and all such r0).
FQ_HOST_DEVICE float inverse(float s, float r0) { return fmaf(fmaf(-s, r0, 1.f), r0, r0); }

}  // namespace fqi

// Which ids min_p keeps (internal): shared by the verification of drafts and the sampler with per-row limits, so that both
// keep the same ones.
#pragma once
#include "common.hpp"

namespace rgd {

// The lowest kept logit of a row of maximum `top`: the smallest float z with
// (double)z - top >= low, so that one fp32 comparison decides as fp64 does.
RGD_DEV float threshold(float top, double low) {
  float f = (float)((double)top + low);
  for (int i = 0; i < 4 && (double)f - (double)top < low; ++i) f = nextafterf(f, INFINITY);
  for (int i = 0; i < 4; ++i) {
    const float g = nextafterf(f, -INFINITY);
    if (!((double)g - (double)top >= low)) break;
    f = g;
  }
  return f;
}

RGD_DEV bool finite_top(float t) { return t > -INFINITY && t < INFINITY; }

}  // namespace rgd

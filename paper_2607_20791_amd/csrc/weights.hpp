// Weights of a truncated softmax in 64 bits (internal): shared by the verification of drafts and the sampler with
// per-row limits, so that both keep the same ids.
#pragma once
#include "common.hpp"

namespace rgd {

// 2^x to 1e-14 for x <= 0: the Taylor series of 2^f, |f| <= 1/2, to f^11.
RGD_DEV double exp2_f64(double x) {
  x = fmax(x, -1100.0);  // below: 0 either way (and -inf - rint(-inf) is not a number)
  const double n = rint(x), g = (x - n) * 0.6931471805599453;
  double s = 1.0 / 39916800.0;
  s = fma(s, g, 1.0 / 3628800.0);
  s = fma(s, g, 1.0 / 362880.0);
  s = fma(s, g, 1.0 / 40320.0);
  s = fma(s, g, 1.0 / 5040.0);
  s = fma(s, g, 1.0 / 720.0);
  s = fma(s, g, 1.0 / 120.0);
  s = fma(s, g, 1.0 / 24.0);
  s = fma(s, g, 1.0 / 6.0);
  s = fma(s, g, 0.5);
  s = fma(s, g, 1.0);
  s = fma(s, g, 1.0);
  return ldexp(s, (int)n);
}

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

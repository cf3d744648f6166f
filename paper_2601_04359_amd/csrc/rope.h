// The angles of the 3D rotary embedding: frequencies of every pair of dims (host) and their sines (device).
#pragma once

#include <math.h>

#include "common.h"

namespace pc {

constexpr int kMaxPairs = 128;    // D <= 256

struct RopeFreq {
  double inv_freq[kMaxPairs];  // base^(-2i/s) of every pair, section by section
  uint8_t axis[kMaxPairs];     // which coordinate (0 = t, 1 = h, 2 = w) turns the pair
};

// The frequencies of the last (sections, base) this host thread asked for: a model uses one set, and
// its pow() calls are a quarter of the host time of a small call.
inline const RopeFreq& rope_freq(const int (&secs)[3], double base) {
  thread_local RopeFreq fr;
  thread_local int of_secs[3] = {-1, -1, -1};
  thread_local double of_base = 0.0;
  if (secs[0] == of_secs[0] && secs[1] == of_secs[1] && secs[2] == of_secs[2] && base == of_base) return fr;
  int p = 0;
  for (int a = 0; a < 3; ++a)
    for (int i = 0; i < secs[a] / 2; ++i, ++p) {
      fr.inv_freq[p] = pow(base, -2.0 * i / secs[a]);
      fr.axis[p] = static_cast<uint8_t>(a);
    }
  for (; p < kMaxPairs; ++p) {
    fr.inv_freq[p] = 0.0;
    fr.axis[p] = 0;
  }
  for (int a = 0; a < 3; ++a) of_secs[a] = secs[a];
  of_base = base;
  return fr;
}

// sin and cos of x in fp64: Cody-Waite reduction to |r| <= pi/4 (pi/2 in two parts; k has at most 32
// bits here, so x - k pi/2 is good to the last bit of r), then the Taylor series (remainders below
// 1e-13 of the result, which is rounded to fp32).  A quarter of the instructions of the general
// function, which carries a reduction for any x; beyond 2^32 that one is called.
__device__ __forceinline__ void sincos_f64(double x, double* sn, double* cs) {
  if (fabs(x) > 4294967296.0) {
    sincos(x, sn, cs);
    return;
  }
  const double k = rint(x * 0.63661977236758134308);
  double r = fma(-k, 1.57079632679489661923, x);
  r = fma(-k, 6.12323399573676603587e-17, r);
  const double q = r * r;
  double s = fma(q, 1.0 / 6227020800.0, -1.0 / 39916800.0);
  s = fma(q, s, 1.0 / 362880.0);
  s = fma(q, s, -1.0 / 5040.0);
  s = fma(q, s, 1.0 / 120.0);
  s = fma(q, s, -1.0 / 6.0);
  s = fma(q * r, s, r);
  double c = fma(q, -1.0 / 87178291200.0, 1.0 / 479001600.0);
  c = fma(q, c, -1.0 / 3628800.0);
  c = fma(q, c, 1.0 / 40320.0);
  c = fma(q, c, -1.0 / 720.0);
  c = fma(q, c, 1.0 / 24.0);
  c = fma(q, c, -0.5);
  c = fma(q, c, 1.0);
  const int quadrant = static_cast<int>(k - 4.0 * floor(k * 0.25));   // 0..3 (NaN: anything)
  const double a = (quadrant & 1) ? c : s, b = (quadrant & 1) ? s : c;
  *sn = (quadrant & 2) ? -a : a;
  *cs = (quadrant == 1 || quadrant == 2) ? -b : b;
}

// Sixteen bytes of a row turned by their pairs' (cos, sin), one rounding per element.
template <typename T>
__device__ __forceinline__ void turn_16B(u32x4& raw, const float2* cs) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 r = cs[k];
      const float a0 = bf16_to_f32(static_cast<uint16_t>(raw[k] & 0xFFFFu));
      const float a1 = bf16_to_f32(static_cast<uint16_t>(raw[k] >> 16));
      raw[k] = pack_bf16x2(fmaf(a0, r.x, -(a1 * r.y)), fmaf(a1, r.x, a0 * r.y));
    }
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float2 r = cs[k];
      const float a0 = __uint_as_float(raw[2 * k]), a1 = __uint_as_float(raw[2 * k + 1]);
      raw[2 * k] = __float_as_uint(fmaf(a0, r.x, -(a1 * r.y)));
      raw[2 * k + 1] = __float_as_uint(fmaf(a1, r.x, a0 * r.y));
    }
  }
}

}  // namespace pc

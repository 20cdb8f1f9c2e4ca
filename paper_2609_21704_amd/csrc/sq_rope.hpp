// Rotary position embedding (gfx950 device code).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

namespace sq {

// The rotation shared by the kernels that write a cache and the attention that rotates its own query rows and new
// entries (the same bits): pair (t, t + 64) of a head
// turns by pos * theta^(-2t/128), the angle and its cosine and sine in fp64,
// the turn itself in fp32 with every product rounded on its own.
// Both functions are short series here: the library's pow and sincos, with their
// branches for every argument, are code that a launch fetches to run once
// (with the items' shorter code a rotating attention of 4 x 9 rows over 64
// positions took 12.1 us, 14.1 before; the attention alone 8.0).
struct RopeBase {  // ln theta = hi + lo
  double hi, lo;
};

// theta^(-2t/128) = exp(-(t / 64) ln theta), the exponent in two parts, the exponential by its Taylor series to
// degree 13 on |r| <= ln 2 / 2 (next term 4e-18).
__device__ __forceinline__ double rope_freq(int t, RopeBase base) {
  const double s = (double)t * (-1.0 / 64.0);
  const double x = s * base.hi, xl = __builtin_fma(s, base.hi, -x) + s * base.lo;
  const double n = rint(x * 0x1.71547652b82fep+0);
  double r = __builtin_fma(n, -0x1.62e42fefa39efp-1, x);
  r = __builtin_fma(n, -0x1.abc9e3b39803fp-56, r) + xl;
  double p = 1.0 / 6227020800.0;
  const double c[] = {1.0 / 479001600.0, 1.0 / 39916800.0, 1.0 / 3628800.0, 1.0 / 362880.0, 1.0 / 40320.0,
                      1.0 / 5040.0,      1.0 / 720.0,      1.0 / 120.0,     1.0 / 24.0,     1.0 / 6.0,
                      0.5,               1.0,              1.0};
#pragma unroll
  for (int i = 0; i < 13; ++i) p = __builtin_fma(p, r, c[i]);
  return ldexp(p, (int)n);
}

// Cosine and sine of pos * freq: the angle less n pi / 2 by fused steps with pi / 2 in three parts (the first is
// exact below 2^31), what the second rounds off carried along, and the Taylor series to degrees 16 and 17 on
// |r| <= pi / 4 (next terms below 5e-17); 2.3e-16 of the values at most over angles up to 1e6.
__device__ __forceinline__ float2 rope_cos_sin(int64_t pos, double freq) {
  const double x = (double)pos * freq;
  const double n = rint(x * 0x1.45f306dc9c883p-1);
  const double r1 = __builtin_fma(-n, 0x1.921fb54442d18p+0, x);
  const double r = __builtin_fma(-n, 0x1.1a62633145c07p-54, r1);
  const double tail = __builtin_fma(-n, -0x1.f1976b7ed8fbcp-110, __builtin_fma(-n, 0x1.1a62633145c07p-54, r1 - r));
  const double z = r * r;
  double ps = 1.0 / 355687428096000.0, pc = 1.0 / 20922789888000.0;
  const double cs[] = {-1.0 / 1307674368000.0, 1.0 / 6227020800.0, -1.0 / 39916800.0, 1.0 / 362880.0,
                       -1.0 / 5040.0,          1.0 / 120.0,        -1.0 / 6.0};
  const double cc[] = {-1.0 / 87178291200.0, 1.0 / 479001600.0, -1.0 / 3628800.0, 1.0 / 40320.0, -1.0 / 720.0,
                       1.0 / 24.0};
#pragma unroll
  for (int i = 0; i < 7; ++i) ps = __builtin_fma(ps, z, cs[i]);
#pragma unroll
  for (int i = 0; i < 6; ++i) pc = __builtin_fma(pc, z, cc[i]);
  const double sn = r + __builtin_fma(r * z, ps, tail);
  const double co = __builtin_fma(-0.5, z, 1.0) + __builtin_fma(z * z, pc, -r * tail);
  const int q = (int)(int64_t)n & 3;
  const double a = q & 1 ? sn : co, b = q & 1 ? co : sn;  // |cosine|, |sine| of the angle
  return make_float2((float)((q + 1) & 2 ? -a : a), (float)(q & 2 ? -b : b));
}

__device__ __forceinline__ void rope_turn(float a, float e, float2 cs, float& ra, float& re) {
#pragma clang fp contract(off)
  ra = a * cs.x - e * cs.y;
  re = e * cs.x + a * cs.y;
}

inline RopeBase rope_base(double theta) {
  const long double ln = std::log((long double)theta);
  const double hi = (double)ln;
  return {hi, (double)(ln - (long double)hi)};
}

}  // namespace sq

// Arithmetic shared by the quantizers (gfx950 device code).
#pragma once

#include "sq_device.hpp"

namespace sq {

// Division by a reciprocal estimate, one Newton step on it and one correction
// of the quotient by its exact fused remainder: Markstein, Computation of
// elementary functions on the IBM RISC System/6000 processor, 1990.
//
// 1 / s correctly rounded or within one ulp of it, for s > 0 whose reciprocal
// is a normal float.
__device__ __forceinline__ float recip(float s) {
#pragma clang fp contract(off)
  const float r = __builtin_amdgcn_rcpf(s);
  return __builtin_fmaf(__builtin_fmaf(-s, r, 1.0f), r, r);
}

// v / s to within half an ulp (+ 2^-20 of one): the exact remainder of the
// first estimate corrects it.  A quotient with few bits comes out exactly.
__device__ __forceinline__ float quotient(float v, float s, float rs) {
#pragma clang fp contract(off)
  const float q0 = v * rs;
  return __builtin_fmaf(__builtin_fmaf(-q0, s, v), rs, q0);
}

// Smallest binary16 value >= s for a finite s > 0 that is a normal double.
// The binary16 grid near s has spacing 2^(e-10) (e = floor(log2 s) >= -14) or
// 2^-24 (subnormal range); scaling by that spacing is exact, so ceil() picks
// the next grid point exactly.
__device__ __forceinline__ double f16_ceil(double s) {
#pragma clang fp contract(off)
  const uint64_t bits = (uint64_t)__double_as_longlong(s);
  const int e = (int)((bits >> 52) & 0x7FF) - 1023;
  const int sp = (e < -14) ? -24 : e - 10;
  return ldexp(ceil(ldexp(s, -sp)), sp);
}

}  // namespace sq

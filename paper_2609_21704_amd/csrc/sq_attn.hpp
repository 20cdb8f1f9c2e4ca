// Device-side pieces shared by the attention and cache kernels (gfx950).
#pragma once

#include "sq_device.hpp"

namespace sq {

constexpr int kHd = 128;  // head dimension of the family

typedef _Float16 half4_t __attribute__((ext_vector_type(4)));

constexpr uint16_t kNanF16 = 0x7E00;

__device__ __forceinline__ void flag(int32_t* status, int32_t bit) {
  if (status) atomicOr(status, bit);
}

// v_exp_f32 alone: exp2f's extra steps only serve results below 2^-126.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// max / sum over the four lanes li + 16 (0..3) that share a query row
template <class OP>
__device__ __forceinline__ float quad_fold(float v, OP op) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  const auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t p0 = p[0], p1 = p[1];
  const uint32_t w = __builtin_bit_cast(uint32_t, op(__builtin_bit_cast(float, p0), __builtin_bit_cast(float, p1)));
  const auto r = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  const uint32_t r0 = r[0], r1 = r[1];
  return op(__builtin_bit_cast(float, r0), __builtin_bit_cast(float, r1));
}
__device__ __forceinline__ float quad_max(float v) {
  return quad_fold(v, [](float x, float y) { return fmaxf(x, y); });
}
__device__ __forceinline__ float quad_sum(float v) {
  return quad_fold(v, [](float x, float y) { return x + y; });
}

}  // namespace sq

// Softmax arithmetic in fp64 and the exact integer sums over its weights, shared by the acceptance and the sampling
// kernels (gfx950 device code).
#pragma once

#include <math.h>

#include "sq_device.hpp"

#pragma clang fp contract(off)

namespace sq {
namespace {

__device__ __forceinline__ double quotient(double a, double b, double rb) {
  const double q = a * rb;
  return __builtin_fma(__builtin_fma(-q, b, a), rb, q);
}

// What the softmax arithmetic of a thread holds in registers.  These kernels
// are bound by fp64 instructions (one per four cycles) where there are many
// rows, so the two expensive operations have forms of their own:
//   z = l / T and p = exp / S: an estimate by the reciprocal plus one
//     exact-remainder correction (Markstein 1990, on the IBM RISC System/6000),
//     the correctly rounded quotient for three operations instead of a dozen; kOne: T == 1, z = l;
//   exp of x <= 0: n = rint(x / ln 2) (Cody and Waite's two-part reduction),
//     then the minimax polynomial of degree 11 on |r| <= ln(2) / 2 (Remez
//     exchange, relative error 3.1e-18, below the rounding of its evaluation)
//     and the scaling by 2^n: 17 operations, without the library's range
//     selections.  Below -1100 (a masked logit's -inf too) it gives 0.
// The coefficients sit in vector registers, so that every step is one
// three-operand fma (72 rows of 151936 logits, statistics: 21.6 -> 13.3 us).
template <bool kOne>
struct Soft {
  static constexpr bool one = kOne;
  double t, rt;
  double c[10], l2e, magic, hi, lo;

  __device__ __forceinline__ explicit Soft(float temp)
      : t((double)temp), rt(kOne ? 1.0 : 1.0 / (double)temp),
        c{0x1.ad66168f6ec16p-26, 0x1.28b31c3ff65e9p-22, 0x1.71df45378dcabp-19, 0x1.a01992c5bfed9p-16,
          0x1.a01a0110431a9p-13, 0x1.6c16c187853cdp-10, 0x1.1111111130e38p-7, 0x1.555555554f35cp-5,
          0x1.55555555554a2p-3, 0x1.0000000000010p-1},
        l2e(0x1.71547652b82fep+0), magic(0x1.8p52), hi(-0x1.62e42fefa2000p-1), lo(-0x1.9ef35793c7673p-41) {
#pragma unroll
    for (int i = 0; i < 10; ++i) asm("" : "+v"(c[i]));
    asm("" : "+v"(l2e), "+v"(magic), "+v"(hi), "+v"(lo));
  }

  __device__ __forceinline__ double exp(double x) const {
    x = fmax(x, -1100.0);
    const double k = __builtin_fma(x, l2e, magic);  // rint(x / ln 2) in the low mantissa bits
    const double n = k - magic;
    const double r = __builtin_fma(n, lo, __builtin_fma(n, hi, x));
    double p = __builtin_fma(c[0], r, c[1]);
#pragma unroll
    for (int i = 2; i < 10; ++i) p = __builtin_fma(p, r, c[i]);
    p = __builtin_fma(p, r, 1.0);
    p = __builtin_fma(p, r, 1.0);
    return ldexp(p, (int)(uint32_t)__builtin_bit_cast(uint64_t, k));
  }

  // A masked logit (-inf) becomes a finite value far below every logit's
  // quotient (a remainder of infinities would be NaN).
  __device__ __forceinline__ double z(float l) const {
    if constexpr (kOne) return (double)l;
    return quotient(fmax((double)l, -1e250), t, rt);
  }
};

// ---- wavefront reductions and scans on DPP moves (a permute through LDS costs several times the latency)
template <int Ctrl, int RowMask = 0xF>
__device__ __forceinline__ uint32_t dpp32(uint32_t v) {  // lanes without a source, or outside RowMask: 0
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, Ctrl, RowMask, 0xF, false);
}

template <int Ctrl, int RowMask = 0xF, class T>
__device__ __forceinline__ T dpp_move(T v) {
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(T, dpp32<Ctrl, RowMask>(__builtin_bit_cast(uint32_t, v)));
  } else {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = dpp32<Ctrl, RowMask>((uint32_t)u), hi = dpp32<Ctrl, RowMask>((uint32_t)(u >> 32));
    return __builtin_bit_cast(T, (uint64_t)hi << 32 | lo);
  }
}

// op over the 64 lanes, a fixed tree; every lane receives the result.
template <class T, class Op>
__device__ __forceinline__ T wave_all(T v, Op op) {
  v = op(v, dpp_move<0xB1>(v));   // quad_perm [1,0,3,2]
  v = op(v, dpp_move<0x4E>(v));   // quad_perm [2,3,0,1]
  v = op(v, dpp_move<0x141>(v));  // row_half_mirror
  v = op(v, dpp_move<0x140>(v));  // row_mirror: every lane holds its row of 16's result
  constexpr int N = sizeof(T) / 4;
  struct W {
    uint32_t w[N];
  };
  W x = __builtin_bit_cast(W, v), y;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const auto p = __builtin_amdgcn_permlane16_swap(x.w[i], x.w[i], false, false);
    const uint32_t p0 = p[0], p1 = p[1];  // scalar copies: vector element lvalues are misread
    x.w[i] = p0;
    y.w[i] = p1;
  }
  v = op(__builtin_bit_cast(T, x), __builtin_bit_cast(T, y));
  x = __builtin_bit_cast(W, v);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const auto p = __builtin_amdgcn_permlane32_swap(x.w[i], x.w[i], false, false);
    const uint32_t p0 = p[0], p1 = p[1];
    x.w[i] = p0;
    y.w[i] = p1;
  }
  return op(__builtin_bit_cast(T, x), __builtin_bit_cast(T, y));
}

__device__ __forceinline__ float wave_max_f32(float v) {
  return wave_all(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ double wave_max_f64(double v) {
  return wave_all(v, [](double a, double b) { return fmax(a, b); });
}
__device__ __forceinline__ double wave_sum_f64(double v) {
  return wave_all(v, [](double a, double b) { return a + b; });
}
__device__ __forceinline__ int64_t wave_sum_i64(int64_t v) {
  return wave_all(v, [](int64_t a, int64_t b) { return a + b; });
}

// Inclusive prefix sum over the 64 lanes.
__device__ __forceinline__ int64_t wave_scan_i64(int64_t v) {
  v += dpp_move<0x111>(v);       // row_shr:1
  v += dpp_move<0x112>(v);       // row_shr:2
  v += dpp_move<0x114>(v);       // row_shr:4
  v += dpp_move<0x118>(v);       // row_shr:8
  v += dpp_move<0x142, 0xA>(v);  // row_bcast:15 into rows 1 and 3
  v += dpp_move<0x143, 0xC>(v);  // row_bcast:31 into rows 2 and 3
  return v;
}

// Exclusive prefix sum of v over the workgroup in thread order; `total`
// receives the workgroup's sum.  Integer, so exact.  sh: one cell per wavefront.
template <int kWaves>
__device__ int64_t block_exclusive_scan_i64(int64_t v, int64_t* sh, int64_t& total) {
  const int w = threadIdx.x >> 6;
  const int64_t x = wave_scan_i64(v);
  if ((threadIdx.x & 63) == 63) sh[w] = x;
  __syncthreads();
  int64_t base = 0, t = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    base += i < w ? sh[i] : 0;
    t += sh[i];
  }
  total = t;
  __syncthreads();
  return base + x - v;
}

template <int kWaves>
__device__ int64_t block_sum_i64(int64_t v, int64_t* sh) {
  v = wave_sum_i64(v);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  int64_t t = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) t += sh[i];
  __syncthreads();
  return t;
}

// ---- parts published to a last workgroup
__device__ __forceinline__ void publish(int64_t* p, int64_t v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ int64_t published(const int64_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// One thread's arrival, after its parts are published: true for the last of n
// (every part is visible to it).  The parts are written through to the level
// all XCDs share, so the wait for their stores is all the release needs (a
// release fence would also write back the whole L2, measured at about 2 us),
// and they are read from there.
__device__ __forceinline__ bool arrive(int32_t* counter, int n) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  return n == 1 || __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == n - 1;
}

}  // namespace
}  // namespace sq

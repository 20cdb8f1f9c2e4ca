// C ABI of the sampling calls: host-side argument validation and dispatch.
#include "abi_checks.hpp"
#include "specquant_sample.h"
#include "sq_internal.hpp"

namespace {

sq_status sample(const float* logits, int32_t m, int64_t v, int64_t ld, const float* temperature, const int32_t* top_k,
                 const float* top_p, const float* min_p, const uint32_t* u24, int32_t* token, float* out,
                 int32_t* status, hipStream_t stream) {
  if (m < 1 || m > (1 << 20) || v < 1 || v > (int64_t(1) << 26) || ld < v || ld > kMaxN) return SQ_ERR_SHAPE;
  if (!logits || (!out && (!u24 || !token))) return SQ_ERR_NULL;
  if (!aligned(logits, 4) || !aligned(temperature, 4) || !aligned(top_k, 4) || !aligned(top_p, 4) || !aligned(min_p, 4) ||
      !aligned(u24, 4) || !aligned(token, 4) || !aligned(out, 4) || !aligned(status, 4))
    return SQ_ERR_ALIGN;
  const size_t rows = ((size_t)(m - 1) * (size_t)ld + (size_t)v) * 4, words = (size_t)m * 4;
  const Range outs[] = {{out, rows}, {token, words}, {status, 4}};
  const Range ins[] = {{out == logits ? nullptr : logits, rows}, {temperature, words}, {top_k, words}, {top_p, words},
                       {min_p, words},                           {u24, words}};
  if (any_alias(outs, ins)) return SQ_ERR_ALIAS;
  (void)hipGetLastError();
  return device_status(sq::launch_sample(logits, m, (int)v, ld, temperature, top_k, top_p, min_p, u24, token, out, status,
                                         stream));
}

}  // namespace

extern "C" {

sq_status sq_sample_f32(const float* logits, int32_t m, int64_t v, int64_t ld, const float* temperature,
                        const int32_t* top_k, const float* top_p, const float* min_p, const uint32_t* u24,
                        int32_t* token, int32_t* status, hipStream_t stream) {
  return sample(logits, m, v, ld, temperature, top_k, top_p, min_p, u24, token, nullptr, status, stream);
}

sq_status sq_filter_logits_f32(const float* logits, int32_t m, int64_t v, int64_t ld, const float* temperature,
                               const int32_t* top_k, const float* top_p, const float* min_p, float* out,
                               int32_t* status, hipStream_t stream) {
  if (!out) return SQ_ERR_NULL;
  return sample(logits, m, v, ld, temperature, top_k, top_p, min_p, nullptr, nullptr, out, status, stream);
}

}  // extern "C"

// C ABI of the calls over packed rows and the 4-bit cache: host-side argument validation and dispatch.
#include <math.h>

#include "abi_checks.hpp"
#include "specquant_packed.h"
#include "sq_internal.hpp"

namespace {

struct Call {
  const int32_t* row_start;
  int32_t b;
  int64_t rows, max_rows;
  int32_t hq, hkv;
  const int32_t* pos_base;
  int64_t len_bound, capacity;
};

constexpr int64_t kMaxRows = int64_t(1) << 20;
// The prompt kernel's lanes reach seven rows of values past a scalar base with 32-bit byte offsets.
constexpr int64_t kMaxAttnCapacity = int64_t(1) << 28;

sq_status check_sizes(const Call& c) {
  if (c.max_rows < 1 || c.max_rows > kMaxRows || c.rows < 0 || c.rows > kMaxRows) return SQ_ERR_SHAPE;
  const sq_status bs = check_block(c.b, 1, c.hq, c.hkv, c.len_bound, c.capacity);
  if (bs != SQ_OK) return bs;
  if (!c.row_start && c.rows != c.b * c.max_rows) return SQ_ERR_SHAPE;
  return SQ_OK;
}

// The arrays every call has: row_start, pos_base and the cache.
sq_status check_arrays(const Call& c, const sq::KvCache& kv, bool q4) {
  if (!c.pos_base || (q4 ? !kv.k4 || !kv.ks || !kv.v4 || !kv.vs : !kv.k || !kv.v)) return SQ_ERR_NULL;
  if (!aligned(c.row_start, 4) || !aligned(c.pos_base, 4) || !aligned(kv.k, 16) || !aligned(kv.v, 16) ||
      !aligned(kv.k4, 16) || !aligned(kv.ks, 16) || !aligned(kv.v4, 16) || !aligned(kv.vs, 16))
    return SQ_ERR_ALIGN;
  return SQ_OK;
}

struct CacheRanges {
  Range r[4];
};
CacheRanges cache_ranges(const Call& c, const sq::KvCache& kv, bool q4) {
  const size_t e = (size_t)c.b * c.hkv * c.capacity;
  if (q4) return {{{kv.k4, e * 64}, {kv.ks, e * 8}, {kv.v4, e * 64}, {kv.vs, e * 8}}};
  return {{{kv.k, e * 256}, {kv.v, e * 256}, {nullptr, 0}, {nullptr, 0}}};
}

sq::PackedRows packed(const Call& c) {
  return {c.row_start, c.b, (int)c.rows, (int)(c.max_rows < c.rows ? c.max_rows : c.rows)};
}

sq_status rope_kv(const Call& c, const sq::KvCache& kv, bool q4, const float* qkv, const uint16_t* bias,
                  int32_t pos_offset, double theta, uint16_t* q_out, int32_t* status, hipStream_t stream) {
  sq_status st = check_sizes(c);
  if (st != SQ_OK) return st;
  if (!isfinite(theta)) return SQ_ERR_NONFINITE;
  if (!(theta > 1.0)) return SQ_ERR_SHAPE;
  if (c.rows == 0) return SQ_OK;
  if (!qkv || !q_out) return SQ_ERR_NULL;
  st = check_arrays(c, kv, q4);
  if (st != SQ_OK) return st;
  if (!aligned(qkv, 16) || !aligned(bias, 16) || !aligned(q_out, 16) || !aligned(status, 4)) return SQ_ERR_ALIGN;
  const size_t nh = (size_t)c.hq + 2 * (size_t)c.hkv;
  const CacheRanges cr = cache_ranges(c, kv, q4);
  const Range outs[] = {{q_out, (size_t)c.rows * c.hq * 256}, cr.r[0], cr.r[1], cr.r[2], cr.r[3], {status, 4}};
  const Range ins[] = {{qkv, (size_t)c.rows * nh * 512},
                       {bias, nh * 256},
                       {c.row_start, ((size_t)c.b + 1) * 4},
                       {c.pos_base, (size_t)c.b * 4}};
  if (any_alias(outs, ins)) return SQ_ERR_ALIAS;
  (void)hipGetLastError();
  return device_status(sq::launch_packed_rope_kv(qkv, bias, packed(c), c.hq, c.hkv, c.pos_base, pos_offset,
                                                 c.len_bound, c.capacity, theta, q_out, kv, status, stream));
}

sq_status attention(const Call& c, const sq::KvCache& kv, bool q4, const uint16_t* q, int32_t pos_offset,
                    uint16_t* out, hipStream_t stream) {
  sq_status st = check_sizes(c);
  if (st != SQ_OK) return st;
  if (!q4 && c.capacity > kMaxAttnCapacity) return SQ_ERR_SHAPE;
  if (c.rows == 0) return SQ_OK;
  if (!q || !out) return SQ_ERR_NULL;
  st = check_arrays(c, kv, q4);
  if (st != SQ_OK) return st;
  if (!aligned(q, 16) || !aligned(out, 16)) return SQ_ERR_ALIGN;
  const CacheRanges cr = cache_ranges(c, kv, q4);
  const size_t qb = (size_t)c.rows * c.hq * 256;
  const Range outs[] = {{out, qb}};
  const Range ins[] = {{q, qb}, cr.r[0], cr.r[1], cr.r[2], cr.r[3], {c.row_start, ((size_t)c.b + 1) * 4},
                       {c.pos_base, (size_t)c.b * 4}};
  if (any_alias(outs, ins)) return SQ_ERR_ALIAS;
  (void)hipGetLastError();
  return device_status(sq::launch_packed_attention(q, packed(c), c.hq, c.hkv, c.pos_base, pos_offset, c.len_bound,
                                                   c.capacity, kv, out, stream));
}

uint16_t* mut(const uint16_t* p) { return const_cast<uint16_t*>(p); }  // read-only in the attention and the read
uint8_t* mut(const uint8_t* p) { return const_cast<uint8_t*>(p); }

}  // namespace

extern "C" {

sq_status sq_packed_rope_kv_f16(const float* qkv, const uint16_t* bias, const int32_t* row_start, int32_t b,
                                int64_t rows, int64_t max_rows, int32_t hq, int32_t hkv, const int32_t* pos_base,
                                int32_t pos_offset, int64_t len_bound, int64_t capacity, double theta,
                                uint16_t* q_out, uint16_t* k_cache, uint16_t* v_cache, int32_t* status,
                                hipStream_t stream) {
  return rope_kv({row_start, b, rows, max_rows, hq, hkv, pos_base, len_bound, capacity},
                 {k_cache, v_cache, nullptr, nullptr, nullptr, nullptr}, false, qkv, bias, pos_offset, theta, q_out,
                 status, stream);
}

sq_status sq_packed_rope_kv_q4(const float* qkv, const uint16_t* bias, const int32_t* row_start, int32_t b,
                               int64_t rows, int64_t max_rows, int32_t hq, int32_t hkv, const int32_t* pos_base,
                               int32_t pos_offset, int64_t len_bound, int64_t capacity, double theta, uint16_t* q_out,
                               uint8_t* k_codes, uint16_t* k_scales, uint8_t* v_codes, uint16_t* v_scales,
                               int32_t* status, hipStream_t stream) {
  return rope_kv({row_start, b, rows, max_rows, hq, hkv, pos_base, len_bound, capacity},
                 {nullptr, nullptr, k_codes, k_scales, v_codes, v_scales}, true, qkv, bias, pos_offset, theta, q_out,
                 status, stream);
}

sq_status sq_packed_kv_read_q4(const uint8_t* k_codes, const uint16_t* k_scales, const uint8_t* v_codes,
                               const uint16_t* v_scales, const int32_t* row_start, int32_t b, int64_t rows,
                               int64_t max_rows, int32_t hkv, const int32_t* pos_base, int32_t pos_offset,
                               int64_t len_bound, int64_t capacity, uint16_t* k_out, uint16_t* v_out,
                               hipStream_t stream) {
  const Call c{row_start, b, rows, max_rows, hkv, hkv, pos_base, len_bound, capacity};
  const sq::KvCache kv{nullptr, nullptr, mut(k_codes), mut(k_scales), mut(v_codes), mut(v_scales)};
  sq_status st = check_sizes(c);
  if (st != SQ_OK) return st;
  if (rows == 0) return SQ_OK;
  if (!k_out || !v_out) return SQ_ERR_NULL;
  st = check_arrays(c, kv, true);
  if (st != SQ_OK) return st;
  if (!aligned(k_out, 16) || !aligned(v_out, 16)) return SQ_ERR_ALIGN;
  const CacheRanges cr = cache_ranges(c, kv, true);
  const size_t ob = (size_t)rows * hkv * 256;
  const Range outs[] = {{k_out, ob}, {v_out, ob}};
  const Range ins[] = {cr.r[0], cr.r[1], cr.r[2], cr.r[3], {row_start, ((size_t)b + 1) * 4}, {pos_base, (size_t)b * 4}};
  if (any_alias(outs, ins)) return SQ_ERR_ALIAS;
  (void)hipGetLastError();
  return device_status(sq::launch_packed_kv_read(packed(c), hkv, pos_base, pos_offset, len_bound, capacity, kv, k_out,
                                                 v_out, stream));
}

sq_status sq_packed_attention_f16(const uint16_t* q, const uint16_t* k_cache, const uint16_t* v_cache,
                                  const int32_t* row_start, int32_t b, int64_t rows, int64_t max_rows, int32_t hq,
                                  int32_t hkv, const int32_t* pos_base, int32_t pos_offset, int64_t len_bound,
                                  int64_t capacity, uint16_t* out, hipStream_t stream) {
  return attention({row_start, b, rows, max_rows, hq, hkv, pos_base, len_bound, capacity},
                   {mut(k_cache), mut(v_cache), nullptr, nullptr, nullptr, nullptr}, false, q, pos_offset, out, stream);
}

sq_status sq_packed_attention_q4(const uint16_t* q, const uint8_t* k_codes, const uint16_t* k_scales,
                                 const uint8_t* v_codes, const uint16_t* v_scales, const int32_t* row_start, int32_t b,
                                 int64_t rows, int64_t max_rows, int32_t hq, int32_t hkv, const int32_t* pos_base,
                                 int32_t pos_offset, int64_t len_bound, int64_t capacity, uint16_t* out,
                                 hipStream_t stream) {
  return attention({row_start, b, rows, max_rows, hq, hkv, pos_base, len_bound, capacity},
                   {nullptr, nullptr, mut(k_codes), mut(k_scales), mut(v_codes), mut(v_scales)}, true, q, pos_offset,
                   out, stream);
}

}  // extern "C"

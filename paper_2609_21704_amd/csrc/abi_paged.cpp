// C ABI of paged caches: host-side argument validation and dispatch.
#include <math.h>

#include "abi_checks.hpp"
#include "specquant_paged.h"
#include "sq_internal.hpp"

static_assert(sq::kPage == SQ_PAGE, "one page size");
static_assert(sq::kPosIdle == SQ_POS_IDLE, "one mark of idle sequences");

namespace {

constexpr int64_t kMaxPages = int64_t(1) << 20;  // (and a table's width)
constexpr int32_t kMaxAhead = 1 << 20;
constexpr int32_t kMaxForks = 1024;  // a thread each
constexpr int64_t kMaxRows = int64_t(1) << 20;

// ---------------------------------------------------------------- the state
sq_status check_state(const int32_t* table, const int32_t* held, const int32_t* refs, int32_t b, int64_t width,
                      int64_t pages) {
  if (b < 1 || b > 65535 || width < 1 || width > kMaxPages || pages < 1 || pages > kMaxPages) return SQ_ERR_SHAPE;
  if (!table || !held || !refs) return SQ_ERR_NULL;
  if (!aligned(table, 4) || !aligned(held, 4) || !aligned(refs, 4)) return SQ_ERR_ALIGN;
  return SQ_OK;
}

size_t words(int64_t n) { return (size_t)n * 4; }

sq::PageState state(int32_t* table, const int32_t* held, int32_t* refs, int32_t b, int64_t width, int64_t pages) {
  return {table, const_cast<int32_t*>(held), refs, b, (int)width, (int)pages};  // (held: read only in compact)
}

// ------------------------------------------------------------ the paged calls
struct Call {
  const int32_t* row_start;
  int32_t b;
  int64_t rows, max_rows;
  int32_t hq, hkv;
  const int32_t* pos_base;
  int64_t len_bound;
  const int32_t* table;
  int64_t width, pages;
};

sq_status check_sizes(const Call& c) {
  if (c.max_rows < 1 || c.max_rows > kMaxRows || c.rows < 0 || c.rows > kMaxRows) return SQ_ERR_SHAPE;
  if (c.width < 1 || c.width > kMaxPages || c.pages < 1 || c.pages > kMaxPages) return SQ_ERR_SHAPE;
  const sq_status bs = check_block(c.b, 1, c.hq, c.hkv, c.len_bound, c.width * SQ_PAGE);
  if (bs != SQ_OK) return bs;
  if (!c.row_start && c.rows != c.b * c.max_rows) return SQ_ERR_SHAPE;
  return SQ_OK;
}

sq_status check_arrays(const Call& c, const sq::KvCache& kv, bool q4) {
  if (!c.pos_base || !c.table || (q4 ? !kv.k4 || !kv.ks || !kv.v4 || !kv.vs : !kv.k || !kv.v)) return SQ_ERR_NULL;
  if (!aligned(c.row_start, 4) || !aligned(c.pos_base, 4) || !aligned(c.table, 4) || !aligned(kv.k, 16) ||
      !aligned(kv.v, 16) || !aligned(kv.k4, 16) || !aligned(kv.ks, 16) || !aligned(kv.v4, 16) || !aligned(kv.vs, 16))
    return SQ_ERR_ALIGN;
  return SQ_OK;
}

struct CacheRanges {
  Range r[4];
};
CacheRanges cache_ranges(const Call& c, const sq::KvCache& kv, bool q4) {
  const size_t e = (size_t)c.pages * c.hkv * SQ_PAGE;
  if (q4) return {{{kv.k4, e * 64}, {kv.ks, e * 8}, {kv.v4, e * 64}, {kv.vs, e * 8}}};
  return {{{kv.k, e * 256}, {kv.v, e * 256}, {nullptr, 0}, {nullptr, 0}}};
}

sq::PackedRows packed(const Call& c) {
  return {c.row_start, c.b, (int)c.rows, (int)(c.max_rows < c.rows ? c.max_rows : c.rows)};
}

sq::KvCache paged(const Call& c, sq::KvCache kv) {
  kv.table = c.table;
  kv.width = (int)c.width;
  kv.pages = (int)c.pages;
  return kv;
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
                       {c.row_start, words(c.b + 1)},
                       {c.pos_base, words(c.b)},
                       {c.table, words(c.b * c.width)}};
  if (any_alias(outs, ins)) return SQ_ERR_ALIAS;
  (void)hipGetLastError();
  return device_status(sq::launch_packed_rope_kv(qkv, bias, packed(c), c.hq, c.hkv, c.pos_base, pos_offset,
                                                 c.len_bound, c.width * SQ_PAGE, theta, q_out, paged(c, kv), status,
                                                 stream));
}

sq_status attention(const Call& c, const sq::KvCache& kv, bool q4, const uint16_t* q, int32_t pos_offset,
                    uint16_t* out, hipStream_t stream) {
  sq_status st = check_sizes(c);
  if (st != SQ_OK) return st;
  if (c.rows == 0) return SQ_OK;
  if (!q || !out) return SQ_ERR_NULL;
  st = check_arrays(c, kv, q4);
  if (st != SQ_OK) return st;
  if (!aligned(q, 16) || !aligned(out, 16)) return SQ_ERR_ALIGN;
  const CacheRanges cr = cache_ranges(c, kv, q4);
  const size_t qb = (size_t)c.rows * c.hq * 256;
  const Range outs[] = {{out, qb}};
  const Range ins[] = {{q, qb}, cr.r[0], cr.r[1], cr.r[2], cr.r[3], {c.row_start, words(c.b + 1)},
                       {c.pos_base, words(c.b)}, {c.table, words(c.b * c.width)}};
  if (any_alias(outs, ins)) return SQ_ERR_ALIAS;
  (void)hipGetLastError();
  return device_status(sq::launch_packed_attention(q, packed(c), c.hq, c.hkv, c.pos_base, pos_offset, c.len_bound,
                                                   c.width * SQ_PAGE, paged(c, kv), out, stream));
}

uint16_t* mut(const uint16_t* p) { return const_cast<uint16_t*>(p); }  // read-only in the attention and the read
uint8_t* mut(const uint8_t* p) { return const_cast<uint8_t*>(p); }

}  // namespace

extern "C" {

sq_status sq_pages_reserve(int32_t* table, int32_t* held, int32_t* refs, int32_t b, int64_t width, int64_t pages,
                           const int32_t* pos_base, int32_t ahead, int32_t* status, hipStream_t stream) {
  const sq_status st = check_state(table, held, refs, b, width, pages);
  if (st != SQ_OK) return st;
  if (ahead < 0 || ahead > kMaxAhead) return SQ_ERR_SHAPE;
  if (!pos_base) return SQ_ERR_NULL;
  if (!aligned(pos_base, 4) || !aligned(status, 4)) return SQ_ERR_ALIGN;
  const Range outs[] = {{table, words(b * width)}, {held, words(b)}, {refs, words(pages)}, {status, 4}};
  const Range ins[] = {{pos_base, words(b)}};
  if (any_alias(outs, ins)) return SQ_ERR_ALIAS;
  (void)hipGetLastError();
  return device_status(
      sq::launch_pages_reserve(state(table, held, refs, b, width, pages), pos_base, ahead, status, stream));
}

sq_status sq_pages_trim(int32_t* table, int32_t* held, int32_t* refs, int32_t b, int64_t width, int64_t pages,
                        const int32_t* keep, int32_t* status, hipStream_t stream) {
  const sq_status st = check_state(table, held, refs, b, width, pages);
  if (st != SQ_OK) return st;
  if (!keep) return SQ_ERR_NULL;
  if (!aligned(keep, 4) || !aligned(status, 4)) return SQ_ERR_ALIGN;
  const Range outs[] = {{table, words(b * width)}, {held, words(b)}, {refs, words(pages)}, {status, 4}};
  const Range ins[] = {{keep, words(b)}};
  if (any_alias(outs, ins)) return SQ_ERR_ALIAS;
  (void)hipGetLastError();
  return device_status(sq::launch_pages_trim(state(table, held, refs, b, width, pages), keep, status, stream));
}

sq_status sq_pages_fork(int32_t* table, int32_t* held, int32_t* refs, int32_t b, int64_t width, int64_t pages,
                        const int32_t* parent, const int32_t* child, const int32_t* length, int32_t n, int32_t* src,
                        int32_t* dst, int32_t* count, int32_t* status, hipStream_t stream) {
  const sq_status st = check_state(table, held, refs, b, width, pages);
  if (st != SQ_OK) return st;
  if (n < 0 || n > kMaxForks) return SQ_ERR_SHAPE;
  if (!count || (n > 0 && (!parent || !child || !length || !src || !dst))) return SQ_ERR_NULL;
  if (!aligned(parent, 4) || !aligned(child, 4) || !aligned(length, 4) || !aligned(src, 4) || !aligned(dst, 4) ||
      !aligned(count, 4) || !aligned(status, 4))
    return SQ_ERR_ALIGN;
  const Range outs[] = {{table, words(b * width)}, {held, words(b)}, {refs, words(pages)}, {src, words(n)},
                        {dst, words(n)},           {count, 4},       {status, 4}};
  const Range ins[] = {{parent, words(n)}, {child, words(n)}, {length, words(n)}};
  if (any_alias(outs, ins)) return SQ_ERR_ALIAS;
  (void)hipGetLastError();
  return device_status(sq::launch_pages_fork(state(table, held, refs, b, width, pages), parent, child, length, n, src,
                                             dst, count, status, stream));
}

sq_status sq_pages_compact(int32_t* table, const int32_t* held, int32_t* refs, int32_t b, int64_t width, int64_t pages,
                           int32_t* src, int32_t* dst, int32_t* count, int32_t* used, int32_t* status,
                           hipStream_t stream) {
  const sq_status st = check_state(table, held, refs, b, width, pages);
  if (st != SQ_OK) return st;
  if (!count || !used || (pages > 1 && (!src || !dst))) return SQ_ERR_NULL;
  if (!aligned(src, 4) || !aligned(dst, 4) || !aligned(count, 4) || !aligned(used, 4) || !aligned(status, 4))
    return SQ_ERR_ALIGN;
  const Range outs[] = {{table, words(b * width)}, {refs, words(pages)}, {src, words(pages / 2)},
                        {dst, words(pages / 2)},   {count, 4},           {used, 4},
                        {status, 4}};
  const Range ins[] = {{held, words(b)}};
  if (any_alias(outs, ins)) return SQ_ERR_ALIAS;
  (void)hipGetLastError();
  return device_status(
      sq::launch_pages_compact(state(table, held, refs, b, width, pages), src, dst, count, used, status, stream));
}

sq_status sq_page_copy(void* pool, int32_t layers, int64_t pages, int64_t page_bytes, const int32_t* src,
                       const int32_t* dst, const int32_t* count, int64_t n, int32_t* status, hipStream_t stream) {
  if (layers < 1 || layers > 65535 || pages < 1 || pages > kMaxPages || page_bytes < 16 ||
      page_bytes > (int64_t(1) << 30) || page_bytes % 16 != 0 || n < 0 || n > kMaxPages)
    return SQ_ERR_SHAPE;
  if (layers * pages >= (int64_t(1) << 46) / page_bytes) return SQ_ERR_SHAPE;
  if (n == 0) return SQ_OK;
  if (!pool || !src || !dst || !count) return SQ_ERR_NULL;
  if (!aligned(pool, 16) || !aligned(src, 4) || !aligned(dst, 4) || !aligned(count, 4) || !aligned(status, 4))
    return SQ_ERR_ALIGN;
  const Range outs[] = {{pool, (size_t)(layers * pages * page_bytes)}, {status, 4}};
  const Range ins[] = {{src, words(n)}, {dst, words(n)}, {count, 4}};
  if (any_alias(outs, ins)) return SQ_ERR_ALIAS;
  (void)hipGetLastError();
  return device_status(
      sq::launch_page_copy(pool, layers, (int)pages, page_bytes, src, dst, count, (int)n, status, stream));
}

sq_status sq_paged_rope_kv_f16(const float* qkv, const uint16_t* bias, const int32_t* row_start, int32_t b,
                               int64_t rows, int64_t max_rows, int32_t hq, int32_t hkv, const int32_t* pos_base,
                               int32_t pos_offset, int64_t len_bound, const int32_t* table, int64_t width,
                               int64_t pages, double theta, uint16_t* q_out, uint16_t* k_pages, uint16_t* v_pages,
                               int32_t* status, hipStream_t stream) {
  return rope_kv({row_start, b, rows, max_rows, hq, hkv, pos_base, len_bound, table, width, pages},
                 {k_pages, v_pages, nullptr, nullptr, nullptr, nullptr}, false, qkv, bias, pos_offset, theta, q_out,
                 status, stream);
}

sq_status sq_paged_rope_kv_q4(const float* qkv, const uint16_t* bias, const int32_t* row_start, int32_t b, int64_t rows,
                              int64_t max_rows, int32_t hq, int32_t hkv, const int32_t* pos_base, int32_t pos_offset,
                              int64_t len_bound, const int32_t* table, int64_t width, int64_t pages, double theta,
                              uint16_t* q_out, uint8_t* k_codes, uint16_t* k_scales, uint8_t* v_codes,
                              uint16_t* v_scales, int32_t* status, hipStream_t stream) {
  return rope_kv({row_start, b, rows, max_rows, hq, hkv, pos_base, len_bound, table, width, pages},
                 {nullptr, nullptr, k_codes, k_scales, v_codes, v_scales}, true, qkv, bias, pos_offset, theta, q_out,
                 status, stream);
}

sq_status sq_paged_kv_read_q4(const uint8_t* k_codes, const uint16_t* k_scales, const uint8_t* v_codes,
                              const uint16_t* v_scales, const int32_t* table, int64_t width, int64_t pages,
                              const int32_t* row_start, int32_t b, int64_t rows, int64_t max_rows, int32_t hkv,
                              const int32_t* pos_base, int32_t pos_offset, int64_t len_bound, uint16_t* k_out,
                              uint16_t* v_out, hipStream_t stream) {
  const Call c{row_start, b, rows, max_rows, hkv, hkv, pos_base, len_bound, table, width, pages};
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
  const Range ins[] = {cr.r[0], cr.r[1], cr.r[2], cr.r[3], {row_start, words(b + 1)}, {pos_base, words(b)},
                       {table, words(b * width)}};
  if (any_alias(outs, ins)) return SQ_ERR_ALIAS;
  (void)hipGetLastError();
  return device_status(sq::launch_packed_kv_read(packed(c), hkv, pos_base, pos_offset, len_bound, width * SQ_PAGE,
                                                 paged(c, kv), k_out, v_out, stream));
}

sq_status sq_paged_attention_f16(const uint16_t* q, const uint16_t* k_pages, const uint16_t* v_pages,
                                 const int32_t* table, int64_t width, int64_t pages, const int32_t* row_start,
                                 int32_t b, int64_t rows, int64_t max_rows, int32_t hq, int32_t hkv,
                                 const int32_t* pos_base, int32_t pos_offset, int64_t len_bound, uint16_t* out,
                                 hipStream_t stream) {
  return attention({row_start, b, rows, max_rows, hq, hkv, pos_base, len_bound, table, width, pages},
                   {mut(k_pages), mut(v_pages), nullptr, nullptr, nullptr, nullptr}, false, q, pos_offset, out, stream);
}

sq_status sq_paged_attention_q4(const uint16_t* q, const uint8_t* k_codes, const uint16_t* k_scales,
                                const uint8_t* v_codes, const uint16_t* v_scales, const int32_t* table, int64_t width,
                                int64_t pages, const int32_t* row_start, int32_t b, int64_t rows, int64_t max_rows,
                                int32_t hq, int32_t hkv, const int32_t* pos_base, int32_t pos_offset,
                                int64_t len_bound, uint16_t* out, hipStream_t stream) {
  return attention({row_start, b, rows, max_rows, hq, hkv, pos_base, len_bound, table, width, pages},
                   {nullptr, nullptr, mut(k_codes), mut(k_scales), mut(v_codes), mut(v_scales)}, true, q, pos_offset, out,
                   stream);
}

}  // extern "C"

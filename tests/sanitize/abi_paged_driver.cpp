// Drives the calls over paged caches and the sampling calls (csrc/abi_paged.cpp,
// csrc/abi_sample.cpp) through valid, invalid and limit-sized arguments under
// AddressSanitizer and UndefinedBehaviorSanitizer, and checks what reaches the
// launchers.  Addresses are fake and never dereferenced (the launchers here
// only record their arguments).
#include <stdint.h>
#include <stdio.h>

#include <cmath>

#include "specquant_paged.h"
#include "specquant_sample.h"
#include "sq_internal.hpp"

extern "C" hipError_t hipGetLastError(void) { return hipSuccess; }

static struct {
  int calls, n, layers;
  int64_t bytes, ld, len_bound, capacity;
  sq::PackedRows rows;
  sq::KvCache cache;
  sq::PageState state;
  hipError_t result;
} seen;

namespace sq {
static hipError_t record(const PackedRows& pr, int64_t len_bound, int64_t capacity, const KvCache& cache) {
  ++seen.calls;
  seen.rows = pr;
  seen.len_bound = len_bound;
  seen.capacity = capacity;
  seen.cache = cache;
  return seen.result;
}
hipError_t launch_packed_rope_kv(const float*, const uint16_t*, const PackedRows& pr, int, int, const int32_t*, int,
                                 int64_t len_bound, int64_t capacity, double, uint16_t*, const KvCache& cache, int32_t*,
                                 hipStream_t) {
  return record(pr, len_bound, capacity, cache);
}
hipError_t launch_packed_kv_read(const PackedRows& pr, int, const int32_t*, int, int64_t len_bound, int64_t capacity,
                                 const KvCache& cache, uint16_t*, uint16_t*, hipStream_t) {
  return record(pr, len_bound, capacity, cache);
}
hipError_t launch_packed_attention(const uint16_t*, const PackedRows& pr, int, int, const int32_t*, int,
                                   int64_t len_bound, int64_t capacity, const KvCache& cache, uint16_t*, hipStream_t) {
  return record(pr, len_bound, capacity, cache);
}
static hipError_t state(const PageState& p, int n) {
  ++seen.calls;
  seen.state = p;
  seen.n = n;
  return seen.result;
}
hipError_t launch_pages_reserve(const PageState& p, const int32_t*, int ahead, int32_t*, hipStream_t) {
  return state(p, ahead);
}
hipError_t launch_pages_trim(const PageState& p, const int32_t*, int32_t*, hipStream_t) { return state(p, 0); }
hipError_t launch_pages_fork(const PageState& p, const int32_t*, const int32_t*, const int32_t*, int n, int32_t*, int32_t*,
                             int32_t*, int32_t*, hipStream_t) {
  return state(p, n);
}
hipError_t launch_pages_compact(const PageState& p, int32_t*, int32_t*, int32_t*, int32_t*, int32_t*, hipStream_t) {
  return state(p, 0);
}
hipError_t launch_page_copy(void*, int layers, int pages, int64_t bytes, const int32_t*, const int32_t*, const int32_t*,
                            int n, int32_t*, hipStream_t) {
  ++seen.calls;
  seen.layers = layers;
  seen.state.pages = pages;
  seen.bytes = bytes;
  seen.n = n;
  return seen.result;
}
hipError_t launch_sample(const float*, int m, int v, int64_t ld, const float*, const int32_t*, const float*, const float*,
                         const uint32_t*, int32_t*, float*, int32_t*, hipStream_t) {
  ++seen.calls;
  seen.n = m;
  seen.layers = v;
  seen.ld = ld;
  return seen.result;
}
}  // namespace sq

static int failures = 0;
#define CHECK(ok)                                    \
  do {                                               \
    if (!(ok)) {                                     \
      printf("FAIL line %d: %s\n", __LINE__, #ok);   \
      ++failures;                                    \
    }                                                \
  } while (0)

template <class T>
static T* at(int i) {  // far apart: 2^56 bytes each
  return reinterpret_cast<T*>((uint64_t)(i + 1) << 56);
}

struct Sizes {
  bool start;
  int32_t b;
  int64_t rows, max_rows;
  int32_t hq, hkv;
  int64_t len_bound, width, pages;
};

static int attention(bool q4, const Sizes& s, int32_t off) {
  const int32_t* start = s.start ? at<int32_t>(1) : nullptr;
  if (q4)
    return sq_paged_attention_q4(at<uint16_t>(0), at<uint8_t>(4), at<uint16_t>(5), at<uint8_t>(6), at<uint16_t>(7),
                                 at<int32_t>(8), s.width, s.pages, start, s.b, s.rows, s.max_rows, s.hq, s.hkv,
                                 at<int32_t>(2), off, s.len_bound, at<uint16_t>(3), nullptr);
  return sq_paged_attention_f16(at<uint16_t>(0), at<uint16_t>(4), at<uint16_t>(5), at<int32_t>(8), s.width, s.pages, start,
                                s.b, s.rows, s.max_rows, s.hq, s.hkv, at<int32_t>(2), off, s.len_bound, at<uint16_t>(3),
                                nullptr);
}
static int rope(bool q4, const Sizes& s, int32_t off, double theta = 1e6) {
  const int32_t* start = s.start ? at<int32_t>(1) : nullptr;
  if (q4)
    return sq_paged_rope_kv_q4(at<float>(0), at<uint16_t>(9), start, s.b, s.rows, s.max_rows, s.hq, s.hkv, at<int32_t>(2),
                               off, s.len_bound, at<int32_t>(8), s.width, s.pages, theta, at<uint16_t>(3), at<uint8_t>(4),
                               at<uint16_t>(5), at<uint8_t>(6), at<uint16_t>(7), at<int32_t>(10), nullptr);
  return sq_paged_rope_kv_f16(at<float>(0), nullptr, start, s.b, s.rows, s.max_rows, s.hq, s.hkv, at<int32_t>(2), off,
                              s.len_bound, at<int32_t>(8), s.width, s.pages, theta, at<uint16_t>(3), at<uint16_t>(4),
                              at<uint16_t>(5), nullptr, nullptr);
}
static int read(const Sizes& s, int32_t off) {
  return sq_paged_kv_read_q4(at<uint8_t>(4), at<uint16_t>(5), at<uint8_t>(6), at<uint16_t>(7), at<int32_t>(8), s.width,
                             s.pages, s.start ? at<int32_t>(1) : nullptr, s.b, s.rows, s.max_rows, s.hkv, at<int32_t>(2),
                             off, s.len_bound, at<uint16_t>(0), at<uint16_t>(3), nullptr);
}

static bool reached(const Sizes& s, bool q4) {
  return seen.rows.b == s.b && seen.rows.rows == s.rows &&
         seen.rows.max_rows == (s.max_rows < s.rows ? s.max_rows : s.rows) && seen.len_bound == s.len_bound &&
         seen.capacity == 64 * s.width && seen.cache.table == at<int32_t>(8) && seen.cache.width == s.width &&
         seen.cache.pages == s.pages && (q4 ? seen.cache.k4 == at<uint8_t>(4) && !seen.cache.k
                                            : seen.cache.k == at<uint16_t>(4) && !seen.cache.k4);
}

int main() {
  const int64_t most = int64_t(1) << 20, lmin = INT64_MIN, lmax = INT64_MAX;
  const int32_t imin = (int32_t)0x80000000, imax = 0x7FFFFFFF;
  const Sizes good[] = {{true, 2, 10, 8, 4, 2, 100, 2, 9},         {false, 3, 12, 4, 28, 4, 2048, 32, 1},
                        {true, 65535, most, most, 128, 1, 64 * most, most, most}, {false, 1, most, most, 128, 128, 1, 1, most}};
  for (const Sizes& s : good)
    for (int32_t off : {0, -1, imax, imin})
      for (bool q4 : {false, true}) {
        int before = seen.calls;
        CHECK(rope(q4, s, off) == SQ_OK && seen.calls == before + 1 && reached(s, q4));
        CHECK(attention(q4, s, off) == SQ_OK && seen.calls == before + 2 && reached(s, q4));
        CHECK(read(s, off) == SQ_OK && seen.calls == before + 3 && reached(s, true));
      }
  const Sizes bad[] = {{true, 0, 10, 8, 4, 2, 100, 2, 9},    {true, imin, 10, 8, 4, 2, 100, 2, 9},
                       {true, imax, 10, 8, 4, 2, 100, 2, 9}, {true, 2, lmin, 8, 4, 2, 100, 2, 9},
                       {true, 2, lmax, 8, 4, 2, 100, 2, 9},  {true, 2, 10, lmax, 4, 2, 100, 2, 9},
                       {true, 2, 10, 8, 4, imin, 100, 2, 9}, {true, 2, 10, 8, imin, imin, 100, 2, 9},
                       {true, 2, 10, 8, 4, 2, lmin, 2, 9},   {true, 2, 10, 8, 4, 2, lmax, 2, 9},
                       {true, 2, 10, 8, 4, 2, 129, 2, 9},    {true, 2, 10, 8, 4, 2, 1, 0, 9},
                       {true, 2, 10, 8, 4, 2, 1, lmax, 9},   {true, 2, 10, 8, 4, 2, 1, lmin, 9},
                       {true, 2, 10, 8, 4, 2, 1, most + 1, 9}, {true, 2, 10, 8, 4, 2, 1, 2, 0},
                       {true, 2, 10, 8, 4, 2, 1, 2, most + 1}, {true, 2, 10, 8, 4, 2, 1, 2, lmin},
                       {true, 2, 10, 8, 4, 2, 1, 2, lmax},   {false, 2, 10, 4, 4, 2, 100, 2, 9}};
  int before = seen.calls;
  for (const Sizes& s : bad) {
    for (bool q4 : {false, true}) CHECK(rope(q4, s, 0) == SQ_ERR_SHAPE && attention(q4, s, 0) == SQ_ERR_SHAPE);
    CHECK(read(s, 0) == SQ_ERR_SHAPE);
  }
  CHECK(rope(false, good[0], 0, std::nan("")) == SQ_ERR_NONFINITE && rope(true, good[0], 0, 0.5) == SQ_ERR_SHAPE);
  CHECK(seen.calls == before);

  // the state
  int32_t *table = at<int32_t>(0), *held = at<int32_t>(1), *refs = at<int32_t>(2), *in = at<int32_t>(3);
  struct Pool {
    int32_t b;
    int64_t width, pages;
  };
  for (const Pool& p : {Pool{1, 1, 1}, Pool{7, 30, 100}, Pool{65535, most, most}}) {
    for (int32_t ahead : {0, 1, 1 << 20}) {
      CHECK(sq_pages_reserve(table, held, refs, p.b, p.width, p.pages, in, ahead, nullptr, nullptr) == SQ_OK);
      CHECK(seen.n == ahead && seen.state.b == p.b && seen.state.width == p.width && seen.state.pages == p.pages);
    }
    CHECK(sq_pages_trim(table, held, refs, p.b, p.width, p.pages, in, at<int32_t>(4), nullptr) == SQ_OK);
    for (int32_t n : {0, 1, 1024})
      CHECK(sq_pages_fork(table, held, refs, p.b, p.width, p.pages, in, at<int32_t>(4), at<int32_t>(5), n, at<int32_t>(6),
                          at<int32_t>(7), at<int32_t>(8), nullptr, nullptr) == SQ_OK &&
            seen.n == n);
    CHECK(sq_pages_compact(table, held, refs, p.b, p.width, p.pages, at<int32_t>(6), at<int32_t>(7), at<int32_t>(8),
                           at<int32_t>(9), nullptr, nullptr) == SQ_OK);
  }
  CHECK(sq_pages_fork(table, held, refs, 3, 3, 9, nullptr, nullptr, nullptr, 0, nullptr, nullptr, at<int32_t>(8), nullptr,
                      nullptr) == SQ_OK);
  before = seen.calls;
  for (const Pool& p : {Pool{0, 1, 1}, Pool{imin, 1, 1}, Pool{imax, 1, 1}, Pool{1, 0, 1}, Pool{1, lmin, 1}, Pool{1, lmax, 1},
                        Pool{1, 1, 0}, Pool{1, 1, lmin}, Pool{1, 1, lmax}, Pool{1, most + 1, 1}, Pool{1, 1, most + 1}}) {
    CHECK(sq_pages_reserve(table, held, refs, p.b, p.width, p.pages, in, 1, nullptr, nullptr) == SQ_ERR_SHAPE);
    CHECK(sq_pages_trim(table, held, refs, p.b, p.width, p.pages, in, nullptr, nullptr) == SQ_ERR_SHAPE);
    CHECK(sq_pages_fork(table, held, refs, p.b, p.width, p.pages, in, in, in, 1, at<int32_t>(6), at<int32_t>(7),
                        at<int32_t>(8), nullptr, nullptr) == SQ_ERR_SHAPE);
    CHECK(sq_pages_compact(table, held, refs, p.b, p.width, p.pages, at<int32_t>(6), at<int32_t>(7), at<int32_t>(8),
                           at<int32_t>(9), nullptr, nullptr) == SQ_ERR_SHAPE);
  }
  for (int32_t n : {-1, 1025, imin, imax})
    CHECK(sq_pages_fork(table, held, refs, 2, 2, 9, in, at<int32_t>(4), at<int32_t>(5), n, at<int32_t>(6), at<int32_t>(7),
                        at<int32_t>(8), nullptr, nullptr) == SQ_ERR_SHAPE);
  for (int32_t ahead : {-1, imin, imax, (1 << 20) + 1})
    CHECK(sq_pages_reserve(table, held, refs, 2, 2, 9, in, ahead, nullptr, nullptr) == SQ_ERR_SHAPE);
  CHECK(seen.calls == before);

  // copies
  struct Copy {
    int32_t layers;
    int64_t pages, bytes, n;
  };
  for (const Copy& c : {Copy{1, 1, 16, 1}, Copy{28, 500, 65536, 250}, Copy{65535, 1, int64_t(1) << 29, most},
                        Copy{1, most - 1, int64_t(1) << 26, most}})
    CHECK(sq_page_copy(at<void>(0), c.layers, c.pages, c.bytes, in, at<int32_t>(4), at<int32_t>(5), c.n, nullptr, nullptr) ==
              SQ_OK &&
          seen.layers == c.layers && seen.state.pages == c.pages && seen.bytes == c.bytes && seen.n == c.n);
  before = seen.calls;
  CHECK(sq_page_copy(nullptr, 1, 1, 16, nullptr, nullptr, nullptr, 0, nullptr, nullptr) == SQ_OK);
  for (const Copy& c : {Copy{0, 1, 16, 1}, Copy{imin, 1, 16, 1}, Copy{65536, 1, 16, 1}, Copy{1, 0, 16, 1}, Copy{1, lmax, 16, 1},
                        Copy{1, 1, 0, 1}, Copy{1, 1, 24, 1}, Copy{1, 1, lmin, 1}, Copy{1, 1, lmax - 15, 1}, Copy{1, 1, 16, -1},
                        Copy{1, 1, 16, lmax}, Copy{65535, most, 1040, 1}, Copy{1, most, int64_t(1) << 26, 1}})
    CHECK(sq_page_copy(at<void>(0), c.layers, c.pages, c.bytes, in, at<int32_t>(4), at<int32_t>(5), c.n, nullptr, nullptr) ==
          SQ_ERR_SHAPE);
  CHECK(seen.calls == before);

  // sampling
  struct Rows {
    int32_t m;
    int64_t v, ld;
  };
  auto draw = [&](const Rows& r) {
    return sq_sample_f32(at<float>(0), r.m, r.v, r.ld, at<float>(1), nullptr, at<float>(2), nullptr, at<uint32_t>(3),
                         at<int32_t>(4), at<int32_t>(5), nullptr);
  };
  auto filter = [&](const Rows& r, float* out) {
    return sq_filter_logits_f32(at<float>(0), r.m, r.v, r.ld, nullptr, at<int32_t>(1), nullptr, at<float>(2), out, nullptr,
                                nullptr);
  };
  for (const Rows& r : {Rows{1, 1, 1}, Rows{64, 151936, 152064}, Rows{1 << 20, 1 << 26, imax}}) {
    CHECK(draw(r) == SQ_OK && seen.n == r.m && seen.layers == r.v && seen.ld == r.ld);
    CHECK(filter(r, at<float>(3)) == SQ_OK && filter(r, at<float>(0)) == SQ_OK && seen.ld == r.ld);
  }
  before = seen.calls;
  for (const Rows& r : {Rows{0, 1, 1}, Rows{imin, 1, 1}, Rows{imax, 1, 1}, Rows{1, 0, 1}, Rows{1, lmin, 1}, Rows{1, lmax, lmax},
                        Rows{1, 2, 1}, Rows{1, 1, lmin}, Rows{1, 1, lmax}, Rows{1, (1 << 26) + 1, imax}})
    CHECK(draw(r) == SQ_ERR_SHAPE && filter(r, at<float>(3)) == SQ_ERR_SHAPE);
  // the last logit of the last row, 2^53 bytes on
  const Rows far{1 << 20, 1 << 26, imax};
  CHECK(filter(far, at<float>(0) + ((int64_t)far.m - 1) * far.ld + far.v - 1) == SQ_ERR_ALIAS);
  CHECK(seen.calls == before);
  // what a launcher reports
  seen.result = hipErrorStreamCaptureUnsupported;
  CHECK(draw({1, 1, 1}) == SQ_ERR_CAPTURE && attention(false, good[0], 0) == SQ_ERR_CAPTURE);
  CHECK(sq_pages_reserve(table, held, refs, 2, 2, 9, in, 1, nullptr, nullptr) == SQ_ERR_CAPTURE);
  seen.result = hipErrorOutOfMemory;
  CHECK(filter({1, 1, 1}, at<float>(3)) == SQ_ERR_DEVICE && rope(true, good[0], 0) == SQ_ERR_DEVICE);
  printf(failures ? "FAILED %d\n" : "ABI OK\n", failures);
  return failures ? 1 : 0;
}

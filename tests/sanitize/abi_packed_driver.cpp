// Drives the calls over packed rows and the 4-bit cache (csrc/abi_packed.cpp)
// through valid, invalid and limit-sized arguments under AddressSanitizer and
// UndefinedBehaviorSanitizer, and checks what reaches the launchers.  Addresses
// are fake and never dereferenced (the launchers here only record their arguments).
#include <stdint.h>
#include <stdio.h>

#include <cmath>

#include "specquant_packed.h"
#include "sq_internal.hpp"

extern "C" hipError_t hipGetLastError(void) { return hipSuccess; }

static struct {
  int calls, hq, hkv, pos_offset;
  int64_t len_bound, capacity;
  sq::PackedRows rows;
  sq::KvCache cache;
  hipError_t result;
} seen;

namespace sq {
static hipError_t record(const PackedRows& pr, int hq, int hkv, int pos_offset, int64_t len_bound, int64_t capacity,
                         const KvCache& cache) {
  ++seen.calls;
  seen.rows = pr;
  seen.hq = hq;
  seen.hkv = hkv;
  seen.pos_offset = pos_offset;
  seen.len_bound = len_bound;
  seen.capacity = capacity;
  seen.cache = cache;
  return seen.result;
}
hipError_t launch_packed_rope_kv(const float*, const uint16_t*, const PackedRows& pr, int hq, int hkv, const int32_t*,
                                 int pos_offset, int64_t len_bound, int64_t capacity, double, uint16_t*,
                                 const KvCache& cache, int32_t*, hipStream_t) {
  return record(pr, hq, hkv, pos_offset, len_bound, capacity, cache);
}
hipError_t launch_packed_kv_read(const PackedRows& pr, int hkv, const int32_t*, int pos_offset, int64_t len_bound,
                                 int64_t capacity, const KvCache& cache, uint16_t*, uint16_t*, hipStream_t) {
  return record(pr, 0, hkv, pos_offset, len_bound, capacity, cache);
}
hipError_t launch_packed_attention(const uint16_t*, const PackedRows& pr, int hq, int hkv, const int32_t*,
                                   int pos_offset, int64_t len_bound, int64_t capacity, const KvCache& cache,
                                   uint16_t*, hipStream_t) {
  return record(pr, hq, hkv, pos_offset, len_bound, capacity, cache);
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
static T* at(uint64_t a) {
  return reinterpret_cast<T*>(a);
}
// far apart: 2^56 bytes each
static uint64_t place(int i) { return (uint64_t)(i + 1) << 56; }

struct Sizes {
  bool start;
  int32_t b;
  int64_t rows, max_rows;
  int32_t hq, hkv;
  int64_t len_bound, capacity;
};

static int rope(bool q4, const Sizes& s, int32_t off, double theta = 1e6) {
  const float* qkv = at<float>(place(0));
  const int32_t *start = s.start ? at<int32_t>(place(1)) : nullptr, *pos = at<int32_t>(place(2));
  uint16_t* q = at<uint16_t>(place(3));
  if (q4)
    return sq_packed_rope_kv_q4(qkv, at<uint16_t>(place(8)), start, s.b, s.rows, s.max_rows, s.hq, s.hkv, pos, off,
                                s.len_bound, s.capacity, theta, q, at<uint8_t>(place(4)), at<uint16_t>(place(5)),
                                at<uint8_t>(place(6)), at<uint16_t>(place(7)), at<int32_t>(place(9)), nullptr);
  return sq_packed_rope_kv_f16(qkv, nullptr, start, s.b, s.rows, s.max_rows, s.hq, s.hkv, pos, off, s.len_bound,
                               s.capacity, theta, q, at<uint16_t>(place(4)), at<uint16_t>(place(5)), nullptr, nullptr);
}
static int attention(bool q4, const Sizes& s, int32_t off) {
  const uint16_t* q = at<uint16_t>(place(0));
  const int32_t *start = s.start ? at<int32_t>(place(1)) : nullptr, *pos = at<int32_t>(place(2));
  uint16_t* out = at<uint16_t>(place(3));
  if (q4)
    return sq_packed_attention_q4(q, at<uint8_t>(place(4)), at<uint16_t>(place(5)), at<uint8_t>(place(6)),
                                  at<uint16_t>(place(7)), start, s.b, s.rows, s.max_rows, s.hq, s.hkv, pos, off,
                                  s.len_bound, s.capacity, out, nullptr);
  return sq_packed_attention_f16(q, at<uint16_t>(place(4)), at<uint16_t>(place(5)), start, s.b, s.rows, s.max_rows,
                                 s.hq, s.hkv, pos, off, s.len_bound, s.capacity, out, nullptr);
}
static int read(const Sizes& s, int32_t off) {
  return sq_packed_kv_read_q4(at<uint8_t>(place(4)), at<uint16_t>(place(5)), at<uint8_t>(place(6)),
                              at<uint16_t>(place(7)), s.start ? at<int32_t>(place(1)) : nullptr, s.b, s.rows,
                              s.max_rows, s.hkv, at<int32_t>(place(2)), off, s.len_bound, s.capacity,
                              at<uint16_t>(place(8)), at<uint16_t>(place(9)), nullptr);
}

static bool reached(const Sizes& s, int32_t off, int64_t max_rows, bool q4) {
  return seen.rows.start == (s.start ? at<int32_t>(place(1)) : nullptr) && seen.rows.b == s.b &&
         seen.rows.rows == s.rows && seen.rows.max_rows == max_rows && seen.hkv == s.hkv && seen.pos_offset == off &&
         seen.len_bound == s.len_bound && seen.capacity == s.capacity &&
         (q4 ? !seen.cache.k && !seen.cache.v && seen.cache.k4 == at<uint8_t>(place(4)) &&
                   seen.cache.ks == at<uint16_t>(place(5)) && seen.cache.v4 == at<uint8_t>(place(6)) &&
                   seen.cache.vs == at<uint16_t>(place(7))
             : seen.cache.k == at<uint16_t>(place(4)) && seen.cache.v == at<uint16_t>(place(5)) && !seen.cache.k4 &&
                   !seen.cache.ks && !seen.cache.v4 && !seen.cache.vs);
}

int main() {
  const int64_t most = int64_t(1) << 20, cap31 = (int64_t(1) << 31) - 64, cap28 = int64_t(1) << 28;
  // valid: ordinary, and at every limit
  const Sizes good[] = {{true, 2, 10, 8, 4, 2, 100, 128},
                        {false, 3, 12, 4, 28, 4, 2048, 2048},
                        {true, 65535, most, most, 128, 1, cap28, cap28},
                        {true, 8191, most, 1, 128, 8, 1, 64},
                        {false, 65535, 65535 * 16, 16, 1, 1, cap28, cap28},
                        {false, 1, most, most, 128, 128, cap28, cap28},
                        {true, 1, 1, most, 7, 1, 64, 64}};
  for (const Sizes& s : good) {
    const int64_t clipped = s.max_rows < s.rows ? s.max_rows : s.rows;
    for (int32_t off : {0, -1, 0x7FFFFFFF, (int32_t)0x80000000}) {
      for (bool q4 : {false, true}) {
        int before = seen.calls;
        CHECK(rope(q4, s, off) == SQ_OK && seen.calls == before + 1 && reached(s, off, clipped, q4) && seen.hq == s.hq);
        before = seen.calls;
        CHECK(attention(q4, s, off) == SQ_OK && seen.calls == before + 1 && reached(s, off, clipped, q4) &&
              seen.hq == s.hq);
      }
      const int before = seen.calls;
      CHECK(read(s, off) == SQ_OK && seen.calls == before + 1 && reached(s, off, clipped, true));
    }
  }
  // the longest capacity: all but the attention over fp16 entries
  const Sizes longest{true, 65535, most, most, 1, 1, cap31, cap31};
  CHECK(rope(false, longest, 0) == SQ_OK && reached(longest, 0, most, false));
  CHECK(rope(true, longest, 0) == SQ_OK && attention(true, longest, 0) == SQ_OK && read(longest, 0) == SQ_OK);
  CHECK(attention(false, longest, 0) == SQ_ERR_SHAPE);
  // nothing to do, and refused sizes: no launch
  const int before = seen.calls;
  const Sizes none{true, 2, 0, 8, 4, 2, 100, 128};
  CHECK(rope(false, none, 0) == SQ_OK && rope(true, none, 0) == SQ_OK && read(none, 0) == SQ_OK &&
        attention(false, none, 0) == SQ_OK && attention(true, none, 0) == SQ_OK);
  const int32_t imin = (int32_t)0x80000000, imax = 0x7FFFFFFF;
  const int64_t lmin = INT64_MIN, lmax = INT64_MAX;
  const Sizes bad[] = {{true, 0, 10, 8, 4, 2, 100, 128},        {true, imin, 10, 8, 4, 2, 100, 128},
                       {true, imax, 10, 8, 4, 2, 100, 128},     {true, 65536, 10, 8, 4, 1, 100, 128},
                       {true, 2, -1, 8, 4, 2, 100, 128},        {true, 2, lmin, 8, 4, 2, 100, 128},
                       {true, 2, lmax, 8, 4, 2, 100, 128},      {true, 2, most + 1, 8, 4, 2, 100, 128},
                       {true, 2, 10, 0, 4, 2, 100, 128},        {true, 2, 10, lmin, 4, 2, 100, 128},
                       {true, 2, 10, lmax, 4, 2, 100, 128},     {false, 2, 10, 4, 4, 2, 100, 128},
                       {false, 65535, 0, most, 4, 1, 100, 128}, {true, 2, 10, 8, 4, 0, 100, 128},
                       {true, 2, 10, 8, 4, imin, 100, 128},     {true, 2, 10, 8, imin, imin, 100, 128},
                       {true, 2, 10, 8, 129, 129, 100, 128},    {true, 2, 10, 8, 4, 2, lmin, 128},
                       {true, 2, 10, 8, 4, 2, lmax, 128},       {true, 2, 10, 8, 4, 2, 64, 63},
                       {true, 2, 10, 8, 4, 2, 64, lmin},        {true, 2, 10, 8, 4, 2, 64, lmax - 63},
                       {true, 2, 10, 8, 4, 2, 64, cap31 + 64}};
  for (const Sizes& s : bad) {
    for (bool q4 : {false, true}) CHECK(rope(q4, s, 0) == SQ_ERR_SHAPE && attention(q4, s, 0) == SQ_ERR_SHAPE);
    CHECK(read(s, 0) == SQ_ERR_SHAPE);
  }
  CHECK(rope(false, good[0], 0, std::nan("")) == SQ_ERR_NONFINITE && rope(true, good[0], 0, 0.5) == SQ_ERR_SHAPE);
  CHECK(seen.calls == before);
  // ranges: a cache of 2^28 positions reaches into what lies 2^38 bytes on
  CHECK(sq_packed_attention_f16(at<uint16_t>(place(0)), at<uint16_t>(place(1)), at<uint16_t>(place(2)), nullptr, 8, 8, 1,
                                4, 4, at<int32_t>(place(3)), 0, 64, cap28, at<uint16_t>(place(1) + (1ull << 38)),
                                nullptr) == SQ_ERR_ALIAS);
  CHECK(sq_packed_kv_read_q4(at<uint8_t>(place(4)), at<uint16_t>(place(5)), at<uint8_t>(place(6)),
                             at<uint16_t>(place(7)), nullptr, 1, most, most, 128, at<int32_t>(place(2)), 0, 64, 64,
                             at<uint16_t>(place(8)), at<uint16_t>(place(8) + (most * 128 - 1) * 256), nullptr) ==
        SQ_ERR_ALIAS);
  CHECK(seen.calls == before);
  // what a launcher reports
  seen.result = hipErrorStreamCaptureUnsupported;
  CHECK(attention(true, good[0], 0) == SQ_ERR_CAPTURE);
  seen.result = hipErrorOutOfMemory;
  CHECK(attention(false, good[0], 0) == SQ_ERR_DEVICE && rope(true, good[0], 0) == SQ_ERR_DEVICE &&
        read(good[0], 0) == SQ_ERR_DEVICE);
  printf(failures ? "FAILED %d\n" : "ABI OK\n", failures);
  return failures ? 1 : 0;
}

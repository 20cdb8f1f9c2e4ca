// Sampling and filtering of vocabulary rows: temperature, top-k, top-p, min-p (include/specquant_sample.h has the
// definition).  No row is sorted: top-k and top-p keep a prefix of the order (logit descending, index ascending), so each
// is a cut through it, and the last kept token (logit, index) says which are kept.
//   1. range_kernel   per (row, segment) the largest and smallest logit
//   2. bins_kernel    per (row, segment) the weights' sums and counts in 1024 bins of the distance from the maximum;
//                     the row's last workgroup finds the bins that the cuts go through
//   3. cut_kernel     gathers the tokens of those bins (a few) and sums the weights that are kept for sure; the row's
//                     last workgroup ranks the gathered tokens against each other, which gives the cuts, and draws
//   4. filter_kernel  writes the kept logits
// A row without top-k and top-p is drawn from by step 2.  Where the bins of the cuts hold too many tokens to rank (ties,
// rows whose logits lie close together but for a few), the last workgroup finds the cuts by a radix selection over the
// row (11 bits of the logit's key a pass).
// Weights are whole numbers, so their sums do not depend on any order.  Rows are cut into segments so that a call fills
// the chip from one row on; last workgroups are found by counting arrivals (counters that step 1 clears).
// Bound by latency in few rows, by fp64 instructions in many (a weight is about 30 of them).
#include <limits.h>

#include "sq_internal.hpp"
#include "sq_softmax.hpp"

#pragma clang fp contract(off)

namespace sq {
namespace {

constexpr int32_t kNoDist = 8, kBadParam = 256;  // the SQ_DEV_* values of the C headers
constexpr int kThreads = 1024, kWaves = kThreads / kWave;
constexpr int kBins = kThreads;   // one a thread where they are scanned
constexpr int kMost = 2048;       // gathered tokens of a row that are ranked
constexpr int kMaxSegments = 16;  // of a row
constexpr int kMinSegment = 4096; // tokens
constexpr double kSpan = 32.0;    // nats below the maximum that the bins cover (e^-32 < 2^-46)

struct SampleArgs {
  const float* logits;
  int v;
  int64_t ld;
  const float *temperature, *top_p, *min_p;
  const int32_t* top_k;
  const uint32_t* u24;
  int32_t* token;  // null: filter
  float* out;
  int32_t* status;
  int segments, len;  // of a row; tokens of a segment
  int shift;          // log2 of the largest weight
};

struct Cell {  // of a segment; bad: a NaN or +inf
  float hi, lo;
  int at, bad;
};

// What step 2 finds of a row, for step 3, and what step 3 finds, for step 4.
struct Cut {
  int mode;         // kDone, kAll (nothing is cut), kCut
  int sure;         // bins below it are kept
  int g0, g1;       // bins through which top-p's cut goes, g0 > g1: none
  int bk, rk;       // bin through which top-k's cut goes, and how many of it are kept; bk < 0: none
  int64_t before;   // sum of R below g0
  int64_t before_k; // below bk (bk < 0: of everything that top-k keeps)
  float hi, scale;  // bins
  float last;       // the last kept token
  int last_at;
};
enum : int { kDone = 0, kAll = 1, kCut = 2, kNan = 3, kSame = 4 };

struct Scratch {
  Cell* cells;       // [m][segments]
  int64_t* sums;     // [m][segments][kBins], then [m][segments] of step 3
  int64_t* kept;
  int64_t* counts;   // [m][segments][kBins]
  int64_t* list;     // [m][kMost]: logit in the low half, index in the high one
  Cut* cuts;         // [m]
  int32_t* counters; // [m][4]: arrivals of steps 2 and 3, gathered tokens
};

__device__ __forceinline__ void flag(int32_t* status, int32_t bit) {
  if (status) atomicOr(status, bit);
}

struct Params {
  float t, top_p, min_p;
  int top_k;  // 0: off
  bool bad;
  __device__ __forceinline__ Params(const SampleArgs& a, int row) {
    t = a.temperature ? a.temperature[row] : 1.f;
    top_p = a.top_p ? a.top_p[row] : 1.f;
    min_p = a.min_p ? a.min_p[row] : 0.f;
    top_k = a.top_k ? a.top_k[row] : 0;
    bad = !(t >= 0.f && t < INFINITY) || !(top_p >= 0.f) || !(min_p >= 0.f);
    min_p = fminf(min_p, 1.f);
    if (top_k < 0 || top_k >= a.v) top_k = 0;
  }
};

// The weight of a logit, and on the grid.
struct Weight {
  Soft<false> sf;
  double zmax, grid;
  __device__ __forceinline__ Weight(float t, float hi, int shift) : sf(t), zmax(sf.z(hi)), grid(ldexp(1.0, shift)) {}
  __device__ __forceinline__ float w(float l) const { return (float)sf.exp(sf.z(l) - zmax); }
  __device__ __forceinline__ int64_t r(float w) const { return llrint((double)w * grid); }
};

// Bins of the distance from the maximum, in the order of the logits: differences, products and minima round monotonically.
__device__ __forceinline__ int bin_of(float hi, float scale, float l) {
  return (int)fminf((hi - l) * scale, (float)(kBins - 1));
}

// A key whose order is that of the logits, descending (-0 as 0).
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t u = __builtin_bit_cast(uint32_t, l + 0.f);
  return (u >> 31) ? u : ~(u | 0x80000000u);
}

// `last`, `at` in (and everything before it in the order) against (l, j)
__device__ __forceinline__ bool up_to(float l, int j, float last, int at) { return l > last || (l == last && j <= at); }

// Tokens of a segment in steps of kBatch a thread, their loads in flight together; f(l, j) for every one.
constexpr int kBatch = 8;
template <class F>
__device__ __forceinline__ void each_token(const float* row, int from, int to, F f) {
  for (int base = from; base < to; base += kThreads * kBatch) {  // uniform
    float x[kBatch];
#pragma unroll
    for (int e = 0; e < kBatch; ++e) x[e] = row[min(base + e * kThreads + (int)threadIdx.x, to - 1)];
#pragma unroll
    for (int e = 0; e < kBatch; ++e) {
      const int j = base + e * kThreads + (int)threadIdx.x;
      if (j < to) f(x[e], j);
    }
  }
}

// True in every thread of the row's last workgroup to arrive, after whose return it sees what all of them published.
__device__ __forceinline__ bool last_of_row(int32_t* counter, int n, int* sh) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) *sh = arrive(counter, n);
  __syncthreads();
  return *sh != 0;
}

// ------------------------------------------------------------------- step 1
__global__ __launch_bounds__(kThreads) void range_kernel(SampleArgs a, Scratch sc) {
  __shared__ Cell sh[kWaves];
  const int row = blockIdx.x / a.segments, seg = blockIdx.x - row * a.segments;
  const int from = seg * a.len, to = min(from + a.len, a.v);
  if (seg == 0 && threadIdx.x < 4) sc.counters[4 * (int64_t)row + threadIdx.x] = 0;
  Cell c = {-INFINITY, INFINITY, INT_MAX, 0};
  each_token(a.logits + row * a.ld, from, to, [&](float l, int j) {
    c.bad |= isnan(l) || l == INFINITY ? 1 : 0;
    if (l > c.hi) {
      c.hi = l;
      c.at = j;
    }
    if (l > -INFINITY) c.lo = fminf(c.lo, l);
  });
  auto merge = [](Cell x, Cell y) {
    const bool other = y.hi > x.hi || (y.hi == x.hi && y.at < x.at);
    return Cell{other ? y.hi : x.hi, fminf(x.lo, y.lo), other ? y.at : x.at, x.bad | y.bad};
  };
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1)
    c = merge(c, Cell{__shfl_xor(c.hi, d), __shfl_xor(c.lo, d), __shfl_xor(c.at, d), __shfl_xor(c.bad, d)});
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = c;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < kWaves; ++w) c = merge(c, sh[w]);
    sc.cells[(int64_t)row * a.segments + seg] = c;
  }
}

__device__ __forceinline__ Cell row_cell(const SampleArgs& a, const Scratch& sc, int row) {
  Cell c = sc.cells[(int64_t)row * a.segments];
  for (int s = 1; s < a.segments; ++s) {
    const Cell y = sc.cells[(int64_t)row * a.segments + s];
    if (y.hi > c.hi) {  // (the first of equal ones stays)
      c.hi = y.hi;
      c.at = y.at;
    }
    c.lo = fminf(c.lo, y.lo);
    c.bad |= y.bad;
  }
  return c;
}

// ------------------------------------------------------------------ drawing
// The smallest j in [from, to) whose running sum of f(l, j) exceeds t (from <= every j; t < the sum of all): the wavefronts
// sum a run each, then the workgroup the one that holds it.
template <class F>
__device__ __forceinline__ int locate(const float* row, int from, int to, int64_t t, F f, int64_t* sh, int* shi) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int run = (to - from + kWaves - 1) / kWaves;
  const int r0 = from + min(w * run, to - from), r1 = min(r0 + run, to);
  int64_t s = 0;
  for (int base = r0; base < r1; base += kWave * kBatch) {
    float x[kBatch];
#pragma unroll
    for (int e = 0; e < kBatch; ++e) x[e] = row[min(base + e * kWave + lane, r1 - 1)];
#pragma unroll
    for (int e = 0; e < kBatch; ++e) {
      const int j = base + e * kWave + lane;
      if (j < r1) s += f(x[e], j);
    }
  }
  s = wave_sum_i64(s);
  __syncthreads();
  if (lane == 0) sh[w] = s;
  __syncthreads();
  int mine = kWaves - 1;
  int64_t before = 0;
  for (int i = 0; i < kWaves; ++i) {
    if (t < before + sh[i]) {
      mine = i;
      break;
    }
    before += sh[i];
  }
  const int b0 = from + min(mine * run, to - from), b1 = min(b0 + run, to);
  __syncthreads();
  // every thread a few consecutive tokens
  const int per = (b1 - b0 + kThreads - 1) / kThreads;
  const int p0 = b0 + min((int)threadIdx.x * per, b1 - b0), p1 = min(p0 + per, b1);
  int64_t part = 0;
  for (int j = p0; j < p1; ++j) part += f(row[j], j);
  int64_t total;
  int64_t at = before + block_exclusive_scan_i64<kWaves>(part, sh, total);
  if (part > 0 && at <= t && t < at + part) {
    int j = p0;
    for (; j < p1 - 1; ++j) {
      at += f(row[j], j);
      if (t < at) break;
    }
    *shi = j;
  }
  __syncthreads();
  return *shi;
}

__device__ __forceinline__ int64_t draw_at(uint32_t u24, int64_t z) {  // floor(u z / 2^24)
  const int64_t u = u24 & 0xFFFFFF;
  return u * (z >> 24) + ((u * (z & 0xFFFFFF)) >> 24);
}

// A token of a row with the sums of R of its segments in seg_sum (LDS) and the weight f of a kept token.
template <class F>
__device__ __forceinline__ void draw(const SampleArgs& a, int row, const int64_t* seg_sum, F f, int64_t* sh, int* shi) {
  int64_t z = 0;
  for (int s = 0; s < a.segments; ++s) z += seg_sum[s];
  int64_t t = draw_at(a.u24[row], z);
  int seg = 0;
  while (seg + 1 < a.segments && t >= seg_sum[seg]) t -= seg_sum[seg++];
  const int from = seg * a.len, to = min(from + a.len, a.v);
  const int j = locate(a.logits + row * a.ld, from, to, t, f, sh, shi);
  if (threadIdx.x == 0) a.token[row] = j;
}

// ------------------------------------------------------------------- step 2
__device__ __forceinline__ int64_t need_of(float top_p, int64_t z) {
  const int64_t n = (int64_t)ceil((double)top_p * (double)z);
  return n < 1 ? 1 : n;
}

__global__ __launch_bounds__(kThreads) void bins_kernel(SampleArgs a, Scratch sc) {
  __shared__ int64_t sums[kBins];
  __shared__ uint32_t counts[kBins];
  __shared__ int64_t sh[kWaves], seg_sum[kMaxSegments];
  __shared__ int shi;
  __shared__ Cut cut;
  const int row = blockIdx.x / a.segments, seg = blockIdx.x - row * a.segments, tid = threadIdx.x;
  const float* logits = a.logits + row * a.ld;
  const Params p(a, row);
  const Cell c = row_cell(a, sc, row);
  if (p.bad || c.bad || !(c.hi > -INFINITY) || p.t == 0.f) {  // uniform
    if (seg == 0 && tid == 0) {
      const bool none = c.bad || !(c.hi > -INFINITY);
      if (p.bad)
        flag(a.status, kBadParam);
      else if (none)
        flag(a.status, kNoDist);
      if (a.token) a.token[row] = p.bad || none ? -1 : c.at;
      cut = {};
      cut.mode = a.token ? kDone : (p.bad ? kNan : (none ? kSame : kCut));
      cut.last = c.hi;  // T = 0: the first of the order alone
      cut.last_at = c.at;
      sc.cuts[row] = cut;
    }
    return;
  }
  const Weight wt(p.t, c.hi, a.shift);
  const int from = seg * a.len, to = min(from + a.len, a.v);
  const bool by_count = p.top_k > 0, by_mass = p.top_p < 1.f;
  if (!by_count && !by_mass) {  // uniform: nothing to cut
    if (!a.token) {
      if (seg == 0 && tid == 0) {
        cut = {};
        cut.mode = kAll;
        cut.hi = c.hi;
        sc.cuts[row] = cut;
      }
      return;
    }
    auto weight = [&](float l, int) {
      const float w = wt.w(l);
      return w >= p.min_p ? wt.r(w) : 0;
    };
    int64_t s = 0;
    each_token(logits, from, to, [&](float l, int j) { s += weight(l, j); });
    s = block_sum_i64<kWaves>(s, sh);
    if (tid == 0) publish(&sc.kept[(int64_t)row * a.segments + seg], s);
    if (!last_of_row(&sc.counters[4 * (int64_t)row], a.segments, &shi)) return;
    if (tid < a.segments) seg_sum[tid] = published(&sc.kept[(int64_t)row * a.segments + tid]);
    if (tid == 0) sc.cuts[row].mode = kDone;
    __syncthreads();
    draw(a, row, seg_sum, weight, sh, &shi);
    return;
  }
  sums[tid] = 0;
  counts[tid] = 0;
  __syncthreads();
  const double span = fmin((double)c.hi - (double)c.lo, kSpan * (double)p.t);
  const float scale = span > 0.0 ? (float)((double)kBins / span) : 0.f;
  each_token(logits, from, to, [&](float l, int) {
    const int b = bin_of(c.hi, scale, l);
    if (by_count) atomicAdd(&counts[b], 1u);
    if (by_mass) {
      const int64_t r = wt.r(wt.w(l));
      if (r) atomicAdd((unsigned long long*)&sums[b], (unsigned long long)r);
    }
  });
  __syncthreads();
  const int64_t slice = (int64_t)row * a.segments * kBins;
  if (by_mass) publish(&sc.sums[slice + seg * kBins + tid], sums[tid]);
  if (by_count) publish(&sc.counts[slice + seg * kBins + tid], counts[tid]);
  if (!last_of_row(&sc.counters[4 * (int64_t)row], a.segments, &shi)) return;
  // the row's last workgroup: a thread a bin
  int64_t mass = 0, n = 0;
#pragma unroll 4
  for (int s = 0; s < a.segments; ++s) {
    if (by_mass) mass += published(&sc.sums[slice + s * kBins + tid]);
    if (by_count) n += published(&sc.counts[slice + s * kBins + tid]);
  }
  int64_t all, tokens;
  const int64_t m0 = block_exclusive_scan_i64<kWaves>(mass, sh, all);
  const int64_t n0 = block_exclusive_scan_i64<kWaves>(n, sh, tokens);
  if (tid == 0) {
    cut = {};
    cut.mode = kCut;
    cut.sure = kBins;
    cut.g0 = 1;
    cut.g1 = 0;
    cut.bk = -1;
    cut.before_k = all;
    cut.hi = c.hi;
    cut.scale = scale;
    cut.last = INFINITY;
    cut.last_at = -1;
  }
  __shared__ int64_t upper;  // of the sum of what top-k keeps
  if (tid == 0) upper = all;
  __syncthreads();
  if (by_count && n0 < p.top_k && p.top_k <= n0 + n) {
    cut.sure = tid;
    cut.bk = tid;
    cut.rk = (int)(p.top_k - n0);
    cut.before_k = m0;
    upper = m0 + mass;
    if (cut.rk == n) {  // the whole bin
      cut.sure = tid + 1;
      cut.bk = -1;
      cut.before_k = m0 + mass;
    }
  }
  __syncthreads();
  if (by_mass) {
    const int64_t n_lo = need_of(p.top_p, cut.before_k), n_hi = need_of(p.top_p, upper);
    __syncthreads();
    // top-p's cut lies between the bins where the sums reach the needs of the least and the most that top-k keeps
    if (m0 < n_lo && n_lo <= m0 + mass) {
      cut.g0 = tid;
      cut.sure = tid;
      cut.before = m0;
    }
    if (m0 < n_hi && n_hi <= m0 + mass) cut.g1 = tid;
  }
  __syncthreads();
  if (tid == 0) sc.cuts[row] = cut;
}

// ------------------------------------------------------------------- step 3
// The cuts of a whole row by radix selection, one workgroup.
struct RadixCut {
  float last;
  int last_at;
};

// The key K (descending order) where the running sum of f over keys passes `target` (>= 1): before K it is less, with K's
// own tokens it is not.  `passed`: the sum before K.
template <class F>
__device__ uint32_t radix_key(const float* row, int v, int64_t target, F f, int64_t* hist, int64_t* sh, int* shi,
                              int64_t& passed) {
  uint32_t prefix = 0;
  passed = 0;
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int low = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bits = pass == 2 ? 10 : 11;
    __syncthreads();
    for (int i = threadIdx.x; i < 2048; i += kThreads) hist[i] = 0;
    __syncthreads();
    each_token(row, 0, v, [&](float l, int j) {
      const uint32_t k = key_of(l);
      if (pass > 0 && (k >> (low + bits)) != prefix) return;
      const int64_t x = f(l, j);
      if (x) atomicAdd((unsigned long long*)&hist[(k >> low) & ((1u << bits) - 1)], (unsigned long long)x);
    });
    __syncthreads();
    const int64_t x0 = hist[2 * threadIdx.x], x1 = hist[2 * threadIdx.x + 1];
    int64_t total;
    const int64_t at = passed + block_exclusive_scan_i64<kWaves>(x0 + x1, sh, total);
    __shared__ int64_t found;
    if (at < target && target <= at + x0) {
      *shi = 2 * threadIdx.x;
      found = at;
    } else if (at + x0 < target && target <= at + x0 + x1) {
      *shi = 2 * threadIdx.x + 1;
      found = at + x0;
    }
    __syncthreads();
    prefix = prefix << bits | (uint32_t)*shi;
    passed = found;
  }
  __syncthreads();
  return prefix;
}

__global__ __launch_bounds__(kThreads) void cut_kernel(SampleArgs a, Scratch sc) {
  __shared__ __align__(16) int64_t lr[kMost];  // weights of the gathered tokens; the histogram of a radix pass
  __shared__ float ll[kMost];
  __shared__ int lj[kMost], lkeep[kMost];
  __shared__ int64_t sh[kWaves], seg_sum[kMaxSegments], z1;
  __shared__ int shi, most_at;
  const int row = blockIdx.x / a.segments, seg = blockIdx.x - row * a.segments, tid = threadIdx.x;
  const Cut cut = sc.cuts[row];
  const Params p(a, row);
  if (cut.mode != kCut || p.t == 0.f || p.bad) return;  // uniform
  const float* logits = a.logits + row * a.ld;
  const Weight wt(p.t, cut.hi, a.shift);
  const int from = seg * a.len, to = min(from + a.len, a.v);
  int32_t* gathered = &sc.counters[4 * (int64_t)row + 2];
  int64_t s = 0;
  each_token(logits, from, to, [&](float l, int j) {
    const int b = bin_of(cut.hi, cut.scale, l);
    if (b < cut.sure) {
      if (a.token) {
        const float w = wt.w(l);
        s += w >= p.min_p ? wt.r(w) : 0;
      }
    } else if (b == cut.bk || (b >= cut.g0 && b <= cut.g1)) {
      const int at = __hip_atomic_fetch_add(gathered, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (at < kMost)
        publish(&sc.list[(int64_t)row * kMost + at], (int64_t)j << 32 | __builtin_bit_cast(uint32_t, l));
    }
  });
  s = block_sum_i64<kWaves>(s, sh);
  if (tid == 0) publish(&sc.kept[(int64_t)row * a.segments + seg], s);
  if (!last_of_row(&sc.counters[4 * (int64_t)row + 1], a.segments, &shi)) return;
  if (tid < a.segments) seg_sum[tid] = published(&sc.kept[(int64_t)row * a.segments + tid]);
  const int n = __hip_atomic_load(gathered, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const bool by_mass = p.top_p < 1.f;
  float last = INFINITY;
  int last_at = -1;
  int sure = cut.sure;
  if (n <= kMost) {  // uniform: rank them
    for (int i = tid; i < n; i += kThreads) {
      const int64_t x = published(&sc.list[(int64_t)row * kMost + i]);
      ll[i] = __builtin_bit_cast(float, (uint32_t)x);
      lj[i] = (int)(x >> 32);
      lr[i] = wt.r(wt.w(ll[i]));
    }
    __syncthreads();
    auto ahead = [&](int i, int j) { return i != j && up_to(ll[j], lj[j], ll[i], lj[i]); };
    auto bin = [&](int i) { return bin_of(cut.hi, cut.scale, ll[i]); };
    // top-k: what it keeps of its bin, and their weights
    int64_t part = 0;
    for (int i = tid; i < n; i += kThreads) {
      int keep = 1;
      if (cut.bk >= 0 && bin(i) == cut.bk) {
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += bin(j) == cut.bk && ahead(i, j) ? 1 : 0;
        keep = rank < cut.rk;
        if (keep) part += lr[i];
      }
      lkeep[i] = keep;
    }
    part = block_sum_i64<kWaves>(part, sh);
    if (tid == 0) z1 = cut.before_k + part;
    __syncthreads();
    if (by_mass) {
      const int64_t need = need_of(p.top_p, z1);
      bool in[kMost / kThreads];
#pragma unroll
      for (int x = 0; x < kMost / kThreads; ++x) {
        const int i = tid + x * kThreads;
        in[x] = false;
        if (i >= n || !lkeep[i] || bin(i) > cut.g1) continue;
        int64_t before = cut.before;
        for (int j = 0; j < n; ++j) before += lkeep[j] && ahead(i, j) ? lr[j] : 0;
        in[x] = before < need;
      }
      __syncthreads();
#pragma unroll
      for (int x = 0; x < kMost / kThreads; ++x)
        if (tid + x * kThreads < n) lkeep[tid + x * kThreads] = in[x];
    }
    __syncthreads();
    // the last one kept, and the kept weights by segment
    if (tid == 0) most_at = -1;
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
      if (!lkeep[i]) continue;
      bool final = true;
      for (int j = 0; j < n; ++j) final = final && !(lkeep[j] && ahead(j, i));
      if (final) most_at = i;
      const float w = wt.w(ll[i]);
      if (w >= p.min_p) atomicAdd((unsigned long long*)&seg_sum[lj[i] / a.len], (unsigned long long)lr[i]);
    }
    __syncthreads();
    if (most_at >= 0) {
      last = ll[most_at];
      last_at = lj[most_at];
    }
  } else {
    // too many to rank: the cuts from the whole row
    sure = 0;
    int64_t passed;
    uint32_t key = 0xFFFFFFFFu;
    int at = INT_MAX;
    if (p.top_k > 0) {
      key = radix_key(logits, a.v, p.top_k, [](float, int) { return (int64_t)1; }, lr, sh, &shi, passed);
      at = locate(logits, 0, a.v, p.top_k - passed - 1, [&](float l, int) { return (int64_t)(key_of(l) == key); }, sh, &shi);
    }
    auto by_k = [&](float l, int j) { return key_of(l) < key || (key_of(l) == key && j <= at); };
    if (by_mass) {
      auto weight = [&](float l, int j) { return by_k(l, j) ? wt.r(wt.w(l)) : 0; };
      int64_t z = 0;
      each_token(logits, 0, a.v, [&](float l, int j) { z += weight(l, j); });
      z = block_sum_i64<kWaves>(z, sh);
      const int64_t need = need_of(p.top_p, z);
      const uint32_t kp = radix_key(logits, a.v, need, weight, lr, sh, &shi, passed);
      // tokens of one key weigh the same: the sum passes need with the first of them at which (running sum) >= need
      at = locate(logits, 0, a.v, need - passed - 1,
                  [&](float l, int j) { return key_of(l) == kp ? weight(l, j) : 0; }, sh, &shi);
      key = kp;
    }
    last = __builtin_bit_cast(float, (key >> 31) ? key : ~(key | 0x80000000u));
    last_at = at;
  }
  if (!a.token) {
    if (tid == 0) {
      sc.cuts[row].sure = sure;
      sc.cuts[row].last = last;
      sc.cuts[row].last_at = last_at;
    }
    return;
  }
  auto weight = [&](float l, int j) -> int64_t {
    if (!(bin_of(cut.hi, cut.scale, l) < sure || up_to(l, j, last, last_at))) return 0;
    const float w = wt.w(l);
    return w >= p.min_p ? wt.r(w) : 0;
  };
  if (n > kMost) {  // the segments' sums anew
    for (int g = 0; g < a.segments; ++g) {
      int64_t z = 0;
      each_token(logits, g * a.len, min((g + 1) * a.len, a.v), [&](float l, int j) { z += weight(l, j); });
      z = block_sum_i64<kWaves>(z, sh);
      if (tid == 0) seg_sum[g] = z;
    }
    __syncthreads();
  }
  draw(a, row, seg_sum, weight, sh, &shi);
}

// ------------------------------------------------------------------- step 4
__global__ __launch_bounds__(kThreads) void filter_kernel(SampleArgs a, Scratch sc) {
  const int row = blockIdx.x / a.segments, seg = blockIdx.x - row * a.segments;
  const Cut cut = sc.cuts[row];
  const Params p(a, row);
  const int from = seg * a.len, to = min(from + a.len, a.v);
  float* out = a.out + row * a.ld;
  const bool greedy = p.t == 0.f;
  const Weight wt(greedy ? 1.f : p.t, cut.hi, a.shift);
  each_token(a.logits + row * a.ld, from, to, [&](float l, int j) {
    bool keep = true;
    if (cut.mode == kCut) keep = greedy ? j == cut.last_at
                                        : bin_of(cut.hi, cut.scale, l) < cut.sure || up_to(l, j, cut.last, cut.last_at);
    if ((cut.mode == kCut || cut.mode == kAll) && !greedy && keep && p.min_p > 0.f) keep = wt.w(l) >= p.min_p;
    out[j] = cut.mode == kNan ? __builtin_nanf("") : (keep ? l : -INFINITY);
  });
}

constexpr int kRowsAtOnce = 1024;  // rows whose scratch is held at once

size_t rounded(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

hipError_t launch_sample(const float* logits, int m, int v, int64_t ld, const float* temperature, const int32_t* top_k,
                         const float* top_p, const float* min_p, const uint32_t* u24, int32_t* token, float* out,
                         int32_t* status, hipStream_t stream) {
  const int rows = m < kRowsAtOnce ? m : kRowsAtOnce;
  SampleArgs a{logits, v, ld, temperature, top_p, min_p, top_k, u24, token, out, status, 1, v, 62};
  while (a.shift > 0 && (int64_t(1) << (62 - a.shift)) < v) --a.shift;
  // segments: a workgroup a CU over all rows, none shorter than pays
  int segments = (cu_count() + rows - 1) / rows;
  const int most = (v + kMinSegment - 1) / kMinSegment;
  segments = segments > kMaxSegments ? kMaxSegments : segments;
  a.segments = segments > most ? most : segments;
  a.len = (v + a.segments - 1) / a.segments;
  a.segments = (v + a.len - 1) / a.len;
  const size_t rs = (size_t)rows * a.segments;
  const size_t bytes[] = {rs * sizeof(Cell),      rs * kBins * 8,         rs * 8,          rs * kBins * 8,
                          (size_t)rows * kMost * 8, (size_t)rows * sizeof(Cut), (size_t)rows * 16};
  size_t total = 0;
  for (size_t n : bytes) total += rounded(n);
  void* ws = nullptr;
  const hipError_t e = workspace(total, stream, &ws);
  if (e != hipSuccess) return e;
  char* at = static_cast<char*>(ws);
  auto take = [&](int i) {
    char* p = at;
    at += rounded(bytes[i]);
    return p;
  };
  Scratch sc;
  sc.cells = reinterpret_cast<Cell*>(take(0));
  sc.sums = reinterpret_cast<int64_t*>(take(1));
  sc.kept = reinterpret_cast<int64_t*>(take(2));
  sc.counts = reinterpret_cast<int64_t*>(take(3));
  sc.list = reinterpret_cast<int64_t*>(take(4));
  sc.cuts = reinterpret_cast<Cut*>(take(5));
  sc.counters = reinterpret_cast<int32_t*>(take(6));
  for (int r0 = 0; r0 < m; r0 += rows) {
    const int n = m - r0 < rows ? m - r0 : rows;
    SampleArgs b = a;
    b.logits += r0 * ld;
    if (b.temperature) b.temperature += r0;
    if (b.top_k) b.top_k += r0;
    if (b.top_p) b.top_p += r0;
    if (b.min_p) b.min_p += r0;
    if (b.u24) b.u24 += r0;
    if (b.token) b.token += r0;
    if (b.out) b.out += r0 * ld;
    const dim3 grid((unsigned)(n * a.segments)), block(kThreads);
    hipLaunchKernelGGL(range_kernel, grid, block, 0, stream, b, sc);
    hipLaunchKernelGGL(bins_kernel, grid, block, 0, stream, b, sc);
    if (top_k || top_p) hipLaunchKernelGGL(cut_kernel, grid, block, 0, stream, b, sc);
    if (out) hipLaunchKernelGGL(filter_kernel, grid, block, 0, stream, b, sc);
  }
  return hipGetLastError();
}

}  // namespace sq

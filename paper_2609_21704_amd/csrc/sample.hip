// Sampling and filtering of vocabulary rows: temperature, top-k, top-p, min-p (include/specquant_sample.h has the
// definition).  No row is sorted: top-k and top-p keep a prefix of the order (logit descending, index ascending), so each
// is a cut through it, and the last kept token (logit, index) says which are kept.
//   1. range_kernel   per (row, segment) the largest and smallest logit
//   2. bins_kernel    per (row, segment) the weights' sums and counts in 1024 bins of the distance from the maximum;
//                     the row's last workgroup finds the bins that the cuts go through
//   3. cut_kernel     gathers the tokens of those bins and sums the weights that are kept for sure; the row's last
//                     workgroup finds the cuts among the gathered tokens (1024 bins of the bin, then ranks) and draws
//   4. filter_kernel  writes the kept logits
// A row without top-k and top-p is drawn from by step 2.  Where the bins of the cuts hold too many tokens (ties, rows
// whose logits lie close together but for a few, rows with fewer finite logits than top-k keeps, whose cut goes through the
// -inf ones), the last workgroup finds the cuts by a radix selection over the row (11 bits of the logit's key a pass): 5
// finite logits of 151936 under top-k 50 take 475 us a row and 502 for 64 rows, ordinary rows 23 and 42.
// Weights are whole numbers, so their sums do not depend on any order.  Rows are cut into segments so that a call fills
// the chip from one row on, and a segment into runs, one a wavefront, whose sums say where a draw has to look.  Last
// workgroups are found by counting arrivals (counters that step 1 clears).
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
constexpr int kHeld = 2;          // gathered tokens a thread holds
constexpr int kMost = kHeld * kThreads;
constexpr int kFew = 512;         // tokens that are ranked against each other
constexpr int kDirect = 96;       // gathered ones that are, without bins of theirs
constexpr int kMaxSegments = 32;  // of a row
constexpr int kMaxRuns = kMaxSegments * kWaves;
constexpr int kMinSegment = 4096; // tokens
constexpr int kLongSegment = 16384;
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
  int segments, run;  // of a row, of kWaves runs each; tokens of a run, a multiple of four
  bool aligned;       // rows start on 16 bytes and are a multiple of them long
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
  int64_t* sums;     // [m][segments][kBins]
  int64_t* kept;     // [m][segments * kWaves]: of the runs
  int32_t* counts;   // [m][segments][kBins]
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

// The weight of a logit, and on the grid: exp((l - hi) / T) = 2^y with y = (l - hi) log2(e) / T in fp64, split into a whole
// number and |f| <= 1/2; 2^f = 1 + f Q(f), Q of degree 7 by Remez exchange on the relative error (2^-39.8), which is exactly 1
// at the maximum; one rounding to fp32, off by 2^-15 of half a step more than the nearest.
struct Weight {
  double hi, c, q[8], magic;
  int shift;
  __device__ __forceinline__ Weight(float t, float hi, int shift)
      : hi(hi),
        c(0x1.71547652b82fep+0 / (double)t),
        q{0x1.63d13637ddc42p-20, 0x1.00dc4a532dcb6p-16, 0x1.4308ac85a9890p-13, 0x1.5d8745a728475p-10,
          0x1.3b2ab7181b75cp-7,  0x1.c6b08dd6fd234p-5,  0x1.ebfbdff823cedp-3,  0x1.62e42fef84cf0p-1},
        magic(0x1.8p52),
        shift(shift) {
#pragma unroll
    for (int i = 0; i < 8; ++i) asm("" : "+v"(q[i]));
  }
  // A weight as the fp32 of 2^f and its power of two.
  struct Value {
    float m;
    int n;
  };
  __device__ __forceinline__ Value operator()(float l) const {
    const double y = fmax(((double)l - hi) * c, -2000.0);  // (-inf too)
    const double k = y + magic;  // rint(y) in the low mantissa bits
    const double f = y - (k - magic);
    double p = q[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) p = __builtin_fma(p, f, q[i]);
    p = __builtin_fma(p, f, 1.0);
    return {(float)p, (int)(uint32_t)__builtin_bit_cast(uint64_t, k)};
  }
  static __device__ __forceinline__ float fp32(Value v) { return ldexpf(v.m, v.n); }
  // rint(w 2^shift), ties to even: what the sum with 2^52 holds in its mantissa (shift <= 51)
  __device__ __forceinline__ int64_t grid(Value v) const {
    const double x = ldexp((double)v.m, v.n + shift) + 0x1p52;
    return __builtin_bit_cast(int64_t, x) - 0x4330000000000000;
  }
  // the same of a token that min_p keeps, 0 for the others
  __device__ __forceinline__ int64_t kept(float l, float min_p) const {
    const Value v = (*this)(l);
    return fp32(v) >= min_p ? grid(v) : 0;
  }
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

// f(l, j) for the tokens from .. to (from a multiple of four), four consecutive ones a load: of the fours a wavefront (stride
// 64) or the workgroup takes every stride-th, the next two on their way while one is worked on (in registers of their own:
// handed on from one to the next they would be waited for).
template <class F>
__device__ __forceinline__ void each_token(const SampleArgs& a, const float* row, int from, int to, int first, int stride,
                                           F f) {
  if (from >= to) return;
  const int q1 = (to + 3) >> 2;
  auto load = [&](int q) {
    float4_t v;
    if (a.aligned) {  // uniform; (rows are a multiple of four long, so the last load lies in its row)
      v = reinterpret_cast<const float4_t*>(row)[min(q, q1 - 1)];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = row[min(4 * q + i, to - 1)];
    }
    return v;
  };
  auto use = [&](float4_t v, int q) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f(v[i], 4 * q + i);
  };
  int base = from >> 2;
  float4_t x = load(base + first), y = load(base + stride + first);
#pragma unroll 1
  for (; base + 2 * stride <= to >> 2; base += 2 * stride) {  // uniform: all lanes' fours are whole
    use(x, base + first);
    x = load(base + 2 * stride + first);
    use(y, base + stride + first);
    y = load(base + 3 * stride + first);
  }
#pragma unroll 1
  for (int e = 0; e < 2; ++e) {  // the rest
    const int j = 4 * (base + e * stride + first);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (j + i < to) f(e ? y[i] : x[i], j + i);
  }
}
// ... of this wavefront's run of a segment
template <class F>
__device__ __forceinline__ void each_of_run(const SampleArgs& a, const float* row, int run, F f) {
  const int from = (int)min((int64_t)run * a.run, (int64_t)a.v), to = (int)min((int64_t)from + a.run, (int64_t)a.v);
  each_token(a, row, from, to, threadIdx.x & 63, kWave, f);
}
// ... and of the whole row
template <class F>
__device__ __forceinline__ void each_of_row(const SampleArgs& a, const float* row, F f) {
  each_token(a, row, 0, a.v, threadIdx.x, kThreads, f);
}

// Exclusive prefix sum over the workgroup in thread order, and the workgroup's sum: as the acceptance's, but the wavefronts'
// sums are scanned over the lanes, in a third of the code.
__device__ __forceinline__ int64_t lane_of(int64_t v, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((int)v, lane), hi = __builtin_amdgcn_readlane((int)(v >> 32), lane);
  return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ int64_t scan(int64_t v, int64_t* sh, int64_t& total) {
  static_assert(kWaves == 16, "a row of lanes");
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t x = wave_scan_i64(v);
  if (lane == 63) sh[w] = x;
  __syncthreads();
  int64_t y = sh[lane & 15];
  y += dpp_move<0x111>(y);  // row_shr:1
  y += dpp_move<0x112>(y);
  y += dpp_move<0x114>(y);
  y += dpp_move<0x118>(y);
  __syncthreads();
  total = lane_of(y, 15);
  return x - v + (w ? lane_of(y, w - 1) : 0);
}
__device__ __forceinline__ int64_t sum_of(int64_t v, int64_t* sh) {
  int64_t total;
  scan(v, sh, total);
  return total;
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
__device__ __forceinline__ Cell merge(Cell x, Cell y) {
  const bool other = y.hi > x.hi || (y.hi == x.hi && y.at < x.at);
  return Cell{other ? y.hi : x.hi, fminf(x.lo, y.lo), other ? y.at : x.at, x.bad | y.bad};
}
template <int kLanes>
__device__ __forceinline__ Cell merge_lanes(Cell c) {
#pragma unroll
  for (int d = kLanes / 2; d >= 1; d >>= 1)
    c = merge(c, Cell{__shfl_xor(c.hi, d), __shfl_xor(c.lo, d), __shfl_xor(c.at, d), __shfl_xor(c.bad, d)});
  return c;
}

__global__ __launch_bounds__(kThreads) void range_kernel(SampleArgs a, Scratch sc) {
  __shared__ Cell sh[kWaves];
  const int row = blockIdx.x / a.segments, seg = blockIdx.x - row * a.segments, w = threadIdx.x >> 6;
  if (seg == 0 && threadIdx.x < 4) sc.counters[4 * (int64_t)row + threadIdx.x] = 0;
  Cell c = {-INFINITY, INFINITY, INT_MAX, 0};
  each_of_run(a, a.logits + row * a.ld, seg * kWaves + w, [&](float l, int j) {
    c.bad |= isnan(l) || l == INFINITY ? 1 : 0;
    if (l > c.hi) {
      c.hi = l;
      c.at = j;
    }
    if (l > -INFINITY) c.lo = fminf(c.lo, l);
  });
  c = merge_lanes<kWave>(c);
  if ((threadIdx.x & 63) == 0) sh[w] = c;
  __syncthreads();
  if (threadIdx.x < kWaves) {
    c = merge_lanes<kWaves>(sh[threadIdx.x]);
    if (threadIdx.x == 0) sc.cells[(int64_t)row * a.segments + seg] = c;
  }
}

// Of the whole row, by every wavefront for itself.
__device__ __forceinline__ Cell row_cell(const SampleArgs& a, const Scratch& sc, int row) {
  const int s = min((int)threadIdx.x & (kMaxSegments - 1), a.segments - 1);
  return merge_lanes<kMaxSegments>(sc.cells[(int64_t)row * a.segments + s]);
}

// ------------------------------------------------------------------ drawing
// The smallest j in [from, to) at which base + the running sum of f(l, j) exceeds t (base <= t < base + the sum).
template <class F>
__device__ __forceinline__ int locate_in(const float* row, int from, int to, int64_t base, int64_t t, F f, int64_t* sh,
                                         int* shi) {
  const int per = (to - from + kThreads - 1) / kThreads;  // consecutive tokens of a thread
  const int p0 = from + min((int)threadIdx.x * per, to - from), p1 = min(p0 + per, to);
  int64_t part = 0;
  for (int j = p0; j < p1; ++j) part += f(row[j], j);
  int64_t total;
  int64_t at = base + scan(part, sh, total);
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

// The same over a row whose runs' sums are in LDS.
template <class F>
__device__ __forceinline__ int locate(const SampleArgs& a, const float* row, const int64_t* runs, int64_t t, F f, int64_t* sh,
                                      int* shi) {
  __shared__ int64_t base;
  const int n = a.segments * kWaves;  // at most a thread each
  const int64_t mine = (int)threadIdx.x < n ? runs[threadIdx.x] : 0;
  int64_t total;
  const int64_t at = scan(mine, sh, total);
  if (mine > 0 && at <= t && t < at + mine) {
    *shi = threadIdx.x;
    base = at;
  }
  __syncthreads();
  const int from = (int)min((int64_t)*shi * a.run, (int64_t)a.v), to = (int)min((int64_t)from + a.run, (int64_t)a.v);
  const int64_t b = base;
  __syncthreads();
  return locate_in(row, from, to, b, t, f, sh, shi);
}

// Sums of f over the runs, to LDS; the wavefronts take them in turn.
template <class F>
__device__ __forceinline__ void sum_runs(const SampleArgs& a, const float* row, int64_t* runs, F f) {
  __syncthreads();
  for (int r = threadIdx.x >> 6; r < a.segments * kWaves; r += kWaves) {
    int64_t s = 0;
    each_of_run(a, row, r, [&](float l, int j) { s += f(l, j); });
    s = wave_sum_i64(s);
    if ((threadIdx.x & 63) == 0) runs[r] = s;
  }
  __syncthreads();
}

__device__ __forceinline__ int64_t draw_at(uint32_t u24, int64_t z) {  // floor(u z / 2^24)
  const int64_t u = u24 & 0xFFFFFF;
  return u * (z >> 24) + ((u * (z & 0xFFFFFF)) >> 24);
}

// A token of a row with the runs' sums in LDS and the weight f of a kept token.
template <class F>
__device__ __forceinline__ void draw(const SampleArgs& a, int row, const int64_t* runs, F f, int64_t* sh, int* shi) {
  const uint32_t u = a.u24[row];
  const int64_t z = sum_of((int)threadIdx.x < a.segments * kWaves ? runs[threadIdx.x] : 0, sh);
  const int j = locate(a, a.logits + row * a.ld, runs, draw_at(u, z), f, sh, shi);
  if (threadIdx.x == 0) a.token[row] = j;
}

// ------------------------------------------------------------------- step 2
__device__ __forceinline__ int64_t need_of(float top_p, int64_t z) {
  const int64_t n = (int64_t)ceil((double)top_p * (double)z);
  return n < 1 ? 1 : n;
}

// The sum of part(s) over the segments, sixteen loads in flight.
template <class F>
__device__ __forceinline__ int64_t slices(int segments, F part) {
  int64_t sum = 0;
  for (int s0 = 0; s0 < segments; s0 += 16) {
    int64_t x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = part(min(s0 + i, segments - 1));
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += s0 + i < segments ? x[i] : 0;
  }
  return sum;
}

// (eight wavefronts a SIMD, two workgroups a CU: 27.6 us for 34.7 at 64 rows of 151936 logits)
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(8, 8))) void bins_kernel(SampleArgs a, Scratch sc) {
  __shared__ int64_t sums[kBins];
  __shared__ uint32_t counts[kBins];
  __shared__ int64_t sh[kWaves], runs[kMaxRuns];
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
    auto weight = [&](float l, int) { return wt.kept(l, p.min_p); };
    int64_t s = 0;
    each_of_run(a, logits, seg * kWaves + (tid >> 6), [&](float l, int j) { s += weight(l, j); });
    s = wave_sum_i64(s);
    int64_t* kept = sc.kept + (int64_t)row * a.segments * kWaves;
    if ((tid & 63) == 0) publish(&kept[seg * kWaves + (tid >> 6)], s);
    if (!last_of_row(&sc.counters[4 * (int64_t)row], a.segments, &shi)) return;
    if (tid < a.segments * kWaves) runs[tid] = published(&kept[tid]);
    if (tid == 0) sc.cuts[row].mode = kDone;
    __syncthreads();
    draw(a, row, runs, weight, sh, &shi);
    return;
  }
  sums[tid] = 0;
  counts[tid] = 0;
  __syncthreads();
  const double span = fmin((double)c.hi - (double)c.lo, kSpan * (double)p.t);
  const float scale = span > 0.0 ? (float)((double)kBins / span) : 0.f;
  each_of_run(a, logits, seg * kWaves + (tid >> 6), [&](float l, int) {
    const int b = bin_of(c.hi, scale, l);
    if (by_count) atomicAdd(&counts[b], 1u);
    if (by_mass) {
      atomicAdd((unsigned long long*)&sums[b], (unsigned long long)wt.grid(wt(l)));
    }
  });
  __syncthreads();
  const int64_t slice = (int64_t)row * a.segments * kBins;
  if (by_mass) publish(&sc.sums[slice + seg * kBins + tid], sums[tid]);
  if (by_count)
    __hip_atomic_store(&sc.counts[slice + seg * kBins + tid], (int32_t)counts[tid], __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
  if (!last_of_row(&sc.counters[4 * (int64_t)row], a.segments, &shi)) return;
  // the row's last workgroup: a thread a bin
  int64_t mass = 0, n = 0;
  if (by_mass) {
    mass = slices(a.segments, [&](int s) { return published(&sc.sums[slice + s * kBins + tid]); });
  }
  if (by_count) {
    n = slices(a.segments, [&](int s) -> int64_t {
      return __hip_atomic_load(&sc.counts[slice + s * kBins + tid], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    });
  }
  int64_t all, tokens;
  const int64_t m0 = scan(mass, sh, all);
  const int64_t n0 = scan(n, sh, tokens);
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
// The key K (descending order) where the running sum of f over keys passes `target` (>= 1): before K it is less, with K's
// own tokens it is not.  `passed`: the sum before K.
template <class F>
__device__ uint32_t radix_key(const SampleArgs& a, const float* row, int64_t target, F f, int64_t* hist, int64_t* sh, int* shi,
                              int64_t& passed) {
  uint32_t prefix = 0;
  passed = 0;
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int low = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bits = pass == 2 ? 10 : 11;
    __syncthreads();
    for (int i = threadIdx.x; i < 2048; i += kThreads) hist[i] = 0;
    __syncthreads();
    each_of_row(a, row, [&](float l, int j) {
      const uint32_t k = key_of(l);
      if (pass > 0 && (k >> (low + bits)) != prefix) return;
      const int64_t x = f(l, j);
      if (x) atomicAdd((unsigned long long*)&hist[(k >> low) & ((1u << bits) - 1)], (unsigned long long)x);
    });
    __syncthreads();
    const int64_t x0 = hist[2 * threadIdx.x], x1 = hist[2 * threadIdx.x + 1];
    int64_t total;
    const int64_t at = passed + scan(x0 + x1, sh, total);
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

// The token of those that the threads hold at which base + the running sum of val, in the order, reaches `target`: their
// bins (-1: not in question) are a monotone function of the order, so the sum is followed through the bins and then through
// the tokens of one.  False where those are too many.
struct Picked {
  int64_t val[kFew], sum;
  float l[kFew], last;
  int j[kFew], bin, n, at;
};
__device__ __forceinline__ bool pick(const float (&l)[kHeld], const int (&j)[kHeld], const int (&bin)[kHeld],
                                     const int64_t (&val)[kHeld], int held, int64_t base, int64_t target, int64_t* hist,
                                     int64_t* sh, Picked& p) {
  const int tid = threadIdx.x;
  __syncthreads();
  const bool few = held <= kDirect;  // uniform: all of them are ranked
  if (!few) hist[tid] = 0;
  if (tid == 0) {
    p.n = 0;
    p.sum = base;
  }
  __syncthreads();
  if (!few) {
#pragma unroll
    for (int e = 0; e < kHeld; ++e)
      if (bin[e] >= 0) atomicAdd((unsigned long long*)&hist[bin[e]], (unsigned long long)val[e]);
    __syncthreads();
    const int64_t h = hist[tid];
    int64_t total;
    const int64_t at = base + scan(h, sh, total);
    if (at < target && target <= at + h) {
      p.bin = tid;
      p.sum = at;
    }
    __syncthreads();
  }
#pragma unroll
  for (int e = 0; e < kHeld; ++e) {
    if (few ? bin[e] < 0 : bin[e] != p.bin) continue;
    const int slot = atomicAdd(&p.n, 1);
    if (slot < kFew) {
      p.l[slot] = l[e];
      p.j[slot] = j[e];
      p.val[slot] = val[e];
    }
  }
  __syncthreads();
  const int n = p.n;
  if (n > kFew) return false;  // uniform
  // A wavefront a token, a lane one of those before it: a thread a token goes through all of them one LDS read after the
  // other (64 rows of 32000: 46 us for this 36).
  for (int t = tid >> 6; t < n; t += kWaves) {
    const float mine = p.l[t];
    const int my_j = p.j[t];
    int64_t before = 0;
    for (int i = tid & 63; i < n; i += 64) {
      const float other = p.l[i];
      const int64_t x = p.val[i];
      const bool up = (int)(other > mine) | ((int)(other == mine) & (int)(p.j[i] < my_j));
      before += up ? x : 0;
    }
    before = p.sum + wave_sum_i64(before);
    if ((tid & 63) == 0 && before < target && target <= before + p.val[t]) {
      p.last = mine;
      p.at = my_j;
    }
  }
  __syncthreads();
  return true;
}

__global__ __launch_bounds__(kThreads) void cut_kernel(SampleArgs a, Scratch sc) {
  __shared__ __align__(16) int64_t list[kMost];  // gathered by this workgroup; then histograms
  __shared__ Picked pk;
  __shared__ int64_t sh[kWaves], runs[kMaxRuns];
  __shared__ int shi, found;
  const int row = blockIdx.x / a.segments, seg = blockIdx.x - row * a.segments, tid = threadIdx.x;
  const Cut cut = sc.cuts[row];
  const Params p(a, row);
  if (cut.mode != kCut || p.t == 0.f || p.bad) return;  // uniform
  const float* logits = a.logits + row * a.ld;
  const Weight wt(p.t, cut.hi, a.shift);
  if (tid == 0) found = 0;
  __syncthreads();
  int64_t s = 0;
  each_of_run(a, logits, seg * kWaves + (tid >> 6), [&](float l, int j) {
    const int b = bin_of(cut.hi, cut.scale, l);
    if (b < cut.sure) {
      if (a.token) s += wt.kept(l, p.min_p);
    } else if (b == cut.bk || (b >= cut.g0 && b <= cut.g1)) {
      const int at = atomicAdd(&found, 1);
      if (at < kMost) list[at] = (int64_t)j << 32 | __builtin_bit_cast(uint32_t, l);
    }
  });
  s = wave_sum_i64(s);
  int64_t* kept = sc.kept + (int64_t)row * a.segments * kWaves;
  if ((tid & 63) == 0) publish(&kept[seg * kWaves + (tid >> 6)], s);
  __syncthreads();
  int32_t* gathered = &sc.counters[4 * (int64_t)row + 2];
  const int mine = found;
  if (tid == 0 && mine > 0) shi = __hip_atomic_fetch_add(gathered, mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  for (int i = tid; i < mine && shi + i < kMost; i += kThreads) publish(&sc.list[(int64_t)row * kMost + shi + i], list[i]);
  __syncthreads();
  if (!last_of_row(&sc.counters[4 * (int64_t)row + 1], a.segments, &shi)) return;
  if (tid < a.segments * kWaves) runs[tid] = published(&kept[tid]);
  const int n = __hip_atomic_load(gathered, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const bool by_mass = p.top_p < 1.f;
  float last = INFINITY;  // the last kept token; of the bins below `sure` alone where none of the gathered ones is
  int last_at = -1;
  bool settled = n <= kMost;
  if (settled) {
    float l[kHeld];
    int j[kHeld], b[kHeld], bin[kHeld];
    int64_t r[kHeld], val[kHeld];
#pragma unroll
    for (int e = 0; e < kHeld; ++e) {
      const int i = tid + e * kThreads;
      b[e] = -1;
      l[e] = -INFINITY;
      j[e] = 0;
      r[e] = 0;
      if (i < n) {
        const int64_t x = published(&sc.list[(int64_t)row * kMost + i]);
        l[e] = __builtin_bit_cast(float, (uint32_t)x);
        j[e] = (int)(x >> 32);
        b[e] = bin_of(cut.hi, cut.scale, l[e]);
        r[e] = wt.grid(wt(l[e]));
      }
    }
    // the place of a token in its bin, in kBins steps
    auto place = [&](int e) {
      const float x = ((cut.hi - l[e]) * cut.scale - (float)b[e]) * (float)kBins;
      return (int)fminf(fmaxf(x, 0.f), (float)(kBins - 1));
    };
    if (cut.bk >= 0) {
#pragma unroll
      for (int e = 0; e < kHeld; ++e) {
        bin[e] = b[e] == cut.bk ? place(e) : -1;
        val[e] = 1;
      }
      settled = pick(l, j, bin, val, n, 0, cut.rk, list, sh, pk);
      if (settled) {
        last = pk.last;
        last_at = pk.at;
      }
    }
    if (settled && by_mass) {
      int64_t part = 0;
#pragma unroll
      for (int e = 0; e < kHeld; ++e) {
        if (cut.bk >= 0 && b[e] == cut.bk) {
          if (up_to(l[e], j[e], last, last_at))
            part += r[e];
          else
            b[e] = -1;  // dropped by top-k
        }
      }
      part = sum_of(part, sh);
      const int64_t need = need_of(p.top_p, cut.before_k + part);
      // its bin, where it may be one of several: the sums of the gathered bins
      int at_bin = cut.g0;
      int64_t base = cut.before;
      if (cut.g1 > cut.g0) {
        list[tid] = 0;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kHeld; ++e)
          if (b[e] >= cut.g0 && b[e] <= cut.g1) atomicAdd((unsigned long long*)&list[b[e]], (unsigned long long)r[e]);
        __syncthreads();
        const int64_t h = list[tid];
        int64_t total;
        const int64_t at = base + scan(h, sh, total);
        if (at < need && need <= at + h) {
          shi = tid;
          pk.sum = at;
        }
        __syncthreads();
        at_bin = shi;
        base = pk.sum;
      }
#pragma unroll
      for (int e = 0; e < kHeld; ++e) bin[e] = b[e] == at_bin ? place(e) : -1;
      settled = pick(l, j, bin, r, n, base, need, list, sh, pk);
      if (settled) {
        last = pk.last;
        last_at = pk.at;
      }
    }
    if (settled && a.token) {  // the kept ones' weights to their runs
      __syncthreads();
#pragma unroll
      for (int e = 0; e < kHeld; ++e) {
        if (tid + e * kThreads < n && up_to(l[e], j[e], last, last_at) && wt.fp32(wt(l[e])) >= p.min_p)
          atomicAdd((unsigned long long*)&runs[j[e] / a.run], (unsigned long long)r[e]);
      }
      __syncthreads();
    }
  }
  int sure = cut.sure;
  if (!settled) {  // uniform: the cuts from the whole row
    sure = 0;
    int64_t passed;
    uint32_t key = 0xFFFFFFFFu;
    int at = INT_MAX;
    if (p.top_k > 0) {
      key = radix_key(a, logits, p.top_k, [](float, int) { return (int64_t)1; }, list, sh, &shi, passed);
      auto tie = [&](float l, int) { return (int64_t)(key_of(l) == key); };
      sum_runs(a, logits, runs, tie);
      at = locate(a, logits, runs, p.top_k - passed - 1, tie, sh, &shi);
    }
    if (by_mass) {
      auto weight = [&](float l, int j) -> int64_t {
        const uint32_t k = key_of(l);
        return k < key || (k == key && j <= at) ? wt.grid(wt(l)) : 0;
      };
      int64_t z = 0;
      each_of_row(a, logits, [&](float l, int j) { z += weight(l, j); });
      z = sum_of(z, sh);
      const int64_t need = need_of(p.top_p, z);
      const uint32_t kp = radix_key(a, logits, need, weight, list, sh, &shi, passed);
      auto tie = [&](float l, int j) { return key_of(l) == kp ? weight(l, j) : 0; };
      sum_runs(a, logits, runs, tie);
      at = locate(a, logits, runs, need - passed - 1, tie, sh, &shi);
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
    return wt.kept(l, p.min_p);
  };
  if (!settled) sum_runs(a, logits, runs, weight);
  draw(a, row, runs, weight, sh, &shi);
}

// ------------------------------------------------------------------- step 4
__global__ __launch_bounds__(kThreads) void filter_kernel(SampleArgs a, Scratch sc) {
  const int row = blockIdx.x / a.segments, seg = blockIdx.x - row * a.segments;
  const Cut cut = sc.cuts[row];
  const Params p(a, row);
  float* out = a.out + row * a.ld;
  const bool greedy = p.t == 0.f;
  const Weight wt(greedy ? 1.f : p.t, cut.hi, a.shift);
  each_of_run(a, a.logits + row * a.ld, seg * kWaves + (threadIdx.x >> 6), [&](float l, int j) {
    bool keep = true;
    if (cut.mode == kCut) keep = greedy ? j == cut.last_at
                                        : bin_of(cut.hi, cut.scale, l) < cut.sure || up_to(l, j, cut.last, cut.last_at);
    if ((cut.mode == kCut || cut.mode == kAll) && !greedy && keep && p.min_p > 0.f) keep = wt.fp32(wt(l)) >= p.min_p;
    out[j] = cut.mode == kNan ? __builtin_nanf("") : (keep ? l : -INFINITY);
  });
}

constexpr int kRowsAtOnce = 512;  // rows whose scratch is held at once

size_t rounded(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

hipError_t launch_sample(const float* logits, int m, int v, int64_t ld, const float* temperature, const int32_t* top_k,
                         const float* top_p, const float* min_p, const uint32_t* u24, int32_t* token, float* out,
                         int32_t* status, hipStream_t stream) {
  const int rows = m < kRowsAtOnce ? m : kRowsAtOnce;
  SampleArgs a{logits, v, ld, temperature, top_p, min_p, top_k, u24, token, out, status, 1, v, false, 51};
  a.aligned = (uintptr_t)logits % 16 == 0 && ld % 4 == 0;
  while (a.shift > 0 && (int64_t(1) << (62 - a.shift)) < v) --a.shift;
  // Segments: as many workgroups as run at once over all rows (two a CU, one of cut_kernel, whose registers allow no more:
  // at 64 rows of 151936 logits 27 us for 34 with two), none shorter than pays.
  auto cut_up = [&](SampleArgs& b, int at_once) {
    int n = at_once / rows;
    const int most = (v + kMinSegment - 1) / kMinSegment;
    // The last workgroup of a row adds up the bins of all its segments: beyond 16 that costs more than the shorter segments
    // give (16 rows of 152000: 44 us with 32, 37 with 16, 44 with 8) until they are long ones (a row of 2^20: 43 for 56).
    int cap = v / kLongSegment;
    cap = cap < kMaxSegments / 2 ? kMaxSegments / 2 : (cap > kMaxSegments ? kMaxSegments : cap);
    n = n > cap ? cap : n;
    n = n > most ? most : n;
    b.segments = n < 1 ? 1 : n;
    b.run = ((v + b.segments * kWaves - 1) / (b.segments * kWaves) + 3) / 4 * 4;
  };
  cut_up(a, 2 * cu_count());
  const size_t rs = (size_t)rows * a.segments;
  const size_t bytes[] = {rs * sizeof(Cell),        rs * kBins * 8,             rs * kWaves * 8,  rs * kBins * 4,
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
  sc.counts = reinterpret_cast<int32_t*>(take(3));
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
    SampleArgs c = b;
    cut_up(c, cu_count());
    const dim3 grid((unsigned)(n * a.segments)), block(kThreads);
    hipLaunchKernelGGL(range_kernel, grid, block, 0, stream, b, sc);
    hipLaunchKernelGGL(bins_kernel, grid, block, 0, stream, b, sc);
    if (top_k || top_p) hipLaunchKernelGGL(cut_kernel, dim3((unsigned)(n * c.segments)), block, 0, stream, c, sc);
    if (out) hipLaunchKernelGGL(filter_kernel, grid, block, 0, stream, b, sc);
  }
  return hipGetLastError();
}

}  // namespace sq

// Causal grouped-query attention of packed rows over a cache of fp16 or 4-bit entries:
//   out[r][h] = f16( sum_{t <= p} e_t v_t / sum_{t <= p} e_t ),  e_t = exp(q . k_t / sqrt(128))
// for row r at position p of its sequence, the softmax kept as a running maximum and sum while the keys pass once.
// The G = hq / hkv query heads of a kv head read the same keys, so the unit of work is a tile of a sequence's queries
// qi = j G + gg (row j, head gg of the group): one pass over the keys serves all G heads.
//   prompt_attn_kernel  many rows: 32 queries a wavefront, keys through LDS; bound by the matrix cores
//   few_attn_kernel     few rows: every wavefront its own keys; bound by the cache's bytes
//   packed_merge_kernel joins the parts of the keys where they were split over workgroups
// Both keep S^T = K Q^T and O^T = V^T P^T, so that a query is a lane's column in every product: the maximum, the sum
// and the rescaling of O need no exchange but a fold over the lanes of one column.  The keys enter S^T in an order that
// makes a lane's scores consecutive keys, which is the order that P^T's fragments take: P goes from one product to the
// next in registers.
// Scores, maxima, sums and O are fp32.  A weight enters the product with V as two binary16 terms (2^-20 of itself off at
// most) in few rows over fp16 entries, whose bytes bound them: the second product costs nothing there (64 tokens after 2000
// positions 54.9 us for 54.8, 32 blocks of 4 rows 37.7 for 37.1).  It enters as one (2^-11 of itself off, as the output's own
// rounding is, and independent from key to key) where the products bound the kernel, in prompts (16001 rows would take
// 2527 us for 1832, four of about 1170 81 for 65), and over 4-bit entries, whose own steps are a fifteenth of a group's
// range and whose dequantisation fills the rest (64 tokens after 2000 positions 18.6 for 17.5, 16 after 13k to 31k 53 for 49).
// Against 64 bits, relative in the 2-norm, one term is 2.0e-4 to 2.2e-4 off where the output's rounding alone is 2.0e-4 to
// 2.1e-4.  Weights are kept times 2^7, and the reference maximum is
// moved only when a row's maximum passes it by 2^8, so they stay below 2^15 and a weight loses bits only
// below 2^-21 of the row's largest.  The reference is kept as the score it was, unscaled, and joined so: a score's scaling
// rounds by what at 10^9 is many powers of two.
#include <type_traits>

#include "sq_internal.hpp"
#include "sq_packed.hpp"

namespace sq {
namespace {

typedef float float16_t __attribute__((ext_vector_type(16)));

constexpr int kTile = 64;  // keys per step
constexpr float kScale = 1.4426950408889634f * 0.08838834764831845f;  // log2(e) / sqrt(128)
constexpr float kShift = 7.f, kSlack = 8.f / kScale;  // (the slack in unscaled scores)
constexpr float kFar = 4096.f;  // references from which their scaling's rounding (2^-15 here) would matter
constexpr int kMaxParts = 256;  // of one kv head's keys, all sequences
constexpr float kNoMax = -1e30f;  // a finite start, below every score: its weights beside any other's are 0

struct AttnArgs {
  const uint16_t* q;
  KvCache c;
  const int32_t* pos_base;
  int pos_offset, hq, hkv;
  int64_t len_bound, capacity;
  uint16_t* out;
  float* part_o;    // [unit][kv head][query][128], null without splitting
  float2* part_ml;  // [unit][kv head][query]
  int most;         // parts of one kv head, 0 without splitting
  int grain;        // steps that a part's are a multiple of
  bool longest;     // the tiles with the most keys first (they do not all run at once)
};

// max / sum over the two lanes that share a column of a 32 x 32 product
template <class OP>
__device__ __forceinline__ float pair_fold(float v, OP op) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  const auto p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const uint32_t p0 = p[0], p1 = p[1];
  return op(__builtin_bit_cast(float, p0), __builtin_bit_cast(float, p1));
}

// The factor from reference `from` to reference `to`.
__device__ __forceinline__ float rescale(float from, float to) { return exp2_fast((from - to) * kScale); }

// A weight is exp2(score kScale + ref).  Far from zero that would round the product and the reference each on its own, by
// more than a weight's range at the ends of binary16's queries and keys: there the reference is taken from the scores first
// (far: some lane of the wavefront is).
__device__ __forceinline__ bool far_reference(float m) { return __any(fabsf(m) > kFar && m != kNoMax); }
__device__ __forceinline__ float near_reference(float m) { return __builtin_fmaf(m, -kScale, kShift); }

// Two weights as two binary16 terms each: truncated, and what that leaves (exact in fp32), truncated.  Where it leaves
// nothing of a weight, the second term is the least there is: a zero would make an infinite value NaN.
__device__ __forceinline__ void two_terms(float p0, float p1, half2_t& hi, half2_t& lo) {
  hi = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_pkrtz(p0, p1));
  lo = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_pkrtz(p0 - (float)hi[0], p1 - (float)hi[1]));
  lo = __builtin_elementwise_max(lo, __builtin_elementwise_min(hi, half2_t{(half_t)0x1p-24f, (half_t)0x1p-24f}));
}

// How the work is laid over workgroups.  A sequence's queries are `tiles` tiles, each over the sequence's `steps` steps of
// 64 keys, and every tile's steps are cut into parts of `span`: `span` is what keeps the number of parts of all sequences
// within `most` (0: no cutting), so that sequences of different lengths give workgroups of like length.  Every workgroup
// forms it for itself from the device's lengths: with S = sum of tiles * steps and N = sum of tiles, S / (most - N) always
// suffices and S / most never does; the smallest of four values between that does is taken (up to 64 sequences, whose
// sums are one reduction; the first for more).
struct SeqWork {
  int tiles, steps;
  SeqRows rows;
  int64_t p0;  // position of the first row
};
struct Unit {
  int s, tile, part, span, steps;
  SeqRows rows;
  int64_t p0;
};

template <int Ctrl>
__device__ __forceinline__ float dpp_move(float v) {
  return __builtin_bit_cast(float,
                            __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), Ctrl, 0xF, 0xF, false));
}

__device__ __forceinline__ float wave_total(float v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, quad_sum(v));
  float x = __builtin_bit_cast(float, u);
  x = dpp_add<0xB1>(x);   // quad_perm [1,0,3,2]
  x = dpp_add<0x4E>(x);   // quad_perm [2,3,0,1]
  x = dpp_add<0x141>(x);  // row_half_mirror
  return dpp_add<0x140>(x);  // row_mirror
}

__device__ __forceinline__ float wave_most(float v) {
  float x = quad_max(v);
  x = fmaxf(x, dpp_move<0xB1>(x));
  x = fmaxf(x, dpp_move<0x4E>(x));
  x = fmaxf(x, dpp_move<0x141>(x));
  return fmaxf(x, dpp_move<0x140>(x));
}

template <class F>
struct Planner {
  int b, span, lane;
  F work;
  SeqWork mine;

  __device__ __forceinline__ SeqWork at(int base) const {
    if (base == 0) return mine;
    return base + lane < b ? work(base + lane) : SeqWork{};
  }
  static __device__ __forceinline__ int parts(SeqWork w, int span) {
    return w.steps > span ? (w.steps + span - 1) / span : 1;
  }

  __device__ __forceinline__ Planner(int b, int most, int grain, F work) : b(b), span(1 << 30), lane(threadIdx.x & 63), work(work) {
    mine = lane < b ? work(lane) : SeqWork{};
    if (most == 0) return;
    float S = 0.f, N = 0.f;  // (up to 256 sums in fp32: S is taken 2^-13 larger)
    for (int base = 0; base < b; base += kWave) {
      const SeqWork w = at(base);
      S += wave_total((float)w.tiles * (float)w.steps);
      N += wave_total((float)w.tiles);
    }
    S *= 1.f + 0x1p-13f;
    auto up = [&](float x) { return ((int)fminf(x, 0x1p29f) / grain + 1) * grain; };
    const float room = (float)most - N;
    if (room < 1.f) return;  // only where row_start lets sequences share rows
    const int hi = up(S / room);
    span = hi;
    if (b > kWave) return;
    const int lo = up(S / (float)most - 1.f);
#pragma unroll
    for (int i = 3; i >= 0; --i) {
      const int c = lo + (hi - lo) / grain * i / 4 * grain;
      // parts or one more: the quotient in fp32, 2^-20 larger (a tile without keys is a part too)
      const float n = (float)(mine.steps + c - 1) * __builtin_amdgcn_rcpf((float)c) * (1.f + 0x1p-20f);
      if (wave_total((float)mine.tiles * fmaxf(floorf(n), 1.f)) <= (float)most) span = c;
    }
    span = __builtin_amdgcn_readfirstlane(span);
  }

  // what lane l holds of sequence s
  __device__ __forceinline__ void fill(Unit& u, int s, const SeqWork& w, int l) const {
    u.s = __builtin_amdgcn_readfirstlane(s);
    u.span = span;
    u.steps = __builtin_amdgcn_readlane(w.steps, l);
    u.rows.first = __builtin_amdgcn_readlane(w.rows.first, l);
    u.rows.n = __builtin_amdgcn_readlane(w.rows.n, l);
    const uint32_t lo = __builtin_amdgcn_readlane((int)w.p0, l);
    u.p0 = (int64_t)__builtin_amdgcn_readlane((int)(w.p0 >> 32), l) << 32 | lo;
  }

  // Unit `item` of the list (sequence 0: tile 0 with its parts, tile 1, ..; sequence 1: ..); false past its end.
  __device__ __forceinline__ bool find(int item, Unit& u) const {
    int before = 0;
    for (int base = 0; base < b; base += kWave) {
      const SeqWork w = at(base);
      const int np = parts(w, span), n = w.tiles * np;
      const int incl = scan(n);
      const int total = __builtin_amdgcn_readlane(incl, kWave - 1);
      if (item < before + total) {
        const int l = __builtin_ctzll(__ballot(before + incl > item));
        const int k = item - before - (__builtin_amdgcn_readlane(incl, l) - __builtin_amdgcn_readlane(n, l));
        const int pl = __builtin_amdgcn_readlane(np, l);
        fill(u, base + l, w, l);
        u.tile = k / pl;
        u.part = k - u.tile * pl;
        return true;
      }
      before += total;
    }
    return false;
  }

  // Unit `item` of the list of whole tiles by the number of their keys, the most first, for up to 64 sequences (the plain
  // list for more).  TQ queries are G-th as many rows, so a tile's place is its level: the sequence's tiles from its last,
  // after as many as it is shorter than the longest sequence that has tiles (2^23 at most: with the 2^20 tiles there can be
  // a level stays a whole number of fp32, and what lies further apart only loses its order).  B(v), the tiles below level v,
  // is one reduction; the search for the item's level takes three of them a turn.
  __device__ __forceinline__ bool find_longest(int item, int G, int TQ, Unit& u) const {
    if (b > kWave) return find(item, u);
    const float longest = wave_most(mine.tiles > 0 ? (float)mine.steps : 0.f);
    const int off = (int)fmaxf(fminf((longest - (float)mine.steps) * (float)(kTile * G) / (float)TQ, 0x1p23f), 0.f);
    const int levels = (int)wave_most(mine.tiles > 0 ? (float)(off + mine.tiles) : 0.f);
    auto below = [&](int v) {
      const int n = v - off;
      return wave_total((float)(n < 0 ? 0 : (n > mine.tiles ? mine.tiles : n)));
    };
    int lo = 0, hi = levels;  // B(lo) <= item < B(hi)
    if ((float)item >= below(hi)) return false;
    while (hi - lo > 1) {
      const int step = (hi - lo + 3) / 4;
      int cut[3];
      float n[3];
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        cut[i] = lo + step * (i + 1) < hi ? lo + step * (i + 1) : hi;
        n[i] = below(cut[i]);
      }
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (n[i] <= (float)item) lo = cut[i];
      hi = lo + step < hi ? lo + step : hi;
    }
    const bool in = off <= lo && lo < off + mine.tiles;
    const uint64_t set = __ballot(in);
    const int rank = __builtin_amdgcn_mbcnt_hi((uint32_t)(set >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)set, 0));
    const int k = item - (int)below(lo);
    const int l = __builtin_ctzll(__ballot(in && rank == k));
    fill(u, l, mine, l);
    u.tile = lo - __builtin_amdgcn_readlane(off, l);
    u.part = 0;
    return true;
  }

  // Tile `item` of the list without parts, and the index of its first part in the list with them.
  __device__ __forceinline__ bool find_tile_parts(int item, Unit& u, int& first) const {
    int before = 0, before_p = 0;
    for (int base = 0; base < b; base += kWave) {
      const SeqWork w = at(base);
      const int np = parts(w, span);
      const int incl = scan(w.tiles), incl_p = scan(w.tiles * np);
      const int total = __builtin_amdgcn_readlane(incl, kWave - 1);
      if (item < before + total) {
        const int l = __builtin_ctzll(__ballot(before + incl > item));
        const int tl = __builtin_amdgcn_readlane(w.tiles, l), pl = __builtin_amdgcn_readlane(np, l);
        fill(u, base + l, w, l);
        u.tile = item - before - (__builtin_amdgcn_readlane(incl, l) - tl);
        u.part = 0;
        first = before_p + __builtin_amdgcn_readlane(incl_p, l) - tl * pl + u.tile * pl;
        return true;
      }
      before += total;
      before_p += __builtin_amdgcn_readlane(incl_p, kWave - 1);
    }
    return false;
  }

  // sum over the lanes up to this one
  static __device__ __forceinline__ int scan(int n) {
    n += __builtin_amdgcn_update_dpp(0, n, 0x111, 0xF, 0xF, true);  // row_shr:1
    n += __builtin_amdgcn_update_dpp(0, n, 0x112, 0xF, 0xF, true);
    n += __builtin_amdgcn_update_dpp(0, n, 0x114, 0xF, 0xF, true);
    n += __builtin_amdgcn_update_dpp(0, n, 0x118, 0xF, 0xF, true);
    n += __builtin_amdgcn_update_dpp(0, n, 0x142, 0xA, 0xF, false);  // row_bcast:15 into rows 1 and 3
    n += __builtin_amdgcn_update_dpp(0, n, 0x143, 0xC, 0xF, false);  // row_bcast:31 into rows 2 and 3
    return n;
  }
};

// The last key that rows up to position `pl` of a sequence read, and the steps of 64 up to it.
__device__ __forceinline__ int last_key(int64_t pl, int64_t len_bound) {
  const int64_t k = pl < len_bound ? pl : len_bound - 1;  // (rows past the bound are not computed)
  return k < -1 ? -1 : (int)k;
}
__device__ __forceinline__ int steps_to(int klast) { return klast < 0 ? 0 : klast / kTile + 1; }

// Tiles of TQ queries of a sequence, and its steps.
__device__ __forceinline__ SeqWork seq_work(const PackedRows& pr, const AttnArgs& a, int G, int TQ, int s) {
  const int64_t p0 = (int64_t)a.pos_base[s] + a.pos_offset;
  const SeqRows sr = seq_rows(pr, s);
  return {(sr.n * G + TQ - 1) / TQ, steps_to(last_key(p0 + sr.n - 1, a.len_bound)), sr, p0};
}

// ------------------------------------------------------------------ dequant
// Sixteen bytes of codes to 16 halves of the low and 16 of the high nibbles: f16((c - z) s), the difference exact.
template <bool HIGH, class Z, class S>
__device__ __forceinline__ void dequant16(const CodeConsts& k, u32x4 w, Z zero, S scale, half8_t (&o)[2]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    half2_t a, b;
    code_pairs<HIGH>(k, w[i], a, b);
    a = (a - zero(2 * i)) * scale(2 * i);
    b = (b - zero(2 * i + 1)) * scale(2 * i + 1);
    o[i >> 1][4 * (i & 1) + 0] = a[0];
    o[i >> 1][4 * (i & 1) + 1] = a[1];
    o[i >> 1][4 * (i & 1) + 2] = b[0];
    o[i >> 1][4 * (i & 1) + 3] = b[1];
  }
}

// A key's part: 16 elements of each group, with the key's own scales and zeros.
__device__ __forceinline__ void dequant_key(const CodeConsts& k, u32x4 w, uint2 sz, half8_t (&lo)[2], half8_t (&hi)[2]) {
  const half2_t s0 = bits_h2((sz.x & 0xFFFF) * 0x10001u), z0 = zero_pair<false>(bits_h2((sz.x >> 16) * 0x10001u));
  const half2_t s1 = bits_h2((sz.y & 0xFFFF) * 0x10001u), z1 = zero_pair<true>(bits_h2((sz.y >> 16) * 0x10001u));
  dequant16<false>(k, w, [&](int) { return z0; }, [&](int) { return s0; }, lo);
  dequant16<true>(k, w, [&](int) { return z1; }, [&](int) { return s1; }, hi);
}

// Scales and zeros of 16 consecutive positions of a block of values: [4][64] halves, 32 bytes of each row.
struct ValScales {
  u32x4 p[4][2];
};
__device__ __forceinline__ ValScales load_val_scales(const uint16_t* vs) {
  ValScales r;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) r.p[i][h] = *reinterpret_cast<const u32x4*>(vs + 64 * i + 8 * h);
  return r;
}
template <bool HIGH>
__device__ __forceinline__ void dequant_val(const CodeConsts& k, u32x4 w, const ValScales& v, half8_t (&o)[2]) {
  constexpr int si = HIGH ? 2 : 0;
  dequant16<HIGH>(
      k, w,
      [&](int i) {
        const uint32_t z = v.p[si + 1][i >> 2][i & 3];
        return zero_pair<HIGH>(bits_h2(z));
      },
      [&](int i) {
        const uint32_t s = v.p[si][i >> 2][i & 3];
        return bits_h2(s);
      },
      o);
}

// Element `dim` of the value at position `key` of (sequence, kv head) sg.
template <bool Q4>
__device__ __forceinline__ float value_at(const AttnArgs& a, int64_t sg, int64_t key, int dim) {
  if constexpr (!Q4) return f16_bits_to_f32(a.c.v[(sg * kHd + dim) * a.capacity + key]);
  const int64_t blk = sg * a.capacity + (key & ~63);
  const int j = dim & 63, t = (int)key & 63, hi = dim >> 6;
  const uint32_t c = a.c.v4[blk * 64 + j * 64 + swap01(t)] >> (4 * hi) & 15;
  const uint16_t* p = a.c.vs + blk * 4 + 128 * hi + t;
  return (float)(half_t)(((float)c - f16_bits_to_f32(p[64])) * f16_bits_to_f32(p[0]));
}

// The elements of a key's value that are not finite (zero for the others), dims lane and 64 + lane: the lanes hand them
// round, since a lane's own 32 or 64 addresses would be formed ahead of the loop over keys and held in registers.
struct OddValue {
  float v[2];
};
template <bool Q4>
__device__ __forceinline__ OddValue odd_value(const AttnArgs& a, int64_t sg, int64_t key) {
  OddValue r;
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float v = value_at<Q4>(a, sg, key, 64 * i + lane);
    r.v[i] = fabsf(v) <= 65504.f ? 0.f : v;
  }
  return r;
}

// A step past a tile's first row holds keys that some row may not read.  What must not reach a row there: values after
// the last row's position (stale, anything), and values that are not finite, since a zero weight times one is NaN.  Both
// are zeroed for the products; where a value was not finite, odd_values later adds it to the rows that do read it.
// The halves of words of positions e, e + 1 up to the last key `left`:
__device__ __forceinline__ uint32_t keep_mask(int e, int left) {
  return (e <= left ? 0xFFFFu : 0u) | (e + 1 <= left ? 0xFFFF0000u : 0u);
}
// bit 15 of every half that is not finite: a full exponent carries into it
__device__ __forceinline__ uint32_t odd_halves(uint32_t w) { return ((w & 0x7C007C00u) + 0x04000400u) & 0x80008000u; }
__device__ __forceinline__ uint32_t without(uint32_t w, uint32_t odd) { return w & ~(odd | (odd - (odd >> 15))); }

// The same for the scales and zeros of a word's two positions: stale ones become 0, and a scale that is not finite does
// (a zero always is finite), so that the values they give do.
__device__ __forceinline__ uint32_t tame_scales(uint32_t w, int e, int left, bool scale, uint32_t& odd) {
  w &= keep_mask(e, left);
  const uint32_t o = scale ? odd_halves(w) : 0u;
  odd |= o;
  return without(w, o);
}

// ---------------------------------------------------------------- few rows
// One workgroup per (part of the keys, sequence, kv head); its wavefronts take the part's steps of 64 keys in turn, each
// for all the queries (NQT tiles of 16), and meet in LDS.  v_mfma_f32_16x16x32_f16: lane l holds row / column li = l %
// 16 and k = 8 lg .. +8 (lg = l / 16); D[4 lg + i][li].  The rows of the key tiles are keys in an order that gives a lane the
// scores of 16 keys whose values lie in runs of 16 bytes, so that it takes them as they lie.
// A step's keys are loaded while the step before takes its values, and the other way round, each into the registers that
// were just used (fp16 and two tiles: the registers hold only one of the two, loaded when its turn comes).  Up to
// 32 queries: all eight wavefronts take keys; up to 64 (4-bit entries): half of them the first 32, half the rest, over the
// same keys.  fp16 entries: bound by the cache's bytes, 64 tokens after 2000 positions (28 heads on 4, 262 MB) 54.9 us, 4.8 TB/s.
// 4-bit: by reads and arithmetic together, 16 tokens after 13k to 31k positions (207 MB, three caches in turn) 44.0 us and 4.8
// for the merge, 4.7 TB/s without it where a streaming read reaches 6.2 to 6.5.  A few sequences by latency: the plan
// 1 us, the first loads 2, a step of 64 keys 0.7, the meeting in LDS 1, and a CU takes in fp16 entries at about 60 GB/s.
constexpr int kFewWaves = 8;

template <bool Q4, int NQT, int HALVES>
__global__ __launch_bounds__(64 * kFewWaves) __attribute__((amdgpu_waves_per_eu(2))) void few_attn_kernel(PackedRows pr,
                                                                                                        AttnArgs a) {
  constexpr int NW = kFewWaves / HALVES;  // wavefronts that share the keys of a half's queries
  constexpr bool kAhead = Q4 || NQT == 1;
  constexpr bool kTwoTerms = !Q4;
  __shared__ __align__(16) float ob[kFewWaves][16 * NQT][kHd + 4];
  __shared__ float2 ml[kFewWaves][16 * NQT];
  __shared__ __align__(16) uint16_t vsb[Q4 ? kFewWaves : 1][4][64];  // a step's scales and zeros of values, per wavefront
  const int item = blockIdx.x / a.hkv, g = blockIdx.x - item * a.hkv;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lg = lane >> 4;
  const int wave8 = __builtin_amdgcn_readfirstlane(tid >> 6), wave = wave8 / HALVES;
  const int q0 = wave8 % HALVES * (16 * NQT);  // the wavefront's first query
  const int G = a.hq / a.hkv;
  Unit u;
  if (a.most) {
    const Planner plan(pr.b, a.most, a.grain, [&](int i) { return seq_work(pr, a, G, 16 * NQT * HALVES, i); });
    if (!plan.find(item, u)) return;
  } else {  // an item a sequence
    const SeqWork w = seq_work(pr, a, G, 16 * NQT * HALVES, item);
    if (w.tiles == 0) return;
    u = {item, 0, 0, 1 << 30, w.steps, w.rows, w.p0};
  }
  const int64_t sg = (int64_t)u.s * a.hkv + g;
  const SeqRows sr = u.rows;
  const int nq = sr.n * G;
  const int64_t p0 = u.p0;
  const int64_t klast = last_key(p0 + sr.n - 1, a.len_bound);
  const int st0 = u.part * u.span, st1 = st0 + u.span < u.steps ? st0 + u.span : u.steps;

  half8_t qf[NQT][4];
  int lpos[NQT];  // the position of this lane's query, clipped to [-1, 2^31)
#pragma unroll
  for (int t = 0; t < NQT; ++t) {
    const int qi = q0 + 16 * t + li, qc = qi < nq ? qi : nq - 1;
    const int j = qc / G;
    const uint16_t* qp = a.q + ((int64_t)(sr.first + j) * a.hq + g * G + (qc - j * G)) * kHd;
#pragma unroll
    for (int x = 0; x < 4; ++x)
      qf[t][x] = *reinterpret_cast<const half8_t*>(qp + (Q4 ? (x >> 1) * 64 + 16 * lg + 8 * (x & 1) : 32 * x + 8 * lg));
    const int64_t p = p0 + j;
    lpos[t] = p < 0 ? -1 : (p > 0x7FFFFFFF ? 0x7FFFFFFF : (int)p);
  }
  float m[NQT], l[NQT];
  float4_t o[NQT][8];
  half8_t pf[NQT][2], pl[kTwoTerms ? NQT : 1][2];  // the weights, and their second terms
#pragma unroll
  for (int t = 0; t < NQT; ++t) {
    m[t] = kNoMax;
    l[t] = 0.f;
#pragma unroll
    for (int d = 0; d < 8; ++d) o[t][d] = float4_t{0.f, 0.f, 0.f, 0.f};
  }
  const CodeConsts kc;
  // Row li of tile kt is key krow + kt_at(kt), so that a lane ends with the scores of keys run lg .. + run (and, run 8, the
  // same of the step's second half): 16 codes are 16 bytes, 8 halves are, and four lanes' loads are one run of memory.
  constexpr int kRun = Q4 ? 16 : 8;
  const int krow = kRun * (li >> 2) + (li & 3);
  auto kt_at = [](int kt) { return Q4 ? 4 * kt : 32 * (kt >> 1) + 4 * (kt & 1); };
  u32x4 kw[Q4 ? 4 : 16], vw[Q4 ? 4 : 16];  // 4-bit: a key's 16 bytes lg, byte rows 16 j + li; fp16: dims 32 x + 8 lg
  uint2 ksz[4];                            // .. +8 of a key, positions 8 lg .. +8 and 32 + 8 lg .. +8 of dim 16 d + li
  uint2 vsr;  // 4-bit: this lane's 8 of the 512 bytes of a step's scales and zeros of values
  // uniform bases and 32-bit lane offsets: the addresses stay out of the vector registers
  const uint8_t* k4 = a.c.k4 + sg * a.capacity * 64;
  const uint16_t* ks = a.c.ks + sg * a.capacity * 4;
  const uint8_t* v4 = a.c.v4 + sg * a.capacity * 64;
  const uint16_t* vs4 = a.c.vs + sg * a.capacity * 4;
  const uint16_t* k16 = a.c.k + sg * a.capacity * kHd;
  const uint16_t* v16 = a.c.v + sg * kHd * a.capacity;
  const int64_t vlane = (int64_t)li * a.capacity + 8 * lg;
  // `live`: all ones; 0 for loads that nothing will use, which all take one lane's
  auto load_k = [&](int st, uint32_t live) {
    if constexpr (Q4) {
      const uint8_t* kst = k4 + (int64_t)st * (kTile * 64);
      const uint16_t* sst = ks + (int64_t)st * (kTile * 4);
      const uint32_t at = (krow * 64 + 16 * lg) & live, as = krow * 8 & live;
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) {
        kw[kt] = *reinterpret_cast<const u32x4*>(kst + (at + 256 * kt));
        ksz[kt] = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint8_t*>(sst) + (as + 32 * kt));
      }
    } else {
      const uint8_t* kst = reinterpret_cast<const uint8_t*>(k16 + (int64_t)st * (kTile * kHd));
      const uint32_t at = (krow * 256 + 16 * lg) & live;
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int x = 0; x < 4; ++x) kw[4 * kt + x] = *reinterpret_cast<const u32x4*>(kst + (at + 256 * kt_at(kt) + 64 * x));
    }
  };
  auto load_v = [&](int st, uint32_t live) {
    if constexpr (Q4) {
      vsr = reinterpret_cast<const uint2*>(vs4 + (int64_t)st * 256)[(uint32_t)lane & live];
      const uint8_t* vst = v4 + (int64_t)st * 4096;
      const uint32_t at = (li * 64 + 16 * lg) & live;
#pragma unroll
      for (int j = 0; j < 4; ++j) vw[j] = *reinterpret_cast<const u32x4*>(vst + (at + 1024 * j));
    } else {
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        const int64_t vl = live ? vlane : 0;
        const uint16_t* vst = v16 + (int64_t)16 * d * a.capacity + (int64_t)st * kTile;
        vw[2 * d] = *reinterpret_cast<const u32x4*>(vst + vl);
        vw[2 * d + 1] = *reinterpret_cast<const u32x4*>(vst + vl + 32);
      }
    }
  };
  const int end = HALVES == 1 || q0 < nq ? st1 : 0;
  // Of the two wavefronts of a SIMD the older issues first and was done after 22 us of 36 with half of the steps (16
  // sequences, 22k positions on average): the older ones take three of five, steps wave + NW {0, 1, 2} of every 5 NW / 2.
  const bool older = wave < NW / 2;
  int turn = 0;
  auto advance = [&](int st) {
    const int gap = older ? (turn == 2 ? NW / 2 : NW) : (turn == 1 ? NW + NW / 2 : NW);
    turn = turn == (older ? 2 : 1) ? 0 : turn + 1;
    return st + gap;
  };
  if (kAhead && st0 + wave < end) {
    load_k(st0 + wave, ~0u);
    load_v(st0 + wave, ~0u);
  }
  auto product = [&](int d, half8_t v0, half8_t v1) {
#pragma unroll
    for (int t = 0; t < NQT; ++t) {
      if constexpr (kTwoTerms) {
        o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pl[t][0], o[t][d], 0, 0, 0);
        o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pl[t][1], o[t][d], 0, 0, 0);
      }
      o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pf[t][0], o[t][d], 0, 0, 0);
      o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pf[t][1], o[t][d], 0, 0, 0);
    }
  };
  bool odd_seen = false;
  for (int st = st0 + wave, following; st < end; st = following) {
    const int64_t key0 = (int64_t)st * kTile;
    following = advance(st);
    const int next = following < end ? following : st;  // (loads after the last step, too: no branch around loads)
    const uint32_t live = following < end ? ~0u : 0u;
    float4_t sc[NQT][4];
    if constexpr (!kAhead) load_k(st, ~0u);
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
      half8_t kf[4];
      if constexpr (Q4) {
        half8_t lo[2], hi[2];
        dequant_key(kc, kw[kt], ksz[kt], lo, hi);
        kf[0] = lo[0];
        kf[1] = lo[1];
        kf[2] = hi[0];
        kf[3] = hi[1];
      } else {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const u32x4 w = kw[4 * kt + x];
          kf[x] = __builtin_bit_cast(half8_t, w);
        }
      }
#pragma unroll
      for (int t = 0; t < NQT; ++t) {
        float4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < 4; ++x) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[x], qf[t][x], acc, 0, 0, 0);
        sc[t][kt] = acc;
      }
      if constexpr (NQT > 1) __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (kAhead)
      load_k(next, live);
    else
      load_v(st, ~0u);
    __builtin_amdgcn_sched_barrier(0);
    // only a step past the first row's position holds keys that some row may not read
    const bool tail = key0 + kTile - 1 > p0;  // uniform
#pragma unroll
    for (int t = 0; t < NQT; ++t) {
      if (tail) {
        const int lim = (int)(lpos[t] - key0 < kTile ? lpos[t] - key0 : kTile) - kRun * lg;
#pragma unroll
        for (int kt = 0; kt < 4; ++kt)
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[t][kt][i] = kt_at(kt) + i <= lim ? sc[t][kt][i] : -__builtin_inff();
      }
      float cm = sc[t][0][0];
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) cm = fmaxf(cm, sc[t][kt][i]);
      cm = quad_max(cm);
      if (__any(cm > m[t] + kSlack)) {
        const float mn = fmaxf(m[t], cm), alpha = rescale(m[t], mn);
        m[t] = mn;
        l[t] *= alpha;
#pragma unroll
        for (int d = 0; d < 8; ++d) o[t][d] *= alpha;
      }
      float ref = near_reference(m[t]);
      if (far_reference(m[t])) {  // uniform
#pragma unroll
        for (int kt = 0; kt < 4; ++kt)
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[t][kt][i] -= m[t];
        ref = kShift;
      }
      float sum = 0.f;
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          const float p0 = exp2_fast(__builtin_fmaf(sc[t][kt][i], kScale, ref));
          const float p1 = exp2_fast(__builtin_fmaf(sc[t][kt][i + 1], kScale, ref));
          sum += p0;
          sum += p1;
          half2_t hi = {(half_t)p0, (half_t)p1}, lo;
          if constexpr (kTwoTerms) {
            two_terms(p0, p1, hi, lo);
            pl[t][kt >> 1][4 * (kt & 1) + i] = lo[0];
            pl[t][kt >> 1][4 * (kt & 1) + i + 1] = lo[1];
          }
          pf[t][kt >> 1][4 * (kt & 1) + i] = hi[0];
          pf[t][kt >> 1][4 * (kt & 1) + i + 1] = hi[1];
        }
      l[t] += sum;
    }
    if (tail) {
      uint32_t odd = 0;
      if constexpr (Q4) {
        const int left = (int)(klast - key0 < kTile ? klast - key0 : kTile) - 4 * li;  // row lg of the four
        vsr.x = tame_scales(vsr.x, 0, left, (lg & 1) == 0, odd);
        vsr.y = tame_scales(vsr.y, 2, left, (lg & 1) == 0, odd);
      } else {
        const int left = (int)(klast - key0 < kTile ? klast - key0 : kTile) - kRun * lg;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const uint32_t keep = keep_mask(kt_at(x >> 1) + 2 * (x & 1), left);
#pragma unroll
          for (int d = 0; d < 8; ++d) vw[2 * d + (x >> 2)][x & 3] &= keep;
        }
        if (sr.n > 1) {  // (a single row reads every key that is left)
#pragma unroll
          for (int x = 0; x < 16; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t o = odd_halves(vw[x][i]);
              odd |= o;
              vw[x][i] = without(vw[x][i], o);
            }
        }
      }
      odd_seen |= __any(odd != 0);
    }
    if constexpr (Q4) {
      // every lane needs the scales and zeros of its keys: handed round in LDS, two of the four rows at a time
      reinterpret_cast<uint2*>(vsb[wave8])[lane] = vsr;
      ValScales vs;
      auto rows = [&](int r) {
#pragma unroll
        for (int i = r; i < r + 2; ++i)
#pragma unroll
          for (int x = 0; x < 2; ++x) vs.p[i][x] = *reinterpret_cast<const u32x4*>(&vsb[wave8][i][16 * lg + 8 * x]);
      };
      rows(0);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        half8_t x[2];
        dequant_val<false>(kc, vw[j], vs, x);
        product(j, x[0], x[1]);
        if constexpr (NQT > 1) __builtin_amdgcn_sched_barrier(0);
      }
      rows(2);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        half8_t x[2];
        dequant_val<true>(kc, vw[j], vs, x);
        product(4 + j, x[0], x[1]);
        if constexpr (NQT > 1) __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        const u32x4 w0 = vw[2 * d], w1 = vw[2 * d + 1];
        product(d, __builtin_bit_cast(half8_t, w0), __builtin_bit_cast(half8_t, w1));
      }
    }
    if constexpr (kAhead) load_v(next, live);
    __builtin_amdgcn_sched_barrier(0);
  }
  if (odd_seen) {
    turn = 0;
#pragma unroll 1
    for (int st = st0 + wave; st < end; st = advance(st)) {
      const int64_t key0 = (int64_t)st * kTile;
      if (key0 + kTile - 1 <= p0) continue;
#pragma unroll 1
      for (int64_t key = key0; key < key0 + kTile && key <= klast; ++key) {
        const OddValue ov = odd_value<Q4>(a, sg, key);
        if (!__any(ov.v[0] != 0.f || ov.v[1] != 0.f)) continue;
#pragma unroll
        for (int d = 0; d < 8; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float v = __shfl(ov.v[d >> 2], 16 * (d & 3) + 4 * lg + i, kWave);
#pragma unroll
            for (int t = 0; t < NQT; ++t) o[t][d][i] += key <= lpos[t] ? v : 0.f;
          }
      }
    }
  }
  // the wavefronts' sums meet
  const int nq_pad = 16 * NQT * HALVES, parts = u.steps > u.span ? (u.steps + u.span - 1) / u.span : 1;
#pragma unroll
  for (int t = 0; t < NQT; ++t) {
    const float lt = quad_sum(l[t]);
    if (lg == 0) ml[wave8][16 * t + li] = make_float2(m[t], lt);
#pragma unroll
    for (int d = 0; d < 8; ++d) *reinterpret_cast<float4_t*>(&ob[wave8][16 * t + li][16 * d + 4 * lg]) = o[t][d];
  }
  __syncthreads();
  auto answer = [&](int qi, int d0, const float (&r)[8], float L) {
    const int j = qi / G;
    const int64_t pos = p0 + j;
    const bool bad = pos < 0 || pos >= a.len_bound;
    half8_t h;
#pragma unroll
    for (int x = 0; x < 8; ++x) h[x] = bad ? __builtin_bit_cast(half_t, kNanF16) : (half_t)(r[x] / L);
    *reinterpret_cast<half8_t*>(a.out + ((int64_t)(sr.first + j) * a.hq + g * G + (qi - j * G)) * kHd + d0) = h;
  };
  for (int qi = tid >> 4; qi < nq; qi += 4 * kFewWaves) {
    const int d0 = 8 * (tid & 15), half = qi / (16 * NQT), qx = qi & (16 * NQT - 1);
    float M = kNoMax, L = 0.f, r[8] = {};
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, ml[HALVES * w + half][qx].x);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float2 x = ml[HALVES * w + half][qx];
      const float f = rescale(x.x, M);
      L += f * x.y;
      const float4_t u = *reinterpret_cast<const float4_t*>(&ob[HALVES * w + half][qx][d0]);
      const float4_t v = *reinterpret_cast<const float4_t*>(&ob[HALVES * w + half][qx][d0 + 4]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        r[i] += f * u[i];
        r[4 + i] += f * v[i];
      }
    }
    if (parts > 1) {
      const int64_t at = (int64_t)blockIdx.x * nq_pad + qi;
      float* po = a.part_o + at * kHd + d0;
      reinterpret_cast<float4_t*>(po)[0] = float4_t{r[0], r[1], r[2], r[3]};
      reinterpret_cast<float4_t*>(po)[1] = float4_t{r[4], r[5], r[6], r[7]};
      if ((tid & 15) == 0) a.part_ml[at] = make_float2(M, L);
    } else {
      answer(qi, d0, r, L);
    }
  }
}

// -------------------------------------------------------------- many rows
// One workgroup per (tile of 32 NW queries, kv head, part of the keys): each wavefront 32 queries, KW groups of NW of them the
// keys in turn, in steps of 64 through LDS buffers, one barrier a step.  fp16 entries go from memory to LDS directly, kRing - 1 steps ahead; 4-bit
// ones through registers, one step ahead, and become halves on the way.
// v_mfma_f32_32x32x16_f16: lane l holds row / column lc = l % 32 and k = 8 h .. +8 (h = l / 32), and of D rows 8 (i / 4) +
// 4 h + i % 4 of column lc.  Row r of a key tile is the key r with bits 2 and 3 exchanged, so that a lane's 16 scores
// are keys 16 (i / 8) + 8 h + i % 8: the P^T fragments of two steps of 16 keys.
// LDS: keys as rows of 16 cells (16 B) with cell c at c ^ (r % 16), values as rows of 8 cells (64 positions of a
// dimension) with cell c at c ^ (d / 2 % 8): 16 lanes of one fragment read 16 different 16-byte banks.
// Bound by the matrix cores and, near them, the power: one prompt of 16001 rows (28 heads on 4, 1.84 TFLOP) 1780 us, 1030
// TFLOP/s, at the clock of about 1.5 GHz that this load leaves; a square product of 8192 by the library reaches 1178.  Four
// prompts of about 1170 rows 57.5 us (700 TFLOP/s: the last tiles leave CUs idle).  Two wavefronts a SIMD take 1.57 us a step
// together, one alone 1.26: products and exponentials of the two overlap.
__device__ __forceinline__ int swap23(int i) { return (i & ~12) | ((i & 4) << 1) | ((i & 8) >> 1); }

typedef __attribute__((address_space(3))) void lds_void;

// 16 bytes per lane from memory to LDS: from base + off (off per lane) to the LDS address dst + 16 l for lane l.  In
// assembly, because the compiler waits for all loads of the builtin before any read of LDS, whichever buffer it reads;
// the waits are barrier_after_loads.  There is no result register, and the addresses are read when the load is issued.
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t off, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(dst)
               : "memory", "m0");
}
template <class T>
__device__ __forceinline__ uint32_t lds_address(T* p) {
  return (uint32_t)(uintptr_t)(lds_void*)p;
}

// All but the wavefront's last N loads, and everything it did in LDS, done by every wavefront.
template <int N>
__device__ __forceinline__ void barrier_after_loads() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Where keys are split, a CU has one workgroup: two groups of four wavefronts take its steps in turn and meet in LDS (20.2 us
// for 20.8 with one: three sequences of 20 to 57 rows after 3358 to 8773 cached positions, 28 query heads on 4).
constexpr int kSplitGroups = 2;

// Buffers of 32 KB a group: two for four wavefronts, two groups of which share a CU, three for those of eight.  Where keys are
// split more did not help (one group: 20.8 us with two, 22.5 with three, 24.2 with four).
constexpr int ring(bool q4, int nw) { return q4 || nw < 8 ? 2 : 3; }

template <bool Q4, int NW, int KW, bool SPLIT>
__global__ __launch_bounds__(64 * NW * KW) __attribute__((amdgpu_waves_per_eu(2, 2))) void prompt_attn_kernel(PackedRows pr,
                                                                                                      AttnArgs a) {
  constexpr int NT = 64 * NW, TQ = 32 * NW, kRing = ring(Q4, NW);
  constexpr int kLoads = 16 / NW;                 // fp16: loads of 1 KB of keys (and of values) per wavefront and step
  constexpr int kCodes = NW >= 8 ? 1 : 512 / NT;  // 4-bit: 16-byte cells of codes per thread
  __shared__ __align__(16) u32x4 kb[KW * kRing][1024], vb[KW * kRing][1024];
  __shared__ int odd_seen;  // a value was not finite
  const int G = a.hq / a.hkv;
  const int item = blockIdx.x / a.hkv, g = blockIdx.x - item * a.hkv;
  const int tid = threadIdx.x & (NT - 1), lane = tid & 63, lc = lane & 31, h = lane >> 5;  // in its group of wavefronts
  const int wave8 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = wave8 & (NW - 1), kw = wave8 / NW;
  Unit u;
  {
    const Planner plan(pr.b, SPLIT ? a.most : 0, KW, [&](int i) { return seq_work(pr, a, G, TQ, i); });
    if (!SPLIT && a.longest ? !plan.find_longest(item, G, TQ, u) : !plan.find(item, u)) return;
  }
  const SeqRows sr = u.rows;
  const int nq = sr.n * G;
  const int qt = (nq + TQ - 1) / TQ - 1 - u.tile;  // the latest rows (the most keys) first
  const int64_t p0 = u.p0;
  const int qlast = (qt + 1) * TQ < nq ? (qt + 1) * TQ - 1 : nq - 1;
  const int64_t pmin = p0 + qt * TQ / G;
  const int klast = last_key(p0 + qlast / G, a.len_bound), nst = steps_to(klast);
  const int st0 = SPLIT ? __builtin_amdgcn_readfirstlane(u.part * u.span) : 0;
  const int st1 = SPLIT && st0 + u.span < nst ? st0 + u.span : nst;
  if (SPLIT && u.part > 0 && st0 >= st1) return;  // (part 0 always answers: rows without any key)
  const int64_t sg = (int64_t)__builtin_amdgcn_readfirstlane(u.s) * a.hkv + g;
  const int wq = qt * TQ + 32 * wave;                       // the wavefront's first query
  const bool owner = wq < nq;
  const int qi = wq + lc < nq ? wq + lc : nq - 1, qj = qi / G;
  auto clip = [](int64_t p) { return p < 0 ? -1 : (p > 0x7FFFFFFF ? 0x7FFFFFFF : (int)p); };
  const int lpos = clip(p0 + qj);
  const int wmin = clip(p0 + wq / G);                       // of the wavefront's queries
  const int wmax = clip(p0 + (wq + 31 < nq ? wq + 31 : nq - 1) / G);

  // fp16: load i of a step takes cells 64 (wave + NW i) .. +64 of the keys and of the values; what a cell of LDS holds is
  // chosen by where its lane reads: a scalar base a load and a 32-bit offset a lane (seven rows of values at most)
  const uint16_t* k16 = a.c.k + sg * a.capacity * kHd;
  const uint16_t* v16[kLoads];
  uint32_t koff[kLoads], voff;
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int row = 4 * (wave + NW * i) + (lane >> 4);
    koff[i] = row * 256 + 16 * ((lane & 15) ^ swap23(row & 15));
    v16[i] = a.c.v + (sg * kHd + 8 * (wave + NW * i)) * a.capacity;
  }
  // (dimension d = 8 (wave + NW i) + lane / 8: d / 2 % 8 is 4 (wave % 2) + lane / 16, NW even)
  voff = (uint32_t)(lane >> 3) * (uint32_t)(2 * a.capacity) + 16 * ((lane & 7) ^ (4 * (wave & 1) + (lane >> 4)));
  const uint32_t kdst = lds_address(&kb[kw * kRing][64 * wave]), vdst = lds_address(&vb[kw * kRing][64 * wave]);
  auto issue_step = [&](int st, int buf) {
    const uint16_t* kst = k16 + (int64_t)st * (kTile * kHd);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load_to_lds(kst, koff[i], kdst + 16384 * buf + 1024 * NW * i);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load_to_lds(v16[i] + (int64_t)st * kTile, voff, vdst + 16384 * buf + 1024 * NW * i);
  };
  // ... and in a step past the tile's first position the values are tamed where they lie
  auto tame_step = [&](int st, int buf) {
    uint32_t odd = 0;
#pragma unroll
    for (int i = 0; i < 1024 / NT; ++i) {
      const int c = tid + NT * i, left = klast - (st * kTile + 8 * ((c & 7) ^ ((c >> 4) & 7)));
      u32x4 w = vb[kw * kRing + buf][c];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const uint32_t v = w[x] & keep_mask(2 * x, left), o = odd_halves(v);
        odd |= o;
        w[x] = without(v, o);
      }
      vb[kw * kRing + buf][c] = w;
    }
    if (odd) odd_seen = 1;
  };

  const CodeConsts kc;
  u32x4 pre[Q4 ? kCodes : 1];
  uint2 pre_ks[Q4 ? kCodes : 1];
  ValScales pre_vs;
  // 4-bit cell c: key c / 4, part c % 4 of it (c < 256), byte (c - 256) / 4 of the block of values, positions 16 (c % 4)
  // .. +16; which of the two is uniform across a wavefront
  auto load_step = [&](int st) {
    const int64_t key0 = (int64_t)st * kTile;
#pragma unroll
    for (int i = 0; i < kCodes; ++i) {
      const int c = tid + NT * i;
      if (c < 256) {
        const int64_t e = sg * a.capacity + key0 + (c >> 2);
        pre[i] = reinterpret_cast<const u32x4*>(a.c.k4)[e * 4 + (c & 3)];
        pre_ks[i] = reinterpret_cast<const uint2*>(a.c.ks)[e];
      } else {
        const int c2 = c - 256;
        pre[i] = *reinterpret_cast<const u32x4*>(a.c.v4 + sg * a.capacity * 64 + (int64_t)st * 4096 + 16 * c2);
        pre_vs = load_val_scales(a.c.vs + sg * a.capacity * 4 + (int64_t)st * 256 + 16 * (c2 & 3));
      }
    }
  };
  auto store_step = [&](int st, int buf) {
#pragma unroll
    for (int i = 0; i < kCodes; ++i) {
      const int c = tid + NT * i;
      half8_t lo[2], hi[2];
      if (c < 256) {
        const int key = c >> 2, part = c & 3;
        dequant_key(kc, pre[i], pre_ks[i], lo, hi);
        const int sw = swap23(key & 15);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          kb[kw * kRing + buf][key * 16 + ((2 * part + x) ^ sw)] = __builtin_bit_cast(u32x4, lo[x]);
          kb[kw * kRing + buf][key * 16 + ((8 + 2 * part + x) ^ sw)] = __builtin_bit_cast(u32x4, hi[x]);
        }
      } else {
        const int c2 = c - 256, j = c2 >> 2, part = c2 & 3;
        if (st * (int64_t)kTile + kTile - 1 > pmin) {  // uniform
          uint32_t odd = 0;
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int x = 0; x < 8; ++x)
              pre_vs.p[r][x >> 2][x & 3] =
                  tame_scales(pre_vs.p[r][x >> 2][x & 3], 2 * x, klast - (st * kTile + 16 * part), (r & 1) == 0, odd);
          if (odd) odd_seen = 1;
        }
        dequant_val<false>(kc, pre[i], pre_vs, lo);
        dequant_val<true>(kc, pre[i], pre_vs, hi);
        const int sw = (j >> 1) & 7;  // (of j + 64 too)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          vb[kw * kRing + buf][j * 8 + ((2 * part + x) ^ sw)] = __builtin_bit_cast(u32x4, lo[x]);
          vb[kw * kRing + buf][(j + 64) * 8 + ((2 * part + x) ^ sw)] = __builtin_bit_cast(u32x4, hi[x]);
        }
      }
    }
  };

  if (threadIdx.x == 0) odd_seen = 0;
  if constexpr (Q4) {
    __syncthreads();
    if (st0 + kw < st1) {
      load_step(st0 + kw);
      store_step(st0 + kw, 0);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kRing - 1; ++i)
      if (st0 + kw + KW * i < st1) issue_step(st0 + kw + KW * i, i);
  }
  half8_t qf[8];
  {
    const uint16_t* qp = a.q + ((int64_t)(sr.first + qj) * a.hq + g * G + (qi - qj * G)) * kHd + 8 * h;
#pragma unroll
    for (int x = 0; x < 8; ++x) qf[x] = *reinterpret_cast<const half8_t*>(qp + 16 * x);
    // they have arrived: a wait for them in the loop would be one for the keys in flight too
#pragma unroll
    for (int x = 0; x < 8; ++x) asm volatile("" : "+v"(qf[x]));
  }
  float m = kNoMax, l = 0.f;
  float16_t o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  const int krow = swap23(lc) * 16, vrow = lc * 8, vsw = (lc >> 1) & 7;
  int buf = 0;
  for (int round = st0; round < st1; round += KW) {  // (the same for all wavefronts: they meet at its barriers)
    const int st = round + kw, key0 = st * kTile;
    // uniform: some row of the workgroup may not read some key of the round
    const bool past = (round + KW - 1) * (int64_t)kTile + kTile - 1 > pmin;
    // step st is in its buffer, and every wavefront is done with step st - KW
    if constexpr (Q4) {
      __syncthreads();
      if (st + KW < st1) load_step(st + KW);
    } else {
      if (st + KW * (kRing - 2) < st1)  // the steps st + KW .. st + KW (kRing - 2) may stay in flight
        barrier_after_loads<(kRing - 2) * 2 * kLoads>();
      else
        barrier_after_loads<0>();
      if (st + KW * (kRing - 1) < st1) issue_step(st + KW * (kRing - 1), buf == 0 ? kRing - 1 : buf - 1);
      if (past) {
        if (st < st1 && key0 + kTile - 1 > pmin) tame_step(st, buf);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
      }
    }
    if (owner && key0 <= wmax && (KW == 1 || st < st1)) {  // uniform in the wavefront
      float16_t sc[2];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[b][i] = 0.f;
      // fragment i of the keys: half i % 2 of the tile, dimensions 16 (i / 2) .. +16; kDeep of them ahead of the products
      constexpr int kDeep = Q4 ? 2 : 8;
      u32x4 f[kDeep];
      auto key_frag = [&](int i) { return kb[kw * kRing + buf][(i & 1) * 512 + krow + ((2 * (i >> 1) + h) ^ (lc & 15))]; };
#pragma unroll
      for (int i = 0; i < kDeep; ++i) f[i] = key_frag(i);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const u32x4 w = f[i % kDeep];
        sc[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, w), qf[i >> 1], sc[i & 1], 0, 0, 0);
        if (i + kDeep < 16) f[i % kDeep] = key_frag(i + kDeep);
      }
      // fragment i of the values: dimensions 32 (i % 4) .. +32, keys 16 (i / 4) .. +16
      auto val_frag = [&](int i) { return vb[kw * kRing + buf][(i & 3) * 256 + vrow + ((2 * (i >> 2) + h) ^ vsw)]; };
#pragma unroll
      for (int i = 0; i < kDeep; ++i) f[i] = val_frag(i);
      const bool tail = key0 + kTile - 1 > wmin;  // uniform
      if (tail) {
        const int lim = (lpos - key0 < kTile ? lpos - key0 : kTile) - 8 * h;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            sc[b][i] = 32 * b + 16 * (i >> 3) + (i & 7) <= lim ? sc[b][i] : -__builtin_inff();
      }
      float cm = sc[0][0];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) cm = fmaxf(cm, sc[b][i]);
      cm = pair_fold(cm, [](float x, float y) { return fmaxf(x, y); });
      if (__any(cm > m + kSlack)) {
        const float mn = fmaxf(m, cm), alpha = rescale(m, mn);
        m = mn;
        l *= alpha;
#pragma unroll
        for (int d = 0; d < 4; ++d) o[d] *= alpha;
      }
      float ref = near_reference(m);
      if (far_reference(m)) {  // uniform
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) sc[b][i] -= m;
        ref = kShift;
      }
      half8_t pf[4];
      float sum = 0.f;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p = exp2_fast(__builtin_fmaf(sc[x >> 1][8 * (x & 1) + e], kScale, ref));
          sum += p;
          pf[x][e] = (half_t)p;
        }
      }
      l += sum;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const u32x4 w = f[i % kDeep];
        o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, w), pf[i >> 2], o[i & 3], 0, 0, 0);
        if (i + kDeep < 16) f[i % kDeep] = val_frag(i + kDeep);
      }
    }
    if constexpr (Q4) {
      if (st + KW < st1) store_step(st + KW, buf ^ 1);
    }
    buf = buf + 1 == kRing ? 0 : buf + 1;
  }
  if (KW == 1 && !owner) return;
  if (owner && odd_seen) {  // (written before the last step's barrier)
#pragma unroll 1
    for (int st = st0 + kw; st < st1; st += KW) {
      if (st * (int64_t)kTile + kTile - 1 <= pmin) continue;
#pragma unroll 1
      for (int key = st * kTile; key < st * kTile + kTile && key <= wmax && key <= klast; ++key) {
        const OddValue ov = odd_value<Q4>(a, sg, key);
        if (!__any(ov.v[0] != 0.f || ov.v[1] != 0.f)) continue;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float v = __shfl(ov.v[d >> 1], 32 * (d & 1) + 8 * (i >> 2) + 4 * h + (i & 3), kWave);
            o[d][i] += key <= lpos ? v : 0.f;
          }
      }
    }
  }
  l = pair_fold(l, [](float x, float y) { return x + y; });
  if constexpr (KW == 2) {  // the second group's sums to the first
    u32x4* ob = &kb[0][1024 * wave];  // (four wavefronts of 16 KB)
    float2* ml = reinterpret_cast<float2*>(&vb[0][64 * wave]);
    __syncthreads();  // every wavefront is done with the keys
    if (owner && kw == 1) {
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          ob[64 * (4 * d + x) + lane] =
              __builtin_bit_cast(u32x4, float4_t{o[d][4 * x], o[d][4 * x + 1], o[d][4 * x + 2], o[d][4 * x + 3]});
      ml[lane] = make_float2(m, l);
    }
    __syncthreads();
    if (!owner || kw == 1) return;
    const float2 other = ml[lane];
    const float mn = fmaxf(m, other.x), mine = rescale(m, mn), theirs = rescale(other.x, mn);
    m = mn;
    l = l * mine + other.y * theirs;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const u32x4 w = ob[64 * (4 * d + x) + lane];
        const float4_t v = __builtin_bit_cast(float4_t, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[d][4 * x + i] = o[d][4 * x + i] * mine + v[i] * theirs;
      }
  }
  if constexpr (SPLIT) {
    const int64_t at = (int64_t)blockIdx.x * TQ + 32 * wave + lc;
    float* po = a.part_o + at * kHd + 4 * h;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        *reinterpret_cast<float4_t*>(po + 32 * d + 8 * x) =
            float4_t{o[d][4 * x], o[d][4 * x + 1], o[d][4 * x + 2], o[d][4 * x + 3]};
    if (h == 0) a.part_ml[at] = make_float2(m, l);
  } else {
    const bool real = wq + lc < nq;
    const int64_t pos = p0 + qj;
    const bool bad = pos < 0 || pos >= a.len_bound;
    const float inv = 1.f / l;
    uint16_t* dst = a.out + ((int64_t)(sr.first + qj) * a.hq + g * G + (qi - qj * G)) * kHd + 8 * h;
    // the lane pairs of a query exchange halves of every 16 dimensions, for stores of 16 bytes
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int x = 0; x < 4; x += 2) {
        uint32_t w[2][2];  // dimensions 8 (x + j) + 4 h + 2 e, + 1
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const half2_t v = {(half_t)(o[d][4 * (x + j) + 2 * e] * inv), (half_t)(o[d][4 * (x + j) + 2 * e + 1] * inv)};
            w[j][e] = bad ? kNanF16 * 0x10001u : __builtin_bit_cast(uint32_t, v);
          }
        u32x4 c;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const auto s = __builtin_amdgcn_permlane32_swap(w[0][e], w[1][e], false, false);
          const uint32_t s0 = s[0], s1 = s[1];
          c[e] = s0;
          c[2 + e] = s1;
        }
        if (real) *reinterpret_cast<u32x4*>(dst + 32 * d + 8 * x) = c;
      }
  }
}

// The parts of query qi joined, in their order: lane i the weights of parts i, 64 + i, .. (at most kMost a lane), then every
// lane two dimensions, eight parts' sums in flight.  row0: the query's row of part 0's sums.
template <int kMost>
__device__ __forceinline__ void join(const AttnArgs& a, int G, int g, SeqRows sr, int64_t p0, int qi, int parts,
                                     int64_t row0, int64_t stride) {
  const int lane = threadIdx.x & 63;
  float2 ml[kMost];
  float M = kNoMax, L = 0.f;
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const int p = 64 * i + lane;
    ml[i] = make_float2(kNoMax, 0.f);
    if (p < parts) ml[i] = a.part_ml[row0 + p * stride];
    M = fmaxf(M, ml[i].x);
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) M = fmaxf(M, __shfl_xor(M, d, kWave));
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    ml[i].x = rescale(ml[i].x, M);
    L += ml[i].x * ml[i].y;
  }
  L = wave_sum(L);
  float x = 0.f, y = 0.f;
  const float* po = a.part_o + row0 * kHd + 2 * lane;
  for (int p0i = 0; p0i < parts; p0i += 8) {
    float2 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int p = p0i + i < parts ? p0i + i : parts - 1;
      v[i] = *reinterpret_cast<const float2*>(po + p * stride * kHd);
    }
    float fw = ml[0].x;
#pragma unroll
    for (int i = 1; i < kMost; ++i) fw = (p0i >> 6) == i ? ml[i].x : fw;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float f = p0i + i < parts ? __shfl(fw, (p0i & 63) + i, kWave) : 0.f;
      x += p0i + i < parts ? f * v[i].x : 0.f;
      y += p0i + i < parts ? f * v[i].y : 0.f;
    }
  }
  const int j = qi / G;
  const bool bad = p0 + j < 0 || p0 + j >= a.len_bound;
  const half_t nan = __builtin_bit_cast(half_t, kNanF16);
  half2_t r = {bad ? nan : (half_t)(x / L), bad ? nan : (half_t)(y / L)};
  *reinterpret_cast<half2_t*>(a.out + ((int64_t)(sr.first + j) * a.hq + g * G + (qi - j * G)) * kHd + 2 * lane) = r;
}

// Four queries of a tile a workgroup, one a wavefront (sixteen, in wavefronts or in turn: 7.1 and 11.2 us for 5.0).  A
// sequence's last workgroup could join few parts itself (16 tokens after 22k positions 43.7 us for 45.4), with counters that
// would have to be zero before every call: one pair of calls that overlap would leave them wrong for good.
__global__ __launch_bounds__(256) void packed_merge_kernel(PackedRows pr, AttnArgs a, int TQ, int grain, bool few) {
  const int wave = threadIdx.x >> 6;
  const int G = a.hq / a.hkv;
  const int item = blockIdx.x / a.hkv, g = blockIdx.x - item * a.hkv;
  Unit u;
  int first;
  {
    const Planner plan(pr.b, a.most, grain, [&](int i) { return seq_work(pr, a, G, TQ, i); });
    if (!plan.find_tile_parts(item, u, first)) return;
  }
  const SeqRows sr = u.rows;
  const int nq = sr.n * G, qt = few ? 0 : (nq + TQ - 1) / TQ - 1 - u.tile;
  const int64_t p0 = u.p0;
  const int qlast = (qt + 1) * TQ < nq ? (qt + 1) * TQ - 1 : nq - 1;
  const int nst = steps_to(last_key(p0 + qlast / G, a.len_bound));
  const int parts = nst > u.span ? (nst + u.span - 1) / u.span : 1;
  const int64_t stride = (int64_t)a.hkv * TQ;  // rows of the sums from one part to the next
  const int qx = blockIdx.y * 4 + wave;
  if (qt * TQ + qx >= nq || (few && parts == 1) || first + parts > a.most) return;  // (the latter as in the plan)
  const int64_t row0 = ((int64_t)first * a.hkv + g) * TQ + qx;
  if (parts <= kWave)
    join<1>(a, G, g, sr, p0, qt * TQ + qx, parts, row0, stride);
  else
    join<kMaxParts / kWave>(a, G, g, sr, p0, qt * TQ + qx, parts, row0, stride);
}

struct Plan {
  bool few;
  int tq, grain;    // queries of a tile; steps that a part's are a multiple of
  int tiles, most;  // tiles at most; parts at most (0: the keys are not split)
};

Plan make_plan(const PackedRows& pr, int hq, int hkv, int64_t len_bound, bool q4) {
  const int G = hq / hkv;
  const int64_t steps = (len_bound + kTile - 1) / kTile;
  const int64_t b = pr.b < pr.rows ? pr.b : pr.rows;
  Plan p;
  // Up to 32 queries (4-bit entries: 64), every wavefront its own keys; more share them through LDS.  28 query heads on 4,
  // few_attn_kernel and prompt_attn_kernel: fp16, 32 sequences of 4 rows after 2000 positions 32 and 39 us, of 9 rows (63
  // queries) 47 and 42, one of 9 18.5 and 14.1; 4-bit, 32 of 9 rows 32 and 41, one of 9 14.4 and 14.6.
  p.few = (int64_t)pr.max_rows * G <= (q4 ? 64 : 32);
  int64_t most = kMaxParts / hkv;  // a workgroup a CU
  if (p.few) {
    p.tq = pr.max_rows * G <= 16 ? 16 : (pr.max_rows * G <= 32 ? 32 : 64);
    p.tiles = pr.b;
    // Whole sequences from half a workgroup a CU: in up to 1024 parts, 64 sequences of one row after 2000 positions took
    // 62.7 us for 42.7 (4-bit: 36.7 for 17.1).  Parts of four steps at least (eight: one fp16 sequence after
    // 1000 positions 17.2 us for 12.8, after 4000 17.2 for 13.2).  The merge has to pay: one fp16 row over 8 steps takes 12.2 us
    // whole and 12.7 in parts, over 16 19.1 and 12.8; 4-bit, over 16 9.2 and 10.2, over 21 11.1 and 10.2; 9 rows (63 queries)
    // over 8 13.0 and 14.4, over 16 18.4 and 14.4.
    p.grain = 4;
    if (2 * b > most || steps <= (q4 && p.tq <= 32 ? 4 : 2) * p.grain) most = 0;
  } else {
    auto tiles = [&](int64_t tq) {
      return pr.start ? ((int64_t)pr.rows * G + b * (tq - 1)) / tq
                      : (int64_t)pr.b * (((int64_t)pr.max_rows * G + tq - 1) / tq);
    };
    // Tiles of 256 queries read the keys (and dequantise 4-bit ones) half as often, and leave more CUs idle at the end.  256
    // and 128 over fp16, then 4-bit entries, 28 query heads on 4: one prompt of 12000 rows 996 and 1000 us, 1090 and 1122;
    // eight of 2000 273 and 275, 293 and 308; sixteen of 1000 173 and 171, 188 and 186; one of 2000 55.7 and 49.2, 69.7 and
    // 58.9; forty of 200 49.9 and 46.9, both formats; four of 2000, 40 heads on 8, 204 and 200, 214 and 225.
    p.tq = tiles(256) * hkv >= 1536 ? 256 : 128;
    p.tiles = (int)tiles(p.tq);
    // Split: one sequence of 40 rows after 4000 positions 20.6 us for 76.  Tiles on half of the CUs or more stay whole.
    p.grain = kSplitGroups;
    if (2 * p.tiles > most || steps <= 4) most = 0;
  }
  p.most = (int)most;
  return p;
}

template <bool Q4>
void launch_few(const Plan& p, dim3 grid, const PackedRows& pr, const AttnArgs& a, hipStream_t stream) {
  const dim3 block(64 * kFewWaves);
  if (p.tq == 16)
    hipLaunchKernelGGL((few_attn_kernel<Q4, 1, 1>), grid, block, 0, stream, pr, a);
  else if (p.tq == 32)
    hipLaunchKernelGGL((few_attn_kernel<Q4, 2, 1>), grid, block, 0, stream, pr, a);
  else if constexpr (Q4)
    hipLaunchKernelGGL((few_attn_kernel<true, 2, 2>), grid, block, 0, stream, pr, a);
}

template <bool Q4>
void launch_prompt(const Plan& p, dim3 grid, const PackedRows& pr, const AttnArgs& a, hipStream_t stream) {
  if (p.tq == 256)  // (never split: so many tiles fill the chip)
    hipLaunchKernelGGL((prompt_attn_kernel<Q4, 8, 1, false>), grid, dim3(512), 0, stream, pr, a);
  else if (p.most)
    hipLaunchKernelGGL((prompt_attn_kernel<Q4, 4, kSplitGroups, true>), grid, dim3(256 * kSplitGroups), 0, stream, pr, a);
  else
    hipLaunchKernelGGL((prompt_attn_kernel<Q4, 4, 1, false>), grid, dim3(256), 0, stream, pr, a);
}

}  // namespace

hipError_t launch_packed_attention(const uint16_t* q, const PackedRows& pr, int hq, int hkv, const int32_t* pos_base,
                                   int pos_offset, int64_t len_bound, int64_t capacity, const KvCache& cache,
                                   uint16_t* out, hipStream_t stream) {
  const bool q4 = cache.k4 != nullptr;
  const Plan p = make_plan(pr, hq, hkv, len_bound, q4);
  AttnArgs a{q, cache, pos_base, pos_offset, hq, hkv, len_bound, capacity, out, nullptr, nullptr, p.most, p.grain, false};
  const int units = p.most ? p.most : p.tiles;
  if (p.most) {
    const size_t queries = (size_t)units * hkv * p.tq;
    void* ws = nullptr;
    const hipError_t e = workspace(queries * (kHd * sizeof(float) + sizeof(float2)), stream, &ws);
    if (e != hipSuccess) return e;
    a.part_o = static_cast<float*>(ws);
    a.part_ml = reinterpret_cast<float2*>(a.part_o + queries * kHd);
  }
  const dim3 grid((unsigned)(units * hkv));
  // Longest first where not all tiles run at once, for a few (sequence, kv head) pairs: tiles of more of them side by side
  // no longer find their keys in the L2s, and a tile's level is found by search, which one sequence (in this order as it
  // is) need not pay.  fp16 and 4-bit entries, 28 heads on 4: four prompts of 1171 rows 58.9 us for 61.2 and 63.9 for 69.2,
  // seven of 400, 800 .. 2800 209 for 213 and 223 for 232, eight of up to 2500 42.7 for 45.1 and 81.4 for 95.8; eight of 700
  // 54.3 for 52.1 and 55.5 for 57.9; ten of up to 2500 110 for 105 and 95.0 for 97.1; 29 of 64 .. 1856 360 for 350 and 374 for
  // 366; 40 heads on 8, four of up to 3000 72.3 for 75.6 and 128.4 for 126.5, eight 282 for 275 and 220 for 217.
  const int64_t seqs = pr.b < pr.rows ? pr.b : pr.rows;
  a.longest = !p.few && seqs > 1 && seqs * hkv <= 32 && (int64_t)units * hkv > (p.tq == 256 ? 256 : 512);
  if (p.few) {
    if (q4)
      launch_few<true>(p, grid, pr, a, stream);
    else
      launch_few<false>(p, grid, pr, a, stream);
  } else {
    if (q4)
      launch_prompt<true>(p, grid, pr, a, stream);
    else
      launch_prompt<false>(p, grid, pr, a, stream);
  }
  if (p.most)
    hipLaunchKernelGGL(packed_merge_kernel, dim3((unsigned)(p.tiles * hkv), (unsigned)(p.tq / 4)), dim3(256), 0, stream,
                       pr, a, p.tq, p.grain, p.few);
  return hipGetLastError();
}

}  // namespace sq

// Rows of several sequences packed one after the other, on their way into a cache: bias, rotary embedding and the
// cache write, fp16 or 4-bit, and the read of 4-bit entries as fp16.
//   packed_rope_kernel<false>  fp16 entries: keys [position][128], values position-minor [128][position]
//   packed_rope_kernel<true>   4-bit entries (sq_packed.hpp): keys [position][64 bytes], values in blocks of 64
//                              positions, [64 bytes][64 positions]
//   packed_read_kernel         4-bit entries of the packed rows' positions as fp16 rows
// All three are bound by memory: fp32 projections in, 16-bit queries and the entries out.  fp16, 13128 rows of 40 heads on
// 8 (565 MB): 128 us, 4.4 TB/s; a copy of 1 GiB reaches 4.8.  4-bit, 3091 rows of 28 heads on 4 (89 MB with the read): 20.2 us
// and 5.0 us for the read.  A few rows: 5.5 us, the launch, the list of tiles and two dependent loads.
#include "sq_internal.hpp"
#include "sq_packed.hpp"
#include "sq_quant.hpp"
#include "sq_rope.hpp"

namespace sq {
namespace {

constexpr int32_t kBadPos = 2, kBadRows = 16;  // the SQ_DEV_* values of the C headers

// A workgroup takes the rows of one sequence at 16 positions that start at a multiple of 16 (so that a run of values
// is whole words of memory), and the heads h with h % gridDim.y == blockIdx.y.
constexpr int kTileRows = 16;

struct RowTile {
  int s, row0, nr;   // sequence, first packed row, rows
  int64_t pos0;      // position of row0
  int shift;         // pos0 % 16
};

__device__ __forceinline__ bool row_tile(const PackedRows& pr, const int32_t* pos_base, int pos_offset, int item,
                                         RowTile& rt) {
  int s, t;
  if (!find_tile(pr.b, item,
                 [&](int i) {
                   const int n = seq_rows(pr, i).n;
                   const int sh = (int)(((int64_t)pos_base[i] + pos_offset) & (kTileRows - 1));
                   return n > 0 ? (n + sh + kTileRows - 1) / kTileRows : 0;
                 },
                 s, t))
    return false;
  const SeqRows sr = seq_rows(pr, s);
  const int64_t p0 = (int64_t)pos_base[s] + pos_offset;
  const int sh = (int)(p0 & (kTileRows - 1));
  const int a = t == 0 ? 0 : t * kTileRows - sh;  // first row of the tile within the sequence
  const int e = (t + 1) * kTileRows - sh;
  rt.s = s;
  rt.row0 = sr.first + a;
  rt.nr = (e < sr.n ? e : sr.n) - a;
  rt.pos0 = p0 + a;
  rt.shift = t == 0 ? sh : 0;
  return true;
}

// Workgroups go to the eight XCDs in turn, each with an L2 of its own.  Four tiles in a row hold the values of the same
// 128-byte lines (64 positions of a dimension): of every 32 workgroups, each XCD gets four tiles in a row.
__device__ __forceinline__ int tile_of_block() {
  const int b = blockIdx.x;
  return b < (gridDim.x & ~31) ? (b & ~31) + (b & 7) * 4 + (b >> 3 & 3) : b;
}

template <int Ctrl>
__device__ __forceinline__ half2_t dpp_min2(half2_t v) {
  const int o = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), Ctrl, 0xF, 0xF, false);
  return __builtin_elementwise_min(v, __builtin_bit_cast(half2_t, o));
}

// Scale, zero and four codes of a group of 64 halves held four to a lane by a row of 16 lanes: the arithmetic of
// quantize_int4_kernel (fp64 decisions from fp32 quotients), and where a code would stand for a value past the largest
// binary16, the next one towards the zero.  A group with a NaN or an infinity: codes 0, a NaN scale, zero 0.
struct Q4Group {
  uint16_t scale, zero;
  uint32_t code[4];
};
__device__ __forceinline__ Q4Group quantize_group(const half_t (&w)[4]) {
  half2_t ext = {(half_t)0, (half_t)0};  // minimum, minus maximum
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    bad |= (__builtin_bit_cast(uint16_t, w[i]) & 0x7C00) == 0x7C00;
    ext = __builtin_elementwise_min(ext, half2_t{w[i], -w[i]});
  }
  bad = ((__ballot(bad) >> (threadIdx.x & 48)) & 0xFFFFull) != 0;
  ext = dpp_min2<0xB1>(ext);   // quad_perm [1,0,3,2]
  ext = dpp_min2<0x4E>(ext);   // quad_perm [2,3,0,1]
  ext = dpp_min2<0x141>(ext);  // row_half_mirror
  ext = dpp_min2<0x140>(ext);  // row_mirror
  const float lo = (float)ext[0], hi = -(float)ext[1];
  const double range = bad || hi == lo ? 15.0 : (double)hi - (double)lo;
  const float s = (float)f16_ceil(range / 15.0);
  const float rs = recip(s);
  float z = bad ? 0.f : __builtin_rintf(quotient(-lo, s, rs));
  z = z > 0.f ? (z > 15.f ? 15.f : z) : 0.f;
  Q4Group r;
  r.scale = bad ? (uint16_t)0x7E00 : f32_to_f16_bits(s);
  r.zero = f32_to_f16_bits(z);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float c = __builtin_rintf(quotient((float)w[i], s, rs)) + z;
    c = __builtin_amdgcn_fmed3f(c, 0.f, 15.f);
    if (s >= 4368.f && fabsf((c - z) * s) >= 65520.f) c += c > z ? -1.f : 1.f;  // (exact: 4 by 11 bits)
    r.code[i] = bad ? 0u : (uint32_t)c;
  }
  return r;
}

struct RopeArgs {
  const float* qkv;
  const uint16_t* bias;
  const int32_t* pos_base;
  int pos_offset, hq, hkv;
  int64_t len_bound, capacity;
  RopeBase base;
  uint16_t* q_out;
  KvCache c;
  int32_t* status;
};

// Sixteen lanes take one (row, head): lane t the elements 4 t .. 4 t + 3 and 64 + those, which are four pairs of the
// rotation and one word of codes.  The 16 such groups of a workgroup take a row each and walk its heads, whose rows of
// the projection follow one another in memory, one load ahead; where a tile has fewer rows (blocks, single tokens),
// several groups share a row's heads.
template <bool Q4>
__global__ __launch_bounds__(256) void packed_rope_kernel(PackedRows pr, RopeArgs a) {
  __shared__ float2 tab[kTileRows][64];                             // cosine, sine of (row, pair)
  __shared__ __align__(16) uint16_t vt[Q4 ? 1 : kTileRows][kHd + 4];  // one head's values
  __shared__ __align__(16) uint8_t vc4[Q4 ? kTileRows : 1][68];
  __shared__ uint16_t vs4[Q4 ? 4 : 1][kTileRows];
  const int tid = threadIdx.x, t0 = 4 * (tid & 15), unit = tid >> 4;
  const double freq = rope_freq(tid & 63, a.base);  // (beside the loads of the rows' bounds)
  if (pr.start && a.status && blockIdx.x == 0 && blockIdx.y == 0) {
    for (int s = tid; s < pr.b; s += 256) {
      const int x = pr.start[s], y = pr.start[s + 1];
      if (x < 0 || y < x || y > pr.rows || y - x > pr.max_rows) flag(a.status, kBadRows);
    }
  }
  RowTile rt;
  if (!row_tile(pr, a.pos_base, a.pos_offset, tile_of_block(), rt)) return;  // uniform
  const int nh = a.hq + 2 * a.hkv, turned = a.hq + a.hkv, share = blockIdx.y, shares = gridDim.y;
  const int per = (turned + shares - 1) / shares, head0 = share * per;
  const int head1 = head0 + per < turned ? head0 + per : turned;
  const int lg = rt.nr > 8 ? 0 : (rt.nr > 4 ? 1 : (rt.nr > 2 ? 2 : (rt.nr > 1 ? 3 : 4)));  // 2^lg groups a row
  const int r = unit >> lg, step = 1 << lg;
  const bool busy = r < rt.nr;
  struct Raw {
    float4_t lo, hi;
    half4_t bl, bh;
  };
  auto load = [&](int row, int hh) {
    Raw w;
    const float* src = a.qkv + ((int64_t)(rt.row0 + row) * nh + hh) * kHd + t0;
    w.lo = *reinterpret_cast<const float4_t*>(src);
    w.hi = *reinterpret_cast<const float4_t*>(src + 64);
    if (a.bias) {
      w.bl = *reinterpret_cast<const half4_t*>(a.bias + hh * kHd + t0);
      w.bh = *reinterpret_cast<const half4_t*>(a.bias + hh * kHd + t0 + 64);
    }
    return w;
  };
  auto add_bias = [&](Raw& w) {
    if (a.bias) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        w.lo[x] += (float)w.bl[x];
        w.hi[x] += (float)w.bh[x];
      }
    }
  };
  int hh = head0 + (unit & (step - 1));
  Raw next;
  if (busy && hh < head1) next = load(r, hh);
  for (int i = tid >> 6; i < rt.nr; i += 4) tab[i][tid & 63] = rope_cos_sin(rt.pos0 + i, freq);
  __syncthreads();
  auto valid = [&](int row) { return rt.pos0 + row >= 0 && rt.pos0 + row < a.len_bound; };
  if (share == 0 && tid < rt.nr && !valid(tid)) flag(a.status, kBadPos);
  if (busy) {
    const bool ok = valid(r);
    for (; hh < head1; hh += step) {
      Raw w = next;
      if (hh + step < head1) next = load(r, hh + step);
      add_bias(w);
      half4_t ol, oh;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        float ra, re;
        rope_turn(w.lo[x], w.hi[x], tab[r][t0 + x], ra, re);
        ol[x] = (half_t)ra;
        oh[x] = (half_t)re;
      }
      if (hh < a.hq) {
        const half_t nan = __builtin_bit_cast(half_t, kNanF16);
        if (!ok) ol = oh = half4_t{nan, nan, nan, nan};
        uint16_t* dst = a.q_out + ((int64_t)(rt.row0 + r) * a.hq + hh) * kHd + t0;
        *reinterpret_cast<half4_t*>(dst) = ol;
        *reinterpret_cast<half4_t*>(dst + 64) = oh;
      } else if (Q4) {
        const half_t wl[4] = {ol[0], ol[1], ol[2], ol[3]}, wh[4] = {oh[0], oh[1], oh[2], oh[3]};
        const Q4Group gl = quantize_group(wl), gh = quantize_group(wh);
        if (ok) {
          const int64_t e = ((int64_t)rt.s * a.hkv + (hh - a.hq)) * a.capacity + rt.pos0 + r;
          uint32_t c = 0;
#pragma unroll
          for (int x = 0; x < 4; ++x) c |= (gl.code[x] | gh.code[x] << 4) << (8 * swap01(x));
          reinterpret_cast<uint32_t*>(a.c.k4)[e * 16 + (tid & 15)] = c;
          if ((tid & 15) == 0)
            reinterpret_cast<uint2*>(a.c.ks)[e] = make_uint2(gl.scale | (uint32_t)gl.zero << 16,
                                                             gh.scale | (uint32_t)gh.zero << 16);
        }
      } else if (ok) {
        uint16_t* dst = a.c.k + (((int64_t)rt.s * a.hkv + (hh - a.hq)) * a.capacity + rt.pos0 + r) * kHd + t0;
        *reinterpret_cast<half4_t*>(dst) = ol;
        *reinterpret_cast<half4_t*>(dst + 64) = oh;
      }
    }
  }
  // values: a group a row; each head's rows meet in LDS and leave as runs of positions
  const int64_t base = rt.pos0 - rt.shift;  // a multiple of 16
  auto inside = [&](int c) { return c >= rt.shift && c < rt.shift + rt.nr && valid(c - rt.shift); };
  const bool mine = unit < rt.nr;
  const int c = rt.shift + unit;  // the row's place among the 16 positions
  if (mine && share < a.hkv) next = load(unit, turned + share);
  for (int g = share; g < a.hkv; g += shares) {
    const int64_t sg = (int64_t)rt.s * a.hkv + g;
    if (g != share) __syncthreads();
    if (mine) {
      Raw w = next;
      add_bias(w);
      half_t wl[4], wh[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        wl[x] = (half_t)w.lo[x];
        wh[x] = (half_t)w.hi[x];
      }
      if constexpr (Q4) {
        const Q4Group gl = quantize_group(wl), gh = quantize_group(wh);
        uint32_t b = 0;
#pragma unroll
        for (int x = 0; x < 4; ++x) b |= (gl.code[x] | gh.code[x] << 4) << (8 * x);
        *reinterpret_cast<uint32_t*>(&vc4[c][t0]) = b;
        if ((tid & 15) == 0) {
          vs4[0][c] = gl.scale;
          vs4[1][c] = gl.zero;
          vs4[2][c] = gh.scale;
          vs4[3][c] = gh.zero;
        }
      } else {
        *reinterpret_cast<half4_t*>(&vt[c][t0]) = half4_t{wl[0], wl[1], wl[2], wl[3]};
        *reinterpret_cast<half4_t*>(&vt[c][t0 + 64]) = half4_t{wh[0], wh[1], wh[2], wh[3]};
      }
    }
    if (mine && g + shares < a.hkv) next = load(unit, turned + g + shares);
    __syncthreads();
    if constexpr (Q4) {
      // thread: byte row j, four positions, whose bytes lie exchanged
      const int j = tid & 63, p = 4 * (tid >> 6);
      uint8_t* dst = a.c.v4 + sg * a.capacity * 64 + (base >> 6) * 4096 + j * 64 + (base & 63) + p;
      if (inside(p) && inside(p + 1) && inside(p + 2) && inside(p + 3)) {
        *reinterpret_cast<uint32_t*>(dst) =
            vc4[p][j] | vc4[p + 2][j] << 8 | vc4[p + 1][j] << 16 | (uint32_t)vc4[p + 3][j] << 24;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (inside(p + i)) dst[swap01(i)] = vc4[p + i][j];
      }
      if (tid < 64 && inside(tid & 15))
        a.c.vs[sg * a.capacity * 4 + (base >> 6) * 256 + (base & 63) + (tid >> 4) * 64 + (tid & 15)] =
            vs4[tid >> 4][tid & 15];
    } else {
      // thread: dimension d, eight positions
      const int d = tid & 127, p = 8 * (tid >> 7);
      uint16_t* dst = a.c.v + (sg * kHd + d) * a.capacity + base + p;
      uint16_t e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = vt[p + i][d];
      bool all = true;
#pragma unroll
      for (int i = 0; i < 8; ++i) all &= inside(p + i);
      if (all) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = e[2 * i] | (uint32_t)e[2 * i + 1] << 16;
        *reinterpret_cast<u32x4*>(dst) = w;
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (inside(p + i)) dst[i] = e[i];
      }
    }
  }
}

// The values f16((q - z) s) of the entries at the packed rows' positions; rows at bad positions: NaN.
__global__ __launch_bounds__(256) void packed_read_kernel(PackedRows pr, const int32_t* __restrict__ pos_base,
                                                          int pos_offset, int hkv, int64_t len_bound, int64_t capacity,
                                                          KvCache c, uint16_t* __restrict__ k_out,
                                                          uint16_t* __restrict__ v_out) {
  __shared__ __align__(16) uint8_t vb[64][kTileRows];
  const int tid = threadIdx.x, t = tid & 15, unit = tid >> 4;
  RowTile rt;
  if (!row_tile(pr, pos_base, pos_offset, tile_of_block(), rt)) return;  // uniform
  const int64_t base = rt.pos0 - rt.shift;
  const CodeConsts kc;
  for (int g = blockIdx.y; g < hkv; g += gridDim.y) {
    const int64_t sg = (int64_t)rt.s * hkv + g;
    __syncthreads();
    if (tid < 64 && base >= 0 && base < len_bound)
      *reinterpret_cast<u32x4*>(vb[tid]) = *reinterpret_cast<const u32x4*>(c.v4 + sg * capacity * 64 +
                                                                           (base >> 6) * 4096 + tid * 64 + (base & 63));
    __syncthreads();
    for (int r = unit; r < rt.nr; r += 16) {
      const int64_t pos = rt.pos0 + r;
      const bool ok = pos >= 0 && pos < len_bound;
      const int64_t o = ((int64_t)(rt.row0 + r) * hkv + g) * kHd + 4 * t;
      uint32_t kw = 0, vw = 0;
      uint16_t sz[2][4];
      if (ok) {
        kw = reinterpret_cast<const uint32_t*>(c.k4)[(sg * capacity + pos) * 16 + t];
        const int cc = swap01(rt.shift + r);
#pragma unroll
        for (int x = 0; x < 4; ++x) vw |= (uint32_t)vb[4 * t + x][cc] << (8 * swap01(x));
        const uint16_t* ks = c.ks + (sg * capacity + pos) * 4;
        const uint16_t* vs = c.vs + sg * capacity * 4 + (pos >> 6) * 256 + (pos & 63);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          sz[0][x] = ks[x];
          sz[1][x] = vs[64 * x];
        }
      } else {
#pragma unroll
        for (int x = 0; x < 4; ++x) sz[0][x] = sz[1][x] = kNanF16;
      }
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        uint16_t* dst = (w ? v_out : k_out) + o;
        const half2_t s0 = bits_h2(sz[w][0] * 0x10001u), z0 = bits_h2(sz[w][1] * 0x10001u);
        const half2_t s1 = bits_h2(sz[w][2] * 0x10001u), z1 = bits_h2(sz[w][3] * 0x10001u);
        half2_t p, q;
        code_pairs<false>(kc, w ? vw : kw, p, q);
        p = (p - zero_pair<false>(z0)) * s0;
        q = (q - zero_pair<false>(z0)) * s0;
        *reinterpret_cast<half4_t*>(dst) = half4_t{p[0], p[1], q[0], q[1]};
        code_pairs<true>(kc, w ? vw : kw, p, q);
        p = (p - zero_pair<true>(z1)) * s1;
        q = (q - zero_pair<true>(z1)) * s1;
        *reinterpret_cast<half4_t*>(dst + 64) = half4_t{p[0], p[1], q[0], q[1]};
      }
    }
  }
}

// Workgroups that cover every row tile: a sequence of n rows has at most (n + 30) / 16.
int64_t tile_bound(const PackedRows& pr) {
  if (!pr.start) return (int64_t)pr.b * ((pr.max_rows + 2 * kTileRows - 2) / kTileRows);
  const int64_t b = pr.b < pr.rows ? pr.b : pr.rows;
  return (pr.rows + b * (2 * kTileRows - 2)) / kTileRows;
}

// Shares of the heads: about four workgroups per CU, no share without a whole pass of 16 (row, head) units.
unsigned head_shares(const PackedRows& pr, int64_t tiles, int heads) {
  int64_t shares = ((int64_t)cu_count() * 4 + tiles - 1) / tiles;
  const int64_t rows = pr.max_rows < kTileRows ? pr.max_rows : kTileRows;
  const int64_t most = (rows * heads + 15) / 16;
  shares = shares > most ? most : shares;
  return (unsigned)(shares < 1 ? 1 : (shares > heads ? heads : shares));
}

}  // namespace

hipError_t launch_packed_rope_kv(const float* qkv, const uint16_t* bias, const PackedRows& pr, int hq, int hkv,
                                 const int32_t* pos_base, int pos_offset, int64_t len_bound, int64_t capacity,
                                 double theta, uint16_t* q_out, const KvCache& cache, int32_t* status,
                                 hipStream_t stream) {
  const int64_t tiles = tile_bound(pr);
  const dim3 grid((unsigned)tiles, head_shares(pr, tiles, hq + hkv));
  const RopeArgs a{qkv, bias, pos_base, pos_offset, hq, hkv, len_bound, capacity, rope_base(theta), q_out, cache, status};
  if (cache.k4)
    hipLaunchKernelGGL(packed_rope_kernel<true>, grid, dim3(256), 0, stream, pr, a);
  else
    hipLaunchKernelGGL(packed_rope_kernel<false>, grid, dim3(256), 0, stream, pr, a);
  return hipGetLastError();
}

hipError_t launch_packed_kv_read(const PackedRows& pr, int hkv, const int32_t* pos_base, int pos_offset,
                                 int64_t len_bound, int64_t capacity, const KvCache& cache, uint16_t* k_out,
                                 uint16_t* v_out, hipStream_t stream) {
  const int64_t tiles = tile_bound(pr);
  const dim3 grid((unsigned)tiles, head_shares(pr, tiles, hkv));
  hipLaunchKernelGGL(packed_read_kernel, grid, dim3(256), 0, stream, pr, pos_base, pos_offset, hkv, len_bound, capacity,
                     cache, k_out, v_out);
  return hipGetLastError();
}

}  // namespace sq

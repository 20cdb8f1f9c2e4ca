// Packed rows of several sequences, and the 4-bit cache format (gfx950 device code).
#pragma once

#include "sq_attn.hpp"
#include "sq_internal.hpp"

namespace sq {

// Rows of sequence s: start[s] .. start[s + 1] (at most max_rows of them, clipped to [0, rows)); without `start` every
// sequence has max_rows rows.  Out-of-range or decreasing entries give clipped or no rows, never an access outside.
struct SeqRows {
  int first, n;
};
__device__ __forceinline__ SeqRows seq_rows(const PackedRows& p, int s) {
  if (!p.start) return {s * p.max_rows, p.max_rows};
  int a = p.start[s], e = p.start[s + 1];
  a = a < 0 ? 0 : (a > p.rows ? p.rows : a);
  e = e < a ? a : (e > p.rows ? p.rows : e);
  const int n = e - a;
  return {a, n < p.max_rows ? n : p.max_rows};
}

// Item `item` of the list (sequence 0: tile 0, 1, ..; sequence 1: ..), with tiles(s) tiles in sequence s, found by
// every wavefront for itself: 64 sequences a step, one scan of their counts.  False past the end of the list.
template <class F>
__device__ __forceinline__ bool find_tile(int b, int item, F tiles, int& s, int& t) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int base = 0; base < b; base += kWave) {
    const int n = base + lane < b ? tiles(base + lane) : 0;
    int incl = n;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
      const int o = __shfl_up(incl, d, kWave);
      incl += lane >= d ? o : 0;
    }
    const int total = __builtin_amdgcn_readlane(incl, kWave - 1);
    if (item < before + total) {
      const int l = __builtin_ctzll(__ballot(before + incl > item));
      s = base + l;
      t = item - before - (__builtin_amdgcn_readlane(incl, l) - __builtin_amdgcn_readlane(n, l));
      return true;
    }
    before += total;
  }
  return false;
}

// ------------------------------------------------------------ 4-bit entries
// An entry of 128 elements is two groups of 64 with a scale and a zero each; byte j holds the codes of elements j (low
// nibble) and j + 64 (high).  Four consecutive bytes (of a key: elements; of a block of values: positions) lie in the
// order 0, 2, 1, 3, so that one mask of a word gives a pair of neighbours.
__device__ __forceinline__ int swap01(int i) { return (i & ~3) | ((i & 1) << 1) | ((i >> 1) & 1); }

__device__ __forceinline__ half2_t bits_h2(uint32_t u) { return __builtin_bit_cast(half2_t, u); }

// Word `w` of four bytes to halves: codes 0 .. 3's low (HIGH: high) nibbles as 1024 + c (64 + c): c in the lowest (the
// lowest bits but four) mantissa bits, one v_and_or_b32 a pair.  That instruction takes no literals: the masks are held
// in scalar, the other constants in vector registers, opaque to the compiler, which would split it otherwise.
struct CodeConsts {
  uint32_t mask[2], one[2];
  __device__ __forceinline__ CodeConsts() : mask{0x000F000Fu, 0x00F000F0u}, one{0x64006400u, 0x54005400u} {
    asm("" : "+s"(mask[0]), "+s"(mask[1]), "+v"(one[0]), "+v"(one[1]));
  }
};
template <bool HIGH>
__device__ __forceinline__ void code_pairs(const CodeConsts& k, uint32_t w, half2_t& a, half2_t& b) {
  a = bits_h2((w & k.mask[HIGH]) | k.one[HIGH]);
  b = bits_h2(((w >> 8) & k.mask[HIGH]) | k.one[HIGH]);
}
// What code_pairs adds to the zero: (1024 + c) - (1024 + z) is exact.
template <bool HIGH>
__device__ __forceinline__ half2_t zero_pair(half2_t z) {
  const half_t o = HIGH ? (half_t)64.f : (half_t)1024.f;
  return z + half2_t{o, o};
}

}  // namespace sq

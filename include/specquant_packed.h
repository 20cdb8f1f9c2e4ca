/*
 * specquant_packed.h -- packed sequences, and a key/value cache held in 4 bits.
 *
 * The rotation with its cache write and the attention of specquant.h for rows of
 * several sequences packed one after the other, each sequence with a number of
 * rows of its own: whole prompts of different lengths without padding, parts of
 * prompts after cached ones, drafted blocks, single tokens.  Each comes over the fp16
 * cache of specquant.h and over a cache of 4-bit entries, which takes 144 bytes
 * per position and kv head instead of 512.  A draft may keep such a cache: accepting
 * keeps the parent's distribution whatever the draft's distribution is.  The
 * conventions of specquant.h hold (device pointers, alignment, statuses, the library
 * workspace, one stream per device, SQ_DEV_* bits).
 *
 * Packed rows.  row_start [b + 1] (device, int32): sequence s has the rows
 * row_start[s] .. row_start[s + 1] - 1 of `rows` rows, none where the two are equal.
 * max_rows is a bound on one sequence's rows, known on the host.  It chooses the
 * attention's kernel, and with the rows whether keys are split, for all sequences
 * alike: single tokens after long caches packed with a prompt get the prompt's, one
 * workgroup each (16 tokens after 31000 positions and a prompt of 512 rows, 28 query
 * heads on 4: 557 us, 751 over 4-bit entries).  Two calls over the same packed rows
 * take 196 and 78: the tokens' sequences first, then one call whose row_start is
 * clipped to at most their number of rows, with max_rows 1, and one whose row_start
 * is clipped to at least that (the other sequences are empty, their rows are left).
 * Row row_start[s] + j is at position pos_base[s] + pos_offset + j.
 * Rows before the first and after the last sequence's are left as they were.
 * row_start NULL: max_rows rows for every sequence (rows = b max_rows).
 * Entries of row_start that decrease or lie outside [0, rows], or a sequence of more
 * than max_rows rows: the writing calls set SQ_DEV_BAD_ROWS, and which of the
 * outputs of such a call are written is unspecified (nothing else is).
 *
 * Limits of every call: 1 <= b, b hkv <= 65535; 0 <= rows <= 2^20 (0: nothing to
 * do); 1 <= max_rows <= 2^20; heads, capacity and len_bound as for sq_rope_kv_f16.
 *
 * 4-bit entries.  An fp16 key or value of 128 elements becomes two groups of 64
 * elements (0 .. 63 and 64 .. 127), each with a scale and a zero as
 * sq_quantize_int4_g128 forms them for its groups of 128:
 *   lo = min(0, min w), hi = max(0, max w);  a group of zeros: s = 1, z = 0, q = 0
 *   else s = smallest fp16 >= (hi - lo) / 15, z = clamp(rint(-lo / s), 0, 15),
 *        q = clamp(rint(w / s) + z, 0, 15), of the codes that stand for a finite
 *        fp16 (where |(q - z) s| >= 65520 the next one towards z);
 *   a group with a NaN or an infinity: s = NaN, z = 0, q = 0.
 * The entry stands for f16((q - z) s): |w - that| <= s / 2 + half an fp16 ulp (s
 * where a code had to step).  Layout, of one layer:
 *   k_codes  [b][hkv][capacity][64] u8      byte e(j) of a position holds the codes of
 *                                           elements j (low nibble) and j + 64 (high)
 *   k_scales [b][hkv][capacity][4] fp16     scale and zero of elements 0 .. 63, then
 *                                           those of 64 .. 127
 *   v_codes  [b][hkv][capacity / 64][64][64] u8  per block of 64 positions: byte e(t) of
 *                                           row j holds elements j and j + 64 of the
 *                                           block's position t
 *   v_scales [b][hkv][capacity / 64][4][64] fp16 the four of k_scales, by position
 * with e(i) = i with its two lowest bits exchanged.  All four 16-byte aligned.
 */
#ifndef SPECQUANT_PACKED_H
#define SPECQUANT_PACKED_H

#include "specquant.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SQ_DEV_BAD_ROWS 16 /* row_start decreases, leaves [0, rows] or exceeds max_rows */

/* sq_rope_kv_f16 of packed rows (the same bits): bias, rotation, queries to q_out
 * [rows][hq][128] fp16, entries to the cache.  qkv [rows][(hq + 2 hkv) * 128] f32.
 * A row at a position outside [0, len_bound) writes no entry, gets NaN in q_out and
 * sets SQ_DEV_BAD_POS. */
sq_status sq_packed_rope_kv_f16(const float* qkv, const uint16_t* bias, const int32_t* row_start, int32_t b,
                                int64_t rows, int64_t max_rows, int32_t hq, int32_t hkv, const int32_t* pos_base,
                                int32_t pos_offset, int64_t len_bound, int64_t capacity, double theta,
                                uint16_t* q_out, uint16_t* k_cache, uint16_t* v_cache, int32_t* status,
                                hipStream_t stream);
/* The same into a 4-bit cache: the 4-bit entries of the fp16 ones that
 * sq_packed_rope_kv_f16 writes. */
sq_status sq_packed_rope_kv_q4(const float* qkv, const uint16_t* bias, const int32_t* row_start, int32_t b,
                               int64_t rows, int64_t max_rows, int32_t hq, int32_t hkv, const int32_t* pos_base,
                               int32_t pos_offset, int64_t len_bound, int64_t capacity, double theta, uint16_t* q_out,
                               uint8_t* k_codes, uint16_t* k_scales, uint8_t* v_codes, uint16_t* v_scales,
                               int32_t* status, hipStream_t stream);

/* The fp16 values of the 4-bit entries at the packed rows' positions: k_out, v_out
 * [rows][hkv][128] fp16 (NaN for a row at a position outside [0, len_bound)). */
sq_status sq_packed_kv_read_q4(const uint8_t* k_codes, const uint16_t* k_scales, const uint8_t* v_codes,
                               const uint16_t* v_scales, const int32_t* row_start, int32_t b, int64_t rows,
                               int64_t max_rows, int32_t hkv, const int32_t* pos_base, int32_t pos_offset,
                               int64_t len_bound, int64_t capacity, uint16_t* k_out, uint16_t* v_out,
                               hipStream_t stream);

/* Causal grouped-query attention of packed rows over the cache: out[r][h] as
 * sq_attention_f16 has it, for any number of rows per sequence; scores, softmax
 * sums and outputs in fp32, a weight rounded for its product with the value to two
 * fp16 terms (2^-20 of it) where max_rows hq / hkv <= 32, to one (2^-11) above.
 * q, out [rows][hq][128] fp16.  A row reads its sequence's positions 0 .. its own, which must hold written entries; what is at later positions does
 * not matter (NaN and infinities included); an infinite value it reads with a weight
 * below 2^-31 of its largest may give NaN.  A row at a position outside [0, len_bound)
 * gets NaN.  Few workgroups for the chip: the keys are split over up to 256
 * workgroups, whose sums take at most 17 MiB of the library workspace.
 * capacity <= 2^28. */
sq_status sq_packed_attention_f16(const uint16_t* q, const uint16_t* k_cache, const uint16_t* v_cache,
                                  const int32_t* row_start, int32_t b, int64_t rows, int64_t max_rows, int32_t hq,
                                  int32_t hkv, const int32_t* pos_base, int32_t pos_offset, int64_t len_bound,
                                  int64_t capacity, uint16_t* out, hipStream_t stream);
/* The same over a 4-bit cache: the attention over the fp16 values its entries
 * stand for, each weight as one fp16 term. */
sq_status sq_packed_attention_q4(const uint16_t* q, const uint8_t* k_codes, const uint16_t* k_scales,
                                 const uint8_t* v_codes, const uint16_t* v_scales, const int32_t* row_start, int32_t b,
                                 int64_t rows, int64_t max_rows, int32_t hq, int32_t hkv, const int32_t* pos_base,
                                 int32_t pos_offset, int64_t len_bound, int64_t capacity, uint16_t* out,
                                 hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* SPECQUANT_PACKED_H */

/*
 * specquant_paged.h -- key/value caches of pages that sequences share.
 *
 * A page holds 64 positions of one layer's keys and values, all kv heads.  A cache is a pool of `pages` pages per
 * layer, and per sequence a row of page ids: positions 64 i .. 64 i + 63 of sequence s lie in page table[s][i] of every
 * layer's pool (several pools, the parent's and a draft's, may go by one table).  Sequences take pages as they grow and
 * give them back, and sequences with a common prefix hold the same pages for it, so memory follows the tokens that are
 * there, not batch times capacity.  64 positions are a step of the attention kernels, so a step never crosses a page;
 * a page of one layer and 4 kv heads is 128 KB in fp16.  The conventions of specquant.h and the packed rows of
 * specquant_packed.h hold (device pointers, alignment, statuses, the library workspace, one stream per device,
 * SQ_DEV_* bits, row_start).
 *
 * The state of a pool (device, int32, caller-owned; all zero but table, which is -1 everywhere, where nothing is held):
 *   table [b][width]  page ids; row s has held[s] of them, then -1
 *   held  [b]         pages of row s, 0 .. width
 *   refs  [pages]     rows that hold a page; 0: it is free
 * The calls that change it run on one workgroup each but for the tables of sq_pages_trim and sq_pages_compact; they take
 * free pages lowest id first, so their results do not depend on any order of execution.  Rows whose held is outside
 * [0, width] are left as they are, page ids outside [0, pages) are never followed; both set SQ_DEV_BAD_PAGE.
 * Limits: 1 <= b <= 65535, 1 <= width <= 2^20, 1 <= pages <= 2^20.
 */
#ifndef SPECQUANT_PAGED_H
#define SPECQUANT_PAGED_H

#include "specquant_packed.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SQ_PAGE 64          /* positions of a page */
#define SQ_DEV_NO_PAGES 32  /* a row that needs more pages than are free, or than its table's width: it got none */
#define SQ_DEV_BAD_PAGE 64  /* a page id outside the pool, or held outside the table */
#define SQ_DEV_BAD_FORK 128 /* a fork that names no possible pair of rows: it was left out */

/* Room for the positions below pos_base[s] + ahead: row s gets the pages it lacks, in the order of the rows, as long as
 * free pages last.  The first row for which too few are left gets none, like every later one that needs any.  A row that
 * needs more than its table's width gets none either, and keeps none from the others.  Each sets SQ_DEV_NO_PAGES.
 * pos_base[s] < 0: the row is left alone.  Nothing is taken back.  Pages come as they were left: positions for which a row
 * found no page while they were computed hold nothing of it later.
 * pos_base [b]; 0 <= ahead <= 2^20.  Workspace: 4 bytes a page. */
sq_status sq_pages_reserve(int32_t* table, int32_t* held, int32_t* refs, int32_t b, int64_t width, int64_t pages,
                           const int32_t* pos_base, int32_t ahead, int32_t* status, hipStream_t stream);

/* Row s gives back its pages past position keep[s] (0: all of them); keep[s] < 0: the row is left alone.  A page is
 * free when its last holder has given it back.  keep [b]. */
sq_status sq_pages_trim(int32_t* table, int32_t* held, int32_t* refs, int32_t b, int64_t width, int64_t pages,
                        const int32_t* keep, int32_t* status, hipStream_t stream);

/* Row child[i], which must hold no pages, gets the first length[i] positions of row parent[i] (1 .. 64 held[parent]):
 * whole pages are shared, a partly filled last one becomes a page of its own, whose copy is left to sq_page_copy:
 * src, dst [n] and count [1] get the pages to copy, in the order of i.  So a child's positions from length[i] on may be
 * written; a position before that, only where length[i] was rounded down to it (for a cache whose last entry is written
 * again, fork one position less).  child[i] < 0: nothing.  A pair with a row outside [0, b), a child that holds pages or
 * that an earlier pair names, or an impossible length is left out (SQ_DEV_BAD_FORK); where free pages run out, as in
 * sq_pages_reserve.  0 <= n <= 1024 (0: count = 0).  Workspace: 4 bytes a page. */
sq_status sq_pages_fork(int32_t* table, int32_t* held, int32_t* refs, int32_t b, int64_t width, int64_t pages,
                        const int32_t* parent, const int32_t* child, const int32_t* length, int32_t n, int32_t* src,
                        int32_t* dst, int32_t* count, int32_t* status, hipStream_t stream);

/* The u = used[0] pages in use move to the ids 0 .. u - 1 (those at or past u to the free ids below, both in ascending
 * order) in refs and in every table row; src, dst [pages / 2] and count [1] get the pages whose content sq_page_copy then
 * has to move.  Afterwards the pages from u on are free: the tail of the pool can serve something else.  (width and held
 * stay.)  Workspace: 4 bytes a page. */
sq_status sq_pages_compact(int32_t* table, const int32_t* held, int32_t* refs, int32_t b, int64_t width, int64_t pages,
                           int32_t* src, int32_t* dst, int32_t* count, int32_t* used, int32_t* status,
                           hipStream_t stream);

/* Page dst[i] = page src[i], i < count[0] (at most n), in every layer of one array of a pool: [layers][pages][page_bytes].
 * No page may be a destination twice, or a destination and another pair's source (what such pages then hold is
 * unspecified); src[i] = dst[i] does nothing; pairs with an id outside [0, pages) are left out (SQ_DEV_BAD_PAGE).
 * src, dst [n]; 1 <= layers <= 65535; page_bytes a multiple of 16, at most 2^30; layers pages page_bytes < 2^46;
 * 0 <= n <= 2^20. */
sq_status sq_page_copy(void* pool, int32_t layers, int64_t pages, int64_t page_bytes, const int32_t* src,
                       const int32_t* dst, const int32_t* count, int64_t n, int32_t* status, hipStream_t stream);

/* The calls of specquant_packed.h over pages: every argument as there but for the cache, which is a layer's pool
 *   k_pages [pages][hkv][64][128], v_pages [pages][hkv][128][64] fp16 (values position-minor), or
 *   k_codes [pages][hkv][64][64], v_codes [pages][hkv][64][64] u8, k_scales [pages][hkv][64][4], v_scales
 *   [pages][hkv][4][64] fp16 (one block of 64 positions each of the 4-bit cache's layout)
 * with table [b][width] in the place of the capacity; 1 <= len_bound <= 64 width, width and pages as above.
 * Results are the bits of those calls over a cache with the same entries and capacity, but for the attention of few rows
 * (at most 32 queries of a kv head, 4-bit 64) of more than 128 / hkv sequences: there those calls take a sequence's keys
 * whole, and these cut all sequences' keys into equal shares, whose sums take at most 34 MiB of the library workspace.
 * A position whose table entry is outside [0, pages) has no entry: a row there is treated as one at a bad position
 * (nothing written, NaN in q_out, k_out and v_out) and sets SQ_DEV_BAD_PAGE; a row that reads one gets NaN in out.
 * Writing into a page that several rows hold changes it for all of them.
 * A sequence with pos_base[s] = SQ_POS_IDLE has no rows, whatever row_start gives it: they are left as they were, and no
 * bit is set.  So rows of a batch may be idle without pages. */
sq_status sq_paged_rope_kv_f16(const float* qkv, const uint16_t* bias, const int32_t* row_start, int32_t b,
                               int64_t rows, int64_t max_rows, int32_t hq, int32_t hkv, const int32_t* pos_base,
                               int32_t pos_offset, int64_t len_bound, const int32_t* table, int64_t width,
                               int64_t pages, double theta, uint16_t* q_out, uint16_t* k_pages, uint16_t* v_pages,
                               int32_t* status, hipStream_t stream);
sq_status sq_paged_rope_kv_q4(const float* qkv, const uint16_t* bias, const int32_t* row_start, int32_t b, int64_t rows,
                              int64_t max_rows, int32_t hq, int32_t hkv, const int32_t* pos_base, int32_t pos_offset,
                              int64_t len_bound, const int32_t* table, int64_t width, int64_t pages, double theta,
                              uint16_t* q_out, uint8_t* k_codes, uint16_t* k_scales, uint8_t* v_codes,
                              uint16_t* v_scales, int32_t* status, hipStream_t stream);
sq_status sq_paged_kv_read_q4(const uint8_t* k_codes, const uint16_t* k_scales, const uint8_t* v_codes,
                              const uint16_t* v_scales, const int32_t* table, int64_t width, int64_t pages,
                              const int32_t* row_start, int32_t b, int64_t rows, int64_t max_rows, int32_t hkv,
                              const int32_t* pos_base, int32_t pos_offset, int64_t len_bound, uint16_t* k_out,
                              uint16_t* v_out, hipStream_t stream);
sq_status sq_paged_attention_f16(const uint16_t* q, const uint16_t* k_pages, const uint16_t* v_pages,
                                 const int32_t* table, int64_t width, int64_t pages, const int32_t* row_start,
                                 int32_t b, int64_t rows, int64_t max_rows, int32_t hq, int32_t hkv,
                                 const int32_t* pos_base, int32_t pos_offset, int64_t len_bound, uint16_t* out,
                                 hipStream_t stream);
sq_status sq_paged_attention_q4(const uint16_t* q, const uint8_t* k_codes, const uint16_t* k_scales,
                                const uint8_t* v_codes, const uint16_t* v_scales, const int32_t* table, int64_t width,
                                int64_t pages, const int32_t* row_start, int32_t b, int64_t rows, int64_t max_rows,
                                int32_t hq, int32_t hkv, const int32_t* pos_base, int32_t pos_offset,
                                int64_t len_bound, uint16_t* out, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* SPECQUANT_PAGED_H */

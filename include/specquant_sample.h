/*
 * specquant_sample.h -- sampling with temperature, top-k, top-p and min-p, each row with settings of its own.
 *
 * sq_spec_accept at kd = 0 draws from softmax(logits / T).  These calls draw from what the usual filters leave of it, or
 * write the logits with the tokens that the filters drop as -inf, which sq_spec_accept and sq_spec_accept_multi take as
 * masked: a draft and a parent filtered alike are accepted as ever, and the tokens follow the parent's filtered
 * distribution exactly.  The conventions of specquant.h hold (device pointers, alignment, statuses, the library
 * workspace, one stream per device, SQ_DEV_* bits).
 *
 * Per row, with logits l_j and the order O: l descending, then the lowest j first (-0 is 0):
 *   weights  w_j = exp((l_j - max l) / T) in fp64 to 2^-39, rounded to fp32; R_j = rint(w_j 2^s),
 *            s = min(51, 62 - ceil(log2 v)) (sums of R are exact in int64)
 *   top-k    the first k of O are kept (k <= 0, or k >= v: all)
 *   top-p    of the kept ones the shortest run from the start of O with sum R >= ceil(p Z), Z the sum of R over the
 *            kept ones, p Z and its ceil in fp64, at least the first token (p >= 1: all)
 *   min-p    of those the ones with w_j >= min(m, 1) (m = 0: all)
 *   draw     t = floor(u24 Z' / 2^24), Z' the sum of R over what is kept: the smallest j whose running sum of R over
 *            the kept j' <= j exceeds t; u24 & 0xFFFFFF as in sq_spec_accept
 * T = 0: the first of O alone.  -inf: a token of weight 0.  Without filters the distribution is that of sq_spec_accept
 * to a relative 2^-23 (there each probability is rounded to fp32, here each weight), so a draw may differ where u24 falls
 * that close to a border.
 *
 * A row with a NaN or a +inf among its logits, or without a finite one, has no distribution (SQ_DEV_NO_DIST): token -1,
 * filtered logits as they are.  A row whose T, p or m is NaN, negative or (T) infinite: token -1, NaN in the filtered
 * logits, SQ_DEV_BAD_PARAM.
 *
 * logits [m][ld] f32, of which the first v of each row count; 1 <= m <= 2^20, 1 <= v <= 2^26, v <= ld < 2^31.
 * temperature, top_k, top_p, min_p [m] (f32, int32, f32, f32), each NULL: 1, 0, 1 and 0 for every row.
 * Workspace: at most 32 MB.
 */
#ifndef SPECQUANT_SAMPLE_H
#define SPECQUANT_SAMPLE_H

#include "specquant.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SQ_DEV_BAD_PARAM 256 /* a temperature, top_p or min_p that is NaN, negative or (temperature) infinite */

/* token[r] int32 out: a draw of every row; u24 [m] uint32. */
sq_status sq_sample_f32(const float* logits, int32_t m, int64_t v, int64_t ld, const float* temperature,
                        const int32_t* top_k, const float* top_p, const float* min_p, const uint32_t* u24,
                        int32_t* token, int32_t* status, hipStream_t stream);

/* out [m][ld] f32: logits of kept tokens, -inf for the others; what lies behind the first v of a row is not written.
 * out = logits filters in place. */
sq_status sq_filter_logits_f32(const float* logits, int32_t m, int64_t v, int64_t ld, const float* temperature,
                               const int32_t* top_k, const float* top_p, const float* min_p, float* out,
                               int32_t* status, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* SPECQUANT_SAMPLE_H */

/*
 * ivftq_sample.h -- the next token of each row from a model's logits, for AMD MI355X (gfx950), part of libivftq.
 *
 * Row r has logits x_i, i < vocabulary, and weights w_i = e^((x_i - max x) / temperature).  Of its tokens, ranked by x (ties: the lowest
 * index first), these are kept, each step on what the one before has left:
 *     top_k   the first top_k ranks                                            (0, or not under the vocabulary: all)
 *     top_p   the ranks before which there is less than top_p of the mass      (1 and above: all; the first rank always)
 *     min_p   w_i >= min_p                                                     (0: all; above 1 as 1)
 * The token is the lowest index i with  sum of kept w_j, j <= i  >  u * sum of all kept w_j.  u comes from the caller, so equal calls give
 * equal tokens.  temperature 0: the largest logit's lowest index.
 *
 * Weights are added up as whole multiples of 2^-42 (of the largest weight), so sums do not depend on their order; a token of less than half
 * of that is never drawn.  What is no number counts as -infinity; +infinity leaves only the tokens that have it.  A row of nothing but
 * -infinity gives token -1.
 *
 * Conventions as in ivftq_kv.h: device pointers, asynchronous on `stream`, kernel launches only, nothing allocated or kept.
 */
#ifndef IVFTQ_SAMPLE_H
#define IVFTQ_SAMPLE_H

#include "ivftq.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { IVFTQ_LOGITS_F16 = 0, IVFTQ_LOGITS_BF16 = 1, IVFTQ_LOGITS_F32 = 2 };

/* Logit i of row r at data[r * row_stride + i] (elements; row_stride >= vocabulary).  vocabulary: 1 to 2^20. */
typedef struct ivftq_logits {
    const void* data;
    int64_t row_stride;
    int64_t rows;
    int32_t vocabulary;
    int32_t type;
} ivftq_logits;

/* How rows are sampled: an array of a value for each row (device), or NULL and the one value for all.  In the arrays what is out of range
 * counts as the end of the range that it lies behind, no number as no restriction (temperature: as 0). */
typedef struct ivftq_sampling {
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    float temperature_all;         /* >= 0 */
    int32_t top_k_all;             /* >= 0 */
    float top_p_all;               /* 0 to 1 */
    float min_p_all;               /* 0 to 1 */
} ivftq_sampling;

/* u: rows numbers from [0, 1) (others as the nearest).  tokens: rows.  logprobs, NULL or rows floats: the natural logarithm of the
 * probability that the token had among those kept (token -1: -infinity).  workspace: ivftq_sample_workspace bytes, 256-byte aligned,
 * its content does not matter. */
ivftq_status ivftq_sample_tokens(const ivftq_logits* logits, const float* u, const ivftq_sampling* how, int32_t* tokens, float* logprobs,
                                 void* workspace, int64_t workspace_bytes, void* stream);
/* -1 for logits that ivftq_sample_tokens refuses.  how NULL: enough for any. */
int64_t ivftq_sample_workspace(const ivftq_logits* logits, const ivftq_sampling* how);

#ifdef __cplusplus
}
#endif
#endif /* IVFTQ_SAMPLE_H */

/*
 * mlora_logit_rules -- penalties for repeated tokens, biases and grammar masks on the logits of a draft tree's rows, for AMD
 * MI355X (gfx950), C ABI.  Part of the mlora_w4 library.
 *
 * Row r of stream s (row s * R + r of the call) continues, through parent[], the rows above it up to row 0, the last verified
 * token; the first T rows of a stream are its token rows (as in mlora_ds2d.h), which carry tokens[s][t].  With
 *
 *     c(v) = counts[s][v] + number of token rows t > 0 on the row's path (itself included) with tokens[s][t] = v
 *
 * (row 0's token is the stream's newest: it is counted in counts[]) the call computes, for every token v of every row,
 *
 *     z1 = c <= 0 ? z : z > 0 ? z / repetition[s] : z * repetition[s]
 *     z2 = z1 - (frequency[s] * c + presence[s] * (c > 0)) + bias[bias_row[s]][v]
 *     out = token v is allowed by mask mask_row[row] ? z2 : -infinity           (whatever z2 is, NaN too)
 *
 * in fp32, rounded once at the end; z / repetition[s] is z times the fp32 number next to 1 / repetition[s].  First it adds the
 * stream's new tokens to counts[] (each entry of new_tokens[s] in [0, V) once; other values, such as the -1 behind a short list, are
 * skipped).
 *
 * Conventions as in mlora_w4.h.  Logits need the alignment of one element only.
 */
#ifndef MLORA_LOGIT_RULES_H
#define MLORA_LOGIT_RULES_H

#include "mlora_w4.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { MLORA_RULES_MAX_ROWS = 64 /* rows of a stream (as in mlora_tree_attention) */, MLORA_RULES_MAX_NEW = 4096 };

typedef struct {
    int32_t n_streams;              /* S >= 1; S * R <= MLORA_MAX_ROWS */
    int32_t rows_per_stream;        /* R, 1 .. MLORA_RULES_MAX_ROWS */
    int32_t tokens_per_stream;      /* T, 1 .. R */
    int32_t vocab;                  /* V, 1 .. 2^30 */
    int32_t logits_dtype;           /* MLORA_Y_BF16 or MLORA_Y_FP32, of logits and out */
    const int32_t *parent;          /* device int32 [S * R]: an earlier row of the stream; anything else ends the path there */
    int32_t *counts;                /* device int32 [S][V], in and out, or NULL: the rows of the step are all there is */
    const float *repetition;        /* device fp32 [S], of a magnitude from 2^-126 to 2^126, or NULL: 1 */
    const float *frequency;         /* device fp32 [S], or NULL: 0 */
    const float *presence;          /* device fp32 [S], or NULL: 0 */
    const float *bias;              /* device fp32 [n_bias][V] */
    const int32_t *bias_row;        /* device int32 [S]: a row of bias; outside [0, n_bias): no bias */
    int32_t n_bias;                 /* 0: bias and bias_row may be NULL */
    const uint32_t *masks;          /* device uint32 [n_masks][(V + 31) / 32]: bit v % 32 of word v / 32 set: v is allowed */
    const int32_t *mask_row;        /* device int32 [S * R]: a row of masks; outside [0, n_masks): all tokens are allowed */
    int32_t n_masks;                /* 0: masks and mask_row may be NULL */
} mlora_logit_rules;

/*   logits      [S * R][V]      out  the same shape; may be logits itself
 *   tokens      int32 [S][T]    new_tokens  int32 [S][n_new], NULL where n_new is 0 (always 0 without counts) */
mlora_status mlora_logit_rules_apply(const mlora_logit_rules *d, const void *logits, const int32_t *tokens, const int32_t *new_tokens,
                                     int32_t n_new, void *out, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MLORA_LOGIT_RULES_H */

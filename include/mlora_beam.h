/*
 * mlora_beam -- one step of beam search on the logits, for AMD MI355X (gfx950), C ABI.  Part of the mlora_w4 library.
 *
 * G groups (requests) of W beams; beam b of group g is row g * W + b of the call.  Every beam has a score (the sum of the logarithms of its
 * tokens' probabilities), a length in tokens, and may be finished.  Candidates of a group:
 *     beam b, not finished, with token v:   score_b + z_b[v] - log sum over u of exp z_b[u],   length_b + 1 tokens
 *     beam b, finished:                     score_b as it is, length_b tokens, token `pad`
 * ranked by their score / max(1, tokens)^length_power.  The W best, best first, are the group's new beams; a candidate with token `eos` is
 * finished.  Among equals the lower beam comes first, then the larger logit, then the lower token.
 *
 * There is no candidate with a logit of -infinity, none of a beam whose score is not finite, and none of one whose logits hold NaN
 * or +infinity.  Places that no candidate takes have score -infinity, their own row as source, token `pad`, length 0, and are not finished: beams
 * without candidates.  A search starts from one beam with score 0 and W - 1 with -infinity.
 *
 * Scores are compared in 64 bits, from exponentials in fp32 that are added 64 by 64 in fp32 and beyond that in 64 bits (a logarithm of a sum is
 * off by 10^-8 as a rule, by 2^-17 at most), and rounded once, to the fp32 number that is given out.  Conventions as in mlora_w4.h.
 */
#ifndef MLORA_BEAM_H
#define MLORA_BEAM_H

#include "mlora_w4.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { MLORA_BEAM_MAX_BEAMS = 32, MLORA_BEAM_MAX_VOCAB = 1 << 24 };

typedef struct {
    int32_t n_groups, n_beams;      /* G >= 1, W 1 .. MLORA_BEAM_MAX_BEAMS; G * W <= MLORA_MAX_ROWS */
    int32_t vocab;                  /* 1 .. MLORA_BEAM_MAX_VOCAB */
    int32_t logits_dtype;           /* MLORA_Y_BF16 or MLORA_Y_FP32 */
    int32_t eos;                    /* token that ends a beam; outside the vocabulary: none */
    int32_t pad;
    float length_power;             /* finite, >= 0 */
} mlora_beam;

/* Device scratch of a call (256-byte aligned); its contents need no initialisation and carry nothing from call to call.  0 on a bad
 * descriptor. */
size_t mlora_beam_workspace_bytes(const mlora_beam *d);

/* All of the arrays but the logits have an entry for every row.
 *   logits          [G * W][vocab], alignment of one element (what rows of finished beams hold does not count)
 *   score           fp32;  length, finished  int32 (finished: not 0)
 *   source          out int32: the row that the new beam continues (what mlora_page_cache_reorder takes)
 *   token           out int32
 *   score_out, length_out, finished_out     out, as the inputs, which they may be themselves */
mlora_status mlora_beam_select(const mlora_beam *d, const void *logits, const float *score, const int32_t *length, const int32_t *finished,
                               int32_t *source, int32_t *token, float *score_out, int32_t *length_out, int32_t *finished_out,
                               void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MLORA_BEAM_H */

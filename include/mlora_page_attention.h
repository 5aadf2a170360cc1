/*
 * mlora_page_attention -- attention over a paged cache of 8 bits, with a sliding window and first tokens that stay visible, for AMD
 * MI355X (gfx950), C ABI.  Part of the mlora_w4 library.
 *
 * Row i of stream s is row m = s * R + i of the call.  As in mlora_tree_attention it continues the row parent[m] of its stream (an earlier one;
 * anything else: it stands right behind the stream's tokens).  With d rows above it on this path it stands at position p = len[s] + d, and
 *
 *     out[m][hq] = sum over the tokens row m may see of softmax(scale * q[m][hq] . k)[token] * v[token]
 *
 * where it may see the stream's tokens (positions 0 .. len[s] - 1), itself and the rows it continues, those at positions t with
 * t > p - window or t < sink (window 0: all of them).  Keys and values of full pages are code * scale, those of the tail and of the step's
 * rows are bf16.  Tokens whose table entry names no page of the pool are not there.  Query head hq reads kv head hq / (n_q_heads / n_kv_heads).
 * Position encodings are applied by the caller.
 *
 * What a row may not see does not touch it, infinite or not a number as it may be.  A row that sees NaN, or whose own query vector is not
 * finite, is NaN.  Finite scores scale q . k are of a magnitude below 2^20.
 *
 * Accuracy, for both types of outputs: on pages a query vector's numbers count to 2^-22 of its largest, a weight to 2^-24 of the largest of its page; products, sums
 * and states are exact or fp32, and an output in bf16 is rounded once.
 *
 * Conventions as in mlora_w4.h; results are bit-identical from call to call.
 */
#ifndef MLORA_PAGE_ATTENTION_H
#define MLORA_PAGE_ATTENTION_H

#include "mlora_page_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    mlora_page_cache cache;            /* own is not used; nothing in the cache is written */
    int32_t layer;                     /* of the cache */
    int32_t n_q_heads;                 /* a multiple of n_kv_heads, at most 8 query heads per kv head */
    int32_t rows_per_stream;           /* R, 1 .. 64; S * R <= MLORA_MAX_ROWS */
    float scale;
    int32_t window, sink;              /* >= 0 */
    const void *k_new, *v_new;         /* the rows of the step, bf16 [S * R][H][D], 16-byte aligned */
    const int32_t *parent;             /* device int32 [S * R] */
} mlora_page_attn;

/* Device scratch of a call (256-byte aligned); its contents need no initialisation and carry nothing from call to call.  0 on a bad
 * descriptor. */
size_t mlora_page_attention_workspace_bytes(const mlora_page_attn *t);

/* How such a call would be run, for reading profiles; host only, nothing is launched.  info (HOST memory, 3 int32): as of
 * mlora_tree_attention_plan, [0] tiles of 16 query vectors a block takes, [1] waves of a block, [2] blocks that may share a tile's pages (how
 * many do, and whether streams are taken together, the lengths decide on the device). */
mlora_status mlora_page_attention_plan(const mlora_page_attn *t, int32_t *info);

/*   q    bf16 [S * R][n_q_heads][D], 16-byte aligned
 *   out  [S * R][n_q_heads][D], bf16 (out_dtype = MLORA_Y_BF16, round to nearest even) or fp32, 16-byte aligned */
mlora_status mlora_page_attention(const mlora_page_attn *t, const void *q, void *out, int32_t out_dtype, void *workspace,
                                  size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MLORA_PAGE_ATTENTION_H */

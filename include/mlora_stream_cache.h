/*
 * mlora_stream_cache -- the streams' own cache segments at a bounded size, for AMD MI355X (gfx950), C ABI.  Part of the mlora_w4
 * library.
 *
 * Every layer, stream and kv head has `cap` slots of a key, a value, the attention weight the slot has received so far (mass) and the
 * position of the token it holds.  The slots below len[s] are live; they stand in no order (the attention needs none: keys
 * are rotated before they are stored).  k and v of layer l are what mlora_tree_attention takes as k_stream and v_stream.
 *
 *   append    the accepted rows of a step enter the caches of all layers; where a stream's live slots would pass the budget, the
 *             slots with the least mass give way to them
 *   weights   the attention weights of the newest rows are added to the mass of every slot they saw
 *   compress  the heaviest slots of a long segment (a prompt) are copied, in order, into a smaller cache
 *
 * Rank of a head's live slots: first those that are protected (position >= next_pos - recent, or position < sink), then the
 * others by mass, the larger first and NaN last (-0 equals +0); among equals the lower slot.
 *
 * Rows of a call are listed per stream: rows[s][0 .. n_rows), indexes into the stream's R rows of the step, which count up to
 * the first entry outside [0, R) (mlora_ds2d_step's accepted_rows as they are); NULL: all R rows in order.  len[s] outside
 * [0, cap] counts as the nearer end.
 *
 * Conventions as in mlora_w4.h: no allocation, no synchronisation, no atomics on values: results are bit-identical from call
 * to call.  Calls on one cache that overlap on the GPU race.
 */
#ifndef MLORA_STREAM_CACHE_H
#define MLORA_STREAM_CACHE_H

#include "mlora_w4.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
    MLORA_CACHE_MAX_SLOTS = 1 << 24,   /* cap */
    MLORA_CACHE_TICKET_WORDS = 32,     /* a line of memory per stream */
    MLORA_CACHE_MAX_HEADS = 1 << 20    /* n_layers * n_streams * n_kv_heads */
};

/* Index order and types of the device memory, L = n_layers, S = n_streams, H = n_kv_heads: */
typedef struct {
    int32_t n_layers, n_streams, n_kv_heads;
    int32_t head_dim;                  /* 64 or 128 */
    int32_t cap;                       /* 1 .. MLORA_CACHE_MAX_SLOTS */
    void *k, *v;                       /* bf16 [L][S][H][cap][head_dim], 16-byte aligned */
    float *mass;                       /* fp32 [L][S][H][cap] */
    int32_t *slot_pos;                 /* int32 [L][S][H][cap] */
    int32_t *len;                      /* int32 [S]: live slots, the same in all layers and heads */
    int32_t *next_pos;                 /* int32 [S]: position of the stream's next token */
    uint32_t *tickets;                 /* uint32 [S][MLORA_CACHE_TICKET_WORDS]: zero when a call starts, zero again when it ends (append alone uses them) */
} mlora_stream_cache;

/* Row j of the n that a stream appends goes to slot len + j while the live slots are fewer than max(len, budget); the others go to
 * the e slots of the lowest rank, in the order of the slots, each head its own.  A slot that is written starts with mass 0 and
 * position next_pos + j.  Then len grows by the rows that found room, next_pos by n.
 *   k_new, v_new  bf16 [L][S * rows_per_stream][H][head_dim]
 *   rows          device int32 [S][n_rows] or NULL;  n_rows 1 .. rows_per_stream (ignored without rows)
 *   budget        live slots to keep to: at least the rows of the call, at most cap;  sink, recent >= 0 */
mlora_status mlora_stream_cache_append(const mlora_stream_cache *c, const void *k_new, const void *v_new, int32_t rows_per_stream,
                                       const int32_t *rows, int32_t n_rows, int32_t budget, int32_t sink, int32_t recent, void *stream);

/* The min(len, budget) slots of the highest rank of every head go to the slots 0, 1, .. of `to` in the order of their slots, with mass
 * and position; to->len and to->next_pos are set.  `to` has the same L, S, H and head_dim, cap >= budget and memory of its own;
 * its other slots stay as they are.
 *   kept   out device int32 [L][S][H][budget]: the slots, ascending, -1 beyond */
mlora_status mlora_stream_cache_compress(const mlora_stream_cache *from, const mlora_stream_cache *to, int32_t *kept,
                                         int32_t budget, int32_t sink, int32_t recent, void *stream);

/* Attention weights of the newest rows.  Listed row j of the n of stream s is the token at position next_pos[s] - n + j (the rows have
 * been appended): with its query heads it sees the prefill segment, which all streams share, and the stream's live slots with
 * slot_pos <= its position.  For every layer and kv head
 *     mass[t]         = decay * mass[t]         + sum over rows and query heads of softmax(scale q . k)[t]     (live slots)
 *     mass_prefill[t] = decay * mass_prefill[t] + the same, over all streams
 * (the soft-max runs over both segments; a row that sees nothing, or whose scores are all minus infinity, adds nothing; one with NaN or
 * plus infinity among its scores makes what it sees NaN, and only that; finite scores scale q . k are of a magnitude below 2^30: beyond,
 * fp32 does not hold their differences and weights may be NaN). */
typedef struct {
    mlora_stream_cache cache;
    int32_t n_q_heads;                 /* a multiple of n_kv_heads, at most 8 query heads per kv head */
    int32_t rows_per_stream;           /* R >= 1; S * R <= MLORA_MAX_ROWS */
    float scale;
    const void *k_prefill;             /* bf16 [L][H][len_prefill][head_dim], 16-byte aligned; len 0: pointers may be NULL */
    float *mass_prefill;               /* fp32 [L][H][len_prefill] */
    int32_t len_prefill;               /* 0 .. MLORA_CACHE_MAX_SLOTS */
    float decay;
} mlora_attention_mass;

/* Device scratch of such a call (256-byte aligned), n_rows as in the call, 0 for all rows; 0 on a bad descriptor.  Its contents
 * need no initialisation and carry nothing from call to call. */
size_t mlora_attention_mass_workspace_bytes(const mlora_attention_mass *d, int32_t n_rows);

/*   q     bf16 [L][S * rows_per_stream][n_q_heads][head_dim], rotated, 16-byte aligned
 *   rows  device int32 [S][n_rows] or NULL (all rows; n_rows is ignored) */
mlora_status mlora_attention_mass_add(const mlora_attention_mass *d, const void *q, const int32_t *rows, int32_t n_rows,
                                      void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MLORA_STREAM_CACHE_H */

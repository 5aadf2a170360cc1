/*
 * mlora_page_cache -- a paged cache of keys and values in 8 bits that streams can share, for AMD MI355X (gfx950), C ABI.  Part of the
 * mlora_w4 library.
 *
 * Token t of a stream lies in page t / 64.  Pages come from a pool that all streams share; page i of a stream is the pool's page
 * table[slot][i] in every layer and head.  Full pages never change, so streams that continue the same tokens hold the same pages,
 * counted in refs.  The tokens of a stream's last, unfinished page stay in bf16, in its tail.
 *
 * A page that fills is rounded to 8 bits, keys and values of every layer and head apart: with m the largest magnitude of its 64 *
 * head_dim numbers
 *     scale = m / 127      code = 127 x / m, to the nearest whole number, halves to the even one      (m 0: codes and scale 0)
 * in fp32; a number is off by half a scale at most.  One that is infinite or NaN makes the scale NaN and all codes 0: whoever sees a
 * token of that page in that head gets NaN.  Values are stored feature by feature (the order in which the attention takes them).
 *
 *   append   the accepted rows of a step, or a prompt, enter the caches of all layers
 *   reorder  streams become continuations of others, as beams do; pages are shared, and those that nobody holds or a window has left
 *            behind are free again
 *   copy     streams into another cache, packed
 *
 * Free pages are taken from the lowest on.  Conventions as in mlora_w4.h: no allocation, no synchronisation; results, the choice of pages
 * among them, are bit-identical from call to call.  Calls on one cache that overlap on the GPU race.
 */
#ifndef MLORA_PAGE_CACHE_H
#define MLORA_PAGE_CACHE_H

#include "mlora_w4.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
    MLORA_PAGE_TOKENS = 64,
    MLORA_PAGE_MAX_STREAMS = 1024,     /* n_streams */
    MLORA_PAGE_MAX_PAGES = 1 << 20,    /* n_pages */
    MLORA_PAGE_MAX_COLUMNS = 1 << 18,  /* max_pages: 2^24 tokens */
    MLORA_PAGE_MAX_HEADS = 1 << 20     /* n_layers * n_streams * n_kv_heads */
};

/* Index order and types of the device memory, L = n_layers, S = n_streams, H = n_kv_heads, D = head_dim.  An empty cache is zeros, but
 * for slot (0, 1, .. S - 1) and table (-1). */
typedef struct {
    int32_t n_layers, n_streams, n_kv_heads;
    int32_t head_dim;                  /* 64 or 128 */
    int32_t n_pages;                   /* of the pool */
    int32_t max_pages;                 /* of a stream, which holds up to 64 * max_pages + 63 tokens */
    void *k;                           /* int8 [L][n_pages][H][64][D], 16-byte aligned like all of the data */
    void *v;                           /* int8 [L][n_pages][H][D][64] */
    float *k_scale, *v_scale;          /* fp32 [L][n_pages][H], not negative (or NaN) */
    void *k_tail, *v_tail;             /* bf16 [L][S][H][64][D]: token t of the stream in slot i at [l][i][h][t % 64] */
    int32_t *slot;                     /* int32 [S]: where the stream's tail and table row are; every number once */
    int32_t *len;                      /* int32 [S]: tokens of the stream (outside [0, 64 * max_pages + 63]: the nearer end) */
    int32_t *table;                    /* int32 [S][max_pages], by slot; -1 (or anything outside the pool): no page, tokens that nobody sees */
    int32_t *refs;                     /* int32 [n_pages]: table entries that hold the page; 0: free */
    int32_t *own;                      /* int32 [mlora_page_cache_own_words()]: the library's own, zero at first and after refs was written by others */
} mlora_page_cache;

/* Words of own; 0 if the numbers are outside the limits. */
size_t mlora_page_cache_own_words(int32_t n_streams, int32_t n_pages);

/* Rows enter the streams, each behind its stream's last token.  Listed per stream: rows[s][0 .. n_rows), indexes into the stream's R rows, which
 * count up to the first entry outside [0, R) (mlora_ds2d_step's accepted_rows as they are); NULL: all R rows in order.  A stream enters
 * with all of its rows or none: none where they do not fit its table, and, in the order of the streams, from the first one on whose full pages
 * do not find free ones (streams that fill no page enter all the same).
 *   k_new, v_new  bf16 [L][S * rows_per_stream][H][D], 16-byte aligned;  S * rows_per_stream <= MLORA_MAX_ROWS
 *   rows          device int32 [S][n_rows] or NULL;  n_rows 1 .. rows_per_stream (ignored without rows)
 *   appended      out device int32 [S]: rows that entered, or NULL */
mlora_status mlora_page_cache_append(const mlora_page_cache *c, const void *k_new, const void *v_new, int32_t rows_per_stream,
                                     const int32_t *rows, int32_t n_rows, int32_t *appended, void *stream);

/* Stream s becomes what stream source[s] was (outside [0, S): an empty stream); NULL: all stay.  The first stream that continues
 * a stream takes its slot; the others, and empty ones, take the slots that are left in their order, tail and table row copied.
 * window > 0: pages that lie behind it are given up, those whose tokens t all have t <= len - window (the next token, at position len, sees
 * t > len - window) and that begin at or behind `sink`; sink counts tokens from a stream's first. */
mlora_status mlora_page_cache_reorder(const mlora_page_cache *c, const int32_t *source, int32_t window, int32_t sink, void *stream);

/* Stream i of `to` becomes what stream source[i] of `from` is (outside its streams: an empty one).  `to` holds nothing else afterwards: the
 * pages that these streams hold, each once, in the order of the pool, as its pages 0, 1, ..; what lies in its other pages and behind its streams'
 * tails stays.  If they do not find room (to->n_pages, to->max_pages), all streams of `to` are empty.  `to` has the same L, H and D, and
 * memory of its own.
 *   source   device int32 [to->n_streams]
 *   n_used   out device int32 [1]: pages that the streams hold, whether they find room or not; or NULL */
mlora_status mlora_page_cache_copy(const mlora_page_cache *from, const mlora_page_cache *to, const int32_t *source, int32_t *n_used, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MLORA_PAGE_CACHE_H */

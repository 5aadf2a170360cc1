/*
 * mlora_rope -- rotary position encodings for AMD MI355X (gfx950), C ABI.  Part of the mlora_w4 library.
 *
 * Pair i of a head (of rot / 2 pairs) is turned by the angle position * f_i:
 *
 *     y_a = x_a cos - x_b sin        y_b = x_b cos + x_a sin
 *
 * Features from rot on pass through.  The pair of number i is (i, i + rot / 2) in the half layout, (2i, 2i + 1) in the
 * interleaved one.  The inverse call turns back (the gradient of the rotation).  Frequencies, in radians per position, with
 * t_i = theta^(-2i / rot):
 *     PLAIN    f_i = t_i
 *     LINEAR   f_i = t_i / factor
 *     BASE     f_i = (theta * factor^(rot / (rot - 2)))^(-2i / rot)
 *     TURNS    u = clamp((context * t_i / 2 pi - low) / (high - low), 0, 1):  f_i = (1 - u) t_i / factor + u t_i
 *              (pairs that turn often within `context` positions keep their frequency, slow ones are stretched)
 *
 * Row m of a call stands at position base[m / rows_per_stream] + offset[m % rows_per_stream]; without base: 0; without
 * offset: m % rows_per_stream.  Angles are reduced in 64 bits, so far positions are as exact as near ones.
 *
 * Conventions as in mlora_w4.h.  Tensors need the alignment of one element only.
 */
#ifndef MLORA_ROPE_H
#define MLORA_ROPE_H

#include "mlora_w4.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { MLORA_ROPE_HALF = 0, MLORA_ROPE_INTERLEAVED = 1 };
enum { MLORA_ROPE_PLAIN = 0, MLORA_ROPE_LINEAR = 1, MLORA_ROPE_BASE = 2, MLORA_ROPE_TURNS = 3 };
enum {
    MLORA_ROPE_MAX_DIM = 512,       /* head_dim */
    MLORA_ROPE_MAX_TENSORS = 4,     /* of one call */
    MLORA_ROPE_MAX_ROWS = 1 << 24   /* rows of a call */
};

typedef struct {
    int32_t head_dim;               /* features of a head, 2 .. MLORA_ROPE_MAX_DIM */
    int32_t rot;                    /* features that turn: even, 2 .. head_dim (BASE: from 4) */
    int32_t layout, scaling;
    double theta;                   /* > 0 */
    double factor;                  /* > 0; LINEAR, BASE and TURNS */
    double low, high, context;      /* TURNS: low < high, context > 0 */
} mlora_rope;

/* HOST out: quarter turns per position (f_i * 2 / pi) of every pair, rot / 2 doubles.  Made once; the calls below take a
 * device copy. */
mlora_status mlora_rope_frequencies(const mlora_rope *r, double *quarter_turns);

typedef struct {
    int32_t M;                      /* rows: 0 .. MLORA_ROPE_MAX_ROWS, a multiple of rows_per_stream; 0: tensors may be NULL, nothing is launched */
    int32_t rows_per_stream;
    const int32_t *base;            /* device int32 [M / rows_per_stream], or NULL */
    const int32_t *offset;          /* device int32 [rows_per_stream], or NULL */
    const double *quarter_turns;    /* device fp64 [rot / 2] */
} mlora_rope_rows;

/* Cosines and sines of every row, fp32 [M][rot / 2] each: what mlora_w4_epilogue takes (heads of 64 features, rot 64). */
mlora_status mlora_rope_tables(const mlora_rope *r, const mlora_rope_rows *rows, float *cos_out, float *sin_out, void *stream);

/* One tensor of a call: element (m, head, e) of x lies at m * x_row + head * x_head + e (strides in elements, not negative).  y may be
 * x itself with the same strides, and otherwise overlaps no tensor of the call; its rows and heads do not overlap each other (x's may).
 * rotate 0: the rows are copied. */
typedef struct {
    const void *x;
    void *y;
    int64_t x_row, x_head, y_row, y_head;
    int32_t heads;
    int32_t rotate;
} mlora_rope_tensor;

/* All tensors in one launch.  dtype: MLORA_Y_BF16 (computed in fp32, rounded once to nearest even) or MLORA_Y_FP32.  inverse: 0 or 1. */
mlora_status mlora_rope_apply(const mlora_rope *r, const mlora_rope_rows *rows, const mlora_rope_tensor *tensors, int32_t n_tensors,
                              int32_t dtype, int32_t inverse, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MLORA_ROPE_H */

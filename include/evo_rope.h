/*
 * evo_rope.h -- C ABI of rotary positions and of the norm of every head with
 * the rotation in the same pass (gfx950).
 *
 * Two sets of heads go through one call, set 0 (queries) and set 1 (keys, or
 * n_heads[1] == 0 for none), each with its own head count, length, positions
 * and strides.  Per token t and head, with x the head's d channels:
 *
 *   u = w * x / sqrt(mean(x^2) + eps)     with EVO_ROPE_NORM (w of ones if NULL)
 *   u = x                                 without
 *   y[a] = A (u[a] cos p - u[b] sin p),  y[b] = A (u[a] sin p + u[b] cos p)
 *
 * for the pairs i < rot_dim / 2: (a, b) = (i, i + rot_dim / 2), or (2i, 2i + 1)
 * with EVO_ROPE_INTERLEAVED; channels from rot_dim on are u.  A is `amplitude`,
 * and the angle is p = 2 pi frac(pos[t] * steps[i] / 2^64): steps[i] is the
 * pair's turn per position in units of 2^-64, as a 64-bit integer, so the
 * product's low 64 bits are the fraction of a turn without any rounding, at
 * every int32 position, negative ones too.
 *
 * Backward, from dy: g = the rotation's transpose of dy;
 *   dw = sum over tokens and heads of g * xhat,   xhat = x / sqrt(mean(x^2) + eps)
 *   dx = (g w - xhat mean(g w xhat)) / sqrt(mean(x^2) + eps)
 * (dx = g without the norm, which does not read x).  Sums are fp32 within a
 * workgroup and fp64 over the workgroups, in a fixed order: repeated calls
 * give identical bits.
 *
 * Conventions (dtype and status codes from evo_attn.h): device pointers owned
 * by the caller; nothing is allocated or synchronised; the calls enqueue
 * kernels on `stream` and return, so they may be captured into a HIP graph.
 * Validation happens before any HIP call; errors enqueue nothing.
 * - x, y [N, len, heads, d]: element (r, t, h, c) at r * stride_row + t * stride_tok
 *   + h * d + c.  Addresses and strides allow 16-byte access (EVO_ERR_ALIGNMENT).
 *   y's (row, token) grid does not overlap itself; x's may (stride_row 0: one
 *   row for all), but not where dx, which has x's strides, is written.
 * - y may be x itself (same address, same strides: in place), and dx dy or x; other
 *   overlaps of these are refused, and so are those of one set's output with
 *   the other set's tensors.  Blocks side by side in the tokens of one packed
 *   buffer do not overlap, with one token a row, too.
 * - pos int32: row r starts at r * pos_stride (0: all rows share positions);
 *   steps uint64 [rot_dim / 2], w and dw fp32 [d].
 * - Angles and all arithmetic are fp32 (phases exact), rounded once.  The mean of squares may leave fp32's range, at an
 *   eps of 0 and for large channels: only where 1 / sqrt(mean(x^2) + eps) itself does is dx infinite.
 */
#ifndef EVO_ROPE_H
#define EVO_ROPE_H

#include "evo_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

enum evo_rope_flags { EVO_ROPE_INTERLEAVED = 1, EVO_ROPE_NORM = 2 };

/* Compiled limits: head_dim a multiple of 8, 8..256; rot_dim even, 0..head_dim;
 * n_heads <= 65535; len <= 2^30; n_rows * len * n_heads * head_dim <= 2^40.  An empty set
 * (N, len or n_heads 0) launches nothing for it; its dw is still written (zeros). */
typedef struct evo_rope_dims {
    int32_t dtype;    /* of x and y */
    int32_t head_dim; /* d */
    int32_t rot_dim;  /* rotated channels, the first of each head */
    int32_t flags;    /* enum evo_rope_flags */
    int32_t n_heads[2];
    float eps;        /* of the norm, >= 0 */
    float amplitude;  /* A, finite */
    int64_t n_rows;   /* N >= 0, of both sets */
    int64_t len[2];
    int64_t pos_stride[2];
    int64_t x_stride_row[2], x_stride_tok[2]; /* of x and dx, elements */
    int64_t y_stride_row[2], y_stride_tok[2]; /* of y and dy, elements */
} evo_rope_dims;

int evo_rope_fwd(const evo_rope_dims *dims, const void *x0, const void *x1, const int32_t *pos0,
                 const int32_t *pos1, const uint64_t *steps, const float *w0, const float *w1, void *y0,
                 void *y1, void *stream);

/* dw0, dw1: [d] each, or NULL for a set whose w is NULL (both NULL without the
 * norm); x0, x1 are read with the norm only.  workspace: at least
 * evo_rope_bwd_workspace_size(dims) bytes, 16-byte aligned, contents irrelevant
 * (NULL allowed when that size is 0). */
size_t evo_rope_bwd_workspace_size(const evo_rope_dims *dims);
int evo_rope_bwd(const evo_rope_dims *dims, const void *dy0, const void *dy1, const void *x0, const void *x1,
                 const int32_t *pos0, const int32_t *pos1, const uint64_t *steps, const float *w0,
                 const float *w1, void *dx0, void *dx1, float *dw0, float *dw1, void *workspace,
                 size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* EVO_ROPE_H */

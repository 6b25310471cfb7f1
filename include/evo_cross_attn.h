/*
 * evo_cross_attn.h -- C ABI of the gated attention of queries to states of
 * another length (gfx950): training and single tokens.
 *
 *   o = sigmoid(gate) * softmax(Q K^T / sqrt(d) + bias, over the keys the mask keeps) V
 *
 * evo_attn.h's attention without its limits on length, for queries [N, Lq, H, d]
 * and keys and values [N, Lk, Hk, d]: any lengths, Lq and Lk independent of
 * each other; H a multiple of Hk, query head i reads key head i / (H / Hk).
 *
 * - The bias [B, H, Lq, Lk] (rows r use plane r / rows_per_bias; evo_relpos_fwd
 *   writes one) may start at any element, rows of any length.
 * - key_mask [N, Lk] bytes, nonzero = keep.  What lies in the K and V rows (and
 *   bias columns) of a masked key does not matter, infinities and NaN included;
 *   its dK and dV are zeros.
 * - A query with nothing left to attend to gets o = 0, lse = -inf and zero
 *   gradients: all keys masked, Lk == 0, or no logit above -1e30 (a bias of
 *   -inf or of the type's lowest value at every key is a mask; K and V of keys that
 *   only a bias masks are read, and have to be finite).
 * - Logits are fp32 numbers, and softmax and gradients those of these numbers however far
 *   from zero they lie (at -1e9 a step is 64: equal biases there make keys equally
 *   likely, whatever q k' is).
 * - bf16: inputs to the matrix products are bf16 (the probabilities, their
 *   gradients and sigmoid(gate) * dO are rounded to it once), sums, softmax and
 *   log-sum-exp fp32, results rounded once.  fp32: fp32 throughout.
 * - Every sum runs in a fixed order without atomics: repeated calls give
 *   identical bits.  How the work is split depends on the dims and on whether
 *   there is a bias alone.
 *
 * Conventions (dtype and status codes from evo_attn.h): device pointers owned
 * by the caller; nothing is allocated or synchronised; the calls enqueue
 * kernels on `stream` and return, so they may be captured into a HIP graph.
 * Validation happens before any HIP call; errors enqueue nothing.  Calls that
 * overlap in time need workspaces of their own.
 * - Element (r, t, h, c) of a token tensor is at r * stride_row + t * stride_tok
 *   + h * d + c.  q, gate, dq, dgate share the q strides, k, v, dk, dv the k
 *   strides, out and dout the o strides.  Addresses and strides allow 16-byte
 *   access.  Inputs may repeat rows or tokens (stride 0: one set of states for
 *   all rows); outputs must not overlap themselves (so with repeated states the
 *   backward takes its gradients at other strides: copy the dims, run it on
 *   expanded inputs), each other or an input.  Blocks side by side in the tokens
 *   of one packed buffer do not overlap.
 */
#ifndef EVO_CROSS_ATTN_H
#define EVO_CROSS_ATTN_H

#include "evo_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Compiled limits: head_dim a multiple of 8, 8..128; n_heads <= 65535; len_q * (H / Hk) and
 * len_k <= 2^30; element counts <= 2^40; fewer than 2^24 workgroups a kernel, that is
 * n_rows * Hk * ceil(len_q * H / Hk / 128) and n_rows * Hk * ceil(len_k / 128), with a
 * bias also B * H * ceil(len_q / 64) * ceil(len_k / 64). */
typedef struct evo_cross_dims {
    int32_t dtype;      /* enum evo_attn_dtype */
    int32_t n_heads;    /* H >= 1 */
    int32_t n_kv_heads; /* Hk >= 1, divides H */
    int32_t head_dim;   /* d */
    int64_t n_rows;     /* N >= 0 */
    int64_t len_q, len_k;
    int64_t rows_per_bias; /* >= 1, divides N; ignored when bias is NULL */
    int64_t q_stride_row, q_stride_tok;
    int64_t k_stride_row, k_stride_tok;
    int64_t o_stride_row, o_stride_tok;
} evo_cross_dims;

/*
 * Forward: out (o strides) and lse [N, H, Lq] fp32 (natural log of the sum over
 * the kept keys, bias included; the backward takes it).  gate, bias, key_mask
 * may be NULL.  workspace: at least evo_cross_fwd_workspace_size(dims) bytes,
 * 256-byte aligned, contents irrelevant (NULL allowed when that size is 0).
 * N, Lq == 0: nothing to write, EVO_OK; Lk == 0: k and v may be NULL.
 */
size_t evo_cross_fwd_workspace_size(const evo_cross_dims *dims);
int evo_cross_fwd(const evo_cross_dims *dims, const void *q, const void *k, const void *v, const void *gate,
                  const void *bias, const uint8_t *key_mask, void *out, float *lse, void *workspace,
                  size_t workspace_bytes, void *stream);

/*
 * Backward, from the forward's inputs, out and lse, and dout.  dgate and dbias
 * are NULL if and only if gate and bias are; dbias [B, H, Lq, Lk] has the
 * bias' type (summed in fp32 over the rows of its plane, rounded once).
 */
size_t evo_cross_bwd_workspace_size(const evo_cross_dims *dims, int has_gate, int has_bias);
int evo_cross_bwd(const evo_cross_dims *dims, const void *q, const void *k, const void *v, const void *gate,
                  const void *bias, const uint8_t *key_mask, const void *out, const float *lse,
                  const void *dout, void *dq, void *dk, void *dv, void *dgate, void *dbias, void *workspace,
                  size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* EVO_CROSS_ATTN_H */

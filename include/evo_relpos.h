/*
 * evo_relpos.h -- C ABI of the learned relative position bias (gfx950).
 *
 * One value per head and bucket of the position difference, added to the
 * logits of an attention, written in the [B, H, L, L] bias layout that
 * evo_attn_fwd reads, alone or on top of a pair bias (evo_ln_pair_bias_fwd):
 *
 *   n(b, i, j)      = number of edges e with e <= pos_i[b, i] - pos_j[b, j]
 *                     or n_edges + 1 where seg_i[b, i] != seg_j[b, j]
 *   out[b, h, i, j] = base[b, h, i, j] + table[h, n(b, i, j)]
 *
 * The edges are the ascending first differences of every bucket but the
 * lowest: n_edges edges make n_edges + 1 buckets, numbered from the most
 * negative difference up, and one more for pairs of different segments
 * (chains, packed sequences) when segments are given.  Consecutive integers
 * 1 - K .. K give the 2K + 1 buckets of differences clipped at +-K; growing
 * steps give buckets by distance.  The bias of the transposed attention
 * (triangle attention around the ending node) is that of negated positions.
 *
 * Backward: out depends on the base with gradient one, so its gradient is
 * dbias itself, and
 *   dtable[h, n] = sum over (b, i, j) with n(b, i, j) = n of dbias[b, h, i, j].
 * Buckets that no pair falls into get 0.  Sums are fp32 within a part of the
 * entries and fp64 over the parts, in a fixed order: repeated calls give
 * identical bits.
 *
 * Conventions (dtype and status codes from evo_attn.h): device pointers owned
 * by the caller; nothing is allocated or synchronised; the calls enqueue
 * kernels on `stream` and return, so they may be captured into a HIP graph.
 * Validation happens before any HIP call; errors enqueue nothing.
 * - pos_i [B, Li], pos_j [B, Lj], seg_i [B, Li], seg_j [B, Lj], edges
 *   [n_edges]: contiguous int32, 4-byte aligned (edges may be NULL when
 *   n_edges is 0).  Any values; a difference beyond int32 counts as the int32
 *   nearest to it.  Edges that do not ascend give some bucket in range.
 * - table, dtable: contiguous fp32 [H, buckets], 4-byte aligned.
 * - base: contiguous [B, H, Li, Lj] of the dims' dtype or NULL (zeros); out:
 *   the same shape and type.  Both aligned to their element; out may be base
 *   itself (the bias is added in place), but must not overlap it otherwise.
 * - dbias: contiguous fp32 [B, H, Li, Lj], 4-byte aligned: what evo_attn_bwd
 *   writes.
 * Sums are formed in fp32 and rounded once to nearest even.
 */
#ifndef EVO_RELPOS_H
#define EVO_RELPOS_H

#include "evo_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Compiled limits: n_heads <= 65535, n_edges <= 1022, lengths <= 2^20, n_batch * n_heads
 * * len_i * len_j <= 2^40.  No size is padded; B, Li or Lj == 0 validates and
 * returns EVO_OK (the backward still writes dtable: zeros). */
typedef struct evo_relpos_dims {
    int32_t dtype;    /* of base and out (the backward ignores it but validates it) */
    int32_t n_heads;  /* H >= 1 */
    int32_t n_edges;  /* >= 0 */
    int32_t has_seg;  /* 1: seg_i and seg_j are given, and one bucket more; 0: both NULL */
    int64_t n_batch;  /* B >= 0 */
    int64_t len_i;    /* Li >= 0 */
    int64_t len_j;    /* Lj >= 0 */
    int64_t reserved; /* must be 0 */
} evo_relpos_dims;

int evo_relpos_fwd(const evo_relpos_dims *dims, const int32_t *pos_i, const int32_t *pos_j,
                   const int32_t *seg_i, const int32_t *seg_j, const int32_t *edges, const float *table,
                   const void *base, void *out, void *stream);

/* workspace: at least evo_relpos_bwd_workspace_size(dims) bytes, 16-byte
 * aligned, contents irrelevant (NULL allowed when that size is 0). */
size_t evo_relpos_bwd_workspace_size(const evo_relpos_dims *dims);
int evo_relpos_bwd(const evo_relpos_dims *dims, const int32_t *pos_i, const int32_t *pos_j,
                   const int32_t *seg_i, const int32_t *seg_j, const int32_t *edges, const float *dbias,
                   float *dtable, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* EVO_RELPOS_H */

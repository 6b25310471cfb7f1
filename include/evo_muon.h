/*
 * evo_muon.h -- C ABI of the orthogonalised optimizer step on MI355X (gfx950):
 * Newton-Schulz orthogonalisation of matrices, and the Muon step (momentum,
 * orthogonalised update, weight decay, stochastic weight average) over a
 * packed list of matrices, beside evo_optim.h's Adam step, which keeps the
 * vectors (biases, LayerNorm parameters).
 *
 * Orthogonalisation of a matrix x of rows x cols, r = min, c = max of the two,
 * taken transposed where rows > cols:
 *
 *   X = x / max(|x|_F, eps)
 *   `steps` times:  A = X X^T,  X = a X + (b A + c A^2) X
 *
 * Each step maps the singular values s to a s + b s^3 + c s^5 and keeps the
 * singular vectors; with the usual (3.4445, -4.7750, 2.0315) five steps bring
 * those above about 1/500 of the norm to 0.7 .. 1.2.
 *
 * Muon step, per matrix (fp32), gs = *grad_scale or 1:
 *
 *   g = grad * gs
 *   m = momentum m + (1 - momentum) g
 *   u = nesterov ? (1 - momentum) g + momentum m : m
 *   O = orthogonalised u
 *   p = (1 - lr weight_decay) p - lr update_scale O
 *   w = swa_decay w + (1 - swa_decay) p           (skipped when swa == NULL)
 *
 * Conventions (dtype and status codes from evo_attn.h): device pointers owned
 * by the caller; nothing is allocated or synchronised; the calls enqueue
 * kernels on `stream` and return, so they may be captured into a HIP graph.
 * Validation happens before any HIP call; errors enqueue nothing.  Matrices
 * are contiguous and aligned to their element.  All sums run in a fixed
 * order: repeated calls give identical bits.  Two calls may overlap in time
 * only with workspaces of their own.
 *
 * Coefficients: the iterate is held in a limited range, so
 * coefficients that could take it out of it (singular values above 8, or
 * |a| + |b| s^2 + |c| s^4 above 60, followed from 1 over the steps) are refused
 * with EVO_ERR_UNSUPPORTED.  A matrix with an infinity or a NaN gives NaN.
 *
 * Precision: iterates are pairs of fp16 with fp32 accumulation, 22 bits of an entry down
 * to an absolute end: 2^-40 of max(|x|_F, eps) for X = x / max(|x|_F, eps) and its products
 * at the usual coefficients, 2^-34 where singular values reach 8.  Five steps of fp32 matrices err like
 * fp32 arithmetic over the whole matrix, low-rank ones and norms below eps included.  What is
 * far below the rest of a matrix has that end as its error, grown by a (3.4445) a step like itself:
 * rows 10^6 times smaller than another are off by 2 10^-5 of themselves after any number of steps, 10^8
 * times smaller by 2 10^-3, and with more steps that reaches the whole (10^6: 10^-5 after 12 steps).
 * bf16 matrices take the same steps: their results are those of the same values in fp32,
 * rounded once.
 */
#ifndef EVO_MUON_H
#define EVO_MUON_H

#include "evo_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Compiled limits: rows and cols up to 32768, n_batch up to 2^20, steps 1 .. 64, and
 * fewer than 2^24 tiles of 64 x 64 entries in a call (a plan: by XCD, padding included). */
typedef struct evo_orth_dims {
    int32_t dtype;    /* of x and out: EVO_DTYPE_F32 or EVO_DTYPE_BF16 */
    int32_t steps;    /* >= 1 */
    int64_t n_batch;  /* matrices in the stack, >= 0 */
    int64_t rows;     /* >= 0 */
    int64_t cols;     /* >= 0 */
    double a, b, c;   /* coefficients of the step */
    double eps;       /* > 0: smallest norm divided by */
    int64_t reserved; /* must be 0 */
} evo_orth_dims;

/* out[k] = orthogonalised x[k]; x, out: contiguous [n_batch, rows, cols], not
 * overlapping unless out == x.  workspace: at least
 * evo_orthogonalize_workspace_size(dims) bytes, 256-byte aligned, contents
 * irrelevant (NULL allowed when that size is 0).  An empty stack validates
 * and returns EVO_OK. */
size_t evo_orthogonalize_workspace_size(const evo_orth_dims *dims);
int evo_orthogonalize(const evo_orth_dims *dims, const void *x, void *out, void *workspace,
                      size_t workspace_bytes, void *stream);

typedef struct evo_muon_tensor {
    float *param;        /* updated in place */
    const float *grad;   /* read only */
    float *momentum;     /* updated in place */
    float *swa;          /* averaged parameter, updated in place; NULL = no SWA */
    int64_t rows, cols;  /* >= 0; empty matrices are skipped */
    double update_scale; /* factor of the orthogonalised update, finite */
} evo_muon_tensor;

/* Hyperparameters in double; the library derives 1 - momentum and the like in
 * double and rounds each once to fp32. */
typedef struct evo_muon_hparams {
    double lr, momentum, weight_decay, swa_decay;
    double a, b, c, eps; /* as evo_orth_dims */
    int32_t steps;
    int32_t nesterov;    /* 0 or 1 */
} evo_muon_hparams;

/* The tensors that a step writes (param, momentum, swa) must not overlap each other
 * or a gradient: matrices are worked on at the same time.
 *
 * The plan holds the pointers and the work lists of every matrix.  It is
 * built once on the host (evo_muon_plan_bytes bytes, 8-byte aligned; the size
 * is -1 for invalid sizes) and copied to the device by the caller, who passes
 * both copies to every step; rebuild it if a tensor is reallocated. */
int64_t evo_muon_plan_bytes(const evo_muon_tensor *tensors, int32_t n_tensors);
int evo_muon_build_plan(const evo_muon_tensor *tensors, int32_t n_tensors, void *plan, size_t plan_bytes);
/* bytes of workspace a step with this plan (host copy) needs; 256-byte aligned */
size_t evo_muon_workspace_size(const void *plan);

/* One step.  grad_scale: device fp32 scalar multiplying every gradient (e.g.
 * scale_out of evo_grad_clip_scale) or NULL for 1. */
int evo_muon_step(const evo_muon_hparams *hp, const void *plan, const void *plan_device, const float *grad_scale,
                  void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* EVO_MUON_H */

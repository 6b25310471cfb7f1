// evo_ns.h -- internal data of the Newton-Schulz kernels: what the host plan
// (evo_muon_api.cpp) hands to the kernels (evo_muon.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace evo {

// one matrix; r x c with r <= c is the iterate, the transposed matrix where rows > cols
struct NsMat {
    const void *in;      // gradient (fp32), or the matrix to orthogonalise
    void *out;           // parameter (fp32), or the result
    float *mom, *swa;    // momentum; average or null (Muon only)
    int32_t rows, cols;
    float scale;         // factor of the update
    int32_t part0;       // first partial sum of squares
    int32_t by_matrix, pad;  // 1: a workgroup takes it by itself (X transposed in the workspace)
    int64_t off;         // byte offset of the matrix's buffers in the workspace
};

struct NsTile {
    int32_t mat, ti, tj;  // mat < 0: nothing to do
};

// the matrices of a call and the tiles of a launch: from tables, or (null) of
// a uniform stack, matrix k at k times the strides
struct NsWork {
    const NsMat *mats;
    const NsTile *tiles;
    NsMat uni;
    int64_t in_stride, ws_stride;  // bytes per matrix of in and out, and of the workspace
    int32_t n_mats, nti, ntj;      // stack: matrices, and tiles per matrix of this launch
    char *ws;                      // workspace behind the partial sums
    double *part;                  // partial sums of squares
    int *levels;                   // per matrix: how far its norm lies below eps, see Scales
};

struct NsParams {
    // X and A are held times `scale`, P times a scale of its own, all powers of two.  P's coefficients with what
    // brings A A and A to P's scale, and the factors of the products X X^T, P X and the last P X; growth: log2 of
    // what a step multiplies a singular value with at most, 0 where it shrinks
    float poly_a, poly_b, poly_c, from_gram, from_apply, from_last, growth;
    double scale, eps;
    int steps;
    // Muon (fp32): m = mu m + om_mu g, u = u_g g + u_m m, p = decay p - lr scale O, w = sd w + om_sd p
    float mu, om_mu, u_g, u_m, decay, lr, sd, om_sd;
    const float *grad_scale;
};

// The parts of a call.  n_small matrices from first_small on fit into a
// workgroup's LDS (small_lds bytes) and take one launch.  The others have work lists, each
// a launch's grid: x, tiles of 64 x 64 entries, for norm, scaling and update.  Of them n_wg8 (up to 8
// units of 32 rows) and n_wg4 (up to 4) go through the steps a workgroup each, the rest by the products'
// tiles of `tile` x `tile`: gram, the Gram matrix's upper triangle, and apply, the iterate
struct NsLists {
    int64_t n_small, first_small, small_lds;
    int64_t n_wg8, first_wg8, n_wg4, first_wg4;
    int tile;                         // 64 or 128
    int64_t n_x, n_gram, n_apply;     // entries, padding included
    const NsTile *x, *gram, *apply;   // device tables, or null for a stack
};

constexpr int kNsBlock = 64;  // tiles of the norm and scaling passes

// LDS that a matrix takes as a whole, 0 if it does not fit
int64_t ns_small_bytes(int64_t rows, int64_t cols);
// 8 or 4: the form of workgroup that can take the matrix by itself, 0 if none
int ns_matrix_rows(int64_t rows, int64_t cols);
int64_t ns_matrix_wg_bytes(int64_t rows, int64_t cols);  // its buffers then
// whether matrices of this much work in all, and the largest alone, are done a workgroup each
bool ns_by_matrix(double total, double largest);
// bytes of a matrix's buffers in the workspace where it does not fit
int64_t ns_matrix_bytes(int64_t rows, int64_t cols);
// tiles of the products for a call whose Gram matrices' triangles have this many 128 x 128 tiles
int ns_tile(int64_t gram128);

hipError_t launch_ns(const NsWork &w, const NsLists &l, const NsParams &p, bool muon, bool bf16, hipStream_t s);

}  // namespace evo

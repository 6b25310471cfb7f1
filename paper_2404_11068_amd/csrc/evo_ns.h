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
    int64_t off;         // byte offset of the matrix's buffers in the workspace
};

struct NsTile {
    int32_t mat, ti, tj;
};

// the matrices of a call and the tiles of a launch: from tables, or (null) of
// a uniform stack, matrix k at k times the strides
struct NsWork {
    const NsMat *mats;
    const NsTile *tiles;
    NsMat uni;
    int64_t in_stride, ws_stride;  // bytes per matrix of in and out, and of the workspace
    int32_t nti, ntj;              // tiles per matrix of this launch
    char *ws;                      // workspace behind the partial sums
    double *part;                  // partial sums of squares
};

struct NsParams {
    float a, b, c;
    double eps;
    int steps;
    // Muon (fp32): u = bm_g g + bm_m m
    float mu, om_mu, u_g, u_m, decay, lr, sd, om_sd;
    const float *grad_scale;
};

// bytes of a matrix's buffers in the workspace
int64_t ns_matrix_bytes(int64_t rows, int64_t cols);

constexpr int kNsTile = 64;  // tiles of the lists

hipError_t launch_ns(NsWork w, const NsParams &p, bool muon, bool bf16, int64_t n_x, const NsTile *tiles_x, int64_t n_a,
                     const NsTile *tiles_a, hipStream_t s);

}  // namespace evo

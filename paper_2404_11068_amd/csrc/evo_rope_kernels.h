// evo_rope_kernels.h -- internal launch interface of the rotary kernels (the public ABI is include/evo_rope.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace evo {

struct RopeSet {
    const void *in;   // x (forward), dy (backward)
    const void *x;    // x of the norm's backward
    const int32_t *pos;
    const float *w;
    void *out;        // y, dx
    float *dw;
    int64_t tokens, len, pos_stride;
    int64_t in_row, in_tok, x_row, x_tok, out_row, out_tok;
    int heads;
};

struct RopeArgs {
    RopeSet set[2];
    const uint64_t *steps;
    int bf16, d, rot, interleaved, norm;
    float eps, amplitude;
};

size_t rope_bwd_workspace(const RopeArgs &a);
hipError_t launch_rope_fwd(const RopeArgs &a, hipStream_t s);
hipError_t launch_rope_bwd(const RopeArgs &a, void *ws, hipStream_t s);

}  // namespace evo

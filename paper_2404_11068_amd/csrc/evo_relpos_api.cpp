// evo_relpos_api.cpp -- the C ABI declared in include/evo_relpos.h: validation
// (before any HIP call) and dispatch.
#include "evo_relpos.h"

#include <hip/hip_runtime.h>

#include "evo_kernels.h"

namespace {

bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

int check_relpos(const evo_relpos_dims *d) {
    if (!d || d->reserved != 0) return EVO_ERR_INVALID_ARG;
    if (d->dtype != EVO_DTYPE_F32 && d->dtype != EVO_DTYPE_BF16) return EVO_ERR_UNSUPPORTED;
    if (d->n_heads < 1 || d->n_edges < 0 || (d->has_seg != 0 && d->has_seg != 1) || d->n_batch < 0 || d->len_i < 0 ||
        d->len_j < 0)
        return EVO_ERR_INVALID_ARG;
    const int64_t most_len = int64_t(1) << 20, most = int64_t(1) << 40;
    if (d->n_heads > 65535 || d->n_edges > 1022 || d->len_i > most_len || d->len_j > most_len || d->n_batch > most)
        return EVO_ERR_UNSUPPORTED;
    const int64_t plane = d->len_i * d->len_j;  // <= 2^40
    if (plane > 0 && d->n_batch > most / plane / d->n_heads) return EVO_ERR_UNSUPPORTED;
    if (plane > 0 && d->n_batch * d->n_heads > 0x7fffffff) return EVO_ERR_UNSUPPORTED;
    return EVO_OK;
}

evo::RpArgs rp_args(const evo_relpos_dims *d, const int32_t *pos_i, const int32_t *pos_j, const int32_t *seg_i,
                    const int32_t *seg_j, const int32_t *edges) {
    evo::RpArgs a{};
    a.pos_i = pos_i;
    a.pos_j = pos_j;
    a.seg_i = seg_i;
    a.seg_j = seg_j;
    a.edges = edges;
    a.B = d->n_batch;
    a.H = d->n_heads;
    a.Li = (int)d->len_i;
    a.Lj = (int)d->len_j;
    a.E = d->n_edges;
    a.NB = d->n_edges + 1 + d->has_seg;
    return a;
}

// pointers both directions share
int check_index(const evo_relpos_dims *d, const int32_t *pos_i, const int32_t *pos_j, const int32_t *seg_i,
                const int32_t *seg_j, const int32_t *edges) {
    if (!pos_i || !pos_j || (d->n_edges > 0 && !edges)) return EVO_ERR_INVALID_ARG;
    if ((seg_i != nullptr) != (d->has_seg == 1) || (seg_j != nullptr) != (d->has_seg == 1)) return EVO_ERR_INVALID_ARG;
    if (!aligned(pos_i, 4) || !aligned(pos_j, 4) || !aligned(seg_i, 4) || !aligned(seg_j, 4) || !aligned(edges, 4))
        return EVO_ERR_ALIGNMENT;
    return EVO_OK;
}

}  // namespace

extern "C" {

int evo_relpos_fwd(const evo_relpos_dims *d, const int32_t *pos_i, const int32_t *pos_j, const int32_t *seg_i,
                   const int32_t *seg_j, const int32_t *edges, const float *table, const void *base, void *out,
                   void *stream) {
    int st = check_relpos(d);
    if (st) return st;
    if (d->n_batch == 0 || d->len_i == 0 || d->len_j == 0) return EVO_OK;
    st = check_index(d, pos_i, pos_j, seg_i, seg_j, edges);
    if (st) return st;
    if (!table || !out || (const void *)table == out) return EVO_ERR_INVALID_ARG;
    const size_t es = d->dtype == EVO_DTYPE_BF16 ? 2 : 4;
    if (base && base != out) {  // in place or apart
        const size_t bytes = (size_t)(d->n_batch * d->n_heads * d->len_i * d->len_j) * es;
        const uintptr_t b = (uintptr_t)base, o = (uintptr_t)out;
        if (b < o ? o - b < bytes : b - o < bytes) return EVO_ERR_INVALID_ARG;
    }
    if (!aligned(table, 4) || !aligned(base, es) || !aligned(out, es)) return EVO_ERR_ALIGNMENT;
    evo::RpArgs a = rp_args(d, pos_i, pos_j, seg_i, seg_j, edges);
    a.table = table;
    a.base = base;
    a.out = out;
    a.bf16 = d->dtype == EVO_DTYPE_BF16;
    return evo::launch_relpos_fwd(a, (hipStream_t)stream) == hipSuccess ? EVO_OK : EVO_ERR_HIP;
}

size_t evo_relpos_bwd_workspace_size(const evo_relpos_dims *d) {
    if (check_relpos(d) || d->n_batch == 0 || d->len_i == 0 || d->len_j == 0) return 0;
    return evo::relpos_bwd_workspace(rp_args(d, nullptr, nullptr, nullptr, nullptr, nullptr));
}

int evo_relpos_bwd(const evo_relpos_dims *d, const int32_t *pos_i, const int32_t *pos_j, const int32_t *seg_i,
                   const int32_t *seg_j, const int32_t *edges, const float *dbias, float *dtable, void *workspace,
                   size_t workspace_bytes, void *stream) {
    int st = check_relpos(d);
    if (st) return st;
    if (!dtable) return EVO_ERR_INVALID_ARG;
    if (!aligned(dtable, 4)) return EVO_ERR_ALIGNMENT;
    evo::RpArgs a = rp_args(d, pos_i, pos_j, seg_i, seg_j, edges);
    a.dtable = dtable;
    if (d->n_batch > 0 && d->len_i > 0 && d->len_j > 0) {
        st = check_index(d, pos_i, pos_j, seg_i, seg_j, edges);
        if (st) return st;
        if (!dbias || dbias == dtable) return EVO_ERR_INVALID_ARG;
        if (!aligned(dbias, 4)) return EVO_ERR_ALIGNMENT;
        const size_t need = evo::relpos_bwd_workspace(a);
        if (need > 0 && (!workspace || workspace_bytes < need)) return EVO_ERR_WORKSPACE;
        if (need > 0 && !aligned(workspace, 16)) return EVO_ERR_ALIGNMENT;
        a.dbias = dbias;
    }
    return evo::launch_relpos_bwd(a, workspace, (hipStream_t)stream) == hipSuccess ? EVO_OK : EVO_ERR_HIP;
}

}  // extern "C"

// evo_rope_api.cpp -- the C ABI declared in include/evo_rope.h: validation
// (before any HIP call) and dispatch.
#include "evo_rope.h"

#include <hip/hip_runtime.h>
#include <math.h>

#include "evo_rope_kernels.h"
#include "evo_views.h"

namespace {

bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

bool empty(const evo_rope_dims *d, int i) { return d->n_rows == 0 || d->len[i] == 0 || d->n_heads[i] == 0; }

// the (row, token) grid of blocks of `block` elements does not overlap itself
bool apart(const evo_rope_dims *d, int i, int64_t row, int64_t tok) {
    const int64_t block = (int64_t)d->n_heads[i] * d->head_dim, n = d->n_rows, l = d->len[i];
    if ((l > 1 && tok < block) || (n > 1 && row < block)) return false;
    if (n == 1 || l == 1) return true;
    return row >= (l - 1) * tok + block || tok >= (n - 1) * row + block;
}

int check_dims(const evo_rope_dims *d, bool bwd) {
    if (!d) return EVO_ERR_INVALID_ARG;
    if (d->dtype != EVO_DTYPE_F32 && d->dtype != EVO_DTYPE_BF16) return EVO_ERR_UNSUPPORTED;
    if (d->flags & ~(EVO_ROPE_INTERLEAVED | EVO_ROPE_NORM)) return EVO_ERR_INVALID_ARG;
    if (d->head_dim < 1 || d->rot_dim < 0 || d->rot_dim > d->head_dim || d->rot_dim % 2 != 0) return EVO_ERR_INVALID_ARG;
    if (d->head_dim % 8 != 0 || d->head_dim > 256) return EVO_ERR_UNSUPPORTED;
    if (d->n_rows < 0 || !isfinite(d->amplitude)) return EVO_ERR_INVALID_ARG;
    if ((d->flags & EVO_ROPE_NORM) && !(d->eps >= 0.0f && isfinite(d->eps))) return EVO_ERR_INVALID_ARG;
    const int64_t most = int64_t(1) << 40, es = d->dtype == EVO_DTYPE_BF16 ? 2 : 4;
    for (int i = 0; i < 2; ++i) {
        if (d->n_heads[i] < (i == 0 ? 1 : 0) || d->len[i] < 0 || d->pos_stride[i] < 0) return EVO_ERR_INVALID_ARG;
        if (d->n_heads[i] > 65535 || d->len[i] > (int64_t(1) << 30) || d->n_rows > most || d->pos_stride[i] > most)
            return EVO_ERR_UNSUPPORTED;
        if (empty(d, i)) continue;
        const int64_t block = (int64_t)d->n_heads[i] * d->head_dim;
        if (d->n_rows > most / block / d->len[i]) return EVO_ERR_UNSUPPORTED;
        const int64_t st[4] = {d->x_stride_row[i], d->x_stride_tok[i], d->y_stride_row[i], d->y_stride_tok[i]};
        for (int64_t v : st) {
            if (v < 0) return EVO_ERR_INVALID_ARG;
            if (v > most) return EVO_ERR_UNSUPPORTED;
            if (v * es % 16 != 0) return EVO_ERR_ALIGNMENT;
        }
        // the strides times their counts stay far inside 64 bits
        if (d->n_rows > (most << 10) / (st[0] + 1) || d->n_rows > (most << 10) / (st[2] + 1) ||
            d->len[i] > (most << 10) / (st[1] + 1) || d->len[i] > (most << 10) / (st[3] + 1) ||
            d->n_rows > (most << 10) / (d->pos_stride[i] + 1))
            return EVO_ERR_UNSUPPORTED;
        if (bwd ? !apart(d, i, st[0], st[1]) : !apart(d, i, st[2], st[3])) return EVO_ERR_INVALID_ARG;
    }
    return EVO_OK;
}

evo::View view(const evo_rope_dims *d, int i, const void *p, int64_t row, int64_t tok) {
    const int64_t es = d->dtype == EVO_DTYPE_BF16 ? 2 : 4;
    return evo::View{(uintptr_t)p, row * es, tok * es, d->n_rows, d->len[i], (int64_t)d->n_heads[i] * d->head_dim * es};
}

// in place (one address, one pair of strides) or apart
bool overlap_ok(const evo_rope_dims *d, int i, const void *in, int64_t ir, int64_t it, const void *out, int64_t orow,
                int64_t otok) {
    if (in == out && (ir == orow || d->n_rows == 1) && (it == otok || d->len[i] == 1)) return true;
    return evo::views_apart(view(d, i, in, ir, it), view(d, i, out, orow, otok));
}

// what one set writes and another tensor of the other set: apart, which blocks of one packed buffer are, too
bool sets_ok(const evo_rope_dims *d, int i, const void *out, int64_t orow, int64_t otok, int j, const void *other,
             int64_t row, int64_t tok) {
    if (empty(d, i) || empty(d, j) || !other) return true;
    return evo::views_apart(view(d, i, out, orow, otok), view(d, j, other, row, tok));
}

void fill(const evo_rope_dims *d, evo::RopeArgs *a) {
    for (int i = 0; i < 2; ++i) {
        evo::RopeSet &s = a->set[i];
        s.heads = d->n_heads[i];
        s.len = d->len[i] > 0 ? d->len[i] : 1;
        s.tokens = empty(d, i) ? 0 : d->n_rows * d->len[i];
        s.pos_stride = d->pos_stride[i];
    }
    a->bf16 = d->dtype == EVO_DTYPE_BF16;
    a->d = d->head_dim;
    a->rot = d->rot_dim;
    a->interleaved = (d->flags & EVO_ROPE_INTERLEAVED) != 0;
    a->norm = (d->flags & EVO_ROPE_NORM) != 0;
    a->eps = d->eps;
    a->amplitude = d->amplitude;
}

}  // namespace

extern "C" {

int evo_rope_fwd(const evo_rope_dims *d, const void *x0, const void *x1, const int32_t *pos0, const int32_t *pos1,
                 const uint64_t *steps, const float *w0, const float *w1, void *y0, void *y1, void *stream) {
    int st = check_dims(d, false);
    if (st) return st;
    const void *x[2] = {x0, x1};
    const int32_t *pos[2] = {pos0, pos1};
    const float *w[2] = {w0, w1};
    void *y[2] = {y0, y1};
    evo::RopeArgs a{};
    fill(d, &a);
    if (!a.norm && (w0 || w1)) return EVO_ERR_INVALID_ARG;
    for (int i = 0; i < 2; ++i) {
        if (empty(d, i)) continue;
        if (!x[i] || !y[i] || (d->rot_dim > 0 && (!pos[i] || !steps))) return EVO_ERR_INVALID_ARG;
        if (!aligned(x[i], 16) || !aligned(y[i], 16) || !aligned(pos[i], 4) || !aligned(steps, 8) || !aligned(w[i], 4))
            return EVO_ERR_ALIGNMENT;
        if (!overlap_ok(d, i, x[i], d->x_stride_row[i], d->x_stride_tok[i], y[i], d->y_stride_row[i], d->y_stride_tok[i]))
            return EVO_ERR_INVALID_ARG;
        evo::RopeSet &s = a.set[i];
        s.in = x[i];
        s.pos = pos[i];
        s.w = w[i];
        s.out = y[i];
        s.in_row = d->x_stride_row[i];
        s.in_tok = d->x_stride_tok[i];
        s.out_row = d->y_stride_row[i];
        s.out_tok = d->y_stride_tok[i];
    }
    for (int i = 0; i < 2; ++i)
        if (!sets_ok(d, i, y[i], d->y_stride_row[i], d->y_stride_tok[i], 1 - i, x[1 - i], d->x_stride_row[1 - i],
                     d->x_stride_tok[1 - i]) ||
            !sets_ok(d, i, y[i], d->y_stride_row[i], d->y_stride_tok[i], 1 - i, y[1 - i], d->y_stride_row[1 - i],
                     d->y_stride_tok[1 - i]))
            return EVO_ERR_INVALID_ARG;
    a.steps = steps;
    return evo::launch_rope_fwd(a, (hipStream_t)stream) == hipSuccess ? EVO_OK : EVO_ERR_HIP;
}

size_t evo_rope_bwd_workspace_size(const evo_rope_dims *d) {
    if (check_dims(d, true)) return 0;
    evo::RopeArgs a{};
    fill(d, &a);
    return evo::rope_bwd_workspace(a);
}

int evo_rope_bwd(const evo_rope_dims *d, const void *dy0, const void *dy1, const void *x0, const void *x1,
                 const int32_t *pos0, const int32_t *pos1, const uint64_t *steps, const float *w0, const float *w1,
                 void *dx0, void *dx1, float *dw0, float *dw1, void *workspace, size_t workspace_bytes, void *stream) {
    int st = check_dims(d, true);
    if (st) return st;
    const void *dy[2] = {dy0, dy1}, *x[2] = {x0, x1};
    const int32_t *pos[2] = {pos0, pos1};
    const float *w[2] = {w0, w1};
    void *dx[2] = {dx0, dx1};
    float *dw[2] = {dw0, dw1};
    evo::RopeArgs a{};
    fill(d, &a);
    if (!a.norm && (w0 || w1)) return EVO_ERR_INVALID_ARG;
    for (int i = 0; i < 2; ++i) {
        if ((w[i] != nullptr) != (dw[i] != nullptr)) return EVO_ERR_INVALID_ARG;
        if (!aligned(dw[i], 4) || !aligned(w[i], 4)) return EVO_ERR_ALIGNMENT;
        a.set[i].dw = dw[i];
        if (empty(d, i)) continue;
        if (!dy[i] || !dx[i] || (a.norm && !x[i]) || (d->rot_dim > 0 && (!pos[i] || !steps))) return EVO_ERR_INVALID_ARG;
        if (!aligned(dy[i], 16) || !aligned(dx[i], 16) || !aligned(x[i], 16) || !aligned(pos[i], 4) || !aligned(steps, 8))
            return EVO_ERR_ALIGNMENT;
        if (!overlap_ok(d, i, dy[i], d->y_stride_row[i], d->y_stride_tok[i], dx[i], d->x_stride_row[i], d->x_stride_tok[i]))
            return EVO_ERR_INVALID_ARG;
        if (a.norm && !overlap_ok(d, i, x[i], d->x_stride_row[i], d->x_stride_tok[i], dx[i], d->x_stride_row[i], d->x_stride_tok[i]))
            return EVO_ERR_INVALID_ARG;
        evo::RopeSet &s = a.set[i];
        s.in = dy[i];
        s.x = x[i];
        s.pos = pos[i];
        s.w = w[i];
        s.out = dx[i];
        s.in_row = d->y_stride_row[i];
        s.in_tok = d->y_stride_tok[i];
        s.x_row = s.out_row = d->x_stride_row[i];
        s.x_tok = s.out_tok = d->x_stride_tok[i];
    }
    if (dw0 && dw0 == dw1) return EVO_ERR_INVALID_ARG;
    for (int i = 0; i < 2; ++i)
        if (!sets_ok(d, i, dx[i], d->x_stride_row[i], d->x_stride_tok[i], 1 - i, dy[1 - i], d->y_stride_row[1 - i],
                     d->y_stride_tok[1 - i]) ||
            !sets_ok(d, i, dx[i], d->x_stride_row[i], d->x_stride_tok[i], 1 - i, dx[1 - i], d->x_stride_row[1 - i],
                     d->x_stride_tok[1 - i]) ||
            (a.norm && !sets_ok(d, i, dx[i], d->x_stride_row[i], d->x_stride_tok[i], 1 - i, x[1 - i],
                                d->x_stride_row[1 - i], d->x_stride_tok[1 - i])))
            return EVO_ERR_INVALID_ARG;
    a.steps = steps;
    const size_t need = evo::rope_bwd_workspace(a);
    if (need > 0 && (!workspace || workspace_bytes < need)) return EVO_ERR_WORKSPACE;
    if (need > 0 && !aligned(workspace, 16)) return EVO_ERR_ALIGNMENT;
    return evo::launch_rope_bwd(a, workspace, (hipStream_t)stream) == hipSuccess ? EVO_OK : EVO_ERR_HIP;
}

}  // extern "C"

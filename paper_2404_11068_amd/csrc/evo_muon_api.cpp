// evo_muon_api.cpp -- the C ABI declared in include/evo_muon.h: host-side
// plans, validation (before any HIP call) and dispatch.
#include "evo_muon.h"

#include <hip/hip_runtime.h>
#include <math.h>
#include <string.h>

#include "evo_ns.h"

namespace {

using evo::kNsTile;
using evo::NsMat;
using evo::NsTile;

constexpr int64_t kMostSide = 32768;

bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

int64_t tiles_of(int64_t n) { return (n + kNsTile - 1) / kNsTile; }

// whether the iterate stays in the kernels' range: the largest singular value,
// followed from 1 (no singular value of X exceeds the Frobenius norm) through
// the steps' polynomial, sampled finely enough that a step between two samples
// adds less than the margin left below the range's end
int check_coefs(double a, double b, double c, double eps, int steps) {
    if (!isfinite(a) || !isfinite(b) || !isfinite(c) || !(eps > 0.0) || !isfinite(eps) || steps < 1)
        return EVO_ERR_INVALID_ARG;
    if (steps > 64) return EVO_ERR_UNSUPPORTED;
    double top = 1.0;
    for (int k = 0; k < steps; ++k) {
        const double t2 = top * top;
        if (!(top <= 8.0) || !(fabs(a) + fabs(b) * t2 + fabs(c) * t2 * t2 <= 60.0)) return EVO_ERR_UNSUPPORTED;
        double next = 0.0;
        for (int i = 0; i <= 1024; ++i) {
            const double s = top * i / 1024.0, s2 = s * s;
            next = fmax(next, fabs(s * (a + s2 * (b + s2 * c))));
        }
        top = next;
    }
    return top <= 8.0 ? EVO_OK : EVO_ERR_UNSUPPORTED;
}

// ---- Muon plan: header, matrices, tiles of the iterate, tiles of the Gram matrix
struct PlanHeader {
    uint64_t magic;
    int64_t bytes, n_mats, n_x, n_a, ws_bytes, part_bytes;
    int64_t off_mats, off_x, off_a;
};
constexpr uint64_t kMagic = 0x45564f4d554f4e31ull;

int64_t round256(int64_t n) { return (n + 255) & ~int64_t(255); }

bool measure(const evo_muon_tensor *t, int32_t n, PlanHeader &h) {
    if (n < 0 || (n > 0 && !t)) return false;
    h = PlanHeader{};
    for (int32_t i = 0; i < n; ++i) {
        if (t[i].rows < 0 || t[i].cols < 0 || t[i].rows > kMostSide || t[i].cols > kMostSide) return false;
        if (t[i].rows == 0 || t[i].cols == 0) continue;
        const int64_t r = t[i].rows < t[i].cols ? t[i].rows : t[i].cols, c = t[i].rows + t[i].cols - r;
        ++h.n_mats;
        h.n_x += tiles_of(r) * tiles_of(c);
        h.n_a += tiles_of(r) * tiles_of(r);
        h.ws_bytes += evo::ns_matrix_bytes(t[i].rows, t[i].cols);
        if (h.n_x > 0x7fffffff) return false;
    }
    h.magic = kMagic;
    h.part_bytes = round256(h.n_x * 8);
    h.ws_bytes += h.part_bytes;
    h.off_mats = round256(sizeof(PlanHeader));
    h.off_x = h.off_mats + round256(h.n_mats * (int64_t)sizeof(NsMat));
    h.off_a = h.off_x + round256(h.n_x * (int64_t)sizeof(NsTile));
    h.bytes = h.off_a + round256(h.n_a * (int64_t)sizeof(NsTile));
    return true;
}

int check_orth(const evo_orth_dims *d) {
    if (!d || d->reserved != 0) return EVO_ERR_INVALID_ARG;
    if (d->dtype != EVO_DTYPE_F32 && d->dtype != EVO_DTYPE_BF16) return EVO_ERR_UNSUPPORTED;
    if (d->n_batch < 0 || d->rows < 0 || d->cols < 0) return EVO_ERR_INVALID_ARG;
    if (d->n_batch > (1 << 20) || d->rows > kMostSide || d->cols > kMostSide) return EVO_ERR_UNSUPPORTED;
    if (d->n_batch * tiles_of(d->rows) * tiles_of(d->cols) > 0x7fffffff) return EVO_ERR_UNSUPPORTED;
    return check_coefs(d->a, d->b, d->c, d->eps, d->steps);
}

bool orth_empty(const evo_orth_dims *d) { return d->n_batch == 0 || d->rows == 0 || d->cols == 0; }

size_t orth_workspace(const evo_orth_dims *d) {
    return (size_t)(round256(d->n_batch * tiles_of(d->rows) * tiles_of(d->cols) * 8) +
                    d->n_batch * evo::ns_matrix_bytes(d->rows, d->cols));
}

}  // namespace

extern "C" {

size_t evo_orthogonalize_workspace_size(const evo_orth_dims *d) {
    if (check_orth(d) || orth_empty(d)) return 0;
    return orth_workspace(d);
}

int evo_orthogonalize(const evo_orth_dims *d, const void *x, void *out, void *workspace, size_t workspace_bytes,
                      void *stream) {
    const int st = check_orth(d);
    if (st) return st;
    if (orth_empty(d)) return EVO_OK;
    if (!x || !out) return EVO_ERR_INVALID_ARG;
    const int64_t es = d->dtype == EVO_DTYPE_BF16 ? 2 : 4, each = d->rows * d->cols * es;
    if (x != out) {
        const uintptr_t p = (uintptr_t)x, q = (uintptr_t)out, all = (uintptr_t)(d->n_batch * each);
        if (p < q ? q - p < all : p - q < all) return EVO_ERR_INVALID_ARG;
    }
    if (!aligned(x, es) || !aligned(out, es)) return EVO_ERR_ALIGNMENT;
    const size_t need = orth_workspace(d);
    if (!workspace || workspace_bytes < need) return EVO_ERR_WORKSPACE;
    if (!aligned(workspace, 256)) return EVO_ERR_ALIGNMENT;
    const int64_t r = d->rows < d->cols ? d->rows : d->cols, c = d->rows + d->cols - r;
    const int64_t n_x = tiles_of(r) * tiles_of(c), n_a = tiles_of(r) * tiles_of(r);
    evo::NsWork w{};
    w.uni.in = x;
    w.uni.out = out;
    w.uni.rows = (int32_t)d->rows;
    w.uni.cols = (int32_t)d->cols;
    w.in_stride = each;
    w.ws_stride = evo::ns_matrix_bytes(d->rows, d->cols);
    w.part = (double *)workspace;
    w.ws = (char *)workspace + round256(d->n_batch * n_x * 8);
    evo::NsParams p{};
    p.a = (float)d->a;
    p.b = (float)d->b;
    p.c = (float)d->c;
    p.eps = d->eps;
    p.steps = d->steps;
    return evo::launch_ns(w, p, false, d->dtype == EVO_DTYPE_BF16, d->n_batch * n_x, nullptr, d->n_batch * n_a, nullptr,
                          (hipStream_t)stream) == hipSuccess
               ? EVO_OK
               : EVO_ERR_HIP;
}

int64_t evo_muon_plan_bytes(const evo_muon_tensor *tensors, int32_t n_tensors) {
    PlanHeader h;
    return measure(tensors, n_tensors, h) ? h.bytes : -1;
}

int evo_muon_build_plan(const evo_muon_tensor *tensors, int32_t n_tensors, void *plan, size_t plan_bytes) {
    PlanHeader h;
    if (!measure(tensors, n_tensors, h) || !plan) return EVO_ERR_INVALID_ARG;
    if (!aligned(plan, 8)) return EVO_ERR_ALIGNMENT;
    if (plan_bytes < (size_t)h.bytes) return EVO_ERR_WORKSPACE;
    for (int32_t i = 0; i < n_tensors; ++i) {
        const evo_muon_tensor &t = tensors[i];
        if (t.rows == 0 || t.cols == 0) continue;
        if (!t.param || !t.grad || !t.momentum || !isfinite(t.update_scale)) return EVO_ERR_INVALID_ARG;
        if (!aligned(t.param, 4) || !aligned(t.grad, 4) || !aligned(t.momentum, 4) || !aligned(t.swa, 4))
            return EVO_ERR_ALIGNMENT;
    }
    memset(plan, 0, (size_t)h.bytes);
    memcpy(plan, &h, sizeof h);
    NsMat *mats = (NsMat *)((char *)plan + h.off_mats);
    NsTile *tx = (NsTile *)((char *)plan + h.off_x), *ta = (NsTile *)((char *)plan + h.off_a);
    int32_t m = 0, part = 0;
    int64_t off = 0;
    for (int32_t i = 0; i < n_tensors; ++i) {
        const evo_muon_tensor &t = tensors[i];
        if (t.rows == 0 || t.cols == 0) continue;
        const int64_t r = t.rows < t.cols ? t.rows : t.cols, c = t.rows + t.cols - r;
        NsMat &M = mats[m];
        M.in = t.grad;
        M.out = t.param;
        M.mom = t.momentum;
        M.swa = t.swa;
        M.rows = (int32_t)t.rows;
        M.cols = (int32_t)t.cols;
        M.scale = (float)t.update_scale;
        M.part0 = part;
        M.off = off;
        off += evo::ns_matrix_bytes(t.rows, t.cols);
        for (int32_t ti = 0; ti < tiles_of(r); ++ti)
            for (int32_t tj = 0; tj < tiles_of(c); ++tj, ++part) *tx++ = NsTile{m, ti, tj};
        for (int32_t ti = 0; ti < tiles_of(r); ++ti)
            for (int32_t tj = 0; tj < tiles_of(r); ++tj) *ta++ = NsTile{m, ti, tj};
        ++m;
    }
    return EVO_OK;
}

size_t evo_muon_workspace_size(const void *plan) {
    const PlanHeader *h = (const PlanHeader *)plan;
    return h && h->magic == kMagic ? (size_t)h->ws_bytes : 0;
}

int evo_muon_step(const evo_muon_hparams *hp, const void *plan, const void *plan_device, const float *grad_scale,
                  void *workspace, size_t workspace_bytes, void *stream) {
    if (!hp || !plan || !aligned(plan, 8)) return EVO_ERR_INVALID_ARG;
    const PlanHeader &h = *(const PlanHeader *)plan;
    if (h.magic != kMagic) return EVO_ERR_INVALID_ARG;
    const double f[] = {hp->lr, hp->momentum, hp->weight_decay, hp->swa_decay};
    for (double x : f)
        if (!isfinite(x)) return EVO_ERR_INVALID_ARG;
    if (hp->momentum < 0.0 || hp->momentum >= 1.0 || hp->swa_decay < 0.0 || hp->swa_decay > 1.0 ||
        (hp->nesterov != 0 && hp->nesterov != 1))
        return EVO_ERR_INVALID_ARG;
    const int st = check_coefs(hp->a, hp->b, hp->c, hp->eps, hp->steps);
    if (st) return st;
    if (h.n_mats == 0) return EVO_OK;
    if (!plan_device) return EVO_ERR_INVALID_ARG;
    if (!aligned(plan_device, 8) || !aligned(grad_scale, 4)) return EVO_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < (size_t)h.ws_bytes) return EVO_ERR_WORKSPACE;
    if (!aligned(workspace, 256)) return EVO_ERR_ALIGNMENT;
    const char *dev = (const char *)plan_device;
    evo::NsWork w{};
    w.mats = (const NsMat *)(dev + h.off_mats);
    w.part = (double *)workspace;
    w.ws = (char *)workspace + h.part_bytes;
    evo::NsParams p{};
    p.a = (float)hp->a;
    p.b = (float)hp->b;
    p.c = (float)hp->c;
    p.eps = hp->eps;
    p.steps = hp->steps;
    p.mu = (float)hp->momentum;
    p.om_mu = (float)(1.0 - hp->momentum);
    p.u_g = hp->nesterov ? p.om_mu : 0.0f;
    p.u_m = hp->nesterov ? p.mu : 1.0f;
    p.decay = (float)(1.0 - hp->lr * hp->weight_decay);
    p.lr = (float)hp->lr;
    p.sd = (float)hp->swa_decay;
    p.om_sd = (float)(1.0 - hp->swa_decay);
    p.grad_scale = grad_scale;
    return evo::launch_ns(w, p, true, false, h.n_x, (const NsTile *)(dev + h.off_x), h.n_a,
                          (const NsTile *)(dev + h.off_a), (hipStream_t)stream) == hipSuccess
               ? EVO_OK
               : EVO_ERR_HIP;
}

}  // extern "C"

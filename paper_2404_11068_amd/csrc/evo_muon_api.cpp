// evo_muon_api.cpp -- the C ABI declared in include/evo_muon.h: host-side
// plans, validation (before any HIP call) and dispatch.
#include "evo_muon.h"

#include <hip/hip_runtime.h>
#include <math.h>
#include <string.h>

#include <algorithm>
#include <vector>

#include "evo_ns.h"

namespace {

using evo::NsLists;
using evo::NsMat;
using evo::NsTile;

constexpr int64_t kMostSide = 32768;
// workgroups of a launch: HIP takes fewer than 2^32 threads, and up to 256 are in one here
constexpr int64_t kMostBlocks = (int64_t(1) << 24) - 1;

bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

int64_t tiles_of(int64_t n, int64_t tile) { return (n + tile - 1) / tile; }
int64_t triangle(int64_t n) { return n * (n + 1) / 2; }
int64_t blocks_of(int64_t rows, int64_t cols) { return tiles_of(rows, evo::kNsBlock) * tiles_of(cols, evo::kNsBlock); }

// Whether the iterate stays in range: the largest singular value, followed from 1 (no
// singular value of X exceeds the Frobenius norm) through the steps.  Each takes s of [0, top] to
// |a s + b s^3 + c s^5|, whose largest value lies at the end or where a + 3 b t + 5 c t^2 = 0, t = s^2.
// p: the coefficients and scales as the kernels take them
int check_coefs(double a, double b, double c, double eps, int steps, evo::NsParams *p = nullptr) {
    if (!isfinite(a) || !isfinite(b) || !isfinite(c) || !(eps > 0.0) || !isfinite(eps) || steps < 1)
        return EVO_ERR_INVALID_ARG;
    if (steps > 64 || fabs(a) + fabs(b) + fabs(c) > 60.0) return EVO_ERR_UNSUPPORTED;
    auto value = [&](double t) { return fabs(sqrt(t) * (a + t * (b + t * c))); };
    const double disc = 9.0 * b * b - 20.0 * a * c, q = -0.5 * (3.0 * b + copysign(sqrt(fmax(disc, 0.0)), b));
    const double turns[] = {disc >= 0.0 && c != 0.0 ? q / (5.0 * c) : 0.0, disc >= 0.0 && q != 0.0 ? a / q : 0.0};  // (0: none)
    auto largest = [&](double t2) {
        double v = value(t2);
        for (const double t : turns)
            if (t > 0.0 && t < t2) v = fmax(v, value(t));
        return v;
    };
    // `wide` is followed with room for the steps' roundings, far below 2^-12 each, and is what the scales go by
    double top = 1.0, wide = 1.0, most = 1.0;
    for (int k = 0; k < steps; ++k) {
        const double t2 = top * top;
        if (top > 8.0 || fabs(a) + fabs(b) * t2 + fabs(c) * t2 * t2 > 60.0) return EVO_ERR_UNSUPPORTED;
        most = fmax(most, wide);
        top = largest(t2);
        wide = fmin(largest(wide * wide) * (1.0 + 0x1p-12), 16.0);
    }
    if (top > 8.0) return EVO_ERR_UNSUPPORTED;
    if (!p) return EVO_OK;
    // Entries are at most the matrices' largest singular values: `most` for X, its square for A, and for P
    // the largest |a + b t + c t^2| up to there, at an end or where b + 2 c t = 0
    const double t2 = most * most, turn = c != 0.0 ? -b / (2.0 * c) : 0.0;
    double gain = fmax(1.0, fmax(fabs(a), fabs(a + t2 * (b + t2 * c))));
    if (turn > 0.0 && turn < t2) gain = fmax(gain, fabs(a + turn * (b + turn * c)));
    const double xs = exp2(floor(log2(65000.0 / t2))), ps = exp2(floor(log2(65000.0 / gain)));
    p->scale = xs;
    p->poly_a = (float)(a * ps);
    p->poly_b = (float)(b * ps / xs);
    p->poly_c = (float)(c * ps / (xs * xs));
    p->from_gram = (float)(1.0 / xs);
    p->from_apply = (float)(1.0 / ps);
    p->from_last = (float)(1.0 / (xs * ps));
    p->growth = (float)(log2(gain) * (1.0 + 0x1p-12));
    p->eps = eps;
    p->steps = steps;
    return EVO_OK;
}

// ---- Muon plan: header, matrices, tiles of the norm, of the Gram matrix and of the iterate
struct PlanHeader {
    uint64_t magic;
    int64_t bytes, n_mats, ws_bytes, part_bytes;  // part: partial sums of `blocks` tiles, and levels
    int64_t blocks;
    // matrices in this order: by tiles, a workgroup each (8 and 4 units of rows), in LDS
    int64_t n_wg8, n_wg4, n_small, small_lds;
    int64_t tile, n_x, n_gram, n_apply;  // entries of the lists, padding included
    int64_t off_mats, off_x, off_gram, off_apply;
};
constexpr uint64_t kMagic = 0x45564f4d554f4e33ull;

int64_t round256(int64_t n) { return (n + 255) & ~int64_t(255); }

struct Size {
    int64_t r, c;
};
Size size_of(const evo_muon_tensor &t) {
    return t.rows < t.cols ? Size{t.rows, t.cols} : Size{t.cols, t.rows};
}

template <class F>
void each_gram(int64_t r, int64_t tile, F f) {
    const int64_t n = tiles_of(r, tile);
    for (int64_t i = 0; i < n; ++i)
        for (int64_t j = i; j < n; ++j) f((int32_t)i, (int32_t)j);
}
template <class F>
void each_tile(int64_t r, int64_t c, int64_t tile, F f) {
    for (int64_t i = 0; i < tiles_of(r, tile); ++i)
        for (int64_t j = 0; j < tiles_of(c, tile); ++j) f((int32_t)i, (int32_t)j);
}

// lists by XCD -> one list in which entry k belongs to XCD k % 8
struct Lists {
    std::vector<NsTile> by[8];
    int next = 0;
    void add(int xcd, const NsTile &t) {
        if (xcd == 8) {
            xcd = next;
            next = (next + 1) & 7;
        }
        by[xcd].push_back(t);
    }
    int64_t total() const {
        size_t most = 0;
        for (const auto &v : by) most = v.size() > most ? v.size() : most;
        return (int64_t)most * 8;
    }
    void write(NsTile *out) const {
        const int64_t n = total();
        for (int64_t k = 0; k < n; ++k) {
            const auto &v = by[k & 7];
            out[k] = (size_t)(k >> 3) < v.size() ? v[k >> 3] : NsTile{-1, 0, 0};
        }
    }
};

// work of a matrix, about: the products' multiply-adds and the passes over its entries
double cost(const Size &z) { return (double)z.r * z.r * (3.0 * z.c + z.r) + 100.0 * z.c * z.r; }

struct Plan {
    PlanHeader h{};
    std::vector<NsMat> mats;
    Lists x, gram, apply;
};

// false: invalid sizes
bool make_plan(const evo_muon_tensor *t, int32_t n, Plan &p) {
    if (n < 0 || (n > 0 && !t)) return false;
    PlanHeader &h = p.h;
    std::vector<int32_t> order;
    std::vector<char> form((size_t)n);  // 0 tiles, 1 and 2 a workgroup with 8 and 4 units of rows, 3 in LDS
    int64_t gram128 = 0, blocks = 0;
    double total = 0.0, alone = 0.0, largest = 0.0;
    for (int32_t i = 0; i < n; ++i) {
        if (t[i].rows < 0 || t[i].cols < 0 || t[i].rows > kMostSide || t[i].cols > kMostSide) return false;
        if (t[i].rows == 0 || t[i].cols == 0) continue;
        order.push_back(i);
        if (evo::ns_small_bytes(t[i].rows, t[i].cols) > 0) {
            form[i] = 3;
        } else if (const int rb = evo::ns_matrix_rows(t[i].rows, t[i].cols)) {
            form[i] = rb == 8 ? 1 : 2;
            alone += cost(size_of(t[i]));
            largest = cost(size_of(t[i])) > largest ? cost(size_of(t[i])) : largest;
        }
    }
    const bool by_matrix = evo::ns_by_matrix(alone, largest);
    for (const int32_t i : order) {
        if (!by_matrix && form[i] != 3) form[i] = 0;
        const Size z = size_of(t[i]);
        if (form[i] == 1) ++h.n_wg8;
        if (form[i] == 2) ++h.n_wg4;
        if (form[i] == 3) {
            ++h.n_small;
            const int64_t lds = evo::ns_small_bytes(t[i].rows, t[i].cols);
            h.small_lds = lds > h.small_lds ? lds : h.small_lds;
        }
        if (form[i] == 3) continue;
        blocks += blocks_of(z.r, z.c);
        if (blocks > kMostBlocks) return false;
        if (form[i] != 0) continue;
        gram128 += triangle(tiles_of(z.r, 128));
        total += cost(z);
    }
    // each form by falling cost: what takes longest begins first
    std::stable_sort(order.begin(), order.end(), [&](int32_t a, int32_t b) {
        return form[a] != form[b] ? form[a] < form[b] : cost(size_of(t[a])) > cost(size_of(t[b]));
    });
    h.magic = kMagic;
    h.blocks = blocks;
    h.tile = evo::ns_tile(gram128);
    h.n_mats = (int64_t)order.size();
    h.part_bytes = round256(blocks * 8 + h.n_mats * (int64_t)sizeof(int));
    h.ws_bytes = h.part_bytes;
    double load[8] = {};
    int64_t part = 0, off = 0;
    for (int32_t m = 0; m < (int32_t)order.size(); ++m) {
        const evo_muon_tensor &s = t[order[m]];
        const Size z = size_of(s);
        NsMat M{};
        M.in = s.grad;
        M.out = s.param;
        M.mom = s.momentum;
        M.swa = s.swa;
        M.rows = (int32_t)s.rows;
        M.cols = (int32_t)s.cols;
        M.scale = (float)s.update_scale;
        const int f = form[order[m]];
        M.off = off;
        if (f == 3) {
            p.mats.push_back(M);
            continue;
        }
        M.part0 = (int32_t)part;
        M.by_matrix = f != 0;
        part += blocks_of(z.r, z.c);
        off += f == 0 ? evo::ns_matrix_bytes(s.rows, s.cols) : evo::ns_matrix_wg_bytes(s.rows, s.cols);
        p.mats.push_back(M);
        if (f != 0) {
            each_tile(z.r, z.c, evo::kNsBlock, [&](int32_t i, int32_t j) { p.x.add(8, NsTile{m, i, j}); });
            continue;
        }
        const double c = cost(z);
        int xcd = 8;
        if (c * 8 <= total) {
            xcd = 0;
            for (int k = 1; k < 8; ++k)
                if (load[k] < load[xcd]) xcd = k;
            load[xcd] += c;
        }
        each_tile(z.r, z.c, evo::kNsBlock, [&](int32_t i, int32_t j) { p.x.add(xcd, NsTile{m, i, j}); });
        each_gram(z.r, h.tile, [&](int32_t i, int32_t j) { p.gram.add(xcd, NsTile{m, i, j}); });
        each_tile(z.r, z.c, h.tile, [&](int32_t i, int32_t j) { p.apply.add(xcd, NsTile{m, i, j}); });
    }
    h.ws_bytes += off;
    if (h.n_mats > 0 && h.ws_bytes < 256) h.ws_bytes = 256;  // (a size of 0 means that there is nothing to do)
    h.n_x = p.x.total();
    h.n_gram = p.gram.total();
    h.n_apply = p.apply.total();
    if (h.n_x > kMostBlocks || h.n_gram > kMostBlocks || h.n_apply > kMostBlocks) return false;
    h.off_mats = round256(sizeof(PlanHeader));
    h.off_x = h.off_mats + round256(h.n_mats * (int64_t)sizeof(NsMat));
    h.off_gram = h.off_x + round256(h.n_x * (int64_t)sizeof(NsTile));
    h.off_apply = h.off_gram + round256(h.n_gram * (int64_t)sizeof(NsTile));
    h.bytes = h.off_apply + round256(h.n_apply * (int64_t)sizeof(NsTile));
    return true;
}

int check_orth(const evo_orth_dims *d, evo::NsParams *p = nullptr) {
    if (!d || d->reserved != 0) return EVO_ERR_INVALID_ARG;
    if (d->dtype != EVO_DTYPE_F32 && d->dtype != EVO_DTYPE_BF16) return EVO_ERR_UNSUPPORTED;
    if (d->n_batch < 0 || d->rows < 0 || d->cols < 0) return EVO_ERR_INVALID_ARG;
    if (d->n_batch > (1 << 20) || d->rows > kMostSide || d->cols > kMostSide) return EVO_ERR_UNSUPPORTED;
    if ((d->n_batch + 7) * blocks_of(d->rows, d->cols) > kMostBlocks) return EVO_ERR_UNSUPPORTED;  // (see `grid`)
    return check_coefs(d->a, d->b, d->c, d->eps, d->steps, p);
}

bool orth_empty(const evo_orth_dims *d) { return d->n_batch == 0 || d->rows == 0 || d->cols == 0; }

bool orth_by_matrix(const evo_orth_dims *d) {
    return evo::ns_matrix_rows(d->rows, d->cols) > 0 && evo::ns_by_matrix((double)d->n_batch, 1.0);
}

// partial sums and levels
int64_t orth_part(const evo_orth_dims *d) {
    return round256(d->n_batch * (blocks_of(d->rows, d->cols) * 8 + (int64_t)sizeof(int)));
}

// (a stack that fits into the workgroups' LDS still asks for a little: a size of 0 means a refusal)
size_t orth_workspace(const evo_orth_dims *d) {
    if (evo::ns_small_bytes(d->rows, d->cols) > 0) return 256;
    const int64_t each = orth_by_matrix(d) ? evo::ns_matrix_wg_bytes(d->rows, d->cols)
                                           : evo::ns_matrix_bytes(d->rows, d->cols);
    return (size_t)(orth_part(d) + d->n_batch * each);
}

// no C++ exception leaves a C entry: `none` where the plan's memory cannot be had
template <class F>
int guarded(F f, int none) {
    try {
        return f();
    } catch (...) {
        return none;
    }
}

}  // namespace

extern "C" {

size_t evo_orthogonalize_workspace_size(const evo_orth_dims *d) {
    if (check_orth(d) || orth_empty(d)) return 0;
    return orth_workspace(d);
}

int evo_orthogonalize(const evo_orth_dims *d, const void *x, void *out, void *workspace, size_t workspace_bytes,
                      void *stream) {
    evo::NsParams p{};
    const int st = check_orth(d, &p);
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
    const int64_t r = d->rows < d->cols ? d->rows : d->cols, c = d->rows + d->cols - r, n = d->n_batch;
    const bool bf16 = d->dtype == EVO_DTYPE_BF16;
    evo::NsWork w{};
    w.uni.in = x;
    w.uni.out = out;
    w.uni.rows = (int32_t)d->rows;
    w.uni.cols = (int32_t)d->cols;
    w.in_stride = each;
    w.ws_stride = evo::ns_matrix_bytes(d->rows, d->cols);
    w.n_mats = (int32_t)n;
    w.part = (double *)workspace;
    w.levels = (int *)(w.part + n * blocks_of(r, c));
    w.ws = (char *)workspace + orth_part(d);
    NsLists l{};
    l.small_lds = evo::ns_small_bytes(d->rows, d->cols);
    l.tile = evo::ns_tile(n * triangle(tiles_of(r, 128)));
    // work is dealt to the XCDs: whole matrices, or tiles where there are fewer than eight
    const int64_t slots = (n + 7) / 8 * 8, g = tiles_of(r, l.tile);
    auto grid = [&](int64_t per) { return n >= 8 ? slots * per : (n * per + 7) / 8 * 8; };
    if (l.small_lds > 0) {
        l.n_small = n;
    } else {
        l.n_x = grid(blocks_of(r, c));
        if (orth_by_matrix(d)) {
            w.ws_stride = evo::ns_matrix_wg_bytes(d->rows, d->cols);
            w.uni.by_matrix = 1;
            (evo::ns_matrix_rows(d->rows, d->cols) == 8 ? l.n_wg8 : l.n_wg4) = n;
        } else {
            l.n_gram = grid(triangle(g));
            l.n_apply = grid(g * tiles_of(c, l.tile));
        }
    }
    return evo::launch_ns(w, l, p, false, bf16, (hipStream_t)stream) == hipSuccess ? EVO_OK : EVO_ERR_HIP;
}

int64_t evo_muon_plan_bytes(const evo_muon_tensor *tensors, int32_t n_tensors) {
    int64_t bytes = -1;
    guarded(
        [&] {
            Plan p;
            if (make_plan(tensors, n_tensors, p)) bytes = p.h.bytes;
            return 0;
        },
        0);
    return bytes;
}

int evo_muon_build_plan(const evo_muon_tensor *tensors, int32_t n_tensors, void *plan, size_t plan_bytes) {
    return guarded(
        [&]() -> int {
            Plan p;
            if (!make_plan(tensors, n_tensors, p) || !plan) return EVO_ERR_INVALID_ARG;
            if (!aligned(plan, 8)) return EVO_ERR_ALIGNMENT;
            const PlanHeader &h = p.h;
            if (plan_bytes < (size_t)h.bytes) return EVO_ERR_WORKSPACE;
            for (int32_t i = 0; i < n_tensors; ++i) {
                const evo_muon_tensor &t = tensors[i];
                if (t.rows == 0 || t.cols == 0) continue;
                if (!t.param || !t.grad || !t.momentum || !isfinite(t.update_scale)) return EVO_ERR_INVALID_ARG;
                if (!aligned(t.param, 4) || !aligned(t.grad, 4) || !aligned(t.momentum, 4) || !aligned(t.swa, 4))
                    return EVO_ERR_ALIGNMENT;
            }
            char *q = (char *)plan;
            memset(q, 0, (size_t)h.bytes);
            memcpy(q, &h, sizeof h);
            if (!p.mats.empty()) memcpy(q + h.off_mats, p.mats.data(), p.mats.size() * sizeof(NsMat));
            p.x.write((NsTile *)(q + h.off_x));
            p.gram.write((NsTile *)(q + h.off_gram));
            p.apply.write((NsTile *)(q + h.off_apply));
            return EVO_OK;
        },
        EVO_ERR_INVALID_ARG);
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
    evo::NsParams p{};
    const int st = check_coefs(hp->a, hp->b, hp->c, hp->eps, hp->steps, &p);
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
    w.levels = (int *)(w.part + h.blocks);
    w.ws = (char *)workspace + h.part_bytes;
    p.mu = (float)hp->momentum;
    p.om_mu = (float)(1.0 - hp->momentum);
    p.u_g = hp->nesterov ? p.om_mu : 0.0f;
    p.u_m = hp->nesterov ? p.mu : 1.0f;
    p.decay = (float)(1.0 - hp->lr * hp->weight_decay);
    p.lr = (float)hp->lr;
    p.sd = (float)hp->swa_decay;
    p.om_sd = (float)(1.0 - hp->swa_decay);
    p.grad_scale = grad_scale;
    NsLists l{};
    l.n_small = h.n_small;
    l.first_small = h.n_mats - h.n_small;
    l.small_lds = h.small_lds;
    l.n_wg4 = h.n_wg4;
    l.first_wg4 = l.first_small - h.n_wg4;
    l.n_wg8 = h.n_wg8;
    l.first_wg8 = l.first_wg4 - h.n_wg8;
    l.tile = (int)h.tile;
    l.n_x = h.n_x;
    l.n_gram = h.n_gram;
    l.n_apply = h.n_apply;
    l.x = (const NsTile *)(dev + h.off_x);
    l.gram = (const NsTile *)(dev + h.off_gram);
    l.apply = (const NsTile *)(dev + h.off_apply);
    return evo::launch_ns(w, l, p, true, false, (hipStream_t)stream) == hipSuccess ? EVO_OK : EVO_ERR_HIP;
}

}  // extern "C"

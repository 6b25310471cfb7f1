// evo_cross_api.cpp -- the C ABI declared in include/evo_cross_attn.h:
// validation (before any HIP call), plan and dispatch.
#include "evo_cross_attn.h"

#include <hip/hip_runtime.h>
#include <math.h>

#include "evo_cross.h"
#include "evo_views.h"

namespace {

constexpr int64_t kMost = int64_t(1) << 40, kMostLen = int64_t(1) << 30;
constexpr int64_t kGrid = (int64_t(1) << 24) - 1;  // workgroups of 256 threads: a launch counts its threads in 32 bits

bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// a (row, token) grid of blocks that does not overlap itself
bool apart(int64_t n, int64_t len, int64_t block, int64_t row, int64_t tok) {
    if (n == 0 || len == 0) return true;
    if ((len > 1 && tok < block) || (n > 1 && row < block)) return false;
    if (n == 1 || len == 1) return true;
    return row >= (len - 1) * tok + block || tok >= (n - 1) * row + block;
}

int check_stride(int64_t v, int64_t count, int64_t es) {
    if (v < 0) return EVO_ERR_INVALID_ARG;
    if (v > kMost || (v > 0 && count > (kMost << 10) / v)) return EVO_ERR_UNSUPPORTED;
    return v * es % 16 != 0 ? EVO_ERR_ALIGNMENT : EVO_OK;
}

int check(const evo_cross_dims *d, bool has_bias, evo::CrArgs *a) {
    if (!d) return EVO_ERR_INVALID_ARG;
    if (d->dtype != EVO_DTYPE_F32 && d->dtype != EVO_DTYPE_BF16) return EVO_ERR_UNSUPPORTED;
    if (d->n_heads < 1 || d->n_kv_heads < 1 || d->n_heads % d->n_kv_heads != 0 || d->head_dim < 1 || d->n_rows < 0 ||
        d->len_q < 0 || d->len_k < 0)
        return EVO_ERR_INVALID_ARG;
    if (d->head_dim % 8 != 0 || d->head_dim > 128 || d->n_heads > 65535) return EVO_ERR_UNSUPPORTED;
    const int64_t N = d->n_rows, G = d->n_heads / d->n_kv_heads, es = d->dtype == EVO_DTYPE_BF16 ? 2 : 4;
    if (d->len_q > kMostLen / G || d->len_k > kMostLen || N > kMost) return EVO_ERR_UNSUPPORTED;
    const int64_t M = d->len_q * G, qe = d->len_q * d->n_heads * d->head_dim, ke = d->len_k * d->n_kv_heads * d->head_dim;
    if (qe > kMost || ke > kMost || (qe > 0 && N > kMost / qe) || (ke > 0 && N > kMost / ke)) return EVO_ERR_UNSUPPORTED;
    if (has_bias) {
        if (d->rows_per_bias < 1 || N % d->rows_per_bias != 0) return EVO_ERR_INVALID_ARG;
        const int64_t plane = d->n_heads * d->len_q;  // < 2^47
        const int64_t B = N / d->rows_per_bias;
        if (d->rows_per_bias > 0x7fffffff) return EVO_ERR_UNSUPPORTED;
        if (plane > kMost || (plane > 0 && d->len_k > kMost / plane) ||
            (plane > 0 && d->len_k > 0 && B > kMost / (plane * d->len_k)))
            return EVO_ERR_UNSUPPORTED;
        const int64_t wgs = up(d->len_q, 64) * up(d->len_k, 64);  // <= 2^50
        if (wgs > 0 && B * d->n_heads > kGrid / wgs) return EVO_ERR_UNSUPPORTED;
    }
    const int64_t st[6] = {d->q_stride_row, d->q_stride_tok, d->k_stride_row, d->k_stride_tok, d->o_stride_row, d->o_stride_tok};
    for (int i = 0; i < 6; ++i) {
        const int e = check_stride(st[i], i % 2 == 0 ? N : (i == 3 ? d->len_k : d->len_q), es);
        if (e) return e;
    }
    // tiles of one unit in any kernel, before splits: those are made of up to 4096 workgroups, and make at most 4096 more
    // of them (split), far below the limit
    int64_t tiles = up(M, 128) > up(d->len_k, 128) ? up(M, 128) : up(d->len_k, 128);
    if (tiles < 1) tiles = 1;
    if (N > kGrid / tiles / d->n_kv_heads) return EVO_ERR_UNSUPPORTED;
    *a = evo::CrArgs{};
    a->N = N;
    a->rpb = has_bias ? d->rows_per_bias : (N > 0 ? N : 1);
    a->Lq = (int)d->len_q;
    a->Lk = (int)d->len_k;
    a->M = (int)M;
    a->H = d->n_heads;
    a->Hk = d->n_kv_heads;
    a->G = (int)G;
    a->D = d->head_dim;
    a->q_row = st[0], a->q_tok = st[1], a->k_row = st[2], a->k_tok = st[3], a->o_row = st[4], a->o_tok = st[5];
    a->bf16 = d->dtype == EVO_DTYPE_BF16;
    // x / G = x * ceil(2^(31 + s) / G) >> (31 + s), 2^s >= G, exact for x < 2^31 (the excess over x / G stays below 1 / G)
    int s = 0;
    while ((int64_t(1) << s) < G) ++s;
    a->g_mul = (uint32_t)(((uint64_t(1) << (31 + s)) + G - 1) / G);
    a->g_shift = 31 + s;
    a->scale = 1.0f / sqrtf((float)d->head_dim);
    return EVO_OK;
}

bool apart_o(const evo::CrArgs &a) { return apart(a.N, a.Lq, (int64_t)a.H * a.D, a.o_row, a.o_tok); }

// tensors that are not there (or empty) have no block
evo::View view(const evo::CrArgs &a, const void *p, int len, int heads, int64_t row, int64_t tok) {
    const int64_t es = a.bf16 ? 2 : 4;
    return evo::View{(uintptr_t)p, row * es, tok * es, a.N, len, p && len > 0 ? (int64_t)heads * a.D * es : 0};
}
evo::View flat(const void *p, int64_t bytes) { return evo::View{(uintptr_t)p, 0, 0, 1, 1, p ? bytes : 0}; }
bool apart(const evo::View &x, const evo::View &y) { return x.block == 0 || y.block == 0 || evo::views_apart(x, y); }
// outputs first .. n_outs - 1 from every input and from those before them
bool all_apart(const evo::View *outs, int first, int n_outs, const evo::View *ins, int n_ins) {
    for (int i = first; i < n_outs; ++i) {
        for (int j = 0; j < n_ins; ++j)
            if (!apart(outs[i], ins[j])) return false;
        for (int j = 0; j < i; ++j)
            if (!apart(outs[i], outs[j])) return false;
    }
    return true;
}
int64_t bias_bytes(const evo::CrArgs &a, const void *bias) {
    return bias ? a.N / a.rpb * a.H * a.Lq * (int64_t)a.Lk * (a.bf16 ? 2 : 4) : 0;
}

}  // namespace

namespace evo {

// How many workgroups share one tile's walk of `steps`: the count of the lowest
// estimated time, in us.  The workgroups of the fullest CU count (several on a CU have `rate`
// times one's), each 1.5 to begin with and `one` a step; n parts take a launch (5), 0.15 each to be
// read in turn, and their bytes (of one part) at 2 TB/s, the forward's at 5.5 where others are
// still at work while they are written.  Fitted to calls of 32, 64 and 128 channels; e.g.
// forward, 264 tiles of 65 steps at 64 channels: 82 us unsplit, 72, 69, 66, 65, 67 and 71 with 2, 3, 4, 5, 6
// and 8 (estimated 85, 76, 71, 71, 70, 72, 81).
static int split(int64_t tiles, int64_t steps, double one, double bytes, double rate, bool forward) {
    if (tiles <= 0 || steps <= 1) return 1;
    int best = 1;
    double least = 0.0;
    for (int64_t n = 1; n <= steps && n <= 64; ++n) {
        const int64_t per = up(steps, n), load = up(tiles * n, 256);
        if (up(steps, per) != n) continue;
        const double join = 5.0 + n * (0.15 + bytes / (forward && load > 2 ? 5.5e6 : 2e6));
        const double cost = load * (1.5 + per * one) / (load > 1 ? rate : 1.0) + (n > 1 ? join : 0.0);
        if (n == 1 || cost < least) best = (int)n, least = cost;
        if (load > 16) break;  // the GPU is full
    }
    return best;
}

CrPlan cross_plan(const CrArgs &a, bool has_gate, bool has_bias) {
    CrPlan p{};
    const int64_t units = a.N * a.Hk;
    const int few_rows = a.bf16 ? 32 : 64;
    const int64_t key_steps = up(a.Lk, a.bf16 ? 64 : 32);
    const double rows_bytes = 4.0 * units * a.M * a.D, keys_bytes = 8.0 * units * a.Lk * a.D;
    // us a step of the forward: 128 queries by 64 keys, fp32 by 32 (two products at the rate of its matrix
    // instructions); the lanes' rows of a bias take half a us more
    const int d = a.D <= 32 ? 32 : a.D <= 64 ? 64 : 128;
    const double rate = a.bf16 ? 1.3 : 1.0;  // one workgroup keeps fp32's matrix instructions busy
    const double bias_step = has_bias && a.bf16 ? 0.5 : 0.0;
    const double one = (a.bf16 ? 0.33 + 0.0078 * d : 0.1 + 0.031 * d) + bias_step;
    p.few = a.M <= few_rows;
    const int64_t tiles = up(a.M, p.few ? few_rows : 128);
    if (p.few) {
        // reading K and V is all there is to do: two workgroups a CU, of four steps at least.  16 rows of 4 key
        // heads to 4097 keys of 128 channels: 64 us unsplit, 41, 25, 24 and 28 with 2, 4, 8 and 12
        int64_t n = units * tiles > 0 ? 512 / (units * tiles) : 1;
        if (n > key_steps / 4) n = key_steps / 4;
        p.fwd_splits = n < 2 ? 1 : (int)up(key_steps, up(key_steps, n));
    } else {
        p.fwd_splits = split(units * tiles, key_steps, one, rows_bytes, rate, true);
    }
    // few keys: a workgroup (or, for up to 32 queries, a wave) walks over rows of the batch, where there are
    // enough.  A workgroup (a workgroup a row beside it): 256 queries to 77 keys, 8 heads of 32, gate, bias and mask, 16,
    // 32, 64, 128 rows 10.4 us (9.2), 10.9 (12.4), 15.4 (20.0), 24.7 (34.7), without them 7.5 (6.0), 7.9 (7.3), 9.9 (10.6),
    // 16.9 (18.6): from 1024 units and tiles on (64 rows here) no form loses.  A wave: one query to 4 keys, 4 heads of
    // 16, 256, 512, 1024, 2048, 8192 rows 5.7 (5.1), 5.8 (6.5), 6.5 (10.1), 8.9 (17.1), 23.5 (54.2); 8 queries to 60 keys,
    // 4 heads of 64 with a bias, 256, 512, 1024, 2048, 4096 rows 9.6 (6.7), 10.8 (13.5), 22.9 (23.6), 42.4 (40.7), 78.4 (83).
    // More than 32 channels have no form of four waves: with 3 blocks of keys and a bias 32 channels take 216 registers.
    if (a.Lk > 0 && a.Lk <= 128) {
        p.brief_one = a.M <= 32 && units >= 4096 && 16 * up(a.Lk, 32) * 32 * d * (a.bf16 ? 2 : 4) <= 128 * 1024;
        p.brief = p.brief_one || (a.bf16 && a.D <= 32 && a.M > 32 && units * tiles >= 1024);
    }
    if (p.brief) {
        const int64_t base = a.N / a.rpb * a.Hk * (p.brief_one ? 1 : tiles), most = up(a.rpb, p.brief_one ? 8 : 2);
        int64_t n = (p.brief_one ? 1024 : 512) / base;
        n = n < 1 ? 1 : n > most ? most : n;
        p.brief_chunks = (int)up(a.rpb, up(a.rpb, n));
        p.fwd_splits = 1;
    }
    const auto pad = [](size_t x) { return (x + 255) / 256 * 256; };
    if (p.fwd_splits > 1) {
        p.fwd_part = 0;
        p.fwd_ml = pad((size_t)p.fwd_splits * units * a.M * a.D * 4);
        p.fwd_lo = p.fwd_ml + pad((size_t)p.fwd_splits * units * a.M * 8);
        p.fwd_total = p.fwd_lo + pad((size_t)p.fwd_splits * units * a.M * 4);
    }
    // steps of the backward's passes; the keys' four products (128 keys by 64 queries, or 32), the rows' three
    // (128 queries by 64 keys, or 32), a row of the batch for 64 x 64 entries of the bias
    const double step = a.bf16 ? 0.35 + 0.0088 * d : 0.1 + 0.031 * d;
    const bool wide_steps = a.bf16 && a.D <= 64 && !has_bias;
    p.kv_splits = split(units * up(a.Lk, 128), up(a.M, a.bf16 && a.D <= 64 ? 64 : 32), (a.bf16 ? 1.3 : 2.1) * step, keys_bytes, rate, false);
    p.q_splits = split(units * up(a.M, 128), up(a.Lk, wide_steps ? 64 : 32),
                       (a.bf16 ? wide_steps ? 1.2 : 0.6 : 1.6) * step + bias_step, rows_bytes, rate, false);
    p.bias_chunks = 1;
    if (has_bias) {
        const int64_t bias_tiles = a.N / a.rpb * a.H * up(a.Lq, 64) * up(a.Lk, 64);
        p.bias_chunks = split(bias_tiles, a.rpb, 1.2 * step, 4.0 * (a.N / a.rpb) * a.H * a.Lq * (double)a.Lk, rate, false);
    }
    p.bwd_da = pad((size_t)units * a.M * 16);
    p.bwd_part = p.bwd_da + (has_gate || has_bias ? pad((size_t)units * a.M * a.D * (a.bf16 ? 2 : 4)) : 0);
    size_t part = 0;
    const auto more = [&](int splits, size_t one) {
        if (splits > 1 && part < splits * one) part = splits * one;
    };
    more(p.kv_splits, (size_t)units * a.Lk * a.D * 8);
    more(p.q_splits, (size_t)units * a.M * a.D * 4);
    if (has_bias) more(p.bias_chunks, (size_t)(a.N / a.rpb) * a.H * a.Lq * (size_t)a.Lk * 4);
    p.bwd_total = p.bwd_part + pad(part);
    return p;
}

}  // namespace evo

extern "C" {

size_t evo_cross_fwd_workspace_size(const evo_cross_dims *d) {
    evo::CrArgs a;
    if (check(d, false, &a) || a.N == 0 || a.Lq == 0) return 0;
    // with a bias there may be more splits
    const size_t plain = evo::cross_plan(a, false, false).fwd_total, bias = evo::cross_plan(a, false, true).fwd_total;
    return plain > bias ? plain : bias;
}

int evo_cross_fwd(const evo_cross_dims *d, const void *q, const void *k, const void *v, const void *gate, const void *bias,
                  const uint8_t *mask, void *out, float *lse, void *ws, size_t ws_bytes, void *stream) {
    evo::CrArgs a;
    const int st = check(d, bias != nullptr, &a);
    if (st) return st;
    if (!apart_o(a)) return EVO_ERR_INVALID_ARG;
    if (a.N == 0 || a.Lq == 0) return EVO_OK;
    if (!q || !out || !lse || (a.Lk > 0 && (!k || !v))) return EVO_ERR_INVALID_ARG;
    const size_t es = a.bf16 ? 2 : 4;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(gate, 16) || !aligned(out, 16) ||
        !aligned(bias, es) || !aligned(lse, 4))
        return EVO_ERR_ALIGNMENT;
    const evo::CrPlan p = evo::cross_plan(a, gate != nullptr, bias != nullptr);
    const evo::View outs[3] = {view(a, out, a.Lq, a.H, a.o_row, a.o_tok), flat(lse, a.N * a.H * a.Lq * 4), flat(ws, (int64_t)p.fwd_total)};
    const evo::View ins[6] = {view(a, q, a.Lq, a.H, a.q_row, a.q_tok), view(a, gate, a.Lq, a.H, a.q_row, a.q_tok),
                              view(a, k, a.Lk, a.Hk, a.k_row, a.k_tok), view(a, v, a.Lk, a.Hk, a.k_row, a.k_tok),
                              flat(bias, bias_bytes(a, bias)), flat(mask, a.N * a.Lk)};
    if (!all_apart(outs, 0, 2, ins, 6)) return EVO_ERR_INVALID_ARG;
    if (p.fwd_total > 0 && (!ws || ws_bytes < p.fwd_total)) return EVO_ERR_WORKSPACE;
    if (p.fwd_total > 0 && !aligned(ws, 256)) return EVO_ERR_ALIGNMENT;
    if (!all_apart(outs, 2, 3, ins, 6)) return EVO_ERR_INVALID_ARG;
    a.q = q, a.k = k, a.v = v, a.gate = gate, a.bias = bias, a.mask = mask, a.out = out, a.lse = lse;
    return evo::launch_cross_fwd(a, p, ws, (hipStream_t)stream) == hipSuccess ? EVO_OK : EVO_ERR_HIP;
}

size_t evo_cross_bwd_workspace_size(const evo_cross_dims *d, int has_gate, int has_bias) {
    evo::CrArgs a;
    if (check(d, has_bias != 0, &a) || a.N == 0) return 0;
    return evo::cross_plan(a, has_gate != 0, has_bias != 0).bwd_total;
}

int evo_cross_bwd(const evo_cross_dims *d, const void *q, const void *k, const void *v, const void *gate, const void *bias,
                  const uint8_t *mask, const void *out, const float *lse, const void *dout, void *dq, void *dk, void *dv,
                  void *dgate, void *dbias, void *ws, size_t ws_bytes, void *stream) {
    evo::CrArgs a;
    const int st = check(d, bias != nullptr, &a);
    if (st) return st;
    if (!apart(a.N, a.Lq, (int64_t)a.H * a.D, a.q_row, a.q_tok) || !apart(a.N, a.Lk, (int64_t)a.Hk * a.D, a.k_row, a.k_tok))
        return EVO_ERR_INVALID_ARG;
    if (a.N == 0 || (a.Lq == 0 && a.Lk == 0)) return EVO_OK;
    if ((gate != nullptr) != (dgate != nullptr) || (bias != nullptr) != (dbias != nullptr)) return EVO_ERR_INVALID_ARG;
    if (a.Lq > 0 && (!q || !out || !lse || !dout || !dq)) return EVO_ERR_INVALID_ARG;
    if (a.Lk > 0 && (!k || !v || !dk || !dv)) return EVO_ERR_INVALID_ARG;
    const size_t es = a.bf16 ? 2 : 4;
    const void *wide[] = {q, k, v, gate, out, dout, dq, dk, dv, dgate};
    for (const void *x : wide)
        if (!aligned(x, 16)) return EVO_ERR_ALIGNMENT;
    if (!aligned(bias, es) || !aligned(dbias, es) || !aligned(lse, 4)) return EVO_ERR_ALIGNMENT;
    const auto qr = [&](const void *x) { return view(a, x, a.Lq, a.H, a.q_row, a.q_tok); };
    const auto kr = [&](const void *x) { return view(a, x, a.Lk, a.Hk, a.k_row, a.k_tok); };
    const auto orr = [&](const void *x) { return view(a, x, a.Lq, a.H, a.o_row, a.o_tok); };
    const int64_t nb = bias_bytes(a, bias);
    const evo::CrPlan p = evo::cross_plan(a, gate != nullptr, bias != nullptr);
    const evo::View outs[6] = {qr(dq), qr(dgate), kr(dk), kr(dv), flat(dbias, nb), flat(ws, (int64_t)p.bwd_total)};
    const evo::View ins[9] = {qr(q), qr(gate), kr(k), kr(v), orr(out), orr(dout), flat(bias, nb), flat(lse, a.N * a.H * a.Lq * 4),
                              flat(mask, a.N * a.Lk)};
    if (!all_apart(outs, 0, 5, ins, 9)) return EVO_ERR_INVALID_ARG;
    if (p.bwd_total > 0 && (!ws || ws_bytes < p.bwd_total)) return EVO_ERR_WORKSPACE;
    if (p.bwd_total > 0 && !aligned(ws, 256)) return EVO_ERR_ALIGNMENT;
    if (!all_apart(outs, 5, 6, ins, 9)) return EVO_ERR_INVALID_ARG;
    a.q = q, a.k = k, a.v = v, a.gate = gate, a.bias = bias, a.mask = mask, a.out = (void *)out, a.lse = (float *)lse;
    a.dout = dout, a.dq = dq, a.dk = dk, a.dv = dv, a.dgate = dgate, a.dbias = dbias;
    return evo::launch_cross_bwd(a, p, ws, (hipStream_t)stream) == hipSuccess ? EVO_OK : EVO_ERR_HIP;
}

}  // extern "C"

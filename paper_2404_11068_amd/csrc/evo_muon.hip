// evo_muon.hip -- Newton-Schulz orthogonalisation and the Muon step, gfx950.
#include "evo_frag.h"
#include "evo_ns.h"

namespace evo {
namespace {

constexpr int kT = kNsTile;

struct View {  // a matrix of this call and its buffers
    NsMat m;
    int r, c;
    bool tr;            // the iterate is the transposed matrix
    float *x0, *x1, *A, *P;
};

__host__ __device__ int64_t up(int64_t n) { return (n + 63) & ~int64_t(63); }

__device__ View view_of(const NsWork &w, int k) {
    View v;
    if (w.mats) {
        v.m = w.mats[k];
    } else {
        v.m = w.uni;
        v.m.in = (const char *)v.m.in + k * w.in_stride;
        v.m.out = (char *)v.m.out + k * w.in_stride;
        v.m.off = k * w.ws_stride;
    }
    v.tr = v.m.rows > v.m.cols;
    v.r = v.tr ? v.m.cols : v.m.rows;
    v.c = v.tr ? v.m.rows : v.m.cols;
    v.x0 = (float *)(w.ws + v.m.off);
    v.x1 = v.x0 + up((int64_t)v.r * v.c);
    v.A = v.x1 + up((int64_t)v.r * v.c);
    v.P = v.A + up((int64_t)v.r * v.r);
    return v;
}

__device__ NsTile tile_of(const NsWork &w, int k) {
    if (w.tiles) return w.tiles[k];
    const int per = w.nti * w.ntj, e = k % per;
    return NsTile{k / per, e / w.ntj, e % w.ntj};
}

__device__ int64_t place(const View &v, int i, int j) {  // of iterate element (i, j) in the matrix
    return v.tr ? (int64_t)j * v.m.cols + i : (int64_t)i * v.m.cols + j;
}

template <bool MUON, bool BF16>
__device__ float value_in(const View &v, const NsParams &p, float gs, int64_t at) {
    if constexpr (MUON) {
        const float g = ((const float *)v.m.in)[at] * gs;
        return fmaf(p.u_m, v.m.mom[at], p.u_g * g);
    } else if constexpr (BF16) {
        return bf2f(((const uint16_t *)v.m.in)[at]);
    } else {
        return ((const float *)v.m.in)[at];
    }
}

// momentum, and the sum of squares of each tile
template <bool MUON, bool BF16>
__global__ __launch_bounds__(256) void ns_norm_kernel(NsWork w, NsParams p) {
    __shared__ double red[256];
    const NsTile t = tile_of(w, blockIdx.x);
    const View v = view_of(w, t.mat);
    const float gs = MUON && p.grad_scale ? *p.grad_scale : 1.0f;
    double s = 0.0;
    for (int e = threadIdx.x; e < kT * kT; e += 256) {
        const int hi = e / kT, lo = e % kT;
        const int i = t.ti * kT + (v.tr ? lo : hi), j = t.tj * kT + (v.tr ? hi : lo);
        if (i >= v.r || j >= v.c) continue;
        const int64_t at = place(v, i, j);
        if constexpr (MUON) v.m.mom[at] = fmaf(p.mu, v.m.mom[at], p.om_mu * (((const float *)v.m.in)[at] * gs));
        const double u = value_in<MUON, BF16>(v, p, gs, at);
        s += u * u;
    }
    red[threadIdx.x] = s;
    __syncthreads();
    for (int m = 128; m >= 1; m >>= 1) {
        if (threadIdx.x < m) red[threadIdx.x] += red[threadIdx.x + m];
        __syncthreads();
    }
    if (threadIdx.x == 0) w.part[blockIdx.x] = red[0];
}

template <bool MUON, bool BF16>
__global__ __launch_bounds__(256) void ns_scale_kernel(NsWork w, NsParams p) {
    __shared__ double inv;
    const NsTile t = tile_of(w, blockIdx.x);
    const View v = view_of(w, t.mat);
    const float gs = MUON && p.grad_scale ? *p.grad_scale : 1.0f;
    const int n = ((v.r + kT - 1) / kT) * ((v.c + kT - 1) / kT);
    if (threadIdx.x == 0) {
        const double *part = w.part + (w.mats ? v.m.part0 : t.mat * n);
        double s = 0.0;
        for (int k = 0; k < n; ++k) s += part[k];
        s = sqrt(s);
        inv = 1.0 / (s < p.eps ? p.eps : s);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < kT * kT; e += 256) {
        const int hi = e / kT, lo = e % kT;
        const int i = t.ti * kT + (v.tr ? lo : hi), j = t.tj * kT + (v.tr ? hi : lo);
        if (i >= v.r || j >= v.c) continue;
        v.x0[(int64_t)i * v.c + j] = (float)(value_in<MUON, BF16>(v, p, gs, place(v, i, j)) * inv);
    }
}

// acc += the 64 x 64 tile of L R, L[i][k] and R[k][j] by functions; 4 x 4 per thread
template <class FL, class FR>
__device__ void tile_product(float (&acc)[4][4], int K, FL L, FR R) {
    __shared__ float ls[16][kT + 4], rs[16][kT + 4];
    const int tid = threadIdx.x, ty = tid / 16, tx = tid % 16;
    for (int k0 = 0; k0 < K; k0 += 16) {
        for (int e = tid; e < 16 * kT; e += 256) {
            ls[e % 16][e / 16] = L(e / 16, k0 + e % 16);
            rs[e / kT][e % kT] = R(k0 + e / kT, e % kT);
        }
        __syncthreads();
        for (int k = 0; k < 16; ++k)
            for (int x = 0; x < 4; ++x)
                for (int y = 0; y < 4; ++y) acc[x][y] = fmaf(ls[k][ty * 4 + x], rs[k][tx * 4 + y], acc[x][y]);
        __syncthreads();
    }
}

// POLY: P = a I + b A + c A A; otherwise A = X X^T
template <bool POLY>
__global__ __launch_bounds__(256) void ns_gram_kernel(NsWork w, NsParams p, bool odd) {
    const NsTile t = tile_of(w, blockIdx.x);
    const View v = view_of(w, t.mat);
    const float *x = POLY ? v.A : odd ? v.x1 : v.x0;
    const int K = POLY ? v.r : v.c, i0 = t.ti * kT, j0 = t.tj * kT;
    auto at = [&](int row, int k) { return row < v.r && k < K ? x[(int64_t)row * K + k] : 0.0f; };
    float acc[4][4] = {};
    tile_product(acc, K, [&](int i, int k) { return at(i0 + i, k); }, [&](int k, int j) { return at(j0 + j, k); });
    const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
    for (int a = 0; a < 4; ++a)
        for (int b = 0; b < 4; ++b) {
            const int i = i0 + ty * 4 + a, j = j0 + tx * 4 + b;
            if (i >= v.r || j >= v.r) continue;
            const int64_t e = (int64_t)i * v.r + j;
            if constexpr (POLY) v.P[e] = p.b * v.A[e] + p.c * acc[a][b] + (i == j ? p.a : 0.0f);
            else v.A[e] = acc[a][b];
        }
}

// X = P X, or (LAST) the result
template <bool LAST, bool MUON, bool BF16>
__global__ __launch_bounds__(256) void ns_apply_kernel(NsWork w, NsParams p, bool odd) {
    const NsTile t = tile_of(w, blockIdx.x);
    const View v = view_of(w, t.mat);
    const float *x = odd ? v.x1 : v.x0;
    float *y = odd ? v.x0 : v.x1;
    const int i0 = t.ti * kT, j0 = t.tj * kT;
    float acc[4][4] = {};
    tile_product(
        acc, v.r, [&](int i, int k) { return i0 + i < v.r && k < v.r ? v.P[(int64_t)(i0 + i) * v.r + k] : 0.0f; },
        [&](int k, int j) { return k < v.r && j0 + j < v.c ? x[(int64_t)k * v.c + j0 + j] : 0.0f; });
    const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
    for (int a = 0; a < 4; ++a)
        for (int b = 0; b < 4; ++b) {
            const int i = i0 + ty * 4 + a, j = j0 + tx * 4 + b;
            if (i >= v.r || j >= v.c) continue;
            if constexpr (!LAST) {
                y[(int64_t)i * v.c + j] = acc[a][b];
            } else {
                const int64_t e = place(v, i, j);
                if constexpr (MUON) {
                    float *prm = (float *)v.m.out;
                    const float q = fmaf(-p.lr * v.m.scale, acc[a][b], p.decay * prm[e]);
                    prm[e] = q;
                    if (v.m.swa) v.m.swa[e] = fmaf(p.sd, v.m.swa[e], p.om_sd * q);
                } else if constexpr (BF16) {
                    ((uint16_t *)v.m.out)[e] = f2bf(acc[a][b]);
                } else {
                    ((float *)v.m.out)[e] = acc[a][b];
                }
            }
        }
}

template <bool MUON, bool BF16>
hipError_t launch_all(NsWork w, const NsParams &p, int64_t n_x, const NsTile *tx, int64_t n_a, const NsTile *ta,
                      hipStream_t s) {
    NsWork wx = w, wa = w;
    const int r = w.uni.rows < w.uni.cols ? w.uni.rows : w.uni.cols, c = w.uni.rows + w.uni.cols - r;
    wx.tiles = tx;
    wx.nti = (r + kT - 1) / kT;
    wx.ntj = (c + kT - 1) / kT;
    wa.tiles = ta;
    wa.nti = wa.ntj = wx.nti;
    const dim3 gx((unsigned)n_x), ga((unsigned)n_a), b(256);
    hipLaunchKernelGGL((ns_norm_kernel<MUON, BF16>), gx, b, 0, s, wx, p);
    hipLaunchKernelGGL((ns_scale_kernel<MUON, BF16>), gx, b, 0, s, wx, p);
    for (int k = 0; k < p.steps; ++k) {
        hipLaunchKernelGGL(ns_gram_kernel<false>, ga, b, 0, s, wa, p, (k & 1) != 0);
        hipLaunchKernelGGL(ns_gram_kernel<true>, ga, b, 0, s, wa, p, (k & 1) != 0);
        if (k + 1 < p.steps) hipLaunchKernelGGL((ns_apply_kernel<false, MUON, BF16>), gx, b, 0, s, wx, p, (k & 1) != 0);
        else hipLaunchKernelGGL((ns_apply_kernel<true, MUON, BF16>), gx, b, 0, s, wx, p, (k & 1) != 0);
    }
    return hipGetLastError();
}

}  // namespace

int64_t ns_matrix_bytes(int64_t rows, int64_t cols) {
    const int64_t r = rows < cols ? rows : cols, c = rows + cols - r;
    return 4 * (2 * up(r * c) + 2 * up(r * r));
}

hipError_t launch_ns(NsWork w, const NsParams &p, bool muon, bool bf16, int64_t n_x, const NsTile *tx, int64_t n_a,
                     const NsTile *ta, hipStream_t s) {
    if (muon) return launch_all<true, false>(w, p, n_x, tx, n_a, ta, s);
    return bf16 ? launch_all<false, true>(w, p, n_x, tx, n_a, ta, s) : launch_all<false, false>(w, p, n_x, tx, n_a, ta, s);
}

}  // namespace evo

// evo_muon.hip -- Newton-Schulz orthogonalisation and the Muon step, gfx950.
//
//   X = x / max(|x|_F, eps);  steps times:  A = X X^T,  P = a I + b A + c A A,  X = P X
//
// Precision.  A direction that X hardly has grows by up to a^steps = 485, and so do
// the roundings of the iterate.  Every iterate is therefore a pair of fp16
// (value = hi + lo, 22 bits), and each product is hi hi + hi lo + lo hi
// on the fp16 matrix instructions with fp32 accumulation: the error of fp32
// arithmetic (1e-6 .. 1e-5 of the result over five steps, low-rank inputs too; rows far
// below the others have an absolute error, see the range below) at a third of the fp16 rate, which
// is five times the fp32 matrix rate.
// bf16 matrices go through the same steps and are rounded once, at the end: with hi
// alone in the last two steps their error would grow by a tenth (1.84e-3 instead of
// 1.66e-3 of a result), in all steps to 2.4 times their rounding for low-rank inputs.
// fp16's range: X and A are stored times one power of two and P times another, the largest at which no
// entry passes 65504 for the coefficients' singular values (2^15 and 2^14 for the usual ones), so that
// a pair holds 22 bits of what is not below 2^-14 of that, and less ends at 2^-25: 2^-40 of X and A, 2^-39 of P.
// A matrix whose norm is below eps, so that X is small as a whole, has another power of two on top, less of it
// each step as X grows (Scales).
//
// Layout.  Iterates lie in the workspace as units of 32 x 32 entries, 2 KB per
// plane, zero beyond the matrix.  Inside a unit 16-byte chunks (8 entries of a
// row) are ordered so that both ways of reading it touch every LDS bank once:
// an operand fragment by rows (ds_read_b128, lane = row) and one by columns
// (ds_read_b64_tr_b16, four rows of four chunks at a time).  A unit goes from
// memory to LDS as it is, so one copy of X serves X X^T (rows) and P X (columns).
#include "evo_frag.h"
#include "evo_ns.h"

namespace evo {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));

// The scales of X and A before step k, and what a step's products bring to the next ones.  A matrix of norm below
// eps has a level, log2(eps / norm) rounded down: no singular value of its X is above 2^-level before the first step,
// nor above 2^(growth k - level) before step k, so X has room for that much more
constexpr int kMostLevel = 96;  // (what is smaller by more than that keeps fewer bits)
__device__ __forceinline__ int more_at(const NsParams &p, int level, int k) {
    const int e = (int)floorf((float)level - (float)k * p.growth);
    return e > 0 ? e : 0;
}
__device__ __forceinline__ int level_of(const NsParams &p, double norm) {
    // (a norm of infinity or NaN gets an end of int from ilogb, and then one of the range's ends)
    const int l = ilogb(p.eps / norm);
    return l < 0 ? 0 : l < kMostLevel ? l : kMostLevel;
}
// what the entries of a matrix are multiplied with to be those of X before the first step
__device__ __forceinline__ double first_scale(const NsParams &p, double norm, int level) {
    if (norm == 0.0) return 0.0;  // (the smallest eps would make it infinite)
    return ldexp(p.scale, more_at(p, level, 0)) / (norm < p.eps ? p.eps : norm);
}
struct Scales {
    float poly_a, poly_b, poly_c, from_gram, from_last;
    __device__ __forceinline__ Scales(const NsParams &p, int level, int k) {
        const int e = more_at(p, level, k), next = more_at(p, level, k + 1);
        poly_a = ldexpf(p.poly_a, next - e);
        poly_b = ldexpf(p.poly_b, next - 2 * e);
        poly_c = ldexpf(p.poly_c, next - 3 * e);
        from_gram = ldexpf(p.from_gram, -e);
        from_last = ldexpf(p.from_last, -next);
    }
};

constexpr int kPlane = 2048, kPlanes = 2, kUnit = kPlanes * kPlane;  // bytes of a unit's plane, planes, bytes of a unit

__host__ __device__ inline int units(int n) { return (n + 31) / 32; }

// ---- matrices and their buffers

struct View {
    NsMat m;
    int r, c;         // the iterate's rows and columns, r <= c
    int R, C;         // in units
    bool tr;          // the iterate is the transposed matrix
    bool xt;          // a workgroup's matrix: X lies transposed, in x0 alone
    char *x0, *x1, *A, *P;
};

__device__ __forceinline__ View view_of(const NsWork &w, int k) {
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
    v.R = units(v.r);
    v.C = units(v.c);
    v.xt = v.m.by_matrix != 0;
    const int64_t nx = (int64_t)v.R * v.C * kUnit;
    v.x0 = w.ws + v.m.off;
    v.x1 = v.x0 + nx;
    v.A = v.x1 + nx;
    v.P = v.A + (int64_t)v.R * v.R * kUnit;
    return v;
}

// Workgroups go round the eight XCDs, each with an L2 of its own.  A stack of eight matrices
// or more puts matrix k on XCD k % 8, so that the tiles of a matrix share an L2;
// the tables of a plan are ordered likewise on the host.  GRAM: the upper triangle of tiles
template <bool GRAM>
__device__ __forceinline__ NsTile tile_of(const NsWork &w, int k) {
    if (w.tiles) return w.tiles[k];
    const int per = GRAM ? w.nti * (w.nti + 1) / 2 : w.nti * w.ntj;
    int e, mat;
    // workgroup k runs on XCD k % 8: it has every eighth matrix, or an eighth of a few large ones' tiles
    if (w.n_mats >= 8) {
        const int q = k >> 3;
        mat = (k & 7) + 8 * (q / per);
        e = q % per;
        if (mat >= w.n_mats) mat = -1;
    } else {
        const int all = w.n_mats * per, q = (k & 7) * ((all + 7) / 8) + (k >> 3);
        mat = q < all ? q / per : -1;
        e = q % per;
    }
    // Bands of four tile rows, column by column: 32 tiles in a row need 12 panels of the operands (row by
    // row 18 of 16 columns).  A triangle's band begins with the one on its diagonal
    for (int ti = 0;; ti += 4) {
        const int nb = w.nti - ti < 4 ? w.nti - ti : 4, diag = GRAM ? nb * (nb + 1) / 2 : 0;
        const int band = diag + nb * (GRAM ? w.nti - ti - nb : w.ntj);
        if (e >= band && ti + 4 < w.nti) {
            e -= band;
            continue;
        }
        if (e >= diag) {
            e -= diag;
            return NsTile{mat, ti + e % nb, (GRAM ? ti + nb : 0) + e / nb};
        }
        int col = 0;
        while (e > col) {
            ++col;
            e -= col;
        }
        return NsTile{mat, ti + e, ti + col};
    }
}

// ---- units

// byte of chunk `half` (k 8 half .. + 7 of 16-entry block blk) of a row inside a plane
__device__ __forceinline__ int chunk(int row, int half, int blk) {
    const int g = row >> 2;
    return g * 256 + (((row & 3) | ((half ^ (g & 1)) << 2) | ((blk ^ ((g >> 1) & 1)) << 3)) << 4);
}

// operand fragment of 16 contraction entries from a unit's plane in LDS: lane
// = row, entries 16 s + 8 (lane / 32) ..
__device__ __forceinline__ half8 frag_rows(const char *plane, int lane, int s) {
    return *(const half8 *)(plane + chunk(lane & 31, lane >> 5, s));
}
// the same with lane = column of the unit, contraction over its rows
__device__ __forceinline__ half8 frag_cols(const char *plane, int lane, int s) {
    const int G = lane >> 4, i = lane & 15;
    const int row = 16 * s + 8 * (G >> 1) + (i >> 2);
    const int half = (i >> 1) & 1, blk = G & 1, sub = (i & 1) * 8;
    typedef __attribute__((address_space(3))) short4tr lds4;
    const short4tr a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(plane + chunk(row, half, blk) + sub));
    const short4tr b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(plane + chunk(row + 4, half, blk) + sub));
    return __builtin_bit_cast(half8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Four values f v as two fp16 each that sum up to them within 22 bits.  Conversions
// two at a time, the remainder in one mixed fused multiply-add: 3 operations per value
typedef float float2v __attribute__((ext_vector_type(2)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void split4(const float (&v)[4], float f, half4 (&p)[kPlanes]) {
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
        const half2v hi = __builtin_convertvector((float2v{v[e] * f, v[e + 1] * f}), half2v);
        p[0][e] = hi.x;
        p[0][e + 1] = hi.y;
        const half2v lo =
            __builtin_convertvector((float2v{fmaf(v[e], f, -(float)hi.x), fmaf(v[e + 1], f, -(float)hi.y)}), half2v);
        p[1][e] = lo.x;
        p[1][e + 1] = lo.y;
    }
}

template <int N> struct Int { static constexpr int value = N; };

struct Frag { half8 p[kPlanes]; };

// the product's t-th term, the small ones first: lo hi, hi lo, hi hi
constexpr int kTerms = 3;
__device__ __forceinline__ void mma_term(f32x16 &acc, const Frag &a, const Frag &b, int t) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a.p[t == 0], b.p[t == 1], acc, 0, 0, 0);
}
__device__ __forceinline__ void mma(f32x16 &acc, const Frag &a, const Frag &b) {
#pragma unroll
    for (int t = 0; t < kTerms; ++t) mma_term(acc, a, b, t);
}

// ---- norm, scaling and update: a thread owns 4 x 4 entries of a 64 x 64 tile.  Streams, bound by HBM:
// 73 M entries of a model in 185, 198 and 299 us, 12, 12 and 20 bytes each (4.5 to 4.9 TB/s)

// four consecutive entries of a memory row, zeros past its end
__device__ __forceinline__ void load4(float (&v)[4], const float *p, int left) {
    if (left >= 4) {
        __builtin_memcpy(v, p, 16);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = e < left ? p[e] : 0.0f;
    }
}
__device__ __forceinline__ void load4(float (&v)[4], const uint16_t *p, int left) {
    uint16_t u[4] = {0, 0, 0, 0};
    if (left >= 4) {
        __builtin_memcpy(u, p, 8);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = e < left ? p[e] : 0;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = bf2f(u[e]);
}
__device__ __forceinline__ void store4(const float (&v)[4], float *p, int left) {
    if (left >= 4) {
        __builtin_memcpy(p, v, 16);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) p[e] = v[e];
    }
}

// the thread's entries u[4][4] by memory rows; UPDATE: the momentum is formed
// and written, otherwise it is read as written
template <bool MUON, bool BF16, bool UPDATE>
__device__ __forceinline__ void load_block(float (&u)[4][4], const View &v, const NsParams &p, int row0, int col0) {
    const float gs = MUON && p.grad_scale ? *p.grad_scale : 1.0f;
    float m[4][4];
#pragma unroll
    for (int a = 0; a < 4; ++a) {
        const int left = row0 + a < v.m.rows ? v.m.cols - col0 : 0;
        const int64_t at = (int64_t)(row0 + a) * v.m.cols + col0;
        if constexpr (BF16) load4(u[a], (const uint16_t *)v.m.in + at, left);
        else load4(u[a], (const float *)v.m.in + at, left);
        if constexpr (MUON) load4(m[a], v.m.mom + at, left);
    }
    if constexpr (MUON) {
#pragma unroll
        for (int a = 0; a < 4; ++a) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float g = u[a][e] * gs;
                if constexpr (UPDATE) m[a][e] = fmaf(p.mu, m[a][e], p.om_mu * g);
                u[a][e] = fmaf(p.u_m, m[a][e], p.u_g * g);
            }
            if constexpr (UPDATE)
                store4(m[a], v.m.mom + (int64_t)(row0 + a) * v.m.cols + col0,
                       row0 + a < v.m.rows ? v.m.cols - col0 : 0);
        }
    }
}

// the thread's entries times f into the units of X, or (TRANSPOSED) of its transpose
template <bool TRANSPOSED>
__device__ __forceinline__ void pack_block(const float (&u)[4][4], const View &v, char *x0, int row0, int col0, double f) {
    const bool by_cols = v.tr != TRANSPOSED;  // a unit's rows are the columns in memory
    const int rows = TRANSPOSED ? v.C : v.R, cols = TRANSPOSED ? v.R : v.C;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        // row i, columns j .. j + 3
        const int i = by_cols ? col0 + x : row0 + x, j = by_cols ? row0 : col0;
        if ((i >> 5) >= rows || (j >> 5) >= cols) continue;
        float q[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) q[y] = (float)((double)(by_cols ? u[y][x] : u[x][y]) * f);
        half4 hh[kPlanes];
        split4(q, 1.0f, hh);
        char *unit = x0 + ((int64_t)(i >> 5) * cols + (j >> 5)) * kUnit;
        const int k = j & 31, at = chunk(i & 31, (k >> 3) & 1, k >> 4) + (k & 4) * 2;
#pragma unroll
        for (int z = 0; z < kPlanes; ++z) *(half4 *)(unit + z * kPlane + at) = hh[z];
    }
}

// momentum, and the sum of squares of each tile (fp64: no overflow or underflow of fp32 squares)
template <bool MUON, bool BF16>
__global__ __launch_bounds__(256) void ns_norm_kernel(NsWork w, NsParams p) {
    __shared__ double red[4];
    const NsTile t = tile_of<false>(w, blockIdx.x);
    if (t.mat < 0) return;
    const View v = view_of(w, t.mat);
    const int tid = threadIdx.x;
    const int mi = v.tr ? t.tj : t.ti, mj = v.tr ? t.ti : t.tj;
    float u[4][4];
    load_block<MUON, BF16, true>(u, v, p, mi * kNsBlock + (tid >> 4) * 4, mj * kNsBlock + (tid & 15) * 4);
    double s = 0.0;
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) s += (double)u[a][e] * u[a][e];
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m, 64);
    if ((tid & 63) == 0) red[tid >> 6] = s;
    __syncthreads();
    const int ntj = (v.c + kNsBlock - 1) / kNsBlock, nti = (v.r + kNsBlock - 1) / kNsBlock;
    const int64_t first = w.mats ? v.m.part0 : (int64_t)t.mat * nti * ntj;
    if (tid == 0) w.part[first + t.ti * ntj + t.tj] = ((red[0] + red[1]) + red[2]) + red[3];
}

// X = u / max(|u|, eps), in units, transposed for a workgroup's matrix
template <bool MUON, bool BF16>
__global__ __launch_bounds__(256) void ns_scale_kernel(NsWork w, NsParams p) {
    __shared__ double red[4];
    const NsTile t = tile_of<false>(w, blockIdx.x);
    if (t.mat < 0) return;
    const View v = view_of(w, t.mat);
    const int tid = threadIdx.x;
    const int mi = v.tr ? t.tj : t.ti, mj = v.tr ? t.ti : t.tj;
    const int row0 = mi * kNsBlock + (tid >> 4) * 4, col0 = mj * kNsBlock + (tid & 15) * 4;
    float u[4][4];
    load_block<MUON, BF16, false>(u, v, p, row0, col0);
    // every workgroup sums the matrix's partial sums itself, in the same order
    const int ntj = (v.c + kNsBlock - 1) / kNsBlock, nti = (v.r + kNsBlock - 1) / kNsBlock, n = nti * ntj;
    const double *part = w.part + (w.mats ? v.m.part0 : (int64_t)t.mat * n);
    double s = 0.0;
    for (int k = tid; k < n; k += 256) s += part[k];
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m, 64);
    if ((tid & 63) == 0) red[tid >> 6] = s;
    __syncthreads();
    const double norm = sqrt(((red[0] + red[1]) + red[2]) + red[3]);
    const int level = level_of(p, norm);
    if (tid == 0 && t.ti == 0 && t.tj == 0) w.levels[t.mat] = level;
    const double f = first_scale(p, norm, level);
    if (v.xt) pack_block<true>(u, v, v.x0, row0, col0, f);
    else pack_block<false>(u, v, v.x0, row0, col0, f);
}

// p = decay p - lr scale O, w = sd w + om_sd p, with O as the last product left it in buffer `odd` of X:
// 32 x 32 floats in the place of each unit, by memory rows
__global__ __launch_bounds__(256) void ns_update_kernel(NsWork w, NsParams p, int odd) {
    const NsTile t = tile_of<false>(w, blockIdx.x);
    if (t.mat < 0) return;
    const View v = view_of(w, t.mat);
    const int tid = threadIdx.x;
    const int mi = v.tr ? t.tj : t.ti, mj = v.tr ? t.ti : t.tj;
    const int row0 = mi * kNsBlock + (tid >> 4) * 4, col0 = mj * kNsBlock + (tid & 15) * 4;
    const int i = (v.tr ? col0 : row0) >> 5, j = (v.tr ? row0 : col0) >> 5;  // unit of the iterate
    if (i >= v.R || j >= v.C) return;
    const char *x = v.xt || !odd ? v.x0 : v.x1;
    const float *o = (const float *)(x + (v.xt ? (int64_t)j * v.R + i : (int64_t)i * v.C + j) * (2 * kPlane));
    float *const prm = (float *)v.m.out, *const swa = v.m.swa;
    const float f = -p.lr * v.m.scale;
    float q[4][4], a[4][4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int64_t at = (int64_t)(row0 + r) * v.m.cols + col0;
        const int left = row0 + r < v.m.rows ? v.m.cols - col0 : 0;
        load4(q[r], prm + at, left);
        if (swa) load4(a[r], swa + at, left);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int64_t at = (int64_t)(row0 + r) * v.m.cols + col0;
        const int left = row0 + r < v.m.rows ? v.m.cols - col0 : 0;
        const f32x4 u = *(const f32x4 *)(o + ((row0 + r) & 31) * 32 + (col0 & 31));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            q[r][e] = fmaf(f, u[e], p.decay * q[r][e]);
            if (swa) a[r][e] = fmaf(p.sd, a[r][e], p.om_sd * q[r][e]);
        }
        store4(q[r], prm + at, left);
        if (swa) store4(a[r], swa + at, left);
    }
}

// ---- results

// entries of P = a I + b A + c A A from those of the product A A and of A, all with their scales, three operations
// each (mixed fused multiply-adds take the halves as they are); diagonal: whether the unit lies on it
// (wave-uniform), and then which of the four does, if any
__device__ __forceinline__ void poly4(float (&q)[4], const half4 (&old)[kPlanes], const Scales &p, bool diagonal, int which) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        q[e] = fmaf((float)old[0][e], p.poly_b, p.poly_c * q[e]);
        q[e] = fmaf((float)old[1][e], p.poly_b, q[e]);
    }
    if (diagonal) {
#pragma unroll
        for (int e = 0; e < 4; ++e) q[e] += e == which ? p.poly_a : 0.0f;
    }
}

// acc (a unit: lane = row, registers = columns) times f as packed quarters
__device__ __forceinline__ void pack_unit(const f32x16 &acc, float f, half4 (&out)[4][kPlanes]) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        float q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) q[e] = acc[4 * g + e];
        split4(q, f, out[g]);
    }
}
__device__ __forceinline__ void store_unit(char *unit, const half4 (&out)[4][kPlanes], int n, int h) {
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int z = 0; z < kPlanes; ++z) *(half4 *)(unit + z * kPlane + chunk(n, g & 1, g >> 1) + h * 8) = out[g][z];
}

// One unit's entries of the result, the lanes along the memory rows.  A buffer begins at the unit's
// first row and ends with the matrix (or 2 GB on, past the unit): rows beyond it read
// nothing and are not written, so no entry takes a branch; columns beyond it are sent there
template <bool BF16>
struct UnitOut {
    rsrc_t r;
    uint32_t lane, row;  // byte offset of the lane's first entry, bytes of a memory row
    __device__ __forceinline__ UnitOut(const View &v, const void *base, int iu, int ju, int h, int n) {
        constexpr uint32_t ES = BF16 ? 2 : 4;
        asm volatile("" : "+v"(h), "+v"(n));  // (or a loop over units has all of their addresses made before it)
        const int row0 = __builtin_amdgcn_readfirstlane((v.tr ? ju : iu) * 32), col0 = (v.tr ? iu : ju) * 32;
        const int64_t first = (int64_t)row0 * v.m.cols;
        const int64_t left = ((int64_t)v.m.rows * v.m.cols - first) * ES;
        r = make_buf((const char *)base + first * ES, (uint32_t)(left < 0x7ffffff0 ? left : 0x7ffffff0));
        row = (uint32_t)v.m.cols * ES;
        lane = col0 + n < v.m.cols ? (uint32_t)(4 * h) * row + (uint32_t)(col0 + n) * ES : kOOB;
    }
    __device__ __forceinline__ uint32_t at(int e) const { return lane + (uint32_t)(8 * (e >> 2) + (e & 3)) * row; }
};

template <bool MUON, bool BF16>
struct Result {
    float p[16], w[16];
    __device__ __forceinline__ void before(const View &v, int iu, int ju, int h, int n) {
        if constexpr (MUON) {
            const UnitOut<false> a(v, v.m.out, iu, ju, h, n);
#pragma unroll
            for (int e = 0; e < 16; ++e) p[e] = __uint_as_float(bload4(a.r, a.at(e)));
            if (v.m.swa) {
                const UnitOut<false> b(v, v.m.swa, iu, ju, h, n);
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = __uint_as_float(bload4(b.r, b.at(e)));
            }
        }
    }
    __device__ __forceinline__ void store(const View &v, const NsParams &P, float from_last, const f32x16 &acc, int iu, int ju, int h, int n) {
        const UnitOut<BF16> a(v, v.m.out, iu, ju, h, n);
        if constexpr (MUON) {
            const float f = -P.lr * v.m.scale * from_last;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                p[e] = fmaf(f, acc[e], P.decay * p[e]);
                bstore4(__float_as_uint(p[e]), a.r, a.at(e));
            }
            if (v.m.swa) {
                const UnitOut<false> b(v, v.m.swa, iu, ju, h, n);
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    bstore4(__float_as_uint(fmaf(P.sd, w[e], P.om_sd * p[e])), b.r, b.at(e));
            }
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                if constexpr (BF16) __builtin_amdgcn_raw_buffer_store_b16(f2bf(acc[e] * from_last), a.r, a.at(e), 0, 0);
                else bstore4(__float_as_uint(acc[e] * from_last), a.r, a.at(e));
            }
        }
    }
};

// the last product's unit: for Muon as floats by memory rows in the unit's place, for ns_update_kernel,
// otherwise the result itself
template <bool MUON, bool BF16>
__device__ __forceinline__ void store_last(const View &v, const NsParams &p, float from_last, const f32x16 &acc, char *unit, int iu,
                                           int ju, int h, int n) {
    if constexpr (MUON) {
        float *const o = (float *)unit + 128 * h + n;
#pragma unroll
        for (int e = 0; e < 16; ++e) o[(8 * (e >> 2) + (e & 3)) * 32] = acc[e] * from_last;
    } else {
        Result<MUON, BF16> res;
        res.store(v, p, from_last, acc, iu, ju, h, n);
    }
}

// ---- products
//
// A workgroup of 4 waves forms a T x T tile, a wave a quarter of it, from units staged
// in LDS, one unit column (32 contraction entries) per stage, copied by
// global_load_lds 16 bytes a lane, S - 1 stages ahead: the copies are counted
// by hand (vmcnt), one barrier per stage.  The matrix instructions bound large
// products, the chain of stages and the launch small
// ones: 8 matrices of 2048 x 2048 in pairs, Gram 216 us (1.0 PFLOP/s of fp16 products), polynomial 222,
// P X 355 (1.2); one such matrix 37, 40 and 47 us; 52 of 128 x 512 6.9, 5.1 and 9.7.

enum { kGram, kPoly, kApply, kLast };
struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };

// a wave-uniform address, in scalar registers whatever the compiler makes of its terms
__device__ __forceinline__ const char *scalar(const char *p) {
    const uint64_t a = (uint64_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a), hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
    return (const char *)(((uint64_t)hi << 32) | lo);
}

// 16 bytes per lane from base + off to LDS at lds + 16 lane.  In asm because the compiler would
// wait for all copies in flight before every LDS read; nothing but the counter below waits for these.
// (M0 holds the LDS address; nothing else in these kernels uses it)
__device__ __forceinline__ void copy_to_lds(const char *base, uint32_t off, uint32_t lds) {
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %1, %2"
        :
        : "s"(lds), "v"(off), "s"(base)
        : "memory");
}
template <int N>
__device__ __forceinline__ void wait_copies_and_barrier() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(N) : "memory");
}

// a barrier for what lies in LDS alone
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory"); }

template <int T, int S, int KIND, bool MUON, bool BF16>
__global__ __launch_bounds__(256) void ns_product_kernel(NsWork w, NsParams p, int k0) {
    constexpr int U = T / 64;             // units of a wave's tile in each direction
    constexpr int N = T / 32;             // units of the workgroup's
    constexpr int STAGE = 2 * N * kUnit;
    constexpr int COPIES = U * kUnit / 1024;  // of a wave and stage
    constexpr bool SQUARE = KIND == kGram || KIND == kPoly;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const NsTile t = tile_of<SQUARE>(w, blockIdx.x);
    if (t.mat < 0) return;
    const View v = view_of(w, t.mat);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = wave >> 1, wc = wave & 1, h = lane >> 5, n = lane & 31;
    const bool odd = k0 & 1;
    const char *x = KIND == kPoly ? v.A : odd ? v.x1 : v.x0;
    const Scales sc(p, KIND == kApply ? 0 : w.levels[t.mat], k0);
    const int K = KIND == kGram ? v.C : v.R;  // unit columns of the contraction

    // this wave's share of a stage: U units; units past the matrix repeat its
    // last one, for results that are not stored
    const char *src[U];
    int64_t step;
#pragma unroll
    for (int q = 0; q < U; ++q) {
        const int e = wave * U + q, op = e / N, k = e % N;  // operand (wave-uniform: N is a multiple of U)
        const int first = (op == 0 ? t.ti : t.tj) * N + k;
        if (SQUARE) {
            const int row = first < v.R ? first : v.R - 1;
            src[q] = x + (int64_t)row * K * kUnit;
            step = kUnit;
        } else if (op == 0) {
            const int row = first < v.R ? first : v.R - 1;
            src[q] = v.P + (int64_t)row * v.R * kUnit;
            step = kUnit;
        } else {
            const int col = first < v.C ? first : v.C - 1;
            src[q] = x + (int64_t)col * kUnit;
            step = (int64_t)v.C * kUnit;
        }
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    auto copy = [&](int k, int c) {  // the wave's c-th KB of stage k
        const int q = c / (kUnit / 1024), e = c % (kUnit / 1024);
        copy_to_lds(scalar(src[q] + k * step), (uint32_t)(e * 1024 + lane * 16),
                    lds0 + (uint32_t)(k % S) * STAGE + (uint32_t)(wave * U + q) * kUnit + e * 1024);
    };

    f32x16 acc[U][U];  // [row unit or, where the operands are swapped, ...]: see below
#pragma unroll
    for (int a = 0; a < U; ++a)
#pragma unroll
        for (int b = 0; b < U; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[a][b][e] = 0.0f;

    // operand 0's fragments f0 (tile rows), operand 1's f1 (tile columns).  D = f0 f1 has lane = column,
    // registers = rows; D = f1 f0 the other way round, which is what an iterate's units store
    // (lane = row, four consecutive columns)
    // Four waves, one per SIMD: whatever holds up a wave's issue leaves its matrix core idle.  The operands of
    // a half stage are read while the other half's products run, one at a time between them, and so are the
    // copies issued (in a row each costs a fifth of the time)
    auto products = [&](auto swapped) {
        constexpr int MMAS = kTerms * U * U, READS = 2 * U * kPlanes;  // of a half
        constexpr bool AHEAD = S > 2;  // the next stage's first half is read, too, while this one's products run
#pragma unroll
        for (int k = 0; k < S - 1; ++k)
            if (k < K) {
#pragma unroll
                for (int c = 0; c < COPIES; ++c) copy(k, c);
            }
        Frag f0[2][U], f1[2][U];  // of the two halves of a stage
        // r-th operand of half s, in the order of their use: the left ones' lo, the right ones' hi, ...
        auto read = [&](int k, int s, int r) {
            const int a = r % U, z = r / U, left = z == 0 || z == 3, q = z == 0 || z == 2;
            const char *at = lds + (k % S) * STAGE + q * kPlane + ((left ? wr * U : N + wc * U) + a) * kUnit;
            if (left) f0[s][a].p[q] = frag_rows(at, lane, s);
            else f1[s][a].p[q] = SQUARE ? frag_rows(at, lane, s) : frag_cols(at, lane, s);
        };
        // the products of half s, and between them the reads of the next half (one past the end is read, but
        // not used: a branch around the read would turn the next wait into one for all reads)
        auto half = [&](int k, int s, auto copying) {
#pragma unroll
            for (int t = 0; t < kTerms; ++t)
#pragma unroll
                for (int a = 0; a < U; ++a)
#pragma unroll
                    for (int b = 0; b < U; ++b) {
                        if constexpr (decltype(swapped)::value) mma_term(acc[a][b], f1[s][b], f0[s][a], t);
                        else mma_term(acc[a][b], f0[s][a], f1[s][b], t);
                        const int m = (t * U + a) * U + b, n = s * MMAS + m;
                        __builtin_amdgcn_sched_barrier(0);
                        constexpr int EACH = (READS + MMAS - 1) / MMAS;
#pragma unroll
                        for (int r = m * EACH; r < (m + 1) * EACH && r < READS; ++r)
                            if (AHEAD || s == 0) read(k + s, 1 - s, r);
                        if constexpr (decltype(copying)::value) {
#pragma unroll
                            for (int c = n * COPIES / (2 * MMAS); c < (n + 1) * COPIES / (2 * MMAS); ++c) copy(k + S - 1, c);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
        };
        int k = 0;
        auto stage = [&](auto copying) {  // stage k + 1 has arrived, too
            if (!AHEAD || k == 0) {
#pragma unroll
                for (int r = 0; r < READS; ++r) read(k, 0, r);
            }
            half(k, 0, copying);
            half(k, 1, copying);
        };
        for (; k + S - 1 < K; ++k) {
            wait_copies_and_barrier<AHEAD ? (S - 3) * COPIES : 0>();
            stage(Yes{});
        }
        for (; k < K; ++k) {
            wait_copies_and_barrier<0>();
            stage(No{});
        }
    };
    const int i0 = t.ti * N + wr * U, j0 = t.tj * N + wc * U;  // this wave's first units
    if constexpr (SQUARE) {
        // lane = column: stored as row `column` of the symmetric matrix's unit (j, i)
        products(No{});
        __syncthreads();  // the stages become scratch
        char *const scratch = lds + wave * kUnit;
        char *const dst = KIND == kPoly ? v.P : v.A;
#pragma unroll
        for (int a = 0; a < U; ++a)
#pragma unroll
            for (int b = 0; b < U; ++b) {
                const int i = i0 + a, j = j0 + b;
                if (i >= v.R || j >= v.R) continue;  // wave-uniform
                const int64_t at = ((int64_t)j * v.R + i) * kUnit;
                half4 out[4][kPlanes];
#pragma unroll
                for (int g = 0; g < 4; ++g) {  // rows 8 g + 4 h .. + 3 of the tile
                    const int pos = chunk(n, g & 1, g >> 1) + h * 8;
                    float q[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) q[e] = acc[a][b][4 * g + e];
                    if constexpr (KIND == kPoly) {
                        half4 old[kPlanes];
#pragma unroll
                        for (int z = 0; z < kPlanes; ++z) old[z] = *(const half4 *)(v.A + at + z * kPlane + pos);
                        poly4(q, old, sc, i == j, n - 8 * g - 4 * h);
                    }
                    split4(q, KIND == kPoly ? 1.0f : sc.from_gram, out[g]);
#pragma unroll
                    for (int z = 0; z < kPlanes; ++z) *(half4 *)(dst + at + z * kPlane + pos) = out[g][z];
                }
                if (t.ti != t.tj) {  // the mirrored unit (i, j), through LDS by columns
#pragma unroll
                    for (int g = 0; g < 4; ++g)
#pragma unroll
                        for (int z = 0; z < kPlanes; ++z)
                            *(half4 *)(scratch + z * kPlane + chunk(n, g & 1, g >> 1) + h * 8) = out[g][z];
                    __builtin_amdgcn_wave_barrier();
                    const int64_t mirrored = ((int64_t)i * v.R + j) * kUnit;
#pragma unroll
                    for (int z = 0; z < kPlanes; ++z)
#pragma unroll
                        for (int s = 0; s < 2; ++s)
                            *(half8 *)(dst + mirrored + z * kPlane + chunk(n, h, s)) = frag_cols(scratch + z * kPlane, lane, s);
                    __builtin_amdgcn_wave_barrier();
                }
            }
    } else if constexpr (KIND == kApply) {
        products(Yes{});  // lane = row, registers = columns
        char *const dst = odd ? v.x0 : v.x1;
#pragma unroll
        for (int a = 0; a < U; ++a)
#pragma unroll
            for (int b = 0; b < U; ++b) {
                const int i = i0 + a, j = j0 + b;
                if (i >= v.R || j >= v.C) continue;
                char *unit = dst + ((int64_t)i * v.C + j) * kUnit;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    float q[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) q[e] = acc[a][b][4 * g + e];
                    half4 out[kPlanes];
                    split4(q, p.from_apply, out);
#pragma unroll
                    for (int z = 0; z < kPlanes; ++z)
                        *(half4 *)(unit + z * kPlane + chunk(n, g & 1, g >> 1) + h * 8) = out[z];
                }
            }
    } else {
        // the lanes go along the matrix's memory rows: columns of the iterate, or its rows where it is transposed
        if (v.tr) products(Yes{});
        else products(No{});
#pragma unroll
        for (int a = 0; a < U; ++a)
#pragma unroll
            for (int b = 0; b < U; ++b) {
                const int i = i0 + a, j = j0 + b;
                if (i >= v.R || j >= v.C) continue;
                store_last<MUON, BF16>(v, p, sc.from_last, acc[a][b], (odd ? v.x0 : v.x1) + ((int64_t)i * v.C + j) * kUnit, i, j, h, n);
            }
    }
}

// A symmetric matrix in LDS as the units of one triangle: unit (r, k), r >= k, holds rows r, contraction
// k.  An operand of the other triangle is the mirrored unit read by columns
__device__ __forceinline__ char *tri_unit(char *base, int r, int k) {
    return base + (r * (r + 1) / 2 + k) * kUnit;
}
// rows of unit row r, contraction over unit column k (both wave-uniform)
__device__ __forceinline__ void tri_frag(Frag &f, char *base, int r, int k, int s, int lane) {
    if (r >= k) {
        const char *u = tri_unit(base, r, k);
#pragma unroll
        for (int z = 0; z < kPlanes; ++z) f.p[z] = frag_rows(u + z * kPlane, lane, s);
    } else {
        const char *u = tri_unit(base, k, r);
#pragma unroll
        for (int z = 0; z < kPlanes; ++z) f.p[z] = frag_cols(u + z * kPlane, lane, s);
    }
}

// ---- matrices that fit into LDS: everything in one workgroup
//
// X and the triangle of A, then of P in its place, lie in LDS: 128 x 224 entries, 64 x 576,
// 32 x 1216.  P's entries wait in registers until every wave has read A.  One launch does the norm, the steps and the
// update: memory sees each entry once.  Each of 16 waves takes a unit of the
// triangle (10 of them at 128 x 128), then unit columns of X.  What bounds it are the
// chains of a unit, LDS reads, matrix instructions, splitting and storing: at 128 x 128
// 4000 cycles a step for the Gram matrix, 6200 for the polynomial and 6200 for P X,
// against 1900, 1900 and 3100 of matrix instructions on the busiest SIMD; so the next operands
// are read before the matrix instructions of the last.  128 x 128: 37 us; 256
// matrices of 128 x 224 70 us, of 96 x 352 65.

constexpr int kSmallUnits = 40;
constexpr int kSmallLds = 39 * kUnit;
static_assert(kSmallLds + 1024 <= 160 * 1024, "X, the triangle and the partial sums fill a workgroup's LDS at most");
constexpr int kSmallWaves = 16;

__host__ __device__ inline bool fits_small(int R, int C) {
    return R * C <= kSmallUnits && (R * C + R * (R + 1) / 2) * kUnit <= kSmallLds;
}

template <bool MUON, bool BF16>
__global__ __launch_bounds__(64 * kSmallWaves) void ns_small_kernel(NsWork w, NsParams p, int first) {
    constexpr int THREADS = 64 * kSmallWaves;
    constexpr int BLOCKS = (kSmallUnits * 64 + THREADS - 1) / THREADS;  // 4 x 4 blocks of a thread
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    __shared__ double red[kSmallWaves];
    const View v = view_of(w, first + blockIdx.x);
    const int tid = threadIdx.x;
    int lane = tid & 63, h = lane >> 5, n = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int R = v.R, C = v.C;
    char *const X = lds, *const A = lds + R * C * kUnit;

    int level;
    {  // X = u / max(|u|, eps)
        const int per_row = 8 * (v.tr ? R : C), blocks = 64 * R * C;
        float u[BLOCKS][4][4];
        double s = 0.0;
#pragma unroll
        for (int q = 0; q < BLOCKS; ++q) {
            const int k = q * THREADS + tid;
            if (q * THREADS < blocks) {
                const int br = k / per_row, bc = k - br * per_row;
                load_block<MUON, BF16, true>(u[q], v, p, br * 4, bc * 4);
#pragma unroll
                for (int a = 0; a < 4; ++a)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s += (double)u[q][a][e] * u[q][a][e];
            }
        }
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m, 64);
        if (lane == 0) red[wave] = s;
        __syncthreads();
        s = red[0];
#pragma unroll
        for (int k = 1; k < kSmallWaves; ++k) s += red[k];
        const double norm = sqrt(s);
        level = level_of(p, norm);
        const double f = first_scale(p, norm, level);
#pragma unroll
        for (int q = 0; q < BLOCKS; ++q) {
            const int k = q * THREADS + tid;
            if (k < blocks) {
                const int br = k / per_row, bc = k - br * per_row;
                pack_block<false>(u[q], v, X, br * 4, bc * 4, f);
            }
        }
        __syncthreads();
    }

    const int tri = R * (R + 1) / 2;
    // t-th unit (b, a), b >= a, of the triangle; past its end the last one, not stored
    auto unit_of = [&](int t, int &a, int &b) {
        b = 0;
        while (t > b) {
            ++b;
            t -= b;
        }
        a = t;
    };
    auto zero = [](f32x16 &x) {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = 0.0f;
    };
    // sum over k of left(k) right(k), each a loader of the operands of unit column k
    auto contract = [&](f32x16 &acc, int K, auto left, auto right) {
        zero(acc);
        Frag l[2], r[2];  // one half (16 entries) ahead
        left(l[0], 0, 0);
        right(r[0], 0, 0);
        for (int k = 0; k < K; ++k) {
            left(l[1], k, 1);
            right(r[1], k, 1);
            mma(acc, l[0], r[0]);
            // (past the end the last ones again, not used: a branch here would make the next wait one for all reads)
            left(l[0], k + 1 < K ? k + 1 : k, 0);
            right(r[0], k + 1 < K ? k + 1 : k, 0);
            mma(acc, l[1], r[1]);
        }
    };
    auto x_rows = [&](int a) {
        return [&, a](Frag &f, int k, int s) {
#pragma unroll
            for (int z = 0; z < kPlanes; ++z) f.p[z] = frag_rows(X + (a * C + k) * kUnit + z * kPlane, lane, s);
        };
    };
    auto x_cols = [&](int b) {
        return [&, b](Frag &f, int k, int s) {
#pragma unroll
            for (int z = 0; z < kPlanes; ++z) f.p[z] = frag_cols(X + (k * C + b) * kUnit + z * kPlane, lane, s);
        };
    };
    auto a_rows = [&](int a) { return [&, a](Frag &f, int k, int s) { tri_frag(f, A, a, k, s, lane); }; };

    const bool mine = wave < tri;  // (R <= 4: ten units at most)
    int ta, tb;
    unit_of(mine ? wave : 0, ta, tb);
    auto columns = [&](auto rows) {
        constexpr int RR = decltype(rows)::value;
        for (int b = wave; b < C; b += kSmallWaves) {
            f32x16 acc[RR];  // lane = row, registers = columns
#pragma unroll
            for (int a = 0; a < RR; ++a) zero(acc[a]);
            Frag x[2], f[2];  // operands one ahead: P's of the next row, X's of the next half unit
            x_cols(b)(x[0], 0, 0);
            tri_frag(f[0], A, 0, 0, 0, lane);
#pragma unroll
            for (int at = 0; at < 2 * RR * RR; ++at) {
                const int a = at % RR, half = at / RR, next = at + 1;
                if (a == 0 && half + 1 < 2 * RR) x_cols(b)(x[(half + 1) & 1], (half + 1) >> 1, (half + 1) & 1);
                if (next < 2 * RR * RR) tri_frag(f[next & 1], A, next % RR, next / RR >> 1, next / RR & 1, lane);
                __builtin_amdgcn_sched_barrier(0);
                mma(acc[a], x[half & 1], f[at & 1]);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int a = 0; a < RR; ++a) {
                half4 out[4][kPlanes];
                pack_unit(acc[a], p.from_apply, out);
                store_unit(X + (a * C + b) * kUnit, out, n, h);
            }
        }
    };
    auto one_step = [&](int step, bool last) {  // the last leaves P
        const Scales sc(p, level, step);
        // (every address is the lane's part plus the unit's: made anew, or the compiler makes all of them
        // before the loop and spills them)
        asm volatile("" : "+v"(lane));
        h = lane >> 5;
        n = lane & 31;
        char *const at = tri_unit(A, tb, ta);
        if (mine) {
            f32x16 acc;  // lane = row of tb, registers = rows of ta
            contract(acc, C, x_rows(ta), x_rows(tb));
            half4 out[4][kPlanes];
            pack_unit(acc, sc.from_gram, out);
            store_unit(at, out, n, h);
        }
        __syncthreads();
        {
            half4 out[4][kPlanes];
            if (mine) {
                f32x16 acc;
                contract(acc, R, a_rows(ta), a_rows(tb));
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    float q[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) q[e] = acc[4 * g + e];
                    half4 old[kPlanes];
#pragma unroll
                    for (int z = 0; z < kPlanes; ++z)
                        old[z] = *(const half4 *)(at + z * kPlane + chunk(n, g & 1, g >> 1) + h * 8);
                    poly4(q, old, sc, ta == tb, n - 8 * g - 4 * h);
                    split4(q, 1.0f, out[g]);
                }
            }
            __syncthreads();
            if (mine) store_unit(at, out, n, h);
            __syncthreads();
        }
        if (last) return;
        // X = P X: a wave takes whole unit columns, reads each X operand once for all its rows and stores
        // them in their place, which no other wave reads
        if (R == 1) columns(Int<1>{});
        else if (R == 2) columns(Int<2>{});
        else if (R == 3) columns(Int<3>{});
        else columns(Int<4>{});
        __syncthreads();
    };
    for (int step = 0; step < p.steps; ++step) one_step(step, step + 1 == p.steps);
    // the last step's P X: the lanes go along the matrix's memory rows
    const float from_last = Scales(p, level, p.steps - 1).from_last;
    for (int t = wave; t < R * C; t += kSmallWaves) {
        const int a = t / C, b = t - a * C;
        Result<MUON, BF16> res;
        res.before(v, a, b, h, n);
        f32x16 acc;
        if (v.tr) contract(acc, R, x_cols(b), a_rows(a));
        else contract(acc, R, a_rows(a), x_cols(b));
        res.store(v, p, from_last, acc, a, b, h, n);
    }
}

// ---- matrices of up to 256 rows, one workgroup each
//
// A workgroup of eight waves takes a matrix through all steps.  (The norm, the
// scaling and Muon's update are passes of their own: a CU by itself keeps too little in flight for them.)  The Gram
// matrix and then P lie in LDS, as the units of one triangle (36 of them, 144
// KB, for 256 rows): an operand of the other triangle is the mirrored
// unit read by columns.  X lies in the workspace, transposed, so that the
// fragments of P X come straight from memory, 1 KB a load: each wave takes unit
// columns of its own and writes the result in their place, without a barrier.  Memory
// then sees X read twice and written once per step: 240 matrices of 256 x 256 take 268 us, of
// 256 x 1024 800 (with A and P in the workspace, too, the former moved 2.7 GB at 6.4 TB/s and took 430).
// Over a model's matrices the matrix instructions take 41% of the time and the LDS 18%: two waves per SIMD, which
// wait for memory, LDS and barriers 46% of theirs, cover no more of each other's chains.
// A call with too few matrices for the CUs is done sooner by the tiles above.

constexpr int kWgWaves = 8;

template <int RB, bool MUON, bool BF16>
struct MatrixWg {
    static constexpr int STAGE = RB * kUnit, STAGES = 4;               // of the Gram matrix: a unit column of X
    static constexpr int TRI = RB * (RB + 1) / 2;
    static constexpr int LDS = TRI * kUnit > STAGES * STAGE ? TRI * kUnit : STAGES * STAGE;

    const NsParams &p;
    const View &v;
    char *lds;
    uint32_t lds0;
    int lane, wave, h, n;

    // Every address below is the lane's part plus the unit's; out of the loop over the steps the
    // compiler would compute all sums once and spill them, so each phase makes its own lane's part
    __device__ __forceinline__ MatrixWg fresh() const {
        MatrixWg g = *this;
        asm volatile("" : "+v"(g.lane));
        g.h = g.lane >> 5;
        g.n = g.lane & 31;
        return g;
    }

    __device__ __forceinline__ char *tri(int r, int k) const { return tri_unit(lds, r, k); }
    __device__ __forceinline__ void frag(Frag &f, int r, int k, int s) const { tri_frag(f, lds, r, k, s, lane); }

    // operands of unit rows r and r + 1 for unit column k, one branch for both
    __device__ __forceinline__ void block_frag(Frag *f, int r, int k, int s) const {
        if (k <= r) {
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int z = 0; z < kPlanes; ++z) f[q].p[z] = frag_rows(tri(r + q, k) + z * kPlane, lane, s);
        } else if (k > r + 1) {
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int z = 0; z < kPlanes; ++z) f[q].p[z] = frag_cols(tri(k, r + q) + z * kPlane, lane, s);
        } else {
#pragma unroll
            for (int z = 0; z < kPlanes; ++z) {
                f[0].p[z] = frag_cols(tri(k, r) + z * kPlane, lane, s);
                f[1].p[z] = frag_rows(tri(k, k) + z * kPlane, lane, s);
            }
        }
    }

    // A = X X^T, then P in its place.  A wave has NU units (ui[u], uj[u]), uj >= ui, of the
    // triangle, products of the unit rows r[0 .. NR) as which[u] says
    template <class W>
    __device__ __forceinline__ void gram_and_poly(const Scales &sc) const {
        const W t(wave);
        f32x16 acc[W::NU];
        Frag f[2][W::NR];
        auto zero = [&] {
#pragma unroll
            for (int u = 0; u < W::NU; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[u][e] = 0.0f;
        };
        auto products = [&](const Frag (&x)[W::NR]) {
#pragma unroll
            for (int u = 0; u < W::NU; ++u) mma(acc[u], x[W::left(u)], x[W::right(u)]);
        };
        const int K = v.C;
        auto copy = [&](int k) {  // unit column k of X: this wave's unit of it
            if (wave < v.R) {
                const char *src = scalar(v.x0 + ((int64_t)k * v.R + wave) * kUnit);
                const uint32_t dst = lds0 + (uint32_t)(k % STAGES) * STAGE + wave * kUnit;
#pragma unroll
                for (int e = 0; e < kUnit / 1024; ++e) copy_to_lds(src, (uint32_t)(e * 1024 + lane * 16), dst + e * 1024);
            }
        };
        zero();
#pragma unroll
        for (int k = 0; k < STAGES - 1; ++k)
            if (k < K) copy(k);
        // f[0] holds the first half of a unit column's operands, f[1] the second, each read while the
        // other's products run: at stage k the copies of stage k + 1 must have arrived, too
        auto staged = [&](Frag (&x)[W::NR], int k, int s) {
            const char *stage = lds + (k % STAGES) * STAGE;
#pragma unroll
            for (int q = 0; q < W::NR; ++q)
#pragma unroll
                for (int z = 0; z < kPlanes; ++z) x[q].p[z] = frag_cols(stage + t.row(q) * kUnit + z * kPlane, lane, s);
        };
        for (int k = 0; k < K; ++k) {
            if (k + 2 < K) wait_copies_and_barrier<kUnit / 1024>();
            else wait_copies_and_barrier<0>();
            if (k + STAGES - 1 < K) copy(k + STAGES - 1);
            if (t.any) {
                if (k == 0) staged(f[0], 0, 0);
                staged(f[1], k, 1);
                products(f[0]);
                staged(f[0], k + 1, 0);  // (past the end: not used)
                products(f[1]);
            }
        }
        wait_copies_and_barrier<0>();  // every wave is past the last stage
        auto mine = [&](int u) { return t.any && t.row(W::right(u)) < v.R; };
#pragma unroll
        for (int u = 0; u < W::NU; ++u)
            if (mine(u)) {
                half4 out[4][kPlanes];
                pack_unit(acc[u], sc.from_gram, out);
                store_unit(tri(t.row(W::right(u)), t.row(W::left(u))), out, n, h);
                __builtin_amdgcn_sched_barrier(0);
            }
        lds_barrier();
        half4 out[W::NU][4][kPlanes];
        if (t.any) {
            zero();
            auto operands = [&](Frag (&x)[W::NR], int k, int s) {
                if constexpr (W::BLOCKS) {
                    block_frag(&x[0], t.row(0), k, s);
                    block_frag(&x[2], t.row(2), k, s);
                } else {
#pragma unroll
                    for (int q = 0; q < W::NR; ++q) frag(x[q], t.row(q), k, s);
                }
            };
            operands(f[0], 0, 0);
            for (int k = 0; k < v.R; ++k) {
                operands(f[1], k, 1);
                products(f[0]);
                operands(f[0], k + 1 < v.R ? k + 1 : k, 0);
                products(f[1]);
            }
#pragma unroll
            for (int u = 0; u < W::NU; ++u)
                if (mine(u)) {
                    const int i = t.row(W::left(u)), j = t.row(W::right(u));
                    const char *at = tri(j, i);
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        half4 old[kPlanes];
#pragma unroll
                        for (int z = 0; z < kPlanes; ++z)
                            old[z] = *(const half4 *)(at + z * kPlane + chunk(n, g & 1, g >> 1) + h * 8);
                        float q[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) q[e] = acc[u][4 * g + e];
                        poly4(q, old, sc, i == j, n - 8 * g - 4 * h);
                        split4(q, 1.0f, out[u][g]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
        }
        lds_barrier();  // every wave has read A
#pragma unroll
        for (int u = 0; u < W::NU; ++u)
            if (mine(u)) store_unit(tri(t.row(W::right(u)), t.row(W::left(u))), out[u], n, h);
        lds_barrier();
    }

    // Shares of the triangle.  Eight unit rows: blocks of two of them, waves 2 to 7 the six blocks above the
    // diagonal (four units of two and two rows), 0 and 1 two of the four on it (three units of two rows each): 8 or 10
    // units per SIMD (wave % 4), the longer waves the older ones, which the SIMD prefers.  Four unit rows: one or two units of a row a wave, 2 or 3 per SIMD
    struct Off {
        static constexpr int NU = 4, NR = 4;
        static constexpr bool BLOCKS = true;
        int i, j;
        static constexpr bool any = true;
        __device__ __forceinline__ Off(int w) : i(w < 5 ? 0 : w < 7 ? 2 : 4), j(w < 5 ? 2 * w - 2 : w < 7 ? 2 * w - 6 : 6) {}
        __device__ __forceinline__ int row(int q) const { return q < 2 ? i + q : j + q - 2; }
        static constexpr int left(int u) { return u >> 1; }
        static constexpr int right(int u) { return 2 + (u & 1); }
    };
    struct Diagonal {
        static constexpr int NU = 6, NR = 4;
        static constexpr bool BLOCKS = true;
        int i, j;
        static constexpr bool any = true;
        __device__ __forceinline__ Diagonal(int w) : i(2 * w), j(2 * w + 4) {}
        __device__ __forceinline__ int row(int q) const { return q < 2 ? i + q : j + q - 2; }
        static constexpr int left(int u) { return 2 * (u / 3) + (u % 3 == 2); }
        static constexpr int right(int u) { return 2 * (u / 3) + (u % 3 > 0); }
    };
    struct Pair {  // units (i, j), (i, j + 1)
        static constexpr int NU = 2, NR = 3;
        static constexpr bool BLOCKS = false;
        int i, j;
        static constexpr bool any = true;
        __device__ __forceinline__ Pair(int w) : i(w < 2 ? 0 : w - 1), j(w == 0 ? 0 : 2) {}
        __device__ __forceinline__ int row(int q) const { return q == 0 ? i : j + q - 1; }
        static constexpr int left(int) { return 0; }
        static constexpr int right(int u) { return 1 + u; }
    };
    struct Single {  // unit (i, i), i = 1, 3; waves 6 and 7 none
        static constexpr int NU = 1, NR = 1;
        static constexpr bool BLOCKS = false;
        int i;
        bool any;
        __device__ __forceinline__ Single(int w) : i(w == 4 ? 1 : 3), any(w < 6) {}
        __device__ __forceinline__ int row(int) const { return i; }
        static constexpr int left(int) { return 0; }
        static constexpr int right(int) { return 0; }
    };

    __device__ __forceinline__ void make_p(const Scales &sc) const {
        if constexpr (RB == 8) {
            if (wave < 2) gram_and_poly<Diagonal>(sc);
            else gram_and_poly<Off>(sc);
        } else {
            if (wave < 4) gram_and_poly<Pair>(sc);  // (0, 0..1), (0, 2..3), (1, 2..3), (2, 2..3)
            else gram_and_poly<Single>(sc);
        }
    }

    // X = P X in place, or (LAST) the result; ALONG: lane = column of the iterate, otherwise its row.
    // (Two waves with four rows of two columns each read P half as often but X twice, and took a fifth longer.)
    template <bool LAST, bool ALONG>
    __device__ __forceinline__ void apply(float from_last) const {
        constexpr int RING = RB > 4 ? 3 : 2;  // units of the column, loaded ahead
        for (int j = wave; j < v.C; j += kWgWaves) {
            char *const col = v.x0 + (int64_t)j * v.R * kUnit;
            Frag x[RING][2];
            auto load = [&](int k) {
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int z = 0; z < kPlanes; ++z)
                        x[k % RING][s].p[z] = *(const half8 *)(col + k * kUnit + z * kPlane + chunk(n, h, s));
            };
            f32x16 acc[RB];
#pragma unroll
            for (int i = 0; i < RB; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][e] = 0.0f;
#pragma unroll
            for (int k = 0; k < RING - 1; ++k)
                if (k < v.R) load(k);
#pragma unroll
            for (int k = 0; k < RB; ++k) {
                if (k < v.R) {
                    if (k + RING - 1 < v.R) load(k + RING - 1);
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
#pragma unroll
                        for (int i = 0; i < RB; ++i) {
                            Frag f;  // (units past the matrix hold anything: those results are not used)
                            frag(f, i, k, s);
                            if constexpr (ALONG || !LAST) mma(acc[i], f, x[k % RING][s]);
                            else mma(acc[i], x[k % RING][s], f);
                        }
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < RB; ++i) {
                if (i < v.R) {
                    if constexpr (LAST) {
                        store_last<MUON, BF16>(v, p, from_last, acc[i], col + i * kUnit, i, j, h, n);
                    } else {
                        half4 out[4][kPlanes];
                        pack_unit(acc[i], p.from_apply, out);
                        store_unit(col + i * kUnit, out, n, h);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        wait_copies_and_barrier<0>();  // (the stores, too)
    }
};

template <int RB, bool MUON, bool BF16>
__device__ __forceinline__ void matrix_steps(const NsWork &w, const NsParams &p, int k, char *lds) {
    const View v = view_of(w, k);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    const MatrixWg<RB, MUON, BF16> g{p, v, lds, lds0, lane, wave, lane >> 5, lane & 31};
    const int level = w.levels[k];
    for (int step = 0;; ++step) {
        const Scales sc(p, level, step);
        g.fresh().make_p(sc);
        if (step + 1 < p.steps) {
            g.fresh().template apply<false, true>(sc.from_last);
        } else {
            if (v.tr) g.fresh().template apply<true, false>(sc.from_last);
            else g.fresh().template apply<true, true>(sc.from_last);
            return;
        }
    }
}

// n matrices from `first` on of up to RB unit rows; where RB is 8, those from n8 on have up to 4
template <int RB, bool MUON, bool BF16>
__global__ __launch_bounds__(64 * kWgWaves) __attribute__((amdgpu_waves_per_eu(RB == 8 ? 2 : 4))) void
ns_matrix_kernel(NsWork w, NsParams p, int first, int n8) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int k = blockIdx.x;
    if constexpr (RB == 8 && MUON) {
        if (k >= n8) {
            matrix_steps<4, MUON, BF16>(w, p, first + k, lds);
            return;
        }
    }
    matrix_steps<RB, MUON, BF16>(w, p, first + k, lds);
}

template <int T, int KIND, bool MUON, bool BF16>
hipError_t launch_product(NsWork w, const NsTile *tiles, int64_t grid, const NsParams &p, int k0, hipStream_t s) {
    w.tiles = tiles;
    const int r = w.uni.rows < w.uni.cols ? w.uni.rows : w.uni.cols, c = w.uni.rows + w.uni.cols - r;
    w.nti = (r + T - 1) / T;
    w.ntj = (c + T - 1) / T;
    auto launch = [&](auto stages) {
        constexpr int S = decltype(stages)::value;
        hipLaunchKernelGGL((ns_product_kernel<T, S, KIND, MUON, BF16>), dim3((unsigned)grid), dim3(256),
                           S * 2 * (T / 32) * kUnit, s, w, p, k0);
    };
    // S stages of copies.  Tiles of 128 x 128 take 32 KB a stage: with four of them a CU has one workgroup, with
    // two stages it has two, which is better once there are enough (96 matrices of 256 x 256 in 287 us
    // instead of 366; 8 of 2048 x 2048 as fast either way) and worse before (one of 2048 x 2048: 798 instead of 630)
    if (T == 128 && grid > 256) launch(Int<T == 128 ? 2 : 4>{});
    else launch(Int<4>{});
    return hipGetLastError();
}

template <int T, bool MUON, bool BF16>
hipError_t launch_step(const NsWork &w, const NsLists &l, const NsParams &p, int k0, hipStream_t s) {
    hipError_t e = launch_product<T, kGram, false, false>(w, l.gram, l.n_gram, p, k0, s);
    if (e != hipSuccess) return e;
    e = launch_product<T, kPoly, false, false>(w, l.gram, l.n_gram, p, k0, s);
    if (e != hipSuccess) return e;
    if (k0 + 1 == p.steps) return launch_product<T, kLast, MUON, BF16>(w, l.apply, l.n_apply, p, k0, s);
    return launch_product<T, kApply, false, false>(w, l.apply, l.n_apply, p, k0, s);
}

template <int T, bool MUON, bool BF16>
hipError_t launch_all(NsWork w, const NsLists &l, const NsParams &p, hipStream_t s) {
    if (l.n_small > 0) {
        hipLaunchKernelGGL((ns_small_kernel<MUON, BF16>), dim3((unsigned)l.n_small), dim3(64 * kSmallWaves), l.small_lds, s, w,
                           p, (int)l.first_small);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (l.n_x == 0) return hipSuccess;
    NsWork wx = w;
    const int r = w.uni.rows < w.uni.cols ? w.uni.rows : w.uni.cols, c = w.uni.rows + w.uni.cols - r;
    wx.tiles = l.x;
    wx.nti = (r + kNsBlock - 1) / kNsBlock;
    wx.ntj = (c + kNsBlock - 1) / kNsBlock;
    const dim3 gx((unsigned)l.n_x), b(256);
    hipLaunchKernelGGL((ns_norm_kernel<MUON, BF16>), gx, b, 0, s, wx, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((ns_scale_kernel<MUON, BF16>), gx, b, 0, s, wx, p);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    // Matrices of more than 128 rows, and in the same launch those of fewer: these fill the CUs that the last of the
    // longer ones leave idle (578 and 157 matrices: 1088 us instead of 909 + 241).  By themselves they take half
    // the LDS and registers, and a CU has two
    if (l.n_wg8 > 0) {
        hipLaunchKernelGGL((ns_matrix_kernel<8, MUON, BF16>), dim3((unsigned)(l.n_wg8 + l.n_wg4)), dim3(64 * kWgWaves),
                           (MatrixWg<8, MUON, BF16>::LDS), s, w, p, (int)l.first_wg8, (int)l.n_wg8);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    } else if (l.n_wg4 > 0) {
        hipLaunchKernelGGL((ns_matrix_kernel<4, MUON, BF16>), dim3((unsigned)l.n_wg4), dim3(64 * kWgWaves),
                           (MatrixWg<4, MUON, BF16>::LDS), s, w, p, (int)l.first_wg4, 0);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    for (int k = 0; k < p.steps && l.n_apply > 0; ++k) {
        e = launch_step<T, MUON, BF16>(w, l, p, k, s);
        if (e != hipSuccess) return e;
    }
    if constexpr (MUON) {
        hipLaunchKernelGGL(ns_update_kernel, gx, b, 0, s, wx, p, p.steps & 1);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

int64_t ns_matrix_bytes(int64_t rows, int64_t cols) {
    const int64_t r = rows < cols ? rows : cols, c = rows + cols - r;
    const int64_t R = (r + 31) / 32, C = (c + 31) / 32;
    return 2 * (R * C + R * R) * kUnit;
}

int64_t ns_small_bytes(int64_t rows, int64_t cols) {
    const int r = (int)(rows < cols ? rows : cols), c = (int)(rows + cols - r);
    const int R = units(r), C = units(c);
    const bool fits = fits_small(R, C);
    return fits ? (int64_t)(R * C + R * (R + 1) / 2) * kUnit : 0;
}

int ns_matrix_rows(int64_t rows, int64_t cols) {
    const int R = units((int)(rows < cols ? rows : cols));
    return R <= 4 ? 4 : R <= 8 ? 8 : 0;
}

int64_t ns_matrix_wg_bytes(int64_t rows, int64_t cols) {
    const int64_t r = rows < cols ? rows : cols, c = rows + cols - r;
    return (r + 31) / 32 * ((c + 31) / 32) * kUnit;
}

// A workgroup takes as long for its matrix as tiles on all CUs for 55 (256 x 256) to 92 (256 x 1024) of them.  The
// rule has one number between: wide matrices in calls of 72 to 90 would be up to a quarter sooner by tiles.  (fp32, by tiles and by workgroups: 48 of 256 x 256 176 and 200 us, 64 238 and 204, 96 287 and 214; 72 of
// 256 x 512 312 and 336, 96 404 and 347; 72 of 256 x 1024 481 and 593, 96 645 and 612, 128 847 and 651; 72 of
// 128 x 512 143 and 123, of 128 x 1024 211 and 218)
bool ns_by_matrix(double total, double largest) { return total >= 72.0 * largest; }

// 128 x 128 tiles read each staged unit twice as often, but the Gram matrix's triangle has few of
// them: below about 120, tiles of a quarter the size do the work sooner (fp32, small and large tiles: 1 matrix
// of 1024 x 4096, 36 large ones, 404 and 527 us; 1 of 1792 x 1792, 105, 504 and 505; 12 of 512 x 512, 120, 262
// and 237; 1 of 2048 x 2048, 136, 765 and 631; 16 of 512 x 2048, 160, 682 and 576)
int ns_tile(int64_t gram128) { return gram128 >= 120 ? 128 : 64; }

hipError_t launch_ns(const NsWork &w, const NsLists &l, const NsParams &p, bool muon, bool bf16, hipStream_t s) {
    if (l.tile == 128)
        return muon ? launch_all<128, true, false>(w, l, p, s)
                    : bf16 ? launch_all<128, false, true>(w, l, p, s) : launch_all<128, false, false>(w, l, p, s);
    return muon ? launch_all<64, true, false>(w, l, p, s)
                : bf16 ? launch_all<64, false, true>(w, l, p, s) : launch_all<64, false, false>(w, l, p, s);
}

}  // namespace evo

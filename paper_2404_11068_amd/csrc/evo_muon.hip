// evo_muon.hip -- Newton-Schulz orthogonalisation and the Muon step, gfx950.
//
//   X = x / max(|x|_F, eps);  steps times:  A = X X^T,  P = a I + b A + c A A,  X = P X
//
// Precision.  A direction that X hardly has grows by up to a^steps = 485, and so do
// the roundings of the iterate.  fp32 matrices therefore keep every iterate
// as a pair of fp16 (value = hi + lo, 22 bits) and form each product as hi hi + hi lo + lo hi
// on the fp16 matrix instructions with fp32 accumulation: the error of fp32
// arithmetic (1e-6 .. 1e-5 of the result over five steps, low-rank inputs
// too) at a third of the fp16 rate, which is five times the fp32 matrix rate.
// bf16 matrices take one fp16 plane: an iterate rounded to 2^-11 costs 2e-3 of
// the result, about its own rounding to bf16 (with bf16 iterates it would be
// 1e-2, and all of it for low-rank inputs).  X and A are stored times 2^10:
// their entries stay below 64 (coefficients that could take them further
// are refused), and those near 1 / sqrt(m n) stay clear of fp16's subnormals.
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

constexpr float kScale = 1024.0f;        // X and A are stored times this, P as it is: P X needs no scaling
constexpr float kUnscale = 1.0f / 1024.0f;
constexpr int kPlane = 2048;                       // bytes of a unit's plane

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

template <int PL>
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
    const int64_t unit = PL * kPlane, nx = (int64_t)v.R * v.C * unit;
    v.x0 = w.ws + v.m.off;
    v.x1 = v.x0 + nx;
    v.A = v.x1 + nx;
    v.P = v.A + (int64_t)v.R * v.R * unit;
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
    if (w.n_mats >= 8) {
        const int q = k >> 3;
        mat = (k & 7) + 8 * (q / per);
        e = q % per;
        if (mat >= w.n_mats) mat = -1;
    } else {
        mat = k / per;
        e = k % per;
    }
    if (!GRAM) return NsTile{mat, e / w.ntj, e % w.ntj};
    int ti = 0;  // rows of nti, nti - 1, ... tiles
    while (e >= w.nti - ti) {
        e -= w.nti - ti;
        ++ti;
    }
    return NsTile{mat, ti, ti + e};
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

// Four values f v as fp16, or as two fp16 each that sum up to them within 22 bits.  Conversions
// two at a time, the remainder in one mixed fused multiply-add: 3 operations per value
typedef float float2v __attribute__((ext_vector_type(2)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
template <int PL>
__device__ __forceinline__ void split4(const float (&v)[4], float f, half4 (&p)[PL]) {
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
        const half2v hi = __builtin_convertvector((float2v{v[e] * f, v[e + 1] * f}), half2v);
        p[0][e] = hi.x;
        p[0][e + 1] = hi.y;
        if constexpr (PL == 2) {
            const half2v lo =
                __builtin_convertvector((float2v{fmaf(v[e], f, -(float)hi.x), fmaf(v[e + 1], f, -(float)hi.y)}), half2v);
            p[1][e] = lo.x;
            p[1][e + 1] = lo.y;
        }
    }
}

template <int PL> struct Frag { half8 p[PL]; };

template <int PL>
__device__ __forceinline__ void mma(f32x16 &acc, const Frag<PL> &a, const Frag<PL> &b) {
    if constexpr (PL == 2) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a.p[1], b.p[0], acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a.p[0], b.p[1], acc, 0, 0, 0);
    }
    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a.p[0], b.p[0], acc, 0, 0, 0);
}

// ---- norm and scaling: a thread owns 4 x 4 entries of a 64 x 64 tile

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
template <int PL, bool TRANSPOSED>
__device__ __forceinline__ void pack_block(const float (&u)[4][4], const View &v, int row0, int col0, double f) {
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
        half4 hh[PL];
        split4<PL>(q, 1.0f, hh);
        char *unit = v.x0 + ((int64_t)(i >> 5) * cols + (j >> 5)) * (PL * kPlane);
        const int k = j & 31, at = chunk(i & 31, (k >> 3) & 1, k >> 4) + (k & 4) * 2;
#pragma unroll
        for (int z = 0; z < PL; ++z) *(half4 *)(unit + z * kPlane + at) = hh[z];
    }
}

// momentum, and the sum of squares of each tile (fp64: no overflow or underflow of fp32 squares)
template <bool MUON, bool BF16, int PL>
__global__ __launch_bounds__(256) void ns_norm_kernel(NsWork w, NsParams p) {
    __shared__ double red[4];
    const NsTile t = tile_of<false>(w, blockIdx.x);
    if (t.mat < 0) return;
    const View v = view_of<PL>(w, t.mat);
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
template <bool MUON, bool BF16, int PL>
__global__ __launch_bounds__(256) void ns_scale_kernel(NsWork w, NsParams p) {
    __shared__ double red[4];
    const NsTile t = tile_of<false>(w, blockIdx.x);
    if (t.mat < 0) return;
    const View v = view_of<PL>(w, t.mat);
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
    const double f = (double)kScale / (norm < p.eps ? p.eps : norm);
    if (v.xt) pack_block<PL, true>(u, v, row0, col0, f);
    else pack_block<PL, false>(u, v, row0, col0, f);
}

// p = decay p - lr scale O, w = sd w + om_sd p, with O as the last product left it in buffer `odd` of X:
// 32 x 32 floats in the place of each unit, by memory rows
__global__ __launch_bounds__(256) void ns_update_kernel(NsWork w, NsParams p, int odd) {
    const NsTile t = tile_of<false>(w, blockIdx.x);
    if (t.mat < 0) return;
    const View v = view_of<2>(w, t.mat);
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

// entries of P = a I + b A + c A A from those of the product (scale 2^20) and of A (2^10);
// diagonal: which of the four lies on it, if any
template <int PL>
__device__ __forceinline__ void poly4(float (&q)[4], const half4 (&old)[PL], const NsParams &p, int diagonal) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float o = (float)old[0][e];
        if constexpr (PL == 2) o += (float)old[1][e];
        q[e] = fmaf(p.c * (kUnscale * kUnscale), q[e], p.b * kUnscale * o);
        q[e] += e == diagonal ? p.a : 0.0f;
    }
}

// acc (a unit: lane = row, registers = columns) times f as packed quarters
template <int PL>
__device__ __forceinline__ void pack_unit(const f32x16 &acc, float f, half4 (&out)[4][PL]) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        float q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) q[e] = acc[4 * g + e];
        split4<PL>(q, f, out[g]);
    }
}
template <int PL>
__device__ __forceinline__ void store_unit(char *unit, const half4 (&out)[4][PL], int n, int h) {
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int z = 0; z < PL; ++z) *(half4 *)(unit + z * kPlane + chunk(n, g & 1, g >> 1) + h * 8) = out[g][z];
}

// One unit's entries of the result, the lanes along the memory rows; before() loads what the update
// needs.  An address is a scalar row plus the lane's part, which is the same in every row
template <bool MUON, bool BF16>
struct Result {
    float p[16], w[16];

    // f(entry, offset of its row in elements, the lane's) for the entries inside the matrix
    template <class F>
    __device__ __forceinline__ static void each(const View &v, int iu, int ju, int h, int n, F f) {
        int row0 = __builtin_amdgcn_readfirstlane((v.tr ? ju : iu) * 32), col0 = (v.tr ? iu : ju) * 32;
        asm volatile("" : "+s"(row0));  // (or a loop over units has all of its rows' addresses made before it)
        asm volatile("" : "+v"(h), "+v"(n));
        const uint32_t lane = (uint32_t)(4 * h) * (uint32_t)v.m.cols + (uint32_t)n;
        const bool in = col0 + n < v.m.cols;
        const int left = v.m.rows - row0 - 4 * h;
        const int64_t first = (int64_t)row0 * v.m.cols + col0;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int r = 8 * (e >> 2) + (e & 3);
            if (in && r < left) f(e, first + (int64_t)r * v.m.cols, lane);
        }
    }
    __device__ __forceinline__ void before(const View &v, int iu, int ju, int h, int n) {
        if constexpr (MUON) {
            const float *const prm = (const float *)v.m.out, *const swa = v.m.swa;
            each(v, iu, ju, h, n, [&](int e, int64_t row, uint32_t lane) { p[e] = (prm + row)[lane]; });
            if (swa) each(v, iu, ju, h, n, [&](int e, int64_t row, uint32_t lane) { w[e] = (swa + row)[lane]; });
        }
    }
    __device__ __forceinline__ void store(const View &v, const NsParams &P, const f32x16 &acc, int iu, int ju, int h, int n) {
        if constexpr (MUON) {
            float *const prm = (float *)v.m.out, *const swa = v.m.swa;
            const float f = -P.lr * v.m.scale * kUnscale;
            each(v, iu, ju, h, n, [&](int e, int64_t row, uint32_t lane) {
                p[e] = fmaf(f, acc[e], P.decay * p[e]);
                (prm + row)[lane] = p[e];
            });
            if (swa)
                each(v, iu, ju, h, n,
                     [&](int e, int64_t row, uint32_t lane) { (swa + row)[lane] = fmaf(P.sd, w[e], P.om_sd * p[e]); });
        } else {
            each(v, iu, ju, h, n, [&](int e, int64_t row, uint32_t lane) {
                if constexpr (BF16) ((uint16_t *)v.m.out + row)[lane] = f2bf(acc[e] * kUnscale);
                else ((float *)v.m.out + row)[lane] = acc[e] * kUnscale;
            });
        }
    }
};

// the last product's unit: for Muon as floats by memory rows in the unit's place, for ns_update_kernel,
// otherwise the result itself
template <bool MUON, bool BF16>
__device__ __forceinline__ void store_last(const View &v, const NsParams &p, const f32x16 &acc, char *unit, int iu, int ju, int h,
                                           int n) {
    if constexpr (MUON) {
        float *const o = (float *)unit + 128 * h + n;
#pragma unroll
        for (int e = 0; e < 16; ++e) o[(8 * (e >> 2) + (e & 3)) * 32] = acc[e] * kUnscale;
    } else {
        Result<MUON, BF16> res;
        res.store(v, p, acc, iu, ju, h, n);
    }
}

// ---- products
//
// A workgroup of 4 waves forms a T x T tile, a wave a quarter of it, from units staged
// in LDS, one unit column (32 contraction entries) per stage, copied by
// global_load_lds 16 bytes a lane, S - 1 stages ahead: the copies are counted
// by hand (vmcnt), one barrier per stage.

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

template <int T, int PL, int S, int KIND, bool MUON, bool BF16>
__global__ __launch_bounds__(256) void ns_product_kernel(NsWork w, NsParams p, int odd) {
    constexpr int U = T / 64;             // units of a wave's tile in each direction
    constexpr int N = T / 32;             // units of the workgroup's
    constexpr int UNIT = PL * kPlane;
    constexpr int STAGE = 2 * N * UNIT;
    constexpr int COPIES = U * UNIT / 1024;  // of a wave and stage
    constexpr bool SQUARE = KIND == kGram || KIND == kPoly;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const NsTile t = tile_of<SQUARE>(w, blockIdx.x);
    if (t.mat < 0) return;
    const View v = view_of<PL>(w, t.mat);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = wave >> 1, wc = wave & 1, h = lane >> 5, n = lane & 31;
    const char *x = KIND == kPoly ? v.A : odd ? v.x1 : v.x0;
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
            src[q] = x + (int64_t)row * K * UNIT;
            step = UNIT;
        } else if (op == 0) {
            const int row = first < v.R ? first : v.R - 1;
            src[q] = v.P + (int64_t)row * v.R * UNIT;
            step = UNIT;
        } else {
            const int col = first < v.C ? first : v.C - 1;
            src[q] = x + (int64_t)col * UNIT;
            step = (int64_t)v.C * UNIT;
        }
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    auto copy_stage = [&](int k) {
        const uint32_t dst = lds0 + (uint32_t)(k % S) * STAGE + (uint32_t)(wave * U) * UNIT;
#pragma unroll
        for (int q = 0; q < U; ++q)
#pragma unroll
            for (int e = 0; e < UNIT / 1024; ++e)
                copy_to_lds(scalar(src[q] + k * step), (uint32_t)(e * 1024 + lane * 16), dst + q * UNIT + e * 1024);
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
    auto products = [&](auto swapped) {
#pragma unroll
        for (int k = 0; k < S - 1; ++k)
            if (k < K) copy_stage(k);
        for (int k = 0; k < K; ++k) {
            // stage k has arrived when at most the later ones' copies are outstanding
            if (k + S - 2 < K) wait_copies_and_barrier<(S - 2) * COPIES>();
            else wait_copies_and_barrier<0>();
            if (k + S - 1 < K) copy_stage(k + S - 1);
            const char *s0 = lds + (k % S) * STAGE + wr * U * UNIT, *s1 = lds + (k % S) * STAGE + (N + wc * U) * UNIT;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                Frag<PL> f0[U], f1[U];
#pragma unroll
                for (int a = 0; a < U; ++a)
#pragma unroll
                    for (int q = 0; q < PL; ++q) {
                        f0[a].p[q] = frag_rows(s0 + a * UNIT + q * kPlane, lane, s);
                        f1[a].p[q] = SQUARE ? frag_rows(s1 + a * UNIT + q * kPlane, lane, s)
                                            : frag_cols(s1 + a * UNIT + q * kPlane, lane, s);
                    }
#pragma unroll
                for (int a = 0; a < U; ++a)
#pragma unroll
                    for (int b = 0; b < U; ++b) {
                        if constexpr (decltype(swapped)::value) mma<PL>(acc[a][b], f1[b], f0[a]);
                        else mma<PL>(acc[a][b], f0[a], f1[b]);
                    }
            }
        }
    };
    const int i0 = t.ti * N + wr * U, j0 = t.tj * N + wc * U;  // this wave's first units
    if constexpr (SQUARE) {
        // lane = column: stored as row `column` of the symmetric matrix's unit (j, i)
        products(No{});
        __syncthreads();  // the stages become scratch
        char *const scratch = lds + wave * UNIT;
        char *const dst = KIND == kPoly ? v.P : v.A;
#pragma unroll
        for (int a = 0; a < U; ++a)
#pragma unroll
            for (int b = 0; b < U; ++b) {
                const int i = i0 + a, j = j0 + b;
                if (i >= v.R || j >= v.R) continue;  // wave-uniform
                const int64_t at = ((int64_t)j * v.R + i) * UNIT;
                half4 out[4][PL];
#pragma unroll
                for (int g = 0; g < 4; ++g) {  // rows 8 g + 4 h .. + 3 of the tile
                    const int pos = chunk(n, g & 1, g >> 1) + h * 8;
                    float q[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) q[e] = acc[a][b][4 * g + e];
                    if constexpr (KIND == kPoly) {
                        half4 old[PL];
#pragma unroll
                        for (int z = 0; z < PL; ++z) old[z] = *(const half4 *)(v.A + at + z * kPlane + pos);
                        poly4<PL>(q, old, p, i == j ? n - 8 * g - 4 * h : -1);
                    }
                    split4<PL>(q, KIND == kPoly ? 1.0f : kUnscale, out[g]);
#pragma unroll
                    for (int z = 0; z < PL; ++z) *(half4 *)(dst + at + z * kPlane + pos) = out[g][z];
                }
                if (t.ti != t.tj) {  // the mirrored unit (i, j), through LDS by columns
#pragma unroll
                    for (int g = 0; g < 4; ++g)
#pragma unroll
                        for (int z = 0; z < PL; ++z)
                            *(half4 *)(scratch + z * kPlane + chunk(n, g & 1, g >> 1) + h * 8) = out[g][z];
                    __builtin_amdgcn_wave_barrier();
                    const int64_t mirrored = ((int64_t)i * v.R + j) * UNIT;
#pragma unroll
                    for (int z = 0; z < PL; ++z)
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
                char *unit = dst + ((int64_t)i * v.C + j) * UNIT;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    float q[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) q[e] = acc[a][b][4 * g + e];
                    half4 out[PL];
                    split4<PL>(q, 1.0f, out);
#pragma unroll
                    for (int z = 0; z < PL; ++z)
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
                store_last<MUON, BF16>(v, p, acc[a][b], (odd ? v.x0 : v.x1) + ((int64_t)i * v.C + j) * UNIT, i, j, h, n);
            }
    }
}

// ---- matrices that fit into LDS: everything in one workgroup
//
// X and A (later P in its place) lie in LDS as units, R C + R R <= 39 of them
// in pairs (128 x 160 entries, 64 x 544, 32 x 1184) and at most kSmallUnits of
// X; a product's results wait in registers until every wave has read its
// operands.  One launch does the norm, the steps and the update: memory sees
// each entry once.  A wave takes units of the upper triangle (10 of 16 at 128
// x 128) or pairs of units of X in turn.

constexpr int kSmallUnits = 40;
constexpr int kSmallLds = 39 * 2 * kPlane;
constexpr int kSmallWaves = 8;

template <int PL>
__host__ __device__ inline bool fits_small(int R, int C) {
    return R * ((C + 1) / 2) <= 3 * kSmallWaves && R * C <= kSmallUnits && (R * C + R * R) * PL * kPlane <= kSmallLds;
}

template <bool MUON, bool BF16, int PL>
__global__ __launch_bounds__(64 * kSmallWaves) void ns_small_kernel(NsWork w, NsParams p, int first) {
    constexpr int UNIT = PL * kPlane, THREADS = 64 * kSmallWaves;
    constexpr int BLOCKS = kSmallUnits * 64 / THREADS;  // 4 x 4 blocks of a thread
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    __shared__ double red[kSmallWaves];
    const View v = view_of<PL>(w, first + blockIdx.x);
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, n = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int R = v.R, C = v.C;
    char *const X = lds, *const A = lds + R * C * UNIT;

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
        const double norm = sqrt(s), f = (double)kScale / (norm < p.eps ? p.eps : norm);
#pragma unroll
        for (int q = 0; q < BLOCKS; ++q) {
            const int k = q * THREADS + tid;
            if (k < blocks) {
                const int br = k / per_row, bc = k - br * per_row;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int i = v.tr ? bc * 4 + x : br * 4 + x, j = v.tr ? br * 4 : bc * 4;
                    float y4[4];
#pragma unroll
                    for (int y = 0; y < 4; ++y) y4[y] = (float)((double)(v.tr ? u[q][y][x] : u[q][x][y]) * f);
                    half4 hh[PL];
                    split4<PL>(y4, 1.0f, hh);
                    const int kk = j & 31, at = chunk(i & 31, (kk >> 3) & 1, kk >> 4) + (kk & 4) * 2;
                    char *unit = X + ((i >> 5) * C + (j >> 5)) * UNIT;
#pragma unroll
                    for (int z = 0; z < PL; ++z) *(half4 *)(unit + z * kPlane + at) = hh[z];
                }
            }
        }
        __syncthreads();
    }

    // rows of units `a` times rows `b` of M (K units each), summed into acc by parts
    auto rows_by_rows = [&](const char *M, int K, int a, int b) {
        f32x16 acc[PL == 2 ? 3 : 1];
#pragma unroll
        for (auto &x : acc)
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = 0.0f;
        for (int k = 0; k < K; ++k) {
            const char *ua = M + (a * K + k) * UNIT, *ub = M + (b * K + k) * UNIT;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const half8 fa = frag_rows(ua, lane, s), fb = frag_rows(ub, lane, s);
                acc[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa, fb, acc[0], 0, 0, 0);
                if constexpr (PL == 2) {
                    const half8 la = frag_rows(ua + kPlane, lane, s), lb = frag_rows(ub + kPlane, lane, s);
                    acc[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa, lb, acc[1], 0, 0, 0);
                    acc[2] = __builtin_amdgcn_mfma_f32_32x32x16_f16(la, fb, acc[2], 0, 0, 0);
                }
            }
        }
        if constexpr (PL == 2) acc[0] += acc[1] + acc[2];
        return acc[0];
    };
    const int tri = R * (R + 1) / 2;
    auto unit_of = [&](int t, int &a, int &b) {  // t-th unit of the upper triangle
        a = 0;
        while (t >= R - a) {
            t -= R - a;
            ++a;
        }
        b = a + t;
    };
    // a unit of a symmetric matrix, lane = row b, registers = columns a, and its mirror
    auto store_pair = [&](const half4 (&out)[4][PL], int a, int b) {
        char *const at = A + (b * R + a) * UNIT;
        store_unit<PL>(at, out, n, h);
        if (a == b) return;
        __builtin_amdgcn_wave_barrier();
        char *const mirror = A + (a * R + b) * UNIT;
#pragma unroll
        for (int z = 0; z < PL; ++z)
#pragma unroll
            for (int s = 0; s < 2; ++s) *(half8 *)(mirror + z * kPlane + chunk(n, h, s)) = frag_cols(at + z * kPlane, lane, s);
    };

    constexpr int TRI = PL == 2 ? 2 : 3;  // units of a wave: R <= 4 in pairs of planes, R <= 6 in one
    constexpr int PAIRS = 3;              // pairs of a wave: R ceil(C / 2) <= 20 for R C <= 40, R <= C (checked below)
    const int half_c = (C + 1) / 2, pairs = R * half_c;
    // pair t of units of P X: row a, columns b0 and b1 (b0 again where there is one)
    auto pair_of = [&](int t, int &a, int &b0, int &b1) {
        a = t / half_c;
        b0 = (t - a * half_c) * 2;
        b1 = b0 + 1 < C ? b0 + 1 : b0;
    };
    // along: lane = column of the iterate, otherwise its row
    auto product = [&](f32x16 (&acc)[2], int a, int b0, int b1, bool along) {
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[y][e] = 0.0f;
        for (int k = 0; k < R; ++k) {
            const char *up = A + (a * R + k) * UNIT, *u0 = X + (k * C + b0) * UNIT, *u1 = X + (k * C + b1) * UNIT;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                Frag<PL> fp, f0, f1;
#pragma unroll
                for (int z = 0; z < PL; ++z) {
                    fp.p[z] = frag_rows(up + z * kPlane, lane, s);
                    f0.p[z] = frag_cols(u0 + z * kPlane, lane, s);
                    f1.p[z] = frag_cols(u1 + z * kPlane, lane, s);
                }
                if (along) {
                    mma<PL>(acc[0], fp, f0);
                    mma<PL>(acc[1], fp, f1);
                } else {
                    mma<PL>(acc[0], f0, fp);
                    mma<PL>(acc[1], f1, fp);
                }
            }
        }
    };
    for (int step = 0; step < p.steps; ++step) {
        for (int t = wave; t < tri; t += kSmallWaves) {
            int a, b;
            unit_of(t, a, b);
            half4 out[4][PL];
            pack_unit<PL>(rows_by_rows(X, C, a, b), kUnscale, out);
            store_pair(out, a, b);
        }
        __syncthreads();
        {
            half4 out[TRI][4][PL];
#pragma unroll
            for (int x = 0; x < TRI; ++x) {
                const int t = wave + x * kSmallWaves;
                if (t < tri) {
                    int a, b;
                    unit_of(t, a, b);
                    const f32x16 acc = rows_by_rows(A, R, a, b);
                    const char *at = A + (b * R + a) * UNIT;
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        float q[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) q[e] = acc[4 * g + e];
                        half4 old[PL];
#pragma unroll
                        for (int z = 0; z < PL; ++z)
                            old[z] = *(const half4 *)(at + z * kPlane + chunk(n, g & 1, g >> 1) + h * 8);
                        poly4<PL>(q, old, p, a == b ? n - 8 * g - 4 * h : -1);
                        split4<PL>(q, 1.0f, out[x][g]);
                    }
                }
            }
            __syncthreads();
#pragma unroll
            for (int x = 0; x < TRI; ++x) {
                const int t = wave + x * kSmallWaves;
                if (t < tri) {
                    int a, b;
                    unit_of(t, a, b);
                    store_pair(out[x], a, b);
                }
            }
            __syncthreads();
        }
        if (step + 1 == p.steps) break;
        half4 out[PAIRS][2][4][PL];
#pragma unroll
        for (int x = 0; x < PAIRS; ++x) {
            const int t = wave + x * kSmallWaves;
            if (t < pairs) {
                int a, b0, b1;
                pair_of(t, a, b0, b1);
                f32x16 acc[2];
                product(acc, a, b0, b1, false);
#pragma unroll
                for (int y = 0; y < 2; ++y) pack_unit<PL>(acc[y], 1.0f, out[x][y]);
            }
        }
        __syncthreads();
#pragma unroll
        for (int x = 0; x < PAIRS; ++x) {
            const int t = wave + x * kSmallWaves;
            if (t < pairs) {
                int a, b0, b1;
                pair_of(t, a, b0, b1);
                store_unit<PL>(X + (a * C + b0) * UNIT, out[x][0], n, h);
                if (b1 != b0) store_unit<PL>(X + (a * C + b1) * UNIT, out[x][1], n, h);
            }
        }
        __syncthreads();
    }
    // the last step: the lanes go along the matrix's memory rows
    for (int t = wave; t < pairs; t += kSmallWaves) {
        int a, b0, b1;
        pair_of(t, a, b0, b1);
        Result<MUON, BF16> r0, r1;
        r0.before(v, a, b0, h, n);
        r1.before(v, a, b1, h, n);
        f32x16 acc[2];
        product(acc, a, b0, b1, !v.tr);
        r0.store(v, p, acc[0], a, b0, h, n);
        if (b1 != b0) r1.store(v, p, acc[1], a, b1, h, n);
    }
}

// ---- matrices of up to 256 rows, one workgroup each
//
// A workgroup of eight waves takes a matrix through all steps.  (The norm, the
// scaling and Muon's update are passes of their own: a CU by itself keeps too little in flight for them.)  The Gram
// matrix and then P lie in LDS, as the units of one triangle (36 of them, 144
// KB, for 256 rows in pairs of planes): an operand of the other triangle is the mirrored
// unit read by columns.  X lies in the workspace, transposed, so that the
// fragments of P X come straight from memory, 1 KB a load: each wave takes unit
// columns of its own and writes the result in their place, without a barrier.  Memory
// then sees X read twice and written once per step; with A and P in the workspace, too,
// 240 matrices of 256 x 256 moved 2.7 GB at 6.4 TB/s and took 430 us.
// A call with too few matrices for the CUs is done sooner by the tiles above.

constexpr int kWgWaves = 8;

template <int RB, int PL, bool MUON, bool BF16>
struct MatrixWg {
    static constexpr int UNIT = PL * kPlane;
    static constexpr int WA = RB == 8 ? 2 : 1, WB = RB == 8 ? 4 : 2;  // units of a wave's tile of the symmetric products
    static constexpr int STAGE = RB * UNIT, STAGES = 4;               // of the Gram matrix: a unit column of X
    static constexpr int TRI = RB * (RB + 1) / 2;
    static constexpr int LDS = TRI * UNIT > STAGES * STAGE ? TRI * UNIT : STAGES * STAGE;

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

    // unit (r, k), r >= k, of the triangle in LDS: row r, contraction k
    __device__ __forceinline__ char *tri(int r, int k) const { return lds + (r * (r + 1) / 2 + k) * UNIT; }
    // rows of unit row r, contraction over unit column k, of the symmetric matrix in LDS
    __device__ __forceinline__ void frag(Frag<PL> &f, int r, int k, int s) const {
        if (r >= k) {
            const char *u = tri(r, k);
#pragma unroll
            for (int z = 0; z < PL; ++z) f.p[z] = frag_rows(u + z * kPlane, lane, s);
        } else {
            const char *u = tri(k, r);
#pragma unroll
            for (int z = 0; z < PL; ++z) f.p[z] = frag_cols(u + z * kPlane, lane, s);
        }
    }

    // The wave's units (i0 + a, j0 + b), b >= a + D, of A = X X^T, then of P in its place
    template <int D>
    __device__ __forceinline__ void gram_and_poly(int i0, int j0) const {
        f32x16 acc[WA][WB];
        auto zero = [&] {
#pragma unroll
            for (int a = 0; a < WA; ++a)
#pragma unroll
                for (int b = 0; b < WB; ++b)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[a][b][e] = 0.0f;
        };
        auto products = [&](const Frag<PL> (&fa)[WA], const Frag<PL> (&fb)[WB]) {
#pragma unroll
            for (int a = 0; a < WA; ++a)
#pragma unroll
                for (int b = 0; b < WB; ++b)
                    if (b >= a + D) mma<PL>(acc[a][b], fa[a], fb[b]);
        };
        constexpr int B0 = D > 0 ? D : 0;
        const int K = v.C;
        auto copy = [&](int k) {  // unit column k of X: this wave's unit of it
            if (wave < v.R) {
                const char *src = scalar(v.x0 + ((int64_t)k * v.R + wave) * UNIT);
                const uint32_t dst = lds0 + (uint32_t)(k % STAGES) * STAGE + wave * UNIT;
#pragma unroll
                for (int e = 0; e < UNIT / 1024; ++e) copy_to_lds(src, (uint32_t)(e * 1024 + lane * 16), dst + e * 1024);
            }
        };
        zero();
#pragma unroll
        for (int k = 0; k < STAGES - 1; ++k)
            if (k < K) copy(k);
        for (int k = 0; k < K; ++k) {
            if (k + STAGES - 2 < K) wait_copies_and_barrier<(STAGES - 2) * (UNIT / 1024)>();
            else wait_copies_and_barrier<0>();
            if (k + STAGES - 1 < K) copy(k + STAGES - 1);
            const char *stage = lds + (k % STAGES) * STAGE;
            if constexpr (D < WB) {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    Frag<PL> fa[WA], fb[WB];
#pragma unroll
                    for (int a = 0; a < WA; ++a)
#pragma unroll
                        for (int z = 0; z < PL; ++z) fa[a].p[z] = frag_cols(stage + (i0 + a) * UNIT + z * kPlane, lane, s);
#pragma unroll
                    for (int b = B0; b < WB; ++b)
#pragma unroll
                        for (int z = 0; z < PL; ++z) fb[b].p[z] = frag_cols(stage + (j0 + b) * UNIT + z * kPlane, lane, s);
                    products(fa, fb);
                    __builtin_amdgcn_sched_barrier(0);  // (both halves' operands at once do not fit the registers)
                }
            }
        }
        wait_copies_and_barrier<0>();  // every wave is past the last stage
        if constexpr (D < WB) {
#pragma unroll
            for (int a = 0; a < WA; ++a)
#pragma unroll
                for (int b = 0; b < WB; ++b)
                    if (b >= a + D && i0 + a < v.R && j0 + b < v.R) {
                        half4 out[4][PL];
                        pack_unit<PL>(acc[a][b], kUnscale, out);
                        store_unit<PL>(tri(j0 + b, i0 + a), out, n, h);
                        __builtin_amdgcn_sched_barrier(0);
                    }
        }
        wait_copies_and_barrier<0>();
        half4 out[WA][WB][4][PL];
        if constexpr (D < WB) {
            zero();
            for (int k = 0; k < v.R; ++k) {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    Frag<PL> fa[WA], fb[WB];
#pragma unroll
                    for (int a = 0; a < WA; ++a) frag(fa[a], i0 + a, k, s);
#pragma unroll
                    for (int b = B0; b < WB; ++b) frag(fb[b], j0 + b, k, s);
                    products(fa, fb);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
#pragma unroll
            for (int a = 0; a < WA; ++a)
#pragma unroll
                for (int b = 0; b < WB; ++b)
                    if (b >= a + D && i0 + a < v.R && j0 + b < v.R) {
                        const char *at = tri(j0 + b, i0 + a);
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            half4 old[PL];
#pragma unroll
                            for (int z = 0; z < PL; ++z)
                                old[z] = *(const half4 *)(at + z * kPlane + chunk(n, g & 1, g >> 1) + h * 8);
                            float q[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) q[e] = acc[a][b][4 * g + e];
                            poly4<PL>(q, old, p, i0 + a == j0 + b ? n - 8 * g - 4 * h : -1);
                            split4<PL>(q, 1.0f, out[a][b][g]);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
        }
        wait_copies_and_barrier<0>();  // every wave has read A
        if constexpr (D < WB) {
#pragma unroll
            for (int a = 0; a < WA; ++a)
#pragma unroll
                for (int b = 0; b < WB; ++b)
                    if (b >= a + D && i0 + a < v.R && j0 + b < v.R) store_unit<PL>(tri(j0 + b, i0 + a), out[a][b], n, h);
        }
        wait_copies_and_barrier<0>();
    }

    __device__ __forceinline__ void make_p() const {
        // unit row and column of the waves' tiles, those at or above the diagonal shared out
        // so that no SIMD (wave % 4) has more than 10 of 36 units, or 3 of 10; d = 8: none
        int i0, j0;
        if constexpr (RB == 8) {
            i0 = wave == 0 ? 0 : wave == 1 ? 2 : wave == 2 ? 0 : wave == 3 ? 4 : wave == 4 ? 4 : wave == 5 ? 6 : wave == 6 ? 2 : 6;
            j0 = wave == 0 || wave == 1 || wave == 3 || wave == 7 ? 4 : 0;
        } else {
            i0 = wave == 0 || wave == 1 ? 0 : wave == 2 || wave == 4 ? 1 : wave == 3 || wave == 6 ? 2 : 3;
            j0 = wave == 1 || wave == 2 || wave == 3 || wave == 5 ? 2 : 0;
        }
        const int d = i0 - j0;
        if (d < 0) gram_and_poly<-8>(i0, j0);
        else if (d == 0) gram_and_poly<0>(i0, j0);
        else if (d < WB) gram_and_poly<WB / 2>(i0, j0);
        else gram_and_poly<8>(i0, j0);
    }

    // X = P X in place, or (LAST) the result; ALONG: lane = column of the iterate, otherwise its row
    template <bool LAST, bool ALONG>
    __device__ __forceinline__ void apply() const {
        for (int j = wave; j < v.C; j += kWgWaves) {
            char *const col = v.x0 + (int64_t)j * v.R * UNIT;
            Frag<PL> x[RB > 4 ? 3 : 2][2];  // units of the column, loaded ahead
            constexpr int RING = RB > 4 ? 3 : 2;
            auto load = [&](int k) {
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int z = 0; z < PL; ++z)
                        x[k % RING][s].p[z] = *(const half8 *)(col + k * UNIT + z * kPlane + chunk(n, h, s));
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
                            Frag<PL> f;  // (units past the matrix hold anything: those results are not used)
                            frag(f, i, k, s);
                            if constexpr (ALONG || !LAST) mma<PL>(acc[i], f, x[k % RING][s]);
                            else mma<PL>(acc[i], x[k % RING][s], f);
                        }
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < RB; ++i) {
                if (i < v.R) {
                    if constexpr (LAST) {
                        store_last<MUON, BF16>(v, p, acc[i], col + i * UNIT, i, j, h, n);
                    } else {
                        half4 out[4][PL];
                        pack_unit<PL>(acc[i], 1.0f, out);
                        store_unit<PL>(col + i * UNIT, out, n, h);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        wait_copies_and_barrier<0>();  // (the stores, too)
    }
};

template <int RB, int PL, bool MUON, bool BF16>
__global__ __launch_bounds__(64 * kWgWaves) __attribute__((amdgpu_waves_per_eu(RB == 8 ? 2 : 4))) void
ns_matrix_kernel(NsWork w, NsParams p, int first) {
    using Wg = MatrixWg<RB, PL, MUON, BF16>;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const View v = view_of<PL>(w, first + blockIdx.x);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    const Wg g{p, v, lds, lds0, lane, wave, lane >> 5, lane & 31};
    for (int step = 0;; ++step) {
        g.fresh().make_p();
        if (step + 1 == p.steps) break;
        g.fresh().template apply<false, true>();
    }
    if (v.tr) g.fresh().template apply<true, false>();
    else g.fresh().template apply<true, true>();
}

// S stages: with the large tile two workgroups per CU, with the small one enough copies in
// flight for a CU that has one
template <int T, int PL> constexpr int kStages = T == 128 ? (PL == 2 ? 2 : 4) : 4;

template <int T, int PL, int KIND, bool MUON, bool BF16>
hipError_t launch_product(NsWork w, const NsTile *tiles, int64_t grid, const NsParams &p, int odd, hipStream_t s) {
    w.tiles = tiles;
    const int r = w.uni.rows < w.uni.cols ? w.uni.rows : w.uni.cols, c = w.uni.rows + w.uni.cols - r;
    w.nti = (r + T - 1) / T;
    w.ntj = (c + T - 1) / T;
    constexpr int S = kStages<T, PL>;
    hipLaunchKernelGGL((ns_product_kernel<T, PL, S, KIND, MUON, BF16>), dim3((unsigned)grid), dim3(256),
                       S * 2 * (T / 32) * PL * kPlane, s, w, p, odd);
    return hipGetLastError();
}

template <int T, bool MUON, bool BF16>
hipError_t launch_all(NsWork w, const NsLists &l, const NsParams &p, hipStream_t s) {
    constexpr int PL = BF16 ? 1 : 2;
    if (l.n_small > 0) {
        hipLaunchKernelGGL((ns_small_kernel<MUON, BF16, PL>), dim3((unsigned)l.n_small), dim3(64 * kSmallWaves), l.small_lds, s, w,
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
    hipLaunchKernelGGL((ns_norm_kernel<MUON, BF16, PL>), gx, b, 0, s, wx, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((ns_scale_kernel<MUON, BF16, PL>), gx, b, 0, s, wx, p);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    // matrices of more than 128 rows, then of fewer
    if (l.n_wg8 > 0) {
        hipLaunchKernelGGL((ns_matrix_kernel<8, PL, MUON, BF16>), dim3((unsigned)l.n_wg8), dim3(64 * kWgWaves),
                           (MatrixWg<8, PL, MUON, BF16>::LDS), s, w, p, (int)l.first_wg8);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (l.n_wg4 > 0) {
        hipLaunchKernelGGL((ns_matrix_kernel<4, PL, MUON, BF16>), dim3((unsigned)l.n_wg4), dim3(64 * kWgWaves),
                           (MatrixWg<4, PL, MUON, BF16>::LDS), s, w, p, (int)l.first_wg4);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    for (int k = 0; k < p.steps && l.n_apply > 0; ++k) {
        const int odd = k & 1;
        e = launch_product<T, PL, kGram, false, false>(w, l.gram, l.n_gram, p, odd, s);
        if (e != hipSuccess) return e;
        e = launch_product<T, PL, kPoly, false, false>(w, l.gram, l.n_gram, p, odd, s);
        if (e != hipSuccess) return e;
        e = k + 1 < p.steps ? launch_product<T, PL, kApply, false, false>(w, l.apply, l.n_apply, p, odd, s)
                            : launch_product<T, PL, kLast, MUON, BF16>(w, l.apply, l.n_apply, p, odd, s);
        if (e != hipSuccess) return e;
    }
    if constexpr (MUON) {
        hipLaunchKernelGGL(ns_update_kernel, gx, b, 0, s, wx, p, p.steps & 1);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

int64_t ns_matrix_bytes(int64_t rows, int64_t cols, int planes) {
    const int64_t r = rows < cols ? rows : cols, c = rows + cols - r;
    const int64_t R = (r + 31) / 32, C = (c + 31) / 32;
    return 2 * (R * C + R * R) * planes * kPlane;
}

int64_t ns_small_bytes(int64_t rows, int64_t cols, int planes) {
    const int r = (int)(rows < cols ? rows : cols), c = (int)(rows + cols - r);
    const int R = units(r), C = units(c);
    const bool fits = planes == 2 ? fits_small<2>(R, C) : fits_small<1>(R, C);
    return fits ? (int64_t)(R * C + R * R) * planes * kPlane : 0;
}

int ns_matrix_rows(int64_t rows, int64_t cols) {
    const int R = units((int)(rows < cols ? rows : cols));
    return R <= 4 ? 4 : R <= 8 ? 8 : 0;
}

int64_t ns_matrix_wg_bytes(int64_t rows, int64_t cols, int planes) {
    const int64_t r = rows < cols ? rows : cols, c = rows + cols - r;
    return (r + 31) / 32 * ((c + 31) / 32) * planes * kPlane;
}

// A workgroup takes as long for its matrix as tiles on all CUs for about forty of them
bool ns_by_matrix(double total, double largest) { return total >= 40.0 * largest; }

// 128 x 128 tiles read each staged unit twice as often; once they do not fill
// the CUs, tiles of a quarter the size do the work sooner
int ns_tile(int64_t tiles128) { return tiles128 >= 256 ? 128 : 64; }

hipError_t launch_ns(const NsWork &w, const NsLists &l, const NsParams &p, bool muon, bool bf16, hipStream_t s) {
    if (l.tile == 128)
        return muon ? launch_all<128, true, false>(w, l, p, s)
                    : bf16 ? launch_all<128, false, true>(w, l, p, s) : launch_all<128, false, false>(w, l, p, s);
    return muon ? launch_all<64, true, false>(w, l, p, s)
                : bf16 ? launch_all<64, false, true>(w, l, p, s) : launch_all<64, false, false>(w, l, p, s);
}

}  // namespace evo

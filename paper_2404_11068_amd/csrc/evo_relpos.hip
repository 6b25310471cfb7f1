// evo_relpos.hip -- learned relative position bias by buckets, and the
// gradient of its table, gfx950.
//
//   out[b, h, i, j] = base[b, h, i, j] + table[h, n],   n = #{e <= pos_i - pos_j}
//   dtable[h, n]    = sum of dbias[b, h, i, j] over the entries of bucket n
//
// Both are streams: the forward writes (and with a base reads) every entry
// once, the backward reads every entry once, against a few operations per
// entry; large calls are bound by HBM, small ones by launch and latency.
#include "evo_frag.h"
#include "evo_kernels.h"

namespace evo {
namespace {

constexpr int kRpThreads = 256;
constexpr int kRpLut = 6144;  // entries of the bucket table, 2 bytes each

// a - b, at the ends of int32 where it lies beyond
__device__ __forceinline__ int rp_sub(int a, int b) { return __builtin_elementwise_sub_sat(a, b); }

// How the buckets of a call are found, the same for all of its entries:
//   kRpUnit    the edges are consecutive integers (differences clipped at +-K, the
//              common form): the bucket is a clamp of the difference
//   kRpTable   from a table in LDS, one entry per difference
//   kRpSteps   from a table over the differences in steps of 1 << shift, whose entry
//              counts the edges up to the step's first difference, then at most
//              `more` comparisons with the edges inside a step
//   kRpSearch  by a branch-free binary search over the edges in LDS, 7 steps for 64
//              to 127 edges, the searches of a lane side by side: for calls too
//              short to pay for a table, and where a step would hold many edges
enum { kRpUnit, kRpTable, kRpSteps, kRpSearch };

struct RpFind {
    const int *edges;     // LDS
    const uint16_t *lut;  // LDS
    int E, mode, lo, hi, shift, more, steps;

    // by all threads of a workgroup of T threads, with barriers; mem: E ints, 16-byte aligned.
    // lut: kRpLut entries, or null for no table
    template <int T>
    __device__ __forceinline__ void stage(int *mem, uint16_t *table, const int32_t *src, int n, int tid) {
        edges = mem;
        lut = table;
        E = n;
        shift = more = 0;
        steps = n > 0 ? 32 - __builtin_clz(n) : 0;
        const int first = n > 0 ? src[0] : 0;
        hi = n > 0 ? src[n - 1] : 0;
        lo = first - 1;  // (where it exists: no mode but the search uses it otherwise)
        int same = 1;
        for (int k = tid; k < n; k += T) {
            const int e = src[k];
            mem[k] = e;
            same &= (int64_t)e - first == k;
        }
        const bool unit = __syncthreads_and(same) != 0;
        const bool has = n > 0 && first > -0x7fffffff && hi >= first;
        mode = unit && has ? kRpUnit : kRpSearch;
        if (!table || mode == kRpUnit || !has) return;
        // differences lo .. hi; each edge is counted from the first step on that
        // starts at or after it: marks, then their running sum
        const int64_t reach = (int64_t)hi - lo + 1;
        while ((reach >> shift) + 2 > kRpLut) ++shift;
        unsigned *const w = (unsigned *)table;
        constexpr int R = kRpLut / T;  // entries of a thread, consecutive
        for (int k = tid; k < kRpLut / 2; k += T) w[k] = 0;
        __syncthreads();
        for (int k = tid; k < n; k += T) {
            const int64_t d = (int64_t)mem[k] - lo, up = (d + ((int64_t)1 << shift) - 1) >> shift;
            const int at = up < 0 ? 0 : up < kRpLut - 1 ? (int)up : kRpLut - 1;
            atomicAdd(&w[at >> 1], 1u << (16 * (at & 1)));
        }
        __syncthreads();
        unsigned v[R / 2], sum = 0, most = 0;
#pragma unroll
        for (int x = 0; x < R / 2; ++x) {
            v[x] = w[tid * (R / 2) + x];
            const unsigned a = v[x] & 0xffffu, b = v[x] >> 16;
            sum += a + b;
            most = max(most, max(a, b));
        }
        unsigned before = sum;  // inclusive scan over the threads, then exclusive
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const unsigned o = __shfl_up(before, m, 64);
            if ((tid & 63) >= m) before += o;
        }
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) most = max(most, (unsigned)__shfl_xor((int)most, m, 64));
        __shared__ unsigned wave_sum[T / 64], wave_most[T / 64];
        if ((tid & 63) == 63) {
            wave_sum[tid >> 6] = before;
            wave_most[tid >> 6] = most;
        }
        __syncthreads();
        before -= sum;
#pragma unroll
        for (int k = 0; k < T / 64; ++k) {
            before += k < (tid >> 6) ? wave_sum[k] : 0u;
            most = max(most, wave_most[k]);
        }
#pragma unroll
        for (int x = 0; x < R / 2; ++x) {
            const unsigned a = before + (v[x] & 0xffffu), b = a + (v[x] >> 16);
            w[tid * (R / 2) + x] = a | (b << 16);
            before = b;
        }
        more = (int)most;
        if (shift == 0) mode = kRpTable;
        else if (more <= steps / 2) mode = kRpSteps;
        __syncthreads();
    }

    // buckets of the differences d, in [0, E] for any edges
    template <int MODE, int N>
    __device__ __forceinline__ void buckets(const int (&d)[N], int (&n)[N]) const {
        if constexpr (MODE == kRpSearch) {
#pragma unroll
            for (int x = 0; x < N; ++x) n[x] = 0;
            for (int s = steps - 1; s >= 0; --s) {
                int at[N], e[N];
#pragma unroll
                for (int x = 0; x < N; ++x) {
                    at[x] = n[x] + (1 << s);
                    e[x] = edges[(at[x] <= E ? at[x] : E) - 1];
                }
#pragma unroll
                for (int x = 0; x < N; ++x) n[x] = at[x] <= E && e[x] <= d[x] ? at[x] : n[x];
            }
        } else {
#pragma unroll
            for (int x = 0; x < N; ++x) {
                const int t = d[x] < lo ? lo : d[x] > hi ? hi : d[x];
                const unsigned at = (unsigned)t - (unsigned)lo;  // (the edges of kRpSteps may span more than an int)
                n[x] = MODE == kRpUnit ? (int)at : MODE == kRpTable ? lut[at] : lut[at >> shift];
            }
            if constexpr (MODE == kRpSteps)
                for (int k = 0; k < more; ++k) {
                    int e[N];
#pragma unroll
                    for (int x = 0; x < N; ++x) e[x] = edges[n[x] < E ? n[x] : 0];
#pragma unroll
                    for (int x = 0; x < N; ++x) n[x] += n[x] < E && e[x] <= d[x];
                }
        }
    }
};

// N consecutive values from a pointer aligned to one of them
template <int N, class T> struct RpPack { T v[N]; };
template <int N, class T>
__device__ __forceinline__ void rp_load(T (&v)[N], const T *p) {
    RpPack<N, T> t;
    __builtin_memcpy(&t, p, sizeof t);
#pragma unroll
    for (int x = 0; x < N; ++x) v[x] = t.v[x];
}
template <int N, class T>
__device__ __forceinline__ void rp_store(const T (&v)[N], T *p) {
    RpPack<N, T> t;
#pragma unroll
    for (int x = 0; x < N; ++x) t.v[x] = v[x];
    __builtin_memcpy(p, &t, sizeof t);
}

// ---------------------------------------------------------------------------
// forward
//
// A lane owns 8 consecutive entries j of a row i in up to 8 heads: one 16-byte
// access per head in bf16 (the ISA takes them at any element's alignment, so
// odd lengths need no other path than the row's last piece).  It finds the
// buckets of its entries once and uses them for all heads of its group.  The
// table lies in LDS with a bucket's heads side by side, so one or two 16-byte
// reads bring an entry's values for the whole group; every eighth bucket adds
// 16 bytes of padding, because neighbouring lanes are 8 buckets apart and
// would otherwise all meet in one bank.  16 planes of 2049 x 2049 in bf16: 34 us,
// 4.0 TB/s of writes; 8 of 256 x 256 onto a base: 4.0 us, a launch.

constexpr int kRpCols = 8;  // consecutive entries of a lane

// floats of the table's LDS copy before bucket n, HG heads each
template <int HG>
__host__ __device__ constexpr int rp_slot(int n) {
    return n * HG + (n >> 3) * (HG < 4 ? HG : 4);
}

__device__ __forceinline__ float rp_value(uint16_t v) { return bf2f(v); }
__device__ __forceinline__ float rp_value(float v) { return v; }
template <class T> __device__ __forceinline__ T rp_round(float v);
template <> __device__ __forceinline__ uint16_t rp_round<uint16_t>(float v) { return f2bf(v); }
template <> __device__ __forceinline__ float rp_round<float>(float v) { return v; }

// the positions (or segments) of a piece's columns; past the row's end its last one
__device__ __forceinline__ void rp_columns(int (&v)[kRpCols], const int32_t *row, int j0, int Lj) {
    if (j0 + kRpCols <= Lj) {
        rp_load(v, row + j0);
    } else {
#pragma unroll
        for (int x = 0; x < kRpCols; ++x) v[x] = row[j0 + x < Lj ? j0 + x : Lj - 1];
    }
}

template <class T, int HG>
__global__ __launch_bounds__(kRpThreads) void relpos_fwd_kernel(RpArgs a, int64_t pieces, int per_row, int table) {
    extern __shared__ __attribute__((aligned(16))) float tab[];
    const int tid = threadIdx.x, h0 = blockIdx.y * HG, heads = a.H - h0 < HG ? a.H - h0 : HG;
    const int64_t b = blockIdx.z;
    // a bucket's heads side by side; the missing heads of the last group stay unset and unused
    for (int x = tid; x < heads * a.NB; x += kRpThreads) {
        const int h = x / a.NB, n = x - h * a.NB;
        tab[rp_slot<HG>(n) + h] = a.table[(int64_t)(h0 + h) * a.NB + n];
    }
    RpFind f;
    {
        int *const em = (int *)(tab + ((rp_slot<HG>(a.NB) + 3) & ~3));
        f.stage<kRpThreads>(em, table ? (uint16_t *)(em + ((a.E + 3) & ~3)) : nullptr, a.edges, a.E, tid);
    }

    const int64_t plane = (int64_t)a.Li * a.Lj;
    for (int64_t c = blockIdx.x * (int64_t)kRpThreads + tid; c < pieces; c += (int64_t)gridDim.x * kRpThreads) {
        int64_t i64;
        if (pieces <= 0x7fffffff) i64 = (uint32_t)c / (uint32_t)per_row;
        else i64 = c / per_row;
        const int i = (int)i64, j0 = (int)(c - i64 * per_row) * kRpCols;
        const int64_t at = (b * a.H + h0) * plane + i64 * a.Lj + j0;
        const T *base = a.base ? (const T *)a.base + at : nullptr;
        T *out = (T *)a.out + at;
        const bool full = j0 + kRpCols <= a.Lj;
        T g[HG][kRpCols];
        if (base && full) {
#pragma unroll
            for (int h = 0; h < HG; ++h)
                if (h < heads) rp_load(g[h], base + h * plane);
        }
        int d[kRpCols], n[kRpCols];
        rp_columns(d, a.pos_j + b * a.Lj, j0, a.Lj);
        const int pi = a.pos_i[b * a.Li + i];
#pragma unroll
        for (int x = 0; x < kRpCols; ++x) d[x] = rp_sub(pi, d[x]);
        if (f.mode == kRpUnit) f.buckets<kRpUnit>(d, n);
        else if (f.mode == kRpTable) f.buckets<kRpTable>(d, n);
        else if (f.mode == kRpSteps) f.buckets<kRpSteps>(d, n);
        else f.buckets<kRpSearch>(d, n);
        if (a.seg_i) {
            rp_columns(d, a.seg_j + b * a.Lj, j0, a.Lj);
            const int si = a.seg_i[b * a.Li + i];
#pragma unroll
            for (int x = 0; x < kRpCols; ++x) n[x] = d[x] == si ? n[x] : a.E + 1;
        }
        float v[kRpCols][HG];
#pragma unroll
        for (int x = 0; x < kRpCols; ++x) {
            const float *row = tab + rp_slot<HG>(n[x]);
            if constexpr (HG >= 4) {
#pragma unroll
                for (int q = 0; q < HG / 4; ++q) {
                    const f32x4 w = *(const f32x4 *)(row + 4 * q);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[x][4 * q + e] = w[e];
                }
            } else {
#pragma unroll
                for (int h = 0; h < HG; ++h) v[x][h] = row[h];
            }
        }
        if (full) {
#pragma unroll
            for (int h = 0; h < HG; ++h) {
                if (h >= heads) break;
                T o[kRpCols];
#pragma unroll
                for (int x = 0; x < kRpCols; ++x)
                    o[x] = rp_round<T>(base ? rp_value(g[h][x]) + v[x][h] : v[x][h]);
                rp_store(o, out + h * plane);
            }
        } else {
#pragma unroll
            for (int x = 0; x < kRpCols; ++x) {
                if (j0 + x >= a.Lj) break;
#pragma unroll
                for (int h = 0; h < HG; ++h)
                    if (h < heads)
                        out[h * plane + x] = rp_round<T>(base ? rp_value(base[h * plane + x]) + v[x][h] : v[x][h]);
            }
        }
    }
}

template <class T, int HG>
hipError_t launch_fwd_hg(const RpArgs &a, hipStream_t s) {
    const int per_row = (a.Lj + kRpCols - 1) / kRpCols;
    const int64_t pieces = (int64_t)a.Li * per_row, wg = (pieces + kRpThreads - 1) / kRpThreads;
    const int64_t groups = (int64_t)((a.H + HG - 1) / HG);
    for (int64_t b0 = 0; b0 < a.B; b0 += 65535) {
        const int64_t nb = a.B - b0 < 65535 ? a.B - b0 : 65535;
        RpArgs c = a;
        const int64_t skip = b0 * a.H * (int64_t)a.Li * a.Lj * (int64_t)sizeof(T);
        c.pos_i += b0 * a.Li;
        c.pos_j += b0 * a.Lj;
        if (a.seg_i) {
            c.seg_i += b0 * a.Li;
            c.seg_j += b0 * a.Lj;
        }
        if (a.base) c.base = (const char *)a.base + skip;
        c.out = (char *)a.out + skip;
        // four workgroups per CU, each walking its share with the table staged
        // once.  The bucket table takes about as long to build as three searches
        int64_t grid = 1024 / (groups * nb);
        if (grid < 1) grid = 1;
        if (grid > wg) grid = wg;
        const int table = a.E > 3 && wg > 3 * grid;
        const size_t lds = (size_t)((rp_slot<HG>(a.NB) + 3) & ~3) * 4 + (size_t)((a.E + 3) & ~3) * 4 + (table ? kRpLut * 2 : 0);
        hipLaunchKernelGGL((relpos_fwd_kernel<T, HG>), dim3((unsigned)grid, (unsigned)groups, (unsigned)nb),
                           dim3(kRpThreads), lds, s, c, pieces, per_row, table);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class T>
hipError_t launch_fwd_t(const RpArgs &a, hipStream_t s) {
    // Heads per group: as many as there are, up to eight, while the groups'
    // workgroups still number the CUs
    const int64_t wg = a.B * (((int64_t)a.Li * ((a.Lj + kRpCols - 1) / kRpCols) + kRpThreads - 1) / kRpThreads);
    auto enough = [&](int hg) { return a.H > hg / 2 && wg * ((a.H + hg - 1) / hg) >= 256; };
    if (enough(8)) return launch_fwd_hg<T, 8>(a, s);
    if (enough(4)) return launch_fwd_hg<T, 4>(a, s);
    if (enough(2)) return launch_fwd_hg<T, 2>(a, s);
    return launch_fwd_hg<T, 1>(a, s);
}

// ---------------------------------------------------------------------------
// backward
//
// Sums by bucket without atomics: the lanes of a wave have columns of their own
// in a histogram in LDS, [bucket][C columns], so the wave's accesses touch
// different banks whatever the buckets are, and nothing depends on timing.
// (LDS float atomics to the same places took 200 cycles an instruction.)
// A lane's piece of four entries is first summed within its buckets, each entry with
// those before it; then it reads its four sums at once, adds, and writes them back
// in order: one LDS round trip per piece instead of four.  At the end the columns
// of every row are summed in a fixed order, and a second kernel adds the
// waves' sums in order, in fp64.
//
// 16 planes of 2048 x 2048, differences clipped: 65 buckets 57 us (4.7 TB/s), 129 65 us, 257 88 us (by a table
// 96), 513 in two passes 162 us.  With more than 67 buckets the turns' chains of LDS reads, additions and writes bound
// it, not HBM: at 257 the LDS is busy 38% and the vector units 43% of the time, and waves wait 36% of theirs.
//
// C is 64, one column per lane, for up to 67 buckets.  With more of them that
// would leave a SIMD fewer than two waves, so 32 (up to 133) or 16 columns serve the
// wave's halves or quarters in turn (257 buckets: 16 columns and two workgroups per CU 88 us a call, 32 and one
// 109; 127 buckets: 32 and two 67, 64 and one 80).
//
// A wave takes one head and a run of 4-entry pieces of its rows, 64 at a time.
// The last piece of a row whose length is no multiple of four starts earlier,
// so that it lies inside the row, and skips the entries it shares with the one
// before: no branch, and every load is a whole one.  AHEAD pieces per lane are
// in flight while as many are added.  More buckets than 512 take several
// passes over the entries, each for some of them.

constexpr int kRpMaxBuckets = 512;
constexpr int kRpWaves = 4;  // per workgroup

struct RpBwdPlan {
    int piece;        // entries of a lane's piece
    int span;         // buckets per pass
    int passes;
    int columns;      // of the histogram
    int64_t pieces;   // per head
    int64_t shares;   // waves per head and pass
    int64_t per_wave; // pieces of a wave, a multiple of 64
};

// LDS of a workgroup: its waves' histograms, the bucket table and the edges
__host__ __device__ inline size_t rp_bwd_lds(int columns, int span, int E) {
    return (size_t)kRpWaves * span * columns * 4 + kRpLut * 2 + (size_t)((E + 3) & ~3) * 4;
}

RpBwdPlan plan_bwd(const RpArgs &a) {
    RpBwdPlan p;
    p.piece = a.Lj >= 4 ? 4 : 1;
    p.passes = (a.NB + kRpMaxBuckets - 1) / kRpMaxBuckets;
    p.span = (a.NB + p.passes - 1) / p.passes;
    const size_t all = 159 * 1024;  // of two workgroups, whose other LDS is 288 bytes each
    p.columns = p.piece == 1 ? 16 : 64;
    while (p.columns > 16 && 2 * rp_bwd_lds(p.columns, p.span, a.E) > all) p.columns /= 2;  // (16: 512 buckets take 147 KB)
    int64_t per_cu = (int64_t)(all / rp_bwd_lds(p.columns, p.span, a.E)) * kRpWaves;
    if (per_cu > 8) per_cu = 8;
    const int64_t per_row = (a.Lj + p.piece - 1) / p.piece;
    p.pieces = a.B * a.Li * per_row;
    // a wave takes four rounds of 64 pieces at least
    int64_t shares = 256 * per_cu / ((int64_t)a.H * p.passes);
    const int64_t most = (p.pieces + 255) / 256;
    if (shares > most) shares = most;
    if (shares < 1) shares = 1;
    p.per_wave = ((p.pieces + shares - 1) / shares + 63) / 64 * 64;
    p.shares = (p.pieces + p.per_wave - 1) / p.per_wave;
    return p;
}

// a lane's place among the pieces: batch entry, row, piece of the row; and the
// way to the piece 64 further on
struct RpPlace {
    int64_t b, left;  // batch entry; pieces from here to the wave's end
    int i, c;
    int step_c, step_i;
    int64_t step_b;

    template <bool MANY>
    __device__ __forceinline__ void start(const RpArgs &a, int64_t first, int64_t last, int lane, int per_row) {
        const int64_t p = first + lane, row = p / per_row;
        left = last - p;
        c = (int)(p - row * per_row);
        b = MANY ? row / a.Li : 0;
        i = (int)(row - b * a.Li);
        step_c = 64 % per_row;
        const int rows = 64 / per_row;
        step_b = MANY ? rows / a.Li : 0;
        step_i = (int)(rows - step_b * a.Li);
    }
    template <bool MANY>
    __device__ __forceinline__ void next(const RpArgs &a, int per_row) {
        c += step_c;
        const bool over = c >= per_row;
        c -= over ? per_row : 0;
        i += step_i + (over ? 1 : 0);
        if constexpr (MANY) {  // at most Li rows on
            const bool wrap = i >= a.Li;
            i -= wrap ? a.Li : 0;
            b += step_b + (wrap ? 1 : 0);
        }
        left -= 64;
    }
};

template <int P, bool SEG>
struct RpLoaded {  // a piece as loaded
    float g[P];
    int pj[P], sj[SEG ? P : 1], pi, si, skip;  // skip: entries that do not count

    template <bool MANY>
    __device__ __forceinline__ void load(const RpArgs &a, const RpPlace &p, const float *head, int64_t plane_b) {
        // past the wave's end the batch's first piece, none of which counts
        const bool ok = p.left > 0;
        const int i = ok ? p.i : 0, j = ok ? p.c * P : 0, js = j + P <= a.Lj ? j : a.Lj - P;
        const int64_t b = MANY ? (ok ? p.b : 0) : 0;
        rp_load(g, head + (MANY ? b * plane_b : 0) + (int64_t)i * a.Lj + js);
        rp_load(pj, a.pos_j + (MANY ? b * a.Lj : 0) + js);
        pi = a.pos_i[(MANY ? b * a.Li : 0) + i];
        if constexpr (SEG) {
            rp_load(sj, a.seg_j + (MANY ? b * a.Lj : 0) + js);
            si = a.seg_i[(MANY ? b * a.Li : 0) + i];
        }
        skip = ok ? j - js : P;
    }
};

template <int MODE, int P, int C, bool SEG, bool MANY, bool PART, int AHEAD>
__device__ __forceinline__ void rp_accumulate(const RpArgs &a, const RpFind &f, int64_t first, int64_t last, int per_row,
                                              int n0, int span, int h, int lane, float *hist) {
    const int64_t plane = (int64_t)a.Li * a.Lj, plane_b = plane * a.H;
    const float *const head = a.dbias + h * plane;
    RpPlace p;
    p.start<MANY>(a, first, last, lane, per_row);
    RpLoaded<P, SEG> now[AHEAD], then[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
        now[u].template load<MANY>(a, p, head, plane_b);
        p.next<MANY>(a, per_row);
    }
    for (int64_t at = first; at < last; at += 64 * AHEAD) {  // (wave-uniform)
        if (at + 64 * AHEAD < last) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                then[u].template load<MANY>(a, p, head, plane_b);
                p.next<MANY>(a, per_row);
            }
        }
        int most = 0;  // entries that do not count are rare: one test for all pieces of the round
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) most |= now[u].skip;
        if (__any(most)) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                for (int x = 0; x < P; ++x) now[u].g[x] = x < now[u].skip ? 0.0f : now[u].g[x];
        }
        int n[AHEAD][P];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            int d[P];
#pragma unroll
            for (int x = 0; x < P; ++x) d[x] = rp_sub(now[u].pi, now[u].pj[x]);
            f.buckets<MODE>(d, n[u]);
            if constexpr (SEG) {
#pragma unroll
                for (int x = 0; x < P; ++x) n[u][x] = now[u].sj[x] == now[u].si ? n[u][x] : a.E + 1;
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            float g[P];
#pragma unroll
            for (int x = 0; x < P; ++x) g[x] = now[u].g[x];
            if constexpr (PART) {  // for a bucket of another pass nothing is added to this pass's last one
#pragma unroll
                for (int x = 0; x < P; ++x) {
                    const unsigned k = (unsigned)(n[u][x] - n0);
                    g[x] = k < (unsigned)span ? g[x] : 0.0f;
                    n[u][x] = (int)(k < (unsigned)span ? k : (unsigned)span - 1);
                }
            }
            // an entry brings along those before it in its bucket: the last one's write holds them all
#pragma unroll
            for (int x = 1; x < P; ++x) {
                float s = 0.0f;
#pragma unroll
                for (int y = 0; y < x; ++y) s = n[u][y] == n[u][x] ? g[y] : s;
                g[x] += s;
            }
#pragma unroll
            for (int turn = 0; turn < 64 / C; ++turn) {
                if (C == 64 || lane / C == turn) {
                    float v[P];
#pragma unroll
                    for (int x = 0; x < P; ++x) v[x] = hist[n[u][x] * C];
#pragma unroll
                    for (int x = 0; x < P; ++x) hist[n[u][x] * C] = v[x] + g[x];
                }
                // the turns' accesses to a column stay in order
                if (C < 64) __builtin_amdgcn_wave_barrier();
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) now[u] = then[u];
    }
}

template <int P, int C, bool SEG, bool MANY, bool PART, int AHEAD>
__global__ __launch_bounds__(64 * kRpWaves) __attribute__((amdgpu_waves_per_eu(1, 2))) void
relpos_bwd_kernel(RpArgs a, int span, int per_row, int64_t pieces, int64_t per_wave, int64_t shares, float *__restrict__ part) {
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = blockIdx.y, n0 = blockIdx.z * span;
    float *const all = lds + wave * span * C;
    for (int k = lane; k < span * C; k += 64) all[k] = 0.0f;
    RpFind f;
    {
        int *const em = (int *)(lds + kRpWaves * span * C);
        f.stage<64 * kRpWaves>(em, (uint16_t *)(em + ((a.E + 3) & ~3)), a.edges, a.E, tid);
    }
    const int64_t share = (int64_t)blockIdx.x * kRpWaves + wave;
    if (share >= shares) return;
    const int64_t first = share * per_wave, last = first + per_wave < pieces ? first + per_wave : pieces;
    float *const hist = all + lane % C;
    if (f.mode == kRpUnit)
        rp_accumulate<kRpUnit, P, C, SEG, MANY, PART, AHEAD>(a, f, first, last, per_row, n0, span, h, lane, hist);
    else if (f.mode == kRpTable)
        rp_accumulate<kRpTable, P, C, SEG, MANY, PART, AHEAD>(a, f, first, last, per_row, n0, span, h, lane, hist);
    else if (f.mode == kRpSteps)
        rp_accumulate<kRpSteps, P, C, SEG, MANY, PART, AHEAD>(a, f, first, last, per_row, n0, span, h, lane, hist);
    else
        rp_accumulate<kRpSearch, P, C, SEG, MANY, PART, AHEAD>(a, f, first, last, per_row, n0, span, h, lane, hist);
    __builtin_amdgcn_wave_barrier();
    // 16 rows at a time, C / 4 columns per lane, from a column of the lane's own on, then the four quarters
    float *const dst = part + ((blockIdx.z * (int64_t)a.H + h) * shares + share) * span;
    const int q = lane >> 4, x = lane & 15;
    constexpr int Q = C / 4;
    for (int k0 = 0; k0 < span; k0 += 16) {
        const int k = k0 + x < span ? k0 + x : span - 1;
        const float *row = all + k * C + q * Q;
        float v[Q], s = 0.0f;
#pragma unroll
        for (int l = 0; l < Q; ++l) v[l] = row[(l + x) & (Q - 1)];
#pragma unroll
        for (int l = 0; l < Q; ++l) s += v[l];
        s += __shfl_xor(s, 16, 64);
        s += __shfl_xor(s, 32, 64);
        if (q == 0 && k0 + x < span) dst[k0 + x] = s;
    }
}

// dtable: the shares of every wave, in order; 16 buckets x 16 slices of the shares per workgroup
__global__ __launch_bounds__(256) void relpos_bwd_sum_kernel(const float *__restrict__ part, int shares, int span, int NB,
                                                            int H, float *__restrict__ dtable) {
    __shared__ double red[16][17];
    const int x = threadIdx.x & 15, y = threadIdx.x >> 4, h = blockIdx.y;
    const int n = blockIdx.x * 16 + x, pass = n / span, k = n - pass * span;
    double s = 0.0;
    if (n < NB) {
        const float *src = part + ((int64_t)pass * H + h) * shares * span + k;
        int w = y;
        for (; w + 48 < shares; w += 64) {  // four in flight, added in order
            float v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = src[(int64_t)(w + 16 * u) * span];
#pragma unroll
            for (int u = 0; u < 4; ++u) s += (double)v[u];
        }
        for (; w < shares; w += 16) s += (double)src[(int64_t)w * span];
    }
    red[y][x] = s;
    __syncthreads();
    if (y == 0 && n < NB) {
#pragma unroll
        for (int w = 1; w < 16; ++w) s += red[w][x];
        dtable[(int64_t)h * NB + n] = (float)s;
    }
}

__global__ __launch_bounds__(256) void relpos_zero_kernel(float *p, int64_t n) {
    const int64_t x = blockIdx.x * (int64_t)256 + threadIdx.x;
    if (x < n) p[x] = 0.0f;
}

template <int P, int C, bool SEG, bool MANY, bool PART, int AHEAD>
hipError_t launch_bwd_as(const RpArgs &a, const RpBwdPlan &p, float *part, hipStream_t s) {
    hipLaunchKernelGGL((relpos_bwd_kernel<P, C, SEG, MANY, PART, AHEAD>),
                       dim3((unsigned)((p.shares + kRpWaves - 1) / kRpWaves), (unsigned)a.H, (unsigned)p.passes),
                       dim3(64 * kRpWaves), rp_bwd_lds(C, p.span, a.E), s, a, p.span, (a.Lj + P - 1) / P, p.pieces,
                       p.per_wave, p.shares, part);
    return hipGetLastError();
}

template <bool SEG, bool MANY>
hipError_t launch_bwd(const RpArgs &a, const RpBwdPlan &p, float *part, hipStream_t s) {
    // rows of one to three entries, and several passes (of 257 buckets and more: 16 columns): rare, in one form each
    if (p.piece == 1) return launch_bwd_as<1, 16, SEG, MANY, true, 4>(a, p, part, s);
    if (p.passes > 1) return launch_bwd_as<4, 16, SEG, MANY, true, 8>(a, p, part, s);
    if (p.columns == 16) return launch_bwd_as<4, 16, SEG, MANY, false, 8>(a, p, part, s);
    if (p.columns == 32) return launch_bwd_as<4, 32, SEG, MANY, false, 8>(a, p, part, s);
    // four pieces ahead in short runs, so that few of a round are empty, and with
    // segments, where eight would leave registers for one wave per SIMD
    if constexpr (!SEG)
        if (p.per_wave >= 1024) return launch_bwd_as<4, 64, SEG, MANY, false, 8>(a, p, part, s);
    return launch_bwd_as<4, 64, SEG, MANY, false, 4>(a, p, part, s);
}

}  // namespace

hipError_t launch_relpos_fwd(const RpArgs &a, hipStream_t s) {
    return a.bf16 ? launch_fwd_t<uint16_t>(a, s) : launch_fwd_t<float>(a, s);
}

size_t relpos_bwd_workspace(const RpArgs &a) {
    const RpBwdPlan p = plan_bwd(a);
    return (size_t)p.passes * a.H * p.shares * p.span * 4;
}

hipError_t launch_relpos_bwd(const RpArgs &a, void *ws, hipStream_t s) {
    if (!a.dbias) {  // no entries
        const int64_t n = (int64_t)a.H * a.NB;
        hipLaunchKernelGGL(relpos_zero_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a.dtable, n);
        return hipGetLastError();
    }
    const RpBwdPlan p = plan_bwd(a);
    float *part = (float *)ws;
    const hipError_t e = a.seg_i ? a.B > 1 ? launch_bwd<true, true>(a, p, part, s) : launch_bwd<true, false>(a, p, part, s)
                                 : a.B > 1 ? launch_bwd<false, true>(a, p, part, s) : launch_bwd<false, false>(a, p, part, s);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(relpos_bwd_sum_kernel, dim3((unsigned)((a.NB + 15) / 16), (unsigned)a.H), dim3(256), 0, s, part,
                       (int)p.shares, p.span, a.NB, a.H, a.dtable);
    return hipGetLastError();
}

}  // namespace evo

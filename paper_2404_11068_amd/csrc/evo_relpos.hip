// evo_relpos.hip -- learned relative position bias by buckets, and the
// gradient of its table, gfx950.
#include "evo_frag.h"
#include "evo_kernels.h"

namespace evo {
namespace {

// difference of two positions, at the ends of int32 where it lies beyond
__device__ __forceinline__ int rp_offset(int i, int j) {
    const int64_t d = (int64_t)i - j;
    return d > 0x7fffffff ? 0x7fffffff : d < -0x7fffffff - 1 ? -0x7fffffff - 1 : (int)d;
}

// number of edges <= d (in [0, E] also where the edges do not ascend)
__device__ __forceinline__ int rp_search(const int32_t *edges, int E, int d) {
    int lo = 0, hi = E;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (edges[mid] <= d) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ int rp_bucket(const RpArgs &a, int64_t b, int i, int j) {
    if (a.seg_i && a.seg_i[b * a.Li + i] != a.seg_j[b * a.Lj + j]) return a.E + 1;
    return rp_search(a.edges, a.E, rp_offset(a.pos_i[b * a.Li + i], a.pos_j[b * a.Lj + j]));
}

__global__ __launch_bounds__(256) void relpos_fwd_kernel(RpArgs a) {
    const int64_t plane = (int64_t)a.Li * a.Lj, all = a.B * a.H * plane;
    for (int64_t x = blockIdx.x * (int64_t)256 + threadIdx.x; x < all; x += (int64_t)gridDim.x * 256) {
        const int64_t bh = x / plane, e = x % plane;
        const int i = (int)(e / a.Lj), j = (int)(e % a.Lj), h = (int)(bh % a.H);
        float v = a.table[(int64_t)h * a.NB + rp_bucket(a, bh / a.H, i, j)];
        if (a.bf16) {
            if (a.base) v += bf2f(((const uint16_t *)a.base)[x]);
            ((uint16_t *)a.out)[x] = f2bf(v);
        } else {
            if (a.base) v += ((const float *)a.base)[x];
            ((float *)a.out)[x] = v;
        }
    }
}

// one workgroup per bucket and head: every entry of the bucket, in a fixed order
__global__ __launch_bounds__(256) void relpos_bwd_kernel(RpArgs a) {
    __shared__ double red[256];
    const int n = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
    const int64_t plane = (int64_t)a.Li * a.Lj;
    double s = 0.0;
    for (int64_t b = 0; b < a.B; ++b) {
        const float *g = a.dbias + (b * a.H + h) * plane;
        for (int64_t e = tid; e < plane; e += 256)
            if (rp_bucket(a, b, (int)(e / a.Lj), (int)(e % a.Lj)) == n) s += (double)g[e];
    }
    red[tid] = s;
    __syncthreads();
    for (int m = 128; m >= 1; m >>= 1) {
        if (tid < m) red[tid] += red[tid + m];
        __syncthreads();
    }
    if (tid == 0) a.dtable[(int64_t)h * a.NB + n] = (float)red[0];
}

}  // namespace

hipError_t launch_relpos_fwd(const RpArgs &a, hipStream_t s) {
    const int64_t all = a.B * a.H * (int64_t)a.Li * a.Lj, wg = (all + 255) / 256;
    hipLaunchKernelGGL(relpos_fwd_kernel, dim3((unsigned)(wg < 8192 ? wg : 8192)), dim3(256), 0, s, a);
    return hipGetLastError();
}

size_t relpos_bwd_workspace(const RpArgs &) { return 0; }

hipError_t launch_relpos_bwd(const RpArgs &a, void *, hipStream_t s) {
    hipLaunchKernelGGL(relpos_bwd_kernel, dim3((unsigned)a.NB, (unsigned)a.H), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace evo

// evo_rope.hip -- rotary positions, and the norm of every head with the
// rotation in the same pass: forward and backward (include/evo_rope.h).
//
// Both directions read each element once and write it once, with a handful of
// operations between: HBM bandwidth bounds them, and for few tokens the launch.
// The angles are the expensive part per value (a 64-bit product, a polynomial
// for the sine and one for the cosine), so a workgroup forms those of its
// tokens once, in LDS, for all heads: one pair in 2 d / rot * heads elements.
//
// Measured: 2 x 8193 tokens of 32 heads of 64 in bf16, rotation alone, 22 us (6.0 TB/s);
// 128 x 256 of 16 heads of 32 in fp32 with the norm 22 us (6.1 TB/s); 4 x 4099 of 20
// heads of 128, 96 rotated, with the norm 40 us forward (4.2 TB/s), 53 us backward (4.8).
//
// A head is a group of GS lanes (the power of two that holds d / VEC chunks of
// 16 bytes); groups walk over the (token, head) units of a workgroup's tokens.
// Sums over a head are butterflies inside the group.
#include "evo_rope_kernels.h"

#include "evo_frag.h"

namespace evo {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTok = 16;  // tokens whose angles a workgroup holds

// How the partner of a channel is found: its own lane (interleaved pairs), the
// lane rot / 2 / VEC chunks away (half layout with whole chunks), or through
// LDS element by element (half layout, rot / 2 not a multiple of VEC).
enum Pairing { kInter, kHalf, kSplit };

struct KArgs {
    RopeArgs a;
    int near[2];         // token strides are small: a block's offsets fit 32 bits
    uint32_t h_mul[2];   // u / heads = u * h_mul >> 32 for a workgroup's units
    uint32_t blocks[2];  // workgroups of each set
    float *part;         // backward: partial sums of dw, [blocks of set 0 + 1][d]
    int tb, gs_log;
};

template <typename E> struct Chunk;  // 16 bytes of a head
template <> struct Chunk<float> {
    static constexpr int VEC = 4;
    static constexpr uint32_t SIGNS = 0x80000000u;
    __device__ __forceinline__ static void get(u32x4 w, float *v) {
        const f32x4 x = __builtin_bit_cast(f32x4, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = x[e];
    }
    __device__ __forceinline__ static u32x4 put(const float *v) {
        return __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]});
    }
};
template <> struct Chunk<uint16_t> {
    static constexpr int VEC = 8;
    static constexpr uint32_t SIGNS = 0x80008000u;
    __device__ __forceinline__ static void get(u32x4 w, float *v) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = __builtin_bit_cast(f32x4, w << 16)[e];
            v[2 * e + 1] = __builtin_bit_cast(f32x4, w & 0xffff0000u)[e];
        }
    }
    __device__ __forceinline__ static u32x4 put(const float *v) {
        bf16x8 w;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = (__bf16)v[e];
        return __builtin_bit_cast(u32x4, w);
    }
};

// (cos, sin) of phase / 2^64 turns.  The upper 32 bits leave 2^-32 turns, far
// below an fp32 step of the result; the nearest quarter turn is taken off
// exactly, and the rest, at most pi / 4, goes into the Taylor series, whose
// first terms left out are below 3e-9.
__device__ __forceinline__ float2 turn(uint64_t phase) {
    const uint32_t p = (uint32_t)(phase >> 32);
    const uint32_t quarter = (p + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(p - (quarter << 30)) * 1.4629180792671596e-9f;  // 2 pi / 2^32
    const float z = x * x;
    float s = fmaf(z, 2.7557319e-6f, -1.9841270e-4f);
    s = fmaf(z, s, 8.3333333e-3f);
    s = fmaf(z, s, -1.6666667e-1f);
    s = fmaf(x * z, s, x);
    float c = fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
    c = fmaf(z, c, -1.3888889e-3f);
    c = fmaf(z, c, 4.1666667e-2f);
    c = fmaf(z, c, -0.5f);
    c = fmaf(z, c, 1.0f);
    const bool odd = quarter & 1;
    const float cc = odd ? s : c, ss = odd ? c : s;
    return float2{quarter == 1 || quarter == 2 ? -cc : cc, quarter >= 2 ? -ss : ss};
}

template <int CTRL> __device__ __forceinline__ float dpp_add(float x) {
    return x + __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), CTRL, 0xf, 0xf, true));
}
// sum over aligned groups of 2^log lanes, the same in all of them: within 16 lanes by lane
// permutations of the vector unit (neighbours, pairs, then mirrored halves, whose fours and
// eights hold equal sums by then)
__device__ __forceinline__ float group_sum(float x, int log) {
    if (log > 0) x = dpp_add<0xB1>(x);
    if (log > 1) x = dpp_add<0x4E>(x);
    if (log > 2) x = dpp_add<0x141>(x);
    if (log > 3) x = dpp_add<0x140>(x);
    if (log > 4) x += __shfl_xor(x, 16, 64);
    if (log > 5) x += __shfl_xor(x, 32, 64);
    return x;
}

// largest over such groups
__device__ __forceinline__ float group_max(float x, int log) {
    for (int m = 1; m < 1 << log; m <<= 1) x = fmaxf(x, __shfl_xor(x, m, 64));
    return x;
}

// Mean squares within these bounds lost nothing that counts to the ends of fp32's range; v_rsq takes
// denormal numbers for zeros, besides.  A head beyond them is scaled by a power of two first.  Looking for such heads
// takes 1% of the forward, 2.5 to 4% of the half layout's backward (8193 tokens of 32 heads of 64: 42.2 us without).
constexpr uint32_t kLeastMean = 27u << 23, kMostMean = 247u << 23;  // 2^-100, 2^120, as bits, which are in order

// That power for a head of these channels (of the lane, of 2^log lanes): of its largest one, or of eps' root; 0 where there is none
template <int VEC> __device__ __forceinline__ int head_exponent(const float *x, int log, float eps) {
    float top = 0.0f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) top = fmaxf(top, fabsf(x[e]));
    const int ex = (int)(__float_as_uint(group_max(top, log)) >> 23) - 127;
    const int least = eps > 0.0f ? ((int)(__float_as_uint(eps) >> 23) - 127) >> 1 : -127;
    return ex == 128 || (ex == -127 && eps == 0.0f && top == 0.0f) ? 0 : max(ex, least);
}

// Workgroup b of the set takes token blocks b, b + blocks, ...
template <typename E, Pairing P, bool NORM, bool BWD>
__device__ __forceinline__ void rope_body(const KArgs &k, float2 *angles, float *line) {
    constexpr int VEC = Chunk<E>::VEC;
    const RopeArgs &a = k.a;
    const int which = blockIdx.x >= k.blocks[0];
    const RopeSet &s = a.set[which];
    const uint32_t b0 = blockIdx.x - (which ? k.blocks[0] : 0), nb = k.blocks[which];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int gs = 1 << k.gs_log, c = lane & (gs - 1), nc = a.d / VEC;
    const int per_wave = 64 >> k.gs_log;
    const int half = a.rot >> 1, H = s.heads;
    const bool live = c < nc;
    const int base = c * VEC;  // the lane's first channel
    const float inv_d = 1.0f / (float)a.d;

    // what stays with the lane: weights, the partner's chunk
    float w[VEC], wp[VEC], acc[VEC];
    int partner = 0;
    bool low = true;  // the lane holds first channels of its pairs
    if (P == kHalf) {
        const int hc = half / VEC;
        low = c < hc;
        partner = low ? lane + hc : lane - hc;
        if (c >= 2 * hc) partner = lane;
    }
    // half layout, angles of a chunk: in order (bf16: 64 bytes a lane, whose reads conflict half of the LDS' time), or
    // with the norm forward in pieces of two pairs, a piece of all chunks side by side.  4 x 4099 tokens of 20
    // heads of 128: 44.7 us in order, 40.8 in pieces; the norm's backward 51.7 in order, 56 in pieces, and without
    // the norm 2 x 8193 tokens of 32 heads of 64 22.5 and 23.3
    constexpr bool PIECES = P == kHalf && NORM && !BWD;
    const int nh = half / VEC, piece = PIECES ? 2 * nh : 2;
    const int angles_at = P == kHalf && base < 2 * half ? (low ? c : c - nh) * (PIECES ? 2 : VEC) : 0;
    // interleaved: whole chunks are rotated or not; the lane's chunk is
    const bool rot_whole = a.rot > 0 && a.rot % VEC == 0, rotated = base < a.rot;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        acc[e] = 0.0f;
        w[e] = NORM && s.w && live ? s.w[base + e] : 1.0f;
        wp[e] = 1.0f;
        if (NORM && !BWD && P == kHalf && s.w && live && base < 2 * half) wp[e] = s.w[low ? base + half + e : base - half + e];
    }

    const int64_t nblocks = (s.tokens + k.tb - 1) / k.tb;
    for (int64_t blk = b0; blk < nblocks; blk += nb) {
        const int64_t t0 = blk * k.tb;
        const int nt = (int)min((int64_t)k.tb, s.tokens - t0);
        // one 64-bit division a block; within it rows and columns are 32 bits (len <= 2^30)
        const int64_t row0 = t0 / s.len;
        const uint32_t col0 = (uint32_t)(t0 - row0 * s.len), len = (uint32_t)s.len;
        // rows that lie between a block's first token and its t-th
        auto rows_on = [&](int t) { return len >= kMaxTok ? (uint32_t)(col0 + t >= len) : (col0 + t) / len; };
        const bool near = k.near[which] && col0 + nt <= len;  // one row, 32-bit offsets from its first token
        // element `rest` of the t-th token
        auto place = [&](const E *p, int64_t row_stride, int64_t tok_stride, int t, uint32_t rest) {
            const E *first = p + row0 * row_stride + (int64_t)col0 * tok_stride;
            if (near) return first + ((uint32_t)t * (uint32_t)tok_stride + rest);
            const uint32_t over = rows_on(t);
            return p + (row0 + over) * row_stride + (int64_t)(col0 + t - over * len) * tok_stride + rest;
        };
        const int units = nt * H, stride = 4 * per_wave;
        struct Unit {
            u32x4 raw, x;
            E *to;
            int t;
            bool on;
        };
        auto fetch = [&](int u0) {
            Unit r;
            const int u = u0 + (lane >> k.gs_log);
            r.on = live && u < units;
            r.t = !r.on || nt == 1 ? 0 : H == 1 ? u : (int)__umulhi((uint32_t)u, k.h_mul[which]);
            const uint32_t rest = r.on ? (uint32_t)(u - r.t * H) * a.d + base : 0;
            r.raw = r.x = u32x4{0, 0, 0, 0};
            r.to = const_cast<E *>(place((const E *)s.out, s.out_row, s.out_tok, r.t, rest));
            if (r.on) {
                r.raw = *reinterpret_cast<const u32x4 *>(place((const E *)s.in, s.in_row, s.in_tok, r.t, rest));
                if (NORM && BWD) r.x = *reinterpret_cast<const u32x4 *>(place((const E *)s.x, s.x_row, s.x_tok, r.t, rest));
            }
            return r;
        };
        // what the norm's forward multiplies by rstd comes last: the rotation is linear
        auto work = [&](const Unit &r) {
            float v[VEC], o[VEC];
            u32x4 raw = r.raw, xraw = r.x;
            float rstd = 1.0f, back = 1.0f;  // of the head as it is worked on, and as it is given
            if (NORM) {
                float xv[VEC], sum = 0.0f;
                Chunk<E>::get(BWD ? xraw : raw, xv);
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum = fmaf(xv[e], xv[e], sum);
                sum = group_sum(sum, k.gs_log);
                float mean = fmaf(sum, inv_d, a.eps);
                const bool odd = __float_as_uint(mean) - kLeastMean > kMostMean - kLeastMean;
                int ex = 0;  // the head is worked on as 2^-ex of itself
                if (__builtin_expect(__any(odd), 0)) {
                    const int own = head_exponent<VEC>(xv, k.gs_log, a.eps);
                    ex = odd ? own : 0;
                    sum = 0.0f;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        xv[e] = ldexpf(xv[e], -ex);
                        sum = fmaf(xv[e], xv[e], sum);
                    }
                    mean = fmaf(group_sum(sum, k.gs_log), inv_d, ldexpf(a.eps, -2 * ex));
                    (BWD ? xraw : raw) = Chunk<E>::put(xv);  // (exactly, but for what is nothing next to the largest)
                }
                // to one step of fp32; units that are not there count nothing, with an eps of 0, too
                rstd = r.on ? __builtin_amdgcn_rsqf(mean) : 0.0f;
                back = ldexpf(rstd, -ex);
            }
            Chunk<E>::get(raw, v);
            if (NORM && !BWD) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[e] *= w[e];
            }
            const float2 *row_angles = angles + r.t * half;
            if (P == kInter) {
                const int j0 = base >> 1;
                if (rot_whole) {
                    const float2 *cs = row_angles + (rotated ? j0 : 0);
#pragma unroll
                    for (int e = 0; e < VEC; e += 2) {
                        o[e] = v[e] * cs[e / 2].x - v[e + 1] * cs[e / 2].y;
                        o[e + 1] = v[e] * cs[e / 2].y + v[e + 1] * cs[e / 2].x;
                    }
                    if (a.rot < a.d) {
#pragma unroll
                        for (int e = 0; e < VEC; ++e) o[e] = rotated ? o[e] : v[e];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < VEC; e += 2) {
                        o[e] = v[e];
                        o[e + 1] = v[e + 1];
                        if (j0 + e / 2 < half) {
                            const float2 cs = row_angles[j0 + e / 2];
                            o[e] = v[e] * cs.x - v[e + 1] * cs.y;
                            o[e + 1] = v[e] * cs.y + v[e + 1] * cs.x;
                        }
                    }
                }
            } else if (P == kHalf) {
                u32x4 praw;
#pragma unroll
                for (int i = 0; i < 4; ++i) praw[i] = (uint32_t)__shfl(raw[i], partner, 64) ^ (low ? Chunk<E>::SIGNS : 0u);
                float pv[VEC];
                Chunk<E>::get(praw, pv);
                if (half > 0) {
                    const float2 *mine = row_angles + angles_at;
#pragma unroll
                    for (int e = 0; e < VEC; e += 2) {
                        const f32x4 cs = *reinterpret_cast<const f32x4 *>(mine + (e >> 1) * piece);
                        if (NORM && !BWD) pv[e] *= wp[e], pv[e + 1] *= wp[e + 1];
                        o[e] = fmaf(pv[e], cs[1], v[e] * cs[0]);
                        o[e + 1] = fmaf(pv[e + 1], cs[3], v[e + 1] * cs[2]);
                    }
                }
                if (a.rot < a.d) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) o[e] = rotated ? o[e] : v[e];
                }
            } else {
                float *mine = line + wave * (64 * VEC) + (lane >> k.gs_log << k.gs_log) * VEC;
#pragma unroll
                for (int e = 0; e < VEC; ++e) mine[base + e] = v[e];
                __builtin_amdgcn_wave_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const int i = base + e;
                    o[e] = v[e];
                    if (i < 2 * half) {
                        const bool lo = i < half;
                        const float2 cs = row_angles[lo ? i : i - half];
                        const float q = mine[lo ? i + half : i - half];
                        o[e] = lo ? v[e] * cs.x - q * cs.y : v[e] * cs.x + q * cs.y;
                    }
                }
                __builtin_amdgcn_wave_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
            if (NORM && !BWD) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) o[e] *= rstd;
            }
            if (NORM && BWD) {
                float xv[VEC], dot = 0.0f;
                Chunk<E>::get(xraw, xv);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    xv[e] *= rstd;
                    acc[e] = fmaf(o[e], xv[e], acc[e]);  // lanes that are off hold zeros
                    o[e] *= w[e];
                    dot = fmaf(o[e], xv[e], dot);
                }
                dot = group_sum(dot, k.gs_log) * -inv_d;
#pragma unroll
                for (int e = 0; e < VEC; ++e) o[e] = back * fmaf(xv[e], dot, o[e]);
            }
            // past the caches' way of keeping what was written last: 2 x 8193 tokens of 32 heads 26.8 -> 24.2 us,
            // 128 x 256 of 16 heads in fp32 25.5 -> 21.6
            if (r.on) __builtin_nontemporal_store(Chunk<E>::put(o), reinterpret_cast<u32x4 *>(r.to));
        };
        // every lane of a wave makes the same number of turns: the shuffles need them all.  Two units are
        // worked on while two are on their way, the first two from before the angles on
        int u0 = wave * per_wave;
        Unit r0 = fetch(u0), r1 = fetch(u0 + stride);
        for (int i = tid; i < nt * half; i += kThreads) {
            const int t = i / half, j = i - t * half;
            const uint32_t over = near ? 0 : rows_on(t);
            const int64_t pos = s.pos[(row0 + over) * s.pos_stride + (col0 + t - over * len)];
            const float2 cs = turn((uint64_t)pos * a.steps[j]);
            const int to = PIECES ? i - j + ((j % VEC) >> 1) * piece + 2 * (j / VEC) + (j & 1) : i;
            angles[to] = float2{cs.x * a.amplitude, (BWD ? -cs.y : cs.y) * a.amplitude};
        }
        __syncthreads();
        while (u0 < units) {
            u0 += 2 * stride;
            const Unit n0 = fetch(u0), n1 = fetch(u0 + stride);
            work(r0);
            work(r1);
            r0 = n0;
            r1 = n1;
        }
        __syncthreads();
    }
    if (NORM && BWD) {
        if (!s.dw) return;
        // groups of a wave, then waves, in a fixed order
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            for (int m = gs; m < 64; m <<= 1) acc[e] += __shfl_xor(acc[e], m, 64);
        if (lane < nc) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) line[wave * 256 + base + e] = acc[e];
        }
        __syncthreads();
        if (tid < a.d)
            k.part[(int64_t)blockIdx.x * a.d + tid] = (line[tid] + line[256 + tid]) + (line[512 + tid] + line[768 + tid]);
    }
}

template <typename E, Pairing P, bool NORM, bool BWD>
__global__ __launch_bounds__(kThreads, 4) void rope_kernel(KArgs k) {
    __shared__ __attribute__((aligned(16))) float2 angles[kMaxTok * 128];
    __shared__ float line[4 * 64 * Chunk<E>::VEC > 1024 ? 4 * 64 * Chunk<E>::VEC : 1024];
    rope_body<E, P, NORM, BWD>(k, angles, line);
}

// dw = sum of the workgroups' parts in fp64: 16 columns a workgroup, 64 threads each
__global__ __launch_bounds__(1024) void rope_dw_kernel(const float *part0, int n0, float *dw0, const float *part1, int n1,
                                                       float *dw1, int d) {
    __shared__ double sums[1024];
    const float *part = blockIdx.y ? part1 : part0;
    float *dw = blockIdx.y ? dw1 : dw0;
    const int n = blockIdx.y ? n1 : n0;
    if (!dw) return;
    const int col = blockIdx.x * 16 + (threadIdx.x & 15), r0 = threadIdx.x >> 4;
    double sum = 0.0;
    if (col < d) {
#pragma unroll 8
        for (int r = r0; r < n; r += 64) sum += (double)part[(int64_t)r * d + col];
    }
    sums[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x < 16 && col < d) {
        for (int i = 1; i < 64; ++i) sum += sums[threadIdx.x + 16 * i];
        dw[col] = (float)sum;
    }
}

// Tokens per workgroup and workgroups per set
void plan(const RopeArgs &a, bool bwd, KArgs *k) {
    const int64_t all = a.set[0].tokens + a.set[1].tokens;
    int tb = 1;
    for (int i = 0; i < 2; ++i)
        k->h_mul[i] = a.set[i].heads > 1 ? (uint32_t)(((uint64_t(1) << 32) + a.set[i].heads - 1) / a.set[i].heads) : 0;
    // (with more heads a workgroup has one token, and h_mul does not count)
    while (tb < kMaxTok && a.set[0].heads <= 8192 && a.set[1].heads <= 8192 && all / (2 * tb) >= 2048) tb *= 2;
    k->tb = tb;
    const int64_t most = int64_t(1) << 24;  // 16 tokens of them, and a token's heads, stay below 2^30 elements
    for (int i = 0; i < 2; ++i) {
        const RopeSet &t = a.set[i];
        k->near[i] = t.in_tok < most && t.x_tok < most && t.out_tok < most && (int64_t)t.heads * a.d < most;
    }
    const int chunks = a.d / (a.bf16 ? 8 : 4);
    k->gs_log = 0;
    while ((1 << k->gs_log) < chunks) ++k->gs_log;
    for (int i = 0; i < 2; ++i) {
        const int64_t blocks = a.set[i].heads > 0 ? (a.set[i].tokens + tb - 1) / tb : 0;
        const int64_t most = bwd && a.norm ? 1024 : (int64_t)1 << 20;
        k->blocks[i] = (uint32_t)(blocks < most ? blocks : most);
    }
}

template <typename E, bool NORM, bool BWD>
void launch(const KArgs &k, hipStream_t s) {
    const dim3 grid(k.blocks[0] + k.blocks[1]);
    const int half = k.a.rot / 2;
    if (k.a.interleaved)
        rope_kernel<E, kInter, NORM, BWD><<<grid, kThreads, 0, s>>>(k);
    else if (half % Chunk<E>::VEC == 0)
        rope_kernel<E, kHalf, NORM, BWD><<<grid, kThreads, 0, s>>>(k);
    else
        rope_kernel<E, kSplit, NORM, BWD><<<grid, kThreads, 0, s>>>(k);
}

template <bool BWD>
hipError_t launch_all(const KArgs &k, hipStream_t s) {
    if (k.blocks[0] + k.blocks[1] == 0) return hipSuccess;
    if (k.a.bf16)
        k.a.norm ? launch<uint16_t, true, BWD>(k, s) : launch<uint16_t, false, BWD>(k, s);
    else
        k.a.norm ? launch<float, true, BWD>(k, s) : launch<float, false, BWD>(k, s);
    return hipGetLastError();
}

}  // namespace

size_t rope_bwd_workspace(const RopeArgs &a) {
    if (!a.norm) return 0;
    KArgs k{};
    plan(a, true, &k);
    return (size_t)(k.blocks[0] + k.blocks[1]) * a.d * sizeof(float);
}

hipError_t launch_rope_fwd(const RopeArgs &a, hipStream_t s) {
    KArgs k{};
    k.a = a;
    plan(a, false, &k);
    return launch_all<false>(k, s);
}

hipError_t launch_rope_bwd(const RopeArgs &a, void *ws, hipStream_t s) {
    KArgs k{};
    k.a = a;
    plan(a, true, &k);
    k.part = (float *)ws;
    hipError_t e = launch_all<true>(k, s);
    if (e != hipSuccess || !(a.set[0].dw || a.set[1].dw)) return e;
    rope_dw_kernel<<<dim3((a.d + 15) / 16, 2), 1024, 0, s>>>(k.part, (int)k.blocks[0], a.set[0].dw,
                                                         k.part + (int64_t)k.blocks[0] * a.d, (int)k.blocks[1],
                                                         a.set[1].dw, a.d);
    return hipGetLastError();
}

}  // namespace evo

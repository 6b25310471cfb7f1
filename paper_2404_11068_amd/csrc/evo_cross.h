// evo_cross.h -- internal launch interface of the attention to states of
// another length, and what its kernels share (public ABI: include/evo_cross_attn.h).
//
// The G = H / Hk query heads of one key head and their Lq tokens are one axis
// of M = Lq * G rows x = t * G + g: a unit (row n of the batch, key head hk) is
// then a plain attention of M queries to Lk keys, a single token of many heads
// fills a tile, and the sums of shared key heads' gradients run along x.
//
// Matrix products are 32x32 tiles; of a result, lane l holds column l % 32 and,
// with half h = l / 32, in register i row 8 (i / 4) + 4 h + i % 4.  A product
// over those rows takes the registers as they are when the other operand's
// contraction slots are read in the same order (`col` below).
#pragma once

#include "evo_frag.h"

namespace evo {

struct CrArgs {
    const void *q, *k, *v, *gate, *bias;
    const uint8_t *mask;
    void *out;
    float *lse;
    // backward
    const void *dout;
    void *da;        // sigmoid(gate) * dout, contiguous [N, Lq, H, d] (with a gate)
    float *dsum;     // [N, Hk, M]
    void *dq, *dk, *dv, *dgate, *dbias;
    // partial sums over splits
    float *part;     // [splits][rows][d]
    float2 *part_ml; // [splits][rows]: running maximum and sum
    int64_t N, rpb, q_row, q_tok, k_row, k_tok, o_row, o_tok;
    int Lq, Lk, M, H, Hk, G, D;
    uint32_t g_mul, g_shift;  // x / G = x * g_mul >> g_shift for x < 2^31
    int tiles, splits, per_split, ntiles;  // tiles of rows, splits of the other axis, its tiles
    float scale;
    int bf16;
};

// plan of a call: splits and workspace
struct CrPlan {
    int fwd_splits, kv_splits, q_splits, bias_chunks;
    bool few;  // forward: a workgroup's waves share its rows and take turns with the keys
    size_t fwd_part, fwd_ml, fwd_total;
    size_t bwd_da, bwd_part, bwd_total;
};
CrPlan cross_plan(const CrArgs &a, bool has_gate, bool has_bias);

hipError_t launch_cross_fwd(CrArgs a, const CrPlan &p, void *ws, hipStream_t s);
hipError_t launch_cross_bwd(CrArgs a, const CrPlan &p, void *ws, hipStream_t s);
// sums the fp32 partials [splits][unit][len][D] into out (strides; G heads per unit row as in x)
hipError_t launch_cross_sum(const CrArgs &a, const float *part, int splits, int64_t units, int len, int group,
                            void *out, int64_t row, int64_t tok, hipStream_t s);

#if defined(__HIPCC__)
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// A query whose largest logit with its bias is below this has no key left: a
// bias of the type's lowest value everywhere is a mask, like -infinity.
constexpr float kNoKey = -1e30f;

// Element type of the tiles: what a lane reads, and the products over it
template <typename T> struct Ty;

template <> struct Ty<bf16_t> {
    using E = uint16_t;
    using Frag = bf16x8;
    static constexpr int VEC = 8;   // elements per 16 bytes
    static constexpr int KS = 16;   // contraction of one product
    static constexpr int PAD = 16;  // of an LDS row: 8 lanes' 16-byte reads of 8 rows, and 4 rows of a transposed read, touch each bank once
    __device__ __forceinline__ static Frag row(const E *p) { return *reinterpret_cast<const bf16x8 *>(p); }
    __device__ __forceinline__ static void mma(f32x16 &acc, const Frag &a, const Frag &b) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0);
    }
    // operand whose row is column c0 + lane % 32 of the tile, contraction rows r0 + 8 (e / 4) + 4 h + e % 4
    __device__ __forceinline__ static Frag col(const E *tile, int stride, int r0, int c0, int lane) {
        const int i = lane & 15, g = lane >> 4;
        const E *src = tile + (r0 + 4 * (g >> 1) + (i >> 2)) * stride + c0 + 16 * (g & 1) + 4 * (i & 3);
        const short4tr lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4tr *)(src));
        const short4tr hi =
            __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4tr *)(src + 8 * stride));
        const short8tr both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(bf16x8, both);
    }
    __device__ __forceinline__ static Frag pack(const f32x16 &p, int s) {
        Frag f;
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (__bf16)p[8 * s + e];
        return f;
    }
    __device__ __forceinline__ static float f(E x) { return bf2f(x); }
    // x where it counts: the choice is made on the bits, before any arithmetic sees what lies there
    __device__ __forceinline__ static float f(E x, bool keep) { return bf2f(keep ? x : (E)0); }
    __device__ __forceinline__ static E e(float x) { return f2bf(x); }
};

template <> struct Ty<float> {
    using E = float;
    using Frag = f32x4;
    static constexpr int VEC = 4, KS = 8, PAD = 4;
    __device__ __forceinline__ static Frag row(const E *p) { return *reinterpret_cast<const f32x4 *>(p); }
    __device__ __forceinline__ static void mma(f32x16 &acc, const Frag &a, const Frag &b) {
#pragma unroll
        for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], acc, 0, 0, 0);
    }
    __device__ __forceinline__ static Frag col(const E *tile, int stride, int r0, int c0, int lane) {
        const E *src = tile + (r0 + 4 * (lane >> 5)) * stride + c0 + (lane & 31);
        return Frag{src[0], src[stride], src[2 * stride], src[3 * stride]};
    }
    __device__ __forceinline__ static Frag pack(const f32x16 &p, int s) {
        return Frag{p[4 * s], p[4 * s + 1], p[4 * s + 2], p[4 * s + 3]};
    }
    __device__ __forceinline__ static float f(E x) { return x; }
    __device__ __forceinline__ static float f(E x, bool keep) { return __uint_as_float(keep ? __float_as_uint(x) : 0u); }
    __device__ __forceinline__ static E e(float x) { return x; }
};

// combined over the lane halves (lanes l and l + 32 hold parts of one column)
__device__ __forceinline__ float half_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ int token_of(const CrArgs &a, int x) {
    return a.G == 1 ? x : (int)(((uint64_t)(uint32_t)x * a.g_mul) >> a.g_shift);
}

// Which of the KT keys from k0 on are kept, one bit each, the same in all lanes
template <int KT> struct KeyBits {
    static constexpr int W = (KT + 63) / 64;
    uint64_t w[W];
    // the lane's mask bytes, requested one step ahead of their use
    struct Bytes { uint8_t b[W]; };
    __device__ __forceinline__ static Bytes request(const uint8_t *mask_row, int k0, int end, int lane) {
        Bytes x;
#pragma unroll
        for (int j = 0; j < W; ++j) {
            const int key = k0 + 64 * j + lane;
            const bool in = key < end && 64 * j + lane < KT;
            x.b[j] = in ? (mask_row ? mask_row[key] : (uint8_t)1) : (uint8_t)0;
        }
        return x;
    }
    __device__ __forceinline__ void set(const Bytes &x) {
#pragma unroll
        for (int j = 0; j < W; ++j) w[j] = __ballot(x.b[j] != 0);
    }
    __device__ __forceinline__ bool any() const {
        uint64_t o = w[0];
#pragma unroll
        for (int j = 1; j < W; ++j) o |= w[j];
        return o != 0;
    }
    __device__ __forceinline__ bool get(int r) const {
        if (W == 1) return (w[0] >> r) & 1;
        return ((r < 64 ? w[0] : w[W - 1]) >> (r & 63)) & 1;
    }
    __device__ __forceinline__ uint32_t sub(int s) const { return (uint32_t)(w[s >> 1] >> (32 * (s & 1))); }
};

// A tile of ROWS tokens of DP channels on its way from memory to LDS, 16 bytes
// a thread at a time.  Rows and channels that are not there are read from a
// valid address and written as zeros (NaN or infinity in a masked place stays
// outside of every product).
template <typename T, int DP, int ROWS, int THREADS> struct Stage {
    using E = typename Ty<T>::E;
    static constexpr int CPR = DP / Ty<T>::VEC, N = ROWS * CPR / THREADS, STR = DP + Ty<T>::PAD;
    static_assert(ROWS * CPR % THREADS == 0, "whole chunks");
    u32x4 v[N];
    template <class Row, class Keep>
    __device__ __forceinline__ void load(const E *safe, int D, int tid, Row row, Keep keep) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = tid + THREADS * i, r = at / CPR, c = at % CPR * Ty<T>::VEC;
            const E *p = keep(r) && c < D ? row(r) + c : safe;
            v[i] = *reinterpret_cast<const u32x4 *>(p);
        }
    }
    template <class Keep> __device__ __forceinline__ void store(E *tile, int D, int tid, Keep keep) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = tid + THREADS * i, r = at / CPR, c = at % CPR * Ty<T>::VEC;
            const u32x4 z = {0, 0, 0, 0};
            *reinterpret_cast<u32x4 *>(tile + r * STR + c) = keep(r) && c < D ? v[i] : z;
        }
    }
};

// the lane's row of a 32-row block as operand: channels KS kk + (KS / 2) h ..
template <typename T, int DP>
__device__ __forceinline__ void load_rows(typename Ty<T>::Frag (&f)[DP / Ty<T>::KS], const typename Ty<T>::E *row, int D, bool on,
                                          int h) {
#pragma unroll
    for (int kk = 0; kk < DP / Ty<T>::KS; ++kk) {
        const int c = Ty<T>::KS * kk + Ty<T>::KS / 2 * h;
        const u32x4 z = {0, 0, 0, 0};
        const u32x4 x = *reinterpret_cast<const u32x4 *>(row + (c < D ? c : 0));
        f[kk] = __builtin_bit_cast(typename Ty<T>::Frag, on && c < D ? x : z);
    }
}

// Four consecutive values of a row that may start at any element, as bits of floats
__device__ __forceinline__ u32x4 load4(const uint16_t *p) {
    uint32_t w[2];
    __builtin_memcpy(w, p, 8);
    return u32x4{w[0] << 16, w[0] & 0xffff0000u, w[1] << 16, w[1] & 0xffff0000u};
}
__device__ __forceinline__ u32x4 load4(const float *p) {
    u32x4 x;
    __builtin_memcpy(&x, p, 16);
    return x;
}

// The lane's bias row: its values for the 16 keys of a block that its registers
// hold.  A block is read in fours of keys; where it ends behind the row, that is
// the next row's beginning, which does not count, and only where it ends behind
// the tensor single values are read.
template <typename T> struct BiasRow {
    using E = typename Ty<T>::E;
    const E *row;
    int room;  // values from the row's start to the tensor's end
    __device__ __forceinline__ BiasRow(const CrArgs &a, int64_t r) {
        const int64_t left = (a.N / a.rpb * a.H * a.Lq - r) * a.Lk;
        row = (const E *)a.bias + r * a.Lk;
        room = left < 0x7fffffff ? (int)left : 0x7fffffff;
    }
    // k0: the block's first key; bits: its kept keys from 4 h on.  What is not kept is 0.
    __device__ __forceinline__ void get(float (&out)[16], int k0, int h, uint32_t bits, bool whole) const {
        u32x4 w[4];
        if (__all(k0 + 32 <= room)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = load4(row + k0 + 8 * i + 4 * h);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const bool keep = (bits >> (8 * (i / 4) + i % 4)) & 1;
                w[i / 4][i % 4] = __float_as_uint(Ty<T>::f(row[keep ? k0 + 8 * (i / 4) + 4 * h + i % 4 : 0]));
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const bool keep = whole || ((bits >> (8 * (i / 4) + i % 4)) & 1);
            out[i] = __uint_as_float(keep ? w[i / 4][i % 4] : 0u);
        }
    }
};
#endif

}  // namespace evo

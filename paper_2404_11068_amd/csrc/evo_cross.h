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
    void *da;        // sigmoid(gate) * dout, contiguous [N, Lq, H, d] (with a gate or a bias)
    f32x4 *stats;    // [N, Hk, M]: (base, D, rest) of a query, base and rest: what its probabilities are formed with
    void *dq, *dk, *dv, *dgate, *dbias;
    // partial sums over splits
    float *part;     // [splits][rows][d]
    float2 *part_ml; // [splits][rows]: reference (hi) and sum
    float *part_lo;  // [splits][rows]: lo
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
    bool brief;       // forward: all keys at once, workgroups walk over the rows of the batch
    int brief_chunks; // of the rows of a bias plane
    bool brief_one;   // a wave a row of the batch, not a workgroup
    size_t fwd_part, fwd_ml, fwd_lo, fwd_total;
    size_t bwd_da, bwd_part, bwd_total;
};
CrPlan cross_plan(const CrArgs &a, bool has_gate, bool has_bias);

hipError_t launch_cross_fwd(CrArgs a, const CrPlan &p, void *ws, hipStream_t s);
hipError_t launch_cross_short(CrArgs a, const CrPlan &p, hipStream_t s);
hipError_t launch_cross_bwd(CrArgs a, const CrPlan &p, void *ws, hipStream_t s);
#if defined(__HIPCC__)
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// A query whose largest logit (natural, with its bias) is not above this has no key left: a
// bias of the type's lowest value everywhere is a mask, like -infinity.
constexpr float kNoKey = -1e30f;

// What probabilities are formed against, in units of base-2 logarithms: of a logit s that is exp2(s to2 - hi - lo).
// hi is a whole number at or above the largest s to2, and lo zero, so that rescaling is exact.  From
// 2^22 on the rounding of that product is no longer small against one, and would be left over in the exponent
// (128 at 1e10): there hi is the rounded product and lo the rest of it, so that the largest logit gives 1.
// The checks for it take up to 2.5% of long calls (64 channels: 172 us without, 177 with them).
struct Ref {
    float hi, lo;
};
constexpr float kFar = 4194304.0f, kLargest = 3.402823466e38f;
__device__ __forceinline__ Ref reference(float top, float to2) {
    const float x = top * to2;
    const bool far = fabsf(x) >= kFar;
    const float hi = far ? fminf(x, kLargest) : __builtin_ceilf(x);
    return Ref{hi, far ? fmaf(top, to2, -hi) : 0.0f};
}
// r is above s
__device__ __forceinline__ bool above(Ref r, Ref s) { return r.hi > s.hi || (r.hi == s.hi && r.lo > s.lo); }
// natural logarithm of a sum of such probabilities
__device__ __forceinline__ float log_of(float sum, Ref r) {
    const float l = __builtin_amdgcn_logf(sum);
    return sum == 0.0f ? -__builtin_inff() : r.lo == 0.0f ? (l + r.hi) * kLn2 : fmaf(r.hi, kLn2, fmaf(r.lo, kLn2, l * kLn2));
}

// Element type of the tiles: what a lane reads, and the products over it
template <typename T> struct Ty;

template <> struct Ty<bf16_t> {
    using E = uint16_t;
    using Frag = bf16x8;
    static constexpr int VEC = 8;   // elements per 16 bytes
    static constexpr int KS = 16;   // contraction of one product
    __device__ __forceinline__ static void mma(f32x16 &acc, const Frag &a, const Frag &b) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0);
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
    static constexpr int VEC = 4, KS = 8;
    __device__ __forceinline__ static void mma(f32x16 &acc, const Frag &a, const Frag &b) {
#pragma unroll
        for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], acc, 0, 0, 0);
    }
    __device__ __forceinline__ static Frag pack(const f32x16 &p, int s) {
        return Frag{p[4 * s], p[4 * s + 1], p[4 * s + 2], p[4 * s + 3]};
    }
    __device__ __forceinline__ static float f(E x) { return x; }
    __device__ __forceinline__ static float f(E x, bool keep) { return __uint_as_float(keep ? __float_as_uint(x) : 0u); }
    __device__ __forceinline__ static E e(float x) { return x; }
};

// A tile of rows of DP channels in LDS, and the two ways it becomes an operand:
//   row(tile, r, kk, h): row r, channels KS kk + KS / 2 h and on
//   col(tile, r0, c0, lane): column c0 + lane % 32, rows r0 + 8 (e / 4) + 4 h + e % 4,
//     the order in which a product's registers hold its rows
template <typename T, int DP> struct Tile;

// The 16-byte chunk k of row r sits at chunk k ^ f(r), so that of 64 four-byte banks 16 lanes reading one
// chunk of 16 rows, 16 lanes writing neighbouring chunks, and 32 lanes of bf16's transposing read (64 bytes
// of four rows) each touch every one once.  Padded rows can have one of the first and the last only (and
// cannot be copied to without registers): at 32 bytes of padding conflicts took 40% of the LDS cycles of
// the forward at 128 channels.
template <int DP> struct Tile<bf16_t, DP> {
    using E = uint16_t;
    static constexpr int CH = DP / 8;
    __device__ __forceinline__ static int f(int r) {
        const int low = (r >> 2) & 3;
        return DP == 32 ? low : DP == 64 ? ((r >> 1) & 1) << 2 | low : (r & 3) << 2 | low;
    }
    __device__ __forceinline__ static int at(int r, int chunk) { return r * DP + ((chunk ^ f(r)) << 3); }
    __device__ __forceinline__ static bf16x8 row(const E *tile, int r, int kk, int h) {
        return *reinterpret_cast<const bf16x8 *>(tile + at(r, 2 * kk + h));
    }
    __device__ __forceinline__ static bf16x8 col(const E *tile, int r0, int c0, int lane) {
        const int i = lane & 15, g = lane >> 4;
        const int r = 4 * (g >> 1) + (i >> 2), chunk = (c0 >> 3) + 2 * (g & 1) + ((i & 3) >> 1), low = 4 * (i & 1);
        const E *lo_at = tile + r0 * DP + at(r, chunk) + low, *hi_at = tile + r0 * DP + at(r + 8, chunk) + low;
        const short4tr lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4tr *)(lo_at));
        const short4tr hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4tr *)(hi_at));
        const short8tr both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(bf16x8, both);
    }
};

// fp32: a column is read by 4-byte reads, 32 lanes a row and the two lane halves four rows apart; f is the
// same for four rows, whose reads differ by a constant then.  Rows are read with conflicts, once for 256
// cycles of matrix instructions.
template <int DP> struct Tile<float, DP> {
    using E = float;
    static constexpr int CH = DP / 4;
    __device__ __forceinline__ static int f(int r) {
        return DP == 32 ? ((r >> 2) & 3) << 1 : ((r >> 2) & 1) << 3 | ((r >> 3) & 1) << 1;
    }
    __device__ __forceinline__ static int at(int r, int chunk) { return r * DP + ((chunk ^ f(r)) << 2); }
    __device__ __forceinline__ static f32x4 row(const E *tile, int r, int kk, int h) {
        return *reinterpret_cast<const f32x4 *>(tile + at(r, 2 * kk + h));
    }
    __device__ __forceinline__ static f32x4 col(const E *tile, int r0, int c0, int lane) {
        const int c = c0 + (lane & 31);
        const E *src = tile + at(r0 + 4 * (lane >> 5), c >> 2) + (c & 3);
        return f32x4{src[0], src[DP], src[2 * DP], src[3 * DP]};
    }
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
    __device__ __forceinline__ bool all() const {
        static_assert(KT == 32 || KT == 64, "one word");
        return w[0] == (KT == 64 ? ~0ull : 0xffffffffull);
    }
    __device__ __forceinline__ bool get(int r) const {
        if (W == 1) return (w[0] >> r) & 1;
        return ((r < 64 ? w[0] : w[W - 1]) >> (r & 63)) & 1;
    }
    __device__ __forceinline__ uint32_t sub(int s) const { return (uint32_t)(w[s >> 1] >> (32 * (s & 1))); }
};

// Narrows the steps [t0, t1) of KT keys to those from the first kept key to the last
template <int KT, int THREADS>
__device__ __forceinline__ void kept_range(const uint8_t *mask_row, int Lk, int tid, int *lds, int &t0, int &t1) {
    const int end = min(t1 * KT, Lk);
    int lo = 0x7fffffff, hi = -1;
    for (int k = t0 * KT + tid * 16; k < end; k += THREADS * 16) {
        uint32_t any = 0;
        if (k + 16 <= end) {
            u32x4 w;
            __builtin_memcpy(&w, mask_row + k, 16);
            any = w[0] | w[1] | w[2] | w[3];
        } else {
            for (int i = k; i < end; ++i) any |= mask_row[i];
        }
        // 16 keys from a multiple of 16 on lie in one step
        if (any) {
            lo = min(lo, k);
            hi = k;
        }
    }
    for (int m = 1; m < 64; m <<= 1) {
        lo = min(lo, __shfl_xor(lo, m, 64));
        hi = max(hi, __shfl_xor(hi, m, 64));
    }
    if ((tid & 63) == 0) lds[2 * (tid >> 6)] = lo, lds[2 * (tid >> 6) + 1] = hi;
    __syncthreads();
    for (int w = 0; w < THREADS / 64; ++w) {
        lo = min(lo, lds[2 * w]);
        hi = max(hi, lds[2 * w + 1]);
    }
    __syncthreads();
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
    t1 = hi < 0 ? t0 : hi / KT + 1;
    if (hi >= 0) t0 = lo / KT;
}

// A tile of ROWS tokens of DP channels from memory to LDS, without registers in between: global_load_lds,
// 16 bytes a lane.  Rows and channels that are not there are copied from zeros (NaN or infinity in a masked
// place stays outside of every product).  The
// copies are counted by hand: copies_done_and_barrier() before a tile is read.
// (The compiler does not see them; its own waits on vector memory count in order
// and only get longer by them.)
// (M0 holds the LDS address.  It is a reserved register: the compiler keeps nothing in it across statements and
// does not take it as a clobber; nothing else in these kernels' code uses it.)
static __device__ const u32x4 kZeros[1] = {};  // what is not there is copied from here
__device__ __forceinline__ void copy16(const void *from, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(lds), "v"(from) : "memory");
}
__device__ __forceinline__ void copies_done_and_barrier() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory"); }

template <typename T, int DP, int ROWS, int THREADS> struct Copy {
    using E = typename Ty<T>::E;
    using L = Tile<T, DP>;
    static constexpr int N = ROWS * L::CH / THREADS;
    static_assert(ROWS * L::CH % THREADS == 0, "whole chunks");
    template <class Row, class Keep>
    __device__ __forceinline__ static void run(E *tile, bool whole, int D, int wave, int lane, Row row, Keep keep) {
        const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)(char *)tile + wave * 1024);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = wave * 64 + THREADS * i + lane, r = at / L::CH, c = ((at % L::CH) ^ L::f(r)) * Ty<T>::VEC;
            const E *p = row(r) + c;
            if (!whole) p = keep(r) && c < D ? p : (const E *)kZeros;
            copy16(p, lds + THREADS * i * 16);
        }
    }
};

// x where on, zeros elsewhere: by a mask, since a choice makes the compiler load x in a branch of its own
// and wait for it there, one load after the other
__device__ __forceinline__ u32x4 where(bool on, u32x4 x) {
    const uint32_t m = on ? 0xffffffffu : 0u;
    return x & u32x4{m, m, m, m};
}

// the lane's row of a 32-row block as operand: channels KS kk + (KS / 2) h ..
template <typename T, int DP>
__device__ __forceinline__ void load_rows(typename Ty<T>::Frag (&f)[DP / Ty<T>::KS], const typename Ty<T>::E *row, int D, bool on,
                                          int h) {
    u32x4 x[DP / Ty<T>::KS];
#pragma unroll
    for (int kk = 0; kk < DP / Ty<T>::KS; ++kk) {
        const int c = Ty<T>::KS * kk + Ty<T>::KS / 2 * h;
        x[kk] = *reinterpret_cast<const u32x4 *>(row + (c < D ? c : 0));
    }
#pragma unroll
    for (int kk = 0; kk < DP / Ty<T>::KS; ++kk)
        f[kk] = __builtin_bit_cast(typename Ty<T>::Frag, where(on && Ty<T>::KS * kk + Ty<T>::KS / 2 * h < D, x[kk]));
}

// Four consecutive values of a row that may start at any element
template <typename E> struct Four;
template <> struct Four<uint16_t> {
    uint32_t w[2];
    __device__ __forceinline__ uint32_t bits(int i) const { return i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16; }
    __device__ __forceinline__ void set(int i, uint16_t x) {
        w[i >> 1] = i & 1 ? (w[i >> 1] & 0xffffu) | (uint32_t)x << 16 : x;
    }
};
template <> struct Four<float> {
    uint32_t w[4];
    __device__ __forceinline__ uint32_t bits(int i) const { return w[i]; }
    __device__ __forceinline__ void set(int i, float x) { w[i] = __float_as_uint(x); }
};
template <typename E> __device__ __forceinline__ Four<E> load4(const E *p) {
    Four<E> x;
    __builtin_memcpy(&x, p, sizeof(x));
    return x;
}

// The lane's bias row: its values for the 32 keys of a block that its registers
// pair with.  A block is read in fours of keys; where it ends behind the row, that
// is the next row's beginning, which does not count, and only where it ends behind
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
    struct Raw { Four<E> x[4]; };
    __device__ __forceinline__ Raw request(int k0, int h) const {
        Raw r;
        if (__all(k0 + 32 <= room)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) r.x[i] = load4(row + k0 + 8 * i + 4 * h);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int key = k0 + 8 * (i / 4) + 4 * h + i % 4;
                r.x[i / 4].set(i % 4, row[key < room ? key : 0]);
            }
        }
        return r;
    }
    __device__ __forceinline__ static float value(const Raw &r, int i) { return __uint_as_float(r.x[i / 4].bits(i % 4)); }
};

// x where the key of register i is kept (bits of a block of 32 keys, the same in all lanes), else the
// float with the bits `other`: one instruction, its lane mask made by scalar ones.  The choice is one of
// bits, so that whatever x came to from a masked bias does not matter.
__device__ __forceinline__ float where_kept(uint32_t bits, int i, float x, uint32_t other) {
    const uint32_t lo = (bits >> (8 * (i / 4) + i % 4)) & 1, hi = (bits >> (8 * (i / 4) + 4 + i % 4)) & 1;
    const uint64_t lanes = (lo ? 0xffffffffull : 0) | (hi ? 0xffffffff00000000ull : 0);
    return __uint_as_float(__builtin_amdgcn_inverse_ballot_w64(lanes) ? __float_as_uint(x) : other);
}
constexpr uint32_t kMinusInf = 0xff800000u;

__device__ __forceinline__ float sigmoid(float x) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-x * kLog2e));  // both to about one step of fp32
}

// 16 channels of a token, c = 16 j and on, as the registers of a product hold them (x[0]: channels c + 4 h
// .. c + 4 h + 3, x[1]: c + 8 + 4 h ..), by 16-byte accesses.  In bf16 a lane reads 8 neighbours and the
// lane halves swap fours.
template <typename E> struct Sixteen;
template <> struct Sixteen<uint16_t> {
    Four<uint16_t> x[2];
    __device__ __forceinline__ void swap() {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const auto r = __builtin_amdgcn_permlane32_swap(x[0].w[i], x[1].w[i], false, false);
            x[0].w[i] = r[0];
            x[1].w[i] = r[1];
        }
    }
    // every lane of the wave takes part; rows that are not there are given a valid address
    __device__ __forceinline__ void load(const uint16_t *row, int c, int D, int h) {
        const u32x4 w = *reinterpret_cast<const u32x4 *>(row + (c + 8 * h < D ? c + 8 * h : 0));
        x[0].w[0] = w[0], x[0].w[1] = w[1], x[1].w[0] = w[2], x[1].w[1] = w[3];
    }
    __device__ __forceinline__ void arrange() { swap(); }  // after load: kept apart, so that it does not wait
    __device__ __forceinline__ void store(uint16_t *row, int c, int D, int h, bool on) {
        swap();
        if (on && c + 8 * h < D) *reinterpret_cast<u32x4 *>(row + c + 8 * h) = u32x4{x[0].w[0], x[0].w[1], x[1].w[0], x[1].w[1]};
    }
    __device__ __forceinline__ void set(int g, const float *v) {
#pragma unroll
        for (int i = 0; i < 2; ++i) x[g].w[i] = (uint32_t)f2bf(v[2 * i]) | (uint32_t)f2bf(v[2 * i + 1]) << 16;
    }
};
template <> struct Sixteen<float> {
    Four<float> x[2];
    __device__ __forceinline__ void load(const float *row, int c, int D, int h) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int at = c + 8 * g + 4 * h;
            const u32x4 w = *reinterpret_cast<const u32x4 *>(row + (at < D ? at : 0));
#pragma unroll
            for (int i = 0; i < 4; ++i) x[g].w[i] = w[i];
        }
    }
    __device__ __forceinline__ void arrange() {}
    __device__ __forceinline__ void store(float *row, int c, int D, int h, bool on) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int at = c + 8 * g + 4 * h;
            if (on && at < D) *reinterpret_cast<u32x4 *>(row + at) = u32x4{x[g].w[0], x[g].w[1], x[g].w[2], x[g].w[3]};
        }
    }
    __device__ __forceinline__ void set(int g, const float *v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[g].w[i] = __float_as_uint(v[i]);
    }
};
#endif

}  // namespace evo

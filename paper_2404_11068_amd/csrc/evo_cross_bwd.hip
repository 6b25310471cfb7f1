// evo_cross_bwd.hip -- attention to states of another length, backward
// (include/evo_cross_attn.h).  With P the probabilities, dA = sigmoid(g) dO:
//   D = sum over channels of dO O,   dP = dA V',   dS = P (dP - D)
//   dV = P' dA,  dK = dS' Q / sqrt d,  dQ = dS K / sqrt d,  dBias = sum over rows of dS
//
// P is formed again from the saved log-sum-exp, in each of three passes:
//   rows:  a wave owns 32 queries (lane = query) and walks the keys: dQ; before that
//          it forms D, dgate and dA of its queries, and leaves them for the others
//   keys:  a wave owns 32 keys (lane = key) and walks the queries: dK, dV
//   bias:  a workgroup owns 64 x 64 entries of one bias plane and walks the
//          rows that share it
//
// The passes are bound like the forward (at 64 channels the matrix units are busy 33 to 37% of
// the time, the vector units 52 to 53%): 2 x 4096 to 4096, 16 heads of 64, bf16, 525 us for all,
// 4096 to 8191, 16 heads of 128, 1200 us (800 TFLOP/s of the seven products).  One pass would save two
// products, and sum dQ over workgroups, by atomics or by partial sums of all of it.
//
// Every sum runs in a fixed order; where the tiles do not fill the GPU, the
// walked axis is split over workgroups, whose fp32 parts a last kernel sums.
#include "evo_cross.h"

namespace evo {
namespace {

constexpr int kThreads = 256;

// A log-sum-exp beyond this no longer holds the logarithm of the sum to 2^-14: fp32's steps there are 2^-13 and more.
// Such a query's wave walks the keys once more, before its pass, for the largest logit and the sum against it, and P is
// formed with those.  With a bias, P = exp(x - base) of a logit x, base = lse, or the largest x with 1 / sum
// multiplied onto D and dA, whose multiples all gradients are: nothing changes for the passes.  Without a bias (where
// dA may be dO itself), P = exp2((s - rest) scale log2 e + base) of s = q k', (base, rest) = (-lse log2 e, 0), or
// (-log2 sum, largest s); steps whose queries all have a rest of 0 leave it out.  Queries without keys: base = inf, -inf.
// With both as terms of every exponent the passes took 2% (64 channels) to 10% longer (32 channels with a bias).
constexpr float kFarLse = 1024.0f;

// dA as the later passes read it: what the first has written, or dO itself without gate and bias
struct DaView {
    int64_t row, tok;
};
__device__ __forceinline__ DaView da_view(const CrArgs &a) {
    return a.da ? DaView{(int64_t)a.Lq * a.H * a.D, (int64_t)a.H * a.D} : DaView{a.o_row, a.o_tok};
}

// ---------------------------------------------------------------------------
// keys: dK, dV
template <typename T, int DP> struct KeysShape {
    static constexpr bool WIDE = sizeof(typename Ty<T>::E) == 4;
    static constexpr int KEYS = 128, XT = WIDE || DP == 128 ? 32 : 64;
    static constexpr int TILE = XT * DP;
    // (bf16 at 64 channels with a bias spills 2 registers around its loop; addresses in scalar registers avoid it and take 44.9 us
    // where this takes 43.4, 2 x 1024 to 1024, 8 heads)
    static constexpr int WAVES = DP == 128 ? 1 : 2;  // per SIMD: the accumulators of 128 channels take half of its registers
};

template <typename T, int DP, bool BIAS>
__global__ __launch_bounds__(kThreads, (KeysShape<T, DP>::WAVES)) void cross_keys_kernel(CrArgs a) {
    using Y = Ty<T>;
    using E = typename Y::E;
    using Frag = typename Y::Frag;
    using LT = Tile<T, DP>;
    using S = KeysShape<T, DP>;
    constexpr int NK = DP / Y::KS, DT = DP / 32;
    __shared__ __attribute__((aligned(16))) E tiles[2][2][S::TILE];
    __shared__ __attribute__((aligned(16))) float stats[2][BIAS ? 2 : 3][S::XT];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    uint32_t u = xcd_unit32(blockIdx.x, gridDim.x);
    const int split = u % a.splits;
    u /= a.splits;
    const int tile = u % a.tiles;
    const uint32_t unit = u / a.tiles;
    const int64_t n = unit / a.Hk;
    const int hk = unit % a.Hk;
    const DaView dv = da_view(a);
    const E *qbase = (const E *)a.q + n * a.q_row + (int64_t)hk * a.G * a.D;
    const E *abase = (const E *)(a.da ? a.da : a.dout) + n * dv.row + (int64_t)hk * a.G * a.D;

    const int key = tile * S::KEYS + wave * 32 + (lane & 31), keyc = min(key, a.Lk - 1);
    const bool keep = key < a.Lk && (!a.mask || a.mask[n * a.Lk + key]);
    Frag kf[NK], vf[NK];
    const int64_t koff = n * a.k_row + (int64_t)keyc * a.k_tok + (int64_t)hk * a.D;
    load_rows<T, DP>(kf, (const E *)a.k + koff, a.D, keep, h);
    load_rows<T, DP>(vf, (const E *)a.v + koff, a.D, keep, h);
    const E *bias = BIAS ? (const E *)a.bias + (n / a.rpb * a.H + hk * a.G) * (int64_t)a.Lq * a.Lk + keyc : nullptr;

    f32x16 dk[DT], dvv[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) dk[i] = dvv[i] = zero16();
    const float to2 = a.scale * kLog2e;

    constexpr int NB = S::XT / 32, GP = 32 / Y::KS;
    using Cp = Copy<T, DP, S::XT, kThreads>;
    float2 stats_in = {};
    float rest_in = 0.0f;
    auto request = [&](int step) {
        const int x0 = step * S::XT;
        auto at = [&](int r, int64_t tok) {
            const int x = x0 + r, t = token_of(a, x);
            return (int64_t)t * tok + (int64_t)(x - t * a.G) * a.D;
        };
        const float *from = (const float *)(a.stats + (int64_t)unit * a.M + min(x0 + lane % S::XT, a.M - 1));
        if (tid < S::XT) stats_in = *reinterpret_cast<const float2 *>(from);
        if (!BIAS) rest_in = from[2];  // (all waves look whether there is one)
        const bool whole = a.D == DP && x0 + S::XT <= a.M;
        auto in = [&](int r) { return x0 + r < a.M; };
        Cp::run(tiles[step & 1][0], whole, a.D, wave, lane, [&](int r) { return qbase + at(r, a.q_tok); }, in);
        Cp::run(tiles[step & 1][1], whole, a.D, wave, lane, [&](int r) { return abase + at(r, dv.tok); }, in);
    };
    // the bias of a step's queries with the lane's key: the 32 keys of a query's row are neighbours
    E braw[BIAS ? NB : 1][16];
    auto request_bias = [&](int step) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int xb = step * S::XT + 32 * b;
            if (a.G == 1 && xb + 32 <= a.M) {
                const E *p = bias + (int64_t)(xb + 4 * h) * a.Lk;
#pragma unroll
                for (int i = 0; i < 16; ++i) braw[BIAS ? b : 0][i] = p[(int64_t)(8 * (i / 4) + i % 4) * a.Lk];
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int x = min(xb + 8 * (i / 4) + 4 * h + i % 4, a.M - 1), t = token_of(a, x);
                    braw[BIAS ? b : 0][i] = bias[((int64_t)(x - t * a.G) * a.Lq + t) * a.Lk];
                }
            }
        }
    };
    const int s0 = split * a.per_split, s1 = min(s0 + a.per_split, a.ntiles);
    // a workgroup whose keys are all masked has zeros to write and nothing to read
    const bool work = __syncthreads_or(keep) && s0 < s1;
    if (work) {
        if (BIAS) request_bias(s0);
        request(s0);
    }
    for (int step = s0; work && step < s1; ++step) {
        const int buf = step & 1;
        const E *qt = tiles[buf][0], *at = tiles[buf][1];
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        if (tid < S::XT) {
            // what lies behind the last query: probability exp(-inf)
            const bool in = step * S::XT + tid < a.M;
            stats[buf][0][tid] = in ? stats_in.x : BIAS ? __builtin_inff() : -__builtin_inff();
            stats[buf][1][tid] = stats_in.y;
            if (!BIAS) stats[buf][BIAS ? 0 : 2][tid] = rest_in;
        }
        const bool any_rest = !BIAS && __any(rest_in != 0.0f);
        copies_done_and_barrier();
        if (step + 1 < s1) request(step + 1);
        f32x16 s[NB], dp[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) s[b] = dp[b] = zero16();
#pragma unroll
        for (int kk = 0; kk < NK; ++kk)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                Y::mma(s[b], LT::row(qt, 32 * b + (lane & 31), kk, h), kf[kk]);
                Y::mma(dp[b], LT::row(at, 32 * b + (lane & 31), kk, h), vf[kk]);
            }
        if (BIAS) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = fmaf(s[b][i], a.scale, Y::f(braw[BIAS ? b : 0][i], keep));
            if (step + 1 < s1) request_bias(step + 1);
        }
        if (any_rest) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] -= stats[buf][BIAS ? 0 : 2][32 * b + 8 * (i / 4) + 4 * h + i % 4];
        }
        // four probabilities of a block, and what the logits' gradients are by them
        auto four = [&](int b, int i) {
            const f32x4 l = *reinterpret_cast<const f32x4 *>(&stats[buf][0][32 * b + 2 * i + 4 * h]);
            const f32x4 d = *reinterpret_cast<const f32x4 *>(&stats[buf][1][32 * b + 2 * i + 4 * h]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[b][i + e] = __builtin_amdgcn_exp2f(BIAS ? (s[b][i + e] - l[e]) * kLog2e : fmaf(s[b][i + e], to2, l[e]));
                dp[b][i + e] = s[b][i + e] * (dp[b][i + e] - d[e]);
            }
        };
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) four(b, i);
            Frag p[GP], ds[GP];
#pragma unroll
            for (int g = 0; g < GP; ++g) p[g] = Y::pack(s[b], g), ds[g] = Y::pack(dp[b], g);
            constexpr int NJ = GP * DT;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const int g = j / DT, d = j % DT;
                Y::mma(dvv[d], LT::col(at, 32 * b + Y::KS * g, 32 * d, lane), p[g]);
                Y::mma(dk[d], LT::col(qt, 32 * b + Y::KS * g, 32 * d, lane), ds[g]);
            }
        }
    }
    if (key >= a.Lk) return;
    const int64_t rows = a.N * a.Hk * (int64_t)a.Lk;
    float *pk = a.part + (((int64_t)split * 2) * rows + (int64_t)unit * a.Lk + key) * a.D, *pv = pk + rows * a.D;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int c = 32 * d + 2 * i + 4 * h;
            if (c >= a.D) continue;
            f32x4 x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
            if (keep) {
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = dk[d][i + e] * a.scale, y[e] = dvv[d][i + e];
            }
            if (a.splits > 1) {
                *reinterpret_cast<f32x4 *>(pk + c) = x;
                *reinterpret_cast<f32x4 *>(pv + c) = y;
            } else {
                E ex[4], ey[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) ex[e] = Y::e(x[e]), ey[e] = Y::e(y[e]);
                E *ok = (E *)a.dk + koff + c, *ov = (E *)a.dv + koff + c;
                __builtin_memcpy(__builtin_assume_aligned(ok, sizeof(ex)), ex, sizeof(ex));
                __builtin_memcpy(__builtin_assume_aligned(ov, sizeof(ey)), ey, sizeof(ey));
            }
        }
    }
}

// ---------------------------------------------------------------------------
// rows: dQ
template <typename T, int DP, bool BIAS> struct RowsShape {
    static constexpr bool WIDE = sizeof(typename Ty<T>::E) == 4;
    static constexpr int KT = WIDE || DP == 128 || BIAS ? 32 : 64, ROWS = 128;
    static constexpr int TILE = KT * DP;
    // (bf16 at 128 channels with a bias does not fit two waves a SIMD: 29 vector registers are spilled, 104 bytes a lane.  2 x 1024
    // to 1024, 8 heads: 150 us for the whole backward; one wave a SIMD was not measured)
    static constexpr int WAVES = WIDE && DP == 128 ? 1 : 2;
};

template <typename T, int DP, bool BIAS>
__global__ __launch_bounds__(kThreads, (RowsShape<T, DP, BIAS>::WAVES)) void cross_rows_kernel(CrArgs a) {
    using Y = Ty<T>;
    using E = typename Y::E;
    using Frag = typename Y::Frag;
    using LT = Tile<T, DP>;
    using S = RowsShape<T, DP, BIAS>;
    constexpr int NK = DP / Y::KS, DT = DP / 32;
    __shared__ __attribute__((aligned(16))) E tiles[2][2][S::TILE];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    uint32_t u = xcd_unit32(blockIdx.x, gridDim.x);
    const int split = u % a.splits;
    u /= a.splits;
    const int tile = u % a.tiles;
    const uint32_t unit = u / a.tiles;
    const int64_t n = unit / a.Hk;
    const int hk = unit % a.Hk;

    const int x = tile * S::ROWS + wave * 32 + (lane & 31);
    const bool on = x < a.M;
    const int xc = on ? x : a.M - 1, t = token_of(a, xc), head = hk * a.G + (xc - t * a.G);
    Frag qf[NK], af[NK];
    const int64_t qoff = n * a.q_row + (int64_t)t * a.q_tok + (int64_t)head * a.D;
    load_rows<T, DP>(qf, (const E *)a.q + qoff, a.D, on, h);
    const float inf = __builtin_inff(), lse = a.lse[(n * a.H + head) * a.Lq + t], to2 = a.scale * kLog2e;
    constexpr int W = Y::KS / 2;
    struct Bits16 { E e[W]; };
    const int64_t oat = n * a.o_row + (int64_t)t * a.o_tok + (int64_t)head * a.D;
    u32x4 oin[NK], din[NK], gin[NK];
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) {
        const int c = Y::KS * kk + W * h, cc = c < a.D ? c : 0;
        oin[kk] = *reinterpret_cast<const u32x4 *>((const E *)a.out + oat + cc);
        din[kk] = *reinterpret_cast<const u32x4 *>((const E *)a.dout + oat + cc);
        gin[kk] = a.gate ? *reinterpret_cast<const u32x4 *>((const E *)a.gate + qoff + cc) : u32x4{};
    }
    const BiasRow<T> brow(a, BIAS ? (n / a.rpb * a.H + head) * a.Lq + t : 0);
    const E *kbase = (const E *)a.k + n * a.k_row + (int64_t)hk * a.D;
    const E *vbase = (const E *)a.v + n * a.k_row + (int64_t)hk * a.D;
    const uint8_t *mrow = a.mask ? a.mask + n * a.Lk : nullptr;

    // the first tiles are on their way while D, dgate and dA are formed: 2 x 1024 to 1024, 8 heads of 64 with a bias 27.4 -> 24.8 us;
    // at 128 channels, where registers are short, 45.4 -> 47.4: there they come after
    using Bits = KeyBits<S::KT>;
    constexpr int NB = S::KT / 32, GP = 32 / Y::KS;
    Bits now, next;
    const bool full_d = a.D == DP;
    auto request = [&](int step, bool whole, auto keep) {
        const int64_t off = (int64_t)step * S::KT * a.k_tok;
        const auto k_row = [&](int r) { return kbase + off + (int64_t)r * a.k_tok; };
        const auto v_row = [&](int r) { return vbase + off + (int64_t)r * a.k_tok; };
        E *kt = tiles[step & 1][0], *vt = tiles[step & 1][1];
        if constexpr (S::KT * LT::CH % kThreads == 0) {
            Copy<T, DP, S::KT, kThreads>::run(kt, whole, a.D, wave, lane, k_row, keep);
            Copy<T, DP, S::KT, kThreads>::run(vt, whole, a.D, wave, lane, v_row, keep);
        } else if (wave < 2) {  // a tile takes half of the workgroup
            Copy<T, DP, S::KT, kThreads / 2>::run(kt, whole, a.D, wave, lane, k_row, keep);
        } else {
            Copy<T, DP, S::KT, kThreads / 2>::run(vt, whole, a.D, wave - 2, lane, v_row, keep);
        }
    };
    typename BiasRow<T>::Raw braw[BIAS ? NB : 1];
    auto request_bias = [&](int step) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
            if (BIAS) braw[BIAS ? b : 0] = brow.request(step * S::KT + 32 * b, h);
    };
    typename Bits::Bytes bytes = {};
    const int t0 = split * a.per_split, t1 = min(t0 + a.per_split, a.ntiles);
    const auto first_tiles = [&] {
        if (t0 >= t1) return;
        const auto first = Bits::request(mrow, t0 * S::KT, a.Lk, lane);
        bytes = Bits::request(mrow, (t0 + 1) * S::KT, a.Lk, lane);
        next.set(first);
        request_bias(t0);
        request(t0, full_d && next.all(), [&](int r) { return next.get(r); });
    };
    if (DP <= 64) first_tiles();

    const bool live = on && lse != -inf, far = live && fabsf(lse) > kFarLse && fabsf(lse) < inf;
    const bool any_far = __any(far);
    float base = BIAS ? (live ? lse : inf) : (live ? -lse * kLog2e : -inf), rest = 0.0f, times = 1.0f;
    if (__builtin_expect(any_far, 0)) {
        // rows of K straight from memory, one a lane: rare, and without barriers that the other waves would have to meet
        const float unit2 = BIAS ? kLog2e : to2;
        float top = -inf, sum = 0.0f;
        for (int k0 = 0; k0 < a.Lk; k0 += 32) {
            const int key = k0 + (lane & 31), keyc = min(key, a.Lk - 1);
            const bool keep = key < a.Lk && (!mrow || mrow[keyc]);
            const uint32_t bits = (uint32_t)__ballot(keep);
            if (!bits) continue;
            Frag kf[NK];
            load_rows<T, DP>(kf, kbase + (int64_t)keyc * a.k_tok, a.D, keep, h);
            f32x16 s = zero16();
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) Y::mma(s, kf[kk], qf[kk]);
            if (BIAS) {
                const auto raw = brow.request(k0, h);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], a.scale, BiasRow<T>::value(raw, i));
            }
            float higher = top;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[i] = where_kept(bits, i, s[i], kMinusInf);
                higher = fmaxf(higher, s[i]);
            }
            higher = half_max(higher);
            const float to = higher > -inf ? higher : 0.0f;
            sum *= __builtin_amdgcn_exp2f((top - to) * unit2);
#pragma unroll
            for (int i = 0; i < 16; ++i) sum += __builtin_amdgcn_exp2f((s[i] - to) * unit2);
            top = higher;
        }
        sum = half_sum(sum);
        if (far && BIAS) base = top, times = 1.0f / sum;
        if (far && !BIAS) base = -__builtin_amdgcn_logf(sum), rest = top;
    }

    // D, dgate and dA of the lane's query, for this pass and, written by the first split, for the next
    float dsum = 0.0f;
    {
        const int64_t daat = ((n * a.Lq + t) * a.H + head) * (int64_t)a.D;
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
            const int c = Y::KS * kk + W * h;
            const bool in = on && c < a.D;
            const Bits16 o = __builtin_bit_cast(Bits16, where(in, oin[kk]));
            Bits16 d = __builtin_bit_cast(Bits16, where(in, din[kk]));
#pragma unroll
            for (int e = 0; e < W; ++e) dsum = fmaf(Y::f(o.e[e]), Y::f(d.e[e]), dsum);
            if (a.gate) {
                const Bits16 g = __builtin_bit_cast(Bits16, gin[kk]);
                Bits16 dg;
#pragma unroll
                for (int e = 0; e < W; ++e) {
                    // sigmoid and one minus it, each without cancellation
                    const float y = Y::f(g.e[e]), z = __builtin_amdgcn_exp2f(-fabsf(y) * kLog2e), r = __builtin_amdgcn_rcpf(1.0f + z);
                    const float sig = y >= 0.0f ? r : z * r, rest = y >= 0.0f ? z * r : r, df = Y::f(d.e[e]);
                    dg.e[e] = Y::e(df * Y::f(o.e[e]) * rest);
                    d.e[e] = Y::e(BIAS ? df * sig * times : df * sig);  // rounded to the type: the operand of two matrix products
                }
                if (in && split == 0) *reinterpret_cast<u32x4 *>((E *)a.dgate + qoff + c) = __builtin_bit_cast(u32x4, dg);
            } else if (BIAS && any_far) {
#pragma unroll
                for (int e = 0; e < W; ++e) d.e[e] = Y::e(Y::f(d.e[e]) * times);
            }
            if ((BIAS || a.gate) && in && split == 0) *reinterpret_cast<u32x4 *>((E *)a.da + daat + c) = __builtin_bit_cast(u32x4, d);
            af[kk] = __builtin_bit_cast(Frag, d);
        }
        dsum = half_sum(dsum);
        if (BIAS) dsum *= times;
        if (on && h == 0 && split == 0) a.stats[(int64_t)unit * a.M + x] = f32x4{base, dsum, rest, 0.0f};
    }
    f32x16 dq[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) dq[i] = zero16();

    if (DP > 64) first_tiles();
    for (int step = t0; step < t1; ++step) {
        const E *kt = tiles[step & 1][0], *vt = tiles[step & 1][1];
        copies_done_and_barrier();
        now = next;
        if (step + 1 < t1) {
            next.set(bytes);
            bytes = Bits::request(mrow, (step + 2) * S::KT, a.Lk, lane);
            request(step + 1, full_d && next.all(), [&](int r) { return next.get(r); });
        }
        if (!now.any()) {
            if (step + 1 < t1) request_bias(step + 1);
            continue;
        }
        f32x16 s[NB], dp[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) s[b] = dp[b] = zero16();
#pragma unroll
        for (int kk = 0; kk < NK; ++kk)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                Y::mma(s[b], LT::row(kt, 32 * b + (lane & 31), kk, h), qf[kk]);
                Y::mma(dp[b], LT::row(vt, 32 * b + (lane & 31), kk, h), af[kk]);
            }
        if (BIAS) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s[b][i] = (fmaf(s[b][i], a.scale, BiasRow<T>::value(braw[BIAS ? b : 0], i)) - base) * kLog2e;
            if (step + 1 < t1) request_bias(step + 1);
        } else {
            if (any_far) {
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[b][i] -= rest;
            }
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = fmaf(s[b][i], to2, base);
        }
        if (!now.all()) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const uint32_t bits = now.sub(b);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = where_kept(bits, i, s[b][i], kMinusInf);
            }
        }
        auto four = [&](int b, int i) {
#pragma unroll
            for (int e = i; e < i + 4; ++e) dp[b][e] = __builtin_amdgcn_exp2f(s[b][e]) * (dp[b][e] - dsum);
        };
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) four(b, i);
            Frag ds[GP];
#pragma unroll
            for (int g = 0; g < GP; ++g) ds[g] = Y::pack(dp[b], g);
            constexpr int NJ = GP * DT;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                Y::mma(dq[j % DT], LT::col(kt, 32 * b + Y::KS * (j / DT), 32 * (j % DT), lane), ds[j / DT]);
            }
        }
    }
    if (!on) return;
    float *part = a.part + ((int64_t)split * a.N * a.Hk * a.M + (int64_t)unit * a.M + x) * a.D;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int c = 32 * d + 2 * i + 4 * h;
            if (c >= a.D) continue;
            f32x4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = dq[d][i + e] * a.scale;
            if (a.splits > 1) {
                *reinterpret_cast<f32x4 *>(part + c) = y;
            } else {
                E ey[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) ey[e] = Y::e(y[e]);
                E *to = (E *)a.dq + qoff + c;
                __builtin_memcpy(__builtin_assume_aligned(to, sizeof(ey)), ey, sizeof(ey));
            }
        }
    }
}

// ---------------------------------------------------------------------------
// bias: dBias.  tiles = 64-query tiles, ntiles = 64-key tiles, splits = chunks of
// per_split rows of a plane
template <typename T, int DP> struct BiasShape {
    static constexpr int TILE = 64 * DP, BYTES = 4 * TILE * (int)sizeof(typename Ty<T>::E);
    static constexpr int BUFS = BYTES <= 64 * 1024 ? 2 : 1;
    static constexpr int WAVES = BUFS * BYTES <= 78 * 1024 ? 2 : 1;
};

template <typename T, int DP>
__global__ __launch_bounds__(kThreads, (BiasShape<T, DP>::WAVES)) void cross_bias_kernel(CrArgs a) {
    using Y = Ty<T>;
    using E = typename Y::E;
    using LT = Tile<T, DP>;
    using S = BiasShape<T, DP>;
    constexpr int NK = DP / Y::KS;
    __shared__ __attribute__((aligned(16))) E tiles[S::BUFS][4][S::TILE];  // Q, dA, K, V
    __shared__ __attribute__((aligned(16))) float stats[S::BUFS][2][64];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    const int qb = wave & 1, kb = wave >> 1;
    uint32_t u = blockIdx.x;
    const int chunk = u % a.splits;
    u /= a.splits;
    const int kt = u % a.ntiles;
    u /= a.ntiles;
    const int qt = u % a.tiles;
    u /= a.tiles;
    const int head = u % a.H;
    const int64_t plane = u / a.H;
    const int hk = head / a.G, g = head % a.G;
    const int t0 = qt * 64, k0 = kt * 64;
    const DaView dv = da_view(a);
    const int64_t n0 = plane * a.rpb + (int64_t)chunk * a.per_split, n1 = min(n0 + a.per_split, (plane + 1) * a.rpb);

    const int key = k0 + kb * 32 + (lane & 31);
    const int64_t brow = (plane * a.H + head) * a.Lq;
    float bias[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int t = min(t0 + qb * 32 + 8 * (i / 4) + 4 * h + i % 4, a.Lq - 1);
        bias[i] = Y::f(((const E *)a.bias)[(brow + t) * a.Lk + min(key, a.Lk - 1)]);
    }
    f32x16 acc = zero16();
    using Bits = KeyBits<64>;
    using Cp = Copy<T, DP, 64, kThreads>;
    Bits now, next;
    auto bytes_of = [&](int64_t n) { return Bits::request(a.mask ? a.mask + n * a.Lk : nullptr, k0, n < n1 ? a.Lk : 0, lane); };
    float2 stats_in = {};
    const bool full_d = a.D == DP, full_q = full_d && t0 + 64 <= a.Lq;
    auto request = [&](int64_t n, int buf) {
        if (tid < 64) stats_in = *reinterpret_cast<const float2 *>(a.stats + ((n * a.Hk + hk) * a.Lq + min(t0 + tid, a.Lq - 1)) * a.G + g);
        const E *q = (const E *)a.q + n * a.q_row + (int64_t)head * a.D;
        const E *da = (const E *)(a.da ? a.da : a.dout) + n * dv.row + (int64_t)head * a.D;
        const E *k = (const E *)a.k + n * a.k_row + (int64_t)hk * a.D, *v = (const E *)a.v + n * a.k_row + (int64_t)hk * a.D;
        const auto in_q = [&](int r) { return t0 + r < a.Lq; };
        const auto keep = [&](int r) { return next.get(r); };
        const bool full_k = full_d && next.all();
        Cp::run(tiles[buf][0], full_q, a.D, wave, lane, [&](int r) { return q + (int64_t)(t0 + r) * a.q_tok; }, in_q);
        Cp::run(tiles[buf][1], full_q, a.D, wave, lane, [&](int r) { return da + (int64_t)(t0 + r) * dv.tok; }, in_q);
        Cp::run(tiles[buf][2], full_k, a.D, wave, lane, [&](int r) { return k + (int64_t)(k0 + r) * a.k_tok; }, keep);
        Cp::run(tiles[buf][3], full_k, a.D, wave, lane, [&](int r) { return v + (int64_t)(k0 + r) * a.k_tok; }, keep);
    };
    typename Bits::Bytes bytes = {};
    if (n0 < n1) {
        const auto first = bytes_of(n0);
        bytes = bytes_of(n0 + 1);
        next.set(first);
        request(n0, 0);
    }
    int buf = 0;
    for (int64_t n = n0; n < n1; ++n) {
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        if (tid < 64) {
            stats[buf][0][tid] = t0 + tid < a.Lq ? stats_in.x : __builtin_inff();
            stats[buf][1][tid] = stats_in.y;
        }
        copies_done_and_barrier();
        now = next;
        const E *const qt_ = tiles[buf][0], *const at_ = tiles[buf][1], *const kt_ = tiles[buf][2], *const vt_ = tiles[buf][3];
        const float *const ls = stats[buf][0], *const ds = stats[buf][1];
        const auto go_on = [&]() {
            if (n + 1 >= n1) return;
            next.set(bytes);
            bytes = bytes_of(n + 2);
            if (S::BUFS == 2) buf ^= 1;
            request(n + 1, buf);
        };
        if (S::BUFS == 2) go_on();
        if (now.any()) {
            f32x16 s = zero16(), dp = zero16();
            const int qr = 32 * qb + (lane & 31), kr = 32 * kb + (lane & 31);
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) {
                Y::mma(s, LT::row(qt_, qr, kk, h), LT::row(kt_, kr, kk, h));
                Y::mma(dp, LT::row(at_, qr, kk, h), LT::row(vt_, kr, kk, h));
            }
            const bool mine = now.get(32 * kb + (lane & 31));
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const f32x4 l = *reinterpret_cast<const f32x4 *>(&ls[32 * qb + 2 * i + 4 * h]);
                const f32x4 d = *reinterpret_cast<const f32x4 *>(&ds[32 * qb + 2 * i + 4 * h]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float b = __uint_as_float(mine ? __float_as_uint(bias[i + e]) : kMinusInf);
                    const float p = __builtin_amdgcn_exp2f((fmaf(s[i + e], a.scale, b) - l[e]) * kLog2e);
                    acc[i + e] = fmaf(p, dp[i + e] - d[e], acc[i + e]);
                }
            }
        }
        if (S::BUFS == 1) {
            __syncthreads();
            go_on();
        }
    }
    if (key >= a.Lk) return;
    const int64_t all = a.N / a.rpb * a.H * a.Lq * (int64_t)a.Lk;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int t = t0 + qb * 32 + 8 * (i / 4) + 4 * h + i % 4;
        if (t >= a.Lq) continue;
        const int64_t at = (brow + t) * a.Lk + key;
        if (a.splits > 1)
            a.part[(int64_t)chunk * all + at] = acc[i];
        else
            ((E *)a.dbias)[at] = Y::e(acc[i]);
    }
}

// ---------------------------------------------------------------------------
// Sums of parts: rows of D channels written at (unit, i < len) -> token and head, or a flat array
// (len 0).  With a second output its parts follow the first's.
template <typename T>
__global__ __launch_bounds__(kThreads) void cross_sum_kernel(CrArgs a, const float *part, int splits, int64_t stride, int64_t count,
                                                             int len, int group, void *out0, void *out1, int64_t row_stride, int64_t tok_stride) {
    using Y = Ty<T>;
    using E = typename Y::E;
    const int64_t at = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 4;
    if (at >= count) return;
    void *out = blockIdx.y ? out1 : out0;
    part += blockIdx.y * count;
    f32x4 sum = {0, 0, 0, 0};
    const bool whole = at + 4 <= count;
#pragma unroll 4
    for (int j = 0; j < splits; ++j) {
        const float *p = part + j * stride + at;
        if (whole) {
            f32x4 x;
            __builtin_memcpy(&x, p, 16);
            sum += x;
        } else {
            for (int e = 0; e < count - at; ++e) sum[e] += p[e];
        }
    }
    if (!len) {
        for (int e = 0; e < 4 && at + e < count; ++e) ((E *)out)[at + e] = Y::e(sum[e]);
        return;
    }
    const int64_t row = at / a.D, unit = row / len, n = unit / a.Hk;
    const int c = (int)(at - row * a.D), x = (int)(row - unit * len), t = group ? token_of(a, x) : x;
    const int head = (int)(unit - n * a.Hk) * (group ? a.G : 1) + (group ? x - t * a.G : 0);
    E e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = Y::e(sum[i]);
    E *to = (E *)out + n * row_stride + (int64_t)t * tok_stride + (int64_t)head * a.D + c;
    __builtin_memcpy(__builtin_assume_aligned(to, sizeof(e)), e, sizeof(e));
}

template <typename T>
void sum_parts(const CrArgs &a, const float *part, int splits, int64_t stride, int64_t count, int len, int group, void *out,
               void *more, int64_t row, int64_t tok, hipStream_t s) {
    const dim3 grid((uint32_t)((count + 4 * kThreads - 1) / (4 * kThreads)), more ? 2 : 1);
    cross_sum_kernel<T><<<grid, kThreads, 0, s>>>(a, part, splits, stride, count, len, group, out, more, row, tok);
}

template <typename T, int DP> void run(CrArgs a, const CrPlan &p, hipStream_t s) {
    const int64_t units = a.N * a.Hk;
    const bool bias = a.bias != nullptr;
    if (a.M > 0) {
        CrArgs k = a;
        const int kt = bias ? RowsShape<T, DP, true>::KT : RowsShape<T, DP, false>::KT;
        k.tiles = (a.M + 127) / 128;
        k.ntiles = (a.Lk + kt - 1) / kt;
        k.splits = p.q_splits;
        k.per_split = (k.ntiles + k.splits - 1) / k.splits;
        const uint32_t grid = (uint32_t)(units * k.tiles * k.splits);
        if (bias)
            cross_rows_kernel<T, DP, true><<<grid, kThreads, 0, s>>>(k);
        else
            cross_rows_kernel<T, DP, false><<<grid, kThreads, 0, s>>>(k);
        if (k.splits > 1) {
            const int64_t count = units * a.M * a.D;
            sum_parts<T>(a, a.part, k.splits, count, count, a.M, 1, a.dq, nullptr, a.q_row, a.q_tok, s);
        }
    }
    if (a.Lk > 0) {
        CrArgs k = a;
        using S = KeysShape<T, DP>;
        k.tiles = (a.Lk + S::KEYS - 1) / S::KEYS;
        k.ntiles = (a.M + S::XT - 1) / S::XT;
        k.splits = p.kv_splits;
        k.per_split = (k.ntiles + k.splits - 1) / k.splits;
        const uint32_t grid = (uint32_t)(units * k.tiles * k.splits);
        if (bias)
            cross_keys_kernel<T, DP, true><<<grid, kThreads, 0, s>>>(k);
        else
            cross_keys_kernel<T, DP, false><<<grid, kThreads, 0, s>>>(k);
        if (k.splits > 1) {
            const int64_t count = units * a.Lk * a.D;
            sum_parts<T>(a, a.part, k.splits, 2 * count, count, a.Lk, 0, a.dk, a.dv, a.k_row, a.k_tok, s);
        }
    }
    if (bias && a.M > 0 && a.Lk > 0) {
        CrArgs k = a;
        k.tiles = (a.Lq + 63) / 64;
        k.ntiles = (a.Lk + 63) / 64;
        k.splits = p.bias_chunks;
        k.per_split = (int)((a.rpb + k.splits - 1) / k.splits);
        const int64_t planes = a.N / a.rpb * a.H;
        cross_bias_kernel<T, DP><<<(uint32_t)(planes * k.tiles * k.ntiles * k.splits), kThreads, 0, s>>>(k);
        if (k.splits > 1) {
            const int64_t count = planes * a.Lq * a.Lk;
            sum_parts<T>(a, a.part, k.splits, count, count, 0, 0, a.dbias, nullptr, 0, 0, s);
        }
    }
}

template <typename T> void run_dim(const CrArgs &a, const CrPlan &p, hipStream_t s) {
    a.D <= 32 ? run<T, 32>(a, p, s) : a.D <= 64 ? run<T, 64>(a, p, s) : run<T, 128>(a, p, s);
}

}  // namespace

hipError_t launch_cross_bwd(CrArgs a, const CrPlan &p, void *ws, hipStream_t s) {
    a.stats = (f32x4 *)ws;
    a.da = a.gate || a.bias ? (char *)ws + p.bwd_da : nullptr;
    a.part = (float *)((char *)ws + p.bwd_part);
    a.bf16 ? run_dim<bf16_t>(a, p, s) : run_dim<float>(a, p, s);
    return hipGetLastError();
}

}  // namespace evo

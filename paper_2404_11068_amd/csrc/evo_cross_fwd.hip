// evo_cross_fwd.hip -- attention to states of another length, forward
// (include/evo_cross_attn.h):  o = sigmoid(g) softmax(q k' / sqrt d + bias) v.
//
// One pass over the keys with the running maximum and sum of the softmax.
// Logits are formed transposed (S' = K Q'): a lane owns a query, so maximum and
// sum stay in the lane but for one exchange between its halves, and the
// probabilities go into O' = V' P' as they lie in their registers, V' by the
// transposing LDS read.  Two shapes of workgroup (four waves):
//   rows: 32 queries a wave, all waves the same keys
//   few:  the waves share 32 (fp32: 64) queries and take turns with the keys;
//         for single tokens, where reading K and V is all there is to do
// and where the tiles of rows do not fill the GPU, the keys are split over
// workgroups whose partial results a second kernel joins.
#include "evo_cross.h"

namespace evo {
namespace {

constexpr int kThreads = 256;

// shape of a workgroup: QW waves of queries times KW waves of keys, KT keys a step
template <typename T, bool FEW> struct Shape {
    static constexpr bool WIDE = sizeof(typename Ty<T>::E) == 4;
    static constexpr int QW = FEW ? (WIDE ? 2 : 1) : 4, KW = 4 / QW;
    static constexpr int KT = FEW ? 32 * KW : (WIDE ? 32 : 64);
    static constexpr int KPW = KT / KW, NS = KPW / 32, ROWS = 32 * QW;
};

template <typename T, int DP, bool FEW> struct Lds {
    using S = Shape<T, FEW>;
    using E = typename Ty<T>::E;
    static constexpr int STR = DP + Ty<T>::PAD, TILE = S::KT * STR;
    static constexpr int BUFS = 2 * 2 * TILE * (int)sizeof(E) <= 150 * 1024 ? 2 : 1;
    static constexpr int BYTES = BUFS * 2 * TILE * (int)sizeof(E);
    static constexpr int JOIN = S::KW > 1 ? 4 * (DP / 32 * 16 + 2) * 64 * 4 : 0;  // the waves' results, at the end
    static constexpr int SIZE = BYTES > JOIN ? BYTES : JOIN;
};

template <typename T, int DP, bool BIAS, bool FEW>
__global__ __launch_bounds__(kThreads, (Lds<T, DP, FEW>::SIZE <= 80 * 1024 ? 2 : 1)) void cross_fwd_kernel(CrArgs a) {
    using Y = Ty<T>;
    using E = typename Y::E;
    using Frag = typename Y::Frag;
    using S = Shape<T, FEW>;
    using L = Lds<T, DP, FEW>;
    constexpr int NK = DP / Y::KS, DT = DP / 32;
    __shared__ __attribute__((aligned(16))) char lds[L::SIZE];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = lane >> 5;
    const int qw = wave % S::QW, kw = wave / S::QW;
    uint32_t u = xcd_unit32(blockIdx.x, gridDim.x);
    const int split = u % a.splits;
    u /= a.splits;
    const int tile = u % a.tiles;
    const uint32_t unit = u / a.tiles;
    const int64_t n = unit / a.Hk;
    const int hk = unit % a.Hk;

    // the lane's query
    const int x = tile * S::ROWS + qw * 32 + (lane & 31);
    const bool on = x < a.M;
    const int xc = on ? x : a.M - 1, t = token_of(a, xc), head = hk * a.G + (xc - t * a.G);
    Frag qf[NK];
    load_rows<T, DP>(qf, (const E *)a.q + n * a.q_row + (int64_t)t * a.q_tok + (int64_t)head * a.D, a.D, on, h);
    const BiasRow<T> brow(a, BIAS ? (n / a.rpb * a.H + head) * a.Lq + t : 0);
    constexpr bool EARLY = DP <= 64;  // the gate's values wait in registers where there is room
    const E *grow = a.gate ? (const E *)a.gate + n * a.q_row + (int64_t)t * a.q_tok + (int64_t)head * a.D : nullptr;
    u32x4 gv[EARLY ? DT * 4 : 1];
    auto gate_at = [&](int d, int i) {
        const int c = 32 * d + 8 * i + 4 * h;
        return load4(grow + (c < a.D ? c : 0));
    };
    if (EARLY && grow) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) gv[EARLY ? d * 4 + i : 0] = gate_at(d, i);
    }

    const E *kbase = (const E *)a.k + n * a.k_row + (int64_t)hk * a.D;
    const E *vbase = (const E *)a.v + n * a.k_row + (int64_t)hk * a.D;
    const uint8_t *mrow = a.mask ? a.mask + n * a.Lk : nullptr;
    const int t0 = split * a.per_split, t1 = min(t0 + a.per_split, a.ntiles);

    f32x16 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = zero16();
    float m = -__builtin_inff(), sum = 0.0f;
    // x is the logit in units of 1 / to2 of base-2 exponents
    const float to2 = BIAS ? kLog2e : a.scale * kLog2e, slack = 8.0f / to2;

    using Bits = KeyBits<S::KT>;
    Bits now, next;
    Stage<T, DP, S::KT, kThreads> ks, vs;
    auto request = [&](int step, auto keep) {
        const int64_t off = (int64_t)step * S::KT * a.k_tok;
        ks.load(kbase, a.D, tid, [&](int r) { return kbase + off + (int64_t)r * a.k_tok; }, keep);
        vs.load(vbase, a.D, tid, [&](int r) { return vbase + off + (int64_t)r * a.k_tok; }, keep);
    };
    typename Bits::Bytes bytes;
    if (t0 < t1) {
        // the first tile does not wait for its mask; of later ones masked keys are not read
        const auto first = Bits::request(mrow, t0 * S::KT, a.Lk, lane);
        request(t0, [&](int r) { return t0 * S::KT + r < a.Lk; });
        bytes = Bits::request(mrow, (t0 + 1) * S::KT, a.Lk, lane);
        next.set(first);
    }
    for (int step = t0; step < t1; ++step) {
        E *kt = (E *)lds + (L::BUFS == 2 ? (step & 1) * 2 * L::TILE : 0), *vt = kt + L::TILE;
        now = next;
        ks.store(kt, a.D, tid, [&](int r) { return now.get(r); });
        vs.store(vt, a.D, tid, [&](int r) { return now.get(r); });
        __syncthreads();
        if (step + 1 < t1) {
            next.set(bytes);
            request(step + 1, [&](int r) { return next.get(r); });
            bytes = Bits::request(mrow, (step + 2) * S::KT, a.Lk, lane);
        }
        if (now.any()) {
            const int sub0 = kw * S::NS;  // the wave's first block of 32 keys
            f32x16 s[S::NS];
            float top = -__builtin_inff();
#pragma unroll
            for (int b = 0; b < S::NS; ++b) {
                const uint32_t bits = now.sub(sub0 + b), mine = bits >> (4 * h);
                if (bits == 0) continue;
                s[b] = zero16();
                const E *row = kt + ((sub0 + b) * 32 + (lane & 31)) * L::STR + Y::KS / 2 * h;
                const bool whole = bits == 0xffffffffu;
                float add[16];
                if (BIAS) brow.get(add, step * S::KT + (sub0 + b) * 32, h, mine, whole);
#pragma unroll
                for (int kk = 0; kk < NK; ++kk) Y::mma(s[b], Y::row(row + Y::KS * kk), qf[kk]);
                if (BIAS) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[b][i] = fmaf(s[b][i], a.scale, add[i]);
                }
                if (!whole) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[b][i] = (mine >> (8 * (i / 4) + i % 4)) & 1 ? s[b][i] : -__builtin_inff();
                }
#pragma unroll
                for (int i = 0; i < 16; i += 2) top = fmaxf(fmaxf(top, s[b][i]), s[b][i + 1]);
            }
            top = half_max(top);
            // the reference maximum rises only when it has fallen behind by 2^8: sums and
            // probabilities stay within fp32 and keep their relative precision
            if (__any(top > m + slack)) {
                const float higher = fmaxf(m, top);
                const float by = m > -__builtin_inff() ? __builtin_amdgcn_exp2f((m - higher) * to2) : 0.0f;
                sum *= by;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] *= by;
                m = higher;
            }
            const float base = m > -__builtin_inff() ? m : 0.0f, shift = -base * to2;
#pragma unroll
            for (int b = 0; b < S::NS; ++b) {
                if (now.sub(sub0 + b) == 0) continue;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    // with a bias the difference comes first: a bias of the type's lowest value times log2 e would be infinite
                    s[b][i] = __builtin_amdgcn_exp2f(BIAS ? (s[b][i] - base) * to2 : fmaf(s[b][i], to2, shift));
                    sum += s[b][i];
                }
#pragma unroll
                for (int g = 0; g < 32 / Y::KS; ++g) {
                    const Frag p = Y::pack(s[b], g);
#pragma unroll
                    for (int d = 0; d < DT; ++d)
                        Y::mma(o[d], Y::col(vt, L::STR, (sub0 + b) * 32 + Y::KS * g, 32 * d, lane), p);
                }
            }
        }
        if (L::BUFS == 1) __syncthreads();
    }

    sum = half_sum(sum);
    if (S::KW > 1) {
        // the waves' maxima, sums and results, joined: wave kw takes every KW-th block of channels
        float *all = (float *)lds;
        constexpr int PER = DT * 16 + 2;
        __syncthreads();
        float *mine = all + wave * PER * 64 + lane;
        mine[0] = m;
        mine[64] = sum;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) mine[(2 + d * 16 + i) * 64] = o[d][i];
        __syncthreads();
        float mj[S::KW], top = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < S::KW; ++j) {
            mj[j] = all[(j * S::QW + qw) * PER * 64 + lane];
            top = fmaxf(top, mj[j]);
        }
        m = top;
        sum = 0.0f;
#pragma unroll
        for (int j = 0; j < S::KW; ++j) {
            mj[j] = mj[j] > -__builtin_inff() ? __builtin_amdgcn_exp2f((mj[j] - top) * to2) : 0.0f;
            sum += mj[j] * all[(j * S::QW + qw) * PER * 64 + 64 + lane];
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            if (d % S::KW != kw) continue;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float v = 0.0f;
#pragma unroll
                for (int j = 0; j < S::KW; ++j) v += mj[j] * all[((j * S::QW + qw) * PER + 2 + d * 16 + i) * 64 + lane];
                o[d][i] = v;
            }
        }
    }
    if (!on) return;
    if (a.splits > 1) {
        const int64_t row = ((int64_t)split * a.N * a.Hk + unit) * a.M + x;
        if (kw == 0 && h == 0) a.part_ml[row] = float2{m, sum};
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            if (S::KW > 1 && d % S::KW != kw) continue;
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int c = 32 * d + 2 * i + 4 * h;
                if (c < a.D) *reinterpret_cast<f32x4 *>(a.part + row * a.D + c) = f32x4{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]};
            }
        }
        return;
    }
    if (BIAS && m < kNoKey) sum = 0.0f;
    const float inv = sum > 0.0f ? 1.0f / sum : (sum == 0.0f ? 0.0f : sum);
    if (kw == 0 && h == 0)
        a.lse[(n * a.H + head) * a.Lq + t] = sum == 0.0f ? -__builtin_inff() : fmaf(__builtin_amdgcn_logf(sum), kLn2, BIAS ? m : m * a.scale);
    E *orow = (E *)a.out + n * a.o_row + (int64_t)t * a.o_tok + (int64_t)head * a.D;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
        if (S::KW > 1 && d % S::KW != kw) continue;
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int c = 32 * d + 2 * i + 4 * h;
            if (c >= a.D) continue;
            E e[4];
            f32x4 g = {1.0f, 1.0f, 1.0f, 1.0f};
            if (grow) {
                g = __builtin_bit_cast(f32x4, EARLY ? gv[EARLY ? d * 4 + i / 4 : 0] : gate_at(d, i / 4));
#pragma unroll
                for (int j = 0; j < 4; ++j) g[j] = 1.0f / (1.0f + __builtin_amdgcn_exp2f(-g[j] * kLog2e));
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) e[j] = Y::e(o[d][i + j] * inv * g[j]);
            __builtin_memcpy(__builtin_assume_aligned(orow + c, sizeof(e)), e, sizeof(e));
        }
    }
}

// Joins the splits of a row: one thread per four channels
template <typename T>
__global__ __launch_bounds__(kThreads) void cross_join_kernel(CrArgs a, int has_bias, int64_t rows) {
    using Y = Ty<T>;
    using E = typename Y::E;
    const int per = a.D / 4;
    const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t row = at / per;
    if (row >= rows) return;
    const int c = (int)(at - row * per) * 4;
    const float to2 = has_bias ? kLog2e : a.scale * kLog2e;
    float top = -__builtin_inff();
    for (int j = 0; j < a.splits; ++j) top = fmaxf(top, a.part_ml[j * rows + row].x);
    float sum = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    if (top > (has_bias ? kNoKey : -__builtin_inff())) {
        for (int j = 0; j < a.splits; ++j) {
            const float2 ml = a.part_ml[j * rows + row];
            if (!(ml.x > -__builtin_inff())) continue;
            const float f = __builtin_amdgcn_exp2f((ml.x - top) * to2);
            sum = fmaf(ml.y, f, sum);
            const f32x4 p = *reinterpret_cast<const f32x4 *>(a.part + (j * rows + row) * a.D + c);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = fmaf(p[i], f, o[i]);
        }
    }
    const int64_t unit = row / a.M, n = unit / a.Hk;
    const int x = (int)(row - unit * a.M), t = token_of(a, x), head = (int)(unit - n * a.Hk) * a.G + x - t * a.G;
    const float inv = sum > 0.0f ? 1.0f / sum : (sum == 0.0f ? 0.0f : sum);
    if (c == 0)
        a.lse[(n * a.H + head) * a.Lq + t] =
            sum == 0.0f ? -__builtin_inff() : fmaf(__builtin_amdgcn_logf(sum), kLn2, has_bias ? top : top * a.scale);
    const int64_t tok = (int64_t)head * a.D + c;
    E e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float g = 1.0f;
        if (a.gate) g = 1.0f / (1.0f + __builtin_amdgcn_exp2f(-Y::f(((const E *)a.gate)[n * a.q_row + (int64_t)t * a.q_tok + tok + i]) * kLog2e));
        e[i] = Y::e(o[i] * inv * g);
    }
    E *out = (E *)a.out + n * a.o_row + (int64_t)t * a.o_tok + tok;
    __builtin_memcpy(__builtin_assume_aligned(out, sizeof(e)), e, sizeof(e));
}

template <typename T, int DP, bool BIAS, bool FEW> void launch(CrArgs &a, hipStream_t s) {
    using S = Shape<T, FEW>;
    a.tiles = (a.M + S::ROWS - 1) / S::ROWS;
    a.ntiles = (a.Lk + S::KT - 1) / S::KT;
    a.per_split = (a.ntiles + a.splits - 1) / a.splits;
    const uint32_t grid = (uint32_t)(a.N * a.Hk * a.tiles * a.splits);
    cross_fwd_kernel<T, DP, BIAS, FEW><<<grid, kThreads, 0, s>>>(a);
}

template <typename T, int DP> void launch_shape(CrArgs &a, bool few, hipStream_t s) {
    if (a.bias)
        few ? launch<T, DP, true, true>(a, s) : launch<T, DP, true, false>(a, s);
    else
        few ? launch<T, DP, false, true>(a, s) : launch<T, DP, false, false>(a, s);
}

template <typename T> void launch_dim(CrArgs &a, bool few, hipStream_t s) {
    a.D <= 32 ? launch_shape<T, 32>(a, few, s) : a.D <= 64 ? launch_shape<T, 64>(a, few, s) : launch_shape<T, 128>(a, few, s);
}

}  // namespace

hipError_t launch_cross_fwd(CrArgs a, const CrPlan &p, void *ws, hipStream_t s) {
    a.splits = p.fwd_splits;
    a.part = (float *)((char *)ws + p.fwd_part);
    a.part_ml = (float2 *)((char *)ws + p.fwd_ml);
    a.bf16 ? launch_dim<bf16_t>(a, p.few, s) : launch_dim<float>(a, p.few, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    const int64_t rows = a.N * a.Hk * a.M, threads = rows * (a.D / 4);
    const uint32_t grid = (uint32_t)((threads + kThreads - 1) / kThreads);
    if (a.bf16)
        cross_join_kernel<bf16_t><<<grid, kThreads, 0, s>>>(a, a.bias != nullptr, rows);
    else
        cross_join_kernel<float><<<grid, kThreads, 0, s>>>(a, a.bias != nullptr, rows);
    return hipGetLastError();
}

}  // namespace evo

// evo_cross_fwd.hip -- attention to states of another length, forward
// (include/evo_cross_attn.h):  o = sigmoid(g) softmax(q k' / sqrt d + bias) v.
//
// One pass over the keys with the running maximum and sum of the softmax.
// Logits are formed transposed (S' = K Q'): a lane owns a query, so maximum and
// sum stay in the lane but for one exchange between its halves, and the
// probabilities go into O' = V' P' as they lie in their registers, V' by the
// transposing LDS read.  Matrix and vector units overlap between the two waves of
// a SIMD.  Within a wave as well (the products with V a step late, among the next
// exponentials) long calls were 0 to 4% slower, 4 rows of 1024 x 1024 at 128 channels
// with a bias 41 us against 37; a few steps with a bias were 2 to 5% faster.  Two shapes of
// workgroup:
//   rows: four waves of 32 queries, all waves the same keys
//   few:  two waves that share 32 queries and take turns with the keys (fp32: 64
//         queries); for single tokens, where reading K and V is all there is to do
// and where the tiles of rows do not fill the GPU, the keys are split over
// workgroups whose partial results a second kernel joins.
//
// The running maximum is kept on whole powers of two (its base-2 logarithm is an
// integer): rescaling is then exact.  Far from zero, where fp32 has no such numbers, it is
// kept as two (Ref).
//
// Long calls keep the matrix and the vector unit busy 49 and 56% of the time at 128
// channels: 4096 queries to 8191 keys, 16 heads, bf16, 274 to 282 us (975 to 1000 TFLOP/s); at 64 channels
// 2 x 4096 to 4096, 16 heads, 173 to 177 us (780 to 800), at 32 114 to 124 us (555 to 600).  fp32 runs at 101 to 116 of the
// 150 TFLOP/s of a library product.  Single tokens are bound by memory: 16 rows, 16 / 4
// heads of 128, 4097 keys 20.6 + 4.0 us (4.6 TB/s of the kept keys).
#include "evo_cross.h"

namespace evo {
namespace {

constexpr int kJoinThreads = 64;

// shape of a workgroup: QW waves of queries times KW waves of keys, KT keys a step
template <typename T, bool FEW> struct Shape {
    static constexpr bool WIDE = sizeof(typename Ty<T>::E) == 4;
    static constexpr int QW = FEW ? (WIDE ? 2 : 1) : 4, KW = FEW && !WIDE ? 2 : 1, THREADS = 64 * QW * KW;
    static constexpr int KT = WIDE ? 32 : 64, KPW = KT / KW, NS = KPW / 32, ROWS = 32 * QW;
};

// K and V of two steps
template <typename T, int DP, bool FEW> struct Lds {
    using S = Shape<T, FEW>;
    static constexpr int TILE = S::KT * DP, SIZE = 4 * TILE * (int)sizeof(typename Ty<T>::E);
    static_assert(S::KW == 1 || 2 * (DP / 32 * 16 + 3) * 256 <= SIZE, "the waves' results fit, at the end");
};

template <typename T, int DP, bool BIAS, bool FEW>
__global__ __launch_bounds__((Shape<T, FEW>::THREADS), (FEW || (Shape<T, FEW>::WIDE && DP == 128) ? 1 : 2)) void cross_fwd_kernel(CrArgs a) {
    using Y = Ty<T>;
    using E = typename Y::E;
    using Frag = typename Y::Frag;
    using S = Shape<T, FEW>;
    using L = Lds<T, DP, FEW>;
    using LT = Tile<T, DP>;
    constexpr int NK = DP / Y::KS, DT = DP / 32, GP = 32 / Y::KS, NS = S::NS;
    __shared__ __attribute__((aligned(16))) char lds[L::SIZE];
    const float inf = __builtin_inff();

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    const int qw = wave % S::QW, kw = wave / S::QW;
    uint32_t u = xcd_unit32(blockIdx.x, gridDim.x);
    const int split = u % a.splits;
    u /= a.splits;
    const int tile = u % a.tiles;
    const uint32_t unit = u / a.tiles;
    const int64_t n = unit / a.Hk;
    const int hk = unit % a.Hk;

    using Bits = KeyBits<S::KT>;
    using Cp = Copy<T, DP, S::KT, S::THREADS>;
    const E *kbase = (const E *)a.k + n * a.k_row + (int64_t)hk * a.D;
    const E *vbase = (const E *)a.v + n * a.k_row + (int64_t)hk * a.D;
    const uint8_t *mrow = a.mask ? a.mask + n * a.Lk : nullptr;
    int t0 = split * a.per_split, t1 = min(t0 + a.per_split, a.ntiles);
    // (a few steps are sooner done than looked for)
    if (mrow && t1 - t0 > 8) kept_range<S::KT, S::THREADS>(mrow, a.Lk, tid, (int *)lds, t0, t1);
    E *const kt0 = (E *)lds, *const vt0 = kt0 + 2 * L::TILE;
    const bool full_d = a.D == DP;
    auto request = [&](int step, bool whole, auto keep) {
        const int64_t off = (int64_t)step * S::KT * a.k_tok;
        Cp::run(kt0 + (step & 1) * L::TILE, whole, a.D, wave, lane, [&](int r) { return kbase + off + (int64_t)r * a.k_tok; }, keep);
        Cp::run(vt0 + (step & 1) * L::TILE, whole, a.D, wave, lane, [&](int r) { return vbase + off + (int64_t)r * a.k_tok; }, keep);
    };
    typename Bits::Bytes bytes = {}, bytes2 = {};
    if (t0 < t1) {
        bytes = Bits::request(mrow, t0 * S::KT, a.Lk, lane);
        bytes2 = Bits::request(mrow, (t0 + 1) * S::KT, a.Lk, lane);
    }

    // the lane's query
    const int x = tile * S::ROWS + qw * 32 + (lane & 31);
    const bool on = x < a.M;
    const int xc = on ? x : a.M - 1, t = token_of(a, xc), head = hk * a.G + (xc - t * a.G);
    Frag qf[NK];
    load_rows<T, DP>(qf, (const E *)a.q + n * a.q_row + (int64_t)t * a.q_tok + (int64_t)head * a.D, a.D, on, h);
    const BiasRow<T> brow(a, BIAS ? (n / a.rpb * a.H + head) * a.Lq + t : 0);
    typename BiasRow<T>::Raw braw[BIAS ? NS : 1];
    auto request_bias = [&](int step) {
#pragma unroll
        for (int b = 0; b < NS; ++b)
            if (BIAS) braw[BIAS ? b : 0] = brow.request(step * S::KT + (kw * NS + b) * 32, h);
    };
    constexpr bool EARLY = DP <= 64;  // the gate's values wait in registers where there is room
    const E *grow = a.gate ? (const E *)a.gate + n * a.q_row + (int64_t)t * a.q_tok + (int64_t)head * a.D : nullptr;
    Four<E> gv[EARLY ? DT * 4 : 1];
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
    Bits now, next;
    next.set(bytes);
    bytes = bytes2;
    if (t0 < t1) {
        request_bias(t0);
        request(t0, full_d && next.all(), [&](int r) { return next.get(r); });
    }

    f32x16 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = zero16();
    // what the running sums are against, as -hi and lo (0, 0 before the first key), how far a logit may rise above it, whether
    // it is far from zero for any of the wave's queries; sum of the lane's half of the keys
    float shift = 0.0f, lo = 0.0f, lag = -inf, sum = 0.0f;
    bool far = false;
    const float to2 = BIAS ? kLog2e : a.scale * kLog2e;
    for (int step = t0; step < t1; ++step) {
        copies_done_and_barrier();
        now = next;
        const E *kt = kt0 + (step & 1) * L::TILE, *vt = vt0 + (step & 1) * L::TILE;
        if (step + 1 < t1) {
            next.set(bytes);
            bytes = Bits::request(mrow, (step + 2) * S::KT, a.Lk, lane);
            request(step + 1, full_d && next.all(), [&](int r) { return next.get(r); });
        }
        f32x16 s[NS];
        float top = -inf;
#pragma unroll
        for (int b = 0; b < NS; ++b) s[b] = zero16();
#pragma unroll
        for (int kk = 0; kk < NK; ++kk)
#pragma unroll
            for (int b = 0; b < NS; ++b) Y::mma(s[b], LT::row(kt, (kw * NS + b) * 32 + (lane & 31), kk, h), qf[kk]);
        if (BIAS) {
#pragma unroll
            for (int b = 0; b < NS; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = fmaf(s[b][i], a.scale, BiasRow<T>::value(braw[BIAS ? b : 0], i));
        }
        if (!now.all()) {
#pragma unroll
            for (int b = 0; b < NS; ++b) {
                const uint32_t bits = now.sub(kw * NS + b);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = where_kept(bits, i, s[b][i], kMinusInf);
            }
        }
#pragma unroll
        for (int b = 0; b < NS; ++b)
#pragma unroll
            for (int i = 0; i < 16; i += 2) top = fmaxf(fmaxf(top, s[b][i]), s[b][i + 1]);
        if (BIAS && step + 1 < t1) request_bias(step + 1);
        top = half_max(top);
        if ((BIAS ? top : top * a.scale) <= kNoKey) top = -inf;  // no key: such logits give exp2(-inf) against 0, too
        // the reference rises only when it has fallen behind by 2^8: sums and probabilities
        // stay within fp32 and keep their relative precision
        float over = fmaf(top, to2, shift);
        if (far) over -= lo;
        if (__any(over > lag)) {
            const bool had = lag > 0.0f;
            Ref to = {-shift, lo};
            if (over > (had ? 0.0f : -inf)) {
                to = reference(top, to2);
                lag = 8.0f;
            }
            const float by = had ? (-shift - to.hi) + (lo - to.lo) : 0.0f, whole = __builtin_rintf(by);
            const int n = (int)fmaxf(whole, -1000.0f);
            sum = ldexpf(sum, n);
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] = ldexpf(o[d][i], n);
            if (__any(by != whole)) {
                const float f = __builtin_amdgcn_exp2f(by - whole);
                sum *= f;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] *= f;
            }
            shift = -to.hi;
            lo = to.lo;
            far = __any(lo != 0.0f);
        }
        float times = to2, plus = shift;
        if (far) {
#pragma unroll
            for (int b = 0; b < NS; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = fmaf(s[b][i], to2, shift) - lo;
            times = 1.0f, plus = 0.0f;
        }
#pragma unroll
        for (int b = 0; b < NS; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[b][i] = __builtin_amdgcn_exp2f(fmaf(s[b][i], times, plus));
                sum += s[b][i];
            }
#pragma unroll
        for (int b = 0; b < NS; ++b)
#pragma unroll
            for (int g = 0; g < GP; ++g) {
                const Frag p = Y::pack(s[b], g);
#pragma unroll
                for (int d = 0; d < DT; ++d) Y::mma(o[d], LT::col(vt, (kw * NS + b) * 32 + Y::KS * g, 32 * d, lane), p);
            }
    }

    sum = half_sum(sum);
    Ref ref = {lag > 0.0f ? -shift : -inf, lo};
    if (S::KW > 1) {
        // the two waves' maxima, sums and results, joined: wave kw takes every other block of channels
        float *all = (float *)lds;
        constexpr int PER = DT * 16 + 3;
        __syncthreads();
        float *mine = all + wave * PER * 64 + lane;
        mine[0] = ref.hi;
        mine[64] = ref.lo;
        mine[128] = sum;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) mine[(3 + d * 16 + i) * 64] = o[d][i];
        __syncthreads();
        Ref rj[S::KW];
        float mj[S::KW];
        ref = Ref{-inf, 0.0f};
#pragma unroll
        for (int j = 0; j < S::KW; ++j) {
            const float *from = all + (j * S::QW + qw) * PER * 64 + lane;
            rj[j] = Ref{from[0], from[64]};
            if (above(rj[j], ref)) ref = rj[j];
        }
        sum = 0.0f;
#pragma unroll
        for (int j = 0; j < S::KW; ++j) {
            mj[j] = rj[j].hi > -inf ? __builtin_amdgcn_exp2f((rj[j].hi - ref.hi) + (rj[j].lo - ref.lo)) : 0.0f;
            sum += mj[j] * all[(j * S::QW + qw) * PER * 64 + 128 + lane];
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            if (d % S::KW != kw) continue;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float v = 0.0f;
#pragma unroll
                for (int j = 0; j < S::KW; ++j) v += mj[j] * all[((j * S::QW + qw) * PER + 3 + d * 16 + i) * 64 + lane];
                o[d][i] = v;
            }
        }
    }
    if (!on) return;
    if (a.splits > 1) {
        const int64_t row = ((int64_t)split * a.N * a.Hk + unit) * a.M + x;
        if (kw == 0 && h == 0) a.part_ml[row] = float2{ref.hi, sum}, a.part_lo[row] = ref.lo;
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
    const float inv = sum > 0.0f ? 1.0f / sum : sum;
    if (kw == 0 && h == 0) a.lse[(n * a.H + head) * a.Lq + t] = log_of(sum, ref);
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
                const Four<E> raw = EARLY ? gv[EARLY ? d * 4 + i / 4 : 0] : gate_at(d, i / 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) g[j] = sigmoid(__uint_as_float(raw.bits(j)));
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) e[j] = Y::e(o[d][i + j] * inv * g[j]);
            __builtin_memcpy(__builtin_assume_aligned(orow + c, sizeof(e)), e, sizeof(e));
        }
    }
}

// Joins the splits of a row: one thread per four channels
template <typename T>
__global__ __launch_bounds__(kJoinThreads) void cross_join_kernel(CrArgs a, int64_t rows) {
    using Y = Ty<T>;
    using E = typename Y::E;
    const int per = a.D / 4;
    const int64_t at = (int64_t)blockIdx.x * kJoinThreads + threadIdx.x;
    const int64_t row = at / per;
    if (row >= rows) return;
    const int c = (int)(at - row * per) * 4;
    const int64_t unit = row / a.M, n = unit / a.Hk;
    const int x = (int)(row - unit * a.M), t = token_of(a, x), head = (int)(unit - n * a.Hk) * a.G + x - t * a.G;
    const int64_t tok = (int64_t)head * a.D + c;
    Four<E> gv = {};
    if (a.gate) gv = load4((const E *)a.gate + n * a.q_row + (int64_t)t * a.q_tok + tok);
    // reference and sum over the splits, read ahead
    const float inf = __builtin_inff();
    Ref ref = {-inf, 0.0f};
    float sum = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int j = 0; j < a.splits; ++j) {
        const float2 ml = a.part_ml[j * rows + row];
        const f32x4 p = *reinterpret_cast<const f32x4 *>(a.part + (j * rows + row) * a.D + c);
        const float higher = fmaxf(ref.hi, ml.x), to = higher > -inf ? higher : 0.0f;
        const float f = __builtin_amdgcn_exp2f(ml.x - to), old = __builtin_amdgcn_exp2f(ref.hi - to);
        sum = fmaf(ml.y, f, sum * old);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = fmaf(p[i], f, o[i] * old);
        ref.hi = higher;
    }
    // (next to a reference near zero those far off count nothing, whatever their lo)
    if (fabsf(ref.hi) >= kFar && ref.hi > -inf) {
        ref = Ref{-inf, 0.0f};
        sum = 0.0f;
        o = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int j = 0; j < a.splits; ++j) {
            const float2 ml = a.part_ml[j * rows + row];
            const Ref r = {ml.x, a.part_lo[j * rows + row]};
            if (r.hi == -inf) continue;
            const Ref to = above(r, ref) ? r : ref;
            const float f = __builtin_amdgcn_exp2f((r.hi - to.hi) + (r.lo - to.lo)), old = __builtin_amdgcn_exp2f((ref.hi - to.hi) + (ref.lo - to.lo));
            sum = fmaf(ml.y, f, sum * old);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = fmaf(a.part[(j * rows + row) * a.D + c + i], f, o[i] * old);
            ref = to;
        }
    }
    const float inv = sum > 0.0f ? 1.0f / sum : sum;
    if (c == 0) a.lse[(n * a.H + head) * a.Lq + t] = log_of(sum, ref);
    E e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float g = a.gate ? sigmoid(__uint_as_float(gv.bits(i))) : 1.0f;
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
    cross_fwd_kernel<T, DP, BIAS, FEW><<<grid, S::THREADS, 0, s>>>(a);
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
    if (p.brief) return launch_cross_short(a, p, s);
    a.splits = p.fwd_splits;
    a.part = (float *)((char *)ws + p.fwd_part);
    a.part_ml = (float2 *)((char *)ws + p.fwd_ml);
    a.part_lo = (float *)((char *)ws + p.fwd_lo);
    a.bf16 ? launch_dim<bf16_t>(a, p.few, s) : launch_dim<float>(a, p.few, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    const int64_t rows = a.N * a.Hk * a.M, threads = rows * (a.D / 4);
    const uint32_t grid = (uint32_t)((threads + kJoinThreads - 1) / kJoinThreads);
    if (a.bf16)
        cross_join_kernel<bf16_t><<<grid, kJoinThreads, 0, s>>>(a, rows);
    else
        cross_join_kernel<float><<<grid, kJoinThreads, 0, s>>>(a, rows);
    return hipGetLastError();
}

}  // namespace evo

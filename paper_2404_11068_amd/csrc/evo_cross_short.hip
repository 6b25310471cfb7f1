// evo_cross_short.hip -- attention to few states (up to 128 keys), forward
// (include/evo_cross_attn.h): residues of every row of an alignment, or of every
// pair, to a handful of states, with one pair bias for all rows.
//
// All logits of a query are in registers at once, and a workgroup walks over rows
// of the batch with the same queries' positions: what is the same for all of them,
// the bias (its rows are read in pieces of 64 bytes, the slowest loads of all), is
// read once, and while a row is worked on, K and V of the next are copied to LDS
// and its queries and gate to registers.  Before, a workgroup a row: 128 rows of 256
// queries to 77 keys, 8 heads of 32, gate, bias, mask took 30 us, the bias' loads
// half of it; now 23 (vector unit 45% busy, waves wait 47% of
// their time: two workgroups a CU fit the registers).
//
// Two shapes: the four waves of a workgroup share a row (32 queries each), or each
// has a row of its own, for up to 32 queries, with no barriers at all.
#include "evo_cross.h"

namespace evo {
namespace {

constexpr int kThreads = 256;

template <typename T, int DP, int NB, bool ONE> struct ShortLds {
    static constexpr int TILE = NB * 32 * DP, GROUPS = ONE ? 4 : 1;
    static constexpr int SIZE = GROUPS * 4 * TILE * (int)sizeof(typename Ty<T>::E);  // K and V of two rows
    static constexpr bool FITS = SIZE <= 128 * 1024;
};

template <typename T, int DP, bool BIAS, int NB, bool ONE>
__global__ __launch_bounds__(kThreads, (ShortLds<T, DP, NB, ONE>::SIZE > 80 * 1024 ? 1 : 2)) void cross_short_kernel(CrArgs a) {
    using Y = Ty<T>;
    using E = typename Y::E;
    using Frag = typename Y::Frag;
    using LT = Tile<T, DP>;
    using L = ShortLds<T, DP, NB, ONE>;
    constexpr int NK = DP / Y::KS, DT = DP / 32, GP = 32 / Y::KS, KT = NB * 32, NW = (KT + 63) / 64;
    __shared__ __attribute__((aligned(16))) E lds[L::SIZE / sizeof(E)];
    const float inf = __builtin_inff();

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    // splits: chunks of per_split rows of a plane, tiles: tiles of queries (ONE: one)
    uint32_t u = xcd_unit32(blockIdx.x, gridDim.x);
    const int tile = u % a.tiles;
    u /= a.tiles;
    const int hk = u % a.Hk;
    u /= a.Hk;
    const int chunk = u % a.splits;
    const int64_t plane = u / a.splits;
    const int64_t p1 = (plane + 1) * a.rpb;
    int64_t n0 = plane * a.rpb + (int64_t)chunk * a.per_split, n1 = min(n0 + a.per_split, p1);
    int64_t stride = 1;
    if (ONE) n0 += wave, stride = 4;

    const int x = (ONE ? 0 : tile * 128 + wave * 32) + (lane & 31);
    const bool on = x < a.M;
    const int xc = on ? x : a.M - 1, t = token_of(a, xc), head = hk * a.G + (xc - t * a.G);
    const int64_t qat = (int64_t)t * a.q_tok + (int64_t)head * a.D, oat = (int64_t)t * a.o_tok + (int64_t)head * a.D;
    const BiasRow<T> brow(a, BIAS ? (plane * a.H + head) * a.Lq + t : 0);
    typename BiasRow<T>::Raw bias[BIAS ? NB : 1];
    if (BIAS) {
#pragma unroll
        for (int b = 0; b < NB; ++b) bias[BIAS ? b : 0] = brow.request(32 * b, h);
    }
    const float to2 = BIAS ? kLog2e : a.scale * kLog2e;

    E *const mine = lds + (ONE ? wave * 4 * L::TILE : 0);
    const bool full_d = a.D == DP;
    // the mask bytes of a row, and K and V of its kept keys
    struct Bytes { uint8_t b[NW]; };
    struct Bits { uint64_t w[NW]; };
    auto bytes_of = [&](int64_t n) {
        Bytes r;
#pragma unroll
        for (int j = 0; j < NW; ++j) {
            const int key = 64 * j + lane;
            r.b[j] = key < a.Lk && n < n1 ? (a.mask ? a.mask[n * a.Lk + key] : (uint8_t)1) : (uint8_t)0;
        }
        return r;
    };
    auto bits_of = [&](const Bytes &r) {
        Bits w;
#pragma unroll
        for (int j = 0; j < NW; ++j) w.w[j] = __ballot(r.b[j] != 0);
        return w;
    };
    auto copy = [&](int64_t n, int buf, const Bits &bits) {
        const E *k = (const E *)a.k + n * a.k_row + (int64_t)hk * a.D, *v = (const E *)a.v + n * a.k_row + (int64_t)hk * a.D;
        E *kt = mine + buf * 2 * L::TILE;
        bool whole = full_d;
#pragma unroll
        for (int j = 0; j < NW; ++j) whole = whole && bits.w[j] == (64 * j + 64 <= KT ? ~0ull : 0xffffffffull);
        auto keep = [&](int r) { return ((r < 64 ? bits.w[0] : bits.w[NW - 1]) >> (r & 63)) & 1; };
        if constexpr (ONE) {
            Copy<T, DP, KT, 64>::run(kt, whole, a.D, 0, lane, [&](int r) { return k + (int64_t)r * a.k_tok; }, keep);
            Copy<T, DP, KT, 64>::run(kt + L::TILE, whole, a.D, 0, lane, [&](int r) { return v + (int64_t)r * a.k_tok; }, keep);
        } else {
            // 32 keys of 32 bf16 channels are half a step of the workgroup
            constexpr int TH = KT * LT::CH >= kThreads && KT * LT::CH % kThreads == 0 ? kThreads : 128;
            if (TH == kThreads || wave < 2) {
                Copy<T, DP, KT, TH>::run(kt, whole, a.D, wave, lane, [&](int r) { return k + (int64_t)r * a.k_tok; }, keep);
                Copy<T, DP, KT, TH>::run(kt + L::TILE, whole, a.D, wave, lane, [&](int r) { return v + (int64_t)r * a.k_tok; }, keep);
            }
        }
    };
    Frag qf[NK], qn[NK];
    Sixteen<E> gate[DT * 2];
    auto tokens_of = [&](int64_t n, Frag (&f)[NK]) {
        load_rows<T, DP>(f, (const E *)a.q + n * a.q_row + qat, a.D, on, h);
        if (a.gate) {
#pragma unroll
            for (int j = 0; j < DT * 2; ++j) gate[j].load((const E *)a.gate + n * a.q_row + qat, 16 * j, a.D, h);
        }
    };

    if (n0 >= n1) return;  // (the waves of a workgroup that meet at barriers have the same rows)
    const auto copies_done = [] { asm volatile("s_waitcnt vmcnt(0)" : : : "memory"); };
    Bytes bytes = bytes_of(n0), bytes2 = bytes_of(n0 + stride);
    tokens_of(n0, qn);
    Bits next = bits_of(bytes);
    copy(n0, 0, next);
    bytes = bytes2;
    copies_done();
    int buf = 0;
    for (int64_t n = n0; n < n1; n += stride, buf ^= 1) {
        // the wave's own copies have come in before the last row's stores: those are not waited for
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
        if (!ONE) asm volatile("s_barrier" : : : "memory");
        const Bits now = next;
        const E *kt = mine + buf * 2 * L::TILE, *vt = kt + L::TILE;
        Sixteen<E> g[DT * 2];
#pragma unroll
        for (int i = 0; i < NK; ++i) qf[i] = qn[i];
#pragma unroll
        for (int i = 0; i < DT * 2; ++i) g[i] = gate[i];
        if (n + stride < n1) {
            next = bits_of(bytes);
            bytes = bytes_of(n + 2 * stride);
            tokens_of(n + stride, qn);
            copy(n + stride, buf ^ 1, next);
        }
        f32x16 s[NB];
        float top = -inf;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const uint32_t bits = (uint32_t)(now.w[b >> 1] >> (32 * (b & 1)));
            const bool whole = bits == 0xffffffffu;
            s[b] = zero16();
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) Y::mma(s[b], LT::row(kt, 32 * b + (lane & 31), kk, h), qf[kk]);
            if (BIAS) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = fmaf(s[b][i], a.scale, BiasRow<T>::value(bias[BIAS ? b : 0], i));
            }
            if (!whole) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = where_kept(bits, i, s[b][i], kMinusInf);
            }
#pragma unroll
            for (int i = 0; i < 16; i += 2) top = fmaxf(fmaxf(top, s[b][i]), s[b][i + 1]);
        }
        // what the sums are against, as in the kernel for many keys
        top = half_max(top);
        if ((BIAS ? top : top * a.scale) <= kNoKey) top = -inf;
        Ref ref = {__builtin_ceilf(top * to2), 0.0f};
        const bool far = __any(fabsf(top * to2) >= kFar && top > -inf);
        float times = to2, plus = top > -inf ? -ref.hi : 0.0f;
        if (far) {
            if (top > -inf) ref = reference(top, to2), plus = -ref.hi;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = fmaf(s[b][i], to2, plus) - ref.lo;
            times = 1.0f, plus = 0.0f;
        }
        float sum = 0.0f;
        f32x16 o[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = zero16();
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[b][i] = __builtin_amdgcn_exp2f(fmaf(s[b][i], times, plus));
                sum += s[b][i];
            }
#pragma unroll
            for (int p = 0; p < GP; ++p) {
                const Frag f = Y::pack(s[b], p);
#pragma unroll
                for (int d = 0; d < DT; ++d) Y::mma(o[d], LT::col(vt, 32 * b + Y::KS * p, 32 * d, lane), f);
            }
        }
        sum = half_sum(sum);
        const float inv = sum > 0.0f ? 1.0f / sum : sum;
        copies_done();
        if (h == 0 && on) a.lse[(n * a.H + head) * a.Lq + t] = log_of(sum, ref);
        E *orow = (E *)a.out + n * a.o_row + oat;
#pragma unroll
        for (int j = 0; j < DT * 2; ++j) {
            Sixteen<E> e;
            if (a.gate) g[j].arrange();
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = o[j / 2][8 * (j & 1) + 4 * p + i] * inv;
                    if (a.gate) v[i] *= sigmoid(__uint_as_float(g[j].x[p].bits(i)));
                }
                e.set(p, v);
            }
            e.store(orow, 16 * j, a.D, h, on);
        }
    }
}

template <typename T, int DP, bool BIAS, int NB> hipError_t launch(const CrArgs &a, bool one, uint32_t grid, hipStream_t s) {
    if constexpr (ShortLds<T, DP, NB, true>::FITS) {
        if (one) {
            cross_short_kernel<T, DP, BIAS, NB, true><<<grid, kThreads, 0, s>>>(a);
            return hipGetLastError();
        }
    }
    // (the plan takes four waves a row in bf16 up to 32 channels only)
    if constexpr (sizeof(typename Ty<T>::E) == 2 && DP == 32) {
        if (!one) {
            cross_short_kernel<T, DP, BIAS, NB, false><<<grid, kThreads, 0, s>>>(a);
            return hipGetLastError();
        }
    }
    return hipErrorInvalidValue;
}

template <typename T, int DP> hipError_t launch_keys(const CrArgs &a, bool one, uint32_t grid, hipStream_t s) {
    switch ((a.Lk + 31) / 32) {
        case 1: return a.bias ? launch<T, DP, true, 1>(a, one, grid, s) : launch<T, DP, false, 1>(a, one, grid, s);
        case 2: return a.bias ? launch<T, DP, true, 2>(a, one, grid, s) : launch<T, DP, false, 2>(a, one, grid, s);
        case 3: return a.bias ? launch<T, DP, true, 3>(a, one, grid, s) : launch<T, DP, false, 3>(a, one, grid, s);
        case 4: return a.bias ? launch<T, DP, true, 4>(a, one, grid, s) : launch<T, DP, false, 4>(a, one, grid, s);
    }
    return hipErrorInvalidValue;
}

template <typename T> hipError_t launch_dim(const CrArgs &a, bool one, uint32_t grid, hipStream_t s) {
    return a.D <= 32 ? launch_keys<T, 32>(a, one, grid, s)
                     : a.D <= 64 ? launch_keys<T, 64>(a, one, grid, s) : launch_keys<T, 128>(a, one, grid, s);
}

}  // namespace

hipError_t launch_cross_short(CrArgs a, const CrPlan &p, hipStream_t s) {
    a.tiles = p.brief_one ? 1 : (a.M + 127) / 128;
    a.splits = p.brief_chunks;
    a.per_split = (int)((a.rpb + a.splits - 1) / a.splits);
    const uint32_t grid = (uint32_t)(a.N / a.rpb * a.splits * a.Hk * a.tiles);
    return a.bf16 ? launch_dim<bf16_t>(a, p.brief_one, grid, s) : launch_dim<float>(a, p.brief_one, grid, s);
}

}  // namespace evo

// evo_views.h -- whether two strided views of memory have a byte in common (host only).
//
// A view is n x len blocks of contiguous bytes, at i * row + j * tok.  Views of one packed
// buffer interleave: their address ranges overlap and their blocks do not.
#pragma once

#include <stdint.h>

namespace evo {

struct View {
    uintptr_t at;
    int64_t row, tok, n, len, block;  // strides (>= 0) and block in bytes, counts >= 1
};

struct ViewAxes {
    int64_t stride[2], count[2], block;  // outer axis first; a count of 1 where there is none
    int64_t span() const { return (count[0] - 1) * stride[0] + (count[1] - 1) * stride[1] + block; }
};

inline ViewAxes view_axes(const View &v) {
    ViewAxes a{{0, 0}, {1, 1}, v.block};
    const bool row_first = v.row >= v.tok;
    int k = 0;
    for (int i = 0; i < 2; ++i) {
        const bool row = (i == 0) == row_first;
        const int64_t s = row ? v.row : v.tok, c = row ? v.n : v.len;
        if (s > 0 && c > 1) a.stride[k] = s, a.count[k] = c, ++k;  // (blocks repeated in one place are one)
    }
    return a;
}

inline int64_t common_divisor(int64_t x, int64_t y) {
    while (y) {
        const int64_t r = x % y;
        x = y, y = r;
    }
    return x;
}

// `by`: from a's first byte to b's
inline bool axes_apart(const ViewAxes &a, const ViewAxes &b, int64_t by) {
    if (by >= a.span() || -by >= b.span()) return true;
    // all of a's blocks in one place within a period of all strides, all of b's in another
    int64_t period = 0;
    for (int i = 0; i < 2; ++i) {
        if (a.count[i] > 1) period = common_divisor(period, a.stride[i]);
        if (b.count[i] > 1) period = common_divisor(period, b.stride[i]);
    }
    if (period == 0) return false;
    const int64_t at = (by % period + period) % period;
    if (at >= a.block && at + b.block <= period) return true;
    // the longest stride, of one or of both, taken apart: the inner axes at the few distances where they could meet
    const int64_t s = a.stride[0] > b.stride[0] ? a.stride[0] : b.stride[0];
    ViewAxes x = a, y = b;
    int64_t nx = 1, ny = 1;
    const auto take = [s](ViewAxes &v, int64_t &n) {
        if (v.count[0] == 1 || v.stride[0] != s) return;
        n = v.count[0];
        v.stride[0] = v.stride[1], v.count[0] = v.count[1];
        v.stride[1] = 0, v.count[1] = 1;
    };
    take(x, nx);
    take(y, ny);
    // -span of y < by + k s < span of x, k from -(nx - 1) to ny - 1
    const auto floor_div = [](int64_t p, int64_t q) { return p >= 0 ? p / q : -((-p + q - 1) / q); };
    int64_t lo = floor_div(-y.span() - by, s) + 1, hi = floor_div(x.span() - by - 1, s);
    if (lo < 1 - nx) lo = 1 - nx;
    if (hi > ny - 1) hi = ny - 1;
    if (hi - lo >= 4) return false;
    for (int64_t k = lo; k <= hi; ++k)
        if (!axes_apart(x, y, by + k * s)) return false;
    return true;
}

// Never true of views that share a byte.  Exact for views whose strides are alike, as those of one packed buffer are;
// false for some others that interleave without touching.
inline bool views_apart(const View &a, const View &b) { return axes_apart(view_axes(a), view_axes(b), (int64_t)(b.at - a.at)); }

}  // namespace evo

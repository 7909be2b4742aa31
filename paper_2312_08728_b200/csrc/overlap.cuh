// Whether two matrices in memory share a byte.  Host side, without CUDA.
#pragma once
#include <cstdint>
#include <initializer_list>

namespace bmgdk {

// `rows` rows of `width` bytes, `ld` bytes apart (at least width).  A null pointer, no rows or no width: nothing.
struct Region {
    const void* base;
    int64_t rows, width, ld;
};
inline Region vector_region(const void* p, int64_t bytes) { return {p, 1, bytes, bytes}; }

typedef __int128 wide_int;
// sum over 0 <= i < n of floor((a i + b) / m), a, b >= 0, m > 0, by Euclid's steps
inline wide_int floor_sum(wide_int n, wide_int m, wide_int a, wide_int b) {
    wide_int sum = 0;
    while (n > 0) {
        sum += n * (n - 1) / 2 * (a / m) + n * (b / m);
        a %= m;
        b %= m;
        const wide_int top = a * n + b;
        if (top < m) break;
        n = top / m;
        b = top % m;
        const wide_int t = m;
        m = a;
        a = t;
    }
    return sum;
}
// sum over 0 <= i < n of floor((a i + c) / m) held between -1 and top, a, m > 0, top >= 0
inline wide_int held_floor_sum(wide_int n, wide_int m, wide_int a, wide_int c, wide_int top) {
    auto first = [&](wide_int least) { const wide_int i = least - c <= 0 ? 0 : (least - c + a - 1) / a; return i < n ? i : n; };  // the first i with a i + c >= least
    const wide_int from = first(0), to = first(top * m);
    return -from + (to > from ? floor_sum(to - from, m, a, a * from + c) : 0) + (n - to) * top;
}

// Row i of x meets the rows j of y with  y + j ly < x + i lx + wx  and  x + i lx < y + j ly + wy:  their number, summed over i, is a difference of two sums.
// Halves of one wide matrix, columns that take turns and the like share nothing, although their ranges of addresses do.
inline bool share_memory(const Region& x, const Region& y) {
    if (!x.base || !y.base || x.rows < 1 || y.rows < 1 || x.width < 1 || y.width < 1) return false;
    const wide_int lx = x.rows > 1 ? x.ld : x.width, ly = y.rows > 1 ? y.ld : y.width;
    const wide_int a = (wide_int)(uintptr_t)x.base, b = (wide_int)(uintptr_t)y.base;
    if (a >= b + (y.rows - 1) * ly + y.width || b >= a + (x.rows - 1) * lx + x.width) return false;
    if (x.rows == 1 && y.rows == 1) return true;
    const wide_int last = y.rows - 1;
    return held_floor_sum(x.rows, ly, lx, a - b + x.width - 1, last) > held_floor_sum(x.rows, ly, lx, a - b - y.width, last);
}
// whether what is written shares nothing with what is read, nor with anything else that is written
inline bool writes_apart(std::initializer_list<Region> written, std::initializer_list<Region> read) {
    for (const Region* w = written.begin(); w != written.end(); ++w) {
        for (const Region& r : read)
            if (share_memory(*w, r)) return false;
        for (const Region* v = written.begin(); v != w; ++v)
            if (share_memory(*w, *v)) return false;
    }
    return true;
}
// the same memory value for value, or none of it
inline bool same_or_apart(const Region& x, const Region& y) {
    return (x.base == y.base && x.rows == y.rows && x.width == y.width && (x.ld == y.ld || x.rows == 1)) || !share_memory(x, y);
}

}  // namespace bmgdk

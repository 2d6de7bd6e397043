// Which buffers of a call overlap. Host code without CUDA.
#pragma once
#include <algorithm>
#include <cstdint>
#include <vector>

struct Interval {
    uintptr_t lo, hi;
    bool out;
};

// An output range may overlap nothing else of the call. Sorts `iv`.
inline bool ranges_clash(std::vector<Interval> &iv)
{
    auto before = [](const Interval &a, const Interval &b) { return a.lo < b.lo; };
    if (!std::is_sorted(iv.begin(), iv.end(), before)) std::sort(iv.begin(), iv.end(), before);
    uintptr_t reach = 0, reach_out = 0;
    for (const Interval &i : iv) {
        if (i.lo < reach_out || (i.out && i.lo < reach)) return true;
        reach = std::max(reach, i.hi);
        if (i.out) reach_out = std::max(reach_out, i.hi);
    }
    return false;
}

// `rows` (at least 1) rows of `width` bytes that start `stride` (at least `width`) bytes apart.
struct RowRange {
    uintptr_t lo, width, stride, rows;
    bool out;
    uintptr_t hi() const { return lo + (rows - 1) * stride + width; }
};

// Whether a row of `m` meets [lo, hi).
inline bool rows_meet(const RowRange &m, uintptr_t lo, uintptr_t hi)
{
    const uintptr_t r = lo < m.lo + m.width ? 0 : (lo - m.lo - m.width) / m.stride + 1;      // the first row that ends behind lo
    return r < m.rows && m.lo + r * m.stride < hi;
}

// Whether rows of two matrices meet. Exact for rows equally far apart, as column slices of one buffer have them; of others the
// whole ranges are taken.
inline bool rows_meet(const RowRange &a, const RowRange &b)
{
    if (a.hi() <= b.lo || b.hi() <= a.lo) return false;
    if (b.lo < a.lo) return rows_meet(b, a);
    if (a.rows == 1) return rows_meet(b, a.lo, a.hi());
    if (b.rows == 1) return rows_meet(a, b.lo, b.hi());
    if (a.stride != b.stride) return true;
    const uintptr_t q = (b.lo - a.lo) / a.stride, d = (b.lo - a.lo) % a.stride;              // b's first row starts behind a's row q
    return (d < a.width && q < a.rows) || (d + b.width > a.stride && q + 1 < a.rows);
}

// The same for plain ranges `iv` and matrices `m` (a few). Sorts `iv`.
inline bool rows_clash(std::vector<Interval> &iv, const std::vector<RowRange> &m)
{
    std::vector<Interval> all(iv);
    for (const RowRange &r : m) all.push_back({r.lo, r.hi(), r.out});
    if (!ranges_clash(all)) return false;            // (nearly always: whole ranges lie apart)
    if (ranges_clash(iv)) return true;
    for (size_t i = 0; i < m.size(); ++i) {
        for (const Interval &x : iv)
            if ((x.out || m[i].out) && rows_meet(m[i], x.lo, x.hi)) return true;
        for (size_t j = 0; j < i; ++j)
            if ((m[i].out || m[j].out) && rows_meet(m[i], m[j])) return true;
    }
    return false;
}

// Checks of arguments that the operators on a filled pool share.
#pragma once

#include <algorithm>
#include <cstdint>
#include <utility>
#include <vector>

namespace pdkv {

constexpr int32_t kMaxTokens = 1 << 30;   // of a sequence or prefix: positions and their next tiles stay below 2^31

inline bool ranges_overlap(const void *a, size_t a_bytes, const void *b, size_t b_bytes)
{
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    return a_bytes && b_bytes && a0 < b0 + b_bytes && b0 < a0 + a_bytes;
}

// Rows of memory of one length at base + sum of i * stride, from `base` to before `end` (nothing where base is null).
struct Rows {
    uintptr_t base = 0, end = 0;
    int64_t bytes = 0, stride[3] = {0, 0, 0}, n[3] = {1, 1, 1};
    Rows(const void *p, int64_t row_bytes) : base(reinterpret_cast<uintptr_t>(p)), end(base + (p ? row_bytes : 0)), bytes(row_bytes) {}
    Rows(const void *p, int64_t row_len, int64_t elem, const int64_t *s, const int64_t *count, int axes) : Rows(p, row_len * elem)
    {
        for (int i = 0; i < axes; ++i) {
            n[i] = count[i];
            stride[i] = count[i] > 1 ? s[i] * elem : 0;
            if (end > base) end = count[i] > 0 ? end + stride[i] * (count[i] - 1) : base;
        }
    }
    std::vector<uintptr_t> starts() const
    {
        std::vector<uintptr_t> at;
        at.reserve((size_t)(n[0] * n[1] * n[2]));
        for (int64_t i = 0; i < n[0]; ++i)
            for (int64_t j = 0; j < n[1]; ++j)
                for (int64_t k = 0; k < n[2]; ++k) at.push_back(base + i * stride[0] + j * stride[1] + k * stride[2]);
        std::sort(at.begin(), at.end());
        return at;
    }
};

// Do a row of `a` and one of `b` share a byte?  Row by row only where their spans meet (views of one buffer).
inline bool meet(const Rows &a, const Rows &b)
{
    if (a.base >= b.end || b.base >= a.end || a.base == a.end || b.base == b.end) return false;
    const std::vector<uintptr_t> x = a.starts(), y = b.starts();
    for (size_t i = 0, j = 0; i < x.size() && j < y.size();) {
        if (x[i] < y[j] + b.bytes && y[j] < x[i] + a.bytes) return true;
        if (x[i] + a.bytes <= y[j])
            ++i;
        else
            ++j;
    }
    return false;
}

// The same where `one` is a single row: by the places of the others along their axes, whatever their number.
inline bool touches(const Rows &one, const Rows &many)
{
    if (one.base >= many.end || many.base >= one.end || one.base == one.end || many.base == many.end) return false;
    int64_t stride[3], n[3];
    int axes = 0;
    for (int i = 0; i < 3; ++i)
        if (many.n[i] > 1 && many.stride[i] > 0) {
            int at = axes++;
            for (; at > 0 && stride[at - 1] < many.stride[i]; --at) {
                stride[at] = stride[at - 1];
                n[at] = n[at - 1];
            }
            stride[at] = many.stride[i];
            n[at] = many.n[i];
        }
    struct Walk {
        const Rows &one;
        const int64_t *stride, *n;
        int axes;
        int64_t bytes;
        bool at(int axis, int64_t base) const   // base: bytes from the start of `one`
        {
            const int64_t end = (int64_t)(one.end - one.base);
            if (axis == axes) return base < end && base + bytes > 0;
            int64_t wide = bytes;
            for (int i = axis + 1; i < axes; ++i) wide += stride[i] * (n[i] - 1);
            const int64_t s = stride[axis], before = -base - wide;   // base + i s + wide > 0,  base + i s < end
            const int64_t first = before < 0 ? 0 : before / s + 1, last = base >= end ? -1 : std::min(n[axis] - 1, (end - base - 1) / s);
            if (last - first >= 2 && s >= wide) return true;   // the second lies inside
            for (int64_t i = first; i <= last; ++i)
                if (at(axis + 1, base + i * s)) return true;
            return false;
        }
    };
    return Walk{one, stride, n, axes, many.bytes}.at(0, (int64_t)(many.base - one.base));
}

// Rows with the axes (sequences, tokens, heads): do all of them lie apart from all of `b`'s by their places within one token?  A
// quick answer for views of one buffer that holds a token's queries, keys and values side by side; false says nothing.
inline bool apart_in_token(const Rows &a, const Rows &b)
{
    const int64_t step = a.n[1] > 1 ? a.stride[1] : b.stride[1];
    if (step <= 0 || (b.n[1] > 1 && b.stride[1] != step) || a.stride[0] % step || b.stride[0] % step) return false;
    const int64_t wide_a = a.bytes + a.stride[2] * (a.n[2] - 1), wide_b = b.bytes + b.stride[2] * (b.n[2] - 1);
    const int64_t d = (int64_t)(b.base - a.base) % step, from = d < 0 ? d + step : d;
    return wide_a <= from && from + wide_b <= step;
}

inline bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

inline int32_t log2_of(int32_t n)
{
    for (int b = 0; b < 31; ++b)
        if (n == 1 << b) return b;
    return -1;
}

// Do rows of `len` entries at i0*s0 + i1*s1 + i2*s2 lie apart from one another?  Axes of one entry do
// not count; the others have to nest (each stride spans everything inside it).
inline bool rows_apart(int64_t len, const int64_t *stride, const int64_t *n, int axes)
{
    std::vector<std::pair<int64_t, int64_t>> ax;
    for (int i = 0; i < axes; ++i) {
        if (n[i] > 1) ax.emplace_back(stride[i], n[i]);
        if (stride[i] < 0) return false;
    }
    std::sort(ax.begin(), ax.end());
    int64_t span = len;
    for (const auto &a : ax) {
        if (a.first < span) return false;
        span += a.first * (a.second - 1);
    }
    return true;
}

}  // namespace pdkv

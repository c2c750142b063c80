// Whether the rows of two tensors share memory.  Host code, without HIP or torch.
#pragma once
#include <algorithm>
#include <cstdint>

namespace xls {

// batch x length rows of `width` bytes, their steps in bytes and not negative.
struct Span {
    int64_t at, batch, length, batch_step, token_step, width;
    bool operator==(const Span &o) const
    {
        return at == o.at && batch == o.batch && length == o.length && width == o.width && (batch <= 1 || batch_step == o.batch_step) && (length <= 1 || token_step == o.token_step);
    }
};

namespace overlap_detail {

inline int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b != 0 && (a < 0) != (b < 0)); }

// Rows that lie next to each other as one, sequences that go on at even steps as one: what is left is as few rows as can be.
inline Span merged(Span s)
{
    if (s.length == 1) {
        s.length = s.batch;
        s.token_step = s.batch_step;
        s.batch = 1;
    } else if (s.batch > 1 && s.batch_step == s.length * s.token_step) {
        s.length *= s.batch;
        s.batch = 1;
    }
    if (s.length > 1 && s.token_step <= s.width) {      // no gaps
        s.width += (s.length - 1) * s.token_step;
        s.length = 1;
    }
    if (s.length == 1 && s.batch > 1) return merged({s.at, 1, s.batch, 0, s.batch_step, s.width});
    if (s.length == 1) s.token_step = 0;
    if (s.batch == 1) s.batch_step = 0;
    return s;
}

// Whether low < at + i * outer + j * inner < high for some i of [i0, i1] and j of [j0, j1].
inline bool meets(int64_t at, int64_t outer, int64_t i0, int64_t i1, int64_t inner, int64_t j0, int64_t j1, int64_t low, int64_t high)
{
    if (outer < inner) {
        std::swap(outer, inner);
        std::swap(i0, j0);
        std::swap(i1, j1);
    }
    if (outer == 0) return low < at && at < high;
    // the i for which some j could do: few, unless the rows of a tensor lie across each other
    i0 = std::max(i0, floor_div(low - at - j1 * inner, outer) + 1);
    i1 = std::min(i1, -floor_div(-(high - at - j0 * inner), outer) - 1);
    if (i1 - i0 > 1 << 16) i1 = i0 + (1 << 16);
    for (int64_t i = i0; i <= i1; ++i) {
        const int64_t a = at + i * outer;
        if (inner == 0 ? low < a && a < high : std::max(j0, floor_div(low - a, inner) + 1) <= std::min(j1, -floor_div(-(high - a), inner) - 1)) return true;
    }
    return false;
}

}  // namespace overlap_detail

// True where a byte of a row of `a` is one of a row of `b`.  Exact for rows at the same steps, for memory without gaps, and wherever one of the two has no more than 4096 rows; tensors with
// more rows than that at other steps whose ranges lie across each other are taken to be apart.
inline bool overlap(const Span &a_, const Span &b_)
{
    using namespace overlap_detail;
    if (a_.batch <= 0 || a_.length <= 0 || a_.width <= 0 || b_.batch <= 0 || b_.length <= 0 || b_.width <= 0) return false;
    const auto end = [](const Span &s) { return s.at + (s.batch - 1) * s.batch_step + (s.length - 1) * s.token_step + s.width; };
    if (end(a_) <= b_.at || end(b_) <= a_.at) return false;
    Span a = merged(a_), b = merged(b_);
    if (a.batch * a.length < b.batch * b.length) std::swap(a, b);
    // b has the fewer rows.  A row of a and one of b meet where the first begins less than its width before the other and less than the other's width behind it.
    if ((b.batch == 1 || a.batch_step == b.batch_step) && (b.length == 1 || a.token_step == b.token_step))
        return meets(a.at - b.at, a.batch_step, 1 - b.batch, a.batch - 1, a.token_step, 1 - b.length, a.length - 1, -a.width, b.width);
    if (b.batch * b.length > 4096) return false;
    for (int64_t i = 0; i < b.batch; ++i)
        for (int64_t j = 0; j < b.length; ++j)
            if (meets(a.at - b.at - i * b.batch_step - j * b.token_step, a.batch_step, 0, a.batch - 1, a.token_step, 0, a.length - 1, -a.width, b.width)) return true;
    return false;
}

// True where two rows of one tensor share a byte.
inline bool overlaps_itself(const Span &s)
{
    if (s.batch <= 0 || s.length <= 0 || s.width <= 0) return false;
    return (s.length > 1 && s.token_step < s.width) ||
           (s.batch > 1 && overlap_detail::meets(0, s.batch_step, 1, s.batch - 1, s.token_step, 1 - s.length, s.length - 1, -s.width, s.width));
}

}  // namespace xls

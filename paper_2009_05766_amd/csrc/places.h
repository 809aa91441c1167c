// Where the operands of a call lie in memory, and whether two of them share any of it: plain host code.
//
// An operand is a batch of matrices: `batch` of them `step` bytes apart, each of `rows` rows of `cols` bytes that start `ld` bytes apart.  Operands that only
// interleave (columns of one wide matrix, slices of workers' rows of parameters) share nothing and are told from those that do by division, not by
// their hulls alone.
#pragma once
#include <stdint.h>

namespace netmax {

struct Place {
    int64_t lo = 0, hi = 0, batch = 0, rows = 0, cols = 0, ld = 0, step = 0;                // hi: behind the last byte; lo == hi: nothing there
    Place() { }
    // `size`: bytes of an element; all others in elements.
    Place(const void *p, int64_t size, int64_t batch_, int64_t rows_, int64_t cols_, int64_t ld_, int64_t step_)
        : batch(batch_), rows(rows_), cols(cols_ * size), ld(ld_ * size), step(step_ * size)
    {
        if (!p || batch <= 0 || rows <= 0 || cols <= 0) { batch = rows = cols = ld = step = 0; return; }
        if (rows > 1 && ld == cols) { cols *= rows; rows = 1; }
        if (rows == 1) ld = 0;
        if (step == 0) batch = 1;
        if (batch > 1 && rows == 1 && step == cols) { cols *= batch; batch = 1; }
        if (batch > 1 && rows > 1 && step == rows * ld) { rows *= batch; batch = 1; }
        if (batch == 1) step = 0;
        lo = (int64_t)(uintptr_t)p;
        hi = lo + (batch - 1) * step + span();
    }
    int64_t span() const { return (rows - 1) * ld + cols; }                                 // of one matrix
    bool operator==(const Place &o) const { return lo == o.lo && batch == o.batch && rows == o.rows && cols == o.cols && ld == o.ld && step == o.step; }
};

inline int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b != 0 && a < 0); }   // b > 0
// The whole numbers n with above < at + n step < below: first .. last.
inline int64_t first_between(int64_t above, int64_t at, int64_t step) { return floor_div(above - at, step) + 1; }
inline int64_t last_between(int64_t below, int64_t at, int64_t step) { return -floor_div(at - below, step) - 1; }
inline bool any_between(int64_t above, int64_t below, int64_t at, int64_t step, int64_t from, int64_t to)
{
    if (step == 0) return from <= to && above < at && at < below;
    const int64_t first = first_between(above, at, step), last = last_between(below, at, step);
    return (first > from ? first : from) <= (last < to ? last : to);
}

// Rows that lie at different distances are compared one by one, pairs of matrices too, up to this many in all; operands that would need more count as sharing memory.
constexpr int64_t MOST_COMPARISONS = 1 << 20;

// Whether a matrix of a and one of b, which starts `off` bytes behind it, have a byte in common.
inline bool matrices_share(const Place &a, const Place &b, int64_t off, int64_t &left)
{
    if (--left < 0) return true;
    if (off >= a.span() || -off >= b.span()) return false;
    if (a.rows == 1) return any_between(-b.cols, a.cols, off, b.ld, 0, b.rows - 1);
    if (b.rows == 1) return any_between(-a.cols, b.cols, -off, a.ld, 0, a.rows - 1);
    if (a.ld == b.ld) return any_between(-b.cols, a.cols, off, a.ld, 1 - a.rows, b.rows - 1);
    const bool swap = b.rows < a.rows;
    const Place &few = swap ? b : a, &many = swap ? a : b;
    const int64_t from = swap ? -off : off;                                                 // of `many` behind `few`
    if ((left -= few.rows) < 0) return true;
    for (int64_t r = 0; r < few.rows; ++r)
        if (any_between(-many.cols, few.cols, from - r * few.ld, many.ld, 0, many.rows - 1)) return true;
    return false;
}

inline bool share_memory(const Place &a, const Place &b)
{
    if (a.lo == a.hi || b.lo == b.hi || a.hi <= b.lo || b.hi <= a.lo) return false;
    const int64_t off = b.lo - a.lo;
    int64_t left = MOST_COMPARISONS;
    if (a.batch > 1 && a.step == b.step) {                          // only the difference of their numbers counts
        int64_t first = first_between(-b.span(), off, a.step), last = last_between(a.span(), off, a.step);
        if (first < 1 - a.batch) first = 1 - a.batch;
        if (last > b.batch - 1) last = b.batch - 1;
        for (int64_t n = first; n <= last; ++n)
            if (matrices_share(a, b, off + n * a.step, left)) return true;
        return false;
    }
    for (int64_t i = 0; i < a.batch; ++i) {
        const int64_t at = off - i * a.step;
        int64_t first = 0, last = b.batch - 1;
        if (b.batch > 1) {
            const int64_t f = first_between(-b.span(), at, b.step), l = last_between(a.span(), at, b.step);
            if (f > first) first = f;
            if (l < last) last = l;
        }
        for (int64_t k = first; k <= last; ++k)
            if (matrices_share(a, b, at + k * b.step, left)) return true;
    }
    return false;
}

// Whether matrices of one batch have a byte in common (their rows do not).
inline bool batch_overlaps(const Place &a)
{
    int64_t left = MOST_COMPARISONS;
    for (int64_t n = 1; n < a.batch && n * a.step < a.span(); ++n)
        if (matrices_share(a, a, n * a.step, left)) return true;
    return false;
}

}  // namespace netmax

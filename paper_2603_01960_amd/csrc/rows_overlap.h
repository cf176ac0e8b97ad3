// Whether two strided sets of rows share memory: for the checks of outputs against what a kernel still reads.
#pragma once
#include <cstdint>

namespace tsdpa {

// Rows of `bytes` adjacent bytes each, the first at `at`, in up to three dimensions (strides in bytes, not negative).  Contiguous
// memory is one row.
struct RowSet {
    struct Dim { int64_t stride, size; };
    int64_t at, bytes;
    int dims = 0;
    Dim dim[3] = {};

    bool empty() const
    {
        for (int i = 0; i < dims; ++i)
            if (dim[i].size <= 0) return true;
        return bytes <= 0;
    }
    int64_t end() const              // one past the last byte
    {
        int64_t last = at + bytes;
        for (int i = 0; i < dims; ++i) last += dim[i].stride * (dim[i].size - 1);
        return last;
    }
};

// Two rows share a byte iff the distance from one's start to the other's is less than a row.  The distances between all pairs are a
// base plus multiples of the strides, each within a range of its own: searched from the greatest stride down, only where
// the smaller ones can still reach.  Views of one tensor that interleave (the heads of Q and of K in a projection's output, which have
// the same strides) take a few tries.  Strides that have little to do with each other could take many; past `kTries` the sets count
// as apart: what is found is certain, not everything is found.
class RowsOverlap {
    static constexpr int kTries = 2000;
    struct Range { int64_t stride, lo, hi; } range[6];
    int64_t below[7], above[7];      // what the ranges from i on can add, least and most
    int n = 0, tries = 0;
    int64_t first, last;             // distances that are an overlap

    void add(int64_t stride, int64_t lo, int64_t hi)
    {
        if (stride == 0 || lo == hi) return;
        int i = 0;
        while (i < n && range[i].stride > stride) ++i;
        if (i < n && range[i].stride == stride) {
            range[i].lo += lo;
            range[i].hi += hi;
            return;
        }
        for (int j = n++; j > i; --j) range[j] = range[j - 1];
        range[i] = Range{stride, lo, hi};
    }
    static int64_t floor_div(int64_t a, int64_t b) { return a >= 0 ? a / b : -((-a + b - 1) / b); }
    bool reach(int i, int64_t distance)
    {
        if (i == n) return distance >= first && distance <= last;
        const Range &r = range[i];
        // distance + x * stride + [below, above] meets [first, last]
        int64_t lo = -floor_div(-(first - distance - above[i + 1]), r.stride), hi = floor_div(last - distance - below[i + 1], r.stride);
        if (lo < r.lo) lo = r.lo;
        if (hi > r.hi) hi = r.hi;
        for (int64_t x = lo; x <= hi; ++x) {
            if (++tries > kTries) return false;
            if (reach(i + 1, distance + x * r.stride)) return true;
        }
        return false;
    }

public:
    bool operator()(const RowSet &a, const RowSet &b)
    {
        if (a.empty() || b.empty() || a.at >= b.end() || b.at >= a.end()) return false;
        for (int i = 0; i < a.dims; ++i) add(a.dim[i].stride, 0, a.dim[i].size - 1);
        for (int i = 0; i < b.dims; ++i) add(b.dim[i].stride, 1 - b.dim[i].size, 0);
        below[n] = above[n] = 0;
        for (int i = n - 1; i >= 0; --i) {
            below[i] = below[i + 1] + range[i].stride * range[i].lo;
            above[i] = above[i + 1] + range[i].stride * range[i].hi;
        }
        first = 1 - a.bytes;
        last = b.bytes - 1;
        return reach(0, a.at - b.at);
    }
};

}  // namespace tsdpa

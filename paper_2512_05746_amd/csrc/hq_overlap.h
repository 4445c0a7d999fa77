// Whether two tensors share memory: host arithmetic for the checks of a caller's result buffers.
#pragma once
#include <stdint.h>

#include <algorithm>

namespace hq {

// n[0] x n[1] rows of neighbouring bytes, stride[.] >= 0 bytes apart.
struct Rows2 {
    int64_t at, n[2], stride[2], bytes;
    bool empty() const { return n[0] <= 0 || n[1] <= 0 || bytes <= 0; }
    int64_t end() const { return at + (n[0] - 1) * stride[0] + (n[1] - 1) * stride[1] + bytes; }
};

// The same bytes in the same order.
inline bool same_rows(const Rows2 &a, const Rows2 &b) {
    const auto axis = [&](int i) { return a.n[i] == b.n[i] && (a.n[i] < 2 || a.stride[i] == b.stride[i]); };
    return a.at == b.at && a.bytes == b.bytes && axis(0) && axis(1);
}

// na rows of `ba` bytes, sa apart, and nb of `bb` bytes, sb apart, that begin `off` bytes further on: rows i and j share
// a byte where -bb < off + j sb - i sa < ba.
inline bool lines_overlap(int64_t off, int64_t na, int64_t sa, int64_t ba, int64_t nb, int64_t sb, int64_t bb) {
    if (sa == sb || na == 1 || nb == 1) {   // j sb - i sa = u s, u from `first` to `last`
        const int64_t s = na == 1 ? sb : sa, first = 1 - na, last = nb - 1;
        if (s == 0) return -bb < off && off < ba;
        const auto floor_div = [](int64_t x, int64_t y) { return x / y - (x % y < 0 ? 1 : 0); };
        return std::max(first, floor_div(-bb - off, s) + 1) <= std::min(last, -floor_div(off - ba, s) - 1);
    }
    if (na > nb) return lines_overlap(-off, nb, sb, bb, na, sa, ba);
    for (int64_t i = 0; i < na; ++i)
        if (lines_overlap(off - i * sa, 1, 0, ba, nb, sb, bb)) return true;
    return false;
}

// Exact.  Ranges of memory that lie apart take no search; views of one buffer with the same strides a step for each index of the
// second axis (heads), with other strides along it one for each pair of them.
inline bool rows_overlap(const Rows2 &a, const Rows2 &b) {
    if (a.empty() || b.empty() || a.end() <= b.at || b.end() <= a.at) return false;
    const auto at = [&](int64_t off) { return lines_overlap(off, a.n[0], a.stride[0], a.bytes, b.n[0], b.stride[0], b.bytes); };
    const int64_t off = b.at - a.at;
    if (a.stride[1] == b.stride[1]) {
        for (int64_t v = 1 - a.n[1]; v < b.n[1]; ++v)
            if (at(off + v * a.stride[1])) return true;
        return false;
    }
    for (int64_t i = 0; i < a.n[1]; ++i)
        for (int64_t j = 0; j < b.n[1]; ++j)
            if (at(off + j * b.stride[1] - i * a.stride[1])) return true;
    return false;
}

}  // namespace hq

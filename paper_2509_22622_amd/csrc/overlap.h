// Whether two tensors of a call share memory (plain C++, checked on the host by tests/check_overlap.cpp).
#pragma once

#include <cstdint>
#include <utility>

namespace ll_api {

// `rows` rows of `row` bytes, `stride` bytes apart, from `at` on; null or without rows: nothing.
struct Extent { const void* at; int64_t rows, stride, row; };
inline Extent extent(const void* at, int64_t bytes) { return Extent{at, 1, bytes, bytes}; }
// Exact where either is without gaps or both have one stride; of others the first row of the one that begins later is looked at.
inline bool overlap(Extent a, Extent b) {
    if (!a.at || !b.at || a.rows <= 0 || b.rows <= 0 || a.row <= 0 || b.row <= 0) return false;
    for (Extent* x : {&a, &b})
        if (x->stride == x->row) *x = extent(x->at, x->rows * x->row);
    if (reinterpret_cast<uintptr_t>(b.at) < reinterpret_cast<uintptr_t>(a.at)) std::swap(a, b);
    const uint64_t off = reinterpret_cast<uintptr_t>(b.at) - reinterpret_cast<uintptr_t>(a.at);
    if (off >= uint64_t((a.rows - 1) * a.stride + a.row)) return false;
    if (a.rows == 1) return true;
    const uint64_t in = off % uint64_t(a.stride);
    return in < uint64_t(a.row) || in + uint64_t(b.row) > uint64_t(a.stride);       // in a row of a, or from the gap behind it into the next one
}
// Whether one of the first `written` of n shares memory with another.
inline bool any_overlap(const Extent* x, int n, int written) {
    for (int i = 0; i < written; ++i)
        for (int j = i + 1; j < n; ++j)
            if (overlap(x[i], x[j])) return true;
    return false;
}

}  // namespace ll_api

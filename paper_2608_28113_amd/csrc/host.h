// Argument checks and sizes shared by the entry points; nothing of HIP.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace {

inline bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline bool overlaps(const void *a, size_t na, const void *b, size_t nb) {
    if (na == 0 || nb == 0) return false;
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    return a0 < b0 + nb && b0 < a0 + na;
}

struct Range {
    const void *p;
    size_t n;
};

// Whether one of the written ranges meets a read one or another written one.
inline bool any_overlap(const Range *w, int nw, const Range *r, int nr) {
    for (int i = 0; i < nw; ++i) {
        for (int j = 0; j < i; ++j)
            if (overlaps(w[i].p, w[i].n, w[j].p, w[j].n)) return true;
        for (int j = 0; j < nr; ++j)
            if (overlaps(w[i].p, w[i].n, r[j].p, r[j].n)) return true;
    }
    return false;
}

// Bytes spanned by `rows` rows of `width` elements at a row stride of `ld`
// elements of `elem` bytes each.
inline size_t span(int64_t rows, int64_t ld, int64_t width, size_t elem) {
    if (rows <= 0 || width <= 0) return 0;
    return ((size_t)(rows - 1) * (size_t)ld + (size_t)width) * elem;
}

inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

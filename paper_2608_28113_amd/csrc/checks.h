// Argument checks of the entry points of the stored layer in use.
#pragma once

#include "common.h"

namespace {

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

}  // namespace

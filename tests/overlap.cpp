// The check for views that share memory (csrc/overlap.h), for the host.
#include "overlap.h"

extern "C" int overlap_(const int64_t *a, const int64_t *b) {  // each: address, element, number of dimensions, (stride, size) ...
    mate_binding::Extent x[2];
    for (int i = 0; i < 2; ++i) {
        const int64_t *e = i ? b : a;
        x[i].address = e[0], x[i].element = e[1];
        for (int64_t d = 0; d < e[2]; ++d) x[i].dims.emplace_back(e[3 + 2 * d], e[4 + 2 * d]);
    }
    return mate_binding::overlap(x[0], x[1]);
}

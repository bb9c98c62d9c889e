// The index arithmetic of the calls on a paged cache (csrc/mate_cache.h), for the host.
#include "mate_cache.h"

extern "C" {
int in_range_(int x, int n) { return mate::in_range(x, n); }
int pages_of_(int len, int page_size) { return mate::pages_of(len, page_size); }
int clip_len_(int len, int most, int *bad) {
    bool b = false;
    const int r = mate::clip_len(len, most, &b);
    *bad = b;
    return r;
}
int owner_of_(const int *off, int n, int r) { return mate::owner_of(off, n, r); }
int owner_of_64(const int64_t *off, int n, int r) { return mate::owner_of(off, n, r); }
}

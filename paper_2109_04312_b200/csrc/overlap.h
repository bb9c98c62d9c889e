// Whether two strided views share memory (host; no torch, so that it can be tested alone).
#pragma once
#include <algorithm>
#include <cstdint>
#include <utility>
#include <vector>

namespace mate_binding {

struct Extent {
    int64_t address;                                // of the first element, in bytes
    int64_t element;                                // bytes
    std::vector<std::pair<int64_t, int64_t>> dims;  // stride in bytes (>= 0), size
};

// Elements at a + sum s_i x_i and b + sum t_j y_j share a byte if the difference lies between -(a's element) and b's, exclusive.  The strides
// are taken from the largest to the smallest (equal ones together, as one number between -(n_b - 1) and n_a - 1), and only
// numbers from which the smaller strides can still reach that range are tried: two or three for each stride of ordinary layouts.
// Layouts that need more than kTries are taken to overlap.
inline bool overlap(const Extent &a, const Extent &b) {
    struct Term {
        int64_t stride, lo, hi;
    };
    std::vector<Term> terms;
    for (int side = 0; side < 2; ++side)
        for (const auto &[stride, size] : (side ? b : a).dims) {
            if (size == 0) return false;
            if (size > 1 && stride > 0) terms.push_back({stride, side ? 1 - size : 0, side ? 0 : size - 1});
        }
    std::sort(terms.begin(), terms.end(), [](const Term &x, const Term &y) { return x.stride > y.stride; });
    size_t n = 0;
    for (const Term &t : terms) {
        if (n && terms[n - 1].stride == t.stride)
            terms[n - 1].lo += t.lo, terms[n - 1].hi += t.hi;
        else
            terms[n++] = t;
    }
    terms.resize(n);
    std::vector<int64_t> least(n + 1, 0), most(n + 1, 0);  // what the terms from i on can add
    for (size_t i = n; i-- > 0;) {
        least[i] = least[i + 1] + terms[i].stride * terms[i].lo;
        most[i] = most[i + 1] + terms[i].stride * terms[i].hi;
    }
    const auto floor_div = [](int64_t x, int64_t y) { return x / y - (x % y != 0 && x < 0); };
    constexpr int kTries = 20000;
    int tries = 0;
    // whether the terms from i on can add up to something between lo and hi
    const auto reaches = [&](const auto &self, size_t i, int64_t lo, int64_t hi) -> bool {
        if (hi < least[i] || lo > most[i]) return false;
        if (i == n) return true;
        if (++tries > kTries) return true;
        const int64_t first = std::max(terms[i].lo, -floor_div(most[i + 1] - lo, terms[i].stride));
        const int64_t last = std::min(terms[i].hi, floor_div(hi - least[i + 1], terms[i].stride));
        for (int64_t x = first; x <= last; ++x)
            if (self(self, i + 1, lo - terms[i].stride * x, hi - terms[i].stride * x)) return true;
        return false;
    };
    const int64_t apart = b.address - a.address;
    return reaches(reaches, 0, apart - a.element + 1, apart + b.element - 1);
}

}  // namespace mate_binding

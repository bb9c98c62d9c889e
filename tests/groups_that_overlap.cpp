// Which entries of a batch are in the groups that they claim (csrc/mate_cache.h), for the host.
#include "mate_cache.h"

extern "C" {
int begins_inside_(const uint32_t *begins, int first, int count) { return mate::begins_inside(begins, first, count); }
// begins: a bit for each entry; member[b]: whether entry b is in its group
void members_(const int32_t *groups, int B, int max_len, uint32_t *begins, int32_t *member) {
    for (int b = 0; b < B; ++b)
        if (mate::begins_group(mate::claim_of(groups, B, b), b, B, max_len)) begins[b / 32] |= 1u << b % 32;
    for (int b = 0; b < B; ++b) {
        const mate::Claim c = mate::claim_of(groups, B, b);
        const int f = c.first < 0 ? 0 : c.first < b ? c.first : b;
        member[b] = mate::is_member(c, b, mate::claim_of(groups, B, f), begins, B, max_len);
    }
}
}

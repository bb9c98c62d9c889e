// What the calls on a paged cache share (not part of the C ABI): argument checks, look-ups, index arithmetic.
#pragma once
#include "mate_internal.h"

namespace mate {

enum { kCacheBad = 1, kCacheFull = 2, kCacheTimeout = 4 };  // bits of mate_cache_t.status

inline size_t elem_size(int dtype) { return dtype == MATE_F32 ? 4 : 2; }
inline bool is_aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// The cache as kernels get it.
struct CacheArgs {
    void *k, *v;  // of one layer, where a call is about one
    int32_t *row_ids, *col_ids, *table, *lens, *prefix, *refs, *status;
    int64_t page_stride, head_stride, slot_stride;
    int32_t pages, page_size, seqs, width;
};
inline CacheArgs cache_args(const mate_cache_t *c, int layer) {
    const size_t at = (size_t)layer * (size_t)c->layer_stride * elem_size(c->dtype);
    return {(char *)c->k + at, (char *)c->v + at, c->row_ids, c->col_ids, c->table, c->lens, c->prefix, c->refs, c->status,
            c->page_stride, c->head_stride, c->slot_stride, c->pages, c->page_size, c->seqs, c->width};
}

// Everything about the struct that can be wrong on the host.
inline int check_cache(const mate_cache_t *c) {
    if (!c || !c->k || !c->v || !c->row_ids || !c->col_ids || !c->table || !c->lens || !c->prefix || !c->refs || !c->status || !c->head_view)
        return MATE_ERR_INVALID_ARG;
    if (c->dtype != MATE_BF16 && c->dtype != MATE_F32) return MATE_ERR_UNSUPPORTED;
    if (c->d <= 0 || c->d % 8 != 0 || c->d > 128) return MATE_ERR_UNSUPPORTED;
    if (c->layers < 1 || c->pages < 1 || c->page_size < 1 || c->seqs < 1 || c->width < 1 || c->heads < 1 || c->kv_heads < 1 ||
        c->heads % c->kv_heads != 0)
        return MATE_ERR_INVALID_ARG;
    // slots, positions and the elements of a page are 32-bit numbers (with room for a block's stride), rows of a page exact in fp32
    constexpr int64_t kMost = 1 << 30;
    if ((int64_t)c->pages * c->page_size > kMost || (int64_t)c->width * c->page_size > kMost ||
        (int64_t)c->kv_heads * c->d > kMost / c->page_size || (int64_t)c->kv_heads * c->page_size > 1 << 20 || c->layers > 32767)
        return MATE_ERR_UNSUPPORTED;
    for (int64_t s : {c->layer_stride, c->page_stride, c->head_stride, c->slot_stride})
        if (s < 0 || s % (int64_t)(16 / elem_size(c->dtype)) != 0) return MATE_ERR_ALIGNMENT;
    if (!is_aligned(c->k, 16) || !is_aligned(c->v, 16)) return MATE_ERR_ALIGNMENT;
    for (int h = 0; h < c->heads; ++h)
        if (c->head_view[h] > MATE_VIEW_EITHER) return MATE_ERR_INVALID_ARG;
    return MATE_OK;
}
// The cache's arrays lie on one device: a call with another one current is refused before anything is launched.
inline int check_cache_device(const mate_cache_t *c) {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return MATE_ERR_CUDA;
    return dev == c->device ? MATE_OK : MATE_ERR_INVALID_ARG;
}
inline int n_sms(int device) {
    int n = 0;
    return cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) == cudaSuccess && n > 0 ? n : 1;
}

// ---- index arithmetic (host and device: the host's side of it is tested without a GPU)

__host__ __device__ inline bool in_range(int x, int n) { return x >= 0 && x < n; }
__host__ __device__ inline int pages_of(int len, int page_size) { return len / page_size + (len % page_size != 0); }
// A sequence's length, clipped to what its row of the table can hold.
__host__ __device__ inline int clip_len(int len, int most, bool *bad) {
    if (len < 0 || len > most) *bad = true;
    return len < 0 ? 0 : len > most ? most : len;
}
// Owner of the r-th of the things that the entries want, off[i] being what those in front of entry i want, off[0] = 0 <= r: the
// last entry with off[i] <= r.
template <typename N>
__host__ __device__ inline int owner_of(const N *off, int n, int r) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (off[mid] <= r)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// What an entry of a batch says of its group (of mate_attn_decode_shared): the first entry of it, how many it has, and the tokens that they share.
struct Claim {
    int first, count, shared;
};
__host__ __device__ inline Claim claim_of(const int32_t *groups, int B, int b) { return {groups[b], groups[B + b], groups[2 * B + b]}; }
// Whether it says that it is in one, and whether that is in range.
__host__ __device__ inline bool claims(const Claim &c) { return c.shared > 0 && c.count > 1; }
__host__ __device__ inline bool fits(const Claim &c, int b, int B, int max_len) {
    return claims(c) && c.first >= 0 && c.first <= b && c.count <= B - c.first && b - c.first < c.count && c.shared <= max_len;
}
__host__ __device__ inline bool begins_group(const Claim &c, int b, int B, int max_len) { return c.first == b && fits(c, b, B, max_len); }
// Whether a group begins among the entries behind the first one of `count`, by a bit for each entry that begins one.  Where none does in any group, no
// two have an entry in common (of two that have, the one that begins later begins inside the other), and all of them together have B entries at most:
// that is what makes their rows, and the places of their results, their own.
__host__ __device__ inline bool begins_inside(const uint32_t *begins, int first, int count) {
    const int from = first + 1, to = first + count;  // to > from
    for (int w = from >> 5; w <= (to - 1) >> 5; ++w) {
        uint32_t those = begins[w];
        if (w == from >> 5) those &= ~0u << (from & 31);
        if (w == (to - 1) >> 5) those &= ~0u >> (31 - ((to - 1) & 31));
        if (those) return true;
    }
    return false;
}
// Whether an entry is in the group that it claims: the group's first entry says the same, and no other group begins inside it.
__host__ __device__ inline bool is_member(const Claim &c, int b, const Claim &of_first, const uint32_t *begins, int B, int max_len) {
    return fits(c, b, B, max_len) && of_first.first == c.first && of_first.count == c.count && of_first.shared == c.shared &&
           !(begins && begins_inside(begins, c.first, c.count));
}
__host__ __device__ inline bool bit_of(const uint32_t *bits, int b) { return bits[b >> 5] >> (b & 31) & 1; }

#ifdef __CUDACC__
// Sequence of entry i of a list (null: i itself), -1 where there is none.
__device__ __forceinline__ int seq_of(const int32_t *seqs, int i, int n_seqs) {
    const int s = seqs ? seqs[i] : i;
    return in_range(s, n_seqs) ? s : -1;
}

// An entry of a batch and its group (of mate_attn_decode_shared).
struct GroupOf {
    int s;  // its sequence; -1: none
    int len, prefix;
    int first, count, shared;  // count 0: it is in none
    bool bad;
};
// What does not fit together on the device leaves an entry without a group: the rows of one group are the same in all of its entries.  none: another
// group is known to begin inside the entry's, which is not looked for here.  (Two rounds of loads, the second one's indexes brought into range
// instead of looked at first.)
__device__ __forceinline__ GroupOf group_of(const CacheArgs &c, const int32_t *seqs, const int32_t *groups, bool none, int B, int b, int max_len) {
    GroupOf e = {};
    const Claim mine = claim_of(groups, B, b);
    const int s = seqs ? seqs[b] : b, at = s < 0 ? 0 : s < c.seqs ? s : c.seqs - 1;
    const int len = c.lens[at], prefix = c.prefix[at];
    const Claim of_first = claim_of(groups, B, mine.first < 0 ? 0 : mine.first < b ? mine.first : b);
    e.s = s == at ? s : -1, e.first = mine.first, e.prefix = prefix < 0 ? 0 : prefix;
    if (s != at || mine.shared < 0) e.bad = true;
    if (s == at) e.len = clip_len(len, max_len, &e.bad);
    if (claims(mine)) {
        if (!none && is_member(mine, b, of_first, nullptr, B, max_len))
            e.count = mine.count, e.shared = mine.shared;
        else
            e.bad = true;
    }
    if (e.count > 0 && e.len < mine.shared) e.bad = true;
    return e;
}
// A bit for each entry that begins a group.  All of a block's NT threads call it, with a barrier behind it.
template <int NT>
__device__ __forceinline__ void find_begins(const int32_t *groups, int B, int max_len, uint32_t *begins) {
#pragma unroll 4
    for (int b0 = threadIdx.x & ~31; b0 < B; b0 += NT) {
        const int b = b0 + (int)(threadIdx.x & 31);
        const unsigned those = __ballot_sync(~0u, b < B && begins_group(claim_of(groups, B, b), b, B, max_len));
        if ((threadIdx.x & 31) == 0) begins[b0 >> 5] = those;
    }
}
#endif

}  // namespace mate

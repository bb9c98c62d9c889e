// Pages of a cache: room for new tokens (mate_cache_extend), sequences that share their pages (mate_cache_fork), pages
// given back (mate_cache_free) and moved together (mate_cache_compact); who shares how many with whom (mate_cache_groups).
//
// What is decided -- who gets which page -- is whole numbers and the same on every launch: one block reads the
// reference counts, each warp a run of consecutive pages, and a scan over the block ranks the free ones; the r-th
// lowest free page goes to the r-th request.  Latency: a few dependent loads and two or three scans.  What is moved
// (rows of keys and values, every layer) is bound by memory and done by a second kernel over all SMs.
//
// A sequence that stands in a list twice: every entry puts its place in the list by atomicMin where the sequence has a word of its
// own, so the first entry wins, whatever the order of the threads: in shared memory, and for more than 4096 sequences in
// their lengths (as INT_MIN + place), which costs two more round trips to L2.
#include "mate_cache.h"
#include "sm100_ptx.cuh"

namespace mate {
namespace {

constexpr int kThreads = 1024;   // of the deciding block
constexpr int kPer = 4;          // entries of a list per thread: lists of up to 4096
constexpr int kMost = kThreads * kPer;
constexpr int kEarly = 16384;    // pages up to which the reference counts are read before it is known whether any is wanted
constexpr int kCopyThreads = 128, kCopyBlocks = 8;  // blocks per SM

// Exclusive sum over the block's threads; *total gets the sum.  All threads call it.
template <typename N>
__device__ N block_scan(N x, N *total) {
    __shared__ N s_warp[kThreads / 32 + 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    N sum = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const N y = __shfl_up_sync(~0u, sum, o);
        if (lane >= o) sum += y;
    }
    __syncthreads();  // an earlier scan has been read
    if (lane == 31) s_warp[warp] = sum;
    __syncthreads();
    if (warp == 0) {
        const N w = s_warp[lane];
        N t = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const N y = __shfl_up_sync(~0u, t, o);
            if (lane >= o) t += y;
        }
        s_warp[lane] = t - w;
        if (lane == 31) s_warp[32] = t;
    }
    __syncthreads();
    *total = s_warp[32];
    return s_warp[warp] + sum - x;
}

// The warp's run of pages, and what can be done with those that are free.
struct PageRun {
    int lo, hi;
    __device__ explicit PageRun(int pages) {
        const int per = ((pages + kThreads - 1) / kThreads) * 32;
        lo = min(pages, (int)(threadIdx.x >> 5) * per), hi = min(pages, lo + per);
    }
    // pages for which f holds, of the lane's
    template <typename F>
    __device__ int count(F &&f) const {
        int n = 0;
#pragma unroll 8
        for (int p = lo + (threadIdx.x & 31); p < hi; p += 32) n += f(p);
        return n;
    }
    // g(page, rank) for the pages for which f holds, in order, ranks from `rank` to below `limit`
    template <typename F, typename G>
    __device__ void each(int rank, int limit, F &&f, G &&g) const {
        const int lane = threadIdx.x & 31;
        for (int p0 = lo; p0 < hi && rank < limit; p0 += 32) {
            const bool is = p0 + lane < hi && f(p0 + lane);
            const unsigned all = __ballot_sync(~0u, is);
            const int mine = rank + __popc(all & ((1u << lane) - 1));
            if (is && mine < limit) g(p0 + lane, mine);
            rank += __popc(all);
        }
    }
};
// Rank of the warp's first among all that were counted (by lanes); *total: how many there are.
__device__ __forceinline__ int warp_rank(int of_lane, int *total) {
    const int of_warp = __reduce_add_sync(~0u, of_lane);
    return __shfl_sync(~0u, block_scan((threadIdx.x & 31) == 0 ? of_warp : 0, total), 0);
}

// Who of the entries with one sequence comes first: put() by all, a barrier, first().  `s_claim`: kMost words of shared memory, cleared by
// clear() and a barrier.
struct Claims {
    int *s_claim;
    const CacheArgs &c;
    __device__ bool shared() const { return c.seqs <= kMost; }
    __device__ void clear() const {
        if (shared())
            for (int i = threadIdx.x; i < c.seqs; i += kThreads) s_claim[i] = INT32_MAX;
    }
    __device__ void put(int seq, int i) const {
        if (shared())
            atomicMin(s_claim + seq, i);
        else
            atomicMin(c.lens + seq, INT32_MIN + i);
    }
    __device__ bool first(int seq, int i) const { return shared() ? s_claim[seq] == i : __ldcg(c.lens + seq) == INT32_MIN + i; }
};

constexpr int kExtendSmem = kMost * (int)(sizeof(int64_t) + 2 * sizeof(int));
__global__ void __launch_bounds__(kThreads, 1) extend_kernel(const __grid_constant__ CacheArgs c, const int32_t *seqs, const int32_t *counts, int n,
                                                             int32_t *granted) {
    extern __shared__ int64_t s_at[];                     // [kMost] where in the table an entry's first new page goes
    int *s_off = reinterpret_cast<int *>(s_at + kMost);   // [kMost] pages that the entries in front of it want
    const Claims claims = {s_off + kMost, c};
    __shared__ int s_used;
    ptx::launch_dependents();
    ptx::wait_prior_grid();
    const int tid = threadIdx.x, i0 = tid * kPer;
    const PageRun run(c.pages);
    const auto is_free = [&](int page) { return c.refs[page] <= 0; };
    const bool early = c.pages <= kEarly;
    int free_here = early ? run.count(is_free) : 0;
    int s[kPer], len[kPer], count[kPer], need[kPer], refused[kPer], status = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        s[j] = -1, need[j] = 0, len[j] = 0, count[j] = 0, refused[j] = 0;
        if (i0 + j >= n) continue;
        s[j] = seq_of(seqs, i0 + j, c.seqs);
        count[j] = counts[i0 + j];
        if (s[j] >= 0) len[j] = c.lens[s[j]];
        const int most = c.width * c.page_size;
        if (s[j] < 0 || count[j] < 0 || len[j] < 0 || len[j] > most)
            refused[j] = kCacheBad;
        else if (count[j] > most - len[j])
            refused[j] = kCacheFull;
        status |= refused[j];
    }
    if (tid == 0) s_used = 0;
    claims.clear();
    __syncthreads();  // every length has been read
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (s[j] >= 0) claims.put(s[j], i0 + j);  // (a refused entry too: it is its sequence's first all the same)
    __syncthreads();
    int64_t sum = 0;  // (the list may want more pages than 32 bits count)
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        if (s[j] >= 0 && !claims.first(s[j], i0 + j)) {
            status |= kCacheBad;  // the second entry of a sequence
            s[j] = -1;
        }
        if (s[j] >= 0 && !refused[j]) need[j] = pages_of(len[j] + count[j], c.page_size) - pages_of(len[j], c.page_size);
        sum += need[j];
    }
    int64_t wanted;
    int64_t off = block_scan(sum, &wanted);
    int n_free = 0, rank = 0;
    if (wanted > 0) {
        if (!early) free_here = run.count(is_free);
        rank = warp_rank(free_here, &n_free);
    }
    // granted: who fits into what is free; the pages that go out are the first `used` free ones
    int used = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int64_t end = off + need[j];
        const bool fits = s[j] >= 0 && !refused[j] && (need[j] == 0 || end <= n_free);
        if (s[j] >= 0 && !refused[j] && !fits) status |= kCacheFull;
        if (fits && need[j] > 0) used = max(used, (int)end);
        if (s[j] >= 0) c.lens[s[j]] = fits ? len[j] + count[j] : len[j];
        if (i0 + j < n) granted[i0 + j] = fits ? count[j] : 0;
        s_off[i0 + j] = (int)min(off, (int64_t)INT32_MAX);
        s_at[i0 + j] = (int64_t)s[j] * c.width + pages_of(len[j], c.page_size);
        off = end;
    }
    if (status) atomicOr(c.status, status);
    if (wanted == 0) return;
    if (used > 0) atomicMax(&s_used, used);
    __syncthreads();
    run.each(rank, s_used, is_free, [&](int page, int r) {
        const int i = owner_of(s_off, min(n, kMost), r);
        c.table[s_at[i] + (r - s_off[i])] = page;
        c.refs[page] = 1;
    });
}

// What mate_cache_fork leaves for its copies, per entry of the list.
struct ForkItem {
    int32_t parent, child;  // child -1: nothing to do
    int32_t full, fill;     // shared pages; filled slots of the page behind them
    int32_t src, dst;       // that page, and the one it is copied to (-1: none)
};

__global__ void __launch_bounds__(kThreads, 1) fork_kernel(const __grid_constant__ CacheArgs c, const int32_t *parents, const int32_t *children,
                                                           int n, ForkItem *items) {
    __shared__ int s_off[kMost], s_dst[kMost];  // (s_dst: the claims at first)
    const Claims claims = {s_dst, c};
    ptx::launch_dependents();
    ptx::wait_prior_grid();
    const int tid = threadIdx.x, i0 = tid * kPer;
    const PageRun run(c.pages);
    const auto is_free = [&](int page) { return c.refs[page] <= 0; };
    const bool early = c.pages <= kEarly;
    int free_here = early ? run.count(is_free) : 0;
    int p[kPer], ch[kPer], len[kPer], child_len[kPer], prefix[kPer], src[kPer], status = 0, sum = 0;
    bool refused[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        p[j] = ch[j] = src[j] = -1, len[j] = child_len[j] = prefix[j] = 0, refused[j] = false;
        if (i0 + j >= n) continue;
        p[j] = seq_of(parents, i0 + j, c.seqs);
        ch[j] = seq_of(children, i0 + j, c.seqs);
        if (p[j] >= 0) len[j] = c.lens[p[j]], prefix[j] = c.prefix[p[j]];
        if (ch[j] >= 0) child_len[j] = c.lens[ch[j]];
        if (p[j] < 0 || ch[j] < 0 || len[j] < 0 || len[j] > c.width * c.page_size || child_len[j] != 0) {
            status |= kCacheBad;
            refused[j] = true;
        } else if (len[j] % c.page_size != 0) {
            src[j] = c.table[(size_t)p[j] * c.width + len[j] / c.page_size];
        }
    }
    claims.clear();
    __syncthreads();  // every length and prefix has been read
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (ch[j] >= 0) claims.put(ch[j], i0 + j);  // (a refused entry too: it is its child's first all the same)
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        if (ch[j] >= 0 && !claims.first(ch[j], i0 + j)) {
            status |= kCacheBad;  // the second entry of a child
            ch[j] = -1;
        }
        sum += ch[j] >= 0 && !refused[j] && len[j] % c.page_size != 0;
    }
    int wanted;
    int off = block_scan(sum, &wanted);  // (its barriers: the claims have been read)
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        if (ch[j] >= 0 && refused[j]) {
            c.lens[ch[j]] = child_len[j];  // (where the claim was put)
            ch[j] = -1;
        }
        s_off[i0 + j] = off;
        s_dst[i0 + j] = -1;
        off += ch[j] >= 0 && len[j] % c.page_size != 0;
    }
    __syncthreads();
    if (wanted > 0) {
        if (!early) free_here = run.count(is_free);
        int n_free;
        const int rank = warp_rank(free_here, &n_free);
        run.each(rank, wanted, is_free, [&](int page, int r) {
            s_dst[owner_of(s_off, min(n, kMost), r)] = page;
            c.refs[page] = 1;
        });
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        if (i0 + j >= n) continue;
        ForkItem it = {p[j], ch[j], 0, 0, -1, -1};
        if (ch[j] >= 0) {
            it.full = len[j] / c.page_size;
            it.fill = len[j] - it.full * c.page_size;
            if (it.fill > 0) {
                it.src = src[j];
                it.dst = s_dst[i0 + j];
                if (it.dst < 0) status |= kCacheFull;
            }
            const bool done = it.fill == 0 || it.dst >= 0;
            c.lens[ch[j]] = done ? len[j] : 0;
            if (done) c.prefix[ch[j]] = prefix[j];
            if (!done) it.child = -1;
            if (done && it.dst >= 0 && !in_range(it.src, c.pages)) {
                status |= kCacheBad;  // nothing to copy from
                it.src = -1;
            }
        }
        items[i0 + j] = it;
    }
    if (status) atomicOr(c.status, status);
}

// How the rows of a page lie.
struct PageShape {
    int64_t page_stride, head_stride, slot_stride, layer_stride;  // bytes
    int heads, per_row, layers, page_size;                        // per_row: units of 16 bytes
    unsigned row_mul;                                             // u / per_row = umulhi(u, row_mul) for u < 2^27; 0: per_row is 1
    int piece, pieces;                                            // units of a piece, pieces of a page
};
// Copies a piece of one page of one layer's keys or values, of whose slots the first `fill` count.  Units of 16 bytes, kFlight of a
// thread under way; slots by way of fp32 (exact: rows are fewer than 2^21, the host sees to that).  Bound by memory as long as
// the arithmetic of a unit is short: quotients by the instruction took the copies of a compaction (230 MB) from 36.3 to 39.8 us.
__device__ __forceinline__ void copy_piece(const PageShape &sh, char *base, int src, int dst, int fill, int piece) {
    const char *from = base + src * sh.page_stride;
    char *to = base + dst * sh.page_stride;
    const int n = min(sh.heads * fill * sh.per_row, (piece + 1) * sh.piece);
    const float by_fill = 1.f / (float)fill;
    constexpr int kFlight = 4;
    for (int i = piece * sh.piece + threadIdx.x; i < n; i += kCopyThreads * kFlight) {
        uint4 v[kFlight];
        int64_t at[kFlight];
#pragma unroll
        for (int j = 0; j < kFlight; ++j) {
            const int u = i + j * kCopyThreads;
            if (u >= n) break;
            const int row = sh.row_mul ? (int)__umulhi((unsigned)u, sh.row_mul) : u, head = (int)(((float)row + 0.5f) * by_fill);
            at[j] = head * sh.head_stride + (row - head * fill) * sh.slot_stride + (u - row * sh.per_row) * 16;
            v[j] = *reinterpret_cast<const uint4 *>(from + at[j]);
        }
#pragma unroll
        for (int j = 0; j < kFlight; ++j)
            if (i + j * kCopyThreads < n) *reinterpret_cast<uint4 *>(to + at[j]) = v[j];
    }
}
__device__ __forceinline__ void copy_ids(const CacheArgs &c, int src, int dst, int fill, int tid, int threads) {
    for (int i = tid; i < fill; i += threads) {
        c.row_ids[(size_t)dst * c.page_size + i] = c.row_ids[(size_t)src * c.page_size + i];
        c.col_ids[(size_t)dst * c.page_size + i] = c.col_ids[(size_t)src * c.page_size + i];
    }
}

// grid: (entry, layer and keys / values, piece of the page); one more layer's block for the table and the ids
__global__ void __launch_bounds__(kCopyThreads, kCopyBlocks) fork_copy_kernel(const __grid_constant__ CacheArgs c, const __grid_constant__ PageShape sh,
                                                                 const ForkItem *items) {
    ptx::launch_dependents();
    ptx::wait_prior_grid();
    const ForkItem it = items[blockIdx.x];
    if (it.child < 0) return;
    const int part = blockIdx.y;
    if (part < 2 * sh.layers) {
        if (it.src < 0 || it.dst < 0) return;
        copy_piece(sh, (char *)(part & 1 ? c.v : c.k) + (part >> 1) * sh.layer_stride, it.src, it.dst, it.fill, blockIdx.z);
        return;
    }
    if (blockIdx.z > 0) return;
    if (it.src >= 0 && it.dst >= 0) copy_ids(c, it.src, it.dst, it.fill, threadIdx.x, kCopyThreads);
    const int32_t *from = c.table + (size_t)it.parent * c.width;
    int32_t *to = c.table + (size_t)it.child * c.width;
    bool bad = false;
    for (int i = threadIdx.x; i < it.full; i += kCopyThreads) {
        const int page = from[i];
        to[i] = page;
        if (in_range(page, c.pages))
            atomicAdd(&c.refs[page], 1);
        else
            bad = true;
    }
    if (threadIdx.x == 0 && it.dst >= 0) to[it.full] = it.dst;
    if (bad) atomicOr(c.status, kCacheBad);
}

__global__ void __launch_bounds__(kCopyThreads) free_kernel(const __grid_constant__ CacheArgs c, const int32_t *seqs) {
    __shared__ int s_len;
    ptx::launch_dependents();
    ptx::wait_prior_grid();
    const int s = seq_of(seqs, blockIdx.x, c.seqs);
    if (s < 0) {
        if (threadIdx.x == 0) atomicOr(c.status, kCacheBad);
        return;
    }
    if (threadIdx.x == 0) s_len = atomicExch(&c.lens[s], 0);  // (of two entries with one sequence one gets its length)
    __syncthreads();
    const int len = s_len;
    bool bad = false;
    const int n = pages_of(clip_len(len, c.width * c.page_size, &bad), c.page_size);
    if (len != 0)
        for (int i = threadIdx.x; i < c.width; i += kCopyThreads) {
            int32_t *at = c.table + (size_t)s * c.width + i;
            if (i < n) {
                const int page = *at;
                if (!in_range(page, c.pages)) {
                    bad = true;
                } else if (atomicSub(&c.refs[page], 1) <= 0) {
                    atomicAdd(&c.refs[page], 1);  // it was free already
                    bad = true;
                }
            }
            *at = -1;
        }
    if (bad) atomicOr(c.status, kCacheBad);
}

// What mate_cache_compact leaves for its copies: the number of moves; from / to of each; the new place of every page
// (-1: it has none).
struct Moves {
    int32_t *n, *from, *to, *place;
};
__global__ void __launch_bounds__(kThreads, 1) compact_kernel(const __grid_constant__ CacheArgs c, Moves m, int32_t *n_live_out) {
    ptx::launch_dependents();
    ptx::wait_prior_grid();
    const PageRun run(c.pages);
    int n_live, n_moves, n_holes;  // (as many holes as moves)
    warp_rank(run.count([&](int p) { return c.refs[p] > 0; }), &n_live);
    const auto is_hole = [&](int p) { return p < n_live && c.refs[p] <= 0; };
    const auto is_mover = [&](int p) { return p >= n_live && c.refs[p] > 0; };
    const int hole = warp_rank(run.count(is_hole), &n_holes), mover = warp_rank(run.count(is_mover), &n_moves);
    for (int p = run.lo + (threadIdx.x & 31); p < run.hi; p += 32) m.place[p] = p < n_live && c.refs[p] > 0 ? p : -1;
    run.each(hole, n_holes, is_hole, [&](int page, int r) { m.to[r] = page; });
    run.each(mover, n_moves, is_mover, [&](int page, int r) { m.from[r] = page; });
    __syncthreads();
    for (int i = threadIdx.x; i < n_moves; i += kThreads) {
        const int from = __ldcg(&m.from[i]), to = __ldcg(&m.to[i]);
        m.place[from] = to;
        c.refs[to] = c.refs[from];
        c.refs[from] = 0;
    }
    if (threadIdx.x == 0) {
        m.n[0] = n_moves;
        *n_live_out = n_live;
    }
}

// Blocks take the tasks in turn, and then the table's rows.
__global__ void __launch_bounds__(kCopyThreads, kCopyBlocks) compact_copy_kernel(const __grid_constant__ CacheArgs c, const __grid_constant__ PageShape sh,
                                                                    Moves m) {
    ptx::launch_dependents();
    ptx::wait_prior_grid();
    // tasks: the pieces of a move's layers' keys and values, and its ids
    const int n_moves = m.n[0], pieces = sh.pieces;
    const int64_t tasks = (int64_t)2 * sh.layers * pieces + 1;
    for (int64_t w = blockIdx.x; w < n_moves * tasks; w += gridDim.x) {
        const int i = (int)(w / tasks), src = m.from[i], dst = m.to[i];
        const int64_t task = w - i * tasks;
        if (task < tasks - 1) {
            const int part = (int)(task / pieces);
            copy_piece(sh, (char *)(part & 1 ? c.v : c.k) + (part >> 1) * sh.layer_stride, src, dst, c.page_size, (int)(task - (int64_t)part * pieces));
        } else {
            copy_ids(c, src, dst, c.page_size, threadIdx.x, kCopyThreads);
        }
    }
    bool bad = false;
    for (int q = blockIdx.x; q < c.seqs; q += gridDim.x) {
        const int n = pages_of(clip_len(c.lens[q], c.width * c.page_size, &bad), c.page_size);
        for (int i = threadIdx.x; i < n; i += kCopyThreads) {
            int32_t *at = c.table + (size_t)q * c.width + i;
            const int page = *at, place = in_range(page, c.pages) ? m.place[page] : -1;
            if (place < 0)
                bad = true;  // no page, or one that nothing counts
            else if (place != page)
                *at = place;
        }
    }
    if (bad) atomicOr(c.status, kCacheBad);
}

// Sequence of entry i, and its full pages; none where there is no such sequence.
__device__ __forceinline__ int full_pages(const CacheArgs &c, const int32_t *seqs, int i, int *s, bool *bad) {
    *s = seq_of(seqs, i, c.seqs);
    if (*s < 0) *bad = true;
    return *s < 0 ? 0 : clip_len(c.lens[*s], c.width * c.page_size, bad) / c.page_size;
}
// Leading full pages that every entry has in common with the one before it.  A block each, kRun pairs of a thread under way: latency,
// as long as a row fits one round of them (2048 pages): with groups_kernel 3.7 us for 64 entries of 512 pages, 4.2 of 2048, 7.5 of 8192.  (Both in one
// cluster of eight blocks: 5.3, 10.5, 30.)
constexpr int kCommonThreads = 128, kRun = 16;
__global__ void __launch_bounds__(kCommonThreads) common_kernel(const __grid_constant__ CacheArgs c, const int32_t *seqs, int32_t *common) {
    __shared__ int s_first;
    ptx::launch_dependents();
    ptx::wait_prior_grid();
    const int i = blockIdx.x, tid = threadIdx.x;
    int s, t = -1;
    bool bad = false, unused = false;
    const int mine = full_pages(c, seqs, i, &s, &bad), n = i > 0 ? min(mine, full_pages(c, seqs, i - 1, &t, &unused)) : 0;
    if (bad && tid == 0) atomicOr(c.status, kCacheBad);
    if (tid == 0) s_first = n;  // the first page that they have not in common
    __syncthreads();
    const int32_t *a = c.table + (size_t)max(s, 0) * c.width, *b = c.table + (size_t)max(t, 0) * c.width;
    for (int p0 = 0; p0 < n; p0 += kCommonThreads * kRun) {
        int x[kRun], y[kRun];
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            const int p = p0 + j * kCommonThreads + tid;
            x[j] = p < n ? a[p] : 0, y[j] = p < n ? b[p] : 0;
        }
        int first = n;
#pragma unroll
        for (int j = kRun - 1; j >= 0; --j) {
            const int p = p0 + j * kCommonThreads + tid;
            if (p < n && (x[j] != y[j] || !in_range(x[j], c.pages))) first = p;
        }
        if (first < n) atomicMin(&s_first, first);
        __syncthreads();
        if (s_first < p0 + kCommonThreads * kRun) break;
        __syncthreads();
    }
    if (tid == 0) common[i] = s_first;
}
// An entry begins a group where it has fewer than `least` pages in common with the one before it.  One block; groups[2 n + i] holds what
// common_kernel found.
__global__ void __launch_bounds__(kThreads, 1) groups_kernel(int page_size, int n, int least, int32_t *groups) {
    __shared__ int s_count[kMost], s_shared[kMost], s_warp[kThreads / 32];
    ptx::launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, i0 = tid * kPer;
    for (int i = tid; i < n; i += kThreads) s_count[i] = 0, s_shared[i] = INT32_MAX;
    ptx::wait_prior_grid();
    int common[kPer], first[kPer], last = 0;  // last: beginning of the group that the thread's last entry belongs to, as far as it knows
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        common[j] = i0 + j < n ? groups[2 * n + i0 + j] : INT32_MAX;
        if (common[j] < least) last = i0 + j;
    }
    int top = last;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) top = max(top, __shfl_up_sync(~0u, top, o));  // (lanes below o get their own)
    if (lane == 31) s_warp[warp] = top;
    const int before = __shfl_up_sync(~0u, top, 1);
    __syncthreads();
    int at = lane > 0 ? before : 0;
    for (int w = 0; w < warp; ++w) at = max(at, s_warp[w]);
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        if (i0 + j >= n) break;
        if (common[j] < least) at = i0 + j;
        first[j] = at;
        atomicAdd(&s_count[at], 1);
        if (at < i0 + j) atomicMin(&s_shared[at], common[j]);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        if (i0 + j >= n) break;
        groups[i0 + j] = first[j];
        groups[n + i0 + j] = s_count[first[j]];
        groups[2 * n + i0 + j] = s_count[first[j]] > 1 ? s_shared[first[j]] * page_size : 0;
    }
}

PageShape page_shape(const mate_cache_t *c) {
    const int64_t size = (int64_t)elem_size(c->dtype);
    const unsigned per_row = (unsigned)(c->d * size / 16), units = (unsigned)(c->kv_heads * c->page_size) * per_row;
    // even pieces of up to 2048 units, whole rounds of the threads (a few pages of 196 KB in two layers moved in 8.4 us; with a page to
    // each block 24.6)
    const unsigned pieces = (units + 2047) / 2048, piece = ((units + pieces - 1) / pieces + kCopyThreads - 1) / kCopyThreads * kCopyThreads;
    return {c->page_stride * size, c->head_stride * size, c->slot_stride * size, c->layer_stride * size,
            c->kv_heads, (int)per_row, c->layers, c->page_size, per_row > 1 ? (unsigned)(((uint64_t)1 << 32) / per_row + 1) : 0,
            (int)piece, (int)((units + piece - 1) / piece)};
}
size_t fork_bytes(int n) { return sizeof(ForkItem) * (size_t)n; }
size_t compact_bytes(const mate_cache_t *c) { return sizeof(int32_t) * (64 + 3 * (size_t)c->pages); }

int check_list(const mate_cache_t *c, const int32_t *list, int n, bool may_be_null) {
    if (n < 0 || (n > 0 && !list && (!may_be_null || n > c->seqs))) return MATE_ERR_INVALID_ARG;
    return n > kMost ? MATE_ERR_UNSUPPORTED : MATE_OK;
}
int check_workspace(const void *workspace, size_t have, size_t need) {
    if (!workspace || have < need) return MATE_ERR_WORKSPACE;
    return is_aligned(workspace, 256) ? MATE_OK : MATE_ERR_ALIGNMENT;
}
int as_status(cudaError_t e) { return e == cudaSuccess ? MATE_OK : MATE_ERR_CUDA; }

}  // namespace

size_t decode_workspace(const mate_cache_t *cache, int B);  // mate_decode.cu

}  // namespace mate

using namespace mate;

extern "C" {

int mate_cache_extend(const mate_cache_t *cache, const int32_t *seqs, const int32_t *counts, int n, int32_t *granted, void *stream) {
    int rc = check_cache(cache);
    if (rc == MATE_OK) rc = check_list(cache, seqs, n, true);
    if (rc == MATE_OK && n > 0 && (!counts || !granted)) rc = MATE_ERR_INVALID_ARG;
    if (rc == MATE_OK) rc = check_cache_device(cache);
    if (rc != MATE_OK || n == 0) return rc;
    static SmemAttrOnce attr;
    rc = attr.ensure((const void *)extend_kernel, kExtendSmem, cache->device);
    if (rc != MATE_OK) return rc;
    return as_status(launch_after(extend_kernel, dim3(1), kThreads, kExtendSmem, (cudaStream_t)stream, cache_args(cache, 0), seqs, counts, n, granted));
}

int mate_cache_fork(const mate_cache_t *cache, const int32_t *parents, const int32_t *children, int n, void *workspace,
                    size_t workspace_bytes, void *stream) {
    int rc = check_cache(cache);
    if (rc == MATE_OK) rc = check_list(cache, parents, n, false);
    if (rc == MATE_OK) rc = check_list(cache, children, n, false);
    if (rc == MATE_OK && n > 0) rc = check_workspace(workspace, workspace_bytes, fork_bytes(n));
    if (rc == MATE_OK) rc = check_cache_device(cache);
    if (rc != MATE_OK || n == 0) return rc;
    const CacheArgs c = cache_args(cache, 0);
    ForkItem *items = static_cast<ForkItem *>(workspace);
    cudaError_t e = launch_after(fork_kernel, dim3(1), kThreads, 0, (cudaStream_t)stream, c, parents, children, n, items);
    if (e == cudaSuccess)
        e = launch_after(fork_copy_kernel, dim3((unsigned)n, 2 * (unsigned)cache->layers + 1, (unsigned)page_shape(cache).pieces), kCopyThreads, 0, (cudaStream_t)stream, c,
                         page_shape(cache), (const ForkItem *)items);
    return as_status(e);
}

int mate_cache_free(const mate_cache_t *cache, const int32_t *seqs, int n, void *stream) {
    int rc = check_cache(cache);
    if (rc == MATE_OK && (n < 0 || (!seqs && n > cache->seqs))) rc = MATE_ERR_INVALID_ARG;
    if (rc == MATE_OK) rc = check_cache_device(cache);
    if (rc != MATE_OK || n == 0) return rc;
    return as_status(launch_after(free_kernel, dim3((unsigned)n), kCopyThreads, 0, (cudaStream_t)stream, cache_args(cache, 0), seqs));
}

int mate_cache_compact(const mate_cache_t *cache, int32_t *n_live, void *workspace, size_t workspace_bytes, void *stream) {
    int rc = check_cache(cache);
    if (rc == MATE_OK && !n_live) rc = MATE_ERR_INVALID_ARG;
    if (rc == MATE_OK) rc = check_workspace(workspace, workspace_bytes, compact_bytes(cache));
    if (rc == MATE_OK) rc = check_cache_device(cache);
    if (rc != MATE_OK) return rc;
    const CacheArgs c = cache_args(cache, 0);
    int32_t *w = static_cast<int32_t *>(workspace);
    const Moves m = {w, w + 64, w + 64 + (size_t)cache->pages, w + 64 + 2 * (size_t)cache->pages};
    cudaError_t e = launch_after(compact_kernel, dim3(1), kThreads, 0, (cudaStream_t)stream, c, m, n_live);
    if (e == cudaSuccess)
        e = launch_after(compact_copy_kernel, dim3((unsigned)(n_sms(cache->device) * kCopyBlocks)), kCopyThreads, 0, (cudaStream_t)stream, c, page_shape(cache), m);
    return as_status(e);
}

int mate_cache_groups(const mate_cache_t *cache, const int32_t *seqs, int n, int min_len, int32_t *groups, void *stream) {
    int rc = check_cache(cache);
    if (rc == MATE_OK) rc = check_list(cache, seqs, n, true);
    if (rc == MATE_OK && (min_len < 0 || (n > 0 && !groups))) rc = MATE_ERR_INVALID_ARG;
    if (rc == MATE_OK) rc = check_cache_device(cache);
    if (rc != MATE_OK || n == 0) return rc;
    const int least = min_len > cache->page_size ? pages_of(min_len, cache->page_size) : 1;
    cudaError_t e = launch_after(common_kernel, dim3((unsigned)n), kCommonThreads, 0, (cudaStream_t)stream, cache_args(cache, 0), seqs, groups + 2 * (size_t)n);
    if (e == cudaSuccess) e = launch_after(groups_kernel, dim3(1), kThreads, 0, (cudaStream_t)stream, cache->page_size, n, least, groups);
    return as_status(e);
}

int mate_cache_workspace_bytes(const mate_cache_t *cache, int n, size_t *fork, size_t *compact, size_t *decode) {
    const int rc = check_cache(cache);
    if (rc != MATE_OK) return rc;
    if (n < 0) return MATE_ERR_INVALID_ARG;
    if (fork) *fork = fork_bytes(n);
    if (compact) *compact = compact_bytes(cache);
    if (decode) *decode = decode_workspace(cache, n);
    return MATE_OK;
}

int mate_cache_status(const mate_cache_t *cache, void *stream) {
    int rc = check_cache(cache);
    if (rc == MATE_OK) rc = check_cache_device(cache);
    if (rc != MATE_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    int32_t s = 0;
    if (cudaMemcpyAsync(&s, cache->status, sizeof s, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaMemsetAsync(cache->status, 0, sizeof s, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess)
        return MATE_ERR_CUDA;
    return s & kCacheTimeout ? MATE_ERR_TIMEOUT : s & kCacheFull ? MATE_ERR_NOMEM : s ? MATE_ERR_INVALID_ARG : MATE_OK;
}

}  // extern "C"

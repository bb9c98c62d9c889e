// Attention of one new token per sequence where sequences share their first tokens (mate_attn_decode_shared): the shared keys and
// values of a group are read once for all of its sequences, whose query heads are the rows of one product,
//     S = Q K^T,  m = max S,  P = exp(S - m),  O = P V / sum P,  LSE = m + ln sum P
// per kv head over the shared tokens, the same over each sequence's own tokens behind them, and the two put together by their m and
// sum P.
//
// Work.  An item is a kv head and a tile of rows of a segment -- a group's shared tokens, or the own tokens of one sequence -- and its
// length in units of kUnit tokens.  Blocks get equal shares of all items' units (found by every block from the lengths, which the host
// does not know): a long segment is spread over the GPU, short ones are put together.  What a block leaves of an item that is not
// a row's whole result -- m, sum P and the sum of values, in fp32 -- is joined by a second kernel, in the order of the tokens: the same bits
// on every launch.
//
// Tokens are looked through 128 at a time by their ids; those that no row of the tile attends are left out before anything of them is read.
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "mate_cache.h"
#include "sm100_ptx.cuh"
#include "tc_tiles.cuh"

namespace mate {
namespace {

constexpr int kUnit = 32;     // tokens of a unit of work: what a warp looks through in one go
constexpr int kOver = 4;      // units that an item costs besides its tokens
constexpr int kMaxBatch = 4096;
constexpr int kMaxHeads = 1024;
constexpr int kNever = INT32_MIN;  // an id that no token has
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Where the results of an item are: [slot] of the block that begins it, then [0] of the next ones up to `last`.
struct Joint {
    int32_t slot, first, last, unused;  // slot < 0: with the rows' whole results
};

struct SharedParams {
    CacheArgs cache;
    const void *Q;
    int64_t q_batch, q_head;
    int B, heads, kv_heads, group, d, max_len;
    int pack, own_tiles;  // entries whose own tokens make an item (their rows fill a tile), or tiles of the rows of one
    const int32_t *seqs, *row_ids, *col_ids, *groups;
    float scale_log2;  // scale / ln 2: weights are powers of two
    int flip;          // tensor-core kernel: the scale above is positive, and the queries change their sign
    void *O;
    float *LSE;
    unsigned page16, head16, slot16;  // strides in 16 bytes; no place is beyond 2^32 of them
    // x / page_size and x / group by multiplication: (umulhi(x, mul) + x) >> shift for x < 2^31
    unsigned page_mul, page_shift, group_mul, group_shift;
    Joint *joints;                    // [2][kv_heads][B own_tiles]: shared tokens, by the first entry of the tile's group, and own ones
    float2 *whole_stats;              // [2][B heads]  m and sum P of rows whose item one block has done
    float *whole;                     // [2][B heads][d]
    float *parts;                     // [blocks][2]: values in groups of four by row, then the rows' m and sum P
    uint32_t views[kMaxHeads / 16];   // two bits a head
};
__device__ __forceinline__ int page_index(const SharedParams &p, int token) {
    return (int)((__umulhi((unsigned)token, p.page_mul) + (unsigned)token) >> p.page_shift);
}
__device__ __forceinline__ int by_group(const SharedParams &p, int row) {
    return (int)((__umulhi((unsigned)row, p.group_mul) + (unsigned)row) >> p.group_shift);
}
__device__ __forceinline__ int view_at(const SharedParams &p, int h) { return p.views[h >> 4] >> 2 * (h & 15) & 3; }
__host__ __device__ constexpr int64_t part_floats(int rows, int d) { return (int64_t)rows * (d + 2); }

// ---- what there is to do

struct Entry {
    int s;           // its sequence; -1: none
    int len;
    int own0, own1;  // its own tokens
    int count;       // of its group, 0: it is in none
    int first, shared;
    int counts;      // the shared tokens are its own too
    int q_row, q_col, prefix;
    int bad;
};
// (called, not put in line: what a block runs through once misses the instruction cache, which holds 32 KB for all of its roles)
// What does not fit together on the device leaves an entry without a group: the rows of one group are the same in all of its entries.  (Two
// rounds of loads, the second one's indexes brought into range instead of looked at first.)
__device__ __noinline__ void entry_of(const SharedParams &p, int b, Entry *to) {
    bool is_bad = false, *bad = &is_bad;
    const int s = p.seqs ? p.seqs[b] : b, q_row = p.row_ids[b], q_col = p.col_ids[b];
    const int first = p.groups[b], count = p.groups[p.B + b], shared = p.groups[2 * p.B + b];
    const int at = min(max(s, 0), p.cache.seqs - 1), f = min(max(first, 0), b);
    int len = p.cache.lens[at];
    const int prefix = p.cache.prefix[at], first_of = p.groups[f], count_of = p.groups[p.B + f], shared_of = p.groups[2 * p.B + f];
    Entry e = {s == at ? s : -1, 0, 0, 0, 0, first, 0, 0, q_row, q_col, max(0, prefix)};
    if (s != at || shared < 0) *bad = true;
    if (s == at) e.len = clip_len(len, p.max_len, bad);
    if (shared > 0 && count > 1) {
        if (first == f && count <= p.B - first && b - first < count && shared <= p.max_len && first_of == first && count_of == count &&
            shared_of == shared)
            e.count = count, e.shared = shared;
        else
            *bad = true;
    }
    const bool has = e.count > 0 && e.len >= shared, padding = q_row < 0 || q_col < 0 || e.s < 0;
    if (e.count > 0 && !has) *bad = true;
    e.counts = has && !padding;
    e.own0 = has ? shared : 0;
    e.own1 = padding ? e.own0 : e.len;
    e.bad = is_bad;
    *to = e;
}
// Units of tokens.  The first kOver units of an item stand for what it costs whatever its length: none of its tokens belong to them.
__host__ __device__ __forceinline__ int units_of(int tokens) { return (tokens + kUnit - 1) / kUnit; }
__device__ __forceinline__ unsigned share(unsigned U, unsigned C, unsigned i) { return U / C * i + U % C * i / C; }
// Items of the shared tokens of the group that entry b is the first of: kv heads and tiles of rows.
__device__ __forceinline__ bool leads(const Entry &e, int b) { return e.count > 0 && e.first == b; }
template <int RT>
__device__ __forceinline__ int group_tiles(const SharedParams &p, const Entry &e) {
    return (e.count * p.group + RT - 1) / RT;
}
// Units of an item of own tokens.  (Without any it has one: its rows have a result too.)
__device__ __forceinline__ int own_units(int tokens_units) { return tokens_units > 0 ? kOver + tokens_units : 1; }

struct Start {
    unsigned total, before;  // units of all; of the batches of `pack` entries in front of `batch`
    unsigned blocks;         // that get any: no more than there are units
    int batch;
};
// All threads call it: the batch that the block's first unit belongs to.  `cost`: [B] in shared memory, free afterwards.
template <int RT, int NT>
__device__ Start find_start(const SharedParams &p, uint2 *cost) {
    __shared__ unsigned s_sum[NT / 32];
    __shared__ Start s_start;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, batches = (p.B + p.pack - 1) / p.pack;
#pragma unroll 1
    for (int b = tid; b < p.B; b += NT) {
        Entry e;
        entry_of(p, b, &e);
        cost[b] = make_uint2(units_of(e.own1 - e.own0), leads(e, b) ? p.kv_heads * group_tiles<RT>(p, e) * (kOver + units_of(e.shared)) : 0);
        if (e.bad && blockIdx.x == 0) atomicOr(p.cache.status, kCacheBad);
    }
    if (tid == 0) s_start = {0, 0, 0, 0};
    __syncthreads();
    // a warp to each batch; its cost replaces that of its first entry
#pragma unroll 1
    for (int i = warp; i < batches; i += NT / 32) {
        unsigned own = 0, shared = 0;
#pragma unroll 1
        for (int b = i * p.pack + lane; b < min(p.B, (i + 1) * p.pack); b += 32) own += cost[b].x, shared += cost[b].y;
        own = __reduce_add_sync(~0u, own), shared = __reduce_add_sync(~0u, shared);
        __syncwarp();
        if (lane == 0) cost[i * p.pack].x = shared + (unsigned)(p.kv_heads * p.own_tiles) * own_units((int)own);
    }
    __syncthreads();
    const int per = (batches + NT - 1) / NT, i0 = min(batches, tid * per), i1 = min(batches, i0 + per);
    unsigned own = 0;
#pragma unroll 1
    for (int i = i0; i < i1; ++i) own += cost[i * p.pack].x;
    unsigned sum = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned y = __shfl_up_sync(~0u, sum, o);
        if (lane >= o) sum += y;
    }
    if (lane == 31) s_sum[warp] = sum;
    __syncthreads();
    unsigned total = 0, before = sum - own;
#pragma unroll 1
    for (int w = 0; w < NT / 32; ++w) {
        if (w < warp) before += s_sum[w];
        total += s_sum[w];
    }
    const unsigned blocks = min(total, gridDim.x);
    if (blockIdx.x < blocks) {
        const unsigned at = share(total, blocks, blockIdx.x);
        if (at >= before && at < before + own) {
            int i = i0;
#pragma unroll 1
            for (; i < i1 - 1 && at >= before + cost[i * p.pack].x; ++i) before += cost[i * p.pack].x;
            s_start = {total, before, blocks, i};
        }
    }
    __syncthreads();
    return s_start;
}

// A part of an item: units [u0, u1) of them.
struct Part {
    int b, seg, kv, tile;  // first entry; shared tokens (0) or own ones (1); tile of rows
    int u0, u1, units;
    int n_rows;
};
enum { kAll, kBegins, kGoesOn };
__device__ __forceinline__ int part_state(const Part &part) { return part.u0 > 0 ? kGoesOn : part.u1 == part.units ? kAll : kBegins; }
// Of a row of the tile: its entry, counted from the part's first, and its place among all rows of the batch.
template <int RT>
__device__ __forceinline__ int member_of(const SharedParams &p, const Part &part, int r) {
    return by_group(p, part.tile * RT + r);
}
template <int RT>
__device__ __forceinline__ size_t row_of(const SharedParams &p, const Part &part, int r, int member) {
    return (size_t)(part.b + member) * p.heads + part.kv * p.group + part.tile * RT + r - member * p.group;
}
// (tiles of a group of n entries: fewer than n own_tiles, so those of different groups have different places)
__device__ __forceinline__ Joint *joint_of(const SharedParams &p, int seg, int kv, int b, int tile) {
    return p.joints + ((size_t)seg * p.kv_heads + kv) * p.B * p.own_tiles + (size_t)b * p.own_tiles + tile;
}
// Of the part that begins an item that goes on in the next blocks (it is the last one of its block's share).
__device__ __noinline__ Joint joint_from(const Part &part, const Start &start, int slot) {
    const int64_t end = (int64_t)share(start.total, start.blocks, blockIdx.x + 1) - (part.u1 - part.u0) + part.units;
    return {slot, (int)blockIdx.x, (int)min((end * start.blocks - 1) / start.total, (int64_t)start.blocks - 1), 0};
}

// ---- who attends what

// A row attends a key if the key's place is below `below` (text keys stand at -1, those of the prefix where they stand; -2: the row attends
// nothing), or one of the ids is the one it wants.
__device__ __forceinline__ bool attends(int want_row, int want_col, int below, int place, int row, int col) {
    return place < below || row == want_row || col == want_col;
}
// The rows of a tile, as those who weigh keys need them,
template <int RT>
struct Rows {
    int want_row[RT], want_col[RT], below[RT];
};
// and as those who look for keys do.
template <int RT>
struct Wishes {
    int least, most;  // of `below` over the rows that are there
    int views;        // 1: some want a row, 2: a column
    int n;            // of a group: without repetitions of the row before
    int2 want[RT];
    __device__ void clear() { least = INT32_MAX, most = INT32_MIN, views = n = 0; }
};
// Keys, with what the rows go by.
struct alignas(16) Key {
    unsigned at;  // in 16 bytes from the cache's beginning
    int place, row, col;
};
constexpr int kList = 256, kScouts = 128;

// kScouts threads walk the parts of the block's share and look through their tokens, four units at a time, a warp to each; the keys that
// count go onto a list.  The next ones' ids, and the pages of the ones behind them, are on their way meanwhile.  Barrier 1 is theirs.
//
// Units of own tokens are numbered through over the entries of the batch, each entry beginning with a new one.
template <int RT>
struct ScoutSmem {
    Entry entries[kScouts];  // of the batch
    int before[kScouts + 1]; // units of own tokens in front of an entry's
    unsigned leaders[4];     // a bit for each entry: it is the first of a group
    Wishes<RT> wishes[2];    // of the parts in turn
    Key list[kList];         // what look() writes is seen behind the next barrier
    uint8_t owners[kList];   // entries of the batch
    int counts[2][4];
};
// Where the loads of a look stand.
struct Asked {
    int j, owner, page;
    bool there;
};
template <int RT>
struct Scout {
    const SharedParams &p;
    ScoutSmem<RT> &sm;
    int tid;
    // the walk: next item of the share
    int batch, entry, item, u, left;  // entry: that leads (of the batch), kScouts: own tokens; left: units of the share
    int held, parts;                  // batch that is in shared memory; parts so far
    // the looks at the present part
    int seg, next, end, pending, list_at, looks;  // next, end: units
    unsigned head_at;
    Asked asked;
    unsigned at;
    int j, owner, row, col;
    bool there, bad;

    __device__ static void sync() { asm volatile("barrier.cta.sync 1, 128;" ::: "memory"); }
    __device__ int entries() const { return min(p.pack, p.B - batch * p.pack); }
    __device__ void hold() {
        held = batch;
        sync();
        int units = 0;
        bool first = false;
        if (tid < entries()) {
            const int b = batch * p.pack + tid;
            entry_of(p, b, sm.entries + tid);
            const Entry &e = sm.entries[tid];
            units = units_of(e.own1 - e.own0), first = leads(e, b);
        }
        int sum = units;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(~0u, sum, o);
            if ((tid & 31) >= o) sum += y;
        }
        const unsigned those = __ballot_sync(~0u, first);
        if ((tid & 31) == 31) sm.counts[0][tid >> 5] = sum, sm.leaders[tid >> 5] = those;
        sync();
        for (int w = 0; w < tid >> 5; ++w) sum += sm.counts[0][w];
        sm.before[tid + 1] = sum;
        if (tid == 0) sm.before[0] = 0;
        sync();
    }
    // The first entry from `entry` on that leads a group, kScouts if there is none.
    __device__ int leader_from(int from) const {
        for (int w = from >> 5; w < 4; ++w) {
            const unsigned those = sm.leaders[w] & (w == from >> 5 ? ~0u << (from & 31) : ~0u);
            if (those) return 32 * w + __ffs(those) - 1;
        }
        return kScouts;
    }
    __device__ int items() const { return p.kv_heads * (entry < kScouts ? group_tiles<RT>(p, sm.entries[entry]) : p.own_tiles); }
    __device__ int units() const { return entry < kScouts ? kOver + units_of(sm.entries[entry].shared) : own_units(sm.before[kScouts]); }
    __device__ void start(const Start &from) {
        const unsigned begin = share(from.total, from.blocks, blockIdx.x);
        unsigned in = begin - from.before;
        batch = from.batch, parts = 0, bad = false, looks = 0;
        left = (int)(share(from.total, from.blocks, blockIdx.x + 1) - begin);
        if (tid == 0) sm.wishes[0].clear();
        hold();
        entry = leader_from(0);
#pragma unroll 1
        while (entry < kScouts && in >= (unsigned)items() * units()) in -= (unsigned)items() * units(), entry = leader_from(entry + 1);
        item = (int)(in / (unsigned)units());
        u = (int)(in - (unsigned)item * units());
        if (u <= kOver) left += u, u = 0;
    }
    // The next part of the share.  (It comes to an end whatever it finds: every part takes a unit off the share.)
    __device__ bool next_part(Part &part) {
#pragma unroll 1
        while (left > 0 && batch * p.pack < p.B) {
            if (held != batch) {
                hold();
                entry = leader_from(0);
            }
            if (item < items()) {
                const int n = units(), u1 = min(n, u + left);
                if (u1 <= kOver && u1 < n) break;  // it ends among the units that stand for the item: the next block takes it
                const int tiles = entry < kScouts ? group_tiles<RT>(p, sm.entries[entry]) : p.own_tiles, kv = item / tiles, tile = item - kv * tiles;
                const int rows = (entry < kScouts ? sm.entries[entry].count : entries()) * p.group;
                part = {batch * p.pack + (entry < kScouts ? entry : 0), entry < kScouts ? 0 : 1, kv, tile, u, u1, n, min(RT, rows - tile * RT)};
                left -= max(1, u1 - u);
                u = 0;
                ++item;
                return true;
            }
            item = 0;
            if (entry == kScouts)
                ++batch;
            else
                entry = leader_from(entry + 1);
        }
        left = 0;
        return false;
    }
    // Who the warp's 32 tokens of unit `unit` belong to, and their pages.
    __device__ void ask_page(int unit) {
        asked = {0, 0, -1, false};
        if (unit >= end) return;
        const int lane = tid & 31;
        int first = 0, stop, from = 0;
        if (seg == 0) {
            asked.owner = leader;
            stop = min(sm.entries[leader].shared, sm.entries[leader].len);
        } else {
            int n = 0;  // entries that begin at the unit or in front of it
#pragma unroll
            for (int i = 0; i < kScouts / 32; ++i) n += sm.before[32 * i + lane] <= unit;
            asked.owner = __reduce_add_sync(~0u, n) - 1;
            // (of entries without tokens the last one that begins there is found: it is the one behind them)
            const Entry &e = sm.entries[asked.owner];
            first = e.own0, stop = e.own1, from = sm.before[asked.owner];
        }
        const int s = sm.entries[asked.owner].s;
        asked.j = first + (unit - from) * kUnit + lane;
        asked.there = asked.j < stop && s >= 0;
        if (asked.there) asked.page = p.cache.table[(size_t)s * p.cache.width + page_index(p, asked.j)];
    }
    __device__ void ask_ids() {  // of the tokens whose page has been asked for
        j = asked.j, owner = asked.owner;
        there = asked.there && in_range(asked.page, p.cache.pages);
        if (asked.there && !there) bad = true;
        if (!there) return;
        const int slot = j - page_index(p, j) * p.cache.page_size, id = asked.page * p.cache.page_size + slot;
        row = p.cache.row_ids[id], col = p.cache.col_ids[id];
        at = (unsigned)asked.page * p.page16 + (unsigned)slot * p.slot16 + head_at;
    }
    int leader;
    // Behind a barrier that the last look at the part before it is in front of.
    __device__ void begin(const Part &part, Rows<RT> &rows) {
        seg = part.seg, leader = part.b - batch * p.pack;
        next = max(0, part.u0 - kOver), end = max(0, part.u1 - kOver);
        if (seg == 1) end = min(end, sm.before[kScouts]);
        head_at = (unsigned)part.kv * p.head16;
        pending = list_at = 0;
        ask_page(next + (tid >> 5));
        Wishes<RT> &w = sm.wishes[parts & 1];
        ++parts;
        if (tid == 0) sm.wishes[parts & 1].clear();
        int want_row = kNever, want_col = kNever, below = -2;
        if (tid < part.n_rows) {
            const int member = member_of<RT>(p, part, tid), view = view_at(p, part.kv * p.group + part.tile * RT + tid - member * p.group);
            Entry e;
            entry_of(p, part.b + member, &e);
            if (seg == 0 ? e.counts && e.first == part.b && e.count > 0 : e.own1 > e.own0) {
                const bool text = e.q_row == MATE_ID_TEXT || e.q_col == MATE_ID_TEXT;
                below = text ? INT32_MAX : e.prefix;
                if (!text && view != MATE_VIEW_COL) want_row = e.q_row;
                if (!text && view != MATE_VIEW_ROW) want_col = e.q_col;
            }
        }
        if (tid < RT) rows.want_row[tid] = want_row, rows.want_col[tid] = want_col, rows.below[tid] = below;
        const int least = __reduce_min_sync(~0u, below < 0 ? INT32_MAX : below), most = __reduce_max_sync(~0u, below);
        const int views = (__any_sync(~0u, want_row != kNever) ? 1 : 0) | (__any_sync(~0u, want_col != kNever) ? 2 : 0);
        const int row_before = __shfl_up_sync(~0u, want_row, 1), col_before = __shfl_up_sync(~0u, want_col, 1);
        const bool again = (tid & 31) > 0 && row_before == want_row && col_before == want_col;
        if ((tid & 31) == 0 && most >= 0) atomicMin(&w.least, least), atomicMax(&w.most, most), atomicOr(&w.views, views);
        if (!again && (want_row != kNever || want_col != kNever)) w.want[atomicAdd(&w.n, 1)] = make_int2(want_row, want_col);
        __syncwarp();
        ask_ids();
        ask_page(next + 4 + (tid >> 5));
        sync();
    }
    __device__ const Wishes<RT> &wishes() const { return sm.wishes[parts + 1 & 1]; }  // of the present part
    __device__ bool more() const { return next < end; }
    __device__ void look() {
        const Wishes<RT> &w = wishes();
        Key key = {at, j, row, col};
        const int of = owner;
        bool is = there && row >= 0 && col >= 0;
        if (is) {
            if (row == MATE_ID_TEXT || col == MATE_ID_TEXT) key.place = -1;
            if (seg == 0) {
                is = key.place < w.most;
#pragma unroll 1
                for (int i = 0; i < w.n && !is; ++i) is = row == w.want[i].x || col == w.want[i].y;
            } else {
                const Entry &e = sm.entries[of];
                is = e.q_row == MATE_ID_TEXT || e.q_col == MATE_ID_TEXT || key.place < e.prefix || ((w.views & 1) && row == e.q_row) ||
                     ((w.views & 2) && col == e.q_col);
            }
        }
        next += 4;
        if (next < end) {
            __syncwarp();
            ask_ids();
            __syncwarp();
            ask_page(next + 4 + (tid >> 5));
        }
        __syncwarp();
        const unsigned those = __ballot_sync(~0u, is);
        int *count = sm.counts[looks++ & 1];
        if ((tid & 31) == 0) count[tid >> 5] = __popc(those);
        sync();
        int before = 0, all = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i < tid >> 5) before += count[i];
            all += count[i];
        }
        const unsigned to = (unsigned)(list_at + pending + before + __popc(those & ((1u << (tid & 31)) - 1))) % kList;
        if (is) sm.list[to] = key, sm.owners[to] = (uint8_t)of;
        pending += all;
    }
    __device__ Key key(int i) const { return sm.list[(unsigned)(list_at + i) % kList]; }
    __device__ int owner_of_key(int i) const { return sm.owners[(unsigned)(list_at + i) % kList]; }
    // Whether every row that a key is for attends it.
    __device__ bool is_plain(const Key &key, int of) const {
        const Entry &e = sm.entries[of];
        return seg == 0 ? key.place < wishes().least : e.q_row == MATE_ID_TEXT || e.q_col == MATE_ID_TEXT || key.place < e.prefix;
    }
    __device__ void taken(int n) { list_at = (int)((unsigned)(list_at + n) % kList), pending -= n; }
};

__device__ __forceinline__ void put(float x, float *y) { *y = x; }
__device__ __forceinline__ void put(float x, __nv_bfloat16 *y) { *y = __float2bfloat16_rn(x); }
__device__ __forceinline__ float natural(float m, float sum) { return sum == 0.f ? -INFINITY : (m + log2f(sum)) * kLn2; }

// ---- the kernel for fp32, without tensor cores: tiles of 64 rows and 32 keys

constexpr int kSimtRows = 64, kSimtKeys = 32, kSimtThreads = 256;

template <int DP>
struct SimtSmem {
    float q[kSimtRows][DP + 4], k[kSimtKeys][DP + 4], v[kSimtKeys][DP];
    float s[kSimtRows][kSimtKeys + 4];
    Rows<kSimtRows> rows;
    ScoutSmem<kSimtRows> scout;
    Part part;
    Key keys[kSimtKeys];
    int owners[kSimtKeys];
    int n, last, plain, done;
};

__device__ __forceinline__ void load16(const float *from, float *to) { *reinterpret_cast<float4 *>(to) = *reinterpret_cast<const float4 *>(from); }

template <int DP>
__global__ void __launch_bounds__(kSimtThreads) shared_simt_kernel(const __grid_constant__ SharedParams p) {
    extern __shared__ __align__(16) char smem_raw[];
    auto &sm = *reinterpret_cast<SimtSmem<DP> *>(smem_raw);
    constexpr int kVec = 4, kCols = DP / 32, kR = kSimtRows / (kSimtThreads / 32);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r0 = warp * kR;
    ptx::wait_prior_grid();
    static_assert(sizeof(sm.q) + sizeof(sm.k) + sizeof(sm.v) + sizeof(sm.s) >= kMaxBatch * sizeof(uint2), "room for the entries' cost");
    const Start start = find_start<kSimtRows, kSimtThreads>(p, reinterpret_cast<uint2 *>(smem_raw));
    if (blockIdx.x >= start.blocks) return;
    for (int i = tid; i < (int)(sizeof(SimtSmem<DP>) / 4); i += kSimtThreads) reinterpret_cast<uint32_t *>(smem_raw)[i] = 0;  // columns that nobody writes
    Scout<kSimtRows> scout = {p, sm.scout, tid};
    __syncthreads();
    if (tid < kScouts) scout.start(start);
    for (int n_parts = 0;; ++n_parts) {
        Part part;
        if (tid < kScouts) {
            const bool is = scout.next_part(part);
            if (is) scout.begin(part, sm.rows);
            if (tid == 0) sm.done = !is, sm.part = part;
        }
        __syncthreads();
        if (sm.done) break;
        part = sm.part;
        for (int i = tid; i < kSimtRows * (p.d / kVec); i += kSimtThreads) {
            const int r = i / (p.d / kVec), c = (i - r * (p.d / kVec)) * kVec;
            if (r >= part.n_rows) continue;
            const int member = member_of<kSimtRows>(p, part, r), head = part.kv * p.group + part.tile * kSimtRows + r - member * p.group;
            load16((const float *)p.Q + (part.b + member) * p.q_batch + head * p.q_head + c, &sm.q[r][c]);
        }
        float o[kR][kCols], m[kR], l[kR];
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            m[r] = -INFINITY, l[r] = 0.f;
#pragma unroll
            for (int c = 0; c < kCols; ++c) o[r][c] = 0.f;
        }
        for (bool more = true; more;) {
            if (tid < kScouts) {
                while (scout.pending < kSimtKeys && scout.more()) scout.look();
                scout.sync();
                const int n = min(scout.pending, kSimtKeys);
                bool every = true;
                if (tid < kSimtKeys) {
                    if (tid < n) sm.keys[tid] = scout.key(tid), sm.owners[tid] = scout.owner_of_key(tid);
                    every = part.seg == 0 && __all_sync(~0u, tid >= n || scout.is_plain(sm.keys[tid], sm.owners[tid]));
                }
                if (tid == 0) sm.n = n, sm.last = scout.pending <= kSimtKeys && !scout.more(), sm.plain = every;
                scout.taken(n);
            }
            __syncthreads();
            const int n = sm.n;
            more = !sm.last;
            bool odd = false;
            for (int i = tid; i < kSimtKeys * (p.d / kVec); i += kSimtThreads) {
                const int k = i / (p.d / kVec), c = (i - k * (p.d / kVec)) * kVec;
                if (k < n) {
                    load16((const float *)p.cache.k + (size_t)sm.keys[k].at * kVec + c, &sm.k[k][c]);
                    load16((const float *)p.cache.v + (size_t)sm.keys[k].at * kVec + c, &sm.v[k][c]);
                    for (int e = 0; e < kVec; ++e) odd |= !(fabsf(sm.v[k][c + e]) < INFINITY);
                } else {
                    for (int e = 0; e < kVec; ++e) sm.k[k][c + e] = sm.v[k][c + e] = 0.f;
                }
            }
            // (a weight 0 does not undo a value that is not a number: where not all rows attend all keys, such tiles are summed key by key)
            const bool apart = __syncthreads_or(odd) && !sm.plain;
            if (r0 < part.n_rows) {
                // scores: two rows and four keys of a lane
                float s[2][4] = {};
                const int qr = r0 + lane / 8 * 2, kc = lane % 8;
                for (int c = 0; c < DP; c += 4) {
                    float4 q[2], k[4];
#pragma unroll
                    for (int i = 0; i < 2; ++i) q[i] = *reinterpret_cast<const float4 *>(&sm.q[qr + i][c]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) k[j] = *reinterpret_cast<const float4 *>(&sm.k[kc + 8 * j][c]);
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            s[i][j] = fmaf(q[i].x, k[j].x, fmaf(q[i].y, k[j].y, fmaf(q[i].z, k[j].z, fmaf(q[i].w, k[j].w, s[i][j]))));
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) sm.s[qr + i][kc + 8 * j] = s[i][j] * p.scale_log2;
                __syncwarp();
                // weights: a key of a lane
                const Key key = sm.keys[lane];
                const int of = sm.owners[lane];
                uint32_t those[kR];
#pragma unroll
                for (int r = 0; r < kR; ++r) {
                    const bool is = lane < n && (part.seg == 0 || of == member_of<kSimtRows>(p, part, r0 + r)) &&
                                    attends(sm.rows.want_row[r0 + r], sm.rows.want_col[r0 + r], sm.rows.below[r0 + r], key.place, key.row, key.col);
                    those[r] = __ballot_sync(~0u, is);
                    const float x = is ? sm.s[r0 + r][lane] : -INFINITY;
                    float top = fmaxf(x, m[r]);
#pragma unroll
                    for (int step = 16; step > 0; step >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, step));
                    const float base = top == -INFINITY ? 0.f : top, keep = ptx::ex2(m[r] - base), w = ptx::ex2(x - base);
                    m[r] = top;
                    l[r] = fmaf(l[r], keep, w);  // of the lane's keys
#pragma unroll
                    for (int c = 0; c < kCols; ++c) o[r][c] *= keep;
                    sm.s[r0 + r][lane] = w;
                }
                __syncwarp();
                if (!apart) {
                    for (int k = 0; k < kSimtKeys; k += 4) {
                        float v[4][kCols];
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int c = 0; c < kCols; ++c) v[j][c] = sm.v[k + j][lane * kCols + c];
#pragma unroll
                        for (int r = 0; r < kR; ++r) {
                            const float4 w = *reinterpret_cast<const float4 *>(&sm.s[r0 + r][k]);
#pragma unroll
                            for (int c = 0; c < kCols; ++c) o[r][c] = fmaf(w.x, v[0][c], fmaf(w.y, v[1][c], fmaf(w.z, v[2][c], fmaf(w.w, v[3][c], o[r][c]))));
                        }
                    }
                } else {
#pragma unroll 1
                    for (int i = 0; i < kSimtKeys; ++i) {
                        const int k = i ^ 3;  // (in the order of the sums above: the same bits as without the others' keys)
#pragma unroll
                        for (int r = 0; r < kR; ++r)
                            if (those[r] >> k & 1) {
#pragma unroll
                                for (int c = 0; c < kCols; ++c) o[r][c] = fmaf(sm.s[r0 + r][k], sm.v[k][lane * kCols + c], o[r][c]);
                            }
                    }
                }
            }
            __syncthreads();
        }
        const int state = part_state(part), slot = n_parts == 0 ? 0 : 1;
        float *to = p.parts + (size_t)(2 * blockIdx.x + slot) * part_floats(kSimtRows, p.d);
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            float sum = l[r];
#pragma unroll
            for (int step = 16; step > 0; step >>= 1) sum += __shfl_xor_sync(~0u, sum, step);
            const int row = r0 + r;
            if (row >= part.n_rows) break;
            const size_t whole = (size_t)part.seg * p.B * p.heads + row_of<kSimtRows>(p, part, row, member_of<kSimtRows>(p, part, row));
            for (int c = 0; c < kCols; ++c) {
                const int e = lane * kCols + c;
                if (e >= p.d) break;
                const float x = sum == 0.f ? 0.f : o[r][c];  // (a row that attends nothing here: whatever the others attend)
                (state == kAll ? p.whole + whole * p.d : to)[state == kAll ? e : (e / 4 * kSimtRows + row) * 4 + e % 4] = x;
            }
            if (lane == 0) (state == kAll ? p.whole_stats[whole] : reinterpret_cast<float2 *>(to + (size_t)p.d * kSimtRows)[row]) = make_float2(m[r], sum);
        }
        if (tid == 0 && state != kGoesOn) {
            Joint *joint = joint_of(p, part.seg, part.kv, part.seg == 0 ? part.b : part.b / p.pack, part.tile);
            if (state == kAll)
                joint->slot = -1;
            else
                *joint = joint_from(part, start, slot);
        }
    }
    if (tid < kScouts && scout.bad) atomicOr(p.cache.status, kCacheBad);
}

// ---- the tensor-core kernel (bf16): tiles of 128 rows and 128 keys, one block to an SM

constexpr int kTcRows = 128, kTcKeys = 128;
constexpr int kSoftmaxWarps = 8;              // two teams, which take the tiles in turn; a thread to a row
constexpr int kLoadWarp0 = kSoftmaxWarps, kLoadWarps = kScouts / 32;
constexpr int kCopyWarp0 = kLoadWarp0 + kLoadWarps, kCopyWarps = 3;
constexpr int kMmaWarp = kCopyWarp0 + kCopyWarps;
constexpr int kTcThreads = 32 * (kMmaWarp + 1);
constexpr int kMetas = 4;                     // tiles whose keys are known
constexpr float kRescale = 8.f;               // log2 units that a score may exceed its row's base by
// tensor memory: O of the teams (fp32), then S of their tiles (fp32), which P takes the place of: of every 16 keys the weights' upper halves
// (8 columns of bf16 pairs) and their lower ones
constexpr uint32_t kTmemCols = 512, kTmemO = 0, kTmemS = 256;

template <int DP>
struct TcShape {
    static constexpr int kTile = kTcKeys * DP * 2;              // bytes; column halves of 64 elements, 128 bytes a row and swizzled
    static constexpr int kHalf = kTcKeys * 128;
    static constexpr int kStages = DP == 64 ? 4 : 2;            // tiles of keys, and of values
    // where 16 bytes of a row go
    __device__ static uint32_t place(uint32_t tile, int row, int chunk) {
        return tile + (chunk >> 3) * kHalf + row * 128 + (((chunk & 7) ^ (row & 7)) << 4);
    }
};
struct alignas(16) Meta {
    int n, first, last;  // keys; of the part.  n < 0: the share is done
    uint32_t plain;      // 0x01010101: every row attends every key that is for it
    int ranged;          // keys lo[m] to hi[m] are for the rows of entry m, else all for all
    uint8_t runs[4];     // of every 32 keys: blocks of TcMaps.run keys that lie one behind the other
    alignas(16) int place[kTcKeys];  // (read four at a time)
    alignas(16) int row[kTcKeys];
    alignas(16) int col[kTcKeys];
    unsigned at[kTcKeys];
    uint8_t lo[kTcRows], hi[kTcRows];
};
// Keys and values as matrices whose rows are a slot stride apart: a run of slots is a box, which comes in by one bulk tensor copy for every
// 64 elements.
struct TcMaps {
    CUtensorMap k, v;
    int run, run_log2;  // rows of a box, 8, 16 or 32; 0: every row is copied by itself
};
template <int DP>
struct TcSmem {  // from a multiple of 1024 bytes on
    uint8_t q[2][TcShape<DP>::kTile];
    uint8_t k[TcShape<DP>::kStages][TcShape<DP>::kTile], v[TcShape<DP>::kStages][TcShape<DP>::kTile];
    Meta meta[kMetas];
    ScoutSmem<kTcRows> scout;
    Rows<kTcRows> rows[2];
    Part part[2];
    float2 stats[2][kTcRows];
    uint64_t q_full[2], q_empty[2], k_full[4], k_empty[4], v_full[4], v_empty[4], meta_full[kMetas], meta_empty[kMetas], s_full[2], p_full[2], pv_done[2],
        team[2], both, final_;
    int odd[2];
    uint32_t tmem;
    int abort;
};

__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void *src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
// Whether one of the scouts says so.  All of them call it.
__device__ __forceinline__ bool any_scout(bool x) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.or.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)x), "n"(kScouts)
        : "memory");
    return r != 0;
}

// Every wait is bounded; the first one to run out raises the flag that ends all of them.
__device__ __noinline__ bool wait_long(uint32_t bar, uint32_t parity, volatile int *abort) {
#pragma unroll 1
    for (uint32_t i = 0; i < ptx::kWaitLimit; ++i) {
        if (ptx::mbar_try_wait(bar, parity)) return true;
        if (*abort) return false;
    }
    *abort = 1;
    return false;
}

// 32 scores of a row: those that do not count become -inf.
__device__ __forceinline__ void mask_scores(uint32_t (&v)[32], const Meta &meta, int c0, int want_row, int want_col, int below) {
#pragma unroll
    for (int e = 0; e < 32; e += 4) {
        const int4 place = *reinterpret_cast<const int4 *>(meta.place + c0 + e), row = *reinterpret_cast<const int4 *>(meta.row + c0 + e),
                   col = *reinterpret_cast<const int4 *>(meta.col + c0 + e);
        if (!attends(want_row, want_col, below, place.x, row.x, col.x)) v[e] = 0xff800000u;
        if (!attends(want_row, want_col, below, place.y, row.y, col.y)) v[e + 1] = 0xff800000u;
        if (!attends(want_row, want_col, below, place.z, row.z, col.z)) v[e + 2] = 0xff800000u;
        if (!attends(want_row, want_col, below, place.w, row.w, col.w)) v[e + 3] = 0xff800000u;
    }
}
__device__ __forceinline__ float top_score(const uint32_t (&v)[32], float top) {
    float t[4] = {top, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int e = 0; e < 32; e += 8)
#pragma unroll
        for (int j = 0; j < 4; ++j) t[j] = ptx::fmax3(t[j], __uint_as_float(v[e + 2 * j]), __uint_as_float(v[e + 2 * j + 1]));
    return fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
}
// Weights 2^(s scale - base) of 32 keys, 16 at a time, as pairs of bf16: rounded, and what the rounding left, rounded (their sum has 16 bits: an error of
// 2^-17 of a weight, which the result's rounding to bf16, 2^-9, hides but for one value in some hundred).  The sums take all of them.
__device__ __forceinline__ void weigh(uint32_t (&v)[32], uint64_t scale2, uint64_t neg_base2, uint64_t (&sum)[2]) {
#pragma unroll
    for (int i = 0; i < 32; i += 16) {
        uint32_t lo[8];
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            float x, y;
            ptx::unpack_f32x2(ptx::fma_f32x2(ptx::pack_f32x2(v[i + e], v[i + e + 1]), scale2, neg_base2), x, y);
            x = ptx::ex2(x), y = ptx::ex2(y);
            const uint64_t xy = ptx::pack_f32x2(x, y);
            sum[e >> 1 & 1] = ptx::add_f32x2(sum[e >> 1 & 1], xy);
            const uint32_t h = ptx::cvt_bf16x2(x, y);
            ptx::unpack_f32x2(ptx::sub_f32x2(xy, ptx::pack_f32x2(h << 16, h & 0xffff0000u)), x, y);
            v[i + (e >> 1)] = h, lo[e >> 1] = ptx::cvt_bf16x2(x, y);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i + 8 + e] = lo[e];
    }
}

template <int DP>
__global__ void __launch_bounds__(kTcThreads, 1) shared_tc_kernel(const __grid_constant__ SharedParams p, const __grid_constant__ TcMaps maps) {
    using namespace ptx;
    using S = TcShape<DP>;
    constexpr int kStages = S::kStages, kHalves = DP / 64;
    constexpr int kPer = DP / 8, kRowsOfCopy = 32 / kPer;  // copies: lanes to a row; rows of an instruction
    extern __shared__ uint8_t tc_smem[];
    TcSmem<DP> &sm = *reinterpret_cast<TcSmem<DP> *>(tc_smem + (-smem_u32(tc_smem) & 1023));
    const int tid = threadIdx.x, warp = __shfl_sync(~0u, tid >> 5, 0), lane = tid & 31;
    const auto bar = [](const uint64_t &b) { return smem_u32(&b); };

    if (warp == 0) {  // (a lane to an index: one after the other they take a third of a microsecond)
        if (lane < 2) {
            mbar_init(bar(sm.q_full[lane]), kLoadWarps);
            mbar_init(bar(sm.q_empty[lane]), kSoftmaxWarps + 1);
            mbar_init(bar(sm.s_full[lane]), 1), mbar_init(bar(sm.pv_done[lane]), 1);
            mbar_init(bar(sm.p_full[lane]), kSoftmaxWarps / 2), mbar_init(bar(sm.team[lane]), kSoftmaxWarps / 2);
            sm.odd[lane] = 0;
        }
        if (lane < kStages) {
            mbar_init(bar(sm.k_full[lane]), kCopyWarps), mbar_init(bar(sm.v_full[lane]), kCopyWarps);
            mbar_init(bar(sm.k_empty[lane]), 1), mbar_init(bar(sm.v_empty[lane]), 1);
        }
        if (lane < kMetas) mbar_init(bar(sm.meta_full[lane]), kLoadWarps), mbar_init(bar(sm.meta_empty[lane]), kSoftmaxWarps + kCopyWarps + 1);
        if (lane == 0) {
            mbar_init(bar(sm.both), kSoftmaxWarps), mbar_init(bar(sm.final_), 1);
            sm.abort = 0;
        }
        fence_mbar_init();
    }
    if (warp == kCopyWarp0 && lane < 2) prefetch_tmap(lane ? &maps.v : &maps.k, maps.run);
    if (warp == kMmaWarp) {
        tmem_alloc(smem_u32(&sm.tmem), kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before();
    wait_prior_grid();
    launch_dependents();  // (what is launched next waits for the end of this before it reads results)
    static_assert(sizeof(sm.k) >= kMaxBatch * sizeof(uint2), "room for the entries' cost");
    const Start start = find_start<kTcRows, kTcThreads>(p, reinterpret_cast<uint2 *>(sm.k));  // (its barriers: the set-up is seen by all)
    tc_fence_after();
    if (p.d < DP && blockIdx.x < start.blocks) {  // columns that no copy writes
#pragma unroll 1
        for (int i = tid; i < (2 + 2 * kStages) * S::kTile / 16; i += kTcThreads) reinterpret_cast<uint4 *>(sm.q)[i] = make_uint4(0, 0, 0, 0);
    }
    fence_proxy_async();  // (what has been written where bulk copies will write)
    __syncthreads();
    const uint32_t tmem = __shfl_sync(~0u, sm.tmem, 0);

    volatile int *abort = &sm.abort;
    const auto wait = [&](const uint64_t &b, uint32_t parity) { return mbar_try_wait(smem_u32(&b), parity) || wait_long(smem_u32(&b), parity, &sm.abort); };

    if (blockIdx.x >= start.blocks) {
    } else if (warp < kSoftmaxWarps) {
        // ------------------------------------------------------------------ softmax and results
        const int team = warp >> 2, r = tid & 127;  // row: the lane of tensor memory
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, tS = tmem + lanes + kTmemS + team * kTcKeys, tO = tmem + lanes + kTmemO + team * 128;
        const uint64_t scale2 = pack_f32x2(p.scale_log2, p.scale_log2);
        int c = 0, mine = 0, parts = 0, teams = 0, boths = 0;  // tiles with keys, and the team's; parts; barriers passed
        const auto sync = [&](const uint64_t &b, int &passed) {  // (bounded like the other waits)
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(b));
            return wait(b, passed++ & 1);
        };
        int want_row = 0, want_col = 0, below = 0, member = 0, tiles = 0, own = 0;  // tiles of the part; the team's
        bool live = false;
        float m = -INFINITY;
        uint64_t sum[2] = {0, 0};
#pragma unroll 1
        for (int t = 0;; ++t) {
            const Meta &meta = sm.meta[t % kMetas];
            if (!wait(sm.meta_full[t % kMetas], t / kMetas & 1)) break;
            const int n = meta.n, qb = parts & 1;
            if (n < 0) break;
            const Part &part = sm.part[qb];
            if (meta.first) {
                if (!wait(sm.q_full[qb], parts / 2 & 1)) break;
                const Rows<kTcRows> &rows = sm.rows[qb];
                want_row = rows.want_row[r], want_col = rows.want_col[r], below = rows.below[r];
                live = (warp & 3) * 32 < part.n_rows;
                member = member_of<kTcRows>(p, part, r);
                tiles = own = 0;
                m = -INFINITY;
                sum[0] = sum[1] = 0;
            }
            const bool last = meta.last;
            if (n > 0 && (c & 1) == team) {
                const bool plain = meta.plain == 0x01010101u;
                // (S is there, so the P V of the team's tile before, whose place it has, is done)
                if (!wait(sm.s_full[team], mine & 1)) break;
                tc_fence_after();
                const int stage = c % kStages;
                bool odd = false;
                if (!plain || meta.ranged) {  // a weight 0 does not undo a value that is not a number: is there one?
                    if (!wait(sm.v_full[stage], c / kStages & 1)) break;
                    __nv_bfloat162 z = __floats2bfloat162_rn(0.f, 0.f);
                    const uint4 *v = reinterpret_cast<const uint4 *>(sm.v[stage]);
#pragma unroll 4
                    for (int i = r; i < kHalves * kTcKeys * 8; i += 128) {
                        const uint4 y = (i >> 3 & (kTcKeys - 1)) < n ? v[i] : make_uint4(0, 0, 0, 0);
                        for (uint32_t w : {y.x, y.y, y.z, y.w})
                            z = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&w), __floats2bfloat162_rn(0.f, 0.f), z);
                    }
                    if (__any_sync(~0u, !(__low2float(z) == 0.f && __high2float(z) == 0.f)) && lane == 0) *(volatile int *)&sm.odd[team] = c + 1;
                    if (!sync(sm.team[team], teams)) break;
                    odd = *(volatile int *)&sm.odd[team] == c + 1;
                }
                // the row's keys: none, where the row attends nothing
                const int m_at = min(member, kTcRows - 1), lo = meta.ranged ? meta.lo[m_at] : 0, hi = below < -1 ? 0 : meta.ranged ? meta.hi[m_at] : n;
                if (live) {
                    const bool any = __any_sync(~0u, lo < hi);
                    const int all_lo = __reduce_max_sync(~0u, lo), all_hi = __reduce_min_sync(~0u, hi);  // keys of all rows
                    float top = -INFINITY;
#pragma unroll 1
                    for (int c0 = 0; any && c0 < n; c0 += 32) {
                        uint32_t v[32];
                        tmem_ld32(tS + c0, v);
                        tc_wait_ld();
                        reg_fence(v);
                        if (!plain || c0 < all_lo || c0 + 32 > all_hi) {
                            const uint32_t on = (hi - c0 >= 32 ? ~0u : hi > c0 ? (1u << (hi - c0)) - 1 : 0u) & ~(lo - c0 >= 32 ? ~0u : lo > c0 ? (1u << (lo - c0)) - 1 : 0u);
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (!(on >> e & 1)) v[e] = 0xff800000u;
                            if (!plain) mask_scores(v, meta, c0, want_row, want_col, below);
                            tmem_st32(tS + c0, v);
                            tc_wait_st();
                        }
                        top = top_score(v, top);
                    }
                    // The base of a row moves when a score exceeds it by kRescale, and with the row's first score.
                    top *= p.scale_log2;
                    const bool moves = top > m + kRescale;
                    if (__any_sync(~0u, moves) || own == 0) {
                        const float keep = moves ? ex2(m - top) : 1.f;
                        if (moves) m = top;
                        const uint64_t keep2 = pack_f32x2(keep, keep);
                        sum[0] = mul_f32x2(sum[0], keep2), sum[1] = mul_f32x2(sum[1], keep2);
#pragma unroll 1
                        for (int i = 0; i < DP; i += 16) {
                            uint32_t o[16] = {};
                            if (own > 0) {
                                tmem_ld16(tO + i, o);
                                tc_wait_ld();
                                reg_fence(o);
                            }
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * keep);
                            tmem_st16(tO + i, o);
                        }
                    }
                    const float neg = m == -INFINITY ? 0.f : -m;
                    const uint64_t neg2 = pack_f32x2(neg, neg);
#pragma unroll 1
                    for (int c0 = 0; c0 < n; c0 += 32) {
                        uint32_t v[32] = {};
                        if (any) {
                            tmem_ld32(tS + c0, v);
                            tc_wait_ld();
                            reg_fence(v);
                            weigh(v, scale2, neg2, sum);
                        }
                        tmem_st32(tS + c0, v);
                    }
                    tc_wait_st();
                }
                if (odd) {
                    // Values that are not numbers: added here to the rows that attend them, and taken out of the tile.
                    const auto at = [&](int key, int e) {
                        return reinterpret_cast<__nv_bfloat16 *>(sm.v[stage] + e / 64 * S::kHalf + key * 128 + ((e / 8 & 7) ^ (key & 7)) * 16 + e % 8 * 2);
                    };
#pragma unroll 1
                    for (int key = 0; key < n && live; ++key) {
                        const bool counts = key >= lo && key < hi && attends(want_row, want_col, below, meta.place[key], meta.row[key], meta.col[key]);
#pragma unroll 1
                        for (int e = 0; e < DP; ++e) {
                            const float y = __bfloat162float(*at(key, e));
                            if (fabsf(y) < INFINITY) continue;
                            const uint32_t col = tS + key / 16 * 16 + key % 16 / 2, hi = tmem_ld1(col), lo = tmem_ld1(col + 8);
                            const uint32_t cut = key & 1 ? 0xffff0000u : 0xffffu, up = key & 1 ? 0 : 16;
                            const float w = __uint_as_float((hi & cut) << up) + __uint_as_float((lo & cut) << up);
                            const float o = __uint_as_float(tmem_ld1(tO + e));
                            tmem_st1(tO + e, __float_as_uint(counts ? fmaf(w, y, o) : o));
                            tc_wait_st();
                        }
                    }
                    if (!sync(sm.team[team], teams)) break;
#pragma unroll 1
                    for (int i = r; i < n * DP; i += 128) {
                        __nv_bfloat16 *y = at(i / DP, i % DP);
                        if (!(fabsf(__bfloat162float(*y)) < INFINITY)) *y = __float2bfloat16_rn(0.f);
                    }
                    fence_proxy_async();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(sm.p_full[team]));
                ++mine, ++own;
            }
            tiles += n > 0, c += n > 0;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sm.meta_empty[t % kMetas]));
            if (!last) continue;

            // The part is done: by both teams, half of the columns each, if it had more than one tile, else by the one that had it (the first
            // team, if it had none).
            const bool joined = tiles > 1;
            if (joined || own > 0 || (tiles == 0 && team == 0)) {
                float a, b;
                unpack_f32x2(add_f32x2(sum[0], sum[1]), a, b);
                float l = a + b, f[2] = {1.f, 1.f};
                if (own > 0 && !wait(sm.pv_done[team], (mine - 1) & 1)) break;
                if (joined) {
                    sm.stats[team][r] = make_float2(m, l);
                    if (!sync(sm.both, boths)) break;
                    const float2 x = sm.stats[0][r], y = sm.stats[1][r];
                    m = fmaxf(x.x, y.x);
                    const float base = m == -INFINITY ? 0.f : m;
                    f[0] = ex2(x.x - base), f[1] = ex2(y.x - base);
                    l = fmaf(x.y, f[0], y.y * f[1]);
                }
                tc_fence_after();
                const int state = part_state(part), slot = parts == 0 ? 0 : 1;
                const size_t whole = (size_t)part.seg * p.B * p.heads + row_of<kTcRows>(p, part, r, member);
                float *to = p.parts + (size_t)(2 * blockIdx.x + slot) * part_floats(kTcRows, p.d);
                if (live) {
                    const bool row = r < part.n_rows;
                    const int col0 = joined ? team * (DP / 2) : 0, col1 = joined ? col0 + DP / 2 : DP;
                    const int y_step = state == kAll ? 1 : kTcRows;
                    float4 *y = state == kAll ? reinterpret_cast<float4 *>(p.whole + whole * p.d + col0) : reinterpret_cast<float4 *>(to) + col0 / 4 * kTcRows + r;
#pragma unroll 1
                    for (int col = col0; col < col1; col += 16) {
                        uint32_t o[16], o2[16] = {};
                        tmem_ld16(tmem + lanes + kTmemO + (joined ? 0 : team * 128) + col, o);
                        if (joined) tmem_ld16(tmem + lanes + kTmemO + 128 + col, o2);
                        tc_wait_ld();
                        reg_fence(o);
                        reg_fence(o2);
                        if (!row) continue;
                        float x[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            x[e] = __uint_as_float(o[e]) * f[0];
                            if (joined) x[e] = fmaf(__uint_as_float(o2[e]), f[1], x[e]);
                            if (l == 0.f) x[e] = 0.f;
                        }
#pragma unroll
                        for (int e = 0; e < 16; e += 8) {
                            if (col + e >= p.d) break;
                            y[0] = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]), y[y_step] = make_float4(x[e + 4], x[e + 5], x[e + 6], x[e + 7]);
                            y += 2 * y_step;
                        }
                    }
                    if (row && (!joined || team == 0))
                        (state == kAll ? p.whole_stats[whole] : reinterpret_cast<float2 *>(to + (size_t)p.d * kTcRows)[r]) = make_float2(m, l);
                }
                if (r == 0 && (!joined || team == 0) && state != kGoesOn) {
                    Joint *joint = joint_of(p, part.seg, part.kv, part.seg == 0 ? part.b : part.b / p.pack, part.tile);
                    if (state == kAll)
                        joint->slot = -1;
                    else
                        *joint = joint_from(part, start, slot);
                }
                tc_fence_before();
                if (joined && !sync(sm.both, boths)) break;  // O has been read
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sm.q_empty[qb]));
            ++parts;
        }
    } else if (warp < kCopyWarp0) {
        // ------------------------------------------------------------------ queries, and which keys are read
        // (These warps meet at barriers: they leave together, when one of them says there that a wait of its own has failed.)
        const int lt = tid - 32 * kLoadWarp0, lw = warp - kLoadWarp0;
        Scout<kTcRows> scout = {p, sm.scout, lt};
        scout.start(start);
        bool ok = true;
        int t = 0;
        Part part;
#pragma unroll 1
        for (int parts = 0; scout.next_part(part); ++parts) {
            const int qb = parts & 1;
            if (parts >= 2) ok &= wait(sm.q_empty[qb], (parts / 2 - 1) & 1);
            if (any_scout(!ok)) break;
            const uint32_t q = smem_u32(sm.q[qb]);
            const int chunk = lane % kPer, sub = lane / kPer, n_here = min(part.n_rows - 32 * lw, 32);  // the warp's rows
            const int member = member_of<kTcRows>(p, part, lt), head = part.kv * p.group + part.tile * kTcRows + lt - member * p.group;
            const int64_t mine = (part.b + member) * p.q_batch + head * p.q_head;  // where the thread's row is
#pragma unroll 4
            for (int i = 0; i < n_here; i += kRowsOfCopy) {
                const int64_t from = __shfl_sync(~0u, mine, i + sub);
                if (i + sub < n_here && chunk < p.d / 8) cp_async16(S::place(q, 32 * lw + i + sub, chunk), (const __nv_bfloat16 *)p.Q + from + chunk * 8);
            }
            __syncwarp();
            scout.begin(part, sm.rows[qb]);
            if (lt == 0) sm.part[qb] = part;
            if (p.flip) {  // a negative scale: its sign goes to the queries
                asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll 1
                for (int i = sub; i < n_here; i += kRowsOfCopy) {
                    uint4 *x = reinterpret_cast<uint4 *>(sm.q[qb] + (S::place(q, 32 * lw + i, chunk) - q));
                    constexpr uint32_t kSigns = 0x80008000u;
                    *x = make_uint4(x->x ^ kSigns, x->y ^ kSigns, x->z ^ kSigns, x->w ^ kSigns);
                }
                __syncwarp();
            }
            cp_async_arrive(bar(sm.q_full[qb]));
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sm.q_full[qb]));
            bool last = false;
#pragma unroll 1
            for (bool first = true; !last; first = false, ++t) {
#pragma unroll 1
                while (scout.pending < kTcKeys && scout.more()) scout.look();
                const int n = min(scout.pending, kTcKeys);
                last = scout.pending <= kTcKeys && !scout.more();
                if (t >= kMetas) ok &= wait(sm.meta_empty[t % kMetas], (t / kMetas - 1) & 1);
                Meta &meta = sm.meta[t % kMetas];
                if (ok) meta.lo[lt] = meta.hi[lt] = 0;
                if (any_scout(!ok)) break;
                Key key = {0, INT32_MAX, kNever + 1, kNever + 1};  // nobody's
                bool plain = true;
                if (lt < n) {
                    key = scout.key(lt);
                    const int of = scout.owner_of_key(lt);
                    plain = scout.is_plain(key, of);
                    if (part.seg == 1) {
                        if (lt == 0 || scout.owner_of_key(lt - 1) != of) meta.lo[of] = (uint8_t)lt;
                        if (lt == n - 1 || scout.owner_of_key(lt + 1) != of) meta.hi[of] = (uint8_t)(lt + 1);
                    }
                }
                meta.place[lt] = key.place, meta.row[lt] = key.row, meta.col[lt] = key.col, meta.at[lt] = key.at;
                plain = __all_sync(~0u, plain);
                if (lane == 0) reinterpret_cast<uint8_t *>(&meta.plain)[lw] = plain;
                const unsigned before = __shfl_up_sync(~0u, key.at, 1);
                const unsigned follows = __ballot_sync(~0u, lt < n && ((lt & (maps.run - 1)) == 0 || key.at == before + p.slot16));
                // (a lane to each of the warp's blocks)
                const bool whole = maps.run && lane < 32 >> maps.run_log2 && __popc(follows >> (lane << maps.run_log2) << (32 - maps.run)) == maps.run;
                const unsigned runs = __ballot_sync(~0u, whole);
                if (lane == 0) meta.runs[lw] = (uint8_t)runs;
                if (lt == 0) meta.n = n, meta.first = first, meta.last = last, meta.ranged = part.seg;
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(sm.meta_full[t % kMetas]));
                scout.taken(n);
            }
            if (!last) break;
        }
        // behind the last one
        if (t >= kMetas) ok &= wait(sm.meta_empty[t % kMetas], (t / kMetas - 1) & 1);
        if (lt == 0) sm.meta[t % kMetas].n = -1;
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(sm.meta_full[t % kMetas]));
        if (scout.bad) atomicOr(p.cache.status, kCacheBad);
    } else if (warp < kMmaWarp) {
        // ------------------------------------------------------------------ copies of keys and values
        const int chunk = lane % kPer, first = (warp - kCopyWarp0) * kRowsOfCopy + lane / kPer;
        const bool copies = chunk < p.d / 8;
        bool ok = true;
#pragma unroll 1
        for (int t = 0, c = 0; ok; ++t) {
            const Meta &meta = sm.meta[t % kMetas];
            if (!wait(sm.meta_full[t % kMetas], t / kMetas & 1)) break;
            const int n = meta.n;
            if (n < 0) break;
            const int stage = c % kStages, rows16 = (n + 15) & ~15, per32 = 32 >> maps.run_log2;
            // the tile's blocks of rows that are copied whole: a bit each, and to every lane of the first warp a block and half of its columns
            const uint32_t runs = maps.run ? meta.runs[0] | meta.runs[1] << per32 | meta.runs[2] << 2 * per32 | meta.runs[3] << 3 * per32 : 0u;
            const int block = lane / kHalves, x = lane % kHalves * 64;
            const bool whole = block < 4 * per32 && (runs >> block & 1);
            const unsigned at0 = whole ? meta.at[block * maps.run] : 0;
            const int bytes = __popc(runs) * kHalves * 128 * maps.run;
            const bool rest = __popc(runs) * maps.run < rows16;
#pragma unroll 1
            for (int kv = 0; kv < 2 && n > 0; ++kv) {
                const uint64_t &full = kv ? sm.v_full[stage] : sm.k_full[stage], &empty = kv ? sm.v_empty[stage] : sm.k_empty[stage];
                if (c >= kStages && !(ok = wait(empty, (c / kStages - 1) & 1))) break;
                const uint32_t tile = smem_u32(kv ? sm.v[stage] : sm.k[stage]);
                const char *from = (const char *)(kv ? p.cache.v : p.cache.k) + chunk * 16;
                if (warp == kCopyWarp0 && whole)
                    tma_load_2d(tile + lane % kHalves * S::kHalf + block * maps.run * 128, kv ? &maps.v : &maps.k, (int)(at0 % p.slot16) * 8 + x,
                                (int)(at0 / p.slot16), bar(full));
                __syncwarp();
                // (places ahead of the copies: a load behind a copy waits its turn, 34 clk per copy instead of 10)
                constexpr int kStep = kCopyWarps * kRowsOfCopy, kBatch = 8;
#pragma unroll 1
                for (int row0 = first; rest && row0 < rows16; row0 += kBatch * kStep) {
                    unsigned at[kBatch];
#pragma unroll
                    for (int i = 0; i < kBatch; ++i) at[i] = meta.at[min(row0 + i * kStep, kTcKeys - 1)];
#pragma unroll
                    for (int i = 0; i < kBatch; ++i) {
                        const int row = row0 + i * kStep;
                        if (copies && row < rows16 && !(runs >> (row >> maps.run_log2) & 1))
                            cp_async16_or_zero(S::place(tile, row, chunk), from + (size_t)at[i] * 16, row < n);
                    }
                }
                __syncwarp();
                cp_async_arrive(bar(full));
                __syncwarp();
                if (lane == 0) mbar_arrive_expect_tx(bar(full), warp == kCopyWarp0 ? bytes : 0);  // (behind all that the warp has asked for)
            }
            c += n > 0;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sm.meta_empty[t % kMetas]));
        }
    } else {
        // ------------------------------------------------------------------ the products
        // S = Q K^T of a tile as soon as its keys are there and the team's last P V is done; O += P V as soon as P is there.
        const bool leader = elect_one();
        int t = 0, parts = 0;     // tile that comes next
        int cs = 0, cp = 0;       // tiles whose S, and whose P V, have been issued
        int n_even = 0, n_odd = 0, n = 0, first = 0, last = 0;  // keys of the teams' tiles; the tile that comes next
        bool known = false, end = false;
        uint32_t idle = 0;
        const auto is = [&](const uint64_t &b, uint32_t parity) { return mbar_test_wait(smem_u32(&b), parity); };
#pragma unroll 1
        while (!end || cp < cs) {
            bool moved = false;
            if (!end && !known && is(sm.meta_full[t % kMetas], t / kMetas & 1)) {
                known = moved = true;
                const Meta &meta = sm.meta[t % kMetas];
                n = meta.n, first = meta.first, last = meta.last;
                end = n < 0;
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(sm.meta_empty[t % kMetas]));
            }
            const int stage = cs % kStages, team = cs & 1;
            if (known && !end && (n == 0 || (is(sm.k_full[stage], cs / kStages & 1) && (!first || is(sm.q_full[parts & 1], parts / 2 & 1)) &&
                                             (cs < 2 || is(sm.pv_done[team], (cs / 2 - 1) & 1))))) {
                if (n > 0) {
                    fence_proxy_async();  // the copies of 16 bytes come through the generic proxy
                    tc_fence_after();
                    const uint32_t idesc = idesc_bf16(kTcRows, (n + 15) & ~15, 0, 0), tS = tmem + kTmemS + team * kTcKeys;
                    const uint32_t q = smem_desc_lo(smem_u32(sm.q[parts & 1])), k = smem_desc_lo(smem_u32(sm.k[stage]));
                    if (leader) {
                        mma_ss_lean<0>(tS, q, k, idesc);
#pragma unroll
                        for (int i = 1; i < DP / 16; ++i) {
                            const uint32_t off = i / 4 * (S::kHalf >> 4) + i % 4 * 2;
                            mma_ss_lean<1>(tS, q + off, k + off, idesc);
                        }
                        mma_commit(bar(sm.s_full[team]));
                        mma_commit(bar(sm.k_empty[stage]));
                    }
                    (team ? n_odd : n_even) = n;
                    ++cs;
                }
                if (last) {
                    if (leader) mma_commit(bar(sm.q_empty[parts & 1]));
                    ++parts;
                }
                __syncwarp();
                ++t;
                known = false;
                moved = true;
            }
            if (cp < cs && is(sm.p_full[cp & 1], cp / 2 & 1) && is(sm.v_full[cp % kStages], cp / kStages & 1)) {
                tc_fence_after();
                fence_proxy_async();
                const int from = cp % kStages, steps = ((cp & 1 ? n_odd : n_even) + 15) / 16;
                const uint32_t idesc = idesc_bf16(kTcRows, 64, 0, 1), v = smem_desc_lo(smem_u32(sm.v[from]));
                const uint32_t tO = tmem + kTmemO + (cp & 1) * 128, tP = tmem + kTmemS + (cp & 1) * kTcKeys;
                if (leader) {
#pragma unroll 1
                    for (int ks = 0; ks < steps; ++ks)
#pragma unroll
                        for (int h = 0; h < kHalves; ++h) {
                            const uint32_t b = v + ks * (16 * 128 >> 4) + h * (S::kHalf >> 4);
                            mma_ts_lean<1>(tO + 64 * h, tP + 16 * ks, b, idesc);
                            mma_ts_lean<1>(tO + 64 * h, tP + 16 * ks + 8, b, idesc);
                        }
                    mma_commit(bar(sm.pv_done[cp & 1]));
                    mma_commit(bar(sm.v_empty[from]));
                }
                __syncwarp();
                ++cp;
                moved = true;
            }
            if (moved) {
                idle = 0;
            } else if (*abort) {
                break;
            } else if (++idle > 1u << 18) {  // (some 20 ms)
                *abort = 1;
            }
        }
        if (leader) mma_commit(bar(sm.final_));  // nothing of this block may still run on the tensor pipe when its memory is freed
        __syncwarp();
        mbar_wait_bounded(bar(sm.final_), 0, kWaitLimit);
    }
    if (*abort)  // copies may still be on their way to shared memory: they take a few microseconds
        for (int i = 0; i < 50; ++i) __nanosleep(1000);
    tc_fence_before();
    __syncthreads();
    if (tid == 0 && *abort) atomicOr(p.cache.status, kCacheTimeout);
    if (warp == kMmaWarp) tmem_dealloc(tmem, kTmemCols);
}

// ---- the results of a row put together

// grid: (eight rows of a kv head, 16 columns); a lane has a row and four columns, the warps take a row's results in turn.
constexpr int kJoinRows = 8, kJoinWarps = 4;
template <typename T, int RT>
__global__ void __launch_bounds__(32 * kJoinWarps) shared_join_kernel(const __grid_constant__ SharedParams p) {
    __shared__ float4 s_sum[kJoinWarps][32];
    __shared__ float2 s_stat[kJoinWarps][32];
    ptx::launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int per_kv = (p.B * p.group + kJoinRows - 1) / kJoinRows, kv = blockIdx.x / per_kv;
    const int at = (blockIdx.x - kv * per_kv) * kJoinRows + lane % kJoinRows, c4 = blockIdx.y * 4 + lane / kJoinRows;
    const int b = at / p.group, g = at - b * p.group;
    const bool exists = b < p.B && c4 * 4 < p.d;
    // the results: of the shared tokens, and of the own ones
    const float *value[2];
    const float2 *stat[2];
    int64_t step[2];        // from one of them to the next, in floats
    int64_t from_first[2];  // from the first one to where the steps are counted from: its slot may be another than the next ones'
    int parts[2] = {0, 0};
    const size_t out = (size_t)b * p.heads + kv * p.group + g;
    // (the batch is looked at ahead of the wait: the kernel in front of this one has waited for whoever wrote it before it let this one start)
    Entry e;
    entry_of(p, min(b, p.B - 1), &e);
    ptx::wait_prior_grid();
    if (exists) {
#pragma unroll
        for (int seg = 0; seg < 2; ++seg) {
            if (seg == 0 && e.count == 0) continue;
            const int row = (seg == 0 ? b - e.first : b % p.pack) * p.group + g, r = row % RT;
            const Joint joint = *joint_of(p, seg, kv, seg == 0 ? e.first : b / p.pack, row / RT);
            if (joint.slot < 0) {
                const size_t whole = (size_t)seg * p.B * p.heads + out;
                value[seg] = p.whole + whole * p.d + c4 * 4, stat[seg] = p.whole_stats + whole;
                step[seg] = from_first[seg] = 0;
                parts[seg] = 1;
            } else {
                const float *from = p.parts + 2 * joint.first * part_floats(RT, p.d);
                value[seg] = from + (size_t)(c4 * RT + r) * 4;
                stat[seg] = reinterpret_cast<const float2 *>(from + (size_t)p.d * RT) + r;
                step[seg] = 2 * part_floats(RT, p.d), from_first[seg] = joint.slot * part_floats(RT, p.d);
                parts[seg] = joint.last - joint.first + 1;
            }
        }
    }
    float m = -INFINITY, l = 0.f;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    {
#pragma unroll
        for (int seg = 0; seg < 2; ++seg) {
            for (int i = warp; i < parts[seg]; i += kJoinWarps) {
                const int64_t off = i == 0 ? from_first[seg] : i * step[seg];
                const float2 s = *(stat[seg] + off / 2);
                const float4 v = *reinterpret_cast<const float4 *>(value[seg] + off);
                const float top = fmaxf(m, s.x), base = top == -INFINITY ? 0.f : top, keep = ptx::ex2(m - base), w = ptx::ex2(s.x - base);
                m = top;
                l = fmaf(l, keep, s.y * w);
                sum.x = fmaf(sum.x, keep, v.x * w), sum.y = fmaf(sum.y, keep, v.y * w);
                sum.z = fmaf(sum.z, keep, v.z * w), sum.w = fmaf(sum.w, keep, v.w * w);
            }
        }
    }
    s_sum[warp][lane] = sum, s_stat[warp][lane] = make_float2(m, l);
    __syncthreads();
    if (warp > 0 || !exists) return;
    for (int w = 0; w < kJoinWarps; ++w) m = fmaxf(m, s_stat[w][lane].x);
    const float base = m == -INFINITY ? 0.f : m;
    l = 0.f, sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int w = 0; w < kJoinWarps; ++w) {
        const float f = ptx::ex2(s_stat[w][lane].x - base);
        const float4 v = s_sum[w][lane];
        l = fmaf(f, s_stat[w][lane].y, l);
        sum.x = fmaf(f, v.x, sum.x), sum.y = fmaf(f, v.y, sum.y), sum.z = fmaf(f, v.z, sum.z), sum.w = fmaf(f, v.w, sum.w);
    }
    T *to = (T *)p.O + out * p.d + c4 * 4;
    put(l == 0.f ? 0.f : sum.x / l, to), put(l == 0.f ? 0.f : sum.y / l, to + 1);
    put(l == 0.f ? 0.f : sum.z / l, to + 2), put(l == 0.f ? 0.f : sum.w / l, to + 3);
    if (c4 == 0) p.LSE[out] = natural(m, l);
}

// ---- host

int rows_of_tile(const mate_cache_t *c) { return c->dtype == MATE_F32 ? kSimtRows : kTcRows; }
int pack_of(const mate_cache_t *c) { return std::max(1, rows_of_tile(c) / (c->heads / c->kv_heads)); }
int own_tiles(const mate_cache_t *c) { return (c->heads / c->kv_heads + rows_of_tile(c) - 1) / rows_of_tile(c); }
int n_blocks(const mate_cache_t *c) { return (c->dtype == MATE_F32 ? 2 : 1) * n_sms(c->device); }

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }
struct Workspace {
    size_t joints, stats, whole, parts, bytes;
};
Workspace workspace_of(const mate_cache_t *c, int B) {
    Workspace w = {};
    w.stats = align256(sizeof(Joint) * 2 * (size_t)c->kv_heads * B * own_tiles(c));
    w.whole = w.stats + align256(sizeof(float2) * 2 * (size_t)B * c->heads);
    w.parts = w.whole + align256(sizeof(float) * 2 * (size_t)B * c->heads * c->d);
    w.bytes = w.parts + sizeof(float) * 2 * (size_t)n_blocks(c) * part_floats(rows_of_tile(c), c->d);
    return w;
}

// Boxes of the highest of 8, 16 and 32 rows that a page is a whole number of, where the rows of all heads and pages lie in one such matrix and 64
// columns from a head's first on are its own, or behind the last one.
TcMaps maps_of(const SharedParams &p, const mate_cache_t *c) {
    TcMaps m = {};
    const int64_t slot = c->slot_stride, rows = slot > 0 ? ((int64_t)(c->pages - 1) * c->page_stride + (c->kv_heads - 1) * c->head_stride) / slot + c->page_size : 0;
    int run = 32;
    while (run > 8 && c->page_size % run != 0) run /= 2;
    bool fits = c->page_size % run == 0 && slot >= c->d && (c->pages == 1 || c->page_stride % slot == 0) && (slot == c->d || c->d % 64 == 0) && rows <= INT32_MAX;
    for (int h = 0; h < c->kv_heads && fits; ++h) fits = h * c->head_stride % slot + c->d <= slot;
    if (fits && make_box_map(&m.k, p.cache.k, (size_t)slot, (size_t)rows, (size_t)slot * 2, run) &&
        make_box_map(&m.v, p.cache.v, (size_t)slot, (size_t)rows, (size_t)slot * 2, run))
        m.run = run;
    for (m.run_log2 = 0; 1 << m.run_log2 < run;) ++m.run_log2;  // (without boxes too: the rows are looked at in blocks all the same)
    return m;
}

template <typename T, int DP>
int launch(const SharedParams &p, const mate_cache_t *cache, int blocks, cudaStream_t st) {
    constexpr bool kTc = sizeof(T) == 2;
    constexpr int kRows = kTc ? kTcRows : kSimtRows, kThreads = kTc ? kTcThreads : kSimtThreads;
    constexpr int kSmem = kTc ? 1024 + (int)sizeof(TcSmem<DP>) : (int)sizeof(SimtSmem<DP>);
    static_assert(kSmem <= 232448, "shared memory of a block");
    static SmemAttrOnce attr;
    cudaError_t e;
    if constexpr (kTc) {
        const int rc = attr.ensure((const void *)shared_tc_kernel<DP>, kSmem, cache->device);
        if (rc != MATE_OK) return rc;
        e = launch_after(shared_tc_kernel<DP>, dim3((unsigned)blocks), kThreads, kSmem, st, p, maps_of(p, cache));
    } else {
        const int rc = attr.ensure((const void *)shared_simt_kernel<DP>, kSmem, cache->device);
        if (rc != MATE_OK) return rc;
        e = launch_after(shared_simt_kernel<DP>, dim3((unsigned)blocks), kThreads, kSmem, st, p);
    }
    const int64_t joins = (int64_t)p.kv_heads * (((int64_t)p.B * p.group + kJoinRows - 1) / kJoinRows);
    if (e == cudaSuccess)
        e = launch_after(shared_join_kernel<T, kRows>, dim3((unsigned)joins, (unsigned)((p.d + 15) / 16)), 32 * kJoinWarps, 0, st, p);
    return e == cudaSuccess ? MATE_OK : MATE_ERR_CUDA;
}

}  // namespace
}  // namespace mate

using namespace mate;

extern "C" {

int mate_cache_shared_workspace_bytes(const mate_cache_t *cache, int n, size_t *bytes) {
    const int rc = check_cache(cache);
    if (rc != MATE_OK) return rc;
    if (n < 0 || !bytes) return MATE_ERR_INVALID_ARG;
    *bytes = n > 0 ? workspace_of(cache, n).bytes : 0;
    return MATE_OK;
}

int mate_attn_decode_shared(const mate_cache_t *cache, int layer, const void *Q, const int64_t *q_stride, int B, const int32_t *seqs,
                            const int32_t *row_ids, const int32_t *col_ids, const int32_t *groups, float scale, int max_len, void *O, float *LSE,
                            void *workspace, size_t workspace_bytes, void *stream) {
    int rc = check_cache(cache);
    if (rc != MATE_OK) return rc;
    if (layer < 0 || layer >= cache->layers || B < 0 || max_len < 0 || (!seqs && B > cache->seqs)) return MATE_ERR_INVALID_ARG;
    if (B > 0 && (!Q || !q_stride || !row_ids || !col_ids || !groups || !O || !LSE)) return MATE_ERR_INVALID_ARG;
    if (!std::isfinite(scale)) return MATE_ERR_INVALID_ARG;
    if (!std::isfinite(scale * kLog2e)) return MATE_ERR_UNSUPPORTED;  // (0 times what it would be is not a number)
    const int64_t reach = (cache->pages - 1) * cache->page_stride + (cache->kv_heads - 1) * cache->head_stride + (cache->page_size - 1) * cache->slot_stride;
    if (cache->heads > kMaxHeads || reach / (int64_t)(16 / elem_size(cache->dtype)) > UINT32_MAX) return MATE_ERR_UNSUPPORTED;
    const int vec = (int)(16 / elem_size(cache->dtype));
    if (B > 0 && (!is_aligned(Q, 16) || !is_aligned(O, 16) || !is_aligned(LSE, 4) || q_stride[0] % vec != 0 || q_stride[1] % vec != 0))
        return MATE_ERR_ALIGNMENT;
    if ((rc = check_cache_device(cache)) != MATE_OK) return rc;
    if (B == 0) return MATE_OK;
    const int most = cache->width * cache->page_size;
    if (max_len == 0 || max_len > most) max_len = most;
    // units of the batch, shared and own, are 32-bit numbers
    if (B > kMaxBatch || (int64_t)B * cache->kv_heads * own_tiles(cache) > INT32_MAX / 2 / (kOver + units_of(max_len))) return MATE_ERR_UNSUPPORTED;
    const Workspace w = workspace_of(cache, B);
    if (!workspace || workspace_bytes < w.bytes) return MATE_ERR_WORKSPACE;
    if (!is_aligned(workspace, 256)) return MATE_ERR_ALIGNMENT;
    SharedParams p = {};
    p.cache = cache_args(cache, layer);
    p.Q = Q, p.q_batch = q_stride[0], p.q_head = q_stride[1];
    p.B = B, p.heads = cache->heads, p.kv_heads = cache->kv_heads, p.group = cache->heads / cache->kv_heads;
    p.d = cache->d, p.max_len = max_len, p.pack = pack_of(cache), p.own_tiles = own_tiles(cache);
    p.seqs = seqs, p.row_ids = row_ids, p.col_ids = col_ids, p.groups = groups;
    p.scale_log2 = scale * kLog2e, p.O = O, p.LSE = LSE;
    for (int h = 0; h < cache->heads; ++h) p.views[h >> 4] |= (uint32_t)cache->head_view[h] << 2 * (h & 15);
    const auto quotients = [](int by, unsigned *mul, unsigned *shift) {
        for (*shift = 0; 1u << *shift < (unsigned)by;) ++*shift;
        *mul = (unsigned)((((uint64_t)1 << 32) * (((uint64_t)1 << *shift) - by)) / by + 1);
    };
    quotients(cache->page_size, &p.page_mul, &p.page_shift);
    quotients(p.group, &p.group_mul, &p.group_shift);
    p.page16 = (unsigned)(cache->page_stride / vec), p.head16 = (unsigned)(cache->head_stride / vec), p.slot16 = (unsigned)(cache->slot_stride / vec);
    char *ws = static_cast<char *>(workspace);
    p.joints = reinterpret_cast<Joint *>(ws + w.joints);
    p.whole_stats = reinterpret_cast<float2 *>(ws + w.stats);
    p.whole = reinterpret_cast<float *>(ws + w.whole);
    p.parts = reinterpret_cast<float *>(ws + w.parts);
    if (cache->dtype == MATE_BF16) {
        // a score of -inf stays one whatever it is multiplied by: a factor above 0, so small for a scale of 0 that every weight is 1
        p.flip = p.scale_log2 < 0.f;
        p.scale_log2 = std::fmax(std::fabs(p.scale_log2), 0x1p-126f);
    }
    cudaStream_t st = (cudaStream_t)stream;
    const int blocks = n_blocks(cache);
    if (cache->dtype == MATE_F32) return cache->d <= 64 ? launch<float, 64>(p, cache, blocks, st) : launch<float, 128>(p, cache, blocks, st);
    return cache->d <= 64 ? launch<__nv_bfloat16, 64>(p, cache, blocks, st) : launch<__nv_bfloat16, 128>(p, cache, blocks, st);
}

}  // extern "C"

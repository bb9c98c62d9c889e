// Attention of one new token per sequence where sequences share their first tokens (mate_attn_decode_shared): the shared keys and
// values of a group are read once for all of its sequences, whose query heads are the rows of one product,
//     S = Q K^T,  m = max S,  P = exp(S - m),  O = P V / sum P,  LSE = m + ln sum P
// per kv head over the shared tokens, the same over the sequences' own tokens behind them, and the two put together by their m and
// sum P.
//
// Work.  An item is a kv head and a tile of rows (128 with bf16, 64 with fp32) of a segment: a group's shared tokens, with the query heads of all of
// its sequences, or the own tokens of as many sequences as their heads fill a tile (reading 32 sequences of 4 heads by turns would be 32 tiles
// of 4 rows; together they are a few tiles of 128 keys, each of which is for the rows of one sequence).  Its length is counted in units of kUnit tokens,
// and kOver units stand for what an item costs whatever its length (8: 39.1 us for 64 questions, 101 for 256 sequences, 30.1 for beams; 4: 40.0, 102,
// 29.5; 16: 40.7, 102, 32.6).  Blocks, one to an SM, get equal shares of all items' units (found by every block from the lengths, which the host does
// not know): a long segment is spread over the GPU, short ones are put together.  What a block leaves of an item that is not a row's whole
// result -- m, sum P and the sum of values, in fp32 -- is joined by a second kernel, in the order of the tokens: the same bits on every
// launch.
//
// Tokens are looked through 256 at a time by their ids; those that no row of the tile attends are left out before anything of them is read.  Which
// row attends which of the rest is found once for all rows that go by the same ids (a bit per key), not by every row.
//
// Roles of a bf16 block.  Four warps look for keys (Scout) and fill tiles of 128 of them; two copy keys and values (sixteen slots that follow one
// another by a bulk tensor copy, the rest in 16 bytes a lane) and the queries; two teams of four warps, a thread to a row, take the tiles in turn and make
// weights of the scores; a warp for each team issues its products.  Tensor memory: O of both teams 2 x 128 columns, S 2 x 128; the weights take
// the place of the scores, 16 keys as 8 columns of bf16 pairs and 8 of what the rounding left.  (Weights as one bf16 would be off by 2^-8, as much as the
// result's rounding.)  fp32: shared_simt_kernel, 64 rows against 32 keys, no tensor cores.
//
// What is lost beside the rounding of the result to bf16 (half a step, 2e-3 to 4e-3 of it): a weight by its 16 bits 2^-16 at most, and the sums in
// tensor memory, which are cut off behind fp32's 24 bits, always towards 0, with every product: of 16 products a tile 64 questions and 256 sequences lose
// 1e-5 of a result, so that one in some 300 rounds to the other bf16; 65536 tokens of one block lose 5e-5 (values of mean 1: 1e-4;
// mate_attn_decode, whose warps have less of a sequence each, 2e-5 and 4e-5), one result in 40.  A third part for every weight, all of the 24 bits, has no
// room beside an O for each team with more than 64 elements.  With one O for both teams it has, but then three times as many products go into a
// sum: 65536 tokens lose 1.2e-4, one result in 18, and 256 sequences take 102 us.  Putting O by, sixteen columns a tile, ends the loss (one
// result in 400, however many tokens) and takes 113 to 121 us.  With 64 elements a third part takes beams from 30.1 to 32.6 us and cells from 43.0
// to 44.9, and no fewer results round to the other bf16.
//
// What bounds it.  The chain of a team's tile, 7.2 thousand cycles of which the other team's overlap half: S 0.5, weights 4 (four chunks of 32 keys, one
// after the other in a warp), P V 1.3, whose weights lie where the next S goes, barriers and the other team's tile 1.4; the products alone would
// take 1.6 a tile.  64 questions about 8192 tokens, 8 kv heads of 4 x 128: 39 us, of which start 10 (lengths and groups in two rounds of loads, pages, ids, then
// the first keys), tiles 18, joining and launches the rest.  Tiles of own keys take 5 thousand cycles each: V has to be looked through ahead of weights of 0
// (0.8), and copies of own runs are short.  Cells (a token attends a few hundred of 4096): looks, 1.1 thousand cycles per 256 tokens.  Measured and
// left out, with what they cost where the rest took 102 us for 256 sequences: chunks of 64 keys (109), S of one half of a tile while the other's weights
// are made (106), three tiles of values and one of queries (106), rows brought to L2 ahead of their copies (103); with 64 elements a third place for
// scores, so that S does not wait for P V (beams 29 -> 30).
//
// Where it is the wrong way: sequences without groups, or in groups of few rows, and own tokens by the thousand, whose tiles multiply 128 rows by keys that
// one sequence's heads count for; see alone_bytes.
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "mate_cache.h"
#include "sm100_ptx.cuh"
#include "tc_tiles.cuh"
#include "wait_together.h"

namespace mate {
// mate_decode.cu
size_t decode_workspace(const mate_cache_t *cache, int B);
int decode(const mate_cache_t *cache, int layer, const void *Q, const int64_t *q_stride, int B, const int32_t *seqs, const int32_t *row_ids,
           const int32_t *col_ids, const int32_t *groups, float scale, int max_len, void *O, float *LSE, void *workspace, size_t workspace_bytes,
           void *stream);
namespace {

constexpr int kUnit = 32;     // tokens of a unit of work: what a warp looks through in one go
constexpr int kOver = 8;      // units that an item costs besides its tokens
constexpr int kMaxBatch = 4096;
constexpr int kMaxHeads = 1024;
constexpr int kNever = INT32_MIN;  // an id that no token has
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Where the results of an item are: [slot] of the block that begins it, then [0] of the next ones up to the one that has the unit in front of
// `end`, of `total`.
struct Joint {
    int32_t slot, first;  // slot < 0: with the rows' whole results
    uint32_t end, total;
};

struct SharedParams {
    CacheArgs cache;
    const void *Q;
    int64_t q_batch, q_head;
    int B, heads, kv_heads, group, d, max_len;
    int own_quarter;  // a unit of own tokens costs a quarter more
    int pack, own_tiles;  // entries whose own tokens make an item (their rows fill a tile), or tiles of the rows of one
    const int32_t *seqs, *row_ids, *col_ids, *groups;
    float scale_log2;  // scale / ln 2: weights are powers of two
    int flip;          // tensor-core kernel: the scale above is positive, and the queries change their sign
    void *O;
    float *LSE;
    // A token's place: page * page_step + slot * slot_step + kv head * head_step, in rows of row16 times 16 bytes; its kv head begins
    // kv head * head16 times 16 bytes behind that.  No place is beyond 2^32 times 16 bytes.
    unsigned page_step, slot_step, head_step, row16, head16;
    // x / page_size and x / group by multiplication: (umulhi(x, mul) + x) >> shift for x < 2^31
    unsigned page_mul, page_shift, group_mul, group_shift;
    Joint *joints;                    // [2][kv_heads][B own_tiles]: shared tokens, by the first entry of the tile's group, and own ones
    float2 *whole_stats;              // [2][B heads]  m and sum P of rows whose item one block has done
    float *whole;                     // [2][B heads][d]
    uint8_t *grouped;                 // [B] whether an entry is in a group, for the kernel that joins
    float *parts;                     // [blocks][2]: values in groups of four by row, then the rows' m and sum P
    int blocks;                       // of the grid
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
// none: as find_start makes it, or null: whether groups have entries in common is not looked at.
// (called, not put in line: what a block runs through once misses the instruction cache, which holds 32 KB for all of its roles)
__device__ __noinline__ void entry_of(const SharedParams &p, int b, const uint32_t *none, Entry *to) {
    const int q_row = p.row_ids[b], q_col = p.col_ids[b];
    const GroupOf g = group_of(p.cache, p.seqs, p.groups, none && bit_of(none, b), p.B, b, p.max_len);
    Entry e = {g.s, g.len, 0, 0, g.count, g.first, g.shared, 0, q_row, q_col, g.prefix};
    const bool has = g.count > 0 && g.len >= g.shared, padding = q_row < 0 || q_col < 0 || g.s < 0;
    e.counts = has && !padding;
    e.own0 = has ? g.shared : 0;
    e.own1 = padding ? e.own0 : e.len;
    e.bad = g.bad;
    *to = e;
}
// Units of tokens.  The first kOver units of an item stand for what it costs whatever its length: none of its tokens belong to them.
__host__ __device__ __forceinline__ int units_of(int tokens) { return (tokens + kUnit - 1) / kUnit; }
// Items of the shared tokens of the group that entry b is the first of: kv heads and tiles of rows.
__device__ __forceinline__ bool leads(const Entry &e, int b) { return e.count > 0 && e.first == b; }
template <int RT>
__device__ __forceinline__ int group_tiles(const SharedParams &p, const Entry &e) {
    return (e.count * p.group + RT - 1) / RT;
}
// Units of an item of own tokens.  (Without any it has one: its rows have a result too.)
__device__ __forceinline__ int own_units(const SharedParams &p, int tokens_units) {
    return tokens_units > 0 ? kOver + tokens_units + (p.own_quarter ? (tokens_units + 3) / 4 : 0) : 1;
}

// Where a block begins: unit `in` of its first batch, for `left` units (0: there is nothing for it to do), the first of them number `at` of all.
struct Start {
    unsigned total, at, in;
    int left, batch;
};
// What the threads look up for it is kept for the first batch, as far as there is room.
constexpr int kKept = 208;
struct Found {
    uint2 cost[kMaxBatch];
    uint32_t begins[kMaxBatch / 32];  // a bit for each entry that begins a group
    Entry entries[kKept];
};
template <int RT>
__device__ __forceinline__ uint2 cost_of(const SharedParams &p, const Entry &e, int b) {
    return make_uint2(units_of(e.own1 - e.own0), leads(e, b) ? p.kv_heads * group_tiles<RT>(p, e) * (kOver + units_of(e.shared)) : 0);
}
// A group that another one begins inside of is none: otherwise two items would have the same rows, and two groups' tiles the same joint.  (Rarely called.)
template <int RT, int NT>
__device__ __noinline__ void leave_out(const SharedParams &p, Found &found, uint32_t *none) {
    uint2 *cost = found.cost;
    const int tid = threadIdx.x, lane = tid & 31;
#pragma unroll 1
    for (int b0 = tid & ~31; b0 < p.B; b0 += NT) {
        const int b = b0 + lane;
        const Claim c = b < p.B ? claim_of(p.groups, p.B, b) : Claim();
        const bool is = fits(c, b, p.B, p.max_len) && begins_inside(found.begins, c.first, c.count);
        const unsigned those = __ballot_sync(~0u, is);
        if (lane == 0) none[b0 >> 5] = those;
        __syncwarp();
        if (!is) continue;
        Entry mine, &e = b < kKept ? found.entries[b] : mine;
        entry_of(p, b, none, &e);
        cost[b] = cost_of<RT>(p, e, b);
        if (blockIdx.x == 0) p.grouped[b] = 0, atomicOr(p.cache.status, kCacheBad);
    }
}
// All threads call it, and each gets it.  `found`: in shared memory, free when the first batch has been taken over.  none: a bit for each entry
// whose group is none because another one begins inside it, there for as long as the block wants entries.
template <int RT, int NT>
__device__ Start find_start(const SharedParams &p, Found &found, uint32_t (&none)[kMaxBatch / 32]) {
    uint2 *cost = found.cost;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, batches = (p.B + p.pack - 1) / p.pack;
#pragma unroll 1
    for (int b0 = tid & ~31; b0 < p.B; b0 += NT) {
        const int b = b0 + lane;
        bool first = false;
        if (b < p.B) {
            Entry mine, &e = b < kKept ? found.entries[b] : mine;
            entry_of(p, b, nullptr, &e);
            cost[b] = cost_of<RT>(p, e, b), first = leads(e, b);
            if (blockIdx.x == 0) p.grouped[b] = e.count > 0;
            if (e.bad && blockIdx.x == 0) atomicOr(p.cache.status, kCacheBad);
        }
        const unsigned those = __ballot_sync(~0u, first);
        if (lane == 0) found.begins[b0 >> 5] = those, none[b0 >> 5] = 0;
    }
    __syncthreads();
    bool inside = false;
#pragma unroll 1
    for (int b = tid; b < p.B; b += NT)
        if (bit_of(found.begins, b)) inside |= begins_inside(found.begins, b, min(p.groups[p.B + b], p.B - b));
    if (__syncthreads_or(inside)) {
        leave_out<RT, NT>(p, found, none);
        __syncthreads();
    }
    // a warp to each batch; its cost replaces that of its first entry
#pragma unroll 1
    for (int i = warp; i < batches; i += NT / 32) {
        unsigned own = 0, shared = 0;
#pragma unroll 1
        for (int b = i * p.pack + lane; b < min(p.B, (i + 1) * p.pack); b += 32) own += cost[b].x, shared += cost[b].y;
        own = __reduce_add_sync(~0u, own), shared = __reduce_add_sync(~0u, shared);
        __syncwarp();
        if (lane == 0) cost[i * p.pack].x = shared + (unsigned)(p.kv_heads * p.own_tiles) * own_units(p, (int)own);
    }
    __syncthreads();
    // every warp for itself, 32 batches at a time: the sum of all, and then the one that has the block's first unit
    Start start = {};
#pragma unroll 1
    for (int i = lane; i < batches; i += 32) start.total += cost[i * p.pack].x;
    start.total = __reduce_add_sync(~0u, start.total);
    const unsigned blocks = min(start.total, (unsigned)p.blocks), i = blockIdx.x;
    if (i >= blocks) return start;
    const unsigned q = start.total / blocks, r = start.total - q * blocks;
    start.at = q * i + r * i / blocks, start.left = (int)(q * (i + 1) + r * (i + 1) / blocks - start.at);
    unsigned before = 0;
#pragma unroll 1
    for (int i0 = 0;; i0 += 32) {
        unsigned sum = i0 + lane < batches ? cost[(i0 + lane) * p.pack].x : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned y = __shfl_up_sync(~0u, sum, o);
            if (lane >= o) sum += y;
        }
        const unsigned behind = __ballot_sync(~0u, before + sum > start.at);
        if (behind) {
            const int k = __ffs(behind) - 1;
            const unsigned front = __shfl_sync(~0u, sum, max(k - 1, 0));
            start.batch = i0 + k, start.in = start.at - before - (k > 0 ? front : 0);
            return start;
        }
        before += __shfl_sync(~0u, sum, 31);
    }
}

// A part of an item.
struct Part {
    int b, seg, kv, tile;  // first entry; shared tokens (0) or own ones (1); tile of rows
    int from, to;          // its units of tokens
    int n_rows;
    int state;
    unsigned end;          // of the item's units, among those of all
};
enum { kAll, kBegins, kGoesOn };
// Of a row of the tile: its entry, counted from the part's first, and its place among all rows of the batch (there are fewer than 2^23).
template <int RT>
__device__ __forceinline__ int member_of(const SharedParams &p, const Part &part, int r) {
    return by_group(p, part.tile * RT + r);
}
template <int RT>
__device__ __forceinline__ int row_of(const SharedParams &p, const Part &part, int r, int member) {
    return (part.b + member) * p.heads + part.kv * p.group + part.tile * RT + r - member * p.group;
}
// (tiles of a group of n entries: n own_tiles at most, so those of different groups, which have no entry in common, have different places)
__device__ __forceinline__ Joint *joint_of(const SharedParams &p, int seg, int kv, int b, int tile) {
    return p.joints + ((size_t)seg * p.kv_heads + kv) * p.B * p.own_tiles + (size_t)b * p.own_tiles + tile;
}
__device__ __forceinline__ void put_joint(const SharedParams &p, const Part &part, int slot, unsigned total) {
    if (part.state == kGoesOn) return;
    *joint_of(p, part.seg, part.kv, part.seg == 0 ? part.b : part.b / p.pack, part.tile) = {part.state == kAll ? -1 : slot, (int)blockIdx.x, part.end, total};
}

// ---- who attends what

// A row attends a key if the key's place is below `below` (text keys stand at -1, those of the prefix where they stand; -2: the row attends
// nothing), or one of the ids is the one it wants.
__device__ __forceinline__ bool attends(int want_row, int want_col, int below, int place, int row, int col) {
    return place < below || row == want_row || col == want_col;
}
constexpr int kScouts = 128, kKinds = 4;
struct alignas(16) Wish {
    int row, col, below;
    int member;  // of own tokens: only those of this entry (of the batch) count
    __device__ bool is_for(const int place, const int of_row, const int of_col) const { return attends(row, col, below, place, of_row, of_col); }
};
// The rows of a tile,
template <int RT>
struct Rows {
    short kind[RT];  // place of a row's wish among those below, -1: it attends nothing
};
// and, as those who look for keys need them, without repetitions of the row before: the rows of a warp have 32 places of their own, up to a
// multiple of kKinds of them in use.
template <int RT>
struct Wishes {
    int least, most;  // of `below` over the rows that are there
    int views;        // 1: some want a row, 2: a column
    uint8_t n[kScouts / 32];
    Wish kind[kScouts];
    __device__ void clear() { least = INT32_MAX, most = INT32_MIN, views = 0; }
};
// Keys, with what the rows go by.
struct alignas(16) Key {
    unsigned at;  // where it lies: see SharedParams
    int place, row, col;
};
constexpr int kList = 512;
constexpr unsigned kNowhere = ~0u;
__device__ __forceinline__ Key nobody() { return {kNowhere, INT32_MAX, kNever + 1, kNever + 1}; }  // a key that no row attends
constexpr int kUnits = 8;  // of a look

// kScouts threads walk the parts of the block's share and look through their tokens, eight units at a time, two to a warp; the keys that
// count go onto a list.  The next ones' ids, and the pages of the ones behind them, are on their way meanwhile.  Barrier 1 is theirs.
//
// Units of own tokens are numbered through over the entries of the batch, each entry beginning with a new one.
template <int RT>
struct ScoutSmem {
    Entry entries[kScouts];  // of the batch
    int before[kScouts + 1]; // units of own tokens in front of an entry's
    unsigned leaders[4];     // a bit for each entry: it is the first of a group
    uint32_t none[kMaxBatch / 32];  // of all entries there are: see find_start
    Wishes<RT> wishes[2];    // of the parts in turn
    Key list[kList];         // what look() writes is seen behind the next barrier
    uint8_t owners[kList];   // entries of the batch
    int counts[2][8];        // of the units' keys; plus kDense
};
constexpr int kDense = 64, kNobody = 255, kRun = 16;
constexpr int kLooked = kUnits * (kUnit + kRun - 1);  // what a look may add to the list, at most
// Where the loads of a look stand.
struct Asked {
    int j, owner, page;
    bool there, first;  // first: the entry's first unit
};
template <int RT>
struct Scout {
    const SharedParams &p;
    ScoutSmem<RT> &sm;
    int tid, run;  // run: keys that lie one behind the other are copied by that many, kRun or 1
    // the walk: next item of the share
    int batch, entry, tiles, n_units, item, u;  // entry: that leads (of the batch), kScouts: own tokens; tiles of rows, units of an item of it
    unsigned in, at_unit;                       // units to pass over yet; number of the next one among those of all
    int left;                                   // units of the share
    int held, parts;                            // batch that is in shared memory; parts so far
    // the looks at the present part
    int seg, next, end, pending, list_at, looks;  // next, end: units
    unsigned head_at;
    Asked asked[2];
    struct {
        unsigned at;
        int j, owner, row, col;
        bool there, first;
    } got[2];
    int leader, shared_end;
    bool bad;

    __device__ static void sync() { asm volatile("barrier.cta.sync 1, 128;" ::: "memory"); }
    __device__ int entries() const { return min(p.pack, p.B - batch * p.pack); }
    __device__ void hold(const Entry *found) {
        held = batch;
        sync();
        int units = 0;
        bool first = false;
        if (tid < entries()) {
            const int b = batch * p.pack + tid;
            if (found && b < kKept)
                sm.entries[tid] = found[b];
            else
                entry_of(p, b, sm.none, sm.entries + tid);
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
    __device__ bool is_leader(int i) const { return sm.leaders[i >> 5] >> (i & 31) & 1; }
    // The first entry from `entry` on that leads a group, kScouts if there is none.
    __device__ int leader_from(int from) const {
        for (int w = from >> 5; w < 4; ++w) {
            const unsigned those = sm.leaders[w] & (w == from >> 5 ? ~0u << (from & 31) : ~0u);
            if (those) return 32 * w + __ffs(those) - 1;
        }
        return kScouts;
    }
    __device__ void start(const Start &from, const Found &found) {
        batch = from.batch, in = from.in, at_unit = from.at, left = from.left;
        parts = looks = item = u = tiles = n_units = 0, entry = -1, bad = false;
        if (tid == 0) sm.wishes[0].clear();
        hold(found.entries);
        // the leader whose items `in` is among: its number less one, with what is left of `in` there
        const unsigned cost = is_leader(tid) ? (unsigned)(p.kv_heads * group_tiles<RT>(p, sm.entries[tid])) * (kOver + units_of(sm.entries[tid].shared)) : 0;
        unsigned sum = cost;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned y = __shfl_up_sync(~0u, sum, o);
            if ((tid & 31) >= o) sum += y;
        }
        if ((tid & 31) == 31) sm.counts[1][tid >> 5] = (int)sum;
        sync();
        for (int w = 0; w < tid >> 5; ++w) sum += (unsigned)sm.counts[1][w];
        if (sum - cost <= in && in < sum) sm.counts[0][0] = tid, sm.counts[0][1] = (int)(in - (sum - cost));
        if (tid == kScouts - 1 && sum <= in) sm.counts[0][0] = kScouts, sm.counts[0][1] = (int)(in - sum);
        sync();
        entry = sm.counts[0][0] - 1, in = (unsigned)sm.counts[0][1];
        sync();
    }
    // The next part of the share.  (It comes to an end whatever it finds: every part takes a unit off the share.)
    __device__ bool next_part(Part &part) {
#pragma unroll 1
        while (left > 0 && batch * p.pack < p.B) {
            if (held != batch) {
                hold(nullptr);
                entry = -1, tiles = item = 0;
            }
            if (item < p.kv_heads * tiles) {
                const int u1 = min(n_units, u + left);
                if (u1 <= kOver && u1 < n_units) break;  // it ends among the units that stand for the item: the next block takes it
                const int kv = item / tiles, tile = item - kv * tiles;
                const int rows = (entry < kScouts ? sm.entries[entry].count : entries()) * p.group;
                const int seg = entry < kScouts ? 0 : 1;
                const auto unit = [&](int cost) { return cost <= kOver ? 0 : seg && p.own_quarter ? cost - kOver - (cost - kOver + 4) / 5 : cost - kOver; };
                part = {batch * p.pack + (seg == 0 ? entry : 0), seg, kv, tile, unit(u), unit(u1),
                        min(RT, rows - tile * RT), u > 0 ? kGoesOn : u1 == n_units ? kAll : kBegins, at_unit - u + n_units};
                left -= max(1, u1 - u);
                at_unit += u1 - u;
                u = 0;
                ++item;
                return true;
            }
            if (entry == kScouts) {
                ++batch;
                continue;
            }
            entry = leader_from(entry + 1), item = 0;
            const bool group = entry < kScouts;
            tiles = group ? group_tiles<RT>(p, sm.entries[entry]) : p.own_tiles;
            n_units = group ? kOver + units_of(sm.entries[entry].shared) : own_units(p, sm.before[kScouts]);
            const unsigned all = (unsigned)(p.kv_heads * tiles) * n_units;
            if (in >= all) {
                in -= all, item = p.kv_heads * tiles;
            } else if (in > 0) {
                item = (int)(in / (unsigned)n_units), u = (int)(in - (unsigned)item * n_units), in = 0;
                if (u <= kOver) left += u, at_unit -= u, u = 0;
            }
        }
        left = 0;
        return false;
    }
    // Who the tokens of the warp's units from `unit` on belong to, and their pages.
    __device__ void ask_pages(int unit0) {
        const int lane = tid & 31;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int unit = unit0 + 2 * (tid >> 5) + k;
            Asked &a = asked[k];
            a = {0, 0, -1, false, false};
            if (unit >= end) continue;
            int first_token = 0, stop, from = 0;
            if (seg == 0) {
                a.owner = leader;
                stop = shared_end;
            } else {
                int n = 0;  // entries that begin at the unit or in front of it
#pragma unroll
                for (int i = 0; i < kScouts / 32; ++i) n += sm.before[32 * i + lane] <= unit;
                a.owner = __reduce_add_sync(~0u, n) - 1;
                // (of entries without tokens the last one that begins there is found: it is the one behind them)
                const Entry &e = sm.entries[a.owner];
                first_token = e.own0, stop = e.own1, from = sm.before[a.owner];
                a.first = unit == from;
            }
            const int s = sm.entries[a.owner].s;
            a.j = first_token + (unit - from) * kUnit + lane;
            a.there = a.j < stop && s >= 0;
            if (a.there) a.page = p.cache.table[(size_t)s * p.cache.width + page_index(p, a.j)];
        }
    }
    __device__ void ask_ids() {  // of the tokens whose pages have been asked for
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const Asked &a = asked[k];
            auto &g = got[k];
            g.j = a.j, g.owner = a.owner, g.first = a.first;
            g.there = a.there && in_range(a.page, p.cache.pages);
            if (a.there && !g.there) bad = true;
            if (!g.there) continue;
            const int slot = a.j - page_index(p, a.j) * p.cache.page_size, id = a.page * p.cache.page_size + slot;
            g.row = p.cache.row_ids[id], g.col = p.cache.col_ids[id];
            g.at = (unsigned)a.page * p.page_step + (unsigned)slot * p.slot_step + head_at;
        }
    }
    // Behind a barrier that the last look at the part before it is in front of.
    __device__ void begin(const Part &part, Rows<RT> &rows) {
        seg = part.seg, leader = part.b - batch * p.pack;
        next = part.from, end = seg == 1 ? min(part.to, sm.before[kScouts]) : part.to;
        head_at = (unsigned)part.kv * p.head_step;
        pending = list_at = 0;
        if (seg == 0) shared_end = min(sm.entries[leader].shared, sm.entries[leader].len);
        ask_pages(next);
        Wishes<RT> &w = sm.wishes[parts & 1];
        ++parts;
        if (tid == 0) sm.wishes[parts & 1].clear();
        Wish x = {kNever, kNever, -2, kNobody};
        if (tid < part.n_rows) {
            const int member = member_of<RT>(p, part, tid), view = view_at(p, part.kv * p.group + part.tile * RT + tid - member * p.group);
            const int held_at = part.b - batch * p.pack + member;
            Entry other;
            if (held_at >= entries()) entry_of(p, part.b + member, sm.none, &other);
            const Entry &e = held_at >= entries() ? other : sm.entries[held_at];
            if (seg == 0 ? e.counts && e.first == part.b && e.count > 0 : e.own1 > e.own0) {
                const bool text = e.q_row == MATE_ID_TEXT || e.q_col == MATE_ID_TEXT;
                x.below = text ? INT32_MAX : e.prefix;
                if (!text && view != MATE_VIEW_COL) x.row = e.q_row;
                if (!text && view != MATE_VIEW_ROW) x.col = e.q_col;
                x.member = seg == 0 ? 0 : member;
            }
        }
        const int lane = tid & 31, least = __reduce_min_sync(~0u, x.below < 0 ? INT32_MAX : x.below), most = __reduce_max_sync(~0u, x.below);
        const int views = (__any_sync(~0u, x.row != kNever) ? 1 : 0) | (__any_sync(~0u, x.col != kNever) ? 2 : 0);
        const bool same = (__shfl_up_sync(~0u, x.row, 1) == x.row) & (__shfl_up_sync(~0u, x.col, 1) == x.col) &
                          (__shfl_up_sync(~0u, x.below, 1) == x.below) & (__shfl_up_sync(~0u, x.member, 1) == x.member);
        const unsigned begins = __ballot_sync(~0u, lane == 0 || !same);
        const int kind = (tid & ~31) + __popc(begins & (2u << lane) - 1) - 1;
        const int kinds = most < 0 ? 0 : (__popc(begins) + kKinds - 1) & -kKinds;
        if (begins >> lane & 1) w.kind[kind] = x;
        if (lane >= __popc(begins) && lane < kinds) w.kind[tid] = {kNever, kNever, -2, kNobody};
        if (lane == 0) {
            w.n[tid >> 5] = (uint8_t)kinds;
            if (most >= 0) atomicMin(&w.least, least), atomicMax(&w.most, most), atomicOr(&w.views, views);
        }
        if (tid < RT) rows.kind[tid] = (short)(x.below < 0 ? -1 : kind);
        __syncwarp();
        ask_ids();
        ask_pages(next + kUnits);
        sync();
    }
    __device__ const Wishes<RT> &wishes() const { return sm.wishes[parts + 1 & 1]; }  // of the present part
    __device__ bool more() const { return next < end; }
    __device__ void look() {
        const Wishes<RT> &w = wishes();
        const int lane = tid & 31, warp = tid >> 5;
        int *count = sm.counts[looks++ & 1];
        Key key[2];
        int of[2];
        bool is[2];
        unsigned those[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const auto &g = got[k];
            key[k] = {g.at, g.row == MATE_ID_TEXT || g.col == MATE_ID_TEXT ? -1 : g.j, g.row, g.col}, of[k] = g.owner;
            is[k] = g.there && g.row >= 0 && g.col >= 0;
            if (!is[k]) key[k] = nobody();
            if (is[k] && seg == 1) {
                const Entry &e = sm.entries[of[k]];
                is[k] = e.q_row == MATE_ID_TEXT || e.q_col == MATE_ID_TEXT || key[k].place < e.prefix || ((w.views & 1) && g.row == e.q_row) ||
                        ((w.views & 2) && g.col == e.q_col);
            }
        }
        if (seg == 0) {
#pragma unroll
            for (int k = 0; k < 2; ++k) is[k] = key[k].place < w.most;
            if (__any_sync(~0u, (key[0].at != kNowhere && !is[0]) || (key[1].at != kNowhere && !is[1])))
#pragma unroll 1
                for (int i = 0; i < kScouts; i += 32)
#pragma unroll 1
                    for (int j = i; j < i + w.n[i / 32]; j += kKinds)
#pragma unroll
                        for (int k = 0; k < kKinds; ++k) {
                            const int row = w.kind[j + k].row, col = w.kind[j + k].col;
                            is[0] |= (key[0].row == row) | (key[0].col == col), is[1] |= (key[1].row == row) | (key[1].col == col);
                        }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            those[k] = __ballot_sync(~0u, is[k]);
            // Own tokens of which none is left out begin at a multiple of `run`, so that they are copied in runs; in front of them are nobody's.
            const bool dense = got[k].first && those[k] == __ballot_sync(~0u, got[k].there) && __popc(those[k]) >= run;
            if (lane == 0) count[2 * warp + k] = __popc(those[k]) + (dense ? kDense : 0);
        }
        next += kUnits;
        if (next < end) {
            ask_ids();
            __syncwarp();
            ask_pages(next + kUnits);
        }
        sync();
        int to[2], gap[2], all = pending;
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const int c = count[i], up = c >= kDense ? (all + run - 1) & -run : all;
            if (i >> 1 == warp) to[i & 1] = up, gap[i & 1] = up - all;
            all = up + (c & (kDense - 1));
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (lane < gap[k]) put_key(to[k] - gap[k] + lane, nobody(), kNobody);
            if (those[k] >> lane & 1) put_key(to[k] + __popc(those[k] & ((1u << lane) - 1)), key[k], of[k]);
        }
        pending = all;
    }
    __device__ void put_key(int i, const Key &key, int of) {
        const unsigned at_list = (unsigned)(list_at + i) % kList;
        sm.list[at_list] = key, sm.owners[at_list] = (uint8_t)of;
    }
    __device__ Key key(int i) const { return sm.list[(unsigned)(list_at + i) % kList]; }
    __device__ int owner_of_key(int i) const { return sm.owners[(unsigned)(list_at + i) % kList]; }
    // Whether every row attends every key that is for it.
    __device__ bool plain() const { return wishes().least == INT32_MAX; }
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

// fp32: eight warps with eight rows each, two rows and four keys of a lane in S, eight rows and DP / 32 columns in P V; scores by shared memory.  Bound
// by its reads of shared memory beside the products: 64 sequences that share 4096 tokens, 8 kv heads of 4 x 128, 268 us, 16 TFLOP/s.
template <int DP>
__global__ void __launch_bounds__(kSimtThreads, 2) shared_simt_kernel(const __grid_constant__ SharedParams p) {
    extern __shared__ __align__(16) char smem_raw[];
    auto &sm = *reinterpret_cast<SimtSmem<DP> *>(smem_raw);
    constexpr int kVec = 4, kCols = DP / 32, kR = kSimtRows / (kSimtThreads / 32);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r0 = warp * kR;
    ptx::wait_prior_grid();
    static_assert(sizeof(sm.q) + sizeof(sm.k) + sizeof(sm.v) + sizeof(sm.s) >= sizeof(Found), "room for the entries");
    Found &found = *reinterpret_cast<Found *>(smem_raw);
    const Start start = find_start<kSimtRows, kSimtThreads>(p, found, sm.scout.none);
    if (start.left == 0) return;
    Scout<kSimtRows> scout = {p, sm.scout, tid, 1};
    if (tid < kScouts) scout.start(start, found);
    __syncthreads();
    for (int i = tid; i < (int)((sizeof(sm.q) + sizeof(sm.k) + sizeof(sm.v) + sizeof(sm.s)) / 4); i += kSimtThreads)
        reinterpret_cast<uint32_t *>(smem_raw)[i] = 0;  // columns that nobody writes
    __syncthreads();
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
                    every = part.seg == 0 && scout.plain();
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
                    const size_t at = ((size_t)sm.keys[k].at * p.row16 + (size_t)part.kv * p.head16) * kVec + c;
                    load16((const float *)p.cache.k + at, &sm.k[k][c]);
                    load16((const float *)p.cache.v + at, &sm.v[k][c]);
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
                const Wishes<kSimtRows> &wishes = sm.scout.wishes[n_parts & 1];
                uint32_t those[kR];
#pragma unroll
                for (int r = 0; r < kR; ++r) {
                    const int kind = sm.rows.kind[r0 + r];
                    const Wish &wish = wishes.kind[max(kind, 0)];
                    const bool is = lane < n && kind >= 0 && (part.seg == 0 || of == wish.member) && wish.is_for(key.place, key.row, key.col);
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
        const int state = part.state, slot = n_parts == 0 ? 0 : 1;
        float *to = p.parts + (size_t)(2 * blockIdx.x + slot) * part_floats(kSimtRows, p.d);
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            float sum = l[r];
#pragma unroll
            for (int step = 16; step > 0; step >>= 1) sum += __shfl_xor_sync(~0u, sum, step);
            const int row = r0 + r;
            if (row >= part.n_rows) break;
            const size_t whole = (size_t)(part.seg * p.B * p.heads) + row_of<kSimtRows>(p, part, row, member_of<kSimtRows>(p, part, row));
            for (int c = 0; c < kCols; ++c) {
                const int e = lane * kCols + c;
                if (e >= p.d) break;
                const float x = sum == 0.f ? 0.f : o[r][c];  // (a row that attends nothing here: whatever the others attend)
                (state == kAll ? p.whole + whole * p.d : to)[state == kAll ? e : (e / 4 * kSimtRows + row) * 4 + e % 4] = x;
            }
            if (lane == 0) (state == kAll ? p.whole_stats[whole] : reinterpret_cast<float2 *>(to + (size_t)p.d * kSimtRows)[row]) = make_float2(m[r], sum);
        }
        if (tid == 0) put_joint(p, part, slot, start.total);
    }
    if (tid < kScouts && scout.bad) atomicOr(p.cache.status, kCacheBad);
}

// ---- the tensor-core kernel (bf16): tiles of 128 rows and 128 keys, one block to an SM

constexpr int kTcRows = 128, kTcKeys = 128;
constexpr int kSoftmaxWarps = 8;              // two teams, which take the tiles in turn; a thread to a row
constexpr int kScoutWarp0 = kSoftmaxWarps, kScoutWarps = kScouts / 32;
constexpr int kCopyWarp0 = kScoutWarp0 + kScoutWarps, kCopyWarps = 2;  // keys, values
constexpr int kMmaWarp = kCopyWarp0 + kCopyWarps, kMmaWarps = 2;       // a team each
constexpr int kTcThreads = 32 * (kMmaWarp + kMmaWarps);
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
};
constexpr int kAhead = kList - kLooked - kTcKeys + 1;  // a look comes while a tile waits for its place, where the list has room for it
static_assert(kAhead >= 0, "room for a look behind what is less than a tile");
enum { kFirst = 1, kLast = 2, kRanged = 4, kBits = 8 };  // tiles of a part; keys lo[m] to hi[m] are for the rows of entry m, or as bits[kind] says, else
                                                          // all keys for all rows that attend anything
struct alignas(16) Meta {
    int n, flags;     // keys; n < 0: the share is done
    unsigned x16;     // where a row's elements begin, in 16 bytes
    uint8_t runs[4];  // of every 32 keys, a bit for each kRun of them: they lie one behind the other
    alignas(16) uint32_t bits[kTcRows][kTcKeys / 32];
    unsigned at[kTcKeys];
    uint8_t lo[kTcRows], hi[kTcRows];
};
// Keys and values as matrices whose rows are a slot stride apart: a run of slots is a box, which comes in by one bulk tensor copy for every
// 64 elements.
struct TcMaps {
    CUtensorMap k, v;
    int run;  // rows of a box: kRun; 0: every row is copied by itself
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
    uint64_t part_full[2], q_full[2], q_empty[2], k_full[4], k_empty[4], v_full[4], v_empty[4], meta_full[kMetas], meta_empty[kMetas], s_full[2], p_full[2],
        pv_done[2], team[2], both, final_;
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

// Every wait is bounded; the first one to run out raises the flag that ends all of them.  A warp passes a wait, or leaves its role, as a whole.
struct Wait {
    uint32_t bar, parity;
    volatile int *abort;
    __device__ bool there() const { return ptx::mbar_try_wait(bar, parity); }
    __device__ bool all(bool x) const { return __all_sync(~0u, x); }
    __device__ bool any(bool x) const { return __any_sync(~0u, x); }
    __device__ bool given_up() const { return *abort; }
    __device__ void give_up() const { *abort = 1; }
};
__device__ __noinline__ bool wait_long(uint32_t bar, uint32_t parity, volatile int *abort) { return wait_together(Wait{bar, parity, abort}, ptx::kWaitLimit); }

__device__ __forceinline__ uint32_t bits_below(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }
__device__ __forceinline__ float top_score(const uint32_t (&v)[32]) {
    float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int e = 0; e < 32; e += 8)
#pragma unroll
        for (int j = 0; j < 4; ++j) t[j] = ptx::fmax3(t[j], __uint_as_float(v[e + 2 * j]), __uint_as_float(v[e + 2 * j + 1]));
    return fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
}
// Weights 2^(s scale - base), 16 keys at a time, as pairs of bf16: rounded, and what the rounding left, half a step of 2^-8, rounded by half a step of that.
// Their sum has 16 bits: a weight is off by 2^-16 at most, the difference of two weights that are 2^-12 apart by 3 %.  The sums take all of them.
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

// The row's O times `keep` (rarely).
__device__ __noinline__ void scale_o(uint32_t tO, int n, float keep) {
    ptx::tc_fence_after();
#pragma unroll 1
    for (int i = 0; i < n; i += 16) {
        uint32_t o[16];
        ptx::tmem_ld16(tO + i, o);
        ptx::tc_wait_ld();
        ptx::reg_fence(o);
#pragma unroll
        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * keep);
        ptx::tmem_st16(tO + i, o);
    }
    ptx::tc_wait_st();
}

// The row's weights of the keys before, where they have not gone into O yet (more rarely still).
__device__ __noinline__ void scale_p(uint32_t tP, int n, float keep) {
    ptx::tc_wait_st();
#pragma unroll 1
    for (int i = 0; i < n; i += 16) {
        uint32_t hi[8], lo[8];
        ptx::tmem_ld8(tP + i, hi);
        ptx::tmem_ld8(tP + i + 8, lo);
        ptx::tc_wait_ld();
        ptx::reg_fence(hi);
        ptx::reg_fence(lo);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = (__uint_as_float(hi[e] << 16) + __uint_as_float(lo[e] << 16)) * keep;
            const float y = (__uint_as_float(hi[e] & 0xffff0000u) + __uint_as_float(lo[e] & 0xffff0000u)) * keep;
            hi[e] = ptx::cvt_bf16x2(x, y);
            lo[e] = ptx::cvt_bf16x2(x - __uint_as_float(hi[e] << 16), y - __uint_as_float(hi[e] & 0xffff0000u));
        }
        ptx::tmem_st8(tP + i, hi);
        ptx::tmem_st8(tP + i + 8, lo);
    }
    ptx::tc_wait_st();
}

template <int DP>
__global__ void __launch_bounds__(kTcThreads, 1) shared_tc_kernel(const __grid_constant__ SharedParams p, const __grid_constant__ TcMaps maps) {
    using namespace ptx;
    using S = TcShape<DP>;
    constexpr int kStages = S::kStages, kHalves = DP / 64;
    extern __shared__ uint8_t tc_smem[];
    TcSmem<DP> &sm = *reinterpret_cast<TcSmem<DP> *>(tc_smem + (-smem_u32(tc_smem) & 1023));
    const int tid = threadIdx.x, warp = __shfl_sync(~0u, tid >> 5, 0), lane = tid & 31;
    const auto bar = [](const uint64_t &b) { return smem_u32(&b); };

    if (warp == 0) {  // (a lane to an index: one after the other they take a third of a microsecond)
        if (lane < 2) {
            mbar_init(bar(sm.part_full[lane]), 1);
            mbar_init(bar(sm.q_full[lane]), kScoutWarps + 1);
            mbar_init(bar(sm.q_empty[lane]), kSoftmaxWarps + kMmaWarps);
            mbar_init(bar(sm.s_full[lane]), 1), mbar_init(bar(sm.pv_done[lane]), 1);
            mbar_init(bar(sm.p_full[lane]), kSoftmaxWarps / 2);
            mbar_init(bar(sm.team[lane]), kSoftmaxWarps / 2);
            sm.odd[lane] = 0;
        }
        if (lane < kStages) {
            mbar_init(bar(sm.k_full[lane]), 1), mbar_init(bar(sm.v_full[lane]), 1);
            mbar_init(bar(sm.k_empty[lane]), 1), mbar_init(bar(sm.v_empty[lane]), 1);
        }
        if (lane < kMetas) mbar_init(bar(sm.meta_full[lane]), kScoutWarps), mbar_init(bar(sm.meta_empty[lane]), kSoftmaxWarps + kCopyWarps + kMmaWarps);
        if (lane == 0) {
            mbar_init(bar(sm.both), kSoftmaxWarps), mbar_init(bar(sm.final_), kMmaWarps);
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
    static_assert(sizeof(sm.k) >= sizeof(Found), "room for the entries");
    Found &found = *reinterpret_cast<Found *>(sm.k);
    const Start start = find_start<kTcRows, kTcThreads>(p, found, sm.scout.none);  // (its barriers: the set-up is seen by all)
    tc_fence_after();
    Scout<kTcRows> scout = {p, sm.scout, tid - 32 * kScoutWarp0, max(1, maps.run)};
    if (start.left && warp >= kScoutWarp0 && warp < kCopyWarp0) scout.start(start, found);
    if (p.d < DP) {  // columns that no copy writes
        __syncthreads();
#pragma unroll 1
        for (int i = tid; i < (2 + 2 * kStages) * S::kTile / 16; i += kTcThreads) reinterpret_cast<uint4 *>(sm.q)[i] = make_uint4(0, 0, 0, 0);
    }
    fence_proxy_async();  // (what has been written where bulk copies will write)
    __syncthreads();
    const uint32_t tmem = __shfl_sync(~0u, sm.tmem, 0);

    volatile int *abort = &sm.abort;
    const auto wait = [&](const uint64_t &b, uint32_t parity) {
        return __all_sync(~0u, mbar_try_wait(smem_u32(&b), parity)) || wait_long(smem_u32(&b), parity, &sm.abort);
    };

    if (start.left == 0) {
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
        int kind = 0, member = 0, tiles = 0, own = 0;  // tiles of the part; the team's
        bool live = false;
        float m = -INFINITY;
        uint64_t sum[2] = {0, 0};
#pragma unroll 1
        for (int t = 0;; ++t) {
            const Meta &meta = sm.meta[t % kMetas];
            if (!wait(sm.meta_full[t % kMetas], t / kMetas & 1)) break;
            const int2 head = *reinterpret_cast<const int2 *>(&meta);
            const int n = head.x, flags = head.y, qb = parts & 1;
            if (n < 0) break;
            const Part &part = sm.part[qb];
            if (flags & kFirst) {
                if (!wait(sm.q_full[qb], parts / 2 & 1)) break;
                kind = sm.rows[qb].kind[r];
                live = (warp & 3) * 32 < part.n_rows;
                member = member_of<kTcRows>(p, part, r);
                tiles = own = 0;
                m = -INFINITY;
                sum[0] = sum[1] = 0;
            }
            if (n > 0 && (c & 1) == team) {
                // (S is there, so the P V of the team's tile before, whose place it has, is done)
                if (!wait(sm.s_full[team], mine & 1)) break;
                tc_fence_after();
                const int stage = c % kStages;
                bool odd = false;
                if (flags & (kRanged | kBits)) {  // a weight 0 does not undo a value that is not a number: is there one?
                    if (!wait(sm.v_full[stage], c / kStages & 1)) break;
                    const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f);
                    __nv_bfloat162 z = zero, z2 = zero;
                    const uint4 *v = reinterpret_cast<const uint4 *>(sm.v[stage]);
#pragma unroll 1
                    for (int h = 0; h < kHalves; ++h, v += kTcKeys * 8)
#pragma unroll 8
                        for (int i = r; i < n * 8; i += 128) {
                            const uint4 y = v[i];
                            for (uint32_t w : {y.x, y.y}) z = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&w), zero, z);
                            for (uint32_t w : {y.z, y.w}) z2 = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&w), zero, z2);
                        }
                    z = __hadd2(z, z2);
                    if (__any_sync(~0u, !(__low2float(z) == 0.f && __high2float(z) == 0.f)) && lane == 0) *(volatile int *)&sm.odd[team] = c + 1;
                    if (!sync(sm.team[team], teams)) break;
                    odd = *(volatile int *)&sm.odd[team] == c + 1;
                }
                // the keys that the row attends
                uint4 on = make_uint4(0, 0, 0, 0);
                if (kind < 0) {
                } else if (flags & kBits) {
                    on = *reinterpret_cast<const uint4 *>(meta.bits[kind]);
                } else {
                    const int lo = flags & kRanged ? meta.lo[member] : 0, hi = flags & kRanged ? meta.hi[member] : n;
                    on = make_uint4(bits_below(hi) & ~bits_below(lo), bits_below(hi - 32) & ~bits_below(lo - 32), bits_below(hi - 64) & ~bits_below(lo - 64),
                                    bits_below(hi - 96) & ~bits_below(lo - 96));
                }
                if (live) {
                    if (own == 0) {
                        uint32_t zero[16] = {};
#pragma unroll 1
                        for (int i = 0; i < DP; i += 16) tmem_st16(tO + i, zero);
                    }
#pragma unroll 1
                    for (int c0 = 0; c0 < n; c0 += 32) {
                        uint32_t v[32] = {};
                        if (__any_sync(~0u, on.x)) {
                            tmem_ld32(tS + c0, v);
                            tc_wait_ld();
                            reg_fence(v);
                            if (!__all_sync(~0u, on.x == ~0u)) {
#pragma unroll
                                for (int e = 0; e < 32; ++e)
                                    if (!(on.x >> e & 1)) v[e] = 0xff800000u;
                            }
                            // The base of a row moves when a score exceeds it by kRescale, and with the row's first score: O, the sum and the
                            // weights of the tile's keys in front of these follow.
                            const float top = top_score(v) * p.scale_log2;
                            const bool moves = top > m + kRescale;
                            const bool first_score = m == -INFINITY;  // (there is nothing yet that would have to follow)
                            const float keep = moves && !first_score ? ex2(m - top) : 1.f;
                            if (moves) m = top;
                            if (__any_sync(~0u, moves && !first_score)) {
                                const uint64_t keep2 = pack_f32x2(keep, keep);
                                sum[0] = mul_f32x2(sum[0], keep2), sum[1] = mul_f32x2(sum[1], keep2);
                                if (own > 0) scale_o(tO, DP, keep);
                                if (c0 > 0) scale_p(tS, c0, keep);
                            }
                            const float neg = m == -INFINITY ? 0.f : -m;
                            weigh(v, scale2, pack_f32x2(neg, neg), sum);
                        }
                        tmem_st32(tS + c0, v);
                        on = make_uint4(on.y, on.z, on.w, on.x);
                    }
                    tc_wait_st();
                }
                if (odd) {
                    for (int i = (n + 31) / 32; i < 4; ++i) on = make_uint4(on.y, on.z, on.w, on.x);  // (back to the first)
                    // Values that are not numbers: added here to the rows that attend them, and taken out of the tile.
                    const auto at = [&](int key, int e) {
                        return reinterpret_cast<__nv_bfloat16 *>(sm.v[stage] + e / 64 * S::kHalf + key * 128 + ((e / 8 & 7) ^ (key & 7)) * 16 + e % 8 * 2);
                    };
#pragma unroll 1
                    for (int key = 0; key < n && live; ++key) {
                        if (key % 32 == 0 && key > 0) on = make_uint4(on.y, on.z, on.w, on.x);
                        const bool counts = on.x >> (key & 31) & 1;
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
            if (!(flags & kLast)) continue;

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
                if (live) {
                    const bool row = r < part.n_rows, all = part.state == kAll;
                    const int slot = parts == 0 ? 0 : 1, whole = part.seg * p.B * p.heads + row_of<kTcRows>(p, part, r, member);
                    float *to = all ? p.whole + (size_t)whole * p.d : p.parts + (size_t)(2 * blockIdx.x + slot) * part_floats(kTcRows, p.d) + 4 * r;
                    float2 *stat = all ? p.whole_stats + whole
                                       : reinterpret_cast<float2 *>(p.parts + (size_t)(2 * blockIdx.x + slot) * part_floats(kTcRows, p.d) + p.d * kTcRows) + r;
                    const int step = all ? 4 : 4 * kTcRows, col0 = joined && team ? DP / 2 : 0, col1 = min(p.d, joined ? col0 + DP / 2 : DP);
                    const uint32_t first_o = tmem + lanes + kTmemO + (joined ? 0 : team * 128);
                    to += col0 / 4 * step;
#pragma unroll 1
                    for (int col = col0; col < col1; col += 16) {
                        uint32_t o[16], o2[16] = {};
                        tmem_ld16(first_o + col, o);
                        if (joined) tmem_ld16(first_o + 128 + col, o2);
                        tc_wait_ld();
                        reg_fence(o);
                        reg_fence(o2);
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            o[e] = l == 0.f ? 0u : __float_as_uint(fmaf(__uint_as_float(o2[e]), f[1], __uint_as_float(o[e]) * f[0]));
                        if (row) {
                            *reinterpret_cast<uint4 *>(to) = make_uint4(o[0], o[1], o[2], o[3]);
                            *reinterpret_cast<uint4 *>(to + step) = make_uint4(o[4], o[5], o[6], o[7]);
                            if (col + 8 < p.d) {
                                *reinterpret_cast<uint4 *>(to + 2 * step) = make_uint4(o[8], o[9], o[10], o[11]);
                                *reinterpret_cast<uint4 *>(to + 3 * step) = make_uint4(o[12], o[13], o[14], o[15]);
                            }
                            to += 4 * step;
                        }
                    }
                    if (row && (!joined || team == 0)) *stat = make_float2(m, l);
                    if (r == 0 && (!joined || team == 0)) put_joint(p, part, slot, start.total);
                }
                tc_fence_before();
                if (joined && !sync(sm.both, boths)) break;  // O has been read
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sm.q_empty[qb]));
            ++parts;
        }
    } else if (warp < kCopyWarp0) {
        // ------------------------------------------------------------------ which keys are read
        // (These warps meet at barriers: they leave together, when one of them says there that a wait of its own has failed.)
        const int lt = tid - 32 * kScoutWarp0, lw = warp - kScoutWarp0;
        bool ok = true;
        int t = 0;
        Part part;
#pragma unroll 1
        for (int parts = 0;; ++parts) {
            const int qb = parts & 1;
            const bool is = scout.next_part(part);
            if (!is) part.n_rows = 0;
            if (parts >= 2) ok &= wait(sm.q_empty[qb], (parts / 2 - 1) & 1);
            if (any_scout(!ok)) break;
            if (lt == 0) {
                sm.part[qb] = part;
                mbar_arrive(bar(sm.part_full[qb]));
            }
            __syncwarp();
            if (!is) break;
            scout.begin(part, sm.rows[qb]);
            if (lane == 0) mbar_arrive(bar(sm.q_full[qb]));
            const bool all_plain = scout.plain();
            bool last = false;
#pragma unroll 1
            for (bool first = true; !last; first = false, ++t) {
#pragma unroll 1
                while (scout.pending < kTcKeys + (first ? 0 : kAhead) && scout.more()) scout.look();
                const int n = min(scout.pending, kTcKeys);
                last = scout.pending <= kTcKeys && !scout.more();
                if (t >= kMetas) ok &= wait(sm.meta_empty[t % kMetas], (t / kMetas - 1) & 1);
                Meta &meta = sm.meta[t % kMetas];
                if (ok) meta.lo[lt] = meta.hi[lt] = 0;
                if (any_scout(!ok)) break;
                Key key = nobody();
                int of = kNobody;
                if (lt < n) key = scout.key(lt), of = scout.owner_of_key(lt);
                const bool plain = all_plain || (part.seg == 0 && !any_scout(lt < n && key.place >= scout.wishes().least));
                if (!plain) {  // a bit for each key, of every kind of row that it may be for
                    const Wishes<kTcRows> &w = scout.wishes();
                    const bool own = part.seg == 1, there = key.at != kNowhere;
                    const unsigned of0 = own ? __reduce_min_sync(~0u, of) : 0, of1 = own ? __reduce_max_sync(~0u, of == kNobody ? 0 : of) : 0;
#pragma unroll 1
                    for (int i = 0; i < kScouts; i += 32) {
                        int k0 = 0, k1 = w.n[i / 32];
                        if (own) {  // those of the keys' owners (they are in order)
                            const int of_kind = lane < k1 ? w.kind[i + lane].member : kNobody;
                            const unsigned kinds = __ballot_sync(~0u, of_kind >= of0 && of_kind <= of1);
                            k0 = kinds ? (__ffs(kinds) - 1) & -kKinds : 32, k1 = 32 - __clz(kinds);
                        }
                        unsigned word = 0;
#pragma unroll 1
                        for (int k = i + k0; k < i + k1; k += kKinds)
#pragma unroll
                            for (int j = 0; j < kKinds; ++j) {
                                const Wish x = w.kind[k + j];
                                const unsigned those = __ballot_sync(~0u, there && (!own || of == x.member) && x.is_for(key.place, key.row, key.col));
                                if (lt % 32 == k + j - i) word = those;
                            }
                        meta.bits[i + lane][lw] = word;
                    }
                } else if (part.seg == 1 && of != kNobody) {
                    if (lt == 0 || scout.owner_of_key(lt - 1) != of) meta.lo[of] = (uint8_t)lt;
                    if (lt == n - 1 || scout.owner_of_key(lt + 1) != of) meta.hi[of] = (uint8_t)(lt + 1);
                }
                meta.at[lt] = key.at;
                const unsigned before = __shfl_up_sync(~0u, key.at, 1);
                const unsigned follows = __ballot_sync(~0u, key.at != kNowhere && (lt % kRun == 0 || key.at == before + p.slot_step));
                const unsigned runs = maps.run ? ((follows & 0xffff) == 0xffff ? 1 : 0) | (follows >> 16 == 0xffff ? 2 : 0) : 0;
                if (lane == 0) meta.runs[lw] = (uint8_t)runs;
                if (lt == 0)
                    meta.n = n, meta.flags = (first ? kFirst : 0) | (last ? kLast : 0) | (!plain ? kBits : part.seg ? kRanged : 0), meta.x16 = (unsigned)part.kv * p.head16;
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(sm.meta_full[t % kMetas]));
                scout.taken(n);
            }
            if (!last) break;
        }
        // behind the last one (where a wait has failed its place may still be read, and the flag ends the other roles)
        if (t >= kMetas) ok &= wait(sm.meta_empty[t % kMetas], (t / kMetas - 1) & 1);
        if (!any_scout(!ok)) {
            if (lt == 0) sm.meta[t % kMetas].n = -1;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sm.meta_full[t % kMetas]));
        }
        if (scout.bad) atomicOr(p.cache.status, kCacheBad);
    } else if (warp < kMmaWarp) {
        // ------------------------------------------------------------------ copies of queries and keys (first warp) and values (second)
        // Runs by one lane, the rest row by row.
        const bool leader = elect_one(), v = warp != kCopyWarp0;
        const CUtensorMap *map = v ? &maps.v : &maps.k;
        const int chunk = lane & 7, sub = lane >> 3;  // of a copy of four rows
        const unsigned stride = p.row16 * 16;
        const auto copy_queries = [&](int qb) {  // of the part that comes next
            const Part &part = sm.part[qb];
            const uint32_t q = smem_u32(sm.q[qb]);
            const int n_rows = part.n_rows, b = part.b, head0 = part.kv * p.group + part.tile * kTcRows, at0 = part.tile * kTcRows;
#pragma unroll 2
            for (int row = sub; row < n_rows; row += 4) {
                const int member = by_group(p, at0 + row);
                const __nv_bfloat16 *from = (const __nv_bfloat16 *)p.Q + (b + member) * p.q_batch + (head0 + row - member * p.group) * p.q_head + chunk * 8;
                const uint32_t to = q + row * 128 + ((chunk ^ (row & 7)) << 4);
#pragma unroll
                for (int h = 0; h < kHalves; ++h)
                    if (h * 8 + chunk < p.d / 8) cp_async16(to + h * S::kHalf, from + 64 * h);
            }
            if (p.flip) {  // a negative scale: its sign goes to the queries
                asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll 1
                for (int row = sub; row < n_rows; row += 4)
#pragma unroll 1
                    for (int h = 0; h < kHalves; ++h) {
                        uint4 *x = reinterpret_cast<uint4 *>(sm.q[qb] + h * S::kHalf + row * 128 + ((chunk ^ (row & 7)) << 4));
                        constexpr uint32_t kSigns = 0x80008000u;
                        *x = make_uint4(x->x ^ kSigns, x->y ^ kSigns, x->z ^ kSigns, x->w ^ kSigns);
                    }
            }
            __syncwarp();
            cp_async_arrive(bar(sm.q_full[qb]));
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sm.q_full[qb]));
        };
        int parts = 0, c = 0;  // parts, tiles that have been asked for
        bool asked = false;    // the queries of part number `parts`
#pragma unroll 1
        for (int t = 0;; ++t) {
            if (!v && !asked) {
                if (!wait(sm.part_full[parts & 1], parts / 2 & 1) || sm.part[parts & 1].n_rows == 0) break;
                copy_queries(parts & 1);
                asked = true;
            }
            const Meta &meta = sm.meta[t % kMetas];
            if (!wait(sm.meta_full[t % kMetas], t / kMetas & 1)) break;
            const int n = meta.n, last = meta.flags & kLast;
            if (n < 0) break;
            if (n > 0) {
                const int stage = c % kStages;
                const uint64_t &full = v ? sm.v_full[stage] : sm.k_full[stage];
                const uint32_t tile = smem_u32(v ? sm.v[stage] : sm.k[stage]);
                const uint32_t blocks = (2u << ((n - 1) / kRun)) - 1;  // that have a key
                const uint32_t runs = blocks & (meta.runs[0] | meta.runs[1] << 2 | meta.runs[2] << 4 | meta.runs[3] << 6);
                const int x16 = (int)meta.x16;
                unsigned at[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) at[i] = meta.at[i * kRun];
                if (c >= kStages && !wait(v ? sm.v_empty[stage] : sm.k_empty[stage], (c / kStages - 1) & 1)) break;
                if (runs && leader) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (runs >> i & 1)
#pragma unroll
                            for (int h = 0; h < kHalves; ++h) tma_load_2d(tile + h * S::kHalf + i * kRun * 128, map, x16 * 8 + 64 * h, (int)at[i], bar(full));
                }
                __syncwarp();
                if (runs != blocks) {
                    const uint32_t first = tile + sub * 128 + ((chunk ^ sub) << 4);
                    const char *from = (const char *)(v ? p.cache.v : p.cache.k) + (size_t)x16 * 16 + chunk * 16;
#pragma unroll 1
                    for (uint32_t rest = blocks & ~runs; rest; rest &= rest - 1) {
                        const int row0 = (__ffs(rest) - 1) * kRun;
                        unsigned place[4];  // (ahead of the copies: a load behind a copy waits its turn)
#pragma unroll
                        for (int i = 0; i < 4; ++i) place[i] = meta.at[row0 + 4 * i + sub];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            // (the row's low three bits permute its 16 bytes: those of sub, and those of 4 i)
                            const bool is = place[i] != kNowhere;
                            const char *row = from + (is ? (size_t)place[i] * stride : 0);
                            const uint32_t to = (first ^ (i & 1) << 6) + (row0 + 4 * i) * 128;
#pragma unroll
                            for (int h = 0; h < kHalves; ++h)
                                if (h * 8 + chunk < p.d / 8) cp_async16_or_zero(to + h * S::kHalf, row + h * 128, is);
                        }
                    }
                    __syncwarp();
                    cp_async_arrive(bar(full));
                    __syncwarp();
                }
                if (lane == 0) mbar_arrive_expect_tx(bar(full), __popc(runs) * kHalves * kRun * 128);  // (behind all that has been asked for)
                ++c;
            }
            if (last) ++parts, asked = false;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sm.meta_empty[t % kMetas]));
        }
        // No copy outlives the block, whoever has given up: the last tile of every stage is waited for.
        asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll 1
        for (int stage = 0; stage < min(c, kStages); ++stage)
            mbar_wait_bounded(bar(v ? sm.v_full[stage] : sm.k_full[stage]), (c - 1 - stage) / kStages & 1, kWaitLimit);
    } else {
        // ------------------------------------------------------------------ the products, a warp to each team
        // S = Q K^T of a tile as soon as its keys are there and the team's last P V, whose weights have the place of S, is done; O += P V as
        // soon as P is there.
        const bool leader = elect_one();
        const int team = warp - kMmaWarp;
        const uint32_t tS = tmem + kTmemS + team * kTcKeys, tO = tmem + kTmemO + team * 128, idesc_pv = idesc_bf16(kTcRows, DP, 0, 1);
        int c = 0, mine = 0, parts = 0;
#pragma unroll 1
        for (int t = 0;; ++t) {
            const Meta &meta = sm.meta[t % kMetas];
            if (!wait(sm.meta_full[t % kMetas], t / kMetas & 1)) break;
            const int n = meta.n, last = meta.flags & kLast;
            if (n < 0) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sm.meta_empty[t % kMetas]));
            if (n > 0 && (c & 1) == team) {
                const int stage = c % kStages, phase = c / kStages & 1, steps = (n + 15) / 16;
                const uint32_t idesc = idesc_bf16(kTcRows, steps * 16, 0, 0);
                if (!wait(sm.q_full[parts & 1], parts / 2 & 1) || !wait(sm.k_full[stage], phase)) break;
                if (mine > 0 && !wait(sm.pv_done[team], (mine - 1) & 1)) break;
                fence_proxy_async();  // the copies of 16 bytes come through the generic proxy
                tc_fence_after();
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
                    if (last) mma_commit(bar(sm.q_empty[parts & 1]));
                }
                __syncwarp();
                if (!wait(sm.v_full[stage], phase) || !wait(sm.p_full[team], mine & 1)) break;
                tc_fence_after();
                fence_proxy_async();
                // (64 columns of V lie kHalf behind the others: the leading byte offset)
                const uint32_t v = (smem_u32(sm.v[stage]) & 0x3ffffu) >> 4 | (uint32_t)(S::kHalf >> 4) << 16;
                if (leader) {
                    const auto step = [&](int ks) {
                        mma_ts_lean<1>(tO, tS + 16 * ks, v + ks * (16 * 128 >> 4), idesc_pv);
                        mma_ts_lean<1>(tO, tS + 16 * ks + 8, v + ks * (16 * 128 >> 4), idesc_pv);
                    };
                    if (steps == kTcKeys / 16) {
#pragma unroll
                        for (int ks = 0; ks < kTcKeys / 16; ++ks) step(ks);
                    } else {
#pragma unroll 1
                        for (int ks = 0; ks < steps; ++ks) step(ks);
                    }
                    mma_commit(bar(sm.pv_done[team]));
                    mma_commit(bar(sm.v_empty[stage]));
                }
                __syncwarp();
                ++mine;
            } else if (last) {
                if (leader) mma_commit(bar(sm.q_empty[parts & 1]));
                __syncwarp();
            }
            c += n > 0, parts += last != 0;
        }
        if (leader) mma_commit(bar(sm.final_));  // nothing of this block may still run on the tensor pipe when its memory is freed
        __syncwarp();
        mbar_wait_bounded(bar(sm.final_), 0, kWaitLimit);
    }
    tc_fence_before();
    __syncthreads();
    if (tid == 0 && *abort) atomicOr(p.cache.status, kCacheTimeout);
    if (warp == kMmaWarp) tmem_dealloc(tmem, kTmemCols);
}

// ---- the results of a row put together

// A block has kJoinRows rows of a kv head; a lane has a row and four columns, a warp 16 columns and every `splits`-th of the results.  Who has
// them is found once for the block.  Latency: the kernel in front leaves no registers, so its blocks come to the SMs when those end, then a
// row's place, its parts, their sum: 5 us with the launch.  (A block to a row: 64 questions 54 us in all instead of 50.)
constexpr int kJoinRows = 8;
struct Results {
    const float *value;     // of the row's first column
    const float2 *stat;
    int64_t first, step;    // floats to the first one, and from number i i times to the others
    int column, parts;      // floats from four columns to the next
};
template <typename T, int RT>
__global__ void __launch_bounds__(1024) shared_join_kernel(const __grid_constant__ SharedParams p, int splits) {
    __shared__ Results s_of[2][kJoinRows];  // shared tokens, own ones
    __shared__ float4 s_sum[32][32];
    __shared__ float2 s_stat[32][32];
    ptx::launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, per_kv = (p.B * p.group + kJoinRows - 1) / kJoinRows, kv = blockIdx.x / per_kv;
    const int at0 = (blockIdx.x - kv * per_kv) * kJoinRows;
    if (tid < 2 * kJoinRows) {
        const int seg = tid / kJoinRows, i = tid % kJoinRows, b = by_group(p, at0 + i), g = at0 + i - b * p.group;
        // (the batch is looked at ahead of the wait: the kernel in front of this one has waited for whoever wrote it before it let this one start)
        Entry e = {};
        if (b < p.B) entry_of(p, b, nullptr, &e);
        ptx::wait_prior_grid();
        Results of = {};
        if (b < p.B && (seg == 1 || e.count > 0)) {
            const int row = (seg == 0 ? b - e.first : b % p.pack) * p.group + g, r = row % RT;
            const bool there = seg == 1 || p.grouped[b];  // (asked for together with what follows)
            const Joint joint = *joint_of(p, seg, kv, seg == 0 ? e.first : b / p.pack, row / RT);
            if (!there) {
            } else if (joint.slot < 0) {
                const size_t whole = (size_t)(seg * p.B + b) * p.heads + kv * p.group + g;
                of = {p.whole + whole * p.d, p.whole_stats + whole, 0, 0, 4, 1};
            } else if (joint.slot <= 1 && in_range(joint.first, p.blocks) && joint.total > 0) {  // (it may be what lay there, after a wait ran out)
                // up to the block that has the item's last unit: the last one whose share begins in front of the item's end
                const int64_t blocks = min((int64_t)joint.total, (int64_t)p.blocks), last = ((int64_t)joint.end * blocks - 1) / joint.total;
                const float *from = p.parts + 2 * joint.first * part_floats(RT, p.d);
                of = {from + 4 * r, reinterpret_cast<const float2 *>(from + (size_t)p.d * RT) + r, joint.slot * part_floats(RT, p.d),
                      2 * part_floats(RT, p.d), 4 * RT, (int)min(last, blocks - 1) - joint.first + 1};
            }
        }
        s_of[seg][i] = of;
    } else {
        ptx::wait_prior_grid();
    }
    __syncthreads();
    const int cols = (p.d + 15) / 16, split = warp / cols, c4 = (warp - split * cols) * 4 + lane / kJoinRows, i = lane % kJoinRows;
    const bool exists = at0 + i < p.B * p.group && c4 * 4 < p.d;
    float m = -INFINITY, l = 0.f;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    const auto add = [&](const float2 s, const float4 v) {
        const float top = fmaxf(m, s.x), base = top == -INFINITY ? 0.f : top, keep = ptx::ex2(m - base), w = ptx::ex2(s.x - base);
        m = top;
        l = fmaf(l, keep, s.y * w);
        sum.x = fmaf(sum.x, keep, v.x * w), sum.y = fmaf(sum.y, keep, v.y * w);
        sum.z = fmaf(sum.z, keep, v.z * w), sum.w = fmaf(sum.w, keep, v.w * w);
    };
#pragma unroll 1
    for (int seg = 0; seg < 2; ++seg) {
        const Results of = s_of[seg][i];
        const int n = exists ? of.parts : 0;
        constexpr int kBatch = 4;
#pragma unroll 1
        for (int k0 = split; k0 < n; k0 += kBatch * splits) {
            float2 s[kBatch];
            float4 v[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const int k = k0 + j * splits;
                const int64_t off = k == 0 ? of.first : k * of.step;
                s[j] = k < n ? *(of.stat + off / 2) : make_float2(-INFINITY, 0.f);
                v[j] = k < n ? *reinterpret_cast<const float4 *>(of.value + off + c4 * of.column) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int j = 0; j < kBatch; ++j) add(s[j], v[j]);
        }
    }
    if (splits > 1) {
        s_sum[warp][lane] = sum, s_stat[warp][lane] = make_float2(m, l);
        __syncthreads();
        if (split > 0) return;
        for (int w = warp + cols; w < cols * splits; w += cols) add(s_stat[w][lane], s_sum[w][lane]);
    }
    if (!exists) return;
    const int b = by_group(p, at0 + i);
    const size_t out = (size_t)b * p.heads + kv * p.group + at0 + i - b * p.group;
    T *to = (T *)p.O + out * p.d + c4 * 4;
    put(l == 0.f ? 0.f : sum.x / l, to), put(l == 0.f ? 0.f : sum.y / l, to + 1);
    put(l == 0.f ? 0.f : sum.z / l, to + 2), put(l == 0.f ? 0.f : sum.w / l, to + 3);
    if (c4 == 0) p.LSE[out] = natural(m, l);
}

// ---- host

// Up to here a batch is read one sequence after another: by keys and values of all sequences at their longest, which is all that the host knows.  us
// one by one and together, 32 own tokens each:
//   bf16, all in one group, 12 heads of 64 or 8 of 4 x 128 elements: 4 sequences of 4096 tokens (51 and 68 MB) 14 and 21, 17 and 20; 16 of 4096 (203
//   and 271 MB) 31 and 22, 36 and 21; 64 of 16384 (4.3 GB) 400 and 51.  In eight groups of 8 they come together later: 1024 tokens (277 MB) 21 and 38,
//   4096 (812 MB and 1.1 GB) 35 and 37, 42 and 35.  Without groups one by one stays the faster way however long they are: 16 of 4096 tokens (203 MB) 23 and
//   49, of 16384 66 and 164, 84 and 134; and so it is where cells leave most tokens out (29 and 43).
//   fp32, whose products are not made by the tensor cores: 64 sequences of 16384 tokens, 2 heads of 3 x 48 (807 MB), 136 and 106; 8 heads of 4 x 128, 16 of
//   4096 (541 MB) 85 and 101, 64 of 4096 (2.2 GB) 292 and 268, 16 of 16384 284 and 241; in eight groups of 8 93 and 225, without groups 158 and 1450.
// So the rule is for batches in one group or a few; what groups there are only the device knows.  A caller who knows of few takes mate_attn_decode.
double alone_bytes(const mate_cache_t *c) { return c->dtype == MATE_F32 ? 1024.0 * (1 << 20) : 192.0 * (1 << 20); }

int rows_of_tile(const mate_cache_t *c) { return c->dtype == MATE_F32 ? kSimtRows : kTcRows; }
int pack_of(const mate_cache_t *c) { return std::max(1, rows_of_tile(c) / (c->heads / c->kv_heads)); }
int own_tiles(const mate_cache_t *c) { return (c->heads / c->kv_heads + rows_of_tile(c) - 1) / rows_of_tile(c); }
int n_blocks(const mate_cache_t *c) { return (c->dtype == MATE_F32 ? 2 : 1) * n_sms(c->device); }

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }
struct Workspace {
    size_t joints, stats, whole, grouped, parts, bytes;
};
Workspace workspace_of(const mate_cache_t *c, int B) {
    Workspace w = {};
    w.stats = align256(sizeof(Joint) * 2 * (size_t)c->kv_heads * B * own_tiles(c));
    w.whole = w.stats + align256(sizeof(float2) * 2 * (size_t)B * c->heads);
    w.grouped = w.whole + align256(sizeof(float) * 2 * (size_t)B * c->heads * c->d);
    w.parts = w.grouped + align256((size_t)B);
    w.bytes = w.parts + sizeof(float) * 2 * (size_t)n_blocks(c) * part_floats(rows_of_tile(c), c->d);
    return w;
}

// Boxes of kRun rows, where a page is a whole number of them, the rows of all heads and pages lie in one such matrix and 64 columns from a
// head's first on are its own, or behind the last one.
TcMaps maps_of(SharedParams &p, const mate_cache_t *c) {
    TcMaps m = {};
    const int64_t slot = c->slot_stride, rows = slot > 0 ? ((int64_t)(c->pages - 1) * c->page_stride + (c->kv_heads - 1) * c->head_stride) / slot + c->page_size : 0;
    const bool fits = c->page_size % kRun == 0 && slot >= c->d && (c->pages == 1 || c->page_stride % slot == 0) && (slot == c->d || c->d % 64 == 0) && rows <= INT32_MAX && slot <= 1 << 27;
    if (fits && (c->kv_heads - 1) * (c->head_stride % slot) + c->d <= slot && make_box_map(&m.k, p.cache.k, (size_t)slot, (size_t)rows, (size_t)slot * 2, kRun) &&
        make_box_map(&m.v, p.cache.v, (size_t)slot, (size_t)rows, (size_t)slot * 2, kRun))
        m.run = kRun;
    if (m.run) {  // places in rows of a slot stride
        p.page_step = (unsigned)(c->page_stride / slot), p.slot_step = 1, p.head_step = (unsigned)(c->head_stride / slot);
        p.row16 = (unsigned)(slot / 8), p.head16 = (unsigned)(c->head_stride % slot / 8);
    }
    return m;
}

template <typename T, int DP>
int launch(SharedParams &p, const mate_cache_t *cache, cudaStream_t st) {
    constexpr bool kTc = sizeof(T) == 2;
    constexpr int kRows = kTc ? kTcRows : kSimtRows, kThreads = kTc ? kTcThreads : kSimtThreads;
    constexpr int kSmem = kTc ? 1024 + (int)sizeof(TcSmem<DP>) : (int)sizeof(SimtSmem<DP>);
    static_assert(kSmem <= 232448, "shared memory of a block");
    static SmemAttrOnce attr;
    cudaError_t e;
    if constexpr (kTc) {
        const int rc = attr.ensure((const void *)shared_tc_kernel<DP>, kSmem, cache->device);
        if (rc != MATE_OK) return rc;
        const TcMaps maps = maps_of(p, cache);
        e = launch_after(shared_tc_kernel<DP>, dim3((unsigned)p.blocks), kThreads, kSmem, st, p, maps);
    } else {
        const int rc = attr.ensure((const void *)shared_simt_kernel<DP>, kSmem, cache->device);
        if (rc != MATE_OK) return rc;
        e = launch_after(shared_simt_kernel<DP>, dim3((unsigned)p.blocks), kThreads, kSmem, st, p);
    }
    // sixteen warps to a block; twice as many where there is not a block to each SM (one sequence in many parts)
    const int joins = p.kv_heads * ((p.B * p.group + kJoinRows - 1) / kJoinRows), cols = (p.d + 15) / 16;
    const int splits = std::min(8, (joins < n_sms(cache->device) ? 32 : 16) / cols);
    if (e == cudaSuccess) e = launch_after(shared_join_kernel<T, kRows>, dim3((unsigned)joins), 32 * cols * splits, 0, st, p, splits);
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
    *bytes = n > 0 ? std::max(workspace_of(cache, n).bytes, decode_workspace(cache, n)) : 0;
    return MATE_OK;
}

int mate_attn_decode_shared(const mate_cache_t *cache, int layer, const void *Q, const int64_t *q_stride, int B, const int32_t *seqs,
                            const int32_t *row_ids, const int32_t *col_ids, const int32_t *groups, float scale, int max_len, unsigned flags,
                            void *O, float *LSE, void *workspace, size_t workspace_bytes, void *stream) {
    int rc = check_cache(cache);
    if (rc != MATE_OK) return rc;
    if (flags & ~(unsigned)MATE_SHARED_ALWAYS) return MATE_ERR_INVALID_ARG;
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
    // units of the batch, shared (of groups that have no entry in common) and own (these by up to a quarter more), are unsigned 32-bit numbers
    if (B > kMaxBatch || (int64_t)B * cache->kv_heads * own_tiles(cache) > INT32_MAX / 2 / (kOver + units_of(max_len))) return MATE_ERR_UNSUPPORTED;
    const Workspace w = workspace_of(cache, B);
    if (!workspace || workspace_bytes < std::max(w.bytes, decode_workspace(cache, B))) return MATE_ERR_WORKSPACE;
    if (!is_aligned(workspace, 256)) return MATE_ERR_ALIGNMENT;
    if (!(flags & MATE_SHARED_ALWAYS) && 2.0 * elem_size(cache->dtype) * B * max_len * cache->kv_heads * cache->d <= alone_bytes(cache)) {
        return decode(cache, layer, Q, q_stride, B, seqs, row_ids, col_ids, groups, scale, max_len, O, LSE, workspace, workspace_bytes, stream);
    }
    SharedParams p = {};
    p.cache = cache_args(cache, layer);
    p.Q = Q, p.q_batch = q_stride[0], p.q_head = q_stride[1];
    p.B = B, p.heads = cache->heads, p.kv_heads = cache->kv_heads, p.group = cache->heads / cache->kv_heads;
    p.d = cache->d, p.max_len = max_len, p.pack = pack_of(cache), p.own_tiles = own_tiles(cache);
    // (whose copies are shorter: 64 questions with 128 tokens of their own, heads of 128 elements, 39.1 us, without it 41.1, 256 sequences 101 and 102.5;
    // heads of 64: beams 30.2 with it and 30.1 without, cells 42.3 and 42.9; when it was chosen an eighth gave 38.8 and three 38.9 where a quarter gave 37.9)
    p.own_quarter = cache->dtype == MATE_BF16 && cache->d > 64;
    p.seqs = seqs, p.row_ids = row_ids, p.col_ids = col_ids, p.groups = groups;
    p.scale_log2 = scale * kLog2e, p.O = O, p.LSE = LSE;
    for (int h = 0; h < cache->heads; ++h) p.views[h >> 4] |= (uint32_t)cache->head_view[h] << 2 * (h & 15);
    const auto quotients = [](int by, unsigned *mul, unsigned *shift) {
        for (*shift = 0; 1u << *shift < (unsigned)by;) ++*shift;
        *mul = (unsigned)((((uint64_t)1 << 32) * (((uint64_t)1 << *shift) - by)) / by + 1);
    };
    quotients(cache->page_size, &p.page_mul, &p.page_shift);
    quotients(p.group, &p.group_mul, &p.group_shift);
    p.page_step = (unsigned)(cache->page_stride / vec), p.slot_step = (unsigned)(cache->slot_stride / vec), p.head_step = (unsigned)(cache->head_stride / vec);
    p.row16 = 1, p.head16 = 0;
    char *ws = static_cast<char *>(workspace);
    p.joints = reinterpret_cast<Joint *>(ws + w.joints);
    p.whole_stats = reinterpret_cast<float2 *>(ws + w.stats);
    p.whole = reinterpret_cast<float *>(ws + w.whole);
    p.grouped = reinterpret_cast<uint8_t *>(ws + w.grouped);
    p.parts = reinterpret_cast<float *>(ws + w.parts);
    if (cache->dtype == MATE_BF16) {
        // a score of -inf stays one whatever it is multiplied by: a factor above 0, so small for a scale of 0 that every weight is 1
        p.flip = p.scale_log2 < 0.f;
        p.scale_log2 = std::fmax(std::fabs(p.scale_log2), 0x1p-126f);
    }
    cudaStream_t st = (cudaStream_t)stream;
    p.blocks = n_blocks(cache);
    if (cache->dtype == MATE_F32) return cache->d <= 64 ? launch<float, 64>(p, cache, st) : launch<float, 128>(p, cache, st);
    return cache->d <= 64 ? launch<__nv_bfloat16, 64>(p, cache, st) : launch<__nv_bfloat16, 128>(p, cache, st);
}

}  // extern "C"

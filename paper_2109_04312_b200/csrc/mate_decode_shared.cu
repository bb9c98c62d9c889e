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

#include <cmath>
#include <type_traits>

#include "mate_cache.h"
#include "sm100_ptx.cuh"

namespace mate {
namespace {

constexpr int kUnit = 128;    // tokens of a unit of work: what is looked through in one go
constexpr int kOver = 1;      // units that an item costs besides its tokens
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
    int own_tiles;  // tiles of rows of an entry's own segment
    const int32_t *seqs, *row_ids, *col_ids, *groups;
    float scale_log2;  // scale / ln 2: weights are powers of two
    void *O;
    float *LSE;
    unsigned page16, head16, slot16;  // strides in 16 bytes; no place is beyond 2^32 of them
    unsigned page_mul, page_shift;    // x / page_size = (umulhi(x, page_mul) + x) >> page_shift for x < 2^31
    Joint *joints;                    // [2][kv_heads][B own_tiles]: shared segments, own ones
    float2 *whole_stats;              // [2][B heads]  m and sum P of rows that one block has done a segment of
    float *whole;                     // [2][B heads][d]
    float *parts;                     // [blocks][2]: values in groups of four by row, then the rows' m and sum P
    uint32_t views[kMaxHeads / 16];   // two bits a head
};
__device__ __forceinline__ int page_index(const SharedParams &p, int token) {
    return (int)((__umulhi((unsigned)token, p.page_mul) + (unsigned)token) >> p.page_shift);
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
    bool counts;     // the shared tokens are its own too
};
// What does not fit together on the device leaves an entry without a group: the rows of one group are the same in all of its entries.
__device__ __forceinline__ Entry entry_of(const SharedParams &p, int b, bool *bad) {
    const int s = p.seqs ? p.seqs[b] : b, q_row = p.row_ids[b], q_col = p.col_ids[b];
    const int first = p.groups[b], count = p.groups[p.B + b], shared = p.groups[2 * p.B + b];
    Entry e = {in_range(s, p.cache.seqs) ? s : -1, 0, 0, 0, 0, first, 0, false};
    if (e.s >= 0)
        e.len = clip_len(p.cache.lens[s], p.max_len, bad);
    else
        *bad = true;
    if (shared < 0) *bad = true;
    if (shared > 0 && count > 1) {
        if (first >= 0 && first <= b && count <= p.B - first && b - first < count && shared <= p.max_len && p.groups[first] == first &&
            p.groups[p.B + first] == count && p.groups[2 * p.B + first] == shared)
            e.count = count, e.shared = shared;
        else
            *bad = true;
    }
    const bool has = e.count > 0 && e.len >= shared, padding = q_row < 0 || q_col < 0 || e.s < 0;
    if (e.count > 0 && !has) *bad = true;
    e.counts = has && !padding;
    e.own0 = has ? shared : 0;
    e.own1 = padding ? e.own0 : e.len;
    return e;
}
// Units of an item of tokens; the first kOver stand for what an item costs whatever its length (none of its tokens belong to them).
__host__ __device__ __forceinline__ int units_of(int tokens) { return kOver + (tokens + kUnit - 1) / kUnit; }
__device__ __forceinline__ unsigned share(unsigned U, unsigned C, unsigned i) { return U / C * i + U % C * i / C; }

// The segments of an entry: [0] the shared tokens of the group that it is the first of, [1] its own.
struct Segment {
    int items, units;  // units of an item; 0: there is nothing to do
};
template <int RT>
__device__ __forceinline__ Segment segment_of(const SharedParams &p, const Entry &e, int b, int seg) {
    if (seg == 0) {
        const bool leads = e.count > 0 && e.first == b;
        return {leads ? p.kv_heads * (int)(((int64_t)e.count * p.group + RT - 1) / RT) : 0, leads ? units_of(e.shared) : 0};
    }
    // (an entry without a token and without a group has a result too)
    return {p.kv_heads * p.own_tiles, e.own1 > e.own0 ? units_of(e.own1 - e.own0) : e.count > 0 ? 0 : 1};
}
template <int RT>
__device__ __forceinline__ unsigned entry_units(const SharedParams &p, int b, bool *bad) {
    const Entry e = entry_of(p, b, bad);
    const Segment x = segment_of<RT>(p, e, b, 0), y = segment_of<RT>(p, e, b, 1);
    return (unsigned)x.items * x.units + (unsigned)y.items * y.units;
}

struct Start {
    unsigned total, before;  // units of the batch; of the entries in front of `entry`
    unsigned blocks;         // that get any: no more than there are units
    int entry;
};
// All threads call it: the entry that the block's first unit belongs to.
template <int RT, int NT>
__device__ Start find_start(const SharedParams &p) {
    __shared__ unsigned s_sum[NT / 32];
    __shared__ Start s_start;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (p.B + NT - 1) / NT, b0 = min(p.B, tid * per), b1 = min(p.B, b0 + per);
    bool bad = false;
    unsigned own = 0;
    for (int b = b0; b < b1; ++b) own += entry_units<RT>(p, b, &bad);
    unsigned sum = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned y = __shfl_up_sync(~0u, sum, o);
        if (lane >= o) sum += y;
    }
    if (lane == 31) s_sum[warp] = sum;
    if (tid == 0) s_start = {0, 0, 0, 0};
    __syncthreads();
    unsigned total = 0, before = sum - own;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
        if (w < warp) before += s_sum[w];
        total += s_sum[w];
    }
    const unsigned blocks = min(total, gridDim.x);
    if (blockIdx.x < blocks) {
        const unsigned at = share(total, blocks, blockIdx.x);
        if (at >= before && at < before + own) {
            int b = b0;
            for (; b < b1 - 1; ++b) {
                const unsigned n = entry_units<RT>(p, b, &bad);
                if (at < before + n) break;
                before += n;
            }
            s_start = {total, before, blocks, b};
        }
    }
    if (bad && blockIdx.x == 0) atomicOr(p.cache.status, kCacheBad);
    __syncthreads();
    return s_start;
}

// A part of an item: units [u0, u1) of them.
struct Part {
    int b, seg, kv, tile;
    int u0, u1, units;
    int t0, t1;      // its tokens
    int n_rows;
    bool grouped;    // the entry is in a group: its rows' results have to be joined
};
enum { kAll, kBegins, kGoesOn };
__device__ __forceinline__ int part_state(const Part &part) { return part.u0 > 0 ? kGoesOn : part.u1 == part.units ? kAll : kBegins; }
// Walks the parts of a block's share.  (It comes to an end whatever it finds: every part takes a unit off the share.)
struct Walk {
    int b, seg, item, u;
    int left;  // units of the share
};
template <int RT>
__device__ bool next_part(const SharedParams &p, Walk &w, Part &part) {
    bool bad = false;
    for (; w.left > 0 && w.b < p.B; w.seg = 0, w.item = 0, w.u = 0, ++w.b) {
        const Entry e = entry_of(p, w.b, &bad);
        for (; w.seg < 2; ++w.seg, w.item = 0, w.u = 0) {
            const Segment s = segment_of<RT>(p, e, w.b, w.seg);
            if (s.units == 0 || w.item >= s.items) continue;
            const int u1 = min(s.units, w.u + w.left);
            if (u1 <= kOver && u1 < s.units) {
                w.left = 0;
                return false;
            }
            const int tiles = s.items / p.kv_heads, kv = w.item / tiles, tile = w.item - kv * tiles;
            const int rows = (w.seg == 0 ? e.count : 1) * p.group;
            const int begin = w.seg == 0 ? 0 : e.own0, end = w.seg == 0 ? min(e.shared, e.len) : e.own1;
            part = {w.b, w.seg, kv, tile, w.u, u1, s.units, begin + max(0, w.u - kOver) * kUnit, min(end, begin + max(0, u1 - kOver) * kUnit),
                    min(RT, rows - tile * RT), e.count > 0};
            w.left -= max(1, u1 - w.u);
            w.u = 0;
            ++w.item;
            return true;
        }
    }
    return false;
}
// The first part of a block's share.
template <int RT>
__device__ __forceinline__ Walk walk_from(const SharedParams &p, const Start &start) {
    const unsigned at = share(start.total, start.blocks, blockIdx.x);
    bool bad = false;
    const Entry e = entry_of(p, start.entry, &bad);
    unsigned in = at - start.before;
    Walk w = {start.entry, 0, 0, 0, (int)(share(start.total, start.blocks, blockIdx.x + 1) - at)};
    Segment s = segment_of<RT>(p, e, w.b, 0);
    if (in >= (unsigned)s.items * s.units) in -= (unsigned)s.items * s.units, w.seg = 1, s = segment_of<RT>(p, e, w.b, 1);
    w.item = (int)(in / max(1, s.units));
    w.u = (int)(in - (unsigned)w.item * s.units);
    if (w.u <= kOver) w.left += w.u, w.u = 0;
    return w;
}
__device__ __forceinline__ Joint *joint_of(const SharedParams &p, int seg, int kv, int b, int tile) {
    return p.joints + ((size_t)seg * p.kv_heads + kv) * p.B * p.own_tiles + (size_t)b * p.own_tiles + tile;
}
// Of the part that begins an item that goes on in the next blocks (it is the last one of its block's share).
__device__ __forceinline__ Joint joint_from(const Part &part, const Start &start, int slot) {
    const int64_t end = (int64_t)share(start.total, start.blocks, blockIdx.x + 1) - (part.u1 - part.u0) + part.units;
    return {slot, (int)blockIdx.x, (int)min((end * start.blocks - 1) / start.total, (int64_t)start.blocks - 1), 0};
}

// ---- who attends what

// A row attends a key if the key's place is below `below` (text keys stand at -1, those of the prefix where they stand), or one of the ids is
// the one it wants.
struct RowInfo {
    int entry, head;  // head -1: there is no such row
    int want_row, want_col, below;
};
template <int RT>
__device__ RowInfo row_info(const SharedParams &p, const Part &part, int r) {
    RowInfo x = {part.b, -1, kNever, kNever, -2};
    if (r >= part.n_rows) return x;
    const int at = part.tile * RT + r, member = part.seg == 0 ? at / p.group : 0;
    x.entry = part.b + member;
    x.head = part.kv * p.group + at - member * p.group;
    bool bad = false;
    const Entry e = entry_of(p, x.entry, &bad);
    if (part.seg == 0 ? !e.counts || e.first != part.b || e.count == 0 : e.own1 <= e.own0) return x;
    const int q_row = p.row_ids[x.entry], q_col = p.col_ids[x.entry], view = view_at(p, x.head);
    if (q_row == MATE_ID_TEXT || q_col == MATE_ID_TEXT) {
        x.below = INT32_MAX;
        return x;
    }
    if (view != MATE_VIEW_COL) x.want_row = q_row;
    if (view != MATE_VIEW_ROW) x.want_col = q_col;
    x.below = max(0, p.cache.prefix[e.s]);
    return x;
}
__device__ __forceinline__ bool attends(int want_row, int want_col, int below, int place, int row, int col) {
    return place < below || row == want_row || col == want_col;
}

// The rows of a tile, as those who look for keys and those who weigh them need them.
template <int RT>
struct Rows {
    int want_row[RT], want_col[RT], below[RT];
    int least, most;     // of `below` over the rows that are there
    int n_want;          // wishes, without repetitions of the row before
    int2 want[RT];
};
// Keys, with what the rows go by.
struct Key {
    unsigned at;  // in 16 bytes from the cache's beginning
    int place, row, col;
};
constexpr int kList = 256;

// 128 threads look through the tokens of a part, 128 at a time.  Those that count go onto the list.
template <int RT>
struct Looker {
    const SharedParams &p;
    const Rows<RT> *rows;
    Key *list;       // [kList]
    int *counts;     // [4]
    int tid;         // of the 128
    int s, end, next, pending, list_at;
    unsigned head_at;
    bool bad;

    __device__ void sync() const { asm volatile("bar.sync 1, 128;" ::: "memory"); }
    __device__ void begin(const Part &part, const Rows<RT> *of) {
        rows = of;
        s = p.seqs ? p.seqs[part.b] : part.b;
        next = part.t0, end = part.t1;
        if (!in_range(s, p.cache.seqs)) end = next;
        head_at = (unsigned)part.kv * p.head16;
        pending = list_at = 0;
    }
    __device__ bool more() const { return next < end; }
    __device__ void look() {
        const int j = next + tid;
        Key key = {0, j, kNever, kNever};
        bool counts_here = false;
        if (j < end) {
            const int i = page_index(p, j), page = p.cache.table[(size_t)s * p.cache.width + i];
            if (in_range(page, p.cache.pages)) {
                const int slot = j - i * p.cache.page_size, id = page * p.cache.page_size + slot;
                key.row = p.cache.row_ids[id], key.col = p.cache.col_ids[id];
                key.at = (unsigned)page * p.page16 + (unsigned)slot * p.slot16 + head_at;
                if (key.row == MATE_ID_TEXT || key.col == MATE_ID_TEXT) key.place = -1;
                counts_here = key.place < rows->most;
                for (int w = 0; w < rows->n_want && !counts_here; ++w) counts_here = key.row == rows->want[w].x || key.col == rows->want[w].y;
                if (key.row < 0 || key.col < 0) counts_here = false;
            } else {
                bad = true;
            }
        }
        const unsigned those = __ballot_sync(~0u, counts_here);
        if ((tid & 31) == 0) counts[tid >> 5] = __popc(those);
        sync();
        int before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (w < tid >> 5) before += counts[w];
            all += counts[w];
        }
        if (counts_here) list[(list_at + pending + before + __popc(those & ((1u << (tid & 31)) - 1))) % kList] = key;
        pending += all;
        next += kUnit;
        sync();
    }
    __device__ void taken(int n) { list_at = (list_at + n) % kList, pending -= n; }
};
// Filled by the 128 (rows RT or fewer).
template <int RT>
__device__ void fill_rows(const SharedParams &p, const Part &part, Rows<RT> &rows, int tid) {
    const auto sync = [] { asm volatile("bar.sync 1, 128;" ::: "memory"); };
    if (tid == 0) rows.least = INT32_MAX, rows.most = INT32_MIN, rows.n_want = 0;
    sync();
    if (tid < RT) {
        const RowInfo x = row_info<RT>(p, part, tid);
        rows.want_row[tid] = x.want_row, rows.want_col[tid] = x.want_col, rows.below[tid] = x.below;
        if (x.below >= 0) {
            atomicMin(&rows.least, x.below);
            atomicMax(&rows.most, x.below);
        }
    }
    sync();
    if (tid < RT) {
        const int a = rows.want_row[tid], b = rows.want_col[tid];
        const bool same = tid > 0 && rows.want_row[tid - 1] == a && rows.want_col[tid - 1] == b;
        if (!same && (a != kNever || b != kNever)) rows.want[atomicAdd(&rows.n_want, 1)] = make_int2(a, b);
    }
    sync();
}

__device__ __forceinline__ void put(float x, float *y) { *y = x; }
__device__ __forceinline__ void put(float x, __nv_bfloat16 *y) { *y = __float2bfloat16_rn(x); }
__device__ __forceinline__ float natural(float m, float sum) { return sum == 0.f ? -INFINITY : (m + log2f(sum)) * kLn2; }

// ---- the kernel without tensor cores: tiles of 64 rows and 32 keys

constexpr int kSimtRows = 64, kSimtKeys = 32, kSimtThreads = 256;

template <int DP>
struct SimtSmem {
    float q[kSimtRows][DP + 4], k[kSimtKeys][DP + 4], v[kSimtKeys][DP];
    float s[kSimtRows][kSimtKeys + 4];
    Rows<kSimtRows> rows;
    Key list[kList], keys[kSimtKeys];
    int counts[4], n, last, plain;
};

template <typename T>
__device__ __forceinline__ void load16(const T *from, float *to) {
    const uint4 x = *reinterpret_cast<const uint4 *>(from);
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<uint4 *>(to) = x;
    } else {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) to[2 * i] = __uint_as_float(w[i] << 16), to[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

template <typename T, int DP>
__global__ void __launch_bounds__(kSimtThreads) shared_simt_kernel(const __grid_constant__ SharedParams p) {
    extern __shared__ __align__(16) char smem_raw[];
    auto &sm = *reinterpret_cast<SimtSmem<DP> *>(smem_raw);
    constexpr int kVec = 16 / sizeof(T), kCols = DP / 32, kR = kSimtRows / (kSimtThreads / 32);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r0 = warp * kR;
    ptx::wait_prior_grid();
    const Start start = find_start<kSimtRows, kSimtThreads>(p);
    if (blockIdx.x >= start.blocks) return;
    for (int i = tid; i < (int)(sizeof(SimtSmem<DP>) / 4); i += kSimtThreads) reinterpret_cast<uint32_t *>(smem_raw)[i] = 0;  // columns that nobody writes
    Walk walk = walk_from<kSimtRows>(p, start);
    Looker<kSimtRows> look = {p, &sm.rows, sm.list, sm.counts, tid};
    look.bad = false;
    __syncthreads();
    Part part;
    for (int n_parts = 0; next_part<kSimtRows>(p, walk, part); ++n_parts) {
        if (tid < 128) {
            fill_rows(p, part, sm.rows, tid);
            look.begin(part, &sm.rows);
        }
        for (int i = tid; i < kSimtRows * (p.d / kVec); i += kSimtThreads) {
            const int r = i / (p.d / kVec), c = (i - r * (p.d / kVec)) * kVec;
            if (r >= part.n_rows) continue;
            const int at = part.tile * kSimtRows + r, member = part.seg == 0 ? at / p.group : 0;
            load16((const T *)p.Q + (part.b + member) * p.q_batch + (part.kv * p.group + at - member * p.group) * p.q_head + c, &sm.q[r][c]);
        }
        float o[kR][kCols], m[kR], l[kR];
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            m[r] = -INFINITY, l[r] = 0.f;
#pragma unroll
            for (int c = 0; c < kCols; ++c) o[r][c] = 0.f;
        }
        for (bool more = true; more;) {
            if (tid < 128) {
                while (look.pending < kSimtKeys && look.more()) look.look();
                const int n = min(look.pending, kSimtKeys);
                bool every = true;
                if (tid < kSimtKeys) {
                    if (tid < n) sm.keys[tid] = look.list[(look.list_at + tid) % kList];
                    every = __all_sync(~0u, tid >= n || sm.keys[tid].place < sm.rows.least);
                }
                if (tid == 0) sm.n = n, sm.last = look.pending <= kSimtKeys && !look.more(), sm.plain = every;
                look.taken(n);
            }
            __syncthreads();
            const int n = sm.n;
            more = !sm.last;
            bool odd = false;
            for (int i = tid; i < kSimtKeys * (p.d / kVec); i += kSimtThreads) {
                const int k = i / (p.d / kVec), c = (i - k * (p.d / kVec)) * kVec;
                if (k < n) {
                    load16((const T *)p.cache.k + (size_t)sm.keys[k].at * kVec + c, &sm.k[k][c]);
                    load16((const T *)p.cache.v + (size_t)sm.keys[k].at * kVec + c, &sm.v[k][c]);
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
                uint32_t those[kR];
#pragma unroll
                for (int r = 0; r < kR; ++r) {
                    const bool is = lane < n && attends(sm.rows.want_row[r0 + r], sm.rows.want_col[r0 + r], sm.rows.below[r0 + r], key.place, key.row, key.col);
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
            const int row = r0 + r, at = part.tile * kSimtRows + row, member = part.seg == 0 ? at / p.group : 0;
            if (row >= part.n_rows) break;
            const size_t out = (size_t)(part.b + member) * p.heads + part.kv * p.group + at - member * p.group;
            const size_t whole = (size_t)part.seg * p.B * p.heads + out;
            for (int c = 0; c < kCols; ++c) {
                const int e = lane * kCols + c;
                if (e >= p.d) break;
                const float x = sum == 0.f ? 0.f : o[r][c];  // (a row that attends nothing here: whatever the others attend)
                if (state != kAll)
                    to[(size_t)(e / 4 * kSimtRows + row) * 4 + e % 4] = x;
                else if (part.grouped)
                    p.whole[whole * p.d + e] = x;
                else
                    put(sum == 0.f ? 0.f : x / sum, (T *)p.O + out * p.d + e);
            }
            if (lane > 0) continue;
            if (state != kAll)
                reinterpret_cast<float2 *>(to + (size_t)p.d * kSimtRows)[row] = make_float2(m[r], sum);
            else if (part.grouped)
                p.whole_stats[whole] = make_float2(m[r], sum);
            else
                p.LSE[out] = natural(m[r], sum);
        }
        if (tid == 0 && state != kGoesOn) {
            Joint *joint = joint_of(p, part.seg, part.kv, part.b, part.tile);
            if (state == kAll)
                joint->slot = -1;
            else
                *joint = joint_from(part, start, slot);
        }
    }
    if (look.bad) atomicOr(p.cache.status, kCacheBad);
}

// ---- the results of a row put together

// grid: (eight rows of a kv head, 16 columns); a lane has a row and four columns, the warps take a row's results in turn.
constexpr int kJoinRows = 8, kJoinWarps = 4;
template <typename T, int RT>
__global__ void __launch_bounds__(32 * kJoinWarps) shared_join_kernel(const __grid_constant__ SharedParams p) {
    __shared__ float4 s_sum[kJoinWarps][32];
    __shared__ float2 s_stat[kJoinWarps][32];
    ptx::launch_dependents();
    ptx::wait_prior_grid();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int per_kv = (p.B * p.group + kJoinRows - 1) / kJoinRows, kv = blockIdx.x / per_kv;
    const int at = (blockIdx.x - kv * per_kv) * kJoinRows + lane % kJoinRows, c4 = blockIdx.y * 4 + lane / kJoinRows;
    const int b = at / p.group, g = at - b * p.group;
    const bool exists = b < p.B && c4 * 4 < p.d;
    bool bad = false;
    // the results: of the shared tokens, and of the own ones
    const float *value[2];
    const float2 *stat[2];
    int64_t step[2];      // from one of them to the next, in floats
    int64_t from_first[2];  // from the first one to where the steps are counted from: its slot may be another than the next ones'
    int parts[2] = {0, 0};
    const size_t out = (size_t)b * p.heads + kv * p.group + g;
    bool direct = !exists;
    if (exists) {
        const Entry e = entry_of(p, b, &bad);
#pragma unroll
        for (int seg = 0; seg < 2; ++seg) {
            if (seg == 0 ? e.count == 0 : segment_of<RT>(p, e, b, 1).units == 0) continue;
            const int row = seg == 0 ? (b - e.first) * p.group + g : g, r = row % RT;
            const Joint joint = *joint_of(p, seg, kv, seg == 0 ? e.first : b, row / RT);
            if (joint.slot < 0) {
                if (e.count == 0) direct = true;
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
    if (__syncthreads_and(direct)) return;
    float m = -INFINITY, l = 0.f;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    if (!direct) {
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
    if (warp > 0 || direct) return;
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

constexpr int kBlocksPerSm = 2;
int rows_of_tile(const mate_cache_t *) { return kSimtRows; }
int own_tiles(const mate_cache_t *c) { return (c->heads / c->kv_heads + rows_of_tile(c) - 1) / rows_of_tile(c); }
int n_blocks(const mate_cache_t *c) { return kBlocksPerSm * n_sms(c->device); }

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

template <typename T, int DP>
int launch(const SharedParams &p, int device, int blocks, cudaStream_t st) {
    static SmemAttrOnce attr;
    const int rc = attr.ensure((const void *)shared_simt_kernel<T, DP>, sizeof(SimtSmem<DP>), device);
    if (rc != MATE_OK) return rc;
    cudaError_t e = launch_after(shared_simt_kernel<T, DP>, dim3((unsigned)blocks), kSimtThreads, sizeof(SimtSmem<DP>), st, p);
    const int64_t joins = (int64_t)p.kv_heads * (((int64_t)p.B * p.group + kJoinRows - 1) / kJoinRows);
    if (e == cudaSuccess)
        e = launch_after(shared_join_kernel<T, kSimtRows>, dim3((unsigned)joins, (unsigned)((p.d + 15) / 16)), 32 * kJoinWarps, 0, st, p);
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
    // units of the batch, shared and own, are 32-bit numbers, and so are the blocks of the second kernel
    if ((int64_t)B * cache->kv_heads * own_tiles(cache) > INT32_MAX / 2 / units_of(max_len) || (int64_t)B * cache->heads > INT32_MAX / 2)
        return MATE_ERR_UNSUPPORTED;
    const Workspace w = workspace_of(cache, B);
    if (!workspace || workspace_bytes < w.bytes) return MATE_ERR_WORKSPACE;
    if (!is_aligned(workspace, 256)) return MATE_ERR_ALIGNMENT;
    SharedParams p = {};
    p.cache = cache_args(cache, layer);
    p.Q = Q, p.q_batch = q_stride[0], p.q_head = q_stride[1];
    p.B = B, p.heads = cache->heads, p.kv_heads = cache->kv_heads, p.group = cache->heads / cache->kv_heads;
    p.d = cache->d, p.max_len = max_len, p.own_tiles = own_tiles(cache);
    p.seqs = seqs, p.row_ids = row_ids, p.col_ids = col_ids, p.groups = groups;
    p.scale_log2 = scale * kLog2e, p.O = O, p.LSE = LSE;
    for (int h = 0; h < cache->heads; ++h) p.views[h >> 4] |= (uint32_t)cache->head_view[h] << 2 * (h & 15);
    for (p.page_shift = 0; 1u << p.page_shift < (unsigned)cache->page_size;) ++p.page_shift;
    p.page_mul = (unsigned)((((uint64_t)1 << 32) * (((uint64_t)1 << p.page_shift) - cache->page_size)) / cache->page_size + 1);
    p.page16 = (unsigned)(cache->page_stride / vec), p.head16 = (unsigned)(cache->head_stride / vec), p.slot16 = (unsigned)(cache->slot_stride / vec);
    char *ws = static_cast<char *>(workspace);
    p.joints = reinterpret_cast<Joint *>(ws + w.joints);
    p.whole_stats = reinterpret_cast<float2 *>(ws + w.stats);
    p.whole = reinterpret_cast<float *>(ws + w.whole);
    p.parts = reinterpret_cast<float *>(ws + w.parts);
    cudaStream_t st = (cudaStream_t)stream;
    const int blocks = n_blocks(cache), device = cache->device;
    if (cache->dtype == MATE_F32) return cache->d <= 64 ? launch<float, 64>(p, device, blocks, st) : launch<float, 128>(p, device, blocks, st);
    return cache->d <= 64 ? launch<__nv_bfloat16, 64>(p, device, blocks, st) : launch<__nv_bfloat16, 128>(p, device, blocks, st);
}

}  // extern "C"

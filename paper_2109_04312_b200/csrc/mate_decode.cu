// Attention of one new token per sequence over the cached ones (mate_attn_decode): per sequence and kv head, the `group` query
// heads that share it (a block of up to 8 or 16 of them) against those cached tokens that one of them attends,
//     S = K q,  m = max S,  P = exp(S - m),  O = V^T P / sum P,  LSE = m + ln sum P.
//
// Bound by memory: a key and a value are read once for the whole group (4 d bytes in bf16 for 4 d flops per head), the ids of all
// cached tokens (4 or 8 bytes each, mostly from L2: the kv heads share them) decide which.  Hence
//   - a warp works alone: it looks through 32 tokens at a time (the next ones' ids and the pages behind them are on their way
//     meanwhile; four tokens per lane at a time took up to 5 % longer when tried), puts the places of those that count into a list, and
//     copies 16 bytes per lane and instruction from there into its own ring of two stages of 8 KB, one under way while the other is
//     read; twelve such warps to an SM keep 96 KB under way.  (Three stages and eight warps: cells 21.9 us instead of
//     18.8, 64 sequences 72.2 instead of 71.7, one long one 49.8 instead of 51.0.)  No block barrier until the sequence's part is done.  What nobody attends is never read, padding's keys and values included.
//   - the products are tensor-core ones (m16n8k16) with the keys as the 16 rows and the heads as the 8 columns, so that a group
//     of up to 8 costs one of them; the tensor pipe is 18 % busy while HBM is the limit.  The weights go from one product's
//     result to the other's operand by transposing 8 x 8 pieces between the lanes, as the sum of three bf16, which is all of their 24
//     bits (one table of 512 tokens 5.67 -> 5.94 us, cells 18.4 -> 18.7, 64 sequences 74.1 -> 74.6 against two, whose 16 bits showed
//     in one result of 500 that rounded to the neighbouring bf16, and in small differences of large weights).  fp32 caches: multiply-adds.
//   - blocks get equal shares of all sequences' tokens in units of kUnit (found by every block from the lengths, which the host does not
//     know), so one long sequence is spread over the GPU and short ones are put together.  A sequence that falls to several
//     blocks is joined by a second kernel from their partial results, in the order of its tokens: the same bits on every launch.
// The kernel lets the next one start at its end only: where three kernels in a row let the next one start at once, their blocks pile
// up, and the SMs do not get three blocks each (calls back to back: cells 23.4 us instead of 18.8, 64 sequences 73.4 instead of 71.7).
// Measured (one B200, calls back to back in a graph): 64 sequences of up to 4096 tokens, 8 kv heads of 128 elements, 399 MB, 71.7 us (5570
// GB/s); one of 131072 tokens, 4 kv heads, 269 MB, 51.0 us (5270 GB/s); cells of 16 tables of up to 8192 tokens 18.6 us, one table
// of 512 tokens 6.0 to 6.2 us: chains of dependent loads (sequence, length, page, ids, keys).
#include <cuda_bf16.h>

#include <cmath>
#include <type_traits>

#include "mate_cache.h"
#include "sm100_ptx.cuh"

namespace mate {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kManyWarps = 8;            // of a block that has an item and an SM to itself
constexpr int kUnit = 32 * kWarps;       // tokens of a unit of work: what the warps look through in one go
constexpr int kStage = 8192;             // bytes of a stage: keys, then values
constexpr int kAlign = 256;              // of the ring: the longest row of tensor-core operands
constexpr int kRing = 2;                 // stages of a warp
constexpr int kList = 64;                // entries of a warp's list of places: less than a stage, and one look
constexpr int kOver = 1;                 // units that an item costs besides its tokens (0, 1, 2, 3: 64 sequences 74.0, 71.7, 72.6, 74.6 us)
// Units of tokens up to which a block takes a whole item: for few items, and for many.  By the bound of the lengths that the host knows.
// Whole and shared out, us: one sequence of 12 heads of 64 elements and 512 tokens 6.0 and 7.7, 768 7.2 and 8.0, 1024 8.5 and 8.0; of 8 kv
// heads of 128 elements and 512 tokens 8.6 and 9.8, 768 10.6 and 9.9; four sequences of 12 heads and 1024 tokens 8.7 and 8.9, 1536 11.1 and
// 10.3; 40 of them, several items to an SM, 512 tokens 17.9 and 16.9, 1024 33.2 and 28.4; of up to 1000 tokens 14.3 and 15.2, and their cells
// 9.2 and 14.5.
constexpr int kWhole = 4, kWholeOfMany = 8, kMany = 32;
constexpr int kMaxHeads = 1024;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Where the results of an item are: [slot] of the block that begins it, then [0] of the next ones up to `last`.
struct Joint {
    int32_t slot, first, last, unused;  // slot < 0: it is done
};

struct DecodeParams {
    CacheArgs cache;
    const void *Q;
    int64_t q_batch, q_head;
    int B, heads, kv_heads, group, blocks_of_group, d, max_len;
    const int32_t *seqs, *row_ids, *col_ids;
    float scale_log2;  // scale / ln 2: weights are powers of two
    void *O;
    float *LSE;
    unsigned page16, head16, slot16;  // strides in 16 bytes; no place is beyond 2^32 of them
    unsigned page_mul, page_shift;  // x / page_size = (umulhi(x, page_mul) + x) >> page_shift for x < 2^31
    Joint *joints;         // [B][items]; null: a block per item
    float *partial;        // [grid][2][rows of a block][d + 2]
    uint32_t views[kMaxHeads / 16];  // two bits a head
};
__device__ __forceinline__ int page_index(const DecodeParams &p, int token) {
    return (int)((__umulhi((unsigned)token, p.page_mul) + (unsigned)token) >> p.page_shift);
}
__device__ __forceinline__ int view_at(const DecodeParams &p, int h) { return p.views[h >> 4] >> 2 * (h & 15) & 3; }

// ---- types

// DP: elements of a row, padded; NB: query heads of a block, in eights with bf16
template <typename T, int DP, int NB>
struct Shape {
    static constexpr int kRows = sizeof(T) == 2 ? 8 * NB : NB;              // query heads of a block
    static constexpr int kRowBytes = DP * (int)sizeof(T);
    static constexpr int kKeys = kStage / 2 / kRowBytes;                    // of a stage
    static constexpr int kChunks = kRowBytes / 16;
    // What a row's chunks are permuted by: eight rows of 16 bytes (bf16: ldmatrix) or the lanes of an eighth of a warp, of which
    // 32 / kKeys share a key (fp32), then fall into different banks.
    static constexpr int kSwizzle = sizeof(T) == 2 ? 1 : 32 / kKeys;
    // (Three need the registers below 168.  With 16 heads of 128 elements that spills 80 bytes, and 32 x 4096 tokens take 23.7 us instead of
    // 18.7; 8 heads of 128 elements of fp32 spill 24.)
    static constexpr int kBlocksPerSm = sizeof(T) == 2 && DP == 128 && NB == 2 ? 2 : 3;
    __device__ static int chunk_at(int key, int chunk) { return key * kRowBytes + ((chunk ^ (key * kSwizzle & 7)) << 4); }
};

__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void *src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}

// ---- shares of the work

// An item is one sequence's kv head and block of its group; items of a sequence follow one another.  Its units are numbered through
// over all items (fewer than 2^31, the host sees to that); block i of C gets units [i U / C, (i + 1) U / C).  The first kOver units
// stand for what an item costs whatever its length (none of its tokens belong to them); a share that ends among them ends in front
// of the item.  An item without tokens, which is written too, has one unit.
__host__ __device__ __forceinline__ int units_of(int len) { return len > 0 ? kOver + (len + kUnit - 1) / kUnit : 1; }
__device__ __forceinline__ unsigned share(unsigned U, unsigned C, unsigned i) { return U / C * i + U % C * i / C; }

// Tokens that entry b of the batch has to look through; none for an entry that is no sequence, or padding.
__device__ __forceinline__ int entry_len(const DecodeParams &p, int b, bool *bad) {
    const int s = p.seqs ? p.seqs[b] : b, q_row = p.row_ids[b], q_col = p.col_ids[b];
    if (!in_range(s, p.cache.seqs)) {
        *bad = true;
        return 0;
    }
    const int len = clip_len(p.cache.lens[s], p.max_len, bad);
    return q_row < 0 || q_col < 0 ? 0 : len;
}

struct Start {
    unsigned total, before;  // units of the batch; of the entries in front of `entry`
    unsigned blocks;         // that get any: no more than there are units
    int entry;
};
// All threads call it: the entry that the block's first unit belongs to.
__device__ Start find_start(const DecodeParams &p, int items) {
    __shared__ unsigned s_sum[kWarps];
    __shared__ Start s_start;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (p.B + kThreads - 1) / kThreads, b0 = min(p.B, tid * per), b1 = min(p.B, b0 + per);
    bool bad = false;
    unsigned own = 0;
    for (int b = b0; b < b1; ++b) own += units_of(entry_len(p, b, &bad));
    own *= items;
    unsigned sum = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned y = __shfl_up_sync(~0u, sum, o);
        if (lane >= o) sum += y;
    }
    if (lane == 31) s_sum[warp] = sum;
    __syncthreads();
    unsigned total = 0, before = sum - own;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += s_sum[w];
        total += s_sum[w];
    }
    const unsigned blocks = min(total, gridDim.x), at = share(total, blocks, min(blockIdx.x, blocks - 1));
    if (at >= before && at < before + own) {
        int b = b0;
        for (; b < b1 - 1; ++b) {
            const unsigned n = units_of(entry_len(p, b, &bad)) * items;
            if (at < before + n) break;
            before += n;
        }
        s_start = {total, before, blocks, b};
    }
    if (bad && blockIdx.x == 0) atomicOr(p.cache.status, kCacheBad);
    __syncthreads();
    return s_start;
}

// A part of an item: units [u0, u1) of entry b's kv head and block of the group.
struct Part {
    int b, item, u0, u1;
    bool whole;
};
// Walks the parts of a block's share.  (It comes to an end whatever it finds: every part takes a unit off the share.)
struct Walk {
    int b, item, u;  // next unit: of entry b, item, unit u
    int left;        // units of the share
};
__device__ __forceinline__ bool next_part(const DecodeParams &p, int items, Walk &w, Part &part, int *len) {
    if (w.left <= 0 || w.b >= p.B) return false;
    bool bad = false;
    *len = entry_len(p, w.b, &bad);
    const int n = units_of(*len);
    part.b = w.b, part.item = w.item, part.u0 = w.u;
    part.u1 = min(n, w.u + w.left);
    if (part.u1 <= kOver && part.u1 < n) return false;
    part.whole = part.u0 == 0 && part.u1 == n;
    w.left -= max(1, part.u1 - part.u0);
    w.u = 0;
    if (++w.item == items) w.item = 0, ++w.b;
    return true;
}

__device__ __forceinline__ void put(float x, float *y) { *y = x; }
__device__ __forceinline__ void put(float x, __nv_bfloat16 *y) { *y = __float2bfloat16_rn(x); }

// ---- the loading side of a warp

struct Meta {  // of a stage
    int n, end;  // keys; the last stage of a part
    uint32_t by_row, by_col;
    int b, item, state, units;  // the part
};
enum { kNoPart = 0, kAll = 1, kBegins = 2, kGoesOn = 3 };  // Meta.state: behind the last one; an item; its first units; others

template <typename T, int DP, int NB, int W>
struct Loader {
    static constexpr int kStep = 32 * W;  // tokens that the block's warps look through in one go
    using S = Shape<T, DP, NB>;
    const DecodeParams &p;
    uint32_t *list;  // places, in 16 bytes from the cache's beginning
    uint8_t *marks;  // 1: attended by row, 2: by column
    Meta *meta;
    uint32_t ring;
    int lane, warp, items;
    Walk walk;
    // the present part
    Part part;
    bool active;
    int s, prefix, q_row, q_col, end;
    unsigned head_at;
    bool text, need_row, need_col;
    int next;                           // first of the 32 tokens that are looked at next; 32 of every kStep are the warp's
    bool there;                         // the lane's token there exists; its ids have been asked for
    unsigned at;
    int row, col;
    int page;                           // page of the one behind it, which has been asked for too
    bool bad;
    int pending, list_at, filled;       // list (list_at: a multiple of a stage's keys); stages so far

    // page of the lane's token `j`
    __device__ void ask_page(int j) { page = j < end ? p.cache.table[(size_t)s * p.cache.width + page_index(p, j)] : -1; }
    // The same of its first token of entry b, while the sequence's length is on its way: kManyWarps only, whose block has one item and
    // begins with its first token (512 tokens, 12 heads of 64 elements, 6.22 -> 6.02 us).
    __device__ void ask_early(int b) {
        const int sequence = p.seqs ? p.seqs[b] : b, j = 32 * warp + lane;
        page = in_range(sequence, p.cache.seqs) && j < p.max_len ? p.cache.table[(size_t)sequence * p.cache.width + page_index(p, j)] : -1;
    }
    // ids of the lane's token of `next`, whose page has come
    __device__ void ask_ids() {
        const int j = next + lane;
        there = j < end && in_range(page, p.cache.pages);
        if (j < end && !there) bad = true;
        if (!there) return;
        const int slot = j - page_index(p, j) * p.cache.page_size, id = page * p.cache.page_size + slot;
        if (need_row) row = p.cache.row_ids[id];
        if (need_col) col = p.cache.col_ids[id];
        at = (unsigned)page * p.page16 + (unsigned)slot * p.slot16 + head_at;
    }
    __device__ void begin() {
        int len, kv, h0, n;
        for (;;) {
            active = next_part(p, items, walk, part, &len);
            if (!active) return;
            kv = part.item / p.blocks_of_group;
            const int block = part.item - kv * p.blocks_of_group;
            h0 = kv * p.group + block * S::kRows, n = min(S::kRows, p.group - block * S::kRows);
            if (len > 0) break;
            // an item without tokens is done with here
            const size_t row = (size_t)part.b * p.heads + h0;
            if (warp == 0) {
                for (int i = lane; i < n * p.d; i += 32) put(0.f, (T *)p.O + row * p.d + i);
                for (int i = lane; i < n; i += 32) p.LSE[row + i] = -INFINITY;
                if (p.joints && lane == 0) p.joints[part.b * items + part.item].slot = -1;
            }
        }
        s = p.seqs ? p.seqs[part.b] : part.b;
        next = max(0, part.u0 - kOver) * kUnit + 32 * warp;
        end = min(len, (part.u1 - kOver) * kUnit);
        if (W != kManyWarps) ask_page(next + lane);
        q_row = p.row_ids[part.b], q_col = p.col_ids[part.b];
        prefix = p.cache.prefix[s];
        text = q_row == MATE_ID_TEXT || q_col == MATE_ID_TEXT;
        head_at = (unsigned)kv * p.head16;
        need_row = need_col = false;
        for (int i = 0; i < n; ++i) {
            const int v = view_at(p, h0 + i);
            need_row |= v != MATE_VIEW_COL;
            need_col |= v != MATE_VIEW_ROW;
        }
        if (text) need_row = true, need_col = false;  // padding has neither
        list_at = 0;
        ask_ids();
        ask_page(next + kStep + lane);
    }
    // One look at 32 tokens: those that count go onto the list, the next ones' ids are asked for.
    __device__ void look() {
        const bool all = text || next + lane < prefix;
        const bool by_row = there && need_row && row >= 0 && (all || row == MATE_ID_TEXT || row == q_row);
        const bool by_col = there && need_col && col >= 0 && (all || col == MATE_ID_TEXT || col == q_col);
        const unsigned counts = __ballot_sync(~0u, by_row || by_col);
        if (by_row || by_col) {
            const int to = (list_at + pending + __popc(counts & ((1u << lane) - 1))) & (kList - 1);
            list[to] = at;
            if (need_row && need_col) marks[to] = (by_row ? 1 : 0) | (by_col ? 2 : 0);
        }
        pending += __popc(counts);
        next += kStep;
        if (next < end) {
            ask_ids();
            ask_page(next + kStep + lane);
        }
    }
    // Copies of the next stage are put under way (or, at the end of the share, none: the groups are counted).
    __device__ void fill() {
        const int slot = filled % kRing;
        if (active) {
            while (pending < S::kKeys && next < end) look();
            __syncwarp();
            const int n = min(pending, S::kKeys);
            const bool last = pending <= S::kKeys && next >= end;
            uint32_t by_row = n < 32 ? (1u << n) - 1 : ~0u, by_col = by_row;
            if (need_row && need_col) {  // heads of both kinds: who attends what
                const int mine = lane < n ? marks[list_at + lane] : 0;
                by_row = __ballot_sync(~0u, mine & 1), by_col = __ballot_sync(~0u, mine & 2);
            }
            if (lane == 0)
                meta[slot] = {n, last, by_row, by_col, part.b, part.item, part.whole ? kAll : part.u0 == 0 ? kBegins : kGoesOn, part.u1 - part.u0};
            // a lane copies a 16-byte column of eight keys
            const int chunk = lane % S::kChunks, first = lane / S::kChunks * 8;
            if (n > 0 && chunk < p.d * (int)sizeof(T) / 16) {
                const uint4 lo = *reinterpret_cast<const uint4 *>(list + list_at + first), hi = *reinterpret_cast<const uint4 *>(list + list_at + first + 4);
                const unsigned from[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
                const char *k = (const char *)p.cache.k + chunk * 16, *v = (const char *)p.cache.v + chunk * 16;
                const uint32_t to = ring + slot * kStage + first * S::kRowBytes;
                if (n == S::kKeys) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t dst = to + S::chunk_at(i, chunk);  // (first is a multiple of 8: the swizzle goes by i)
                        ptx::cp_async16(dst, k + (size_t)from[i] * 16);
                        ptx::cp_async16(dst + kStage / 2, v + (size_t)from[i] * 16);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const bool is = first + i < n;
                        const uint32_t dst = to + S::chunk_at(i, chunk);
                        cp_async16_or_zero(dst, k + (is ? (size_t)from[i] * 16 : 0), is);
                        cp_async16_or_zero(dst + kStage / 2, v + (is ? (size_t)from[i] * 16 : 0), is);
                    }
                }
            }
            list_at = (list_at + n) & (kList - 1);
            pending -= n;
            __syncwarp();  // the list has been read
            if (last) begin();
        } else if (lane == 0) {
            meta[slot] = {0, 1, 0u, 0u, 0, 0, kNoPart, 0};
        }
        ++filled;
        cp_async_commit();
    }
};

// ---- the reading side: running maximum, sum and weighted sum of values of a block's query heads

// Whether some heads of a stage attend keys that others do not (whose weight there is 0), and a value is Inf or NaN, for which 0 times it is not
// 0: the warp then leaves such keys out one by one.  All lanes call it.  (Doing so without a look: 8 heads, half of them by row and half by
// column, of 64 tables of up to 8192 tokens 24.6 us, with a look first 21.9, never 21.3; in fp32, 32 of
// up to 4096, 34.9, 30.0 and 29.0.)
template <typename T>
__device__ __forceinline__ bool leave_out(const Meta &meta, const char *values, int lane) {
    if (meta.by_row == meta.by_col) return false;
    float zero = 0.f;
    __nv_bfloat162 zeros = __floats2bfloat162_rn(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kStage / 2 / 16; i += 32) {
        const uint4 x = *reinterpret_cast<const uint4 *>(values + (i + lane) * 16);
        for (uint32_t w : {x.x, x.y, x.z, x.w}) {
            if (sizeof(T) == 4)
                zero = fmaf(__uint_as_float(w), 0.f, zero);
            else
                zeros = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&w), __floats2bfloat162_rn(0.f, 0.f), zeros);
        }
    }
    return __any_sync(~0u, sizeof(T) == 4 ? zero != 0.f : __low2float(zeros) != 0.f || __high2float(zeros) != 0.f);
}

template <typename T, int DP, int NB>
struct Reader;

template <int DP, int NB>
struct Reader<__nv_bfloat16, DP, NB> {
    using S = Shape<__nv_bfloat16, DP, NB>;
    static constexpr int kTiles = S::kKeys / 16;
    static constexpr int kParts = 3;  // bf16 numbers whose sum is a weight
    uint32_t q[DP / 16][NB][2];      // B operand: k = element, n = head
    float o[DP / 16][NB][4];         // rows: elements lane / 4 (+ 8), columns: heads 2 (lane % 4) + {0, 1}
    float m[NB][2], l[NB][2];        // of those heads; l: of the lane's own keys
    uint32_t rows_of[NB][2], cols_of[NB][2];  // all ones where the head attends by row / by column

    __device__ void begin(const DecodeParams &p, int b, int h0, int n_rows, int lane, float *) {
        const __nv_bfloat16 *Q = (const __nv_bfloat16 *)p.Q + b * p.q_batch;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int r = nb * 8 + lane / 4;
#pragma unroll
            for (int k = 0; k < DP / 16; ++k)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int e = k * 16 + half * 8 + 2 * (lane & 3);
                    q[k][nb][half] = r < n_rows && e < p.d ? *reinterpret_cast<const uint32_t *>(Q + (h0 + r) * p.q_head + e) : 0u;
                }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int h = nb * 8 + 2 * (lane & 3) + c, v = view_at(p, h < n_rows ? h0 + h : h0);
                rows_of[nb][c] = v != MATE_VIEW_COL ? ~0u : 0u;
                cols_of[nb][c] = v != MATE_VIEW_ROW ? ~0u : 0u;
                m[nb][c] = -INFINITY, l[nb][c] = 0.f;
            }
        }
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[k][nb][i] = 0.f;
    }
    __device__ void add(const DecodeParams &p, const char *at, const Meta &meta, int lane, float *) {
        const uint32_t stage = ptx::smem_u32(at);
        const bool apart = leave_out<__nv_bfloat16>(meta, at + kStage / 2, lane);
        float s[kTiles][NB][4];
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[t][nb][i] = 0.f;
        // (a stage begins at a multiple of its rows' length, so the swizzled column 2 k + i of a lane is column i's address ^ 32 k)
        const uint32_t key_at = stage + S::chunk_at(lane & 15, lane >> 4);
        const uint32_t value_at = stage + kStage / 2 + S::chunk_at((lane & 7) + (lane >> 4) * 8, lane >> 3 & 1);
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                uint32_t a[4];
                ldmatrix4(a, (key_at ^ 32 * k) + t * 16 * S::kRowBytes);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) mma16816(s[t][nb], a, q[k][nb]);
            }
        constexpr uint32_t kFull = S::kKeys < 32 ? (1u << S::kKeys) - 1 : ~0u;
        const bool all = (meta.by_row & meta.by_col) == kFull;
        uint32_t w[kParts][kTiles][NB][2];
        float keep[NB][2];
        bool moved = false;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float top = m[nb][c];
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int half = 0; half < 2; ++half) s[t][nb][2 * half + c] *= p.scale_log2;
                if (!all) {
                    const uint32_t counts = ((meta.by_row & rows_of[nb][c]) | (meta.by_col & cols_of[nb][c])) >> lane / 4;
#pragma unroll
                    for (int t = 0; t < kTiles; ++t)
#pragma unroll
                        for (int half = 0; half < 2; ++half)
                            if (!(counts >> (t * 16 + half * 8) & 1)) s[t][nb][2 * half + c] = -INFINITY;
                }
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int half = 0; half < 2; ++half) top = fmaxf(top, s[t][nb][2 * half + c]);
                top = fmaxf(top, __shfl_xor_sync(~0u, top, 4));
                top = fmaxf(top, __shfl_xor_sync(~0u, top, 8));
                top = fmaxf(top, __shfl_xor_sync(~0u, top, 16));
                const float base = top == -INFINITY ? 0.f : top;
                moved |= top != m[nb][c];
                keep[nb][c] = ptx::ex2(m[nb][c] - base);
                m[nb][c] = top;
                float sum = 0.f;
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        float &x = s[t][nb][2 * half + c];
                        x = ptx::ex2(x - base);
                        sum += x;
                    }
                l[nb][c] = fmaf(l[nb][c], keep[nb][c], sum);
            }
        if (__any_sync(~0u, moved)) {
#pragma unroll
            for (int k = 0; k < DP / 16; ++k)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[k][nb][i] *= keep[nb][i & 1];
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    float x = s[t][nb][2 * half], y = s[t][nb][2 * half + 1];
#pragma unroll
                    for (int i = 0; i < kParts; ++i) {
                        const uint32_t xy = ptx::cvt_bf16x2(x, y);
                        w[i][t][nb][half] = transpose8(xy);
                        x -= __uint_as_float(xy << 16), y -= __uint_as_float(xy & 0xffff0000u);
                    }
                }
        if (!apart) {
#pragma unroll
            for (int k = 0; k < DP / 16; ++k)
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    uint32_t a[4];
                    ldmatrix4_trans(a, (value_at ^ 32 * k) + t * 16 * S::kRowBytes);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int i = 0; i < kParts; ++i) mma16816(o[k][nb], a, w[i][t][nb]);
                }
            return;
        }
        // One product for each kind of heads, with 0 for the values that it leaves out, of which the heads of that kind keep theirs.
#pragma unroll 1
        for (int view = MATE_VIEW_ROW; view <= MATE_VIEW_EITHER; ++view) {
            const uint32_t kept = (view != MATE_VIEW_COL ? meta.by_row : 0u) | (view != MATE_VIEW_ROW ? meta.by_col : 0u);
            bool mine[NB][2], any = false;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    mine[nb][c] = (rows_of[nb][c] != 0u) == (view != MATE_VIEW_COL) && (cols_of[nb][c] != 0u) == (view != MATE_VIEW_ROW);
                    any |= mine[nb][c];
                }
            if (!__any_sync(~0u, any)) continue;
            uint32_t keep_values[kTiles][2];  // of a lane's two keys in an operand's register
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint32_t two = kept >> (t * 16 + half * 8 + 2 * (lane & 3));
                    keep_values[t][half] = (two & 1 ? 0xffffu : 0u) | (two & 2 ? 0xffff0000u : 0u);
                }
#pragma unroll
            for (int k = 0; k < DP / 16; ++k) {
                float sum[NB][4];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[nb][i] = o[k][nb][i];
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    uint32_t a[4];
                    ldmatrix4_trans(a, (value_at ^ 32 * k) + t * 16 * S::kRowBytes);
#pragma unroll
                    for (int i = 0; i < 4; ++i) a[i] &= keep_values[t][i / 2];
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int i = 0; i < kParts; ++i) mma16816(sum[nb], a, w[i][t][nb]);
                }
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[k][nb][i] = mine[nb][i & 1] ? sum[nb][i] : o[k][nb][i];
            }
        }
    }
    // The warp's result: [n_rows][d] un-normalised, then maxima and sums.
    __device__ void store(float *out, float *stats, int n_rows, int d, int lane) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float sum = l[nb][c];
                sum += __shfl_xor_sync(~0u, sum, 4);
                sum += __shfl_xor_sync(~0u, sum, 8);
                sum += __shfl_xor_sync(~0u, sum, 16);
                const int r = nb * 8 + 2 * (lane & 3) + c;
                if (r >= n_rows) continue;
                if (lane < 4) stats[2 * r] = m[nb][c], stats[2 * r + 1] = sum;
#pragma unroll
                for (int k = 0; k < DP / 16; ++k)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int e = k * 16 + half * 8 + lane / 4;
                        if (e < d) out[r * d + e] = o[k][nb][2 * half + c];
                    }
            }
    }
};

template <int DP, int NB>
struct Reader<float, DP, NB> {
    using S = Shape<float, DP, NB>;
    static constexpr int kShare = 32 / S::kKeys;  // lanes that share a key
    static constexpr int kCols = DP / 32;         // columns of a lane
    float m[S::kRows], l[S::kRows], o[S::kRows][kCols];
    uint32_t views;  // two bits a head

    // `own`: queries [kRows][DP] (of the block; every warp writes the same), then the warps' weights [kRows][kKeys] each
    __device__ void begin(const DecodeParams &p, int b, int h0, int n_rows, int lane, float *own) {
        const float *Q = (const float *)p.Q + b * p.q_batch;
        __syncwarp();
#pragma unroll
        for (int i = 0; i < S::kRows * DP / 32; ++i) {
            const int r = (i * 32 + lane) / DP, e = (i * 32 + lane) % DP;
            own[i * 32 + lane] = r < n_rows && e < p.d ? Q[(h0 + r) * p.q_head + e] : 0.f;
        }
        __syncwarp();
        views = 0;
#pragma unroll
        for (int r = 0; r < S::kRows; ++r) {
            views |= (uint32_t)(r < n_rows ? view_at(p, h0 + r) : MATE_VIEW_EITHER) << 2 * r;
            m[r] = -INFINITY, l[r] = 0.f;
#pragma unroll
            for (int c = 0; c < kCols; ++c) o[r][c] = 0.f;
        }
    }
    __device__ uint32_t attended(const Meta &meta, int r) const {  // keys that head r attends
        const int v = views >> 2 * r & 3;
        return (v != MATE_VIEW_COL ? meta.by_row : 0u) | (v != MATE_VIEW_ROW ? meta.by_col : 0u);
    }
    __device__ static void value(const char *stage, int key, int lane, float (&v)[kCols]) {  // the lane's columns
        const char *at = stage + kStage / 2 + S::chunk_at(key, lane * kCols / 4) + (lane * kCols % 4) * 4;
        if (kCols == 4) {
            const float4 x = *reinterpret_cast<const float4 *>(at);
            v[0] = x.x, v[1] = x.y, v[kCols - 2] = x.z, v[kCols - 1] = x.w;
        } else {
            const float2 x = *reinterpret_cast<const float2 *>(at);
            v[0] = x.x, v[1] = x.y;
        }
    }
    // (all kRows rows, also where the block has fewer heads: branches between them cost more than the multiply-adds)
    __device__ void add(const DecodeParams &p, const char *stage, const Meta &meta, int lane, float *own) {
        const int key = lane / kShare, part = lane % kShare;
        float *weights = own + S::kRows * (DP + (threadIdx.x >> 5) * S::kKeys);
        float s[S::kRows];
#pragma unroll
        for (int r = 0; r < S::kRows; ++r) s[r] = 0.f;
#pragma unroll
        for (int i = 0; i < S::kChunks / kShare; ++i) {
            const int chunk = i * kShare + part;
            const float4 k = *reinterpret_cast<const float4 *>(stage + S::chunk_at(key, chunk));
#pragma unroll
            for (int r = 0; r < S::kRows; ++r) {
                const float4 x = *reinterpret_cast<const float4 *>(own + r * DP + chunk * 4);
                s[r] = fmaf(x.x, k.x, fmaf(x.y, k.y, fmaf(x.z, k.z, fmaf(x.w, k.w, s[r]))));
            }
        }
#pragma unroll
        for (int step = 1; step < kShare; step <<= 1)
#pragma unroll
            for (int r = 0; r < S::kRows; ++r) s[r] += __shfl_xor_sync(~0u, s[r], step);
        float top[S::kRows];
#pragma unroll
        for (int r = 0; r < S::kRows; ++r) {
            s[r] = attended(meta, r) >> key & 1 ? s[r] * p.scale_log2 : -INFINITY;
            top[r] = fmaxf(m[r], s[r]);
        }
#pragma unroll
        for (int step = kShare; step < 32; step <<= 1)
#pragma unroll
            for (int r = 0; r < S::kRows; ++r) top[r] = fmaxf(top[r], __shfl_xor_sync(~0u, top[r], step));
#pragma unroll
        for (int r = 0; r < S::kRows; ++r) {
            const float base = top[r] == -INFINITY ? 0.f : top[r], keep = ptx::ex2(m[r] - base), w = ptx::ex2(s[r] - base);
            m[r] = top[r];
            l[r] = fmaf(l[r], keep, w);  // (kShare lanes count the same key)
#pragma unroll
            for (int c = 0; c < kCols; ++c) o[r][c] *= keep;
            if (part == 0) weights[r * S::kKeys + key] = w;
        }
        __syncwarp();
        if (!leave_out<float>(meta, stage + kStage / 2, lane)) {
#pragma unroll
            for (int k0 = 0; k0 < S::kKeys; k0 += 4) {
                float v[4][kCols];
#pragma unroll
                for (int k = 0; k < 4; ++k) value(stage, k0 + k, lane, v[k]);
#pragma unroll
                for (int r = 0; r < S::kRows; ++r) {
                    const float4 w = *reinterpret_cast<const float4 *>(weights + r * S::kKeys + k0);
#pragma unroll
                    for (int c = 0; c < kCols; ++c)
                        o[r][c] = fmaf(w.x, v[0][c], fmaf(w.y, v[1][c], fmaf(w.z, v[2][c], fmaf(w.w, v[3][c], o[r][c]))));
                }
            }
        } else {
#pragma unroll 1
            for (int i = 0; i < S::kKeys; ++i) {
                const int k = i ^ 3;  // (in the order of the sums above: the same bits as without the others' keys)
                float v[kCols];
                value(stage, k, lane, v);
#pragma unroll
                for (int r = 0; r < S::kRows; ++r)
                    if (attended(meta, r) >> k & 1) {
#pragma unroll
                        for (int c = 0; c < kCols; ++c) o[r][c] = fmaf(weights[r * S::kKeys + k], v[c], o[r][c]);
                    }
            }
        }
        __syncwarp();  // the weights have been read
    }
    __device__ void store(float *out, float *stats, int n_rows, int d, int lane) {
#pragma unroll
        for (int r = 0; r < S::kRows; ++r) {
            if (r >= n_rows) break;
            float sum = lane % kShare == 0 ? l[r] : 0.f;
#pragma unroll
            for (int step = 1; step < 32; step <<= 1) sum += __shfl_xor_sync(~0u, sum, step);
            if (lane == 0) stats[2 * r] = m[r], stats[2 * r + 1] = sum;
#pragma unroll
            for (int c = 0; c < kCols; ++c)
                if (lane * kCols + c < d) out[r * d + lane * kCols + c] = o[r][c];
        }
    }
};

// Bytes of shared memory behind the ring: fp32's queries and weights.
template <typename T, int DP, int NB, int W>
constexpr int kExtra = sizeof(T) == 4 ? 4 * Shape<T, DP, NB>::kRows * (DP + W * Shape<T, DP, NB>::kKeys) : 0;

// W = kManyWarps: every block takes an item
template <typename T, int DP, int NB, int W>
__global__ void __launch_bounds__(32 * W, W == kWarps ? Shape<T, DP, NB>::kBlocksPerSm : 1) decode_kernel(const __grid_constant__ DecodeParams p) {
    using S = Shape<T, DP, NB>;
    extern __shared__ char smem_raw[];
    char *smem = smem_raw + (-ptx::smem_u32(smem_raw) & (kAlign - 1));
    __shared__ __align__(16) uint32_t s_list[W][kList];
    __shared__ uint8_t s_marks[W][kList];
    __shared__ Meta s_meta[W][kRing];
    __shared__ __align__(8) float s_stats[W][2 * S::kRows];
    __shared__ int s_out_at[W];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, items = p.kv_heads * p.blocks_of_group;
    const int max_rows = min(S::kRows, p.group);
    float *own = reinterpret_cast<float *>(smem + W * kRing * kStage);
    if (p.d < DP)  // columns that no copy writes
        for (int i = tid; i < W * kRing * kStage / 16; i += 32 * W) reinterpret_cast<uint4 *>(smem)[i] = make_uint4(0, 0, 0, 0);
    ptx::wait_prior_grid();

    Loader<T, DP, NB, W> load = {p, s_list[warp], s_marks[warp], s_meta[warp], ptx::smem_u32(smem) + warp * kRing * kStage, lane, warp, items};
    load.bad = false, load.pending = load.list_at = load.filled = 0;
    Walk walk;
    Start start = {};
    if (W == kWarps && p.joints) {
        start = find_start(p, items);
        if (blockIdx.x >= start.blocks) return;
        const unsigned at = share(start.total, start.blocks, blockIdx.x);
        walk.left = (int)(share(start.total, start.blocks, blockIdx.x + 1) - at);
        bool bad = false;
        const unsigned n = units_of(entry_len(p, start.entry, &bad));
        walk.b = start.entry;
        walk.item = min(items - 1, (int)((at - start.before) / n));
        walk.u = (int)(at - start.before - walk.item * n);
        if (walk.u <= kOver) walk.left += walk.u, walk.u = 0;
    } else {
        bool bad = false;
        walk.b = blockIdx.x / items, walk.item = blockIdx.x - walk.b * items, walk.u = 0;
        if (W == kManyWarps) load.ask_early(walk.b);
        walk.left = units_of(entry_len(p, walk.b, &bad));
        if (bad && tid == 0) atomicOr(p.cache.status, kCacheBad);
        __syncthreads();
    }

    load.walk = walk;
    load.begin();
    for (int i = 0; i < kRing - 1; ++i) load.fill();

    __syncwarp();

    Reader<T, DP, NB> read;
    bool first = true;
    for (int t = 0;;) {
        Meta meta = s_meta[warp][t % kRing];
        if (meta.state == kNoPart) break;
        const Meta part = meta;
        const int kv = part.item / p.blocks_of_group, block = part.item - kv * p.blocks_of_group;
        const int h0 = kv * p.group + block * S::kRows, n_rows = min(S::kRows, p.group - block * S::kRows);
        read.begin(p, part.b, h0, n_rows, lane, own);
        for (bool more = true; more; ++t) {
            cp_async_wait<kRing - 2>();
            __syncwarp();
            load.fill();
            meta = s_meta[warp][t % kRing];
            if (meta.n > 0) read.add(p, smem + (warp * kRing + t % kRing) * kStage, meta, lane, own);
            more = !meta.end;
        }
        __syncwarp();
        // the warp's result goes into the stage that was read last, which the next fill() is the first to write
        static_assert(S::kRows * DP * 4 <= kStage, "a warp's result fits a stage");
        const int out_at = (t - 1) % kRing * kStage;
        read.store(reinterpret_cast<float *>(smem + warp * kRing * kStage + out_at), s_stats[warp], n_rows, p.d, lane);
        if (lane == 0) s_out_at[warp] = warp * kRing * kStage + out_at;
        __syncthreads();
        // the warps' results together: the whole item's, or a partial one
        const int slot = first ? 0 : 1, e = tid % DP;
        float *to = p.partial + (size_t)(2 * blockIdx.x + slot) * max_rows * (p.d + 2);
#pragma unroll 4
        for (int r = tid / DP; r < n_rows; r += 32 * W / DP) {
            float2 stat[W];
            float x[W], top = -INFINITY;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                stat[w] = *reinterpret_cast<const float2 *>(&s_stats[w][2 * r]);
                x[w] = e < p.d ? *reinterpret_cast<const float *>(smem + s_out_at[w] + 4 * (r * p.d + e)) : 0.f;
                top = fmaxf(top, stat[w].x);
            }
            const float base = top == -INFINITY ? 0.f : top;
            float sum = 0.f, y = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float f = ptx::ex2(stat[w].x - base);
                sum = fmaf(f, stat[w].y, sum);
                y = fmaf(f, x[w], y);
            }
            if (e >= p.d) continue;
            if (part.state == kAll) {
                const size_t row = (size_t)part.b * p.heads + h0 + r;
                put(sum == 0.f ? 0.f : y / sum, (T *)p.O + row * p.d + e);
                if (e == 0) p.LSE[row] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
            } else {
                to[r * (p.d + 2) + 2 + e] = y;
                if (e == 0) *reinterpret_cast<float2 *>(to + r * (p.d + 2)) = make_float2(top, sum);
            }
        }
        __syncthreads();
        if (p.d < DP)
            for (int i = lane; i < kStage / 16; i += 32) reinterpret_cast<uint4 *>(smem + warp * kRing * kStage + out_at)[i] = make_uint4(0, 0, 0, 0);
        first = false;
        if (W == kWarps && p.joints && tid == 0) {
            Joint &joint = p.joints[part.b * items + part.item];
            if (part.state == kAll) joint.slot = -1;
            if (part.state == kBegins) {  // the share's last part: who has the item's last unit?
                bool bad = false;
                const int64_t end = (int64_t)share(start.total, start.blocks, blockIdx.x + 1) - part.units + units_of(entry_len(p, part.b, &bad));
                joint = {slot, (int)blockIdx.x, (int)min((end * start.blocks - 1) / start.total, (int64_t)start.blocks - 1), 0};
            }
        }
    }
    ptx::launch_dependents();
    cp_async_wait<0>();
    if (load.bad) atomicOr(p.cache.status, kCacheBad);
}

// Joins the partial results of an item that fell to several blocks of the kernel before.  grid: (item, row of its block of the group)
template <typename T, int kN>
__global__ void __launch_bounds__(kN) join_kernel(const __grid_constant__ DecodeParams p, int block_rows) {
    extern __shared__ float s_weight[];  // of every part
    __shared__ float s_red[2][kN / 32], s_sum[2 * kN];
    ptx::launch_dependents();
    ptx::wait_prior_grid();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = blockIdx.y, width = p.d + 2, items = p.kv_heads * p.blocks_of_group;
    const Joint joint = p.joints[blockIdx.x];
    const int b = blockIdx.x / items, item = blockIdx.x - b * items;
    const int kv = item / p.blocks_of_group, part = item - kv * p.blocks_of_group, max_rows = min(block_rows, p.group);
    const int parts = joint.last - joint.first + 1;
    if (joint.slot < 0 || r >= p.group - part * block_rows) return;
    auto result = [&](int i) { return p.partial + ((size_t)(2 * (joint.first + i) + (i == 0 ? joint.slot : 0)) * max_rows + r) * width; };
    // pairs of columns; groups of threads take the parts in turn, the first kBatch of them ahead of the weights
    constexpr int kBatch = 8;
    const int pairs = p.d / 2, groups = kN / pairs, group = tid / pairs, c = tid - group * pairs;
    float2 v[kBatch];
    auto load = [&](int i0) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (i0 + j * groups < parts) v[j] = *reinterpret_cast<const float2 *>(result(i0 + j * groups) + 2 + 2 * c);
    };
    if (group < groups) load(group);
    float top = -INFINITY;
    for (int i = tid; i < parts; i += kN) top = fmaxf(top, s_weight[i] = *result(i));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
    if (lane == 0) s_red[0][warp] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kN / 32; ++w) top = fmaxf(top, s_red[0][w]);
    const float base = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    for (int i = tid; i < parts; i += kN) {
        const float w = ptx::ex2(s_weight[i] - base);
        s_weight[i] = w;
        sum = fmaf(w, result(i)[1], sum);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    if (lane == 0) s_red[1][warp] = sum;
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < kN / 32; ++w) sum += s_red[1][w];
    if (group < groups) {
        float x = 0.f, y = 0.f;
        for (int i0 = group; i0 < parts; i0 += kBatch * groups) {
            if (i0 > group) load(i0);
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                if (i0 + j * groups >= parts) break;
                const float w = s_weight[i0 + j * groups];
                x = fmaf(w, v[j].x, x), y = fmaf(w, v[j].y, y);
            }
        }
        s_sum[2 * tid] = x, s_sum[2 * tid + 1] = y;
    }
    __syncthreads();
    const size_t row = (size_t)b * p.heads + kv * p.group + part * block_rows + r;
    if (tid < p.d) {
        float z = 0.f;
        for (int g = 0; g < groups; ++g) z += s_sum[g * p.d + tid];
        put(sum == 0.f ? 0.f : z / sum, (T *)p.O + row * p.d + tid);
    }
    if (tid == 0) p.LSE[row] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

// ---- host

// Query heads of a block: 8 or 16 with bf16, 2, 4 or 8 with fp32
int block_rows(const mate_cache_t *c) {
    const int group = c->heads / c->kv_heads;
    return c->dtype == MATE_BF16 ? group > 8 ? 16 : 8 : group > 4 ? 8 : group > 2 ? 4 : 2;
}
int blocks_of_group(const mate_cache_t *c) { return (c->heads / c->kv_heads + block_rows(c) - 1) / block_rows(c); }
// Blocks that share the work, 0 where each takes one item.
int shares(const mate_cache_t *c, int B, int max_len) {
    const int64_t items = (int64_t)B * c->kv_heads * blocks_of_group(c), units = items * units_of(max_len);
    const bool large = c->dtype == MATE_BF16 && c->d > 64 && block_rows(c) == 16;
    const int most = (large ? Shape<__nv_bfloat16, 128, 2>::kBlocksPerSm : Shape<__nv_bfloat16, 64, 1>::kBlocksPerSm) * n_sms(c->device);
    return units <= (kOver + (items < kMany ? kWhole : kWholeOfMany)) * items ? 0 : (int)(units < most ? units : most);
}

template <typename T, int DP, int NB, int W>
int launch_warps(const DecodeParams &p, unsigned grid, int device, cudaStream_t st) {
    static SmemAttrOnce attr;
    constexpr int kSmem = kAlign + W * kRing * kStage + kExtra<T, DP, NB, W>;
    const int rc = attr.ensure((const void *)decode_kernel<T, DP, NB, W>, kSmem, device);
    if (rc != MATE_OK) return rc;
    return launch_after(decode_kernel<T, DP, NB, W>, dim3(grid), 32 * W, kSmem, st, p) == cudaSuccess ? MATE_OK : MATE_ERR_CUDA;
}
template <typename T, int DP, int NB>
int launch(const DecodeParams &p, int blocks, int device, cudaStream_t st) {
    constexpr int kRows = Shape<T, DP, NB>::kRows;
    const int rows = kRows < p.group ? kRows : p.group, items = p.kv_heads * p.blocks_of_group;
    const int64_t all = (int64_t)p.B * items;
    // An item to each block; where there is an SM for each, eight warps: 12 items of 64 elements and 256 or 512 tokens 4.7 and 6.0 us
    // (with four 5.6 and 7.7), 8 items of 4 heads of 128 elements 6.5 and 8.6 (8.5 and 12.3).
    if (!blocks)
        return all <= n_sms(device) ? launch_warps<T, DP, NB, kManyWarps>(p, (unsigned)all, device, st)
                                    : launch_warps<T, DP, NB, kWarps>(p, (unsigned)all, device, st);
    const int rc = launch_warps<T, DP, NB, kWarps>(p, (unsigned)blocks, device, st);
    if (rc != MATE_OK) return rc;
    // few items in many parts: more threads each
    const dim3 joins((unsigned)all, (unsigned)rows);
    const size_t bytes = sizeof(float) * blocks;
    return (blocks > 16 * all ? launch_after(join_kernel<T, 1024>, joins, 1024, bytes, st, p, kRows)
                                      : launch_after(join_kernel<T, 128>, joins, 128, bytes, st, p, kRows)) == cudaSuccess
               ? MATE_OK
               : MATE_ERR_CUDA;
}

}  // namespace

size_t decode_workspace(const mate_cache_t *c, int B) {
    const int blocks = B > 0 ? shares(c, B, c->width * c->page_size) : 0;
    const int group = c->heads / c->kv_heads, rows = block_rows(c) < group ? block_rows(c) : group;
    return blocks ? sizeof(Joint) * B * c->kv_heads * blocks_of_group(c) + sizeof(float) * 2 * rows * (c->d + 2) * (size_t)blocks : 0;
}

}  // namespace mate

extern "C" int mate_attn_decode(const mate_cache_t *cache, int layer, const void *Q, const int64_t *q_stride, int B, const int32_t *seqs,
                                const int32_t *row_ids, const int32_t *col_ids, float scale, int max_len, void *O, float *LSE,
                                void *workspace, size_t workspace_bytes, void *stream) {
    using namespace mate;
    int rc = check_cache(cache);
    if (rc != MATE_OK) return rc;
    if (layer < 0 || layer >= cache->layers || B < 0 || max_len < 0 || (!seqs && B > cache->seqs)) return MATE_ERR_INVALID_ARG;
    if (B > 0 && (!Q || !q_stride || !row_ids || !col_ids || !O || !LSE)) return MATE_ERR_INVALID_ARG;
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
    if ((int64_t)B * cache->kv_heads * blocks_of_group(cache) > INT32_MAX / units_of(max_len)) return MATE_ERR_UNSUPPORTED;
    DecodeParams p = {};
    p.cache = cache_args(cache, layer);
    p.Q = Q, p.q_batch = q_stride[0], p.q_head = q_stride[1];
    p.B = B, p.heads = cache->heads, p.kv_heads = cache->kv_heads, p.group = cache->heads / cache->kv_heads;
    p.blocks_of_group = blocks_of_group(cache), p.d = cache->d;
    p.max_len = max_len;
    p.seqs = seqs, p.row_ids = row_ids, p.col_ids = col_ids;
    p.scale_log2 = scale * kLog2e, p.O = O, p.LSE = LSE;
    for (int h = 0; h < cache->heads; ++h) p.views[h >> 4] |= (uint32_t)cache->head_view[h] << 2 * (h & 15);
    for (p.page_shift = 0; 1u << p.page_shift < (unsigned)cache->page_size;) ++p.page_shift;
    p.page_mul = (unsigned)((((uint64_t)1 << 32) * (((uint64_t)1 << p.page_shift) - cache->page_size)) / cache->page_size + 1);
    p.page16 = (unsigned)(cache->page_stride / vec), p.head16 = (unsigned)(cache->head_stride / vec), p.slot16 = (unsigned)(cache->slot_stride / vec);
    const int blocks = shares(cache, B, p.max_len);
    if (blocks) {
        if (!workspace || workspace_bytes < decode_workspace(cache, B)) return MATE_ERR_WORKSPACE;
        if (!is_aligned(workspace, 256)) return MATE_ERR_ALIGNMENT;
        p.joints = static_cast<Joint *>(workspace);
        p.partial = reinterpret_cast<float *>(p.joints + (size_t)B * cache->kv_heads * p.blocks_of_group);
    }
    cudaStream_t st = (cudaStream_t)stream;
    const auto run = [&](auto wide) {
        constexpr int DP = wide ? 128 : 64;
        switch (block_rows(cache)) {
            case 2: return launch<float, DP, 2>(p, blocks, cache->device, st);
            case 4: return launch<float, DP, 4>(p, blocks, cache->device, st);
            case 16: return launch<__nv_bfloat16, DP, 2>(p, blocks, cache->device, st);
            default:
                return cache->dtype == MATE_F32 ? launch<float, DP, 8>(p, blocks, cache->device, st)
                                                : launch<__nv_bfloat16, DP, 1>(p, blocks, cache->device, st);
        }
    };
    return cache->d <= 64 ? run(std::false_type()) : run(std::true_type());
}

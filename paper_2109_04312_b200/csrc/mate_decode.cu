// Attention of one new token per sequence over the cached ones (mate_attn_decode): per sequence and kv head, the `group` query
// heads that share it (a block of up to 8 or 16 of them) against those cached tokens that one of them attends,
//     S = K q,  m = max S,  P = exp(S - m),  O = V^T P / sum P,  LSE = m + ln sum P.
//
// Bound by memory: a key and a value are read once for the whole group (4 d bytes in bf16 for 4 d flops per head), the ids of all
// cached tokens (4 or 8 bytes each, mostly from L2: the kv heads share them) decide which.  Hence
//   - a warp works alone: it looks through 32 tokens at a time (page, ids; the next 32 are on their way meanwhile), puts the
//     places of those that count into a list, and copies 16 bytes per lane and instruction from there into its own ring of stages
//     of 8 KB, with kRing - 1 stages under way; no block barrier until the sequence's part is done.  What nobody attends is never
//     read, padding's keys and values included.
//   - the products are tensor-core ones (m16n8k16) with the keys as the 16 rows and the heads as the 8 columns, so that a group
//     of up to 8 costs one of them; they take a tenth of the time that the copies take.  The weights go from one product's
//     result to the other's operand by transposing 8 x 8 pieces between the lanes.  fp32 caches: multiply-adds.
//   - blocks get equal shares of all sequences' tokens in units of kUnit (found by every block from the lengths, which the host does not
//     know), so one long sequence is spread over the GPU and short ones are put together.  A sequence that falls to several
//     blocks is joined by a second kernel from their partial results, in the order of its tokens: the same bits on every launch.
#include <cuda_bf16.h>

#include "mate_cache.h"
#include "sm100_ptx.cuh"

namespace mate {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kUnit = 32 * kWarps;       // tokens of a unit: what the warps look through in one go
constexpr int kStage = 8192;             // bytes of a stage: keys, then values
constexpr int kRing = 3;                 // stages of a warp
constexpr int kList = 64;                // entries of a warp's list of places
constexpr int kBlocksPerSm = 2;
constexpr int kJoinThreads = 256;
constexpr int kMaxHeads = 1024;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct DecodeParams {
    CacheArgs cache;
    const void *Q;
    int64_t q_batch, q_head;
    int B, heads, kv_heads, group, blocks_of_group, d, max_len;
    const int32_t *seqs, *row_ids, *col_ids;
    float scale_log2;  // scale / ln 2: weights are powers of two
    void *O;
    float *LSE;
    float *partial;    // [grid][2][rows of a block][d + 2]; null: a block per sequence, kv head and block of the group
    uint32_t views[kMaxHeads / 16];  // two bits a head
};
__device__ __forceinline__ int view_at(const DecodeParams &p, int h) { return p.views[h >> 4] >> 2 * (h & 15) & 3; }

// ---- types

template <typename T, int DP, int NB>
struct Shape {
    static constexpr int kRows = 8 * NB;                                    // query heads of a block
    static constexpr int kRowBytes = DP * (int)sizeof(T);
    static constexpr int kKeys = kStage / 2 / kRowBytes;                    // of a stage
    static constexpr int kChunks = kRowBytes / 16;
    // What a row's chunks are permuted by: eight rows of 16 bytes (bf16: ldmatrix) or the lanes of an eighth of a warp, of which
    // 32 / kKeys share a key (fp32), then fall into different banks.
    static constexpr int kSwizzle = sizeof(T) == 2 ? 1 : 32 / kKeys;
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
// over all items; block i of C gets units [i U / C, (i + 1) U / C).  (Every item has a unit: empty ones are written too.)
__device__ __forceinline__ int units_of(int len) { return len > kUnit ? (len + kUnit - 1) / kUnit : 1; }
__device__ __forceinline__ int64_t share(int64_t U, int C, int i) { return U * i / C; }

// Length that counts of entry b of the batch, 0 where the entry is none.
__device__ __forceinline__ int entry_len(const DecodeParams &p, int b, bool *bad) {
    const int s = seq_of(p.seqs, b, p.cache.seqs);
    if (s < 0) {
        *bad = true;
        return 0;
    }
    return clip_len(p.cache.lens[s], p.max_len, bad);
}

struct Start {
    int64_t total, before;  // units of the batch; of the entries in front of `entry`
    int entry;
};
// All threads call it: the entry that unit `at` belongs to (fixed < 0), or the units in front of entry `fixed`.
template <int kN>
__device__ Start find_start(const DecodeParams &p, int items, int fixed, int block, int blocks) {
    __shared__ int64_t s_sum[kN / 32];
    __shared__ Start s_start;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (p.B + kN - 1) / kN, b0 = min(p.B, tid * per), b1 = min(p.B, b0 + per);
    bool bad = false;
    int64_t own = 0;
    for (int b = b0; b < b1; ++b) own += units_of(entry_len(p, b, &bad));
    own *= items;
    int64_t sum = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(~0u, sum, o);
        if (lane >= o) sum += y;
    }
    if (lane == 31) s_sum[warp] = sum;
    __syncthreads();
    int64_t total = 0, before = sum - own;
#pragma unroll
    for (int w = 0; w < kN / 32; ++w) {
        if (w < warp) before += s_sum[w];
        total += s_sum[w];
    }
    const int64_t at = share(total, blocks, block);
    if (b0 < b1 && (fixed < 0 ? at >= before && at < before + own : fixed >= b0 && fixed < b1)) {
        int b = b0;
        for (; b < b1 - 1; ++b) {
            const int64_t n = (int64_t)units_of(entry_len(p, b, &bad)) * items;
            if (fixed < 0 ? at < before + n : b == fixed) break;
            before += n;
        }
        s_start = {total, before, b};
    }
    if (bad && block == 0) atomicOr(p.cache.status, kCacheBad);
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
    int b, item, u;       // next unit: of entry b, item, unit u
    int64_t left;         // units of the share
};
__device__ __forceinline__ bool next_part(const DecodeParams &p, int items, Walk &w, Part &part, int *len) {
    if (w.left <= 0 || w.b >= p.B) return false;
    bool bad = false;
    *len = entry_len(p, w.b, &bad);
    const int n = units_of(*len);
    part.b = w.b, part.item = w.item, part.u0 = w.u;
    part.u1 = (int)min((int64_t)n, w.u + w.left);
    part.whole = part.u0 == 0 && part.u1 == n;
    w.left -= max(1, part.u1 - part.u0);
    w.u = 0;
    if (++w.item == items) w.item = 0, ++w.b;
    return true;
}

// ---- the loading side of a warp

struct Meta {  // of a stage
    int n, end;           // keys; the last stage of a part
    uint32_t by_row, by_col;
    int b, item, whole, more;  // the part; whether there is one (behind the last one: no)
};

template <typename T, int DP, int NB>
struct Loader {
    using S = Shape<T, DP, NB>;
    const DecodeParams &p;
    int64_t *list;
    Meta *meta;
    uint32_t ring;
    int lane, warp, items;
    Walk walk;
    // the present part
    Part part;
    bool active;
    int s, prefix, q_row, q_col, first, end;  // tokens [first, end) of the warp, in steps of kUnit
    int64_t head_at;
    bool text, need_row, need_col;
    int next;                            // first of the 32 tokens that are looked at next
    int page, page2, slot, row, col;     // of the lane's token there: its ids have been asked for; page2: of the one a step on
    bool there;
    bool bad;
    int pending, list_at, filled;        // list; stages so far

    __device__ void look_page(int j, int &pg) {
        pg = -1;
        if (j < end) {
            pg = p.cache.table[(size_t)s * p.cache.width + j / p.cache.page_size];
            if (!in_range(pg, p.cache.pages)) bad = true, pg = -1;
        }
    }
    __device__ void look_ids(int j) {
        there = j < end && page >= 0;
        if (there) {
            slot = j % p.cache.page_size;
            const size_t at = (size_t)page * p.cache.page_size + slot;
            if (need_row || text) row = p.cache.row_ids[at];
            if (need_col && !text) col = p.cache.col_ids[at];
        }
    }
    __device__ void begin() {
        int len;
        active = next_part(p, items, walk, part, &len);
        if (!active) return;
        s = seq_of(p.seqs, part.b, p.cache.seqs);
        q_row = p.row_ids[part.b], q_col = p.col_ids[part.b];
        prefix = s >= 0 ? p.cache.prefix[s] : 0;
        text = q_row == MATE_ID_TEXT || q_col == MATE_ID_TEXT;
        if (q_row < 0 || q_col < 0) len = 0;
        const int kv = part.item / p.blocks_of_group, block = part.item - kv * p.blocks_of_group;
        head_at = kv * p.cache.head_stride;
        need_row = need_col = false;
        const int h0 = kv * p.group + block * S::kRows, n = min(S::kRows, p.group - block * S::kRows);
        for (int i = 0; i < n; ++i) {
            const int v = view_at(p, h0 + i);
            need_row |= v != MATE_VIEW_COL;
            need_col |= v != MATE_VIEW_ROW;
        }
        next = part.u0 * kUnit + warp * 32;
        end = min(len, part.u1 * kUnit);
        look_page(next + lane, page);
        look_ids(next + lane);
        look_page(next + kUnit + lane, page2);
    }
    // One look at 32 tokens: those that count go onto the list, the next ones' ids are asked for.
    __device__ void look() {
        const int j = next + lane;
        const bool all = text || j < prefix;
        const bool by_row = there && (need_row || text) && row >= 0 && (all || row == MATE_ID_TEXT || row == q_row);
        const bool by_col = text ? by_row : there && need_col && col >= 0 && (all || col == MATE_ID_TEXT || col == q_col);
        const unsigned counts = __ballot_sync(~0u, by_row || by_col);
        if (by_row || by_col) {
            const int64_t at = (page * p.cache.page_stride + slot * p.cache.slot_stride + head_at) * (int64_t)sizeof(T);
            list[(list_at + pending + __popc(counts & ((1u << lane) - 1))) & (kList - 1)] = at | (by_row ? 1 : 0) | (by_col ? 2 : 0);
        }
        pending += __popc(counts);
        next += kUnit;
        page = page2;
        look_ids(next + lane);
        look_page(next + kUnit + lane, page2);
    }
    // Copies of the next stage are put under way (or, at the end of the share, none: the groups are counted).
    __device__ void fill() {
        if (active) {
            while (pending < S::kKeys && next < end) look();
            __syncwarp();
            const int n = min(pending, S::kKeys), slot_of_ring = filled % kRing;
            const bool last = pending <= S::kKeys && next >= end;
            const int64_t mine = lane < n ? list[(list_at + lane) & (kList - 1)] : 0;
            const uint32_t by_row = __ballot_sync(~0u, mine & 1), by_col = __ballot_sync(~0u, mine & 2);
            if (lane == 0) meta[slot_of_ring] = {n, last, by_row, by_col, part.b, part.item, part.whole, 1};
            const uint32_t to = ring + slot_of_ring * kStage;
            constexpr int kPerPass = 32 / S::kChunks > 0 ? 32 / S::kChunks : 1;  // keys of a pass (rows have 8, 16 or 32 chunks)
            const int chunk = lane % S::kChunks, chunks = p.d * (int)sizeof(T) / 16;
            if (n > 0 && chunk < chunks) {
#pragma unroll
                for (int i = 0; i < S::kKeys / kPerPass; ++i) {
                    const int key = i * kPerPass + lane / S::kChunks;
                    const bool there_is = key < n;
                    const int64_t at = there_is ? (list[(list_at + key) & (kList - 1)] & ~(int64_t)15) + chunk * 16 : 0;
                    const uint32_t dst = to + S::chunk_at(key, chunk);
                    cp_async16_or_zero(dst, (const char *)p.cache.k + at, there_is);
                    cp_async16_or_zero(dst + kStage / 2, (const char *)p.cache.v + at, there_is);
                }
            }
            list_at = (list_at + n) & (kList - 1);
            pending -= n;
            __syncwarp();  // the list has been read
            if (last) begin();
        } else if (lane == 0) {
            meta[filled % kRing] = {0, 1, 0u, 0u, 0, 0, 0, 0};
        }
        ++filled;
        cp_async_commit();
    }
};

// ---- the reading side: running maximum, sum and weighted sum of values of a block's query heads

template <typename T, int DP, int NB>
struct Reader;

template <int DP, int NB>
struct Reader<__nv_bfloat16, DP, NB> {
    using S = Shape<__nv_bfloat16, DP, NB>;
    static constexpr int kTiles = S::kKeys / 16;
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
                const int h = nb * 8 + 2 * (lane & 3) + c, v = h < n_rows ? view_at(p, h0 + h) : MATE_VIEW_EITHER;
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
    __device__ void add(const DecodeParams &p, uint32_t stage, const Meta &meta, int lane, float *) {
        float s[kTiles][NB][4];
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[t][nb][i] = 0.f;
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                uint32_t a[4];
                ldmatrix4(a, stage + S::chunk_at(t * 16 + (lane & 15), 2 * k + (lane >> 4)));
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) mma16816(s[t][nb], a, q[k][nb]);
            }
        uint32_t w[kTiles][NB][2];
        float keep[NB][2];
        bool moved = false;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const uint32_t counts = (meta.by_row & rows_of[nb][c]) | (meta.by_col & cols_of[nb][c]);
                float top = m[nb][c];
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        float &x = s[t][nb][2 * half + c];
                        x = counts >> (t * 16 + half * 8 + lane / 4) & 1 ? x * p.scale_log2 : -INFINITY;
                        top = fmaxf(top, x);
                    }
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
                for (int half = 0; half < 2; ++half) w[t][nb][half] = transpose8(ptx::cvt_bf16x2(s[t][nb][2 * half], s[t][nb][2 * half + 1]));
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                uint32_t a[4];
                ldmatrix4_trans(a, stage + kStage / 2 + S::chunk_at(t * 16 + (lane & 7) + (lane >> 4) * 8, 2 * k + (lane >> 3 & 1)));
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) mma16816(o[k][nb], a, w[t][nb]);
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
    int n;

    // `own`: the warp's queries [kRows][DP], then weights [kRows][kKeys]
    __device__ void begin(const DecodeParams &p, int b, int h0, int n_rows, int lane, float *own) {
        const float *Q = (const float *)p.Q + b * p.q_batch;
        n = n_rows;
        __syncwarp();
        for (int i = lane; i < S::kRows * DP; i += 32) {
            const int r = i / DP, e = i % DP;
            own[i] = r < n_rows && e < p.d ? Q[(h0 + r) * p.q_head + e] : 0.f;
        }
        __syncwarp();
#pragma unroll
        for (int r = 0; r < S::kRows; ++r) {
            m[r] = -INFINITY, l[r] = 0.f;
#pragma unroll
            for (int c = 0; c < kCols; ++c) o[r][c] = 0.f;
        }
        views = 0;
        for (int r = 0; r < n_rows; ++r) views |= (uint32_t)view_at(p, h0 + r) << 2 * r;
    }
    uint32_t views;
    __device__ void add(const DecodeParams &p, uint32_t stage, const Meta &meta, int lane, float *own) {
        const int key = lane / kShare, part = lane % kShare;
        float *weights = own + S::kRows * DP;
        float s[S::kRows];
#pragma unroll
        for (int r = 0; r < S::kRows; ++r) s[r] = 0.f;
#pragma unroll
        for (int i = 0; i < S::kChunks / kShare; ++i) {
            const int chunk = i * kShare + part;
            const float4 k = ptx::ld_shared_f4(stage + S::chunk_at(key, chunk));
#pragma unroll
            for (int r = 0; r < S::kRows; ++r) {
                if (r >= n) break;
                const float4 x = *reinterpret_cast<const float4 *>(own + r * DP + chunk * 4);
                s[r] = fmaf(x.x, k.x, fmaf(x.y, k.y, fmaf(x.z, k.z, fmaf(x.w, k.w, s[r]))));
            }
        }
#pragma unroll
        for (int r = 0; r < S::kRows; ++r) {
            if (r >= n) break;
            const int v = views >> 2 * r & 3;
            const uint32_t counts = (v != MATE_VIEW_COL ? meta.by_row : 0u) | (v != MATE_VIEW_ROW ? meta.by_col : 0u);
            float x = s[r];
#pragma unroll
            for (int step = 1; step < kShare; step <<= 1) x += __shfl_xor_sync(~0u, x, step);
            x = counts >> key & 1 ? x * p.scale_log2 : -INFINITY;
            float top = fmaxf(m[r], x);
#pragma unroll
            for (int step = kShare; step < 32; step <<= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, step));
            const float base = top == -INFINITY ? 0.f : top, keep = ptx::ex2(m[r] - base), w = ptx::ex2(x - base);
            m[r] = top;
            l[r] = fmaf(l[r], keep, w);  // (kShare lanes count the same key)
#pragma unroll
            for (int c = 0; c < kCols; ++c) o[r][c] *= keep;
            if (part == 0) weights[r * S::kKeys + key] = w;
        }
        __syncwarp();
#pragma unroll
        for (int k0 = 0; k0 < S::kKeys; k0 += 4) {
            float v[4][kCols];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t at = stage + kStage / 2 + S::chunk_at(k0 + k, lane * kCols / 4) + (lane * kCols % 4) * 4;
                if (kCols == 4) {
                    const float4 x = ptx::ld_shared_f4(at);
                    v[k][0] = x.x, v[k][1] = x.y, v[k][kCols - 2] = x.z, v[k][kCols - 1] = x.w;
                } else {
                    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v[k][0]), "=f"(v[k][1]) : "r"(at));
                }
            }
#pragma unroll
            for (int r = 0; r < S::kRows; ++r) {
                if (r >= n) break;
                const float4 w = *reinterpret_cast<const float4 *>(weights + r * S::kKeys + k0);
#pragma unroll
                for (int c = 0; c < kCols; ++c) o[r][c] = fmaf(w.x, v[0][c], fmaf(w.y, v[1][c], fmaf(w.z, v[2][c], fmaf(w.w, v[3][c], o[r][c]))));
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

__device__ __forceinline__ void put(float x, float *y) { *y = x; }
__device__ __forceinline__ void put(float x, __nv_bfloat16 *y) { *y = __float2bfloat16_rn(x); }

// Floats of shared memory behind the ring: results of the warps, their maxima and sums; fp32: a warp's queries and weights.
template <typename T, int DP, int NB>
__host__ __device__ constexpr int extra_floats(int rows, int d) {
    return kWarps * rows * (d + 2) + (sizeof(T) == 4 ? kWarps * Shape<T, DP, NB>::kRows * (DP + Shape<T, DP, NB>::kKeys) : 0);
}

template <typename T, int DP, int NB>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) decode_kernel(const __grid_constant__ DecodeParams p) {
    using S = Shape<T, DP, NB>;
    extern __shared__ __align__(128) char smem[];
    __shared__ int64_t s_list[kWarps][kList];
    __shared__ Meta s_meta[kWarps][kRing];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, items = p.kv_heads * p.blocks_of_group;
    const int max_rows = min(S::kRows, p.group);
    float *own = reinterpret_cast<float *>(smem + kWarps * kRing * kStage) + (sizeof(T) == 4 ? warp * S::kRows * (DP + S::kKeys) : 0);
    float *s_out = reinterpret_cast<float *>(smem + kWarps * kRing * kStage) + (sizeof(T) == 4 ? kWarps * S::kRows * (DP + S::kKeys) : 0);
    float *s_stats = s_out + kWarps * max_rows * p.d;
    ptx::launch_dependents();
    if (p.d < DP)  // columns that no copy writes
        for (int i = tid; i < kWarps * kRing * kStage / 16; i += kThreads) reinterpret_cast<uint4 *>(smem)[i] = make_uint4(0, 0, 0, 0);
    ptx::wait_prior_grid();

    Walk walk;
    if (p.partial) {
        const Start start = find_start<kThreads>(p, items, -1, blockIdx.x, gridDim.x);
        const int64_t at = share(start.total, gridDim.x, blockIdx.x);
        walk.left = share(start.total, gridDim.x, blockIdx.x + 1) - at;
        if (walk.left == 0) return;
        bool bad = false;
        const int n = units_of(entry_len(p, start.entry, &bad));
        walk.b = start.entry;
        walk.item = min(items - 1, (int)((at - start.before) / n));
        walk.u = (int)(at - start.before - (int64_t)walk.item * n);
    } else {
        bool bad = false;
        walk.b = blockIdx.x / items, walk.item = blockIdx.x - walk.b * items, walk.u = 0;
        walk.left = units_of(entry_len(p, walk.b, &bad));
        if (bad && tid == 0) atomicOr(p.cache.status, kCacheBad);
        __syncthreads();
    }

    Loader<T, DP, NB> load = {p, s_list[warp], s_meta[warp], ptx::smem_u32(smem) + warp * kRing * kStage, lane, warp, items, walk};
    load.bad = false, load.pending = load.list_at = load.filled = 0;
    load.begin();
    for (int i = 0; i < kRing - 1; ++i) load.fill();

    __syncwarp();

    Reader<T, DP, NB> read;
    bool first = true;
    for (int t = 0;;) {
        Meta meta = s_meta[warp][t % kRing];
        if (!meta.more) break;
        const Meta part = meta;
        const int kv = part.item / p.blocks_of_group, block = part.item - kv * p.blocks_of_group;
        const int h0 = kv * p.group + block * S::kRows, n_rows = min(S::kRows, p.group - block * S::kRows);
        read.begin(p, part.b, h0, n_rows, lane, own);
        for (bool more = true; more; ++t) {
            cp_async_wait<kRing - 2>();
            __syncwarp();
            load.fill();
            meta = s_meta[warp][t % kRing];
            if (meta.n > 0) read.add(p, ptx::smem_u32(smem) + (warp * kRing + t % kRing) * kStage, meta, lane, own);
            more = !meta.end;
        }
        __syncwarp();
        read.store(s_out + warp * max_rows * p.d, s_stats + warp * max_rows * 2, n_rows, p.d, lane);
        __syncthreads();
        // the warps' results together: the whole item's, or a partial one
        float *to = p.partial + (size_t)(2 * blockIdx.x + (first ? 0 : 1)) * max_rows * (p.d + 2);
        for (int i = tid; i < n_rows * p.d; i += kThreads) {
            const int r = i / p.d, e = i - r * p.d;
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_stats[(w * max_rows + r) * 2]);
            const float base = top == -INFINITY ? 0.f : top;
            float sum = 0.f, x = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float f = ptx::ex2(s_stats[(w * max_rows + r) * 2] - base);
                sum = fmaf(f, s_stats[(w * max_rows + r) * 2 + 1], sum);
                x = fmaf(f, s_out[(w * max_rows + r) * p.d + e], x);
            }
            if (part.whole) {
                const size_t row = (size_t)part.b * p.heads + h0 + r;
                put(sum == 0.f ? 0.f : x / sum, (T *)p.O + row * p.d + e);
                if (e == 0) p.LSE[row] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
            } else {
                to[r * (p.d + 2) + 2 + e] = x;
                if (e == 0) to[r * (p.d + 2)] = top, to[r * (p.d + 2) + 1] = sum;
            }
        }
        __syncthreads();
        first = false;
    }
    cp_async_wait<0>();
    if (load.bad) atomicOr(p.cache.status, kCacheBad);
}

// Joins the partial results of an item that fell to several blocks of the kernel before.  grid: (entry, item)
template <typename T>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ DecodeParams p, int blocks, int block_rows) {
    extern __shared__ float s_join[];  // weights [rows][parts], then sums [groups][rows][d]
    ptx::launch_dependents();
    ptx::wait_prior_grid();
    const int tid = threadIdx.x, items = p.kv_heads * p.blocks_of_group, b = blockIdx.x, item = blockIdx.y;
    const Start start = find_start<kJoinThreads>(p, items, b, 1, blocks);
    bool bad = false;
    const int n = units_of(entry_len(p, b, &bad));
    const int64_t U = start.total, s = start.before + (int64_t)item * n, e = s + n;
    // block i has unit x: the largest i with i U / blocks <= x
    const int i0 = (int)(((s + 1) * blocks - 1) / U), i1 = (int)((e * blocks - 1) / U);
    if (i0 == i1) return;
    const int kv = item / p.blocks_of_group, part = item - kv * p.blocks_of_group, max_rows = min(block_rows, p.group);
    const int h0 = kv * p.group + part * block_rows, rows = min(block_rows, p.group - part * block_rows), width = p.d + 2, parts = i1 - i0 + 1;
    // (a block without units has no result; an item's first part in a block that has begun another one before is its second)
    auto result = [&](int i) -> const float * {
        const int64_t lo = share(U, blocks, i);
        if (lo == share(U, blocks, i + 1)) return nullptr;
        return p.partial + (size_t)(2 * i + (s <= lo ? 0 : 1)) * max_rows * width;
    };
    float *s_w = s_join, *s_sum = s_join + rows * parts;
    for (int r = tid >> 5; r < rows; r += kJoinThreads / 32) {
        const int lane = tid & 31;
        float top = -INFINITY;
        for (int i = lane; i < parts; i += 32)
            if (const float *x = result(i0 + i)) top = fmaxf(top, x[r * width]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
        const float base = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
        for (int i = lane; i < parts; i += 32) {
            const float *x = result(i0 + i);
            const float w = x ? ptx::ex2(x[r * width] - base) : 0.f;
            s_w[r * parts + i] = w;
            if (x) sum = fmaf(w, x[r * width + 1], sum);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
        const float inverse = sum == 0.f ? 0.f : 1.f / sum;
        for (int i = lane; i < parts; i += 32) s_w[r * parts + i] *= inverse;
        if (lane == 0) p.LSE[(size_t)b * p.heads + h0 + r] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
    }
    __syncthreads();
    // pairs of columns, and for few of them several groups of threads that take the parts in turn
    const int pairs = rows * p.d / 2, groups = max(1, kJoinThreads / pairs), group = tid / pairs;
    for (int c = groups > 1 ? tid % pairs : tid; c < pairs && group < groups; c += groups > 1 ? pairs : kJoinThreads) {
        const int r = c / (p.d / 2), at = r * width + 2 + 2 * (c - r * (p.d / 2));
        float x = 0.f, y = 0.f;
#pragma unroll 4
        for (int i = groups > 1 ? group : 0; i < parts; i += groups)
            if (const float *z = result(i0 + i)) {
                const float2 v = *reinterpret_cast<const float2 *>(z + at);
                x = fmaf(s_w[r * parts + i], v.x, x), y = fmaf(s_w[r * parts + i], v.y, y);
            }
        if (groups == 1) {
            T *to = (T *)p.O + ((size_t)b * p.heads + h0) * p.d + 2 * c;
            put(x, to), put(y, to + 1);
            continue;
        }
        s_sum[(group * pairs + c) * 2] = x, s_sum[(group * pairs + c) * 2 + 1] = y;
    }
    if (groups == 1) return;
    __syncthreads();
    for (int c = tid; c < 2 * pairs; c += kJoinThreads) {
        float x = 0.f;
        for (int g = 0; g < groups; ++g) x += s_sum[g * pairs * 2 + c];
        put(x, (T *)p.O + ((size_t)b * p.heads + h0) * p.d + c);
    }
}

// ---- host

int block_rows(const mate_cache_t *c) { return c->dtype == MATE_BF16 && c->heads / c->kv_heads > 8 ? 16 : 8; }
int blocks_of_group(const mate_cache_t *c) { return (c->heads / c->kv_heads + block_rows(c) - 1) / block_rows(c); }
// Blocks that share the work, 0 where each takes one item.
int shares(const mate_cache_t *c, int B, int max_len) {
    const int64_t items = (int64_t)B * c->kv_heads * blocks_of_group(c), units = items * ((max_len + kUnit - 1) / kUnit);
    const int most = kBlocksPerSm * n_sms(c->device);
    return units == items ? 0 : (int)(units < most ? units : most);
}

template <typename T, int DP, int NB>
int launch(const DecodeParams &p, int blocks, int device, cudaStream_t st) {
    static SmemAttrOnce attr, join_attr;
    using S = Shape<T, DP, NB>;
    const int rows = S::kRows < p.group ? S::kRows : p.group;
    constexpr int kMostSmem = kWarps * kRing * kStage + 4 * extra_floats<T, DP, NB>(S::kRows, DP);
    const int smem = kWarps * kRing * kStage + 4 * extra_floats<T, DP, NB>(rows, p.d);
    int rc = attr.ensure((const void *)decode_kernel<T, DP, NB>, kMostSmem, device);
    if (rc != MATE_OK) return rc;
    const int64_t items = (int64_t)p.kv_heads * p.blocks_of_group, grid = blocks ? blocks : p.B * items;
    if (grid > INT32_MAX) return MATE_ERR_UNSUPPORTED;
    if (launch_after(decode_kernel<T, DP, NB>, dim3((unsigned)grid), kThreads, (size_t)smem, st, p) != cudaSuccess) return MATE_ERR_CUDA;
    if (!blocks) return MATE_OK;
    const size_t join = sizeof(float) * ((size_t)rows * blocks + 2 * kJoinThreads);
    rc = join_attr.ensure((const void *)join_kernel<T>, 100 * 1024, device);
    if (rc != MATE_OK) return rc;
    return launch_after(join_kernel<T>, dim3((unsigned)p.B, (unsigned)items), kJoinThreads, join, st, p, blocks, S::kRows) == cudaSuccess ? MATE_OK
                                                                                                                                  : MATE_ERR_CUDA;
}

}  // namespace

size_t decode_workspace(const mate_cache_t *c, int B) {
    const int blocks = B > 0 ? shares(c, B, c->width * c->page_size) : 0;
    const int group = c->heads / c->kv_heads, rows = block_rows(c) < group ? block_rows(c) : group;
    return sizeof(float) * 2 * (size_t)blocks * rows * (c->d + 2);
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
    if (cache->heads > kMaxHeads) return MATE_ERR_UNSUPPORTED;
    const int vec = (int)(16 / elem_size(cache->dtype));
    if (B > 0 && (!is_aligned(Q, 16) || !is_aligned(O, 16) || !is_aligned(LSE, 4) || q_stride[0] % vec != 0 || q_stride[1] % vec != 0))
        return MATE_ERR_ALIGNMENT;
    if ((rc = check_cache_device(cache)) != MATE_OK) return rc;
    if (B == 0) return MATE_OK;
    DecodeParams p = {};
    p.cache = cache_args(cache, layer);
    p.Q = Q, p.q_batch = q_stride[0], p.q_head = q_stride[1];
    p.B = B, p.heads = cache->heads, p.kv_heads = cache->kv_heads, p.group = cache->heads / cache->kv_heads;
    p.blocks_of_group = blocks_of_group(cache), p.d = cache->d;
    const int most = cache->width * cache->page_size;
    p.max_len = max_len > 0 && max_len < most ? max_len : most;
    p.seqs = seqs, p.row_ids = row_ids, p.col_ids = col_ids;
    p.scale_log2 = scale * kLog2e, p.O = O, p.LSE = LSE;
    for (int h = 0; h < cache->heads; ++h) p.views[h >> 4] |= (uint32_t)cache->head_view[h] << 2 * (h & 15);
    const int blocks = shares(cache, B, p.max_len);
    if (blocks) {
        if (!workspace || workspace_bytes < decode_workspace(cache, B)) return MATE_ERR_WORKSPACE;
        if (!is_aligned(workspace, 256)) return MATE_ERR_ALIGNMENT;
        p.partial = static_cast<float *>(workspace);
    }
    cudaStream_t st = (cudaStream_t)stream;
    const bool narrow = cache->d <= 64;
    if (cache->dtype == MATE_F32)
        return narrow ? launch<float, 64, 1>(p, blocks, cache->device, st) : launch<float, 128, 1>(p, blocks, cache->device, st);
    if (block_rows(cache) == 8)
        return narrow ? launch<__nv_bfloat16, 64, 1>(p, blocks, cache->device, st) : launch<__nv_bfloat16, 128, 1>(p, blocks, cache->device, st);
    return narrow ? launch<__nv_bfloat16, 64, 2>(p, blocks, cache->device, st) : launch<__nv_bfloat16, 128, 2>(p, blocks, cache->device, st);
}

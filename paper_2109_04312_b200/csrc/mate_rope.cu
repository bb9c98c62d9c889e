// Rotary positions (mate_rope) and new tokens into the pages of a cache (mate_cache_append): one kernel, which turns
// rows of up to three tensors (queries, keys; values are only copied) and writes them by strides or through a page table.
//
// A pair (a, b) becomes m (a cos t - b sin t, a sin t + b cos t), t = position * freqs[pair]; the transpose has -t.  The
// angle is reduced in 64 bits (position * freqs / 2 pi, minus the nearest whole number of turns), which leaves an error
// of 1e-9 of a turn at positions of 10^7; sine and cosine of what is left are taken in fp32 by sincospif.
//
// Bound by memory: one read and one write of every element.  A block takes up to kTokens tokens and a slice of the heads:
// all its loads are under way (kUnits of them per thread, 16 bytes each half) before the tokens' sines and cosines are worked
// out, once per block into shared memory, for all heads of the slice.
#include <cuda_bf16.h>

#include "mate_cache.h"
#include "sm100_ptx.cuh"

namespace mate {
namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 16;  // tokens of a block, at most (wide rows: 8, 4, 2 or 1)
constexpr int kUnits = 4;    // units of a thread: a unit is two runs of VEC elements of one head of one token

struct Side {
    const void *x;
    void *y;  // null: into the cache's pages (of keys or of values)
    int64_t xs[3], ys[3];
    int heads;
    int turned, to_keys;
};
struct RopeParams {
    Side side[3];
    int n_sides, n_heads;  // heads of all sides together
    int B, N, d, rot, interleaved;
    const int32_t *positions;
    int64_t position_stride;
    const double *freqs;
    float mscale, sign;
    int n_chunks, turned_chunks;      // units of a head, and how many of them are pairs
    unsigned magic;                   // x / n_chunks = x * magic >> 20 for x below 2^10 and up to 2^10 chunks
    int heads_per_block, token_bits;  // (2^token_bits tokens)
    // new tokens of a cache
    int paged;
    CacheArgs cache;
    const int32_t *seqs, *counts, *row_ids, *col_ids;
};

template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Run {
    T v[VEC];
};
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f32(float x, float &y) { y = x; }
__device__ __forceinline__ void from_f32(float x, __nv_bfloat16 &y) { y = __float2bfloat16_rn(x); }

// Element offsets of a unit's two runs within a row; the second one is missing at the end of an odd row.
struct Place {
    int a, b;
    bool has_b;
};
template <int VEC>
__device__ __forceinline__ Place place(const RopeParams &p, int chunk, bool turned) {
    if (turned && chunk < p.turned_chunks)
        return p.interleaved ? Place{2 * VEC * chunk, 2 * VEC * chunk + VEC, true} : Place{VEC * chunk, p.rot / 2 + VEC * chunk, true};
    const int at = turned ? p.rot + 2 * VEC * (chunk - p.turned_chunks) : 2 * VEC * chunk;
    return {at, at + VEC, at + VEC < p.d};
}

template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads) rope_kernel(const __grid_constant__ RopeParams p) {
    extern __shared__ float s_trig[];  // [tokens][rot / 2] cosines, then sines
    __shared__ int64_t s_from[3][kTokens], s_to[3][kTokens];
    __shared__ int s_pos[kTokens];
    ptx::launch_dependents();
    ptx::wait_prior_grid();
    const int tid = threadIdx.x, pairs = p.rot / 2, tokens = 1 << p.token_bits;
    const int64_t first = (int64_t)blockIdx.x << p.token_bits, n_tokens = (int64_t)p.B * p.N;
    const int h0 = blockIdx.y * p.heads_per_block, n_heads = min(p.heads_per_block, p.n_heads - h0);

    // where the tokens' rows are: -1 = nowhere
    if (tid < tokens) {
        const int64_t t = first + tid;
        const bool exists = t < n_tokens;
        const int b = exists ? (int)(t / p.N) : 0, n = exists ? (int)(t - (int64_t)b * p.N) : 0;
        int position = 0;
        int64_t page_at = -1;
        if (p.paged && exists) {
            bool bad = false;
            const int s = seq_of(p.seqs, b, p.cache.seqs), count = p.counts ? p.counts[b] : p.N;
            if (s < 0 || count < 0 || count > p.N) {
                bad = true;
            } else if (n < count) {
                const int at = clip_len(p.cache.lens[s], p.cache.width * p.cache.page_size, &bad) - count + n;
                position = at;
                if (at < 0) bad = true;
                if (!bad) {
                    const int i = at / p.cache.page_size, slot = at - i * p.cache.page_size;
                    const int page = p.cache.table[(size_t)s * p.cache.width + i];
                    if (!in_range(page, p.cache.pages)) {
                        bad = true;
                    } else {
                        page_at = page * p.cache.page_stride + slot * p.cache.slot_stride;
                        if (p.row_ids && blockIdx.y == 0) {
                            const size_t to = (size_t)page * p.cache.page_size + slot;
                            p.cache.row_ids[to] = p.row_ids[t];
                            p.cache.col_ids[to] = p.col_ids[t];
                        }
                    }
                }
            }
            if (bad && blockIdx.y == 0) atomicOr(p.cache.status, kCacheBad);
        }
        if (exists && p.positions) position = p.positions[b * p.position_stride + n];
        s_pos[tid] = position;
        for (int i = 0; i < p.n_sides; ++i) {
            const Side &s = p.side[i];
            const bool goes = exists && (s.y || page_at >= 0);
            s_from[i][tid] = goes ? b * s.xs[0] + n * s.xs[2] : -1;
            s_to[i][tid] = s.y ? b * s.ys[0] + n * s.ys[2] : page_at;
        }
    }
    __syncthreads();

    Run<T, VEC> a[kUnits], b[kUnits];
    const int units = (n_heads << p.token_bits) * p.n_chunks;
    // head (within the slice), token and chunk of a unit: chunks next to one another, then tokens, then heads
    auto locate = [&](int u, int &side, int &head, int &token, int &chunk) {
        const int row = (int)((unsigned)u * p.magic >> 20);
        chunk = u - row * p.n_chunks;
        token = row & (tokens - 1);
        head = h0 + (row >> p.token_bits);
        side = 0;
        while (side + 1 < p.n_sides && head >= p.side[side].heads) head -= p.side[side++].heads;
    };
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const int u = tid + i * kThreads;
        if (u >= units) break;
        int side, head, token, chunk;
        locate(u, side, head, token, chunk);
        const Side &s = p.side[side];
        if (s_from[side][token] < 0) continue;
        const T *x = (const T *)s.x + s_from[side][token] + head * s.xs[1];
        const Place at = place<VEC>(p, chunk, s.turned);
        a[i] = *reinterpret_cast<const Run<T, VEC> *>(x + at.a);
        if (at.has_b) b[i] = *reinterpret_cast<const Run<T, VEC> *>(x + at.b);
    }
    for (int i = tid; i < tokens * pairs; i += kThreads) {
        const int token = i / pairs, pair = i - token * pairs;
        const double turns = (double)s_pos[token] * (p.freqs[pair] * 0.15915494309189533577);
        float sn, cs;
        sincospif(2.f * (float)(turns - rint(turns)), &sn, &cs);
        s_trig[i] = cs * p.mscale;
        s_trig[tokens * pairs + i] = sn * p.mscale * p.sign;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const int u = tid + i * kThreads;
        if (u >= units) break;
        int side, head, token, chunk;
        locate(u, side, head, token, chunk);
        const Side &s = p.side[side];
        if (s_from[side][token] < 0) continue;
        const Place at = place<VEC>(p, chunk, s.turned);
        if (s.turned && chunk < p.turned_chunks) {
            const float *cs = s_trig + token * pairs + chunk * VEC, *sn = cs + tokens * pairs;
            if (p.interleaved && VEC > 1) {  // pairs lie side by side: VEC / 2 in each run
#pragma unroll
                for (int e = 0; e < VEC; e += 2)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        T *r = half ? &b[i].v[e & (VEC - 1)] : &a[i].v[e & (VEC - 1)];
                        const float c = cs[half * VEC / 2 + e / 2], z = sn[half * VEC / 2 + e / 2], x = to_f32(r[0]), y = to_f32(r[1 & (VEC - 1)]);
                        from_f32(x * c - y * z, r[0]);
                        from_f32(x * z + y * c, r[1 & (VEC - 1)]);
                    }
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float c = cs[e], z = sn[e], x = to_f32(a[i].v[e]), y = to_f32(b[i].v[e]);
                    from_f32(x * c - y * z, a[i].v[e]);
                    from_f32(x * z + y * c, b[i].v[e]);
                }
            }
        }
        T *y = (T *)(s.y ? s.y : s.to_keys ? p.cache.k : p.cache.v) + s_to[side][token] + head * (s.y ? s.ys[1] : p.cache.head_stride);
        *reinterpret_cast<Run<T, VEC> *>(y + at.a) = a[i];
        if (at.has_b) *reinterpret_cast<Run<T, VEC> *>(y + at.b) = b[i];
    }
}

template <typename T, int VEC>
int launch(RopeParams &p, cudaStream_t st) {
    p.turned_chunks = p.rot / 2 / VEC;
    p.n_chunks = VEC == 1 ? (p.d + 1) / 2 : p.d / (2 * VEC);
    p.magic = ((1u << 20) + p.n_chunks - 1) / p.n_chunks;
    // a block's units are at most kUnits for each thread
    int tokens = kTokens;
    p.token_bits = 4;
    while (kUnits * kThreads < tokens * p.n_chunks) tokens >>= 1, --p.token_bits;
    static_assert(kUnits * kThreads >= 512, "a row has up to 512 units");
    const int most = kUnits * kThreads / (tokens * p.n_chunks);
    p.heads_per_block = most < p.n_heads ? most : p.n_heads;
    const int64_t tiles = ((int64_t)p.B * p.N + tokens - 1) / tokens;
    const int64_t slices = ((int64_t)p.n_heads + p.heads_per_block - 1) / p.heads_per_block;
    if (tiles > INT32_MAX || slices > 65535) return MATE_ERR_UNSUPPORTED;
    return launch_after(rope_kernel<T, VEC>, dim3((unsigned)tiles, (unsigned)slices), kThreads, sizeof(float) * tokens * p.rot, st, p) == cudaSuccess
               ? MATE_OK
               : MATE_ERR_CUDA;
}

// Whole runs of 16 bytes where the pairs, the rest of the row, every address and every stride allow it, else one
// element at a time.
int run(RopeParams &p, int dtype, cudaStream_t st) {
    if (p.B == 0 || p.N == 0 || p.n_heads == 0) return MATE_OK;
    const size_t size = elem_size(dtype);
    const int vec = (int)(16 / size);
    bool wide = p.rot % (2 * vec) == 0 && p.d % (2 * vec) == 0;
    for (int i = 0; i < p.n_sides && wide; ++i) {
        const Side &s = p.side[i];
        wide = is_aligned(s.x, 16) && (!s.y || is_aligned(s.y, 16));
        for (int j = 0; j < 3 && wide; ++j) wide = s.xs[j] % vec == 0 && (!s.y || s.ys[j] % vec == 0);
    }
    if (dtype == MATE_F32) return wide ? launch<float, 4>(p, st) : launch<float, 1>(p, st);
    return wide ? launch<__nv_bfloat16, 8>(p, st) : launch<__nv_bfloat16, 1>(p, st);
}

bool set_angles(RopeParams &p, const int32_t *positions, int64_t stride, const double *freqs, int rot, float mscale, unsigned flags) {
    if (flags & ~(unsigned)(MATE_ROPE_INTERLEAVED | MATE_ROPE_BACKWARD)) return false;
    p.positions = positions;
    p.position_stride = stride;
    p.freqs = freqs;
    p.rot = rot;
    p.mscale = mscale;
    p.interleaved = (flags & MATE_ROPE_INTERLEAVED) != 0;
    p.sign = flags & MATE_ROPE_BACKWARD ? -1.f : 1.f;
    return true;
}

}  // namespace
}  // namespace mate

extern "C" int mate_rope(const mate_rope_tensor_t *tensors, int n_tensors, int B, int N, int d, int dtype, const int32_t *positions,
                         int64_t position_stride, const double *freqs, int rot, float mscale, unsigned flags, void *stream) {
    using namespace mate;
    if (!tensors || n_tensors < 1 || n_tensors > 2 || B < 0 || N < 0 || d < 1 || rot < 0 || rot > d || rot % 2 != 0) return MATE_ERR_INVALID_ARG;
    if ((dtype != MATE_BF16 && dtype != MATE_F32) || d > 1024) return MATE_ERR_UNSUPPORTED;
    RopeParams p = {};
    if (!set_angles(p, positions, position_stride, freqs, rot, mscale, flags)) return MATE_ERR_INVALID_ARG;
    if (rot > 0 && (!freqs || !positions)) return MATE_ERR_INVALID_ARG;
    p.B = B, p.N = N, p.d = d;
    for (int i = 0; i < n_tensors; ++i) {
        const mate_rope_tensor_t &t = tensors[i];
        if (!t.x || !t.y || t.heads < 0) return MATE_ERR_INVALID_ARG;
        if (!is_aligned(t.x, elem_size(dtype)) || !is_aligned(t.y, elem_size(dtype))) return MATE_ERR_ALIGNMENT;
        if (t.heads == 0) continue;
        Side &s = p.side[p.n_sides++];
        s.x = t.x, s.y = t.y, s.heads = t.heads, s.turned = rot > 0;
        for (int j = 0; j < 3; ++j) s.xs[j] = t.x_stride[j], s.ys[j] = t.y_stride[j];
        if (p.n_heads > INT32_MAX - t.heads) return MATE_ERR_UNSUPPORTED;
        p.n_heads += t.heads;
    }
    return run(p, dtype, (cudaStream_t)stream);
}

extern "C" int mate_cache_append(const mate_cache_t *cache, int layer, const void *K, const void *V, const int64_t *k_stride,
                                 const int64_t *v_stride, int B, int N, const int32_t *seqs, const int32_t *counts,
                                 const int32_t *row_ids, const int32_t *col_ids, const int32_t *positions, const double *freqs, int rot,
                                 float mscale, unsigned flags, const void *Q, const int64_t *q_stride, void *Q_out,
                                 const int64_t *q_out_stride, void *stream) {
    using namespace mate;
    int rc = check_cache(cache);
    if (rc != MATE_OK) return rc;
    if (layer < 0 || layer >= cache->layers || !K || !V || !k_stride || !v_stride || B < 0 || N < 0 || (!row_ids) != (!col_ids))
        return MATE_ERR_INVALID_ARG;
    if (!seqs && B > cache->seqs) return MATE_ERR_INVALID_ARG;
    if (freqs ? rot < 0 || rot > cache->d || rot % 2 != 0 : rot != 0) return MATE_ERR_INVALID_ARG;
    if (Q ? !freqs || !Q_out || !q_stride || !q_out_stride : Q_out != nullptr) return MATE_ERR_INVALID_ARG;
    RopeParams p = {};
    if (!set_angles(p, positions, N, freqs, rot, mscale, flags)) return MATE_ERR_INVALID_ARG;
    const size_t size = elem_size(cache->dtype);
    for (const void *t : {K, V, Q, (const void *)Q_out})
        if (!is_aligned(t, size)) return MATE_ERR_ALIGNMENT;
    if ((rc = check_cache_device(cache)) != MATE_OK) return rc;
    p.B = B, p.N = N, p.d = cache->d;
    auto add = [&](const void *x, void *y, const int64_t *xs, const int64_t *ys, int heads, bool turned, bool to_keys) {
        Side &s = p.side[p.n_sides++];
        s.x = x, s.y = y, s.heads = heads, s.turned = turned, s.to_keys = to_keys;
        for (int j = 0; j < 3; ++j) s.xs[j] = xs[j], s.ys[j] = ys ? ys[j] : 0;
        p.n_heads += heads;
    };
    if (Q) add(Q, Q_out, q_stride, q_out_stride, cache->heads, rot > 0, false);
    add(K, nullptr, k_stride, nullptr, cache->kv_heads, rot > 0, true);
    add(V, nullptr, v_stride, nullptr, cache->kv_heads, false, false);
    p.paged = 1;
    p.cache = cache_args(cache, layer);
    p.seqs = seqs, p.counts = counts, p.row_ids = row_ids, p.col_ids = col_ids;
    return run(p, cache->dtype, (cudaStream_t)stream);
}

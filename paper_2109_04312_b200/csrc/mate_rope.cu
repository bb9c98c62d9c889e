// Rotary positions of one axis or several (mate_rope, mate_rope_axes) and new tokens into the pages of a cache (mate_cache_append,
// mate_cache_append_axes): one kernel, which turns rows of up to three tensors (queries, keys; values are only copied) and writes them by
// strides or through a page table.
//
// A pair (a, b) becomes m (a cos t - b sin t, a sin t + b cos t), t = position * freqs[pair]; the transpose has -t.  The
// angle's whole turns do not matter, so a frequency is kept as a 64-bit fraction of a turn per position and multiplied by the
// position modulo 2^64: exact but for the fraction's own rounding (2^-65 turns per position and the 2^-53 of the 64-bit
// frequency), for three integer instructions.  (In 64-bit floating point the same took most of the kernel's time.)  Sine and
// cosine of the fraction that is left are taken in fp32 by sincospif, with 32 bits of it: fp32 holds 24, what they leave (9e-8 rad at
// most) is added to first order where the elements are fp32.
//
// Bound by memory: one read and one write of every element.  A thread has one token and one unit of its rows -- two runs of VEC
// elements, which are VEC pairs -- works out their sines and cosines once and takes the heads of its slice in turn, kFlight at
// a time with all their loads under way (the first ones before the sines).
#include <cuda_bf16.h>

#include "mate_cache.h"
#include "sm100_ptx.cuh"

namespace mate {
namespace {

constexpr int kThreads = 128;
constexpr int kFlight = 4;  // heads of a thread that are under way together

struct Side {
    const void *x;
    void *y;  // null: into the cache's pages (of keys or of values)
    int64_t xs[3], ys[3];
    int heads;
    int turned, to_keys;
    int first_slice;  // slices of heads are numbered through over the sides
};
struct RopeParams {
    static constexpr bool kAxes = false;
    Side side[3];
    int n_sides;
    int B, N, d, rot, interleaved;
    const int32_t *positions;
    int64_t position_stride;
    const double *freqs;
    float mscale, sign;
    int n_chunks, turned_chunks;  // units of a head, and how many of them are pairs
    int heads_of_thread;
    // new tokens of a cache
    int paged;
    CacheArgs cache;
    const int32_t *seqs, *counts, *row_ids, *col_ids;
};
// Positions of several axes, of which every pair goes by one: a thread takes its token's up to four positions and picks a pair's by two bits, 4 x
// 2048 tokens, 12 and 12 heads of 64 11.0 us (one axis 10.0), 32768 tokens, 32 and 8 heads of 128 backward 107 (106).  (Parameters of their own:
// those of one axis are copied with every launch.)
constexpr int kMaxAxes = 4, kMaxPairs = 512;
struct AxesParams : RopeParams {
    static constexpr bool kAxes = true;
    int n_axes;
    int64_t axis_stride;
    uint32_t axis[kMaxPairs / 16];  // two bits a pair; the pairs of a unit lie in one word
};

// VEC elements, as they lie in memory and as numbers
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Run {
    T v[VEC];
};
template <int VEC>
__device__ __forceinline__ void unpack(const Run<float, VEC> &r, float (&x)[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = r.v[i];
}
template <int VEC>
__device__ __forceinline__ void pack(const float (&x)[VEC], Run<float, VEC> &r) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) r.v[i] = x[i];
}
__device__ __forceinline__ void unpack(const Run<__nv_bfloat16, 1> &r, float (&x)[1]) { x[0] = __bfloat162float(r.v[0]); }
__device__ __forceinline__ void pack(const float (&x)[1], Run<__nv_bfloat16, 1> &r) { r.v[0] = __float2bfloat16_rn(x[0]); }
template <int VEC>
__device__ __forceinline__ void unpack(const Run<__nv_bfloat16, VEC> &r, float (&x)[VEC]) {
    const uint32_t *w = reinterpret_cast<const uint32_t *>(&r);
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
}
template <int VEC>
__device__ __forceinline__ void pack(const float (&x)[VEC], Run<__nv_bfloat16, VEC> &r) {
    uint32_t *w = reinterpret_cast<uint32_t *>(&r);
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) w[i] = ptx::cvt_bf16x2(x[2 * i], x[2 * i + 1]);
}

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

template <typename T, int VEC, typename P>
__global__ void __launch_bounds__(kThreads, 6) rope_kernel(const __grid_constant__ P p) {
    extern __shared__ uint64_t s_turn[];  // [rot / 2] turns per position, in 2^-64
    ptx::launch_dependents();
    ptx::wait_prior_grid();
    const double freq = threadIdx.x < p.rot / 2 ? p.freqs[threadIdx.x] : 0.;  // (ahead of all else: what it becomes is waited for by all)
    const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x, t = at / p.n_chunks;
    const int chunk = (int)(at - t * p.n_chunks), b = (int)(t / p.N), n = (int)(t - (int64_t)b * p.N);
    const int side = (int)(p.n_sides > 1 && blockIdx.y >= p.side[1].first_slice) + (int)(p.n_sides > 2 && blockIdx.y >= p.side[2].first_slice);
    const Side &s = p.side[side];
    const int h0 = (blockIdx.y - s.first_slice) * p.heads_of_thread, n_heads = min(s.heads - h0, p.heads_of_thread);
    const bool exists = b < p.B;
    // a row of queries always goes somewhere; one of keys or values if its sequence has the token
    int q = 0, count = p.N;
    if (p.paged && exists) {
        q = seq_of(p.seqs, b, p.cache.seqs);
        if (p.counts) count = p.counts[b];
        if ((q < 0 || count < 0 || count > p.N) && chunk == 0 && blockIdx.y == 0) atomicOr(p.cache.status, kCacheBad);
        if (q < 0 || count > p.N) count = 0;
    }
    bool goes = exists && (s.y || n < count);
    const Place place_of = place<VEC>(p, chunk, s.turned);
    const int second = place_of.b - place_of.a;  // from one run to the other
    const bool two = VEC > 1 || place_of.has_b;
    const T *from = (const T *)s.x + b * s.xs[0] + h0 * s.xs[1] + n * s.xs[2] + place_of.a;
    const int64_t from_step = s.xs[1], to_step = s.y ? s.ys[1] : p.cache.head_stride;
    Run<T, VEC> x[kFlight], y[kFlight];
    auto load = [&](int h) {
        if (!goes) return;
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            if (h + i >= n_heads) break;
            x[i] = *reinterpret_cast<const Run<T, VEC> *>(from);
            if (two) y[i] = *reinterpret_cast<const Run<T, VEC> *>(from + second);
            from += from_step;
        }
    };
    load(0);

    // the token's position and, in a cache, its slot (the loads above are under way)
    int position = p.positions && exists ? p.positions[b * p.position_stride + n] : 0;
    [[maybe_unused]] int others[kMaxAxes - 1];  // its positions of the other axes
    [[maybe_unused]] uint32_t axes = 0;         // of the unit's pairs
    if constexpr (P::kAxes) {
#pragma unroll
        for (int a = 1; a < kMaxAxes; ++a)
            others[a - 1] = p.positions && exists && a < p.n_axes ? p.positions[a * p.axis_stride + b * p.position_stride + n] : 0;
        if (s.turned && chunk < p.turned_chunks) axes = p.axis[chunk * VEC / 16] >> 2 * (chunk * VEC % 16);
    }
    int64_t page_at = 0;
    if (p.paged && exists && n < count) {
        bool bad = false;
        const int place_in = clip_len(p.cache.lens[q], p.cache.width * p.cache.page_size, &bad) - count + n;
        if (!p.positions) position = place_in;
        int page = -1;
        if (place_in >= 0 && !bad) {
            const int i = place_in / p.cache.page_size, slot = place_in - i * p.cache.page_size;
            page = p.cache.table[(size_t)q * p.cache.width + i];
            if (in_range(page, p.cache.pages)) {
                page_at = page * p.cache.page_stride + slot * p.cache.slot_stride;
                if (p.row_ids && blockIdx.y == 0 && chunk == 0) {
                    const size_t id = (size_t)page * p.cache.page_size + slot;
                    p.cache.row_ids[id] = p.row_ids[t];
                    p.cache.col_ids[id] = p.col_ids[t];
                }
            }
        }
        if (!in_range(page, p.cache.pages)) {
            if (blockIdx.y == 0 && chunk == 0) atomicOr(p.cache.status, kCacheBad);
            goes = s.y;
        }
    }
    T *to = s.y ? (T *)s.y + b * s.ys[0] + h0 * s.ys[1] + n * s.ys[2] + place_of.a
                : (T *)(s.to_keys ? p.cache.k : p.cache.v) + page_at + h0 * p.cache.head_stride + place_of.a;

    for (int i = threadIdx.x; i < p.rot / 2; i += kThreads) {
        const double turns = (i < kThreads ? freq : p.freqs[i]) * 0.15915494309189533577;
        s_turn[i] = (uint64_t)__double2ull_rn((turns - floor(turns)) * 18446744073709551616.0);
    }
    __syncthreads();
    if (!goes) return;
    const bool turned = s.turned && chunk < p.turned_chunks;
    float cs[VEC], sn[VEC];
    if (turned) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            int at_axis = position;
            if constexpr (P::kAxes) {
                const uint32_t a = axes >> 2 * e & 3;
                at_axis = a & 2 ? (a & 1 ? others[2] : others[1]) : (a & 1 ? others[0] : position);
            }
            const int64_t turn = (int64_t)(s_turn[chunk * VEC + e] * (uint64_t)(int64_t)at_axis);
            const int32_t half_turns = (int32_t)(turn >> 32);  // in 2^-31
            const float rounded = (float)half_turns;
            sincospif(rounded * 4.656612873077393e-10f, &sn[e], &cs[e]);  // 2^-31
            if (sizeof(T) == 4) {  // bf16 does not show what the rounding left
                const float rest = (float)(half_turns - __float2int_rn(rounded)) * 1.4629180792671596e-9f;  // pi 2^-31
                const float c = cs[e];
                cs[e] = fmaf(-sn[e], rest, c);
                sn[e] = fmaf(c, rest, sn[e]);
            }
            cs[e] *= p.mscale;
            sn[e] *= p.mscale * p.sign;
        }
    }
    for (int h = 0; h < n_heads; h += kFlight) {
        if (h > 0) load(h);
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            if (h + i >= n_heads) break;
            if (turned) {
                float u[VEC], w[VEC];
                unpack(x[i], u);
                unpack(y[i], w);
                if (p.interleaved && VEC > 1) {  // pairs lie side by side, VEC / 2 in each run
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        float &c = (e < VEC / 2 ? u : w)[2 * e % VEC], &d = (e < VEC / 2 ? u : w)[(2 * e + 1) % VEC];
                        const float c0 = c;
                        c = c0 * cs[e] - d * sn[e];
                        d = c0 * sn[e] + d * cs[e];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float u0 = u[e];
                        u[e] = u0 * cs[e] - w[e] * sn[e];
                        w[e] = u0 * sn[e] + w[e] * cs[e];
                    }
                }
                pack(u, x[i]);
                pack(w, y[i]);
            }
            *reinterpret_cast<Run<T, VEC> *>(to) = x[i];
            if (two) *reinterpret_cast<Run<T, VEC> *>(to + second) = y[i];
            to += to_step;
        }
    }
}

template <typename T, int VEC, typename P>
int launch(P &p, int device, cudaStream_t st) {
    p.turned_chunks = p.rot / 2 / VEC;
    p.n_chunks = VEC == 1 ? (p.d + 1) / 2 : p.d / (2 * VEC);
    if ((int64_t)p.B * p.N > (int64_t)INT32_MAX * kThreads / p.n_chunks) return MATE_ERR_UNSUPPORTED;
    const int64_t threads = (int64_t)p.B * p.N * p.n_chunks, blocks = (threads + kThreads - 1) / kThreads;
    // As many heads to a thread as leave every SM 1024 of them, in whole batches (4 x 2048 tokens, 12 and 12 heads: 9.0 us; with 2048
    // threads, that is four heads each, 12.8).  New tokens of a cache, whose slots have to be looked up first: 2048 (eight tables in
    // 23.0 us; 23.9 with 1024, 28.1 with 4096).
    int64_t n_heads = 0, slices = 0;
    for (int i = 0; i < p.n_sides; ++i) n_heads += p.side[i].heads;
    const double per_thread = (double)threads * n_heads / ((p.paged ? 2048. : 1024.) * n_sms(device));  // (the product passes 64 bits)
    const int64_t heads = per_thread < n_heads ? (int64_t)per_thread : n_heads;
    p.heads_of_thread = heads <= 2 ? (heads < 1 ? 1 : (int)heads) : (int)(heads + kFlight - 1) / kFlight * kFlight;
    constexpr int kSlices = 65535 - 3;  // of a launch, less the last ones of three tensors, which are not full
    if (n_heads > (int64_t)kSlices * p.heads_of_thread) p.heads_of_thread = (int)((n_heads + kSlices - 1) / kSlices);
    for (int i = 0; i < p.n_sides; ++i) {
        p.side[i].first_slice = (int)slices;
        slices += (p.side[i].heads + p.heads_of_thread - 1) / p.heads_of_thread;
    }
    return launch_after(rope_kernel<T, VEC, P>, dim3((unsigned)blocks, (unsigned)slices), kThreads, sizeof(uint64_t) * (p.rot / 2), st, p) == cudaSuccess
               ? MATE_OK
               : MATE_ERR_CUDA;
}

// Runs of 16 bytes, or of 8, where the pairs, the rest of the row, every address and every stride allow it, else one element at
// a time.  (4 x 4096 tokens, 12 and 12 heads of 80 elements, 40 of them turned: runs of 8 bytes 23.6 us, single elements 46.0.)
template <typename P>
int run(P &p, int dtype, cudaStream_t st) {
    if (p.B == 0 || p.N == 0 || p.n_sides == 0) return MATE_OK;
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess) return MATE_ERR_CUDA;
    const int size = (int)elem_size(dtype);
    const auto fits = [&](int bytes) {
        const int vec = bytes / size;
        if (p.rot % (2 * vec) != 0 || p.d % (2 * vec) != 0) return false;
        for (int i = 0; i < p.n_sides; ++i) {
            const Side &s = p.side[i];
            if (!is_aligned(s.x, bytes) || (s.y && !is_aligned(s.y, bytes))) return false;
            for (int j = 0; j < 3; ++j)
                if (s.xs[j] % vec != 0 || (s.y && s.ys[j] % vec != 0)) return false;
        }
        return true;
    };
    const bool wide = fits(16), half = fits(8);
    if (dtype == MATE_F32) return wide ? launch<float, 4>(p, device, st) : half ? launch<float, 2>(p, device, st) : launch<float, 1>(p, device, st);
    return wide   ? launch<__nv_bfloat16, 8>(p, device, st)
           : half ? launch<__nv_bfloat16, 4>(p, device, st)
                  : launch<__nv_bfloat16, 1>(p, device, st);
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

bool set_axes(RopeParams &, const uint8_t *, int, int64_t, int) { return true; }
bool set_axes(AxesParams &p, const uint8_t *axes, int n_axes, int64_t stride, int rot) {
    if (n_axes < 1 || (rot > 0 && !axes)) return false;
    p.n_axes = n_axes;
    p.axis_stride = stride;
    for (int i = 0; i < rot / 2; ++i) {
        if (axes[i] >= n_axes) return false;
        p.axis[i / 16] |= (uint32_t)axes[i] << 2 * (i % 16);
    }
    return true;
}

template <typename P>
int turn(const mate_rope_tensor_t *tensors, int n_tensors, int B, int N, int d, int dtype, const int32_t *positions, int64_t position_stride,
         const uint8_t *axes, int n_axes, int64_t axis_stride, const double *freqs, int rot, float mscale, unsigned flags, void *stream) {
    if (!tensors || n_tensors < 1 || n_tensors > 2 || B < 0 || N < 0 || d < 1 || rot < 0 || rot > d || rot % 2 != 0) return MATE_ERR_INVALID_ARG;
    if ((dtype != MATE_BF16 && dtype != MATE_F32) || d > 2 * kMaxPairs || n_axes > kMaxAxes) return MATE_ERR_UNSUPPORTED;
    P p = {};
    if (!set_angles(p, positions, position_stride, freqs, rot, mscale, flags)) return MATE_ERR_INVALID_ARG;
    if (!set_axes(p, axes, n_axes, axis_stride, rot)) return MATE_ERR_INVALID_ARG;
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
    }
    return run(p, dtype, (cudaStream_t)stream);
}

template <typename P>
int append(const mate_cache_t *cache, int layer, const void *K, const void *V, const int64_t *k_stride, const int64_t *v_stride, int B, int N,
           const int32_t *seqs, const int32_t *counts, const int32_t *row_ids, const int32_t *col_ids, const int32_t *positions,
           const uint8_t *axes, int n_axes, const double *freqs, int rot, float mscale, unsigned flags, const void *Q, const int64_t *q_stride,
           void *Q_out, const int64_t *q_out_stride, void *stream) {
    int rc = check_cache(cache);
    if (rc != MATE_OK) return rc;
    if (layer < 0 || layer >= cache->layers || !K || !V || !k_stride || !v_stride || B < 0 || N < 0 || (!row_ids) != (!col_ids))
        return MATE_ERR_INVALID_ARG;
    if (!seqs && B > cache->seqs) return MATE_ERR_INVALID_ARG;
    if (freqs ? rot < 0 || rot > cache->d || rot % 2 != 0 : rot != 0) return MATE_ERR_INVALID_ARG;
    if (Q ? !freqs || !Q_out || !q_stride || !q_out_stride : Q_out != nullptr) return MATE_ERR_INVALID_ARG;
    if (n_axes > kMaxAxes) return MATE_ERR_UNSUPPORTED;
    P p = {};
    if (!set_angles(p, positions, N, freqs, rot, mscale, flags)) return MATE_ERR_INVALID_ARG;
    if (!set_axes(p, axes, n_axes, (int64_t)B * N, rot) || (P::kAxes && rot > 0 && !positions)) return MATE_ERR_INVALID_ARG;
    const size_t size = elem_size(cache->dtype);
    for (const void *t : {K, V, Q, (const void *)Q_out})
        if (!is_aligned(t, size)) return MATE_ERR_ALIGNMENT;
    if ((rc = check_cache_device(cache)) != MATE_OK) return rc;
    p.B = B, p.N = N, p.d = cache->d;
    auto add = [&](const void *x, void *y, const int64_t *xs, const int64_t *ys, int heads, bool turned, bool to_keys) {
        Side &s = p.side[p.n_sides++];
        s.x = x, s.y = y, s.heads = heads, s.turned = turned, s.to_keys = to_keys;
        for (int j = 0; j < 3; ++j) s.xs[j] = xs[j], s.ys[j] = ys ? ys[j] : 0;
    };
    if (Q) add(Q, Q_out, q_stride, q_out_stride, cache->heads, rot > 0, false);
    add(K, nullptr, k_stride, nullptr, cache->kv_heads, rot > 0, true);
    add(V, nullptr, v_stride, nullptr, cache->kv_heads, false, false);
    p.paged = 1;
    p.cache = cache_args(cache, layer);
    p.seqs = seqs, p.counts = counts, p.row_ids = row_ids, p.col_ids = col_ids;
    return run(p, cache->dtype, (cudaStream_t)stream);
}

}  // namespace
}  // namespace mate

using namespace mate;

extern "C" {

int mate_rope(const mate_rope_tensor_t *tensors, int n_tensors, int B, int N, int d, int dtype, const int32_t *positions,
              int64_t position_stride, const double *freqs, int rot, float mscale, unsigned flags, void *stream) {
    return turn<RopeParams>(tensors, n_tensors, B, N, d, dtype, positions, position_stride, nullptr, 1, 0, freqs, rot, mscale, flags, stream);
}

int mate_rope_axes(const mate_rope_tensor_t *tensors, int n_tensors, int B, int N, int d, int dtype, const int32_t *positions,
                   int64_t axis_stride, int64_t position_stride, const uint8_t *axes, int n_axes, const double *freqs, int rot, float mscale,
                   unsigned flags, void *stream) {
    return turn<AxesParams>(tensors, n_tensors, B, N, d, dtype, positions, position_stride, axes, n_axes, axis_stride, freqs, rot, mscale, flags,
                            stream);
}

int mate_cache_append(const mate_cache_t *cache, int layer, const void *K, const void *V, const int64_t *k_stride, const int64_t *v_stride,
                      int B, int N, const int32_t *seqs, const int32_t *counts, const int32_t *row_ids, const int32_t *col_ids,
                      const int32_t *positions, const double *freqs, int rot, float mscale, unsigned flags, const void *Q,
                      const int64_t *q_stride, void *Q_out, const int64_t *q_out_stride, void *stream) {
    return append<RopeParams>(cache, layer, K, V, k_stride, v_stride, B, N, seqs, counts, row_ids, col_ids, positions, nullptr, 1, freqs, rot,
                              mscale, flags, Q, q_stride, Q_out, q_out_stride, stream);
}

int mate_cache_append_axes(const mate_cache_t *cache, int layer, const void *K, const void *V, const int64_t *k_stride,
                           const int64_t *v_stride, int B, int N, const int32_t *seqs, const int32_t *counts, const int32_t *row_ids,
                           const int32_t *col_ids, const int32_t *positions, const uint8_t *axes, int n_axes, const double *freqs, int rot,
                           float mscale, unsigned flags, const void *Q, const int64_t *q_stride, void *Q_out, const int64_t *q_out_stride,
                           void *stream) {
    if (!freqs || !positions) return MATE_ERR_INVALID_ARG;
    return append<AxesParams>(cache, layer, K, V, k_stride, v_stride, B, N, seqs, counts, row_ids, col_ids, positions, axes, n_axes, freqs, rot,
                              mscale, flags, Q, q_stride, Q_out, q_out_stride, stream);
}

}  // extern "C"

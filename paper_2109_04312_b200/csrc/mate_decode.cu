// Attention of one new token per sequence over the cached ones (mate_attn_decode).
#include <cuda_bf16.h>

#include "mate_cache.h"
#include "sm100_ptx.cuh"

namespace mate {
namespace {

constexpr int kThreads = 128;

struct DecodeParams {
    CacheArgs cache;
    const void *Q;
    int64_t q_batch, q_head;
    int B, heads, group, d, max_len;
    const int32_t *seqs, *row_ids, *col_ids;
    float scale;
    void *O;
    float *LSE;
    uint32_t views[64];  // two bits a head
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f32(float x, float &y) { y = x; }
__device__ __forceinline__ void from_f32(float x, __nv_bfloat16 &y) { y = __float2bfloat16_rn(x); }

// One block per (sequence, head): 128 keys at a time, one per thread, then one column of V per thread.
template <typename T>
__global__ void __launch_bounds__(kThreads) decode_kernel(const __grid_constant__ DecodeParams p) {
    __shared__ float s_q[128], s_p[kThreads], s_red[4];
    __shared__ int64_t s_at[kThreads];
    ptx::launch_dependents();
    ptx::wait_prior_grid();
    const int b = blockIdx.y, h = blockIdx.x, tid = threadIdx.x, kv = h / p.group;
    const CacheArgs &c = p.cache;
    const int view = p.views[h >> 4] >> 2 * (h & 15) & 3;
    const int s = seq_of(p.seqs, b, c.seqs), q_row = p.row_ids[b], q_col = p.col_ids[b];
    bool bad = s < 0;
    int len = bad ? 0 : clip_len(c.lens[s], p.max_len, &bad);
    if (q_row < 0 || q_col < 0) len = 0;
    const int prefix = s < 0 ? 0 : c.prefix[s];
    const bool text = q_row == MATE_ID_TEXT || q_col == MATE_ID_TEXT;
    if (tid < p.d) s_q[tid] = to_f32(((const T *)p.Q)[b * p.q_batch + h * p.q_head + tid]) * p.scale;
    float m = -INFINITY, l = 0.f, acc = 0.f;
    for (int j0 = 0; j0 < len; j0 += kThreads) {
        const int j = j0 + tid;
        int64_t at = -1;
        if (j < len) {
            const int i = j / c.page_size, slot = j - i * c.page_size, page = c.table[(size_t)s * c.width + i];
            if (!in_range(page, c.pages)) {
                bad = true;
            } else {
                const int row = c.row_ids[(size_t)page * c.page_size + slot], col = c.col_ids[(size_t)page * c.page_size + slot];
                const bool all = text || j < prefix;
                const bool by_row = row >= 0 && (all || row == MATE_ID_TEXT || row == q_row);
                const bool by_col = col >= 0 && (all || col == MATE_ID_TEXT || col == q_col);
                if (view == MATE_VIEW_ROW ? by_row : view == MATE_VIEW_COL ? by_col : by_row || by_col)
                    at = page * c.page_stride + kv * c.head_stride + slot * c.slot_stride;
            }
        }
        __syncthreads();
        float x = -INFINITY;
        if (at >= 0) {
            x = 0.f;
            const T *k = (const T *)c.k + at;
            for (int e = 0; e < p.d; ++e) x = fmaf(s_q[e], to_f32(k[e]), x);
        }
        float top = x;
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
        if ((tid & 31) == 0) s_red[tid >> 5] = top;
        s_at[tid] = at;
        __syncthreads();
        const float m2 = fmaxf(fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3])), m);
        const float base = m2 == -INFINITY ? 0.f : m2;
        s_p[tid] = expf(x - base);
        __syncthreads();
        const float keep = expf(m - base);
        m = m2;
        l *= keep, acc *= keep;
        for (int i = 0; i < kThreads; ++i) {
            if (s_at[i] < 0) continue;
            l += s_p[i];
            if (tid < p.d) acc = fmaf(s_p[i], to_f32(((const T *)c.v)[s_at[i] + tid]), acc);
        }
    }
    const size_t row = (size_t)b * p.heads + h;
    if (tid < p.d) from_f32(l > 0.f ? acc / l : 0.f, ((T *)p.O)[row * p.d + tid]);
    if (tid == 0) p.LSE[row] = l > 0.f ? m + logf(l) : -INFINITY;
    if (bad) atomicOr(c.status, kCacheBad);
}

}  // namespace

size_t decode_workspace(const mate_cache_t *, int) { return 0; }

}  // namespace mate

extern "C" int mate_attn_decode(const mate_cache_t *cache, int layer, const void *Q, const int64_t *q_stride, int B, const int32_t *seqs,
                                const int32_t *row_ids, const int32_t *col_ids, float scale, int max_len, void *O, float *LSE,
                                void *workspace, size_t workspace_bytes, void *stream) {
    using namespace mate;
    int rc = check_cache(cache);
    if (rc != MATE_OK) return rc;
    if (layer < 0 || layer >= cache->layers || B < 0 || max_len < 0 || (!seqs && B > cache->seqs)) return MATE_ERR_INVALID_ARG;
    if (B > 0 && (!Q || !q_stride || !row_ids || !col_ids || !O || !LSE)) return MATE_ERR_INVALID_ARG;
    if (cache->heads > 1024 || B > 65535) return MATE_ERR_UNSUPPORTED;
    const int vec = (int)(16 / elem_size(cache->dtype));
    if (B > 0 && (!is_aligned(Q, 16) || !is_aligned(O, 16) || !is_aligned(LSE, 4) || q_stride[0] % vec != 0 || q_stride[1] % vec != 0))
        return MATE_ERR_ALIGNMENT;
    if ((rc = check_cache_device(cache)) != MATE_OK) return rc;
    if (B == 0) return MATE_OK;
    DecodeParams p = {};
    p.cache = cache_args(cache, layer);
    p.Q = Q, p.q_batch = q_stride[0], p.q_head = q_stride[1];
    p.B = B, p.heads = cache->heads, p.group = cache->heads / cache->kv_heads, p.d = cache->d;
    const int most = cache->width * cache->page_size;
    p.max_len = max_len > 0 && max_len < most ? max_len : most;
    p.seqs = seqs, p.row_ids = row_ids, p.col_ids = col_ids;
    p.scale = scale, p.O = O, p.LSE = LSE;
    for (int h = 0; h < cache->heads; ++h) p.views[h >> 4] |= (uint32_t)cache->head_view[h] << 2 * (h & 15);
    const dim3 grid((unsigned)cache->heads, (unsigned)B);
    const cudaError_t e = cache->dtype == MATE_F32 ? launch_after(decode_kernel<float>, grid, kThreads, 0, (cudaStream_t)stream, p)
                                                   : launch_after(decode_kernel<__nv_bfloat16>, grid, kThreads, 0, (cudaStream_t)stream, p);
    return e == cudaSuccess ? MATE_OK : MATE_ERR_CUDA;
}

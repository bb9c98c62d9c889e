/*
 * libmate -- multi-view (row head / column head / global prefix) sparse self-attention for
 * flattened tables, hand-written CUDA for sm_100a.
 *
 * The operation is the one defined in Section 3 of "MATE: Multi-view Attention for Table
 * Transformer Efficiency": for head i and token position k the output is a softmax-weighted sum of
 * the values of the positions in the attention pattern A^i_k,
 *     k in Q (the query/text prefix)  ->  A = every position (except padding)
 *     row head,    k not in Q         ->  A = Q  u  { j : r_j = r_k }
 *     column head, k not in Q         ->  A = Q  u  { j : c_j = c_k }
 * applied after the Q/K/V projections (Q, K, V are inputs here).  Section 3.1's observation that
 * every head may traverse the tokens in its own data-dependent, deterministic order is what
 * mate_plan pre-computes: in a head's view order each table token's keys are one contiguous
 * segment plus the prefix block.
 *
 * Conventions (the paper leaves them open):
 *   - Q is the first prefix_len positions; their row and column ids must be 0.
 *   - a negative id marks padding (both arrays must agree).  Padding keys are never attended;
 *     padding query rows return O = 0, LSE = -inf and zero gradients; values stored at padding
 *     positions are ignored, whatever they are.  (A NaN or Inf at a valid position may also reach rows
 *     of its example that do not attend it: tiles are multiplied whole, masked pairs with weight 0.)
 *   - a table token whose id is 0 is an ordinary table token (segment 0).
 *   - masking removes a key from the softmax support; `scale` multiplies q.k before the softmax.
 *   - LSE is the natural-log logsumexp of the scaled scores over A.
 *
 * All tensor pointers are DEVICE pointers unless a comment says "host".  The library never keeps
 * or frees caller memory.  Every call returns a status (0 = MATE_OK, negative = error); nothing
 * throws across this boundary.  Calls taking a `stream` (a cudaStream_t passed as void*) enqueue
 * work on it and return without waiting, except mate_plan, which waits for its own kernels.
 */
#ifndef MATE_H_
#define MATE_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct mate_plan_s mate_plan_t;

enum {
    MATE_OK = 0,
    MATE_ERR_INVALID_ARG = -1, /* null pointer, bad size, ids that break the conventions above     */
    MATE_ERR_UNSUPPORTED = -2, /* head dim / dtype / implementation not available for these sizes   */
    MATE_ERR_ALIGNMENT = -3,   /* a tensor pointer is not 16-byte aligned                           */
    MATE_ERR_CUDA = -4,        /* a CUDA runtime call failed (the CUDA error is left in place)      */
    MATE_ERR_TIMEOUT = -5,     /* a bounded wait inside a kernel expired (see mate_plan_status)     */
    MATE_ERR_NOMEM = -6,       /* host or device allocation failed                                  */
    MATE_ERR_WORKSPACE = -7,   /* workspace pointer null or smaller than mate_attn_workspace_bytes  */
    MATE_ERR_TOO_LARGE = -8    /* problem exceeds the built-in scratch of mate_attn_bwd_noalloc      */
};

enum { MATE_BF16 = 0, MATE_F32 = 1 };          /* element type of Q, K, V, O, dO, dQ, dK, dV */
enum { MATE_VIEW_ROW = 0, MATE_VIEW_COL = 1 }; /* entries of head_view                      */

/* flags for mate_attn_fwd / mate_attn_bwd: which implementation runs.
 *   AUTO     tensor-core (tcgen05) kernels when dtype = bf16 and d = 64, otherwise the SIMT kernels
 *   SIMT     fp32-arithmetic kernels without tensor cores (any dtype, d <= 128)
 *   TCGEN05  tensor-core kernels or MATE_ERR_UNSUPPORTED */
enum { MATE_IMPL_AUTO = 0, MATE_IMPL_SIMT = 1, MATE_IMPL_TCGEN05 = 2 };

/* further flag bits (or-ed to the implementation choice):
 *   VIEW_ORDER   (mate_attn_fwd only) Q, K, V are laid out, head by head, in that head's own order
 *                (row b, h, t of a tensor holds the token at position t of the order mate_plan computed
 *                for the head's view), and O and LSE are returned in the same order: what a producer
 *                that writes its projections through the plan's order provides (Section 3.1: the
 *                reordering can be folded into the neighbouring steps).  No gather, no scatter; the
 *                tensor-core kernel then fetches every full K/V tile with bulk tensor copies.  Not for
 *                mate_plan_sat plans and not for mate_attn_bwd (MATE_ERR_UNSUPPORTED).
 *   BULK_TILES   the tensor-core forward fetches the full K/V tiles (and those of a multiple of 16
 *                columns) that are contiguous in the tensors -- of the prefix block of every head and, for
 *                a row-major table, of the row view -- with bulk tensor copies (one per tile and matrix)
 *                instead of row-by-row gathers.  Same results bit for bit.  This is the default wherever
 *                the driver provides tensor maps, so the bit only states it.
 *   GATHER_TILES every K/V tile is gathered row by row.  (Timed back to back on sequences of 512 to
 *                8192 positions, bulk copies are up to 0.7 % faster.)  Both bits together: MATE_ERR_INVALID_ARG. */
enum { MATE_FLAG_VIEW_ORDER = 4, MATE_FLAG_BULK_TILES = 8, MATE_FLAG_GATHER_TILES = 16 };

const char *mate_status_string(int status);

/* Pre-computes, for both views, the per-head token order of Section 3.1 (Figure 2): a stable
 * counting sort of the positions by (prefix, table id, padding), i.e. the row-order / column-order
 * traversal of the table, together with the segment offsets and the tile work-lists the attention
 * kernels walk.  Integer work; the result is unique (ties keep the original order).
 *
 *   row_ids, col_ids  device int32 [B, N]
 *   prefix_len        |Q|, 0 <= prefix_len <= N
 *   head_view         HOST uint8 [H], MATE_VIEW_ROW or MATE_VIEW_COL per head (any mix, one view
 *                     may have no head)
 *   max_row_id, max_col_id   inclusive upper bounds of the non-negative ids
 *   out               receives a plan owned by the library; free it with mate_plan_destroy
 *
 * The plan can be reused for any number of forward/backward calls, layers and head dims, on the
 * device that was current when it was made (calls with another device current return
 * MATE_ERR_INVALID_ARG).  It also holds a few scheduling counters of the tensor-core forward, so
 * calls that use ONE plan -- mate_attn_fwd, mate_plan_status -- must not overlap on the GPU: put
 * them on one stream or order them with events.  Work that should overlap (two streams) needs one
 * plan per stream; mate_attn_bwd keeps its counters in its workspace and only needs separate
 * workspaces.  Runs its kernels on `stream` and waits for them (it allocates device memory, so call
 * it outside a stream capture).  Ids that break the conventions give MATE_ERR_INVALID_ARG and no
 * plan. */
int mate_plan(const int32_t *row_ids, const int32_t *col_ids, int B, int N, int prefix_len,
              const uint8_t *head_view, int H, int max_row_id, int max_col_id, void *stream,
              mate_plan_t **out);

/* The same plan for the bucketed, approximate form of the pattern (Section 3.1 and Appendix D: a
 * global section G, which here is the prefix, and a local section cut into buckets of R positions
 * of each head's own order; the paper uses R = 42).  In a head's order the positions behind the
 * prefix form buckets of `radius` consecutive positions; a table token attends the prefix and,
 * of its own row / column, only the keys in its own bucket and the two adjacent ones.  Prefix
 * tokens still attend every non-padding position.  The order (perm, inv_perm, seg_off) is that
 * of mate_plan; only the key ranges, the work-lists and the pair counts differ.  The pattern
 * stays symmetric, so the forward and the backward calls take such a plan unchanged.  A radius
 * at least as long as the longest row / column segment gives back the exact pattern, as the
 * paper notes; radius = 0 means exactly that (mate_plan); radius < 0 is MATE_ERR_INVALID_ARG.
 * All other arguments, ownership and errors as for mate_plan. */
int mate_plan_bucketed(const int32_t *row_ids, const int32_t *col_ids, int B, int N, int prefix_len,
                       const uint8_t *head_view, int H, int max_row_id, int max_col_id, int radius,
                       void *stream, mate_plan_t **out);

/* The bucketed form with a global section that may be longer than the prefix (Section 3.1: the first
 * G tokens of a head's order attend to and from everything, with G at least the length of the
 * question; Appendix A.2 uses G = 116, R = 42): the first global_len[b] positions of each head's
 * own order -- the prefix and, beyond it, the table tokens that come first in that order -- see
 * every non-padding position and are seen by all of them; the positions behind are cut into
 * buckets of `radius`, counted from global_len[b], and attend the global section plus, of their own
 * row / column, their own bucket and the two adjacent ones.  prefix_len and global_len are HOST
 * int32 [B] arrays with prefix_len[b] <= global_len[b] <= N; radius > 0.  global_len = prefix_len
 * is mate_plan_varlen.  All other arguments, ownership and errors as for mate_plan. */
int mate_plan_bucketed_global(const int32_t *row_ids, const int32_t *col_ids, int B, int N, const int32_t *prefix_len,
                              const int32_t *global_len, const uint8_t *head_view, int H, int max_row_id,
                              int max_col_id, int radius, void *stream, mate_plan_t **out);

/* The same with one prefix length per example (the paper's inputs are a question or a passage of
 * varying length followed by the table, Section 3 and Section 5; its formula takes the set Q per
 * example).  prefix_len is a HOST int32 [B] array, 0 <= prefix_len[b] <= N; examples of different
 * total length are padded at the tail with negative ids as for mate_plan.  radius as for
 * mate_plan_bucketed (0 = the exact pattern).  mate_plan and mate_plan_bucketed are this call with
 * B equal entries.  All other arguments, ownership and errors as for mate_plan. */
int mate_plan_varlen(const int32_t *row_ids, const int32_t *col_ids, int B, int N, const int32_t *prefix_len,
                     const uint8_t *head_view, int H, int max_row_id, int max_col_id, int radius,
                     void *stream, mate_plan_t **out);

/* Packed batches: examples of different length stored one behind the other, without padding
 * (the paper's inputs are a question or a passage followed by a table of any size, Section 3 and
 * Section 5; the attention of one example never reaches another).  row_ids, col_ids: DEVICE int32
 * [T], example b owning the tokens cu_seqlens[b] .. cu_seqlens[b + 1] - 1; cu_seqlens: HOST int32
 * [B + 1], cu_seqlens[0] = 0, non-decreasing, cu_seqlens[B] = T; prefix_len: HOST int32 [B],
 * 0 <= prefix_len[b] <= length of example b.  Negative ids inside an example still mark padding.
 * With such a plan every tensor of mate_attn_fwd / mate_attn_bwd / mate_attn_bwd_noalloc is
 * [H, T, d] (LSE [H, T]) in place of [B, H, N, d] ([B, H, N]); the plan's N (mate_plan_get)
 * is the longest example.  The exact pattern only; MATE_FLAG_VIEW_ORDER
 * and mate_cell_mean return MATE_ERR_UNSUPPORTED.  Ownership and errors as for mate_plan. */
int mate_plan_packed(const int32_t *row_ids, const int32_t *col_ids, int B, const int32_t *cu_seqlens,
                     const int32_t *prefix_len, const uint8_t *head_view, int H, int max_row_id, int max_col_id,
                     void *stream, mate_plan_t **out);

/* Plan of the head-independent pattern that the paper describes for its closest comparison system
 * (Section 2, related work: attention restricted to the tokens of the same row and of the same
 * column; one pattern for all heads): a table token attends the prefix and every table token that
 * shares its row id OR its column id; prefix tokens attend every non-padding position; padding as
 * for mate_plan.  The pattern is evaluated exactly, in three passes of the ordinary kernels over
 * disjoint key sets -- (prefix and own row), (rest of the own column in front of the own cell),
 * (rest of the column behind it) -- whose outputs are merged through their logsumexps and whose
 * gradients are summed; mate_attn_workspace_bytes accounts for the passes' intermediate results.
 * The returned plan is used with mate_attn_fwd / mate_attn_bwd like any other (all H heads share
 * the pattern); mate_plan_get returns the row / column orders of mate_plan; mate_plan_useful_pairs
 * counts the pattern's pairs.  mate_attn_bwd_noalloc does not take such a plan
 * (MATE_ERR_UNSUPPORTED).  Arguments, ownership and errors as for mate_plan;
 * (max_row_id + 1) * (max_col_id + 1) must not exceed 2^28. */
int mate_plan_sat(const int32_t *row_ids, const int32_t *col_ids, int B, int N, int prefix_len, int H,
                  int max_row_id, int max_col_id, void *stream, mate_plan_t **out);

/* Copies one view's order to HOST arrays (any pointer may be null to skip it):
 *   perm      int32 [B, N]          perm[b][t] = original position of the t-th token of the view
 *   inv_perm  int32 [B, N]          inverse of perm
 *   seg_off   int32 [B, max_id+2]   tokens with id s occupy view positions [seg_off[s], seg_off[s+1]);
 *                                   seg_off[0] = prefix_len (of the example), seg_off[max_id+1] = number of
 *                                   non-padding tokens */
int mate_plan_get(const mate_plan_t *plan, int view, int32_t *perm, int32_t *inv_perm,
                  int32_t *seg_off);

/* Number of unmasked (query, key) pairs per example and head (the O(ng + nb) count of Table 1):
 * HOST int64 [B, H].  Forward work is 4*d flops per pair, backward 10*d. */
int mate_plan_useful_pairs(const mate_plan_t *plan, int64_t *pairs);

/* Waits for `stream` and returns MATE_ERR_TIMEOUT if any kernel that used this plan gave up on a
 * bounded wait since the last call (its outputs are then undefined), MATE_ERR_CUDA if the stream
 * reports an error, else MATE_OK. */
int mate_plan_status(const mate_plan_t *plan, void *stream);

/* Test hook (the paper has no counterpart): launches a one-thread kernel that waits, with the
 * bounded helper the attention kernels use and a limit of a few tries (1.4 microseconds each), on a
 * barrier that nothing arrives on; the wait gives up, the kernel raises the plan's time-out word as
 * the attention kernels would, and returns.  The next mate_plan_status on the plan then reports
 * MATE_ERR_TIMEOUT once, and the plan stays usable.  Lets the time-out path be exercised without
 * making any real kernel wait in vain. */
int mate_debug_expire_wait(const mate_plan_t *plan, void *stream);

int mate_plan_destroy(mate_plan_t *plan);

/* Scratch sizes (bytes) the caller must provide to mate_attn_fwd / mate_attn_bwd for head dim d,
 * element type dtype and implementation `flags`.  Either size may be 0. */
int mate_attn_workspace_bytes(const mate_plan_t *plan, int d, int dtype, unsigned flags,
                              size_t *fwd_bytes, size_t *bwd_bytes);

/* Forward: the head formula of Section 3 for every (b, h, k).
 *   Q, K, V   [B, H, N, d] contiguous, dtype elements, 16-byte aligned
 *   O         [B, H, N, d] same type, fully overwritten, original token order
 *   LSE       float32 [B, H, N]
 *   workspace device scratch of at least fwd_bytes (may be null when that is 0), 256-byte aligned;
 *             contents are undefined afterwards; concurrent calls need separate workspaces AND
 *             separate plans (see mate_plan)
 *   scale     any finite value.  The tensor-core forward needs scale > 0; with MATE_IMPL_AUTO other
 *             values run on the SIMT kernels, with MATE_IMPL_TCGEN05 they give MATE_ERR_UNSUPPORTED
 * d must be a multiple of 8 and at most 128.  Asynchronous on `stream`. */
int mate_attn_fwd(const mate_plan_t *plan, const void *Q, const void *K, const void *V, int d,
                  int dtype, float scale, void *O, float *LSE, void *workspace,
                  size_t workspace_bytes, unsigned flags, void *stream);

/* Backward of mate_attn_fwd (derived from the Section 3 head formula; the paper states no
 * backward): given O and LSE of the forward call and dO, writes dQ, dK, dV (fully overwritten,
 * no accumulation into previous contents).  Same layouts, types and rules as the forward, except that
 * the tensor-core backward takes every finite scale. */
int mate_attn_bwd(const mate_plan_t *plan, const void *Q, const void *K, const void *V,
                  const void *O, const float *LSE, const void *dO, int d, int dtype, float scale,
                  void *dQ, void *dK, void *dV, void *workspace, size_t workspace_bytes,
                  unsigned flags, void *stream);

/* Per-cell mean of token scores (cell-selection stage, Section 4.1: the score of a cell is the
 * mean of the scores of its tokens, S(c) = avg_{t in c} S(t)).  A cell is the set of table tokens
 * (positions behind the prefix, non-negative ids) that share a (row id, column id) pair.
 *   logits   float32 [B, N], one score per token (prefix and padding positions are ignored)
 *   col_ids  the int32 [B, N] column ids the plan was made from
 *   mean     float32 [B, max_row_id + 1, max_col_id + 1], fully overwritten; 0 where no token
 *            carries the pair
 *   count    int32, same shape, tokens per cell; may be null
 * Uses the row view of the plan (a row's tokens are contiguous there).  The sum of a cell runs
 * over its tokens in original order, so the result is the same on every launch.  Asynchronous on
 * `stream`; no workspace. */
int mate_cell_mean(const mate_plan_t *plan, const float *logits, const int32_t *col_ids, float *mean,
                   int32_t *count, void *stream);

/* Backward for callers that cannot allocate device memory.  (The paper has no counterpart: this
 * entry point exists for the library's users, not for the method.)
 *
 * Who needs it: code that runs where cudaMalloc is off limits -- a serving or training loop whose
 * framework has handed all device memory to its own pool, a latency-critical section where the
 * device-wide synchronisation of cudaMalloc/cudaFree is not acceptable, or a plug-in that gets
 * tensors but no allocator.  Such a caller cannot create the workspace mate_attn_bwd asks for.
 *
 * Same arguments, results and rules as mate_attn_bwd with flags = MATE_IMPL_SIMT, minus the
 * workspace: the scratch (one float per (example, head, position)) lives in a 4 MiB array that is
 * part of the library itself, so every GPU that loads libmate holds it until the process exits.
 * The call makes no cudaMalloc, cudaFree or other allocating call.
 *
 *   limit       B * H * N <= 1,048,576; larger problems return MATE_ERR_TOO_LARGE and launch nothing
 *   first call  the first call on each device looks up the array's device address (with that
 *               device current); make that first call outside any stream capture
 *   sharing     all calls on a device use the same array.  Its contents are left over from the
 *               previous call; the kernels overwrite every element they later read, so nothing
 *               depends on them.  Two calls that overlap on the GPU (different streams) race on
 *               the array: serialise them.
 * The plan is an input like the tensors; create it ahead of time with mate_plan. */
int mate_attn_bwd_noalloc(const mate_plan_t *plan, const void *Q, const void *K, const void *V,
                          const void *O, const float *LSE, const void *dO, int d, int dtype,
                          float scale, void *dQ, void *dK, void *dV, void *stream);

/* ------------------------------------------------------------------------------------------------
 * Rotary positions.
 *
 * The first `rot` elements of every head are taken as pairs and each pair (a, b) is turned by the
 * angle t = position * freqs[pair] and scaled by mscale:
 *     forward                 a' = mscale (a cos t - b sin t),   b' = mscale (a sin t + b cos t)
 *     MATE_ROPE_BACKWARD      the transpose (t -> -t): gradients of the inputs from those of the outputs
 * Elements rot .. d-1 are passed on.  Pair i is (i, i + rot / 2), with MATE_ROPE_INTERLEAVED (2 i, 2 i + 1).
 *
 *   tensors    n_tensors (1 or 2: queries and keys, whose numbers of heads may differ) views of B x
 *              heads x N rows of d contiguous elements of type dtype; x is read, y is written, by strides in
 *              elements (batch, head, token) of their own.  y == x with equal strides works in place;
 *              otherwise a y must overlap neither an x nor the other y.  Any alignment that fits the type (16 bytes and sizes that
 *              are multiples of it are faster).
 *   positions  device int32, position of token n of example b at positions[b * position_stride + n] (stride 0: one
 *              row for all examples).  Any value: the angle is formed in 64 bits.  For a table whose positions start
 *              again in every cell the caller says so here.
 *   freqs      device float64 [rot / 2], radians per position, finite (scaled for long contexts as the caller likes)
 * rot is even, 0 <= rot <= d <= 1024.  For packed batches B = 1 and N = T.  Asynchronous on `stream`; no
 * workspace.  Bound by memory: every element is read once and written once. */
typedef struct {
    const void *x;
    void *y;
    int64_t x_stride[3], y_stride[3]; /* batch, head, token */
    int32_t heads;
} mate_rope_tensor_t;

enum { MATE_ROPE_INTERLEAVED = 1, MATE_ROPE_BACKWARD = 2 };

int mate_rope(const mate_rope_tensor_t *tensors, int n_tensors, int B, int N, int d, int dtype, const int32_t *positions,
              int64_t position_stride, const double *freqs, int rot, float mscale, unsigned flags, void *stream);

/* The same with positions of several axes (the place in a text or cell, row and column of a table; time, height and width of a picture):
 * pair i is turned by positions[axis axes[i]] * freqs[i].
 *   positions  device int32, axis a of token n of example b at positions[a * axis_stride + b * position_stride + n]
 *   axes       HOST [rot / 2], the axis of every pair, each below n_axes; sections or any other order (null where rot = 0)
 *   n_axes     1 to 4
 * Everything else as above: with one axis the same results bit for bit. */
int mate_rope_axes(const mate_rope_tensor_t *tensors, int n_tensors, int B, int N, int d, int dtype, const int32_t *positions,
                   int64_t axis_stride, int64_t position_stride, const uint8_t *axes, int n_axes, const double *freqs, int rot,
                   float mscale, unsigned flags, void *stream);

/* ------------------------------------------------------------------------------------------------
 * One new token at a time: a paged cache of keys and values, and the row of the pattern that belongs to
 * the newest token of every sequence.
 *
 * The cache is the caller's memory, described by this struct, which the calls read while they run on the host and do not
 * keep.  A sequence is a row of `table`: its tokens 0 .. lens[s] - 1 stand in the slots of the pages table[s][0],
 * table[s][1], ..., page_size to a page.  Every cached token has its row id and its column id (as given to mate_plan:
 * negative ones, in both arrays, mark padding, which is never attended, whatever its key and value hold); the first prefix[s]
 * tokens are the prefix.  MATE_ID_TEXT as both ids marks a token that belongs to the text wherever it stands (an answer
 * written behind the table): it attends, and is attended by, every token.
 *
 * A page may be shared by several sequences; refs[page] counts them, 0 = free.  lens, table, refs and prefix are device
 * memory that only the calls below (and the caller, between them) change; every call is asynchronous on its stream
 * and can be captured into a graph.  Calls on one cache must be ordered (one stream, or events).
 *
 * d is a multiple of 8 and at most 128; pages * page_size and width * page_size are at most 2^30, kv_heads * page_size 2^20.
 *
 * What the kernels find on the device and cannot do -- a sequence, length or page out of range, a sequence twice
 * in the list of mate_cache_extend or a child twice in that of mate_cache_fork, no room left -- they leave out, and say so in
 * status[0], which mate_cache_status reads.  No such content makes a kernel read or write outside of the arrays. */
#define MATE_ID_TEXT 0x7fffffff
enum { MATE_VIEW_EITHER = 2 }; /* entry of mate_cache_t.head_view: the same row OR the same column (mate_plan_sat) */

typedef struct {
    void *k, *v;                 /* [layers, pages, kv_heads, page_size, d] by the strides below; 16-byte aligned  */
    int32_t *row_ids, *col_ids;  /* [pages, page_size], shared by all layers                                       */
    int32_t *table;              /* [seqs, width]                                                                   */
    int32_t *lens;               /* [seqs]                                                                          */
    int32_t *prefix;             /* [seqs]                                                                          */
    int32_t *refs;               /* [pages]                                                                         */
    int32_t *status;             /* [1], zero at the start                                                          */
    const uint8_t *head_view;    /* HOST [heads], MATE_VIEW_*; query head h uses kv head h / (heads / kv_heads)    */
    int64_t layer_stride, page_stride, head_stride, slot_stride; /* elements, multiples of 16 bytes, of k and v     */
    int32_t layers, pages, page_size, seqs, width, heads, kv_heads, d, dtype, device;
} mate_cache_t;

/* Makes room: for every i, sequence seqs[i] (null: i) grows by counts[i] >= 0 tokens; lens[s] += counts[i], and the
 * pages that it needs beyond those it has are the lowest free ones, dealt out in the order of the list.
 * granted[i] = counts[i]; 0, and the sequence as it was, where there is no room: the table's row is too short,
 * or no page is free (then nobody behind it in the list who needs pages gets any either).  The second and further
 * entries with the same sequence get nothing, whatever became of the first.  seqs, counts, granted: device int32 [n], n <= 4096. */
int mate_cache_extend(const mate_cache_t *cache, const int32_t *seqs, const int32_t *counts, int n, int32_t *granted, void *stream);

/* Writes the last counts[i] (null: N) tokens of sequence seqs[i] (null: i) into one layer of the cache: token j < counts[i]
 * of entry i goes to position lens[s] - counts[i] + j.  To be called behind mate_cache_extend, with what it granted.
 * A sequence stands at most once in the list; this is not looked for, and of two entries with the same one each element that stays may be
 * of either.
 *   K, V       new rows, [B, kv_heads, N, d] by strides (batch, head, token), outside of the cache
 *   Q, Q_out   queries of the new tokens, [B, heads, N, d] by strides, and where they go rotated (Q itself with equal strides, or
 *              apart from Q, K and V); null: none.  All B N tokens are rotated, whatever counts says
 *   row_ids, col_ids   device int32 [B, N], or both null (the ids in the cache stay: further layers)
 *   freqs      as in mate_rope, applied to K (and Q); null: neither is rotated (and Q must be null)
 *   positions  device int32 [B, N]; null: the tokens' positions in their sequences (queries behind counts[i]: 0)
 * A page that several sequences share must not be written: mate_cache_fork sees to that. */
int mate_cache_append(const mate_cache_t *cache, int layer, const void *K, const void *V, const int64_t *k_stride,
                      const int64_t *v_stride, int B, int N, const int32_t *seqs, const int32_t *counts, const int32_t *row_ids,
                      const int32_t *col_ids, const int32_t *positions, const double *freqs, int rot, float mscale, unsigned flags,
                      const void *Q, const int64_t *q_stride, void *Q_out, const int64_t *q_out_stride, void *stream);

/* The same with positions of several axes (see mate_rope_axes): positions is device int32 [n_axes, B, N], and neither it nor freqs may be
 * null. */
int mate_cache_append_axes(const mate_cache_t *cache, int layer, const void *K, const void *V, const int64_t *k_stride,
                           const int64_t *v_stride, int B, int N, const int32_t *seqs, const int32_t *counts, const int32_t *row_ids,
                           const int32_t *col_ids, const int32_t *positions, const uint8_t *axes, int n_axes, const double *freqs,
                           int rot, float mscale, unsigned flags, const void *Q, const int64_t *q_stride, void *Q_out,
                           const int64_t *q_out_stride, void *stream);

/* For every i: sequence children[i], which must be empty, becomes a copy of parents[i].  Full pages are shared; a
 * last page that is filled in part is copied, in all layers, to the lowest free page (in the order of the list).  lens and
 * prefix are copied.  All parents are read as they are before the call.  A child that is not empty, or that
 * stands in the list for the second time, whatever became of the first, is left as it is; one for whose copy no page is free stays empty.
 * parents, children: device int32 [n], n <= 4096.  workspace: device, mate_cache_workspace_bytes. */
int mate_cache_fork(const mate_cache_t *cache, const int32_t *parents, const int32_t *children, int n, void *workspace,
                    size_t workspace_bytes, void *stream);

/* Every sequence of the list (null: 0 .. n - 1) becomes empty: its pages lose a reference, its row of the table becomes -1, its length 0.
 * Sequences that are empty already are no error, so one may stand in the list twice.  prefix stays as it is. */
int mate_cache_free(const mate_cache_t *cache, const int32_t *seqs, int n, void *stream);

/* Moves the pages in use to the front: afterwards pages 0 .. n_live - 1 are in use and all others free.  The pages
 * in use at n_live and above go, in order, to the free ones below; all layers, ids, refs and the table follow.
 * n_live: device int32 [1].  workspace: device, mate_cache_workspace_bytes. */
int mate_cache_compact(const mate_cache_t *cache, int32_t *n_live, void *workspace, size_t workspace_bytes, void *stream);

/* Which entries of a list of sequences (null: 0 .. n - 1) share their first pages, as mate_cache_fork makes them: entry i belongs to the
 * group of entry i - 1 if both have at least m full pages and the first m of them are the same, m = max(1, min_len / page_size rounded
 * up).  (Sequences that share pages but do not follow one another in the list make groups of their own.)  There is one level of groups: where all
 * sequences begin with the same few pages, instructions say, and some of them share a table behind those, a min_len beyond the instructions gives a
 * group to each table; with less they are all one group, which shares the instructions only.  For every entry:
 *   groups[i]          the first entry of its group
 *   groups[n + i]      the group's entries, which follow one another
 *   groups[2 n + i]    tokens that they all share: the largest number of leading full pages that are the same in all of them, times
 *                      page_size; 0 for a group of one
 * The same sequence may stand in the list twice.  seqs: device int32 [n], groups: device int32 [3, n], n <= 4096. */
int mate_cache_groups(const mate_cache_t *cache, const int32_t *seqs, int n, int min_len, int32_t *groups, void *stream);

/* Scratch of mate_cache_fork with n entries, of mate_cache_compact, and of mate_attn_decode with n tokens (any may be null). */
int mate_cache_workspace_bytes(const mate_cache_t *cache, int n, size_t *fork_bytes, size_t *compact_bytes, size_t *decode_bytes);

/* Waits for `stream`, clears status[0] and returns MATE_ERR_TIMEOUT if a kernel gave up on a bounded wait since the last call (the outputs
 * of its call are then undefined), MATE_ERR_NOMEM if pages, or the pages that a row of the table holds, ran out
 * since the last call, MATE_ERR_INVALID_ARG if something was out of range or not as it must be, else MATE_OK. */
int mate_cache_status(const mate_cache_t *cache, void *stream);

/* The forward's row of one token per sequence: for entry i and head h, with s = seqs[i] (null: i),
 *     O = sum_j softmax_j(scale q.k_j) v_j  over the tokens j < lens[s] that are not padding and that
 *     belong to the prefix or the text, or share the new token's row (row heads) / column (column heads) / either of them;
 *     a new token of the text attends them all.
 * The new token's own key and value are attended like every other, if they have been appended.
 *   Q          [B, heads, d] by strides (batch, head), of the cache's type, 16-byte aligned rows
 *   row_ids, col_ids   device int32 [B], the new token's ids (MATE_ID_TEXT: text; negative: padding, O = 0 and LSE = -inf, as
 *              for a sequence without a token that may be attended).  A new token has no place in its sequence: one of the prefix,
 *              which attends everything, is given as MATE_ID_TEXT, not by the ids that mate_plan takes for it
 *   scale      any finite value of up to 2.3e38 in magnitude (scale / ln 2 is what the kernel multiplies by)
 *   max_len    an upper bound of the sequences' lengths that the caller knows (0: what the table can hold); tokens at
 *              and beyond it do not count, and status says so.  It decides how the work is split: short sequences in a wide table take
 *              longer without it (one of 512 tokens in a table for 8192 9.3 us instead of 6.2)
 *   O, LSE     [B, heads, d] of the cache's type, float32 [B, heads]; fully overwritten.  O may be Q, if that is contiguous; otherwise the
 *              three share no memory
 *   workspace  device, 256-byte aligned, mate_cache_workspace_bytes; contents undefined afterwards; calls that overlap need one each
 * Scores, softmax, weights and sums in fp32; with bf16 only the result is rounded.  A NaN or Inf in the key or value of a token
 * reaches the heads that attend the token and no others (an Inf in a bf16 value as an Inf or as a NaN: it is multiplied by a weight in
 * parts, some of which may be 0).  heads <= 1024.  Asynchronous on `stream`. */
int mate_attn_decode(const mate_cache_t *cache, int layer, const void *Q, const int64_t *q_stride, int B, const int32_t *seqs,
                     const int32_t *row_ids, const int32_t *col_ids, float scale, int max_len, void *O, float *LSE, void *workspace,
                     size_t workspace_bytes, void *stream);

/* mate_attn_decode for a batch whose sequences share their first tokens: the same results (but for the order of the sums), with the
 * shared pages of a group read once for all of its sequences, whose query heads are multiplied with them together.
 *   groups     device int32 [3, B] as mate_cache_groups gives it for the same list; any other way of telling who shares what is
 *              taken too: for every entry the first entry of its group, the number of its entries, which follow one another, and the
 *              tokens that they share, the same in all entries of a group, and each sequence at least as long.  An entry whose third
 *              number is 0 or whose second is 1 is in no group.  The shared tokens are read through the first entry's row of the table, so
 *              the others' must be the same there; each entry has a prefix and ids of its own
 *   workspace  device, 256-byte aligned, mate_cache_shared_workspace_bytes; contents undefined afterwards; calls that overlap need one each
 * Groups that do not fit together, or of more tokens than a sequence (or max_len) has, are left out: their entries are taken
 * alone, or attend their own tokens only, and status says so.  So is a group among whose entries another one begins: an entry is in one
 * group at most.  B is at most 4096.
 *   flags      0: where the batch may read no more than 192 MB (bf16) or 1 GB (fp32) one sequence after another -- B max_len kv_heads
 *              keys and values --, that way is taken: the results are mate_attn_decode's; MATE_SHARED_ALWAYS: the shared
 *              tokens are read once all the same
 * Reading them once pays for many sequences in one group or a few.  Beyond those sizes mate_attn_decode is the faster call for batches
 * without groups (bf16 1.6 to 2.5 times, fp32 9 times), with fp32 for groups of fewer than sixteen or so, and where the new tokens are those of
 * cells that attend little of a long table.
 * The batch's work is counted in 32 bits: MATE_ERR_UNSUPPORTED where B kv_heads ceil(heads / kv_heads / (bf16 ? 128 : 64)) (8 + max_len / 32)
 * is 2^30 or more.
 * Where they are read once and the type is bf16, weights enter the product with the values as the sum of two bf16, with 16 bits
 * (mate_attn_decode: with all of their 24).  Sums of either call are in fp32 by the tensor cores, which cut off, towards 0, what is behind the
 * 24 bits: the more tokens, the more (65536 tokens that one block sums up: 1e-4 of a result, a twentieth of half a step of bf16).  All other
 * arguments, limits and errors as for mate_attn_decode. */
int mate_attn_decode_shared(const mate_cache_t *cache, int layer, const void *Q, const int64_t *q_stride, int B, const int32_t *seqs,
                            const int32_t *row_ids, const int32_t *col_ids, const int32_t *groups, float scale, int max_len, unsigned flags,
                            void *O, float *LSE, void *workspace, size_t workspace_bytes, void *stream);

enum { MATE_SHARED_ALWAYS = 1 };

/* Scratch of mate_attn_decode_shared with n tokens. */
int mate_cache_shared_workspace_bytes(const mate_cache_t *cache, int n, size_t *bytes);

#ifdef __cplusplus
}
#endif
#endif /* MATE_H_ */

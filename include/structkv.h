/*
 * structkv.h -- C ABI of the B200 (sm_100a) StructKV prefill-time KV-compression hot path.
 *
 * The library scores the observation-window queries of one layer against all prompt keys,
 * accumulates the per-token in-degree across depth into the Global In-Degree Centrality,
 * produces the per-layer attention statistics that drive Dynamic Pivot Detection, selects
 * token budgets (top-k union window) and compacts K/V, hidden states and position ids.
 *
 * Conventions
 *   - Every pointer marked "device" is a CUDA device pointer owned by the caller; "host"
 *     pointers are ordinary host memory.  The library allocates no device memory: the
 *     caller passes one workspace at context creation (structkv_workspace_bytes()).
 *   - `stream` is a cudaStream_t passed as void* (NULL = the legacy default stream).  All
 *     calls enqueue work on it and return without synchronising, except structkv_pivot and
 *     structkv_poll_device_status, which synchronise that stream, and structkv_pivot_select and
 *     structkv_prefill, which return once the device has found the pivot.
 *   - Every call returns a status; invalid arguments are rejected on the host before any
 *     launch.  There is no CPU fallback: an unsupported shape returns
 *     STRUCTKV_ERR_UNSUPPORTED.  Device-side waits are bounded; if one expires the kernel
 *     records STRUCTKV_ERR_TIMEOUT in a device status word read by
 *     structkv_poll_device_status().
 *   - A context serialises its calls through its workspace: calls on one context must be
 *     issued on one stream (or be ordered by the caller).  Distinct contexts are independent.
 *   - Results are deterministic: the same inputs give the same bits.
 *   - Work on other streams: kernels whose blocks exchange values are launched so that all of their
 *     blocks run at once (cooperative launches): the scorer of short windows (at most 32 score rows
 *     per KV group; lengths in score_res.cu), which takes up to every SM, and the CUDA-core scorer of
 *     up to 4096 keys.  Beside a kernel of another stream that holds SMs they start when that one
 *     has made room; the other kernels take the SMs that are free.  So nothing may hold SMs until
 *     such a call has finished (a resident kernel that waits for its result, say).
 *
 * Index conventions: N = n_keys prompt tokens, w = window (the last w positions are the
 * observation-window queries, row i sits at position t = N-w+i and attends to keys j <= t),
 * H query heads, H_kv KV heads, G = H / H_kv, head h reads KV head h / G, d = head_dim.
 */
#ifndef STRUCTKV_H_
#define STRUCTKV_H_

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  STRUCTKV_OK = 0,
  STRUCTKV_ERR_INVALID_ARG = 1, /* null pointer, size out of range, misaligned pointer or stride */
  STRUCTKV_ERR_UNSUPPORTED = 2, /* shape or dtype outside the supported set */
  STRUCTKV_ERR_WORKSPACE = 3,   /* workspace missing or too small */
  STRUCTKV_ERR_CUDA = 4,        /* a CUDA runtime / driver call failed */
  STRUCTKV_ERR_TIMEOUT = 5      /* a bounded device-side wait expired */
} structkv_status;

typedef enum { STRUCTKV_BF16 = 0, STRUCTKV_FP32 = 1 } structkv_dtype;

/* Flags of structkv_score_layer. */
#define STRUCTKV_FLAG_NO_HEAD_STATS 1u /* skip Eq. 5-6: metrics_out[1..2] are written as NaN */
#define STRUCTKV_FLAG_FORCE_SIMT 2u    /* use the CUDA-core scorer even where the tensor-core one applies */
/* The caller vouches that q_window and k are complete and visible to the device before the call
 * is enqueued: no kernel still in flight on `stream` writes them (they were written before an
 * earlier synchronisation, or on another stream joined through an event).  A scorer may then read
 * them while the kernels enqueued before it are still draining; results are identical.  (The
 * present scorers set up early but read nothing before that: the flag changes nothing.) */
#define STRUCTKV_FLAG_INPUTS_READY 4u

typedef struct {
  int n_q_heads;        /* H, a multiple of n_kv_heads */
  int n_kv_heads;       /* H_kv */
  int head_dim;         /* d: 64 or 128 */
  int window;           /* w: 1..256 */
  int max_seq;          /* largest n_keys any call will pass */
  structkv_dtype dtype; /* storage type of q_window and k */
} structkv_config;

typedef struct structkv_ctx structkv_ctx; /* opaque, host-side */

/* Library version (major*10000 + minor*100 + patch). */
int structkv_version(void);

/* Static, human-readable name of a status code. */
const char* structkv_status_string(structkv_status s);

/* Bytes of device workspace a context for `cfg` needs (0 if cfg is invalid). */
size_t structkv_workspace_bytes(const structkv_config* cfg);

/* Creates a context on the current CUDA device.  `workspace_dev` (device, 256-byte aligned,
 * at least structkv_workspace_bytes(cfg) bytes) stays owned by the caller and must outlive
 * the context.  The call zeroes the device status word on the default stream and synchronises.
 * Errors: INVALID_ARG (null pointers, bad config), UNSUPPORTED (head_dim, window),
 * WORKSPACE (too small / misaligned), CUDA. */
structkv_status structkv_create(structkv_ctx** ctx_out, const structkv_config* cfg,
                                void* workspace_dev, size_t workspace_bytes);

/* Frees the host-side context (never touches the workspace). NULL is allowed. */
void structkv_destroy(structkv_ctx* ctx);

/*
 * One layer of observation-window scoring.
 *
 * Paper: Section 3.2, Eq. 1 (window attention weights a_{t,j} = softmax over keys of
 * q_t.k_j * scale, causal), Eq. 2 (local saliency S_j = (1/w) sum over window rows and over
 * all query heads of a_{t,j}), Eq. 3 / Algorithm 1 line 6 (C <- lambda*C + S), and Section
 * 3.3, Eq. 4 (attention entropy, natural log, mean over heads and window rows), Eq. 5
 * (sparsity: mean over heads of the mass of the floor(0.1 N) largest entries of the
 * window-pooled per-head attention) and Eq. 6 (variance: mean over heads of the population
 * variance over keys of that pooled vector).
 *
 *   q_window      device, [H, w, d] contiguous, dtype of the config; positional encoding
 *                 already applied.  16-byte aligned.
 *   k             device, element (g, j, c) at k + g*k_stride_head + j*k_stride_token + c
 *                 (strides in elements; d contiguous).  Base 16-byte aligned, strides
 *                 multiples of 16 bytes.  Read-only; V is never read.
 *   n_keys        N, window <= N <= max_seq.
 *   scale         logit scale (1/sqrt(d), times any temperature the caller folds in).
 *   lambda        decay of Eq. 3; used only if c_inout != NULL.
 *   s_out         device, [N] fp32, required: S^(l).
 *   c_inout       device, [N] fp32 or NULL: updated in place, C <- lambda*C + S.
 *   head_cols_out device, [H, N] fp32 or NULL: pooled per-head attention
 *                 abar^(h)_j = (1/w) sum_i a_{i,j} (each row sums to 1).
 *   metrics_out   device, [3] fp32, required: {entropy, sparsity, variance}.
 *   flags         STRUCTKV_FLAG_*.
 *
 * Errors: INVALID_ARG, UNSUPPORTED, CUDA.  Asynchronous on `stream`.
 */
structkv_status structkv_score_layer(structkv_ctx* ctx, const void* q_window, const void* k,
                                     long long k_stride_head, long long k_stride_token, int n_keys,
                                     float scale, float lambda, float* s_out, float* c_inout,
                                     float* head_cols_out, float* metrics_out, unsigned flags,
                                     void* stream);

/*
 * One layer of observation-window scoring for a BATCH of prompts of different lengths
 * (Section 4.1, implementation details: batches whose prompts reach their pivots at different
 * layers are served with a padded addressing mask; every prompt is an independent problem with
 * its own length, statistics, pivot and index sets).  The prompts' keys are packed back to back
 * along the token axis; one launch runs both scorer passes over all prompts, each prompt receiving
 * a share of the tasks in proportion to its length.  Per prompt the results equal those of
 * structkv_score_layer on that prompt alone (same equations: Eq. 1, 2, 3, 4, 5, 6).
 *
 *   q_window      device, [batch, H, w, d] contiguous bf16.
 *   k             device, packed keys: element (g, t, c) at k + g*k_stride_head + t*k_stride_token + c,
 *                 prompt b owning tokens cu_seqlens[b] .. cu_seqlens[b+1]-1.
 *   cu_seqlens    HOST, [batch + 1] ints, cu_seqlens[0] = 0, every length in [w, max_seq].
 *   batch         1 .. 32.
 *   s_out         device, [total] fp32 (total = cu_seqlens[batch]): S^(l) of every prompt, packed.
 *   c_inout       device, [total] fp32 or NULL: C <- lambda*C + S, packed.
 *   head_cols_out device, [H, total] fp32 or NULL.
 *   metrics_out   device, [batch, 3] fp32: {entropy, sparsity, variance} of every prompt.
 *   flags         STRUCTKV_FLAG_NO_HEAD_STATS, STRUCTKV_FLAG_INPUTS_READY or 0.
 *   batch_workspace  device, 256-byte aligned, at least
 *                 structkv_batch_workspace_bytes(cfg, batch, total) bytes, caller-owned; calls that
 *                 share it must be ordered by the caller.
 * Served by the tensor-core scorer only (bf16, head_dim 64 or 128): other configurations
 * return UNSUPPORTED.  Errors: INVALID_ARG, UNSUPPORTED, WORKSPACE, CUDA.  Asynchronous on `stream`.
 */
size_t structkv_batch_workspace_bytes(const structkv_config* cfg, int max_batch, long long max_total_tokens);
structkv_status structkv_score_layer_batch(structkv_ctx* ctx, const void* q_window, const void* k,
                                           long long k_stride_head, long long k_stride_token,
                                           const int* cu_seqlens, int batch, float scale, float lambda,
                                           float* s_out, float* c_inout, float* head_cols_out,
                                           float* metrics_out, unsigned flags, void* batch_workspace,
                                           size_t batch_workspace_bytes, void* stream);

/*
 * Eq. 10 / Eq. 13 for a batch of prompts of different lengths: prompt b selects budgets[b] tokens
 * (window included) from its own scores scores[cu_seqlens[b] .. cu_seqlens[b+1]) and writes them,
 * as positions inside that prompt, ascending, to idx_out + b*idx_stride; the remaining entries of
 * the row are -1 (the padded addressing of a batch: padding is never a token).
 *   cu_seqlens, budgets   HOST arrays, [batch + 1] and [batch]; window <= budgets[b] <= length of b.
 *   idx_out               device, [batch, idx_stride] int32, idx_stride >= max budget.
 * Errors: INVALID_ARG, CUDA.  Asynchronous on `stream`.
 */
structkv_status structkv_select_batch(structkv_ctx* ctx, const float* scores, const int* cu_seqlens,
                                      const int* budgets, int batch, int window, int* idx_out,
                                      long long idx_stride, void* stream);

/*
 * Algorithm 1 lines 3-6 (Eq. 1-4) for SEVERAL layers whose window queries and keys are all
 * resident (a prompt whose KV cache already exists, or a prefill that ran ahead of the scoring).
 * Per layer the results are the very bits structkv_score_layer gives with
 * STRUCTKV_FLAG_NO_HEAD_STATS: S^(l), the pooled per-head attention, the layer's entropy; C is
 * carried through all layers (C <- lambda*C + S^(l), l ascending).  What differs is the order of
 * the work: one persistent launch (per 32 layers) runs both scorer passes of all layers, the first
 * pass ahead of the second, so no SM idles while the slowest CTA of a pass finishes; the sums over
 * heads of all layers are taken by one launch at the end.
 *
 *   q_windows, ks  HOST arrays [n_layers] of device pointers, laid out as for structkv_score_layer
 *                 (one stride pair serves all layers); every tensor must be complete and visible
 *                 before the call is enqueued (as with STRUCTKV_FLAG_INPUTS_READY).
 *   scales        HOST array [n_layers].
 *   s_out         device, fp32: S^(l) at s_out + l*s_layer_stride, s_layer_stride >= n_keys.
 *   c_inout       device, [n_keys] fp32 or NULL.
 *   head_cols_out device, fp32, required: layer l's [H, n_keys] slab at
 *                 head_cols_out + l*head_cols_layer_stride (feed it to structkv_head_stats).
 *   metrics_out   device, [n_layers, 3] fp32: [l][0] = entropy, [l][1..2] = NaN.
 *   layers_workspace  device, 256-byte aligned, at least structkv_layers_workspace_bytes(cfg, n_layers)
 *                 bytes, caller-owned.
 * Shapes the tensor-core scorer does not take are scored layer after layer (same results).
 * Errors: INVALID_ARG, WORKSPACE, CUDA.  Asynchronous on `stream`.
 */
size_t structkv_layers_workspace_bytes(const structkv_config* cfg, int max_layers);
structkv_status structkv_score_layers(structkv_ctx* ctx, int n_layers, const void* const* q_windows,
                                      const void* const* ks, long long k_stride_head,
                                      long long k_stride_token, int n_keys, const float* scales, float lambda,
                                      float* s_out, long long s_layer_stride, float* c_inout,
                                      float* head_cols_out, long long head_cols_layer_stride,
                                      float* metrics_out, void* layers_workspace,
                                      size_t layers_workspace_bytes, void* stream);

/*
 * Eq. 5 and Eq. 6 (Section 3.3) for several layers at once, from the pooled per-head attention
 * that structkv_score_layer wrote to head_cols_out.  A caller that scores many layers passes
 * STRUCTKV_FLAG_NO_HEAD_STATS and a distinct head_cols_out slab per layer, then makes ONE call
 * here before the pivot: the per-head selections of all layers run side by side instead of as
 * a chain of short dependent launches after every layer.
 *
 *   head_cols     device, fp32: entry (l, h, j) at head_cols + l*layer_stride + h*col_stride + j,
 *                 each (l, h) vector non-negative and summing to 1 (Eq. 2's per-head pooling).
 *   n_layers      1 .. 128.
 *   n             N, the number of keys of every vector; col_stride >= n.
 *   metrics       device, [n_layers, 3] fp32: entries [l][1] (sparsity) and [l][2] (variance) are
 *                 written, [l][0] (entropy) is left untouched.
 * Results equal those of structkv_score_layer without the flag.  Uses the context's workspace
 * (calls on one context are ordered by the caller).  Errors: INVALID_ARG, CUDA.  Asynchronous.
 */
structkv_status structkv_head_stats(structkv_ctx* ctx, const float* head_cols, long long layer_stride,
                                    long long col_stride, int n_layers, int n, float* metrics,
                                    void* stream);

/*
 * structkv_score_layer without a context and without a caller workspace.  The paper has no
 * counterpart: this entry point exists for integration only.
 *
 * Some hosts of this library cannot allocate device memory at the point where they score a
 * layer: a serving engine that hands all free HBM to its paged KV-cache pool at start-up has
 * nothing left for cudaMalloc to give, and a step that runs inside a latency budget cannot
 * afford the device-wide synchronisation an allocation or a free implies.  For them the
 * scratch the scorer needs (per-segment row statistics, row log-sum-exp, pooled per-head
 * columns, the status word) lives in one array of STRUCTKV_STATIC_SCRATCH_BYTES that is part
 * of the library image: every GPU that loads the library holds those bytes until the process
 * exits, whether this function is called or not.  The call itself performs no cudaMalloc,
 * cudaFree or other allocating routine; inputs and outputs are still the caller's.
 *
 * Limit: the configuration must satisfy
 *     0 < structkv_workspace_bytes(cfg) <= STRUCTKV_STATIC_SCRATCH_BYTES
 * (a Llama-3-8B shape, 32 query heads, window 64, fits up to max_seq = 56064).  A larger
 * configuration is refused with STRUCTKV_ERR_WORKSPACE before anything is launched.
 *
 * Set-up: the first call on each device (with that device current) resolves the device
 * address of the array and looks up the tensor-map encoder; it synchronises nothing but
 * should happen before any stream capture begins.  Later calls on that device only enqueue.
 *
 * Sharing: all calls on one device use the same array, and it keeps whatever the previous
 * call left.  The function re-initialises on `stream` what has to start from zero, so calls
 * issued one after another on one stream are independent; two calls that can overlap on the
 * GPU (different streams without an ordering between them, or different host threads) race
 * on the scratch and give undefined results.  A device-side bounded wait that expires during
 * this call cannot be polled through this entry point; use a context for that.
 *
 * Arguments: `cfg` host pointer; everything else exactly as structkv_score_layer, with
 * cfg->max_seq >= n_keys.  Errors: INVALID_ARG, UNSUPPORTED, WORKSPACE, CUDA.
 */
#define STRUCTKV_STATIC_SCRATCH_BYTES ((8u << 20) + 1449984u)
structkv_status structkv_score_layer_static(const structkv_config* cfg, const void* q_window,
                                            const void* k, long long k_stride_head,
                                            long long k_stride_token, int n_keys, float scale,
                                            float lambda, float* s_out, float* c_inout,
                                            float* head_cols_out, float* metrics_out,
                                            unsigned flags, void* stream);

/*
 * Dynamic Pivot Detection.  Paper: Section 3.3, Eq. 7 (first differences of each metric over
 * layers l = 1..L-1, min-max normalised to [0,1]; a metric with zero range contributes 0),
 * Eq. 8 (T_l = w1*grad(-entropy) + w2*grad(sparsity) + w3*grad(variance)), Eq. 9 with
 * Algorithm 1 line 8: the pivot is the layer l in [1, L-1] with the largest T_l (first maximum
 * wins), capped at l_limit.  NaN sparsity/variance columns (head statistics disabled) count
 * as constant.  Evaluated in double precision on the host.
 *
 *   metrics_dev device, [n_layers, 3] fp32 rows as written by structkv_score_layer.
 *   weights     host, {w1, w2, w3}.
 *   l_limit     cap on the pivot, or -1 for none.
 *   pivot_out   host, receives L* (0 if n_layers < 2).
 *   t_out       host, [n_layers] or NULL: receives T_l (T_0 = 0).
 *
 * Synchronises `stream`.  Errors: INVALID_ARG, CUDA.
 */
structkv_status structkv_pivot(structkv_ctx* ctx, const float* metrics_dev, int n_layers,
                               const float* weights, int l_limit, int* pivot_out, float* t_out,
                               void* stream);

/*
 * Global In-Degree Centrality at a known pivot.  Paper: Eq. 3,
 * c_out[j] = sum_{l=0..pivot} lambda^(pivot-l) * s_hist[l*row_stride + j], evaluated as the
 * recursion of Algorithm 1 line 6.
 *
 *   s_hist device, fp32 rows of length >= n, row_stride in elements;  c_out device, [n] fp32.
 * Errors: INVALID_ARG, CUDA.  Asynchronous on `stream`.
 */
structkv_status structkv_accumulate(structkv_ctx* ctx, const float* s_hist, long long row_stride,
                                    int pivot, int n, float lambda, float* c_out, void* stream);

/*
 * Budgeted token selection.  Paper: Eq. 10 (I_struct = top-k(C) union I_win) and Eq. 13
 * (I_KV = top-k(S^(l)) union I_win), Algorithm 1 lines 10 and 16.  For each of `batch` score
 * vectors: the (budget - window) highest-scoring tokens of the prefix [0, n - window), ties
 * to the lower index, written in ascending position order, followed by the window positions
 * n-window .. n-1.  A NaN counts as larger than any number.
 *
 *   scores  device, fp32, vector b starts at scores + b*row_stride (elements).
 *   idx_out device, [batch, budget] int32.
 *   window <= budget <= n.
 * Errors: INVALID_ARG, CUDA.  Asynchronous on `stream`.
 */
structkv_status structkv_select(structkv_ctx* ctx, const float* scores, long long row_stride,
                                int batch, int n, int budget, int window, int* idx_out,
                                void* stream);

/*
 * structkv_pivot, structkv_accumulate and structkv_select (for the layers and for the centrality) in one
 * call: Eq. 7-9, Eq. 3 at the pivot, Eq. 10 and Eq. 13, in that order, without a host round trip between
 * them: the pivot is found on the device (same arithmetic, double precision), the host waits only for
 * its value.  Results are those of the separate calls.
 *   s_hist    device, [n_layers] rows of n fp32 scores, row_stride elements apart.
 *   metrics_dev, weights, l_limit, pivot_out, t_out   as for structkv_pivot (t_out may be NULL).
 *   c_star    device, [n] fp32: the centrality at the pivot.
 *   i_kv      device, [n_layers, kv_budget] int32;  i_struct  device, [struct_budget] int32.
 * Returns once the pivot is known; the selections may still be running on `stream`.  Cannot be
 * captured into a graph.  Errors: INVALID_ARG, CUDA.
 */
structkv_status structkv_pivot_select(structkv_ctx* ctx, const float* s_hist, long long row_stride, int n_layers,
                                      int n, const float* metrics_dev, const float* weights, int l_limit,
                                      float lambda, int window, int kv_budget, int* i_kv, int struct_budget,
                                      float* c_star, int* i_struct, int* pivot_out, float* t_out, void* stream);

/*
 * The whole of Algorithm 1 over one prompt whose layers are resident: structkv_score_layers (C starting
 * from zero), structkv_head_stats, structkv_pivot_select, structkv_compact_layers for K/V and structkv_compact
 * for hidden states and position ids, enqueued by one call.  Every field means what the argument of
 * that name means there.  kv_srcs, hidden and positions may be NULL (that gather is left out).
 * Returns once the pivot is known; selections and gathers may still be running on `stream`.  Results are
 * those of the separate calls.  Errors: INVALID_ARG, WORKSPACE, CUDA.
 */
typedef struct {
  int n_layers;                             /* 1 .. 128 */
  const void* const* q_windows;             /* host arrays of device pointers, [n_layers] */
  const void* const* ks;
  const float* scales;                      /* host, [n_layers] */
  long long k_stride_head, k_stride_token;
  int n_keys;
  float lambda;
  float* s_out;                             /* [n_layers] rows s_layer_stride apart */
  long long s_layer_stride;
  float* c_out;                             /* [n_keys]: C over all layers */
  float* head_cols;                         /* [n_layers, H, n_keys] */
  long long head_cols_layer_stride;
  float* metrics;                           /* [n_layers, 3] */
  void* layers_workspace;
  size_t layers_workspace_bytes;
  float weights[3];
  int l_limit;
  int window, kv_budget, struct_budget;
  int* i_kv;
  int* i_struct;
  float* c_star;
  const void* const* kv_srcs;               /* as srcs of structkv_compact_layers; index lists are i_kv */
  long long kv_slab_stride_bytes, kv_row_stride_bytes;
  int kv_row_bytes, kv_slabs, kv_rows;
  void* kv_dst;
  long long kv_dst_layer_stride_bytes;
  const void* hidden;                       /* [n_keys] rows of hidden_row_bytes, hidden_row_stride_bytes apart */
  long long hidden_row_stride_bytes;
  int hidden_row_bytes;
  void* hidden_dst;
  const void* positions;                    /* the same for position ids */
  long long position_row_stride_bytes;
  int position_row_bytes;
  void* positions_dst;
} structkv_prefill_args;
structkv_status structkv_prefill(structkv_ctx* ctx, const structkv_prefill_args* args, int* pivot_out, float* t_out,
                                 void* stream);

/*
 * Row gather / compaction.  Paper: Algorithm 1 line 17 (cache K, V at I_KV), line 13 and
 * Eq. 11-12 (hidden states and position ids at I_struct).  For every slab s and output row r:
 * dst[s, r, 0:row_bytes] = src[s*slab_stride_bytes + idx[r]*row_stride_bytes + 0:row_bytes],
 * a byte-exact copy.
 *
 *   src   device; dst device, [n_slabs, n_idx, row_bytes] contiguous; they must not overlap.
 *   idx   device, [n_idx] int32, each in [0, n_rows_src); an out-of-range index copies
 *         nothing for that row and records STRUCTKV_ERR_INVALID_ARG in the device status word.
 *   row_bytes > 0.  When src, dst, both strides and row_bytes are multiples of 16 the copy
 *   uses 16-byte accesses; otherwise 4-byte or single-byte accesses.
 * Errors: INVALID_ARG, CUDA.  Asynchronous on `stream`.
 */
structkv_status structkv_compact(structkv_ctx* ctx, const void* src, long long slab_stride_bytes,
                                 long long row_stride_bytes, int row_bytes, int n_slabs,
                                 int n_rows_src, const int* idx, int n_idx, void* dst,
                                 void* stream);

/*
 * structkv_compact (Algorithm 1 line 17) for several layers in ONE launch: layer l gathers rows of
 * its own source srcs[l] at its own index list idx + l*idx_layer_stride into
 * dst + l*dst_layer_stride_bytes, laid out [n_slabs, n_idx, row_bytes].  With small budgets a
 * gather per layer is a chain of launches of a few microseconds each; one launch removes it.
 *   srcs      HOST array of n_layers device pointers (1 .. 128 layers), all sources sharing
 *             slab_stride_bytes, row_stride_bytes, row_bytes, n_slabs and n_rows_src.
 *   idx       device, int32, n_idx entries per layer, idx_layer_stride >= n_idx.
 * An out-of-range index copies nothing and records STRUCTKV_ERR_INVALID_ARG in the device status
 * word.  Bit exact.  Errors: INVALID_ARG, CUDA.  Asynchronous on `stream`.
 */
structkv_status structkv_compact_layers(structkv_ctx* ctx, const void* const* srcs, int n_layers,
                                        long long slab_stride_bytes, long long row_stride_bytes, int row_bytes,
                                        int n_slabs, int n_rows_src, const int* idx, long long idx_layer_stride,
                                        int n_idx, void* dst, long long dst_layer_stride_bytes, void* stream);

/*
 * Per-KV-group saliency and per-slab gathers: the per-head variant of the cache selection.
 * Paper: Section 3.2, the sentence before Eq. 2 (attention is aggregated over the query heads
 * that share a KV head); Eq. 13 applied per KV head instead of per layer; and Section 4.1, the
 * masked state transition for batches whose sequences carry different index sets.
 *
 * structkv_group_saliency: group_out[g, j] = sum over the G = H / H_kv query heads h of KV group
 * g of head_cols[h, j], where head_cols is the pooled per-head attention written by
 * structkv_score_layer (head_cols_out).  Summing group_out over g gives S^(l).
 *   head_cols device, [H, n] fp32 rows col_stride apart (elements);  group_out device, [H_kv, n].
 *
 * structkv_compact_per_slab: structkv_compact with one index list per slab,
 * dst[s, r, :] = src[s, idx[s*idx_slab_stride + r], :]  (idx_slab_stride >= n_idx, in elements):
 * one list per KV head (lists from structkv_select over group_out), or one list per sequence
 * of a batch.  All other arguments, the out-of-range rule and the byte exactness are those of
 * structkv_compact.
 * Errors: INVALID_ARG, CUDA.  Asynchronous on `stream`.
 */
structkv_status structkv_group_saliency(structkv_ctx* ctx, const float* head_cols, long long col_stride,
                                        int n, float* group_out, void* stream);
structkv_status structkv_compact_per_slab(structkv_ctx* ctx, const void* src, long long slab_stride_bytes,
                                          long long row_stride_bytes, int row_bytes, int n_slabs,
                                          int n_rows_src, const int* idx, long long idx_slab_stride,
                                          int n_idx, void* dst, void* stream);

/*
 * Block-Level Aggregation for block-based KV memory managers.  Paper: Section 4.1,
 * implementation details: the importance of physical block k is the sum of the token scores
 * (the Global In-Degree Centrality) inside it, S_block_k = sum_{t in block_k} C[t]; blocks with
 * the lowest scores are evicted.  Block k covers tokens [k*block_size, min(n, (k+1)*block_size));
 * the last block may be ragged.  Block-granular selection and gathering then go through
 * structkv_select (scores = block scores, budget and window counted in blocks) and
 * structkv_compact (row = one block of one KV head, when n is a multiple of block_size).
 *
 *   scores           device, fp32, vector b starts at scores + b*row_stride (elements).
 *   block_scores_out device, [batch, ceil(n / block_size)] fp32.
 * Sums run in token order in fp32.  Errors: INVALID_ARG, CUDA.  Asynchronous on `stream`.
 */
structkv_status structkv_block_scores(structkv_ctx* ctx, const float* scores, long long row_stride,
                                      int batch, int n, int block_size, float* block_scores_out,
                                      void* stream);

/*
 * Attention-mass recovery of a retained token set.  Paper: Section 4.4, "Fidelity of Hidden
 * States": the share of the original attention weights covered by the retained tokens, per
 * layer.  With the window attention of Eq. 1-2 every row sums to 1, so for layer l the share is
 * sum_{j in idx} S^(l)_j / sum_j S^(l)_j.
 *
 *   scores       device, fp32, one saliency vector per layer, vector b at scores + b*row_stride.
 *   idx          device, [n_idx] int32 retained positions in [0, n); an out-of-range index adds
 *                nothing and records STRUCTKV_ERR_INVALID_ARG in the device status word.
 *   recovery_out device, [batch] fp32.
 * Errors: INVALID_ARG, CUDA.  Asynchronous on `stream`.
 */
structkv_status structkv_mass_recovery(structkv_ctx* ctx, const float* scores, long long row_stride,
                                       int batch, int n, const int* idx, int n_idx, float* recovery_out,
                                       void* stream);

/*
 * Decoding over a compacted cache.  The paper stops where the cache is compacted; these calls go on from there: attention of the
 * tokens that come next (one a sequence, a few, or a tree of drafted ones), the attention weight that cached tokens gather, and
 * eviction by it.  n_q_heads, n_kv_heads, head_dim and dtype are the context's (its window and max_seq do not matter here);
 * G = H / H_kv query heads read a KV head.
 *
 * A cache holds, for every (sequence b, KV head g), lengths[b, g] tokens in slots 0 .. lengths[b, g] - 1, in any order; every
 * token has the position it has in its prompt.  A caller that keeps all layers in one allocation may count a layer as more
 * sequences (append, commit and evict then serve all layers in one launch).
 *   k, v        device, element (b, g, slot, c) at k + b*stride_batch + g*stride_head + slot*stride_token + c (elements; d
 *               contiguous; bases 16-byte aligned, strides multiples of 16 bytes; sequences, heads and slots do not overlap).
 *   positions   device, [batch, H_kv, capacity] int32, not negative.
 *   weights     device, [batch, H_kv, capacity] fp32, or NULL where nothing is accumulated or evicted.
 *   lengths     device, [batch, H_kv] int32.  The calls read it on the device: one that is negative or leaves no room for the new
 *               tokens records STRUCTKV_ERR_INVALID_ARG in the device status word, and nothing of that KV head is read or written.
 * Calls on one cache are ordered by the caller (one stream).  All of them can be captured into graphs.  The context's device has
 * to be current.
 */
typedef struct {
  void* k;
  void* v;
  long long stride_batch, stride_head, stride_token;
  int* positions;
  float* weights;
  int* lengths;
  int batch, capacity;
} structkv_cache;

#define STRUCTKV_MAX_NEW 64 /* new tokens of a sequence that attend in one call */

/* Rows of new tokens: element (b, i, g, c) at k + b*stride_batch + i*stride_token + g*stride_head + c (16-byte aligned, strides
 * multiples of 16 bytes, any order, 0 for a dimension that is broadcast); positions device, [batch, n_new] int32 contiguous. */
typedef struct {
  const void* k;
  const void* v;
  long long stride_batch, stride_token, stride_head;
  const int* positions;
} structkv_new_rows;

/*
 * Writes the rows of n_new (1 .. capacity) new tokens a sequence to slots lengths .. lengths + n_new - 1, their positions, and weight
 * 0.  `lengths` stays: the tokens count once they are committed.  Errors: INVALID_ARG, CUDA.  Asynchronous on `stream`.
 */
structkv_status structkv_append(structkv_ctx* ctx, const structkv_cache* cache, const structkv_new_rows* rows, int n_new,
                                void* stream);

/*
 * Attention of n_new (1 .. 64) new tokens a sequence over its cache and over themselves.  With n = lengths[b, g], new token i (slot n + i)
 * and query head h of KV head g:
 *     x[j] = scale q.k[j], then softcap tanh(x / softcap) if softcap > 0, then - slopes[h] (position[n + i] - position[j])
 *     lse = log sum_j exp(x[j]),  out = sum_j exp(x[j] - lse) v[j]
 * over the slots j < n and those new tokens n + u that tree[b, i] names (bit u); without a tree u <= i.  A tree's bits from
 * n_new on are ignored; a token usually names its ancestors and itself.  A token that sees nothing gets out 0 and lse minus infinity.
 *   q           device, element (b, i, h, c) at q + b*q_stride_batch + i*q_stride_token + h*q_stride_head + c, dtype of the config,
 *               positional encoding already applied; 16-byte aligned, strides multiples of 16 bytes.
 *   slopes      device, [H] fp32 or NULL.       tree    device, [batch, n_new] 64-bit words or NULL.
 *   rows        host, the new tokens' rows, which are appended first; NULL: they are in the cache already.
 *   out         device, [batch, n_new, H, d] contiguous, dtype of the config, 16-byte aligned.
 *   lse         device, [batch, n_new, H] fp32 or NULL.
 *   accumulate  not 0: weights[j] = decay weights[j] + the sum over the G heads of exp(x[j] - lse), for all lengths + 1 slots;
 *               for n_new = 1 only (a tree's tokens count once they are accepted: structkv_weigh).
 *   workspace   device, 256-byte aligned, at least structkv_attend_workspace_bytes() bytes (0 for arguments that are not valid),
 *               caller-owned; calls that share it are ordered by the caller.
 * Values are accumulated in fp32; for bf16 storage the probabilities are rounded to bf16 for their product with V.  New tokens
 * that a row does not see do not reach it, whatever they hold; V that is not finite makes its column so in every row that sees the
 * token, if the token's score is a number, however small its probability.  Tiles of 64 keys are counted in 31 bits, for every four rows of a KV
 * head (new token, head of the group) and with nine more for each; a call whose cache could hold more is refused, as structkv_weigh
 * is.  Errors: INVALID_ARG, UNSUPPORTED (accumulate with several tokens), WORKSPACE, CUDA.  Asynchronous on `stream`.
 */
typedef struct {
  const void* q;
  long long q_stride_batch, q_stride_token, q_stride_head;
  int n_new;
  float scale, softcap;
  const float* slopes;
  const unsigned long long* tree;
  const structkv_new_rows* rows;
  void* out;
  float* lse;
  int accumulate;
  float decay;
  void* workspace;
  size_t workspace_bytes;
} structkv_attend_args;
size_t structkv_attend_workspace_bytes(const structkv_config* cfg, int batch, int n_new, int capacity);
structkv_status structkv_attend(structkv_ctx* ctx, const structkv_cache* cache, const structkv_attend_args* args, void* stream);

/*
 * Adds the attention weight that accepted new tokens gave: weights[j] = decay weights[j] + the sum of exp(x - lse) over the new
 * tokens i whose bit is set in accepted[b] and the G heads, for all lengths + n_new slots.  Called between structkv_attend and
 * structkv_commit, with the q, scale, softcap, slopes, tree and n_new of the former and the lse that it wrote (rows, out,
 * accumulate and workspace are not looked at).
 *   accepted    device, [batch] 64-bit words; bits from n_new on are ignored.
 * decay is applied once a call, however many tokens were accepted: three tokens one by one decay a weight three times, three at once
 * a single time.  A caller who wants it by the token passes its power.
 * Sums are in fp32; they are added to a weight, which rounds it, once for every 8 (fp32 storage) or 64 rows.  A probability is as exact as
 * lse in fp32 lets it be: off by 2^-23 |lse|, relative.
 * Errors: INVALID_ARG, CUDA.  Asynchronous on `stream`.
 */
structkv_status structkv_weigh(structkv_ctx* ctx, const structkv_cache* cache, const structkv_attend_args* args,
                               const unsigned long long* accepted, void* stream);

/*
 * New tokens become cached ones: of the n_new tokens in the slots behind lengths, sequence b keeps path[b, 0 .. counts[b] - 1]
 * (ascending numbers of new tokens), moved together behind the old ones with their positions and weights, and its lengths grow by
 * counts[b].  Without a path it keeps the first counts[b], without counts all n_new (1 .. capacity; with a path 1 .. 64).
 *   counts      device, [batch] int32 or NULL.     path    device, [batch, n_new] int32 or NULL (then with counts).
 * A count outside 0 .. n_new or a path that does not ascend within it records STRUCTKV_ERR_INVALID_ARG in the device status
 * word and leaves that sequence as it is.  Errors: INVALID_ARG, CUDA.  Asynchronous on `stream`.
 */
structkv_status structkv_commit(structkv_ctx* ctx, const structkv_cache* cache, int n_new, const int* counts, const int* path,
                                void* stream);

/*
 * Eviction by accumulated attention weight: every KV head of more than `budget` (at least 1) tokens keeps `budget` of them: first
 * those whose position is above its newest one less `recent` (recent >= 0; of more than `budget` such ones the lower slots), then
 * by weight, larger first (a NaN counts as larger than any number), ties to the lower slot.  Kept tokens in slots from `budget` on
 * move, in order, into the slots below it whose tokens go, the lowest first; other slots stay as they are, so that slots are not
 * in the order of positions.  lengths becomes `budget`.
 * Errors: INVALID_ARG, CUDA.  Asynchronous on `stream`.
 */
structkv_status structkv_evict(structkv_ctx* ctx, const structkv_cache* cache, int budget, int recent, void* stream);

/*
 * Rotary positions.  Paper: Section 3.4, Eq. 12 (K' = f_RoPE(K, P'): kept tokens keep their positions).  A head's first `dim` elements form
 * dim / 2 pairs (a, b); at position p pair c is turned by p * step[c], counted in 2^-64 of a turn, modulo one turn, and multiplied:
 *     a' = amplitude (a cos - b sin),  b' = amplitude (b cos + a sin);
 * the elements from `dim` on stay.  Angles are exact products of 64 bits: far positions lose nothing.  structkv_rope_init fills the block
 * in, on the host and in extended precision, for frequencies f[c] = base^(-2c / dim) (radians a position), which scaling changes:
 *   PLAIN   f.
 *   LINEAR  f / factor.
 *   BASE    base is base * factor^(dim / (dim - 2)); dim above 2.
 *   BANDS   with turns = original f / 2 pi over the original context and part = (turns - slow) / (fast - slow) within [0, 1]:
 *           part f + (1 - part) f / factor.
 *   RAMP    the same form, part by the pair's number: with pair(t) = dim ln(original / (2 pi t)) / (2 ln base), lo = max(0, floor(pair(fast)))
 *           and hi = min(dim - 1, ceil(pair(slow))): part = 1 - (c - lo) / max(hi - lo, 0.001) within [0, 1]; amplitude = 0.1 ln(factor) + 1
 *           where factor is above 1.
 *   dim         even, 2 .. STRUCTKV_ROPE_MAX_DIM;  interleaved  not 0: pairs are (2c, 2c + 1), else (c, c + dim / 2);  base above 1.
 *   factor, original, slow, fast   what the scaling uses: positive and finite; slow below fast (the others are not looked at).
 * Errors: INVALID_ARG.
 */
#define STRUCTKV_ROPE_MAX_DIM 128
typedef enum {
  STRUCTKV_ROPE_PLAIN = 0,
  STRUCTKV_ROPE_LINEAR = 1,
  STRUCTKV_ROPE_BASE = 2,
  STRUCTKV_ROPE_BANDS = 3,
  STRUCTKV_ROPE_RAMP = 4
} structkv_rope_scaling;
typedef struct {
  int dim, interleaved;
  double amplitude;
  unsigned long long step[STRUCTKV_ROPE_MAX_DIM / 2];
} structkv_rope;
structkv_status structkv_rope_init(structkv_rope* rope, int dim, int interleaved, double base, int scaling, double factor,
                                   double original, double slow, double fast);

/*
 * Rotates heads of the context's dtype and head_dim (any number of heads; rope->dim at most head_dim).
 *   x, out      device, element (b, i, h, c) at x + b*x_stride_batch + i*x_stride_token + h*x_stride_head + c, out alike (bases 16-byte
 *               aligned, strides multiples of 16 bytes; x's may be 0).  out is x with the same strides (in place), or they do
 *               not overlap.
 *   positions   device, token (b, i) at positions + b*positions_stride + i (0: the same for every b).  Any 32-bit number.
 *   inverse     not 0: turned the other way, amplitude as it is: the transpose of the rotation, so the gradient of x from that of out.
 * Computed in fp32 and rounded once.  batch * tokens below 2^31; none of the sizes is negative, and nothing is done where one is 0.
 * Errors: INVALID_ARG, CUDA.  Asynchronous on `stream`.
 */
typedef struct {
  const void* x;
  long long x_stride_batch, x_stride_token, x_stride_head;
  void* out;
  long long out_stride_batch, out_stride_token, out_stride_head;
  const int* positions;
  long long positions_stride;
  int batch, tokens, heads;
  int inverse;
} structkv_rotate_args;
structkv_status structkv_rotate(structkv_ctx* ctx, const structkv_rope* rope, const structkv_rotate_args* args, void* stream);

/*
 * A paged cache in 8 bits.  A page holds page_size tokens for every KV head, K and V as e4m3 codes; STRUCTKV_SCALE_BLOCK neighbouring
 * slots of a head share a scale, a power of two 2^e held as the byte e + 127: a value is code * 2^e.  Sequence b's slot j is slot
 * j mod page_size of page table[b, j / page_size].
 *   k, v        device, element (page, g, slot, c) at k + page*stride_page + g*stride_head + slot*stride_token + c (bytes; d contiguous;
 *               bases 16-byte aligned, strides multiples of 16, not negative, stride_token below 2^22 and stride_page below 2^32; pages, heads and slots
 *               do not overlap).
 *   k_scales, v_scales   device, [pages, H_kv, page_size / STRUCTKV_SCALE_BLOCK] bytes; what the calls write lies in 87 .. 247.
 *   table       device, row b at table + b*table_stride, table_columns entries.  An entry that is looked at and is no page records
 *               STRUCTKV_ERR_INVALID_ARG in the device status word; its slots are neither written nor seen.
 *   lengths     device, [batch] int32, the tokens of a sequence.  One that is negative or leaves no room for the new tokens records
 *               STRUCTKV_ERR_INVALID_ARG in the device status word, and nothing of that sequence is read or written but its rows of
 *               an attention's output, which become those of a row that sees nothing.
 *   page_size   16, 32, 64, 128 or 256.
 * Full pages may be in several sequences' tables.  Calls on one cache are ordered by the caller (one stream).  All of them can be captured into
 * graphs.  The context's device has to be current.
 */
#define STRUCTKV_SCALE_BLOCK 16
typedef struct {
  void *k, *v;
  unsigned char *k_scales, *v_scales;
  long long stride_page, stride_head, stride_token;
  const int* table;
  long long table_stride;
  int table_columns;
  int* lengths;
  int batch, pages, page_size;
} structkv_pages;

/*
 * Quantises the rows of new tokens into slots lengths[b] .. and up; K is rotated on the way.  `lengths` stays: the tokens count once the
 * caller adds them.  Row r of sequence b comes from source token t = index[b, r], or r without an index, and has its position.
 * A block of STRUCTKV_SCALE_BLOCK slots gets the smallest e, at least -40, with which its largest finite magnitude stays within 448 * 2^e;
 * where it holds tokens already, the larger of that and the e that it has, to which their codes are rounded (to nearest, ties to even)
 * anew.  All rows that are written count, whether they stay or not: where a caller drops some of them (its lengths grow by fewer), the e that
 * they raised and the older codes that were rounded to it remain.  What is not finite in fp32 becomes NaN.  Scales and codes are those of the
 * rotated values rounded to fp32 (which are worked out in fp32, and in fp64 where that is too close to a border between two codes or two
 * scales, or to fp32's end, to tell); a code of zero has either sign.
 *   k, v        device, element (b, t, g, c) at k + b*stride_batch + t*stride_token + g*stride_head + c, dtype of the context
 *               (bases 16-byte aligned, strides multiples of 16 bytes, any order, 0 for a dimension that is broadcast).
 *   tokens      source tokens of a sequence.
 *   n_new       1 .. table_columns * page_size rows of a sequence at most; without an index n_new <= tokens.
 *   counts      device, [batch] int32 or NULL: rows of each sequence, 0 .. n_new (else as a length without room).  NULL: n_new.
 *   index       device, row b at index + b*index_stride, n_new entries, or NULL.  One that is no source token records
 *               STRUCTKV_ERR_INVALID_ARG in the device status word; its row becomes 0.
 *   rope        host, or NULL: K is not rotated.
 *   positions   device, source token t of sequence b at positions + b*positions_stride + t; NULL without rope.
 *   q, q_out    device or NULL: n_heads query heads of the new tokens, rotated in the same launch (without an index, with a rope; all n_new
 *               of them, whatever counts says): element (b, i, h, c) at q + b*q_stride_batch + i*q_stride_token + h*q_stride_head + c,
 *               q_out [batch, n_new, H, d] contiguous; q_out is q where that is contiguous, or they do not overlap.
 * Errors: INVALID_ARG, CUDA.  Asynchronous on `stream`.
 */
typedef struct {
  const void *k, *v;
  long long stride_batch, stride_token, stride_head;
  int tokens, n_new;
  const int* counts;
  const int* index;
  long long index_stride;
  const structkv_rope* rope;
  const int* positions;
  long long positions_stride;
  const void* q;
  long long q_stride_batch, q_stride_token, q_stride_head;
  void* q_out;
} structkv_append_pages_args;
structkv_status structkv_append_pages(structkv_ctx* ctx, const structkv_pages* pages, const structkv_append_pages_args* args, void* stream);

/*
 * Attention of n_new (1 .. 64) new tokens a sequence, whose rows are in the slots behind lengths (structkv_append_pages), over the pages.
 * With n = lengths[b], new token i < counts[b] and query head h of KV head g, over the slots j <= n + i:
 *     x[j] = scale q.k[j], then softcap tanh(x / softcap) if softcap > 0;  lse = log sum_j exp(x[j]),  out = sum_j exp(x[j] - lse) v[j]
 * A token i >= counts[b], and one that sees nothing, gets out 0 and lse minus infinity.
 *   q           device, element (b, i, h, c) at q + b*q_stride_batch + i*q_stride_token + h*q_stride_head + c, dtype of the context, rotated
 *               already; 16-byte aligned, strides multiples of 16 bytes.
 *   counts      device, [batch] int32 or NULL: n_new.  Outside 0 .. n_new: as a length without room.
 *   out         device, [batch, n_new, H, d] contiguous, dtype of the context, 16-byte aligned.
 *   lse         device, [batch, n_new, H] fp32 or NULL.
 *   workspace   device, 256-byte aligned, at least structkv_attend_pages_workspace_bytes() bytes (0 for arguments that are not
 *               valid; slots: table_columns * page_size), caller-owned; calls that share it are ordered by the caller.
 * Codes are exact operands; sums are in fp32; probabilities keep 11 bits for their product with V (22 for fp32 storage) where probability
 * times V's scale is at least 2^-20 (2^-9) of the largest such product of its row, and below that are off by 2^-31 of it; a key whose product is below
 * 2^-118 of the largest counts neither in out nor in lse (V's scales would have to be as far apart for it to matter).  A NaN in V makes its
 * column NaN in every row that sees the token, however small its probability; rows that do not see a token are not
 * reached by it.  Errors: INVALID_ARG, WORKSPACE, CUDA.  Asynchronous on `stream`.
 */
typedef struct {
  const void* q;
  long long q_stride_batch, q_stride_token, q_stride_head;
  int n_new;
  const int* counts;
  float scale, softcap;
  void* out;
  float* lse;
  void* workspace;
  size_t workspace_bytes;
} structkv_attend_pages_args;
size_t structkv_attend_pages_workspace_bytes(const structkv_config* cfg, int batch, int n_new, long long slots);
structkv_status structkv_attend_pages(structkv_ctx* ctx, const structkv_pages* pages, const structkv_attend_pages_args* args, void* stream);

/*
 * Self-test of the error path every device-side wait shares (the paper has no counterpart; the
 * conventions at the top of this header define it): launches one thread that waits, with the
 * scorer's bounded-wait helper and a bound of `limit_cycles` SM clock cycles (1 .. 4e9), on a
 * barrier nothing arrives on.  No copy or tensor-core work is in flight; when the bound runs out
 * the kernel records STRUCTKV_ERR_TIMEOUT in the device status word and returns, so the next
 * structkv_poll_device_status() reports TIMEOUT once and OK afterwards.
 * Errors: INVALID_ARG, CUDA.  Asynchronous on `stream`.
 */
structkv_status structkv_selftest_wait_expiry(structkv_ctx* ctx, unsigned long long limit_cycles,
                                              void* stream);

/*
 * Self-test of the scorer of one short layer, whose CTAs draw tasks: with fewer CTAs than tasks, as on a GPU that
 * other work fills, a CTA runs several.  Bounds the CTAs of the launches to come (0: one per task, as at first).
 * Results do not depend on it.  Errors: INVALID_ARG.
 */
structkv_status structkv_selftest_ctas(structkv_ctx* ctx, int ctas);

/* Reads and clears the device status word (bounded-wait expiry, bad gather index).
 * Synchronises `stream`.  Returns STRUCTKV_OK if nothing was recorded. */
structkv_status structkv_poll_device_status(structkv_ctx* ctx, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* STRUCTKV_H_ */

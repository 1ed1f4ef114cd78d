/*
 * relaxkv.h - C ABI of the RelaxKV selective cache-repair hot path for NVIDIA B200 (sm_100a).
 *
 * The library implements, as hand-written CUDA kernels, the two halves of the repair path of
 * "RelaxKV: Recomputation Guided by the Query with Sparse Context Attention":
 *   (a) query-guided anchor selection   - relaxkv_score_select, relaxkv_build_active_sets
 *   (b) sparse-context repair attention - relaxkv_sparse_ctx_attention, relaxkv_scatter_kv
 *
 * General conventions (they hold for every entry point unless it says otherwise)
 * -----------------------------------------------------------------------------
 * Pointers.   A name starting with h_ is a HOST pointer, read during the call only.  Every other
 *             pointer is a DEVICE pointer of the current CUDA device.  All buffers are owned by the
 *             caller; the library allocates nothing, frees nothing and keeps no pointer after the
 *             call returns.  Scratch comes from the caller's `workspace` (device memory, 256-byte
 *             aligned, at least relaxkv_workspace_bytes() bytes).
 * Types.      K, V, Q and attention outputs are bf16 (2 bytes); scores are fp32; every index is
 *             int32.  head_dim is contiguous in memory everywhere.  bf16 base pointers must be
 *             16-byte aligned and the cache strides multiples of 8 elements.
 * Batching.   A call covers n_req independent requests (a ragged batch).  Per-request arrays are
 *             packed back to back; "cu" arrays hold the n_req+1 exclusive prefix offsets.
 * Positions.  Context positions are request-local token indices 0..T_c-1.  Every index list is
 *             ascending and free of duplicates.  Active targets are stored as ranks into the
 *             sorted union U, so a target's causal limit is its own rank.
 * Heads.      Query head h reads KV head h / (n_q_heads / n_kv_heads).
 * Asynchrony. All work is enqueued on `stream`; no call synchronises except
 *             relaxkv_read_device_status.  Data-dependent set sizes stay on the device; the host
 *             passes upper bounds.
 * Errors.     Host-checkable violations (NULL, bad shape, misalignment, workspace too small) return
 *             a status before any launch.  Launch failures return RELAXKV_ERR_CUDA.  Problems only
 *             the device can see (an index out of range, a count above its host bound, a bounded
 *             wait that expired) are recorded in a device status word - the kernel skips the
 *             offending work and returns normally - and are read with relaxkv_read_device_status.
 *             The first problem recorded stays until it is read.  After an expired wait (RELAXKV_ERR_TIMEOUT)
 *             the tensor-core kernels of later calls on that device return at once without writing their
 *             outputs, until the status word has been read (and thereby cleared): a caller that sees garbage
 *             should read the status word first.
 * Graphs.     Every call only enqueues kernels, memsets and copies on `stream`, so calls can be recorded into a CUDA
 *             graph; make the first call of each kind on a device outside the capture (it looks up device
 *             addresses and opts kernels into large shared memory).  The host bounds and the choice of kernel form
 *             are frozen into the graph.
 * Threads.    Calls may be made from several host threads; the per-device values the library looks up once
 *             (device addresses, attribute opt-ins) are published with atomics.  The status word is per device,
 *             not per thread or stream.
 * Precision.  bf16 inputs, fp32 accumulation and softmax, probabilities rounded to bf16 before the
 *             P*V product, bf16 outputs.
 */
#ifndef RELAXKV_H_
#define RELAXKV_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  RELAXKV_OK = 0,
  RELAXKV_ERR_INVALID_ARG = 1,
  RELAXKV_ERR_UNSUPPORTED_SHAPE = 2,
  RELAXKV_ERR_WORKSPACE_TOO_SMALL = 3,
  RELAXKV_ERR_CUDA = 4,
  RELAXKV_ERR_BAD_INDEX = 5,
  RELAXKV_ERR_TIMEOUT = 6
} relaxkv_status;

/* A CUDA stream handle (cudaStream_t) passed as an opaque pointer; NULL is the default stream. */
typedef void* relaxkv_stream;

/* Optional per-call overrides of choices the library otherwise makes from the size of the launch.  Every field:
 * 0 = automatic.  Meant for tests and measurements; results agree within the tolerances either way. */
typedef struct {
  int32_t attention_ctx_splits;  /* > 0: the attention calls split every query tile's context over this many thread   */
                                 /* blocks (up to 32, and as far as the workspace's 2048 row-splits allow) and merge   */
                                 /* the partial results by their log-sum-exp; automatic = only when the call has too   */
                                 /* few query tiles to fill the GPU (a query prefill, a decode step, few targets), and */
                                 /* then, for targets along the context, the longest of them alone                     */
  int32_t attention_persistent;  /* the repair / list attention calls have a persistent form (one thread block per SM  */
                                 /* walks the call's query tiles, longest context first).  0: the library takes it     */
                                 /* for one-split calls over gathered contexts of at most 128 key tiles; 1: for every  */
                                 /* one-split call over a gathered context; 2: never.  Same results bit for bit.       */
  int32_t attention_grid_blocks; /* > 0: number of thread blocks of the persistent form (default: one per SM); the     */
                                 /* automatic choice then cuts no call at its longest targets                          */
} relaxkv_tuning;

/* Shapes shared by all calls. */
typedef struct {
  int32_t n_req;              /* 1 <= B <= 64 requests in the batch                             */
  int32_t n_q_heads;          /* H                                                              */
  int32_t n_kv_heads;         /* H_kv, divides H; the group size G = H / H_kv must be <= 16     */
  int32_t head_dim;           /* D, 64 or 128                                                   */
  const int32_t* h_ctx_len;   /* host [B]: context tokens T_c of each request                   */
  const int32_t* h_q_len;     /* host [B]: query-suffix tokens Q of each request; read by       */
                              /* relaxkv_score_select and relaxkv_workspace_bytes only          */
  float softmax_scale;        /* multiplies q.k before the softmax (usually 1/sqrt(D))          */
  const relaxkv_tuning* h_tuning;  /* host, optional: NULL = every choice automatic             */
} relaxkv_shape;

/* One layer's KV cache.  Element (request b, token i, kv head g, dim d) of K lives at
 * k + (h_req_token_offset[b] + i) * token_stride + g * head_stride + d  (in elements), same for V.
 * This covers [tokens, H_kv, D] and [H_kv, tokens, D] storage. */
typedef struct {
  void* k;
  void* v;
  int64_t token_stride;
  int64_t head_stride;
  const int64_t* h_req_token_offset;   /* host [B]: first token row of each request */
} relaxkv_cache_view;

/* How the recomputation context of a target at position p is built. */
typedef enum {
  RELAXKV_CTX_UNION = 0,        /* C_l(p) = U intersect {j <= p}  (the method)                    */
  RELAXKV_CTX_FULL_PREFIX = 1   /* every position j <= p (the paper's Full-Prefix Control)        */
} relaxkv_ctx_mode;

const char* relaxkv_status_string(int32_t status);

/* Anchors per layer, k = max(1, round(r * T_c)) clamped to T_c; round is to nearest with halves to
 * even on the fp64 product.  (Appendix A.1, anchor-count equation; Section 3.2.)  Host only. */
int32_t relaxkv_anchor_count(int32_t ctx_len, double ratio);

/* Bytes of device scratch that suffice for any call below with these shapes.  h_k may be NULL.
 * Returns 0 for an invalid shape.  Host only. */
size_t relaxkv_workspace_bytes(const relaxkv_shape* shape, int32_t n_layers, const int32_t* h_k);

/*
 * Query-attention scoring and per-layer top-k anchors (Section 3.2, score equation and TopK;
 * Algorithm 1, steps 1-5; Appendix A.1).
 *
 * For each layer l < n_layers and request b, with Q = the request's query-suffix rows:
 *   s[h,t,i]  = softmax_scale * <q[t,h,:], K[i, h/G, :]>                i over all T_c cached tokens
 *   A[h,t,i]  = exp(s[h,t,i] - lse[h,t])     lse = log sum_i exp(s[h,t,i])  unless supplied
 *   raw[i]    = (1/(H*Q)) * sum_h sum_t A[h,t,i]
 *   norm[i]   = (raw[i] - min raw) / (max raw - min raw)                (all zeros if max == min)
 *   anchors   = positions of the k largest raw[i]; equal scores go to the lower position;
 *               written in ascending order.  (MinMax is monotone, so selecting on raw selects the
 *               same set as selecting on norm.)
 *
 * q_layers         host array [n_layers] of device bf16 [sum_b Q_b, H, D] (requests packed).
 * cache_layers     host array [n_layers]; only .k is read.
 * row_lse_layers   NULL, or host array [n_layers] of device fp32 [H, sum_b Q_b] (entry (h, row));
 *                  when given for a layer, its rows' log-normalisers are taken from it (e.g. from the
 *                  query's own forward pass, whose softmax also spans the query tokens) and the
 *                  statistics pass is skipped.  An entry may itself be NULL.
 * h_k              host [B]: anchors per layer for each request, 1 <= k_b <= T_c.
 * raw_scores_out   device fp32 [n_layers, sum_b T_c].
 * norm_scores_out  NULL or device fp32 [n_layers, sum_b T_c].
 * anchors_out      device int32 [n_layers, sum_b k_b]; request-local positions.  NULL: scoring only (no
 *                  selection, norm_scores_out is not written) - for callers that first combine the scores
 *                  of several head shards (mean over shards of equal size) and then call relaxkv_select_topk.
 * Results are deterministic: reductions run in a fixed order (no floating-point atomics).
 */
relaxkv_status relaxkv_score_select(
    const relaxkv_shape* shape, int32_t n_layers,
    const void* const* q_layers, const relaxkv_cache_view* cache_layers,
    const float* const* row_lse_layers, const int32_t* h_k,
    float* raw_scores_out, float* norm_scores_out, int32_t* anchors_out,
    void* workspace, size_t workspace_bytes, relaxkv_stream stream);

/*
 * The selection step of relaxkv_score_select on its own (Appendix A.1, TopK; Section 3.2, MinMax):
 * top-k anchors (and optionally the MinMax-normalised scores) of given raw scores.  Same layouts,
 * tie rule and output order as above.  Exists so the step can be checked and timed by itself.
 */
relaxkv_status relaxkv_select_topk(
    const relaxkv_shape* shape, int32_t n_layers, const int32_t* h_k, const float* raw_scores,
    float* norm_scores_out, int32_t* anchors_out, relaxkv_stream stream);

/*
 * Repair schedule from the per-layer anchors (Section 3.2, definitions of h_i, U, R_l;
 * Algorithm 1, steps 6-12; Appendix A.2: U is kept sorted and its members are numbered once per request).
 *
 *   h_i  = max{ l : i in S_l }  (-1 if i is in no S_l);   U = { i : h_i >= 0 } ascending;
 *   u_rank[i] = index of i in U (or -1);   R_l = { c : h_{U[c]} >= l } as ascending ranks c.
 *
 * anchors            device int32 [n_layers, sum_b k_b] as written by relaxkv_score_select.
 * highest_layer_out  device int32 [sum_b T_c].
 * u_pos_out          device int32, capacity sum_b min(T_c, n_layers*k_b): U of each request, packed.
 * u_cu_out           device int32 [B+1].
 * u_rank_out         device int32 [sum_b T_c].
 * r_rank_out         device int32, capacity n_layers * (capacity of u_pos_out): for layer l and
 *                    request b the ranks of R_{l,b}, packed in (l, b) order.
 * r_cu_out           device int32 [n_layers*B + 1]: offset of segment (l, b) at index l*B + b.
 * h_counts_pinned    NULL or pinned host int32 [B + n_layers*B]: |U_b| then |R_{l,b}|; valid once
 *                    the stream has been synchronised.
 */
relaxkv_status relaxkv_build_active_sets(
    const relaxkv_shape* shape, int32_t n_layers, const int32_t* h_k, const int32_t* anchors,
    int32_t* highest_layer_out, int32_t* u_pos_out, int32_t* u_cu_out, int32_t* u_rank_out,
    int32_t* r_rank_out, int32_t* r_cu_out, int32_t* h_counts_pinned,
    void* workspace, size_t workspace_bytes, relaxkv_stream stream);

/*
 * relaxkv_build_active_sets for callers that have no scratch memory to give.  (The paper has no
 * counterpart; this is a packaging variant of the call above and computes the same outputs.)
 *
 * Who needs it: code that runs inside a host which owns all device memory and lends an extension
 * only its input and output tensors - an inference-server plug-in, an embedded runtime whose
 * memory pool is sealed after start-up.  Such a caller can neither allocate a workspace nor ask
 * its host for one.  Here the scratch (the B + n_layers*B set counts) lives in a fixed array inside
 * the library image; the call allocates nothing and takes no workspace.  Inputs and outputs are
 * still the caller's buffers, exactly as above.
 *
 * Limits and rules:
 *  - B + n_layers*B must not exceed 8192 entries (32 KB, held by every GPU that loads the
 *    library until the process exits); larger problems get RELAXKV_ERR_UNSUPPORTED_SHAPE.
 *  - The first call on each device looks up the array's device address (cudaGetSymbolAddress, with
 *    that device current).  Make that first call outside any stream capture.
 *  - All calls on a device share the one array, and it keeps the previous call's contents.  Nothing
 *    in it needs to start at zero (each call overwrites every entry it later reads), but two calls
 *    that overlap on the GPU - different streams, no ordering between them - race on it: order them.
 *  - h_counts_pinned (optional) is filled in `stream` order, as above.
 */
relaxkv_status relaxkv_build_active_sets_static(
    const relaxkv_shape* shape, int32_t n_layers, const int32_t* h_k, const int32_t* anchors,
    int32_t* highest_layer_out, int32_t* u_pos_out, int32_t* u_cu_out, int32_t* u_rank_out,
    int32_t* r_rank_out, int32_t* r_cu_out, int32_t* h_counts_pinned, relaxkv_stream stream);

/*
 * Sparse-context repair attention of one layer (Section 3.3, C_l(p); Section 3.4, mixed
 * fresh/cached K/V; Algorithm 1, steps 16-19; Appendix A.2).
 *
 * Target row rho of request b has rank c* = r_rank[r_cu_layer[b] + rho] in U_b and position
 * p = u_pos[u_cu[b] + c*].  With the context list X = U_b (RELAXKV_CTX_UNION; limit = c*) or
 * X = (0..T_c-1) (RELAXKV_CTX_FULL_PREFIX; limit = p), and
 *   Kt[x] = k_new[row of x] if X[x] is an active target of this layer, else cache K at X[x]
 * (same for V), the call computes for every query head h
 *   out[rho,h,:] = sum_{x <= limit} softmax_x(softmax_scale * <q_new[rho,h,:], Kt[x, h/G, :]>) * Vt[x, h/G, :]
 * The target itself is part of its context.  The cache is not modified.
 *
 * q_new           device bf16 [n_target_rows, H, D]; the rows of request b start at
 *                 r_cu_layer[b] - r_cu_layer[0] and follow the order of its R list.
 * k_new, v_new    device bf16 [n_target_rows, H_kv, D], or both NULL to read the cache only.
 * u_pos, u_cu     as written by relaxkv_build_active_sets.
 * r_rank          base of the packed rank array written by relaxkv_build_active_sets.
 * r_cu_layer      r_cu_out + l*B for this layer (B+1 offsets into r_rank are read).
 * n_target_rows   rows allocated in q_new/k_new/v_new/out (>= the layer's true total).
 * h_max_targets   host [B]: upper bound of |R_{l,b}|.   h_max_ctx: host [B]: upper bound of |U_b|.
 *                 A true count above its bound is reported through the device status word.
 * out             device bf16 [n_target_rows, H, D].
 * lse_out         NULL or device fp32 [H, n_target_rows]: log-normaliser of each output row.
 */
relaxkv_status relaxkv_sparse_ctx_attention(
    const relaxkv_shape* shape, relaxkv_ctx_mode mode, const relaxkv_cache_view* cache,
    const void* q_new, const void* k_new, const void* v_new,
    const int32_t* u_pos, const int32_t* u_cu, const int32_t* r_rank, const int32_t* r_cu_layer,
    int64_t n_target_rows, const int32_t* h_max_targets, const int32_t* h_max_ctx,
    void* out, float* lse_out,
    void* workspace, size_t workspace_bytes, relaxkv_stream stream);

/*
 * Cache update of one layer (Section 3.4; Algorithm 1, step 21): the fresh K/V of every active
 * target overwrite its cache entry; no other byte of the cache changes.  Idempotent.
 * Arguments as for relaxkv_sparse_ctx_attention; `cache` is written in place.
 */
relaxkv_status relaxkv_scatter_kv(
    const relaxkv_shape* shape, const relaxkv_cache_view* cache,
    const void* k_new, const void* v_new,
    const int32_t* u_pos, const int32_t* u_cu, const int32_t* r_rank, const int32_t* r_cu_layer,
    const int32_t* h_max_targets, relaxkv_stream stream);

/*
 * Materialised mixed context of one layer (Section 3.4 equation; Algorithm 1, steps 17-18):
 * k_ctx_out / v_ctx_out, device bf16 [ctx_rows, H_kv, D], receive for request b, at rows
 * x_cu[b] .. , Kt/Vt of the context list X defined above, where x_cu = u_cu (UNION) or the prefix
 * sums of T_c (FULL_PREFIX).  The 128 rows after the last one are zero-filled (as far as ctx_rows
 * allows).  ctx_rows >= sum_b h_max_ctx[b] (UNION) or sum_b T_c (FULL_PREFIX).
 * relaxkv_sparse_ctx_attention runs this step itself into its workspace; the entry point exists
 * so the step can be checked and timed on its own.
 */
relaxkv_status relaxkv_gather_kv(
    const relaxkv_shape* shape, relaxkv_ctx_mode mode, const relaxkv_cache_view* cache,
    const void* k_new, const void* v_new,
    const int32_t* u_pos, const int32_t* u_cu, const int32_t* r_rank, const int32_t* r_cu_layer,
    const int32_t* h_max_ctx, void* k_ctx_out, void* v_ctx_out, int64_t ctx_rows,
    relaxkv_stream stream);

/*
 * Repair attention for explicit target and context lists - the paper's controlled configurations
 * (Appendix A.3, table of configurations; Section 4.4 ablation; Appendix B): global repair targets P
 * with context C(p) = U intersect {j <= p} (RelaxKV^G, global target sweep), Global Sparse and Layerwise
 * Sparse context sets U_l with the method's targets R_l.  For request b the targets are the positions
 * tgt_pos[tgt_cu[b] .. tgt_cu[b+1]) and the context list is ctx_pos[ctx_cu[b] .. ctx_cu[b+1]), both
 * ascending; tgt_cu[0] must be 0.  Target rho at position p attends to the context entries with
 * position <= p; an entry whose position is itself a target contributes that target's fresh K/V, every
 * other entry the cached K/V (Section 3.4 equation with R_l := the target list).  A target need not be a
 * context entry (then it does not see itself); a target with no visible entry gets a zero output row and
 * lse = -inf (the paper does not define that case).  With ctx = U, tgt = R_l this equals
 * relaxkv_sparse_ctx_attention; with ctx = all positions, its full-prefix mode.
 * q_new/k_new/v_new/out rows follow the packed target order; other arguments as above.
 */
relaxkv_status relaxkv_list_attention(
    const relaxkv_shape* shape, const relaxkv_cache_view* cache,
    const void* q_new, const void* k_new, const void* v_new,
    const int32_t* ctx_pos, const int32_t* ctx_cu, const int32_t* tgt_pos, const int32_t* tgt_cu,
    int64_t n_target_rows, const int32_t* h_max_targets, const int32_t* h_max_ctx,
    void* out, float* lse_out, void* workspace, size_t workspace_bytes, relaxkv_stream stream);

/* Cache update for an explicit target list (Section 3.4): cache entries at tgt_pos receive k_new / v_new. */
relaxkv_status relaxkv_scatter_kv_lists(
    const relaxkv_shape* shape, const relaxkv_cache_view* cache, const void* k_new, const void* v_new,
    const int32_t* tgt_pos, const int32_t* tgt_cu, const int32_t* h_max_targets, relaxkv_stream stream);

/* Across-layer mean score g_i = (1/L) sum_l a_{l,i} (Appendix B; also the Global Sparse context source):
 * scores device fp32 [n_layers, sum_b T_c] -> mean_out device fp32 [sum_b T_c], summed in layer order.
 * Feed mean_out to relaxkv_select_topk (n_layers = 1) for the global target set or the shared context set. */
relaxkv_status relaxkv_mean_scores(const relaxkv_shape* shape, int32_t n_layers, const float* scores,
                                   float* mean_out, relaxkv_stream stream);

/*
 * The user query's own attention at one layer with the context scores taken from the same pass (Section 2,
 * the query's pass over the naive cache is what yields its attention to the context, layer by layer; Section 3.2, score
 * equation with the row normalisers of the query's real forward pass, whose softmax also spans the query's own
 * tokens).  For a serving caller this replaces relaxkv_score_select's scoring for the layer: the statistics pass
 * never runs, the scores come out of the forward pass the query makes anyway.
 *
 * For request b the cache holds the T_c = h_ctx_len[b] context rows followed by the Q_b = h_q_len[b] rows of the
 * query's own K/V (positions T_c .. T_c + Q_b - 1); it must hold h_req_token_offset[b] + T_c + Q_b token rows.
 *   out[t,h,:] = causal attention of query token t (position T_c + t) over positions 0 .. T_c + t of its request
 *   lse[h,t]   = log-normaliser of that row (context keys and the query's own keys up to t)
 *   raw[i]     = (1/(H*Q_b)) * sum_h sum_t exp(softmax_scale * <q[t,h,:], K[i,h/G,:]> - lse[h,t])      for i < T_c
 * q / out         device bf16 [sum_b Q_b, H, D]; lse_out device fp32 [H, sum_b Q_b] (required)
 * raw_scores_out  device fp32 [sum_b T_c], or NULL for the attention alone.  Stack the layers' rows and feed them to
 *                 relaxkv_select_topk for the anchors.
 * workspace       at least relaxkv_workspace_bytes() of the same shape with h_ctx_len[b] = T_c + Q_b.
 * Runs the cache-only attention kernel (which leaves the rows' normalisers), then the column-sum pass of the scoring
 * kernel over the context keys with those normalisers.
 */
relaxkv_status relaxkv_query_prefill_attention(
    const relaxkv_shape* shape, const relaxkv_cache_view* cache, const void* q, void* out, float* lse_out,
    float* raw_scores_out, void* workspace, size_t workspace_bytes, relaxkv_stream stream);

/* scores[l, i] *= factor, in place, for device fp32 [n_layers, sum_b T_c] (factor > 0).  Section 3.2's score is a mean
 * over all H query heads; when the heads are sharded over N devices of equal share, every device scores its own heads
 * (relaxkv_score_select with anchors_out = NULL), the devices' scores are summed by one all-reduce and this call with
 * factor = 1/N turns the sum of the shard means into the mean over all heads; relaxkv_select_topk follows. */
relaxkv_status relaxkv_scale_scores(const relaxkv_shape* shape, int32_t n_layers, float* scores, float factor,
                                    relaxkv_stream stream);

/*
 * ---- Dense block work of the active targets (Algorithm 1, steps 14, 16 and 20; Section 3.3 for the
 * position IDs).  The method leaves the Transformer block as it is and runs it on the |R_l| active rows only; these
 * calls are that block for a Llama-style pre-norm decoder.  All tensors bf16, row-major, 16-byte aligned,
 * feature counts multiples of 8; fp32 arithmetic inside.  The caller owns every buffer. ----
 */

/* y[r, :] = x[r, :] * rsqrt(mean(x[r, :]^2) + eps) * weight[:]      x, y [n_rows, n_cols], weight [n_cols] */
relaxkv_status relaxkv_rmsnorm(const void* x, const void* weight, void* y, int64_t n_rows, int32_t n_cols,
                               float eps, relaxkv_stream stream);

/* y = x weight^T (+ residual)      x [n_rows, n_in], weight [n_out, n_in] (the [out, in] layout),
 * residual NULL or [n_rows, n_out], y [n_rows, n_out] (may alias residual).  tcgen05 GEMM: 256-row tiles on SM pairs
 * for many rows; up to 128 rows (the query's own tokens, a decoded batch) 128 weight rows against all rows of x,
 * K split over a thread-block cluster and summed through distributed shared memory in a fixed order, so that
 * all SMs stream weights; one row (a decode token, the row that goes through the output head), and two to four
 * with a short K, stream the weights once through a plain HBM-bound kernel instead. */
relaxkv_status relaxkv_linear(const void* x, const void* weight, const void* residual, void* y,
                              int64_t n_rows, int32_t n_out, int32_t n_in, relaxkv_stream stream);

/* The attention block's three input projections in one call: q = x Wq^T, k = x Wk^T, v = x Wv^T with
 * w_qkv [n_q + 2 n_kv, n_in] = the rows of Wq, then Wk, then Wv (stacked once when the weights are loaded).
 * x [n_rows, n_in]; q [n_rows, n_q], k and v [n_rows, n_kv]: three separate row-major buffers.  Same arithmetic per
 * output element as relaxkv_linear.  Up to 128 rows (a decode token, the query's own tokens) this is ONE kernel that
 * streams the stacked matrix once; for more rows it is one large GEMM whose epilogue writes the three buffers when
 * n_q and n_kv are multiples of 32, else the three projections one after the other.
 * n_q, n_kv, n_in multiples of 8. */
relaxkv_status relaxkv_linear_qkv(const void* x, const void* w_qkv, void* q, void* k, void* v, int64_t n_rows,
                                  int32_t n_q, int32_t n_kv, int32_t n_in, relaxkv_stream stream);

/* out = silu(x Wg^T) * (x Wu^T) in one kernel (the MLP's first half): the gate and up projections and the
 * activation, with one rounding to bf16.  weight_tiled [2 * n_inter, n_in] holds, for every block t of 128
 * intermediate features, the 128 gate rows Wg[128 t .. 128 t + 127] followed by the 128 up rows Wu[same range]
 * (a fixed re-ordering of the rows of [Wg; Wu], done once when the weights are loaded), so that a 128 x 256
 * output tile of the GEMM carries both halves of the same features.  n_inter a multiple of 128.
 * x [n_rows, n_in], out [n_rows, n_inter]. */
relaxkv_status relaxkv_linear_swiglu(const void* x, const void* weight_tiled, void* out, int64_t n_rows,
                                     int32_t n_inter, int32_t n_in, relaxkv_stream stream);

/* Rotary embedding in place, rotate-half convention: pair i < D/2 of each head vector is rotated by
 * positions[row] * theta^(-2i/D).  x [n_rows, n_heads, head_dim]; positions: device int32 [n_rows], the rows'
 * ORIGINAL global positions (Section 3.3: restricting the context does not renumber tokens).  Rotations
 * compose, so the same call re-aligns the cached keys of a chunk that is placed at another offset than the
 * one it was encoded at (Section 2, positional consistency): pass the offset difference (it may be negative)
 * as every token's position. */
relaxkv_status relaxkv_rope(void* x, int64_t n_rows, int32_t n_heads, int32_t head_dim, const int32_t* positions,
                            float theta, relaxkv_stream stream);

/* The per-head RMSNorm of the projected queries and keys (models that have one; pass NULL weights otherwise) followed by
 * the rotary embedding, on q [n_rows, n_q_heads, head_dim] and k [n_rows, n_kv_heads, head_dim] in place, in ONE
 * launch: the same results as relaxkv_rmsnorm on the head vectors of q and of k followed by relaxkv_rope on q and on
 * k (the normalised values are rounded to bf16 in between, as a store would), meant for the few rows of a query pass
 * or a decode step, where four launches cost more than their work.  w_q_norm, w_k_norm: [head_dim] or both NULL. */
relaxkv_status relaxkv_qk_norm_rope(void* q, void* k, int64_t n_rows, int32_t n_q_heads, int32_t n_kv_heads,
                                    int32_t head_dim, const void* w_q_norm, const void* w_k_norm, float eps,
                                    const int32_t* positions, float theta, relaxkv_stream stream);

/* relaxkv_qk_norm_rope of q and k [n_rows, ..] at positions tgt_pos, then relaxkv_scatter_kv_lists of k and v to the same positions: the
 * rows of a decode step or a query pass, packed in list order (tgt_cu[0] = 0), rotated and appended to the cache in one launch (more
 * than 512 rows: in two).  Errors as for the two calls. */
relaxkv_status relaxkv_qk_norm_rope_append(
    const relaxkv_shape* shape, const relaxkv_cache_view* cache, void* q, void* k, const void* v, int64_t n_rows, const void* w_q_norm,
    const void* w_k_norm, float eps, const int32_t* tgt_pos, const int32_t* tgt_cu, const int32_t* h_max_targets, float theta,
    relaxkv_stream stream);

/* out[r, i] = silu(gate_up[r, i]) * gate_up[r, n_inter + i]      gate_up [n_rows, 2*n_inter], out [n_rows, n_inter] */
relaxkv_status relaxkv_swiglu(const void* gate_up, void* out, int64_t n_rows, int32_t n_inter, relaxkv_stream stream);

/* positions_out[row] = position of target row of this layer (row order = the layer's R lists, requests
 * packed): u_pos[u_cu[b] + r_rank[r_cu_layer[b] + rho]].  Feeds relaxkv_rope. */
relaxkv_status relaxkv_target_positions(const relaxkv_shape* shape, const int32_t* u_pos, const int32_t* u_cu,
                                        const int32_t* r_rank, const int32_t* r_cu_layer,
                                        const int32_t* h_max_targets, int32_t* positions_out, relaxkv_stream stream);

/* Hidden-state carry between layers (Section 3.2: a token stays active through its highest selected layer):
 * h_out gets, in the row order of layer l+1's targets, the rows of h_in (row order of layer l's targets)
 * that stay active.  r_cu_layer = r_cu + l*B, r_cu_next = r_cu + (l+1)*B; h_max_next: host bounds on
 * |R_{l+1,b}|.  h_in, h_out [rows, n_cols], distinct buffers. */
relaxkv_status relaxkv_carry_rows(const relaxkv_shape* shape, const void* h_in, void* h_out, int32_t n_cols,
                                  const int32_t* r_rank, const int32_t* r_cu_layer, const int32_t* r_cu_next,
                                  const int32_t* h_max_next, relaxkv_stream stream);

/*
 * Test utility: the same result as relaxkv_sparse_ctx_attention from a plain SIMT kernel (one warp
 * per output row, fp32 throughout, no tensor cores).  A second opinion for debugging; far slower.
 */
relaxkv_status relaxkv_sparse_ctx_attention_simt(
    const relaxkv_shape* shape, relaxkv_ctx_mode mode, const relaxkv_cache_view* cache,
    const void* q_new, const void* k_new, const void* v_new,
    const int32_t* u_pos, const int32_t* u_cu, const int32_t* r_rank, const int32_t* r_cu_layer,
    int64_t n_target_rows, const int32_t* h_max_targets, const int32_t* h_max_ctx,
    void* out, float* lse_out,
    void* workspace, size_t workspace_bytes, relaxkv_stream stream);

/*
 * Attention of given token positions over the cache's own causal prefix, cache only: target t of request b,
 * at position p = tgt_pos[tgt_cu[b] + t], attends to every cache entry j <= p of its request.  This is the pass
 * the paper runs after the repair loop (the user query's prefill rows and the first decode step read the
 * repaired cache; Section 3.4 and the TTFT protocol of the reproducibility appendix): the caller has appended
 * the K/V of those tokens to the cache, `shape->h_ctx_len[b]` counts them.  No context is gathered: the
 * kernel's tiled loads read the cache through its strides, so the call moves K and V once.
 *   q_new  device bf16 [n_target_rows, H, D], rows in tgt order, requests packed
 *   tgt_pos / tgt_cu  device int32: ascending positions per request, packed; offsets [B + 1], tgt_cu[0] = 0
 *   h_max_targets  host [B] upper bounds on the target counts
 *   out  device bf16 [n_target_rows, H, D]; lse_out optional device fp32 [H, n_target_rows]
 * The cache must hold max_b(h_req_token_offset[b] + h_ctx_len[b]) token rows.  Errors as for
 * relaxkv_sparse_ctx_attention (positions out of range are reported in the device status word).
 * When every h_max_targets[b] <= 1 (a decode step) the call takes a streaming kernel instead of the 128-row tensor-core
 * tiles: K and V tiles through a TMA ring, the request's few query heads in one warp-level MMA fragment, the context
 * split over one wave of thread blocks and merged in a fixed order.
 */
relaxkv_status relaxkv_cache_attention(
    const relaxkv_shape* shape, const relaxkv_cache_view* cache, const void* q_new,
    const int32_t* tgt_pos, const int32_t* tgt_cu, int64_t n_target_rows, const int32_t* h_max_targets,
    void* out, float* lse_out, void* workspace, size_t workspace_bytes, relaxkv_stream stream);

/*
 * ---- Many continuations of a repaired context.  (The paper answers one query per repair; these calls are for the callers that answer
 * from one repaired context many times: several samples, follow-up questions.)  The contexts stay where the repair left them, in a
 * relaxkv_cache_view; every continuation ("sequence") keeps the K/V of its own tokens - the question, the answer so far - in blocks of a
 * paged store.  One step appends some tokens to some sequences (a "row" each) and attends from those rows.  ----
 *
 * In these calls shape->h_ctx_len[b] may be 0 (a sequence without a context), h_q_len is not read, h_tuning neither.
 */

/* The paged store of one layer.  Token t of block x of KV head g lives at k + x * block_stride + t * token_stride + g * head_stride (in
 * elements), same for V: [n_blocks, block_size, H_kv, D] and [n_blocks, H_kv, block_size, D] storage.  Strides are multiples of 8. */
typedef struct {
  void* k;
  void* v;
  int64_t block_stride;
  int64_t token_stride;
  int64_t head_stride;
  int32_t block_size;                  /* tokens of a block: 16, 32, 64 or 128                                  */
  int32_t n_blocks;
} relaxkv_paged_cache;

/* The rows of a step.  Sequences are grouped by their context; row r belongs to sequence row_seq[r] and sees the whole context of that
 * sequence and the first row_len[r] tokens of the sequence's own (itself the last of them, once it has been appended). */
typedef struct {
  int32_t n_seq;                       /* sequences                                                             */
  int32_t table_width;                 /* blocks a row of block_table has room for                              */
  int64_t table_stride;                /* elements between the rows of block_table                              */
  int64_t n_rows;                      /* rows allocated in q / out                                             */
  int32_t max_len;                     /* upper bound of row_len                                                */
  const int32_t* h_seq_cu;             /* host [n_req+1]: sequences [h_seq_cu[b], h_seq_cu[b+1]) continue context b; from 0 to n_seq */
  const int32_t* h_max_rows;           /* host [n_req]: upper bound of the rows of context b                    */
  const int32_t* row_cu;               /* device [n_seq+1]: rows [row_cu[i], row_cu[i+1]) are sequence i's      */
  const int32_t* row_seq;              /* device [n_rows]; -1: no row (left alone)                              */
  const int32_t* row_len;              /* device [n_rows]                                                       */
  const int32_t* block_table;          /* device [n_seq, table_width]: the blocks of every sequence in order    */
} relaxkv_continuation_rows;

/* Bytes of device scratch that suffice for the three calls below that take a workspace, with these shapes, up to n_rows rows and context
 * blocks of block_size tokens (0: no block selection).  Returns 0 for an invalid shape.  Host only. */
size_t relaxkv_continuation_workspace_bytes(const relaxkv_shape* shape, int64_t n_rows, int32_t block_size);

/*
 * Block tables and slot maps of a step from the sequences' lengths, on the device.  Sequence i holds seq_len[i] tokens in the blocks
 * block_table[i, 0 .. ceil(seq_len[i] / block_size)); new_len[i] >= 0 tokens are appended to it, new_len[i] < 0 ends it: its blocks are free
 * again (before new ones are taken) and its length is 0.
 *   stack     free_blocks[0 .. n_free[0]), then the ended sequences' blocks in sequence order
 *   taken     from the end of the stack, in sequence order; written to block_table behind the blocks a sequence has
 *   rows      of sequence i: [row_cu[i], row_cu[i+1]); token j of them has row_seq = i, row_len = seq_len[i] + j + 1,
 *             row_pos = seq_base[i] + seq_len[i] + j (seq_base NULL: 0) and row_slot = block * block_size + place in the block.
 *             Rows from row_cu[n_seq] to n_rows: row_seq = row_slot = -1, row_len = row_pos = 0.
 * seq_len_out and n_free_out receive the lengths and the free blocks left, the next step's inputs (they may not overlap seq_len, new_len and
 * n_free); the stack that is left stands in free_blocks, which is written from entry n_free[0] on only.  Same inputs, same results: the call
 * may be repeated.
 * A sequence with seq_len < 0, more tokens than its row of block_table holds or new_len > n_rows is left as it is; more rows than n_rows, more
 * blocks than there are: nothing is appended to any sequence (ended ones still end); n_free or the blocks given back beyond free_capacity:
 * nothing happens at all.  Each is reported in the device status word.  Block numbers are not looked at here (the calls that use them do).
 * A block is one sequence's: one that stands in two rows of block_table is given back by each of them when it ends.
 * n_seq <= 4096.
 */
relaxkv_status relaxkv_build_block_tables(
    int32_t n_seq, int32_t block_size, const int32_t* seq_len, const int32_t* new_len, const int32_t* seq_base, int32_t* free_blocks,
    int32_t free_capacity, const int32_t* n_free, int32_t* block_table, int32_t table_width, int64_t table_stride, int64_t n_rows,
    int32_t* seq_len_out, int32_t* n_free_out, int32_t* row_cu, int32_t* row_seq, int32_t* row_pos, int32_t* row_len, int32_t* row_slot,
    relaxkv_stream stream);

/* The per-head RMSNorm of the projected queries and keys (weights [head_dim], or both NULL), the rotary embedding at `positions` and the
 * append of K and V to the paged store in ONE pass: q_out = rotated q (may be q itself), store.k[slot] = rotated k, store.v[slot] = v.
 * Arithmetic in fp32 (angles in fp64) with one rounding to bf16 at the end.  q, q_out [n_rows, n_q_heads, head_dim], k and v [n_rows, n_kv_heads,
 * head_dim] (left as they are); positions, slots device int32 [n_rows]; a row with slot -1 is rotated and not stored, another slot outside the
 * store is reported and not stored.  Slots are distinct. */
relaxkv_status relaxkv_qk_norm_rope_append_paged(
    const relaxkv_paged_cache* store, const void* q, const void* k, const void* v, int64_t n_rows, int32_t n_q_heads, int32_t n_kv_heads,
    int32_t head_dim, const void* w_q_norm, const void* w_k_norm, float eps, const int32_t* positions, const int32_t* slots, float theta,
    void* q_out, relaxkv_stream stream);

/*
 * Attention of a step's rows over [the shared context, the sequence's own tokens]: for row r of sequence i of context b
 *   out[r,h,:] = softmax over j < T_b and t < row_len[r] of scale * <q[r,h,:], K>, times V      K = cache rows of context b, then
 *                                                                                              the store's tokens of sequence i
 * A context is read once for all its rows, whatever their number.  cache may be NULL where every context is empty, store NULL where max_len is 0.
 * A row that sees no key at all gets zeros and lse = -inf.
 *   q, out  device bf16 [n_rows, H, D] (16-byte aligned); lse_out NULL or device fp32 [H, n_rows]
 * Rows with row_seq -1 are left alone.  Reported and left alone: row_seq or row_len out of range, rows of a context above h_max_rows, rows that
 * row_cu does not count among those of their sequence's context.  A block number out of range is reported, its tokens are passed over.
 * T_b, max_len and the cache rows that a context spans: up to 2^31 - 256 tokens, more is refused.
 */
relaxkv_status relaxkv_shared_prefix_attention(
    const relaxkv_shape* shape, const relaxkv_cache_view* cache, const relaxkv_paged_cache* store, const relaxkv_continuation_rows* rows,
    const void* q, void* out, float* lse_out, void* workspace, size_t workspace_bytes, relaxkv_stream stream);

/*
 * 8-bit bounds of the keys of every context block (block x of context b: tokens [x * block_size, (x+1) * block_size) of it, the last one what is
 * left).  For block x and KV head g, with hi_d and lo_d the largest and the smallest key element of dim d (NaN are passed over):
 *   scale = the smallest power of two s with |hi_d|, |lo_d| <= 127 s for all d (at least 2^-100; 1 if all are 0)
 *   bounds[x, g, 0, d] = ceil(hi_d / s), bounds[x, g, 1, d] = floor(lo_d / s)       as int8 (beyond +-127: +-127)
 * bounds_out int8 [sum_b n_b, H_kv, 2, D] (16-byte aligned), scale_out fp32 [sum_b n_b, H_kv], n_b = ceil(T_b / block_size); only cache->k is read.
 * block_size 16, 32, 64 or 128.
 */
relaxkv_status relaxkv_block_bounds(const relaxkv_shape* shape, const relaxkv_cache_view* cache, int32_t block_size, int8_t* bounds_out,
                                    float* scale_out, relaxkv_stream stream);

/*
 * The context blocks that a row may need most: with q_h in 8 bits the way the bounds are (scale s_h per row and head, rounded to nearest even),
 *   score[x] = scale[x] * max over the heads h of the KV head's group of s_h * sum_d (max(q_hd, 0) * hi_d + min(q_hd, 0) * lo_d),
 * the largest logit that a key within the bounds could have with this rounded query (of the query itself a logit may lie above).  All terms are whole numbers below 2^24 and powers of two, so scores do not depend on
 * the order of summation.  Selected are the n_select blocks of the highest score, equal scores by the lower number, the first n_first and the last
 * n_last blocks in any case.
 * blocks_out device int32 [n_rows, H_kv, n_select]: ascending, -1 behind them.  n_first + n_last <= n_select.
 * Of rows only h_seq_cu, h_max_rows, n_seq, n_rows, row_cu and row_seq are read; rows with row_seq -1 are left alone.
 */
relaxkv_status relaxkv_select_blocks(
    const relaxkv_shape* shape, int32_t block_size, const int8_t* bounds, const float* scale, const relaxkv_continuation_rows* rows, const void* q,
    int32_t n_select, int32_t n_first, int32_t n_last, int32_t* blocks_out, void* workspace, size_t workspace_bytes, relaxkv_stream stream);

/* relaxkv_shared_prefix_attention with, of each context, only the tokens of the blocks that `blocks` (device int32 [n_rows, H_kv, n_select]) lists
 * for the row and KV head: distinct, in any order, entries -1 are passed over; another number without a block is reported and passed over. */
relaxkv_status relaxkv_block_sparse_attention(
    const relaxkv_shape* shape, const relaxkv_cache_view* cache, const relaxkv_paged_cache* store, const relaxkv_continuation_rows* rows,
    int32_t block_size, const int32_t* blocks, int32_t n_select, const void* q, void* out, float* lse_out, void* workspace, size_t workspace_bytes,
    relaxkv_stream stream);

/*
 * ---- Contexts kept in 8 bits.  (The paper reuses chunk caches without saying how they are kept.)  Chunks, repaired contexts and
 * what sequences add to them live in blocks of a paged store with one byte per element and one power of two per token and head; they
 * are written as they come (out of a cache, or a step's rows with norm and rotation), read back at any position, and attended to
 * where they are.  ----
 */

typedef enum {
  RELAXKV_INT8 = 0,                    /* whole numbers from -127 to 127                                        */
  RELAXKV_E4M3 = 1                     /* 8-bit floating point, 4 bits of exponent, 3 of mantissa, up to 448    */
} relaxkv_quantized_type;

/*
 * The 8-bit store of one layer.  Token t of block x of KV head g: values at k + x * block_stride + t * token_stride + g *
 * head_stride (bytes = elements; head_dim of them side by side), same for V, strides multiples of 16, that of heads below 2^31;
 * exponents at k_exp + (x * n_kv_heads + g) * block_size + t, same for V. An element stands for value * 2^exponent; exponent -128
 * says that all elements of the token and head are NaN; others are -100 to 127. No value byte is a NaN of e4m3
 * (relaxkv_append_quantized writes none).  All pointers 16-byte aligned.
 */
typedef struct {
  void* k;
  void* v;
  int8_t* k_exp;
  int8_t* v_exp;
  int64_t block_stride;
  int64_t token_stride;
  int64_t head_stride;
  int32_t block_size;                  /* tokens of a block: 16, 32, 64 or 128                                  */
  int32_t n_blocks;
  int32_t n_kv_heads;
  int32_t type;                        /* relaxkv_quantized_type                                                */
} relaxkv_quantized_cache;

/*
 * A rotary embedding.  The first `dims` dims of a head (a multiple of 8) are dims / 2 pairs, pair i of them (i, i + dims / 2), or
 * (2i, 2i + 1) where interleaved; at position p it turns by p * freq[i], and grows by amplitude.  Dims behind them stay as they are.
 */
typedef struct {
  const double* freq;                  /* device [dims / 2]: radians per position                               */
  int32_t dims;
  int32_t interleaved;                 /* 0 or 1                                                                */
  float amplitude;                     /* > 0, usually 1                                                        */
} relaxkv_rotary;

/* How frequencies are scaled for contexts that are longer than those a model was first trained on. */
typedef enum {
  RELAXKV_SCALE_NONE = 0,
  RELAXKV_SCALE_LINEAR = 1,            /* freq / factor (position interpolation)                                */
  RELAXKV_SCALE_BANDS = 2,             /* by wavelength: fewer than `low` turns in original_len positions: freq / factor; more than `high`: freq; between  */
                                       /* them linear in the number of turns                                    */
  RELAXKV_SCALE_RAMP = 3               /* by pair number, between those that make `high` and `low` turns in original_len positions; amplitude            */
                                       /* 0.1 ln(factor) + 1 (YaRN)                                             */
} relaxkv_rotary_scaling;

/* freq_out[i] (host [dims / 2]) = theta^(-2i / dims), scaled; *amplitude_out.  factor >= 1, 0 < low < high and original_len >= 1 where they are read.  Host only. */
relaxkv_status relaxkv_rotary_frequencies(int32_t dims, double theta, int32_t scaling, double factor, int32_t original_len, double low, double high,
                                          double* h_freq_out, float* h_amplitude_out);

/*
 * relaxkv_qk_norm_rope for any rotary embedding and any strides: q_out = rotated norm of q, k_out likewise, one rounding to bf16
 * (angles in fp64 up to their remainder, the rest in fp32).  Head h of row r: q + r * q_token_stride + h * q_head_stride, head_dim
 * elements side by side; q_out is laid out like q and may be q itself, k_out like k.  q or k may be NULL, its output with it (only
 * the other one is turned).  Norm weights [head_dim] as in relaxkv_qk_norm_rope.  head_dim 64 or 128, strides multiples of 8, those
 * of heads below 2^31; positions device int32 [n_rows], negative ones turn backwards.
 */
relaxkv_status relaxkv_qk_norm_rotate(
    const void* q, void* q_out, int64_t q_token_stride, int64_t q_head_stride, const void* k, void* k_out, int64_t k_token_stride, int64_t k_head_stride,
    int64_t n_rows, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, const void* w_q_norm, const void* w_k_norm, float eps, const int32_t* positions,
    const relaxkv_rotary* rotary, relaxkv_stream stream);

/*
 * Append of rows to the 8-bit store: row r of K (normed and rotated as above where weights and a rotary are given, NULL: as it is)
 * and of V goes to slot slots[r] = block * block_size + token; q_out = rotated norm of q as above (q NULL: none).  For each row and
 * KV head, with y in fp32 before any rounding and M = 127 or 448:
 *   exponent = the smallest e >= -100 with max |y| <= M 2^e (-100 where all are 0);  value = y 2^-e to the nearest, ties to even
 * (an infinite or NaN element makes the exponent -128 and the values 0).  What relaxkv_read_quantized returns without a rotation
 * stands for the same values when it is appended again, but for heads with an element of almost 2^128 that the rounding to 8 bits
 * has taken there: in bf16 that is infinite. v is laid out like k.  Slots are distinct; a row with slot -1 is turned and not stored,
 * another slot outside the store is reported and not stored.
 */
relaxkv_status relaxkv_append_quantized(
    const relaxkv_quantized_cache* store, const void* q, void* q_out, int64_t q_token_stride, int64_t q_head_stride, const void* k, const void* v,
    int64_t k_token_stride, int64_t k_head_stride, int64_t n_rows, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, const void* w_q_norm,
    const void* w_k_norm, float eps, const int32_t* positions, const relaxkv_rotary* rotary, const int32_t* slots, relaxkv_stream stream);

/*
 * Rows of the 8-bit store in bf16: k_out, v_out row r (laid out as k above, v_out like k_out) = the token at slots[r], its keys
 * turned by positions[r] positions more (positions and rotary both NULL: as they are, which is exact; what stands for 2^128 or more
 * is infinite).  A row with slot -1 is left alone, another slot outside the store is reported and left alone.
 */
relaxkv_status relaxkv_read_quantized(
    const relaxkv_quantized_cache* store, const int32_t* slots, int64_t n_rows, int32_t n_kv_heads, int32_t head_dim, const int32_t* positions,
    const relaxkv_rotary* rotary, void* k_out, void* v_out, int64_t token_stride, int64_t head_stride, relaxkv_stream stream);

/* Bytes of device scratch that suffice for any relaxkv_quantized_attention with these heads.  Returns 0 for an invalid shape.  Host only. */
size_t relaxkv_quantized_workspace_bytes(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim);

/*
 * Attention of a step's rows over their sequence's tokens in the 8-bit store: row r of sequence i sees the first row_len[r] tokens
 * of the blocks block_table[i, ..],
 *   out[r,h,:] = softmax over t < row_len[r] of softmax_scale * <q[r,h,:], K[t]>, times V        (keys and values as the store's bytes stand for them)
 * q and the keys meet as they are (exact products, fp32 sums); weights are rounded to 11 bits, and to 2^-38 of the row's largest
 * (weight times value's scale), before they meet the values.  Any number of rows to a sequence.  With G = n_q_heads / n_kv_heads <=
 * 16 and G times the sequences' rows on average up to 32, a sequence's tokens are read once for 8 / G to 32 / G rows of it; beyond
 * that once for 128 / G, and weights are rounded to 2^-35 of (the row's largest weight times the largest value's scale of the tokens
 * that it sees).  Of rows n_seq, table_width, table_stride, n_rows, max_len, row_cu, row_seq, row_len and block_table are read;
 * n_seq <= 4096; row_len does not fall within a sequence.  A row that sees no token gets zeros and lse = -inf.
 *   q, out  device bf16 [n_rows, n_q_heads, head_dim] (16-byte aligned, not the same); lse_out NULL or device fp32 [n_q_heads, n_rows]
 * Rows with row_seq -1 and rows behind row_cu[n_seq] are left alone.  Reported and left alone: rows of a sequence whose row_cu, or
 * whose last row_len, is out of range, rows whose row_seq is another sequence, whose row_len is negative or above the sequence's
 * last.  A block number out of range is reported, its tokens are passed over.  max_len up to 2^31 - 256.
 */
relaxkv_status relaxkv_quantized_attention(
    const relaxkv_quantized_cache* store, const relaxkv_continuation_rows* rows, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, float softmax_scale,
    const void* q, void* out, float* lse_out, void* workspace, size_t workspace_bytes, relaxkv_stream stream);

/*
 * Test utility for the bounded waits (the paper has no counterpart): launches one thread that waits on
 * a barrier nothing will ever complete.  The wait gives up after its limit (0.4 s), the kernel ends
 * normally and RELAXKV_ERR_TIMEOUT is recorded in the device status word - the same path a stuck
 * pipeline takes in the attention and scoring kernels.  Nothing hangs or faults.
 */
relaxkv_status relaxkv_debug_wait_timeout(relaxkv_stream stream);

/*
 * Chained launches.  The kernels of the calls above (all but the explicit-list maps, the score averages and relaxkv_rope) are
 * launched with CUDA's programmatic stream serialization: the next kernel's blocks become resident
 * while the current kernel finishes, request the head of their weights into L2 (weights depend on
 * no earlier kernel) and then wait, inside the kernel, until every earlier kernel of the stream has
 * completed and its writes are visible.  Results are identical to plain
 * launches; stream order as the caller sees it is unchanged; the launches can be captured into a
 * CUDA graph.  relaxkv_set_chained_launch(0) switches to plain launches for the whole process
 * (1 = chained, the default) and returns the previous setting; it affects calls made after it.
 */
int32_t relaxkv_set_chained_launch(int32_t on);

/*
 * Synchronises `stream`, copies the device status word (a relaxkv_status: RELAXKV_OK,
 * RELAXKV_ERR_BAD_INDEX or RELAXKV_ERR_TIMEOUT, the first problem recorded wins) to
 * *h_status_out and clears it.  h_detail_out (NULL or host int32[4]) receives where it happened:
 * kernel id, block, and two kernel-specific values.
 */
relaxkv_status relaxkv_read_device_status(int32_t* h_status_out, int32_t* h_detail_out, relaxkv_stream stream);

#ifdef __cplusplus
}
#endif
#endif  /* RELAXKV_H_ */

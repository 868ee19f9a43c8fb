/*
 * libcascade: one token-sharded transformer layer on one MI355X (gfx950).
 *
 * The library computes the single-layer forward pass of Cascade (Section 5,
 * Algorithm 1) with every shard resident on one GPU: per-shard linear layers
 * (Algorithm 2, the projection that closes Algorithm 4, the MLP step that closes Algorithm 1), partial
 * attention for every (query-shard, key/value-shard) pair with row maxima m and
 * subtract-max exponential sums e (Algorithm 3), and the log-sum-exp merge of
 * the partials (the merge steps of Algorithm 4).  A plan carries the sharding R of the
 * hidden rows and, optionally, a distinct sharding S of queries / keys / values
 * (cascade_plan_create_rs); cascade_plan_create sets S = R.
 *
 * Conventions
 *  - Every function returns an int32 status (CASCADE_OK = 0).  Nothing aborts,
 *    throws or prints.  After CASCADE_EHIP, cascade_last_hip_error() returns the
 *    HIP runtime code.
 *  - Pointers are DEVICE pointers unless the name ends in _host.  The library
 *    borrows them: the caller allocates and frees.  Tensor memory is never
 *    allocated here; scratch comes from the caller's workspace.  Only
 *    cascade_plan_create allocates (the index maps it owns).
 *  - All work is enqueued on the caller's HIP stream (void* = hipStream_t) and
 *    is asynchronous; there are no hidden synchronisations.
 *  - Row-major everywhere; a weight matrix is [out_features, in_features].
 *  - "Packed" row order: shards in shard-id order, rows inside a shard in
 *    ascending original token index (the concatenation rule of the
 *    Attention-Pass subsection).  perm[r] = original index of packed row r.
 *  - dtype CASCADE_BF16: tensors are bf16, accumulation and m, e, u are fp32.
 *    dtype CASCADE_F32: everything fp32.
 *  - Empty shards are legal.  A query row that sees no key of a shard gets
 *    m = -inf, e = 0, u = 0 and weight 0 in the merge.
 */
#ifndef CASCADE_H
#define CASCADE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define CASCADE_API __attribute__((visibility("default")))
#else
#define CASCADE_API
#endif

/* status codes */
#define CASCADE_OK            0
#define CASCADE_EINVAL        1   /* null pointer or negative / zero size               */
#define CASCADE_ESHAPE        2   /* dimensions inconsistent with each other / the plan */
#define CASCADE_EASSIGN       3   /* shard id outside [0, n_shards)                     */
#define CASCADE_EUNSUPPORTED  4   /* dtype / head_dim / option not built                */
#define CASCADE_EWORKSPACE    5   /* workspace missing or too small                     */
#define CASCADE_EHIP          6   /* HIP runtime error                                  */

#define CASCADE_F32   0
#define CASCADE_BF16  1

#define CASCADE_MASK_NONE    0
#define CASCADE_MASK_CAUSAL  1   /* key visible iff position[key] <= position[query]   */

#define CASCADE_ROWS_ORIGINAL  0 /* row t of a sequence is token t                     */
#define CASCADE_ROWS_PACKED    1 /* row r of a sequence is token perm[r]               */

#define CASCADE_U_UNNORMALISED 0 /* u~ = sum_s exp(a - m) v_s  (= e * u)               */
#define CASCADE_U_NORMALISED   1 /* u  = softmax(a^{S_j S_k}) v^{S_k} (Algorithm 3)    */

#define CASCADE_NORM_NONE      0
#define CASCADE_NORM_LAYERNORM 1
#define CASCADE_NORM_RMSNORM   2

#define CASCADE_ACT_GELU_ERF   0
#define CASCADE_ACT_GELU_TANH  1
#define CASCADE_ACT_SWIGLU     2

#define CASCADE_ATTN_FUSED        0 /* running merge in registers, no partials written */
#define CASCADE_ATTN_MATERIALISED 1 /* partial_attn -> m, e, u~ in HBM -> lse_merge     */

/* epilogue flags of cascade_shard_gemm (bit mask) */
#define CASCADE_EPI_BIAS       1
#define CASCADE_EPI_GELU_ERF   2
#define CASCADE_EPI_GELU_TANH  4
#define CASCADE_EPI_SWIGLU     8   /* Y = silu(X W^T) * (X W_up^T)                      */
#define CASCADE_EPI_ROPE       16  /* rotate the first rope_cols columns head by head   */
#define CASCADE_EPI_RESIDUAL   32  /* Y += residual                                     */

/* ------------------------------------------------------------------ shard plan
 * Section 5.1: the partition of [N] into shards, as index maps.  Built on the
 * host from token_to_shard_host[seq_len] (values in [0, n_shards)), copied to
 * the current device.  positions_host[seq_len] gives each token's position for
 * the causal mask and the rotary embedding (NULL: position t = t).  The same
 * assignment is shared by all `batch` sequences.
 * Errors: EINVAL (null out / host array, sizes <= 0, unknown mask kind),
 * EASSIGN (shard id out of range), EHIP.                                       */
typedef struct cascade_plan cascade_plan;

CASCADE_API int32_t cascade_plan_create(cascade_plan **out, int32_t batch, int32_t seq_len, int32_t n_shards,
                            const int32_t *token_to_shard_host, const int32_t *positions_host,
                            int32_t mask_kind);

/* Device pointers to perm[seq_len], inv_perm[seq_len], offsets[n_shards + 1]
 * (int32, owned by the plan); any out pointer may be NULL.                     */
CASCADE_API int32_t cascade_plan_maps(const cascade_plan *plan, const int32_t **perm_dev,
                          const int32_t **inv_perm_dev, const int32_t **offsets_dev);

/* Host copies of the same maps (owned by the plan).                            */
CASCADE_API int32_t cascade_plan_maps_host(const cascade_plan *plan, const int32_t **perm_host,
                               const int32_t **inv_perm_host, const int32_t **offsets_host);

/* Section 5.1 keeps the sharding of hidden states {R_i} (alpha shards) apart from
 * the sharding of queries / keys / values {S_j} (beta shards); Section 6.4 refines
 * R into S by an m-split.  This variant takes both: token_to_row_shard_host
 * defines the packed row order and the row shards (as token_to_shard_host does
 * above); token_to_kv_shard_host[seq_len] (values in [0, n_kv_shards)) defines the
 * key/value shards S_k.  Partials then have one entry per key/value shard:
 * m, e [B,H,n_kv_shards,N], u [B,n_kv_shards,H,N,d], rows in the row partition's
 * packed order; cascade_lse_merge merges over the n_kv_shards partials.  Keys of
 * S_k are taken in ascending token index (the sorted concatenation rule of the
 * Attention-Pass subsection).  The result of the merged attention does not depend
 * on either partition.  Errors as cascade_plan_create.                          */
CASCADE_API int32_t cascade_plan_create_rs(cascade_plan **out, int32_t batch, int32_t seq_len, int32_t n_row_shards,
                               const int32_t *token_to_row_shard_host, int32_t n_kv_shards,
                               const int32_t *token_to_kv_shard_host, const int32_t *positions_host,
                               int32_t mask_kind);

/* Host copies of the key/value partition's maps (owned by the plan): its shard
 * count, kv_perm[seq_len] (kv-packed row -> token), kv_offsets[n_kv_shards + 1],
 * kv_to_row[seq_len] (kv-packed row -> packed row of the row partition; NULL is
 * returned when the plan has a single partition).  Any out pointer may be NULL.  */
CASCADE_API int32_t cascade_plan_kv_maps_host(const cascade_plan *plan, int32_t *n_kv_shards,
                                  const int32_t **kv_perm_host, const int32_t **kv_offsets_host,
                                  const int32_t **kv_to_row_host);

/* (c, delta)-sharding of Section 6: 0-based token t belongs to shard
 * (t mod delta) div c; writes token_to_shard_host[seq_len] and the shard count
 * ceil(delta / c) (n_shards may be NULL).  Host only.  Errors: EINVAL.           */
CASCADE_API int32_t cascade_cdelta_assignment(int32_t seq_len, int32_t c, int32_t delta,
                                  int32_t *token_to_shard_host, int32_t *n_shards);

/* m-split of Section 6.4: the sorted tokens of row shard i are dealt round-robin
 * into m pieces (piece x takes the elements at sorted indices x, x + m, ...), and
 * piece x of shard i becomes key/value shard m i + x (0-based), so there are
 * m * n_row_shards key/value shards.  Writes token_to_kv_shard_host[seq_len].
 * Host only.  Errors: EINVAL, EASSIGN (row shard id out of range), EUNSUPPORTED. */
CASCADE_API int32_t cascade_m_split(int32_t seq_len, int32_t n_row_shards, const int32_t *token_to_row_shard_host,
                        int32_t m, int32_t *token_to_kv_shard_host);

/* Cost model of the multi-party setting the method was designed for (Equation 1
 * and the rounds count of the Communication Analysis appendix); on one GPU these
 * are the bytes MATERIALISED mode moves through HBM.  Per layer:
 *   stage_a_bytes = beta F d (H + 2 H_KV) N     q, k, v rows to the AttnNodes
 *   stage_b_bytes = beta F (d + 2) H N          m, e, u rows back
 *   rounds        = 2 alpha beta^2, or 2 beta^2 when m_split_scheme != 0
 *                   ((c, delta)-sharding with an m-split: beta = m alpha)
 * with alpha = n_row_shards, beta = n_kv_shards, F = bytes_per_value.  Any out
 * pointer may be NULL.  Host only.  Errors: EINVAL.                              */
CASCADE_API int32_t cascade_comm_cost(int32_t n_row_shards, int32_t n_kv_shards, int32_t m_split_scheme,
                          int32_t bytes_per_value, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads,
                          int64_t seq_len, int64_t *stage_a_bytes, int64_t *stage_b_bytes, int64_t *rounds);

/* Equation 2 (Theoretical Costs): communication time of one layer under perfect
 * parallel transport, node bandwidth B (bytes/s) and inter-node latency tau (s):
 *   stage_a_s = tau + beta F d (H + 2 H_KV) / B * max_i |R_i|
 *   stage_b_s = tau + F (d + 2) H / B * max_j |S_j|
 *   total_s   = stage_a_s + stage_b_s
 * With a plan, beta = its key/value shard count and the two maxima are taken from its
 * partitions (n_kv_shards, max_row_shard, max_kv_shard are then ignored); with
 * plan == NULL the three are the caller's.  Out pointers are HOST doubles, any may be
 * NULL.  Host only.  Errors: EINVAL (non-positive sizes, negative or NaN latency,
 * bandwidth not above zero).                                                      */
CASCADE_API int32_t cascade_comm_time(const cascade_plan *plan, int32_t n_kv_shards, int32_t max_row_shard,
                          int32_t max_kv_shard, int32_t bytes_per_value, int32_t head_dim,
                          int32_t n_heads, int32_t n_kv_heads, double latency_s,
                          double bandwidth_bytes_per_s, double *stage_a_s, double *stage_b_s,
                          double *total_s);

CASCADE_API void cascade_plan_destroy(cascade_plan *plan);

/* Bytes of caller-owned workspace an entry point needs, by operation: desc points to
 * the descriptor type of that operation; flags is the layer count for
 * CASCADE_OP_LAYER_STACK and ignored otherwise.  Operations without a workspace
 * (shard GEMM, LSE merge, decode, norm) and invalid descriptors give 0.  The
 * per-operation queries below return the same numbers.                          */
#define CASCADE_OP_SHARD_GEMM     0   /* cascade_gemm_desc: no workspace               */
#define CASCADE_OP_PARTIAL_ATTN   1   /* cascade_attn_desc                             */
#define CASCADE_OP_LSE_MERGE      2   /* cascade_attn_desc: no workspace               */
#define CASCADE_OP_LAYER_FORWARD  3   /* cascade_layer_desc                            */
#define CASCADE_OP_LAYER_STACK    4   /* cascade_layer_desc, flags = n_layers          */
#define CASCADE_OP_LM_HEAD        5   /* cascade_lm_head_desc                          */
CASCADE_API size_t cascade_workspace_bytes(const cascade_plan *plan, const void *desc, int32_t op, int32_t flags);

/* HIP error code of the last CASCADE_EHIP on this thread (0 if none).          */
CASCADE_API int32_t cascade_last_hip_error(void);

/* ------------------------------------------------------------------ shard GEMM
 * The token-as-batch linear layers (Section 5 overview; Appendix C): for every
 * shard, Y[rows of the shard] = epilogue(X[rows of the shard] W^T).  Weights are
 * shared by all shards, so the groups are row-index lists; one launch covers
 * all shards.  rows must be batch * seq_len of the plan when any row map is
 * CASCADE_ROWS_ORIGINAL-to-packed (see x_rows / y_rows / res_rows).
 *
 * Row maps: the GEMM's own row r (0 <= r < rows) is a PACKED row.  With
 * x_rows = CASCADE_ROWS_ORIGINAL the kernel reads X row b*N + perm[r mod N]
 * (gather); with CASCADE_ROWS_PACKED it reads row r.  y_rows and res_rows do the
 * same for the store of Y (scatter) and the read of the residual.               */
typedef struct cascade_gemm_desc {
    int32_t dtype;      /* element type of X, W, W_up, bias, residual, Y             */
    int32_t rows;       /* M                                                          */
    int32_t k;          /* in_features                                                */
    int32_t n_out;      /* out_features = columns of Y                                */
    int32_t epilogue;   /* CASCADE_EPI_* mask; order: +bias, activation / swiglu,
                           rope, +residual                                            */
    int32_t x_rows;     /* CASCADE_ROWS_*                                             */
    int32_t y_rows;
    int32_t res_rows;
    int32_t rope_cols;  /* EPI_ROPE: columns [0, rope_cols) are rotated, in heads of
                           head_dim columns, half-split pairing (i, i + head_dim/2),
                           angle position * theta^(-2i/head_dim)                      */
    int32_t head_dim;
    float   rope_theta;
} cascade_gemm_desc;

/* X [rows, k]; W [n_out, k]; W_up [n_out, k] (EPI_SWIGLU only, else NULL);
 * bias [n_out] (EPI_BIAS; with SWIGLU unsupported); residual [rows, n_out];
 * Y [rows, n_out].  Y must not alias X.  Y may alias residual only when
 * y_rows == res_rows.
 * A call with the same arguments gives the same bits each time.  The bits of one row
 * may depend on the number of rows of the call: few rows take kernels that add the
 * products of k in another order (in fp32 still).  The same holds for the projections
 * of cascade_layer_forward; cascade_lm_head keeps one order whatever its rows.
 * Errors: EINVAL, ESHAPE (rows != batch*seq_len with a map), EUNSUPPORTED
 * (bf16 needs k % 8 == 0; rope needs head_dim even and rope_cols % head_dim == 0).*/
CASCADE_API int32_t cascade_shard_gemm(const cascade_plan *plan, const cascade_gemm_desc *desc,
                           const void *X, const void *W, const void *W_up, const void *bias,
                           const void *residual, void *Y, void *stream);

/* ------------------------------------------------------------------ attention
 * Strides are in elements; the head_dim axis is contiguous.  A stride of 0
 * means "dense [B, heads, N, d]".                                               */
typedef struct cascade_attn_desc {
    int32_t dtype;        /* of q, k, v and of o                                      */
    int32_t n_heads;      /* H                                                        */
    int32_t n_kv_heads;   /* H_KV, divides H; query head h reads kv head h/(H/H_KV)   */
    int32_t head_dim;     /* d: bf16 path 64 or 128; f32 path any d <= 256            */
    float   scale;        /* a = scale * q k^T + s                                    */
    int32_t row_layout;   /* rows of q, k, v (partial_attn) and of o (lse_merge)      */
    int32_t u_mode;       /* CASCADE_U_*                                              */
    int64_t q_stride_b, q_stride_h, q_stride_n;
    int64_t kv_stride_b, kv_stride_h, kv_stride_n;   /* shared by k and v             */
} cascade_attn_desc;

/* Bytes of workspace cascade_partial_attn needs (0 is possible).                */
CASCADE_API size_t cascade_partial_attn_workspace_bytes(const cascade_plan *plan, const cascade_attn_desc *desc);

/* Algorithm 3 for every pair (j, k).  Outputs are fp32 and in PACKED row order:
 *   m, e [B, H, n_shards, N]   m[b,h,k,r], e[b,h,k,r]: packed query row r against shard k
 *   u    [B, n_shards, H, N, d]
 * m is in the units of a (natural-log domain).  e and the unnormalised u refer to the
 * m that is stored, so m + log e does not depend on what the maximum was rounded to.
 * f32: a NaN score that a query sees makes its e and u NaN (m is the maximum of the
 * other scores); values of keys that a query does not see never reach its outputs.
 * Errors: EINVAL, ESHAPE (H % H_KV), EUNSUPPORTED (head_dim), EWORKSPACE.       */
CASCADE_API int32_t cascade_partial_attn(const cascade_plan *plan, const cascade_attn_desc *desc,
                             const void *q, const void *k, const void *v,
                             float *m, float *e, float *u,
                             void *workspace, size_t workspace_bytes, void *stream);

/* cascade_partial_attn for callers that cannot allocate device memory or hand over
 * a workspace: code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc.  Same arguments, results and errors as cascade_partial_attn
 * (bit-identical outputs: the same kernels run); the scratch memory of the bf16
 * kernels is a static device array of CASCADE_STATIC_SCRATCH_BYTES that every GPU
 * the library runs on holds until the process ends.  The call allocates nothing and
 * frees nothing.  A problem whose cascade_partial_attn_workspace_bytes exceeds
 * CASCADE_STATIC_SCRATCH_BYTES (36 MiB) is refused with CASCADE_EWORKSPACE.  The
 * bf16 kernels need 2 B H_KV d (N + N') bytes, N' = 64 x the number of 64-key
 * tiles of the key/value shards (N rounded up shard by shard); the limit covers
 * 8 kv heads of 128 at N = 8192 in 64-row-aligned shards.  fp32 needs none.
 * All calls on one GPU share that GPU's array: calls that overlap in time on the
 * same GPU (different streams or threads) race and must be serialised by the
 * caller.  Nothing in the array needs to start at zero; every call rewrites what
 * it reads.                                                                      */
#define CASCADE_STATIC_SCRATCH_BYTES (36u << 20)
CASCADE_API int32_t cascade_partial_attn_static(const cascade_plan *plan, const cascade_attn_desc *desc,
                                    const void *q, const void *k, const void *v,
                                    float *m, float *e, float *u, void *stream);

/* The merge of Algorithm 4 (Post-Pass): n = max_k m_k; w = sum_k exp(m_k - n) e_k;
 * o = sum_k exp(m_k - n) e_k u_k / w (u~ form: sum_k exp(m_k - n) u~_k / w).
 * o [B, N, H*d] in desc->dtype, rows per desc->row_layout; lse_out (optional,
 * may be NULL) [B, H, N] fp32 = n + log w, packed rows.                         */
CASCADE_API int32_t cascade_lse_merge(const cascade_plan *plan, const cascade_attn_desc *desc,
                          const float *m, const float *e, const float *u,
                          void *o, float *lse_out, void *stream);

/* ------------------------------------------------------------------ whole layer
 * Algorithm 1 on one GPU: h1 = h + o_proj(attention(norm1(h))),
 * h_out = h1 + FFN(norm2(h1)); pre-norm block.                                  */
/* Where the two norms of the block sit (the Pre-Pass subsection and the last step of
 * Algorithm 1 leave the block's internals to the model):
 *   PRE :  h1 = h + Attn(norm1(h));      out = h1 + MLP(norm2(h1))      (GPT / Llama)
 *   POST:  h1 = norm1(h + Attn(h));      out = norm2(h1 + MLP(h1))      (BERT, the
 *          model of the paper's timing runs; use a plan with CASCADE_MASK_NONE for
 *          its bidirectional attention)                                           */
#define CASCADE_NORM_PRE  0
#define CASCADE_NORM_POST 1

typedef struct cascade_layer_desc {
    int32_t dtype;
    int32_t d_model, n_heads, n_kv_heads, head_dim, d_ff;
    int32_t norm_kind;    /* CASCADE_NORM_LAYERNORM | CASCADE_NORM_RMSNORM            */
    float   norm_eps;
    int32_t act;          /* CASCADE_ACT_*                                            */
    int32_t rope;         /* 0: none, 1: half-split rotary on q and k                 */
    float   rope_theta;
    float   scale;
    int32_t attn_mode;    /* CASCADE_ATTN_*                                           */
    int32_t io_rows;      /* row order of h_in and h_out: CASCADE_ROWS_*              */
    int32_t norm_placement;   /* CASCADE_NORM_PRE (0) | CASCADE_NORM_POST             */
} cascade_layer_desc;

/* Device pointers, borrowed.  Matrices [out, in].  NULL = absent (biases, norm
 * biases, w_gate unless SWIGLU).                                                */
typedef struct cascade_layer_weights {
    const void *wq, *wk, *wv, *wo;          /* [H d, D] [Hkv d, D] [Hkv d, D] [D, H d] */
    const void *w_gate, *w_up, *w_down;     /* [f, D] [f, D] [D, f]                    */
    const void *bq, *bk, *bv, *bo, *b_up, *b_down;
    const void *norm1_g, *norm1_b, *norm2_g, *norm2_b;   /* [D]                        */
} cascade_layer_weights;

CASCADE_API size_t cascade_layer_workspace_bytes(const cascade_plan *plan, const cascade_layer_desc *desc);

/* h_in, h_out [B, N, D]; must not alias.
 * Errors: EINVAL, ESHAPE, EUNSUPPORTED, EWORKSPACE, EHIP.                       */
CASCADE_API int32_t cascade_layer_forward(const cascade_plan *plan, const cascade_layer_desc *desc,
                              const cascade_layer_weights *weights,
                              const void *h_in, void *h_out,
                              void *workspace, size_t workspace_bytes, void *stream);

/* n_layers consecutive layers with the same descriptor and one weight set each
 * (weights[0 .. n_layers-1]): the output of layer l is the input of layer l+1 on
 * the same rows (Single Layer Pipeline subsection).  Only the first layer gathers
 * h_in into packed order and only the last one scatters into h_out (both in
 * desc->io_rows order); between layers the activations stay packed, in two
 * buffers taken from the workspace (cascade_layer_stack_workspace_bytes).
 * h_in, h_out [B, N, D]; must not alias.  Errors as cascade_layer_forward.       */
CASCADE_API size_t cascade_layer_stack_workspace_bytes(const cascade_plan *plan, const cascade_layer_desc *desc,
                                           int32_t n_layers);
CASCADE_API int32_t cascade_layer_stack_forward(const cascade_plan *plan, const cascade_layer_desc *desc,
                                    const cascade_layer_weights *weights, int32_t n_layers,
                                    const void *h_in, void *h_out,
                                    void *workspace, size_t workspace_bytes, void *stream);

/* ---- LM head on sharded rows -------------------------------------------------
 * After the last layer every CompNode applies the LM head to its own hidden rows
 * and holds R_i-sharded logits; the CompNode that holds the last token turns its
 * logits row into the next token (Single Layer Pipeline subsection, the
 * paragraph after Algorithm 1).  logits = W_vocab . norm_f(h): the model's
 * closing normalisation, then the vocabulary projection as one shard GEMM over
 * the packed rows (weights shared by all shards).
 *
 * rows = CASCADE_LM_ALL_ROWS: logits [B, N, vocab] for every token, h_in rows in
 *   in_rows order, logits rows in out_rows order (CASCADE_ROWS_*).
 * rows = CASCADE_LM_LAST_ROW: logits [B, vocab] of the token with the largest
 *   position in each sequence (lowest index among equal positions); out_rows is
 *   ignored.
 * h_in [B, N, D], norm_gain [D], norm_bias [D] or NULL, w_vocab [vocab, D],
 * logits in desc->dtype: device pointers, borrowed.  workspace: device,
 * 256-byte aligned, cascade_lm_head_workspace_bytes (the normalised rows).
 * vocab % 4 == 0.  Errors: EINVAL, ESHAPE, EUNSUPPORTED, EWORKSPACE, EHIP.       */
#define CASCADE_LM_ALL_ROWS 0
#define CASCADE_LM_LAST_ROW 1

typedef struct cascade_lm_head_desc {
    int32_t dtype;
    int32_t d_model, vocab;
    int32_t norm_kind;    /* CASCADE_NORM_LAYERNORM | CASCADE_NORM_RMSNORM            */
    float   norm_eps;
    int32_t rows;         /* CASCADE_LM_ALL_ROWS | CASCADE_LM_LAST_ROW                */
    int32_t in_rows;      /* row order of h_in: CASCADE_ROWS_*                        */
    int32_t out_rows;     /* row order of the logits (ALL_ROWS): CASCADE_ROWS_*       */
} cascade_lm_head_desc;

CASCADE_API size_t cascade_lm_head_workspace_bytes(const cascade_plan *plan, const cascade_lm_head_desc *desc);
CASCADE_API int32_t cascade_lm_head(const cascade_plan *plan, const cascade_lm_head_desc *desc,
                        const void *h_in, const void *norm_gain, const void *norm_bias,
                        const void *w_vocab, void *logits,
                        void *workspace, size_t workspace_bytes, void *stream);

/* Greedy choice: token_out[r] (device int32 [rows]) = lowest index of the
 * largest of logits[r, 0 .. vocab) (device, [rows, vocab] in dtype).  NaNs never
 * win; a row of NaNs gives 0.  Errors: EINVAL, EUNSUPPORTED, EHIP.               */
CASCADE_API int32_t cascade_greedy_token(const void *logits, int32_t dtype, int32_t rows, int32_t vocab,
                             int32_t *token_out, void *stream);

/* The same computation with stage boundaries marked for measurement: HIP event
 * stage_events[i] (hipEvent_t, created by the caller, NULL entries skipped) is
 * recorded on the stream at boundary i.  Boundaries (CASCADE_N_STAGE_EVENTS):
 * 0 start, 1 gather+norm1, 2 qkv GEMM, 3 rotary (same instant as 2 when the
 * rotation ran in the GEMM's epilogue: bf16 pre-norm layers), 4 attention (partial
 * attention), 5 LSE merge (same instant as 4 in FUSED mode), 6 o projection +
 * residual (and norm2 when a split reduction ends in one row kernel), 7 norm2, 8 FFN up/gate GEMM, 9 FFN down + residual + scatter.       */
#define CASCADE_N_STAGE_EVENTS 10
CASCADE_API int32_t cascade_layer_forward_staged(const cascade_plan *plan, const cascade_layer_desc *desc,
                                     const cascade_layer_weights *weights,
                                     const void *h_in, void *h_out,
                                     void *workspace, size_t workspace_bytes, void *stream,
                                     void *const *stage_events, int32_t n_stage_events);

/* After a MATERIALISED cascade_layer_forward: device pointers into the workspace
 * it used, holding m, e [B,H,n_shards,N] and u~ [B,n_shards,H,N,d] (fp32).      */
CASCADE_API int32_t cascade_layer_partials(const cascade_plan *plan, const cascade_layer_desc *desc,
                               void *workspace, float **m, float **e, float **u);

/* After a cascade_layer_forward (either attention mode): device pointer into the
 * workspace it used, to the merged attention output o [B * N, H * d] in desc->dtype,
 * PACKED rows (the input of the o projection; Algorithm 4 before its last step).
 * Exposed so that the fused path can be checked at the same point as
 * cascade_lse_merge's output.  Errors: EINVAL, EUNSUPPORTED.                     */
CASCADE_API int32_t cascade_layer_attention_output(const cascade_plan *plan, const cascade_layer_desc *desc,
                                       void *workspace, void **o);

/* ------------------------------------------------------------------ KV-cache decode
 * Cost Optimizations appendix ("Caching"): in single-token generation only the
 * newest token's query row is attended, by AttnNode_jk for every kv shard k,
 * against the keys and values of S_k cached so far (the new token's own k, v
 * already appended to its shard by the caller).  One partial per shard:
 *   m, e [B, H, n_shards]        (= [B, H, n_shards, 1] of cascade_partial_attn)
 *   u    [B, n_shards, H, d]     fp32, CASCADE_U_* as in desc->u_mode
 * which cascade_lse_merge combines when called with a plan of seq_len 1 and the
 * same n_shards (cascade_plan_create(batch, 1, n_shards, {j}, ...)).
 *   q [B, H, d]; k_cache, v_cache [B, H_KV, n_shards, shard_capacity, d] (dense,
 *   desc->dtype, 16-byte aligned); shard_len_dev [B, n_shards] int32 DEVICE:
 *   rows of each shard that are valid (clamped to shard_capacity; 0 gives
 *   m = -inf, e = 0, u = 0).  No mask: every cached key is at or before the new
 *   position.  From desc: dtype, n_heads, n_kv_heads, head_dim, scale, u_mode
 *   (row_layout and strides are ignored).  head_dim must be 8 * 2^j (bf16) or
 *   4 * 2^j (f32), at most 512 / 256.
 * Errors: EINVAL, ESHAPE (H % H_KV), EUNSUPPORTED (head_dim, alignment), EHIP.   */
CASCADE_API int32_t cascade_decode_partial_attn(const cascade_attn_desc *desc, int32_t batch, int32_t n_shards,
                                    int32_t shard_capacity, const int32_t *shard_len_dev,
                                    const void *q, const void *k_cache, const void *v_cache,
                                    float *m, float *e, float *u, void *stream);

/* Normalisation of `rows` rows of D values (the optional normalisation step of
 * the Pre-Pass subsection, exposed for callers that compose a
 * single-token step themselves): y = norm(x) * gain (+ bias), statistics in
 * fp32.  x, y [rows, D], gain [D], bias [D] or NULL: device, dtype; x == y allowed.
 * Errors: EINVAL, EUNSUPPORTED, EHIP.                                            */
CASCADE_API int32_t cascade_norm(int32_t dtype, int32_t rows, int32_t d_model, int32_t norm_kind, float eps,
                     const void *x, const void *gain, const void *bias, void *y, void *stream);

/* Token-sharded KV cache from a prefill ("Caching": every AttnNode_jk keeps the
 * k, v of its shard S_k between tokens).  Copies the keys (rotary embedding
 * already applied) and values that the last cascade_layer_forward /
 * cascade_layer_stack_forward call with this plan and descriptor left in
 * `workspace` into the slabs cascade_decode_partial_attn reads:
 *   k_cache, v_cache [B, H_KV, n_kv_shards, shard_capacity, d] in desc->dtype;
 *   row r of kv shard k (ascending token index inside the shard) goes to slab
 *   row r; slab rows past the shard's size are left untouched.
 *   shard_len_dev [B, n_kv_shards] int32 DEVICE receives the shard sizes.
 * shard_capacity must hold the largest shard (ESHAPE otherwise).  The workspace
 * must not have been reused since that forward call.
 * Errors: EINVAL, ESHAPE, EUNSUPPORTED, EHIP.                                    */
CASCADE_API int32_t cascade_layer_kv_to_cache(const cascade_plan *plan, const cascade_layer_desc *desc,
                                  const void *workspace, void *k_cache, void *v_cache,
                                  int32_t shard_capacity, int32_t *shard_len_dev, void *stream);

/* ------------------------------------------------------------------ rotary positions
 * The rotation of EPI_ROPE as an operator of its own (queries and keys of a paged cache, whose
 * positions differ from row to row), with the variants that models use.  The first rot_dim
 * columns of every head are turned in rot_dim / 2 pairs (a, b), the rest is passed on:
 *   (a, b) -> amplitude * (a cos - b sin, a sin + b cos),  angle = position * f_i
 *   f_i = theta^(-2i / rot_dim), i < rot_dim / 2
 *   ROPE_LINEAR: f_i / factor
 *   ROPE_RAMP:   f_i ((1 - g) / factor + g), g = clamp((r - low) / (high - low), 0, 1),
 *                r = original_len * f_i / (2 pi): turns that pair i makes over original_len
 * Angles are formed in 64 bits, so that they hold at every int32 position; a negative
 * position turns back.                                                            */
#define CASCADE_ROPE_HALF        0 /* pairs (i, i + rot_dim / 2)                       */
#define CASCADE_ROPE_INTERLEAVED 1 /* pairs (2i, 2i + 1)                               */
#define CASCADE_ROPE_UNSCALED 0
#define CASCADE_ROPE_LINEAR   1
#define CASCADE_ROPE_RAMP     2

typedef struct cascade_rope_desc {
    int32_t layout;       /* CASCADE_ROPE_HALF | CASCADE_ROPE_INTERLEAVED             */
    int32_t rot_dim;      /* even, 2 .. 512, at most the head dimension               */
    int32_t scaling;      /* CASCADE_ROPE_UNSCALED | _LINEAR | _RAMP                  */
    int32_t original_len; /* ROPE_RAMP: above 0                                       */
    double  theta;        /* above 0                                                  */
    double  factor;       /* ROPE_LINEAR, ROPE_RAMP: above 0                          */
    double  low, high;    /* ROPE_RAMP: low < high                                    */
    double  amplitude;    /* of the rotated columns (1: a rotation)                   */
} cascade_rope_desc;

/* x, y: rows of n_heads * head_dim elements, x_stride / y_stride elements apart (0:
 * dense); positions_dev [rows] int32.  y may be x (with the same stride); otherwise
 * they must not overlap.  Errors: EINVAL, ESHAPE (strides below a row, rot_dim above
 * head_dim, y == x with another stride), EUNSUPPORTED (dtype, rot_dim), EHIP.       */
CASCADE_API int32_t cascade_rope(const cascade_rope_desc *desc, int32_t dtype, int32_t rows, int32_t n_heads,
                     int32_t head_dim, const int32_t *positions_dev, const void *x, int64_t x_stride, void *y,
                     int64_t y_stride, void *stream);

/* ------------------------------------------------------------------ paged cache
 * The token-sharded cache of cascade_decode_partial_attn in pages instead of slabs:
 * sequences grow by any number of tokens at a time, share what they have in common,
 * and hold no memory that they do not use.  Every (sequence, key/value shard) pair has
 * a list of pages; row r of shard s (ascending token index inside the shard) lies in
 * page page_table[sequence][s][r / page_size] at row r % page_size.  A page is free if
 * its page_refs is 0.  Only pages whose rows are all in use are ever shared
 * (page_refs above 1): rows are only written behind the end of a list, in a page that
 * list holds alone.  One set of lists serves the pools of all layers.  After the caller
 * has set them up (all lists -1, lengths and references 0), lists, lengths and references
 * are changed by the calls below alone: a list that is cut short from outside keeps pages
 * that the next extension would lose, and may end in one that others share.
 * The descriptor is read during the call; what it points to belongs to the caller.
 * Calls look at all n_seqs sequences, those without new rows too, and attention takes n_seqs for how many have rows
 * when it chooses a kernel.  A descriptor of neighbouring sequences alone (page_table and kv_len moved to the first
 * of them, n_seqs their number) serves every call but cascade_pages_compact, which has to know all lists.
 * Page ids and lengths are read on the device: an id outside [0, n_pages) holds no
 * keys (they are skipped like masked ones), lengths count up to max_pages * page_size. */
typedef struct cascade_paged_cache {
    int32_t dtype;
    int32_t n_layers, n_pages;
    int32_t n_kv_heads, head_dim;     /* head_dim: a multiple of 8 (bf16) or 4 (f32), at most 256 */
    int32_t page_size;                /* rows: a power of two, 16 .. 65536             */
    int32_t n_seqs, n_shards;         /* n_shards: at most 1024; rows of the pools: 31
                                         bits; rows of a list: at most 2^31 - 65; entries
                                         of page_table: at most 2^31 - 4097            */
    int32_t max_pages;                /* of a list                                     */
    void *k_pages, *v_pages;          /* [n_layers, n_pages, H_KV, page_size, d], 16-byte aligned */
    int32_t *page_table;              /* [n_seqs, n_shards, max_pages]; unused entries -1 */
    int32_t *kv_len;                  /* [n_seqs, n_shards] rows                       */
    int32_t *page_refs;               /* [n_pages]                                     */
} cascade_paged_cache;

/* Room for new rows, once per step and before the layers' cascade_paged_append.  The
 * rows of all sequences lie back to back: those of sequence b are q_start_dev[b] ..
 * q_start_dev[b + 1] (q_start_dev [n_seqs + 1], ascending; a sequence may have none).
 * row_shard_dev [rows]: key/value shard of each row (NULL: one shard only).  Pages are
 * taken lowest id first, list by list.  Outputs (device, int32):
 *   slots [rows]              page * page_size + row of the page; -1: row not stored
 *   visible [rows, n_shards]  rows of shard s at or before this row, itself included:
 *                             the causal limit of cascade_paged_attn
 *   accepted [n_seqs]         0: the sequence did not fit (no free page, list full) and
 *                             is as it was, its rows have slot -1 and see nothing
 * and kv_len, page_table, page_refs are brought up to date.  Once a sequence finds no
 * free page, later ones that need one are refused too.  Rows behind the last sequence
 * (a padded batch) have slot -1 and see nothing; so does a row whose shard id is outside
 * [0, n_shards), but it sees what its neighbours see.
 * Errors: EINVAL, EUNSUPPORTED (sizes above, rows above 2^31 - 1025), EHIP.                                 */
CASCADE_API int32_t cascade_paged_extend(const cascade_paged_cache *cache, int32_t rows, const int32_t *q_start_dev,
                             const int32_t *row_shard_dev, int32_t *slots, int32_t *visible, int32_t *accepted,
                             void *stream);

/* Writes the keys and values of `rows` new rows into their slots in layer `layer`'s
 * pages.  k, v: rows of H_KV * d elements, kv_stride apart (0: dense).  With `rope` the
 * keys are rotated on the way (positions_dev [rows]), and so are n_heads queries per row
 * from q to q_out if q is given (rows of n_heads * d elements; q_out may be q with the
 * same stride).  Without `rope`, positions_dev and q are NULL.  A row whose slot is
 * outside [0, n_pages * page_size) is not stored (its queries are rotated all the same);
 * no slot may be named twice.
 * Errors: EINVAL, ESHAPE (strides, rot_dim above head_dim, layer), EUNSUPPORTED, EHIP. */
CASCADE_API int32_t cascade_paged_append(const cascade_paged_cache *cache, int32_t layer, int32_t rows,
                             const int32_t *slots_dev, const void *k, const void *v, int64_t kv_stride,
                             const cascade_rope_desc *rope, const int32_t *positions_dev, int32_t n_heads,
                             const void *q, int64_t q_stride, void *q_out, int64_t q_out_stride, void *stream);

/* Attention of the new rows over the cached keys of their sequence, the partials of all
 * key/value shards merged (Algorithms 3 and 4 on the rows at hand): one token per
 * sequence, a chunk of a prompt, or both at once.  Row t of sequence b, which are the
 * rows q_start_dev[b] .. q_start_dev[b + 1], sees the rows j < visible_dev[t][s] of
 * shard s (at most kv_len of them); visible_dev [rows, n_shards], as
 * cascade_paged_extend writes it.  NULL: all kv_len rows, without a mask (a bidirectional
 * chunk, or cross attention to cached states).  Query head h reads kv head
 * h / (n_heads / H_KV).
 *   o [rows, n_heads * d] in o_dtype; lse [n_heads, rows] fp32 = log sum exp(a) (NULL:
 *   not wanted).  A row that sees nothing: o = 0, lse = -inf.  Rows behind the last
 *   sequence are left as they were.  What a row does not see never reaches it, be it
 *   NaN.  With o in fp32, (lse, 1, o) is a partial that cascade_lse_merge takes
 *   (CASCADE_U_NORMALISED), where other parties hold more shards.
 * q, o 16-byte aligned, strides in elements (0: dense) and multiples of 16 bytes; o must
 * not overlap q.  Calls that may overlap in time need a workspace each (16-byte aligned);
 * its contents need not be kept between calls.  Two sequences must not share rows.
 * Over a bf16 cache the weights enter the product with the values in 16 bits; where a sequence has more than 256 rows
 * times heads of a kv head (head dimensions 64 and 128), rounded to bf16.
 * A call with the same arguments gives the same bits each time; those of a row may depend
 * on the other rows and lengths of the call, which decide how the work is cut.
 * Errors: EINVAL, ESHAPE (n_heads % H_KV, strides, layer), EUNSUPPORTED (alignment,
 * sizes), EWORKSPACE, EHIP.                                                         */
typedef struct cascade_paged_attn_desc {
    int32_t rows, n_heads;
    float   scale;
    int32_t o_dtype;      /* the cache's, or CASCADE_F32                              */
    int64_t q_stride, o_stride;
} cascade_paged_attn_desc;

CASCADE_API size_t cascade_paged_attn_workspace_bytes(const cascade_paged_cache *cache, const cascade_paged_attn_desc *desc);
CASCADE_API int32_t cascade_paged_attn(const cascade_paged_cache *cache, int32_t layer, const cascade_paged_attn_desc *desc,
                           const int32_t *q_start_dev, const int32_t *visible_dev, const void *q, void *o, float *lse,
                           void *workspace, size_t workspace_bytes, void *stream);

/* Pages of finished or dropped sequences: every list of the n sequences seqs_dev [n]
 * becomes empty and its pages lose one reference each.  Ids outside [0, n_seqs) are
 * skipped, one named twice is freed once.  Errors: EINVAL, EUNSUPPORTED, EHIP.      */
CASCADE_API int32_t cascade_pages_free(const cascade_paged_cache *cache, int32_t n, const int32_t *seqs_dev, void *stream);

/* Branches: sequence dst_dev[i] becomes a copy of src_dev[i], i < n.  Full pages are
 * shared; a last page that is partly filled is copied, its used rows in every layer, into
 * the lowest free page.  accepted [n] (device): 0 where a pair was refused and changed
 * nothing: an id out of range, a destination that is not empty or that an earlier pair
 * names too, or no free page (for every later pair that needs one as well).  Sources are
 * taken as they were before the call.  n * n_shards at most 8192.
 * Errors: EINVAL, EUNSUPPORTED, EWORKSPACE, EHIP.                                   */
CASCADE_API size_t cascade_pages_workspace_bytes(const cascade_paged_cache *cache);
CASCADE_API int32_t cascade_pages_fork(const cascade_paged_cache *cache, int32_t n, const int32_t *src_dev,
                           const int32_t *dst_dev, int32_t *accepted, void *workspace, size_t workspace_bytes, void *stream);

/* Moves the pages in use to the front of the pools: afterwards they are 0 .. n_live - 1
 * (n_live: device int32, may be NULL).  Pages behind that move, in ascending order, to
 * the free ones before it; the lists follow.
 * Errors: EINVAL, EUNSUPPORTED, EWORKSPACE, EHIP.                                   */
CASCADE_API int32_t cascade_pages_compact(const cascade_paged_cache *cache, int32_t *n_live, void *workspace,
                              size_t workspace_bytes, void *stream);

/* Copies page src_dev[i] onto page dst_dev[i] in every layer, i < n; pairs with an id
 * outside [0, n_pages) are skipped.  No page may be a destination twice, nor a source
 * and another pair's destination.  Lists and references stay.
 * Errors: EINVAL, EUNSUPPORTED, EHIP.                                               */
CASCADE_API int32_t cascade_pages_copy(const cascade_paged_cache *cache, int32_t n, const int32_t *src_dev,
                           const int32_t *dst_dev, void *stream);

/* ------------------------------------------------------------------ measured ceiling
 * Not a step of the method: the rate (TFLOP/s) this device sustains on back-to-back
 * bf16 16x16x32 MFMAs with random operands, for the roofline figures quoted next
 * to the datasheet peak.  lds_operands = 0: operands stay in registers;
 * 1: operands are re-read from LDS at the shard GEMM's ratio (12 16-byte reads per
 * 32 MFMAs).  One workgroup of 8 wavefronts per compute unit, `iters` (1..2^22)
 * iterations of 32 MFMAs each; runs twice on `stream`, synchronises, and reports
 * the second run.  tflops_out is a HOST pointer.  Allocates 256 bytes of device
 * memory for the duration of the call.  Errors: EINVAL, EHIP.                    */
CASCADE_API int32_t cascade_mfma_ceiling(int32_t lds_operands, int32_t iters, float *tflops_out, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* CASCADE_H */

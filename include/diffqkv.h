/*
 * diffqkv.h -- C ABI of libdiffqkv: DiffQKV attention over a KV cache on NVIDIA B200 (sm_100a).
 *
 * DiffQKV attention (paper Section 2, "Formulation of DiffQKV Attention") is softmax
 * attention in which Q, K and V have their own head counts n_q, n_k, n_v.  Query head h
 * reads K head  hk = floor(h * n_k / n_q)  and V head  hv = floor(h * n_v / n_q)
 * (Section 3.2, Eq. (idx); n_k and n_v must divide n_q, so hk = h / (n_q/n_k)).  For one
 * query vector q_h and the visible cached tokens j:
 *
 *     s_j = scale * <q_h, K[j, hk]>          m = max_j s_j
 *     p_j = exp(s_j - m)                     l = sum_j p_j
 *     out_h = (sum_j p_j * V[j, hv]) / l     lse_h = m + log(l)
 *
 * K and V live in two separate pools (Section 3.1: the key cache and the value cache have
 * different shapes), streamed once per call; that traffic, b*s*(n_k*d_k + n_v*d_v) elements
 * (Eq. (cache_0)), is what bounds decoding.
 *
 * General rules for every call
 *   - Every pointer in the argument lists and structs is a DEVICE pointer unless it is marked
 *     "host".  The structs themselves (diffqkv_cache, diffqkv_shape) are read on the host.
 *   - The library borrows all buffers, owns nothing and, unless an entry point says otherwise,
 *     allocates nothing: scratch memory is a caller-provided workspace.
 *   - Calls enqueue work on `stream` (a cudaStream_t passed as void*) and return without
 *     synchronising.  Buffers must stay valid until the stream has run the work.
 *   - Errors the host can see (null pointers, head counts that do not divide, unsupported head
 *     dimensions, misaligned pointers, a workspace that is too small, a failed launch) return a
 *     status and launch nothing.  Conditions only the device can see (a page id outside the
 *     pool, a bounded wait that ran out) OR the bit (1 << diffqkv_status value) into *dev_status
 *     (when given) and the affected block skips that work; nothing traps.
 *   - Tensors are dense in their last (channel) dimension.  bf16 tensors must be 16-byte
 *     aligned with strides that are multiples of 8 elements; fp32 tensors 16-byte aligned with
 *     strides that are multiples of 4 elements.
 */
#ifndef DIFFQKV_H_
#define DIFFQKV_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  DIFFQKV_OK = 0,
  DIFFQKV_ERR_INVALID_ARG = 1, /* null pointer, non-positive size, n_k or n_v not dividing n_q ... */
  DIFFQKV_ERR_UNSUPPORTED = 2, /* a shape or dtype no kernel covers                                */
  DIFFQKV_ERR_ALIGNMENT = 3,   /* a pointer or stride violates the alignment rules above           */
  DIFFQKV_ERR_WORKSPACE = 4,   /* workspace missing or smaller than the *_workspace_bytes answer   */
  DIFFQKV_ERR_CUDA = 5,        /* a CUDA runtime or driver call failed                             */
  DIFFQKV_ERR_TIMEOUT = 6,     /* device: a bounded wait on a copy ran out                         */
  DIFFQKV_ERR_INDEX = 7,       /* device: page id outside [0, num_blocks)                          */
  DIFFQKV_ERR_PAGES = 8        /* device: a sequence was denied pages because the pool has too few */
} diffqkv_status;

typedef enum { DIFFQKV_BF16 = 0, DIFFQKV_F32 = 1 } diffqkv_dtype;

/*
 * The KV cache: two pools addressed through the same rule.  Token j of sequence b, head hd,
 * channel c of the K pool sits at element offset
 *     blk * k_stride_blk + hd * k_stride_head + slot * k_stride_tok + c
 * with (blk, slot) = (b, j) for a contiguous cache (page_table == NULL) and
 * (blk, slot) = (page_table[b * max_pages_per_seq + j / page_size], j % page_size) for a paged
 * one; likewise for V.  One page table serves both pools.  The paper fixes only the logical
 * shapes (b, s, n_h, d_h) (Section 3.1); strides make head-major and token-major storage
 * both expressible, and the page format is this library's own.
 */
typedef struct {
  void *k_cache;             /* K pool, element type = shape.dtype                                  */
  void *v_cache;             /* V pool                                                              */
  int64_t k_stride_blk, k_stride_head, k_stride_tok; /* in elements                                 */
  int64_t v_stride_blk, v_stride_head, v_stride_tok;
  const int32_t *seqlens;    /* [batch] visible tokens per sequence (decode: includes the new one)  */
  const int32_t *page_table; /* [batch, max_pages_per_seq] physical page ids, or NULL = contiguous  */
  int32_t page_size;         /* tokens per page (paged only; a multiple of 16 for the TMA kernels)  */
  int32_t max_pages_per_seq; /* row length of page_table                                            */
  int32_t num_blocks;        /* extent of the blk dimension: pages in the pool, or batch            */
  int32_t max_seqlen;        /* host-known upper bound of seqlens[]; contiguous: also the token     */
                             /* extent of each (blk, head) slab, so reads never pass it             */
} diffqkv_cache;

typedef struct {
  int32_t batch, n_q, n_k, n_v; /* n_q % n_k == 0 and n_q % n_v == 0                                */
  int32_t d_qk, d_v;            /* channels per head of Q/K and of V                                */
  diffqkv_dtype dtype;          /* storage type of q, K and V; accumulation is always fp32          */
  diffqkv_dtype out_dtype;      /* storage type of `out`                                            */
  float scale;                  /* multiplies the inner product; the paper uses 1/sqrt(d_k)         */
} diffqkv_shape;

/*
 * Split planning for decode (Section 3.2: the split kernel divides K and V into chunks along
 * the sequence).  The sequence axis is cut into chunks of one fixed length; sequence b uses
 * ceil(seqlens[b] / chunk) of the at most S splits.
 *   diffqkv_decode_num_splits: S the library would choose for num_splits = 0 (always >= 1).
 *   diffqkv_decode_workspace_bytes: bytes of workspace diffqkv_decode / gqa_decode need for
 *   this shape, max_seqlen and num_splits (0 = the automatic choice).  Returns 0 on bad input.
 */
int32_t diffqkv_decode_num_splits(const diffqkv_shape *shape, int32_t max_seqlen);
size_t diffqkv_decode_workspace_bytes(const diffqkv_shape *shape, int32_t max_seqlen, int32_t num_splits);

/*
 * diffqkv_decode -- one query token per sequence against the cache (Section 2 formulation with
 * the head map of Eq. (idx); split-sequence execution per Section 3.2).
 *   q          [batch, n_q, d_qk]  shape.dtype, contiguous
 *   cache      see diffqkv_cache; seqlens[b] == 0 gives out = 0 and lse = -inf for that sequence
 *   num_splits 0 = automatic (recommended): bf16 caches that a TMA tensor map can describe use the
 *              persistent TMA kernel, which divides all (sequence, head group, 64-token tile) work
 *              evenly over one block per SM and cuts sequences wherever a block's share ends; other
 *              inputs use fixed chunks.  > 0 = fixed chunks, at most that many per sequence (generic kernel);
 *              more than 8192 returns DIFFQKV_ERR_UNSUPPORTED
 *   workspace  at least diffqkv_decode_workspace_bytes(...) bytes, 256-byte aligned; holds the
 *              per-split partial outputs (fp32 [batch, n_q, S, d_v]) and log-sum-exps
 *              (fp32 [batch, n_q, S]); contents on entry are ignored
 *   out        [batch, n_q, d_v]   shape.out_dtype
 *   lse        [batch, n_q] fp32 natural-log log-sum-exp of the scaled scores, or NULL
 *   dev_status one int32 the kernels OR (1 << diffqkv_status) bits into, or NULL; the caller zeroes it
 * Runs the split kernel and then the combine kernel on `stream`.  With few, short rows (the blocks that share a
 * (sequence, head group) row fill at least 0.85 of the SMs as clusters of 2 to 8 and the cache's capacity for them is
 * small enough that the idle SMs cost less than a second launch) the TMA kernel's blocks of a row form a thread-block
 * cluster and merge on chip instead: one launch, the workspace is not used.
 */
diffqkv_status diffqkv_decode(const void *q, const diffqkv_cache *cache, const diffqkv_shape *shape,
                              int32_t num_splits, void *workspace, size_t workspace_bytes, void *out,
                              float *lse, int32_t *dev_status, void *stream);

/*
 * diffqkv_decode_host -- diffqkv_decode for a query that sits in host memory and a result that is wanted there (the
 * paper has no counterpart; the KV cache is decode state and stays on the device).  On `stream`, in order: copy
 * q_host -> q_dev, diffqkv_decode(q_dev ... out_dev), copy out_dev -> out_host.  Nothing is synchronised: the result
 * is in out_host once the stream has run the last copy.
 *   q_host, out_host  HOST pointers ([batch, n_q, d_qk] shape.dtype and [batch, n_q, d_v] shape.out_dtype);
 *                     page-locked memory keeps the copies asynchronous
 *   q_dev, out_dev    device staging buffers of the same sizes, provided by the caller (the library allocates nothing)
 *   everything else as in diffqkv_decode
 */
diffqkv_status diffqkv_decode_host(const void *q_host, void *q_dev, const diffqkv_cache *cache,
                                   const diffqkv_shape *shape, int32_t num_splits, void *workspace,
                                   size_t workspace_bytes, void *out_dev, void *out_host, float *lse,
                                   int32_t *dev_status, void *stream);

/*
 * diffqkv_decode_static -- diffqkv_decode for callers that cannot provide or allocate a workspace.
 * (The paper has no counterpart; this is a deployment convenience of this library.)
 * Some hosts cannot call cudaMalloc when they decode: all device memory already belongs to their own
 * pool, or they sit behind an interface with no workspace argument, or an allocation would stall a
 * latency-critical loop.  For them the split kernel's partial results go to a fixed 8 MiB array built
 * into the library (each GPU that loads the library carries those 8 MiB until the process exits).
 * Arguments and results are those of diffqkv_decode without `workspace` / `workspace_bytes`.
 *   - Returns DIFFQKV_ERR_WORKSPACE, launching nothing, when
 *     diffqkv_decode_workspace_bytes(shape, cache->max_seqlen, num_splits) exceeds 8 MiB (8388608 bytes);
 *     choose fewer splits or a smaller batch, or use diffqkv_decode with your own buffer.
 *   - Calls no cudaMalloc / cudaFree and no allocating library routine.
 *   - The first call on each device resolves the array's device address (the device of `stream` must be
 *     the current device); make that first call outside any stream capture.
 *   - All calls on one device share the one array: two calls whose kernels may overlap on the GPU
 *     (different streams without ordering, or several host threads) race on it.  Calls on one stream
 *     are safe.  The array keeps the previous call's partials; nothing in it needs clearing because a
 *     call reads only what it has itself written.
 */
diffqkv_status diffqkv_decode_static(const void *q, const diffqkv_cache *cache, const diffqkv_shape *shape,
                                     int32_t num_splits, void *out, float *lse, int32_t *dev_status,
                                     void *stream);

/*
 * gqa_decode -- grouped-query attention, the comparison point of the paper (Appendix B.1: GQA is
 * the special case n_k == n_v).  Same arguments and the same kernels as diffqkv_decode; returns
 * DIFFQKV_ERR_INVALID_ARG when shape.n_k != shape.n_v.
 */
diffqkv_status gqa_decode(const void *q, const diffqkv_cache *cache, const diffqkv_shape *shape,
                          int32_t num_splits, void *workspace, size_t workspace_bytes, void *out,
                          float *lse, int32_t *dev_status, void *stream);

/*
 * diffqkv_combine -- merge per-split partial results (Section 3.2: the combine kernel assembles
 * the output chunks).  With o_s the NORMALISED output of split s and lse_s its log-sum-exp:
 *     lse = log sum_s exp(lse_s),   out = sum_s exp(lse_s - lse) * o_s,
 * splits with lse_s == -inf are skipped; if all are, out = 0 and lse = -inf.
 *   o_partial   [rows, S, d_v] fp32     lse_partial [rows, S] fp32     (rows = batch * n_q)
 *   out         [rows, d_v] out_dtype   lse [rows] fp32 or NULL
 */
diffqkv_status diffqkv_combine(const float *o_partial, const float *lse_partial, int32_t batch, int32_t n_q,
                               int32_t d_v, int32_t num_splits, diffqkv_dtype out_dtype, void *out,
                               float *lse, void *stream);

/*
 * diffqkv_prefill -- causal attention for q_len new tokens per sequence, writing their K and V
 * rows into the cache first (appendix attention listing: cache update, then the causal
 * flash-attention call; head map of Eq. (idx)).
 *   q      [batch, q_len, n_q, d_qk]   k_new [batch, q_len, n_k, d_qk]   v_new [batch, q_len, n_v, d_v]
 *   cache  seqlens[b] = tokens already cached (past_b) on entry; rows past_b .. past_b + q_len - 1 of
 *          both pools are overwritten; seqlens itself is not modified (the caller adds q_len)
 *   out    [batch, q_len, n_q, d_v] out_dtype; query row i sees tokens 0 .. past_b + i
 *   lse    [batch, q_len, n_q] fp32 or NULL
 * bf16 with (d_qk, d_v) = (128, 128), (64, 64) or (64, 128), a positive scale and pages of at least 8 tokens that
 * divide or are multiples of 128 runs on the tensor cores; every other shape diffqkv_decode accepts (fp32, other head
 * dimensions, scale <= 0) runs the same two steps on a plain fp32-FMA kernel, one block per query row, which is a
 * correctness path, not a fast one.
 */
diffqkv_status diffqkv_prefill(const void *q, const void *k_new, const void *v_new, int32_t q_len,
                               const diffqkv_cache *cache, const diffqkv_shape *shape, void *out, float *lse,
                               int32_t *dev_status, void *stream);

/*
 * diffqkv_augq -- the augmented-Q projection that produces the queries (Section 2, Observation 3;
 * appendix attention listing: q_proj followed by q_down_proj(act(q_gate_proj(x)) * q_up_proj(x))).
 * act is read as SiLU, there are no biases, and weights use the nn.Linear layout [out, in]:
 *     x = h W_Q^T,   a = silu(x W_gate^T) * (x W_up^T),   q = a W_down^T
 *   h [T, d_model]   W_Q [d_q0, d_model]   W_gate, W_up [d_aug, d_q0]   W_down [d_out, d_aug]   all bf16
 *   workspace  diffqkv_augq_workspace_bytes(T, d_q0, d_aug) bytes, 256-byte aligned, for x and a
 *   q_out [T, d_out] bf16
 *   dev_status as in diffqkv_decode, or NULL
 * Products accumulate in fp32 on the tensor cores; x and a are rounded to bf16 once each (they are the next
 * product's bf16 operands).  All dimensions must be multiples of 128 except T; T == 0 does nothing.
 */
size_t diffqkv_augq_workspace_bytes(int64_t T, int32_t d_q0, int32_t d_aug);
diffqkv_status diffqkv_augq(const void *h, const void *W_Q, const void *W_gate, const void *W_up,
                            const void *W_down, int64_t T, int32_t d_model, int32_t d_q0, int32_t d_aug,
                            int32_t d_out, void *workspace, size_t workspace_bytes, void *q_out,
                            int32_t *dev_status, void *stream);

/*
 * diffqkv_augq_rope -- diffqkv_augq followed by the rotary position embedding of the appendix attention listing
 * (apply_rotary_pos_emb on the query), fused into the last product's epilogue: the rotation acts on the fp32
 * result before it is rounded to bf16.  The listing only names the call; it is read as the rotate-half pairing:
 * within a head of width head_dim, channel i < head_dim/2 pairs with channel i + head_dim/2,
 *     y_i = x_i cos[t, i] - x_{i+head_dim/2} sin[t, i],   y_{i+head_dim/2} = x_{i+head_dim/2} cos[t, i] + x_i sin[t, i].
 *   cos, sin  [T, head_dim / 2] fp32 tables of the caller (angle of pair i at position pos: pos * theta^(-2 i / head_dim));
 *             both NULL = no rotation
 *   head_dim  64 or 128; d_out must be a multiple of it
 * Everything else as diffqkv_augq.
 */
diffqkv_status diffqkv_augq_rope(const void *h, const void *W_Q, const void *W_gate, const void *W_up,
                                 const void *W_down, int64_t T, int32_t d_model, int32_t d_q0, int32_t d_aug,
                                 int32_t d_out, int32_t head_dim, const float *cos, const float *sin, void *workspace,
                                 size_t workspace_bytes, void *q_out, int32_t *dev_status, void *stream);

/*
 * diffqkv_project -- a plain projection of the attention listing (k_proj, v_proj): y = x W^T with W in the
 * nn.Linear layout [d_out, d_in], no bias, on the tensor cores with fp32 accumulation; with cos / sin given, the
 * rotary embedding above is applied per head before rounding (the key projection), without them it is a plain
 * product (the value projection).
 *   x [T, d_in] bf16   W [d_out, d_in] bf16   y [T, d_out] bf16   d_in and d_out multiples of 128
 * The result [T, n_heads, head_dim] is the k_new / v_new layout of diffqkv_prefill and diffqkv_cache_append.
 */
diffqkv_status diffqkv_project(const void *x, const void *W, int64_t T, int32_t d_in, int32_t d_out, int32_t head_dim,
                               const float *cos, const float *sin, void *y, int32_t *dev_status, void *stream);

/*
 * diffqkv_cache_append -- the cache update of the attention listing on its own (diffqkv_prefill does the same
 * before it attends): k_new [batch, q_len, n_k, d_qk] and v_new [batch, q_len, n_v, d_v] are written to token
 * positions seqlens[b] .. seqlens[b] + q_len - 1 of the pools (any strides, paged or contiguous, bf16 or fp32).
 * seqlens itself is not modified.  Positions at or past max_seqlen, and page ids outside the pool, are skipped
 * and reported as DIFFQKV_ERR_INDEX in *dev_status.  A decode step is: append the new token's rows, add 1 to
 * seqlens, call diffqkv_decode.
 */
diffqkv_status diffqkv_cache_append(const void *k_new, const void *v_new, int32_t q_len, const diffqkv_cache *cache,
                                    const diffqkv_shape *shape, int32_t *dev_status, void *stream);

/*
 * diffqkv_decode_frontend -- everything one decode step computes from the hidden states before it attends
 * (appendix attention listing: q_proj and the augmented-Q chain, k_proj, v_proj, rotary embedding, cache update), for
 * one new token per sequence:
 *     q_out[b] = rope(aug-Q(h[b]))                      as diffqkv_augq_rope with T = batch rows
 *     K cache row at position seqlens[b]  = rope(h[b] W_K^T)     V cache row at seqlens[b] = h[b] W_V^T
 *   h [batch, d_model] bf16; W_Q [n_q d_qk, d_model], W_gate, W_up [d_aug, n_q d_qk], W_down [n_q d_qk, d_aug],
 *   W_K [n_k d_qk, d_model], W_V [n_v d_v, d_model], all bf16 in the nn.Linear layout
 *   cos, sin   [batch, d_qk / 2] fp32 tables of the new tokens' positions, or both NULL for no rotation
 *   cache      bf16 pools; seqlens[b] = tokens already cached; seqlens is not modified (the caller adds 1 and calls
 *              diffqkv_decode with q_out); positions at or past max_seqlen and page ids outside the pool are
 *              reported as DIFFQKV_ERR_INDEX in *dev_status and skipped
 *   workspace  diffqkv_decode_frontend_workspace_bytes(shape, d_aug) bytes, 256-byte aligned
 *   q_out      [batch, n_q, d_qk] bf16
 * With at most 64 sequences this is three launches (the products of h share one, which writes k and v straight into
 * the cache); with more it is the separate steps of diffqkv_augq_rope, diffqkv_project and diffqkv_cache_append.
 * d_model, d_aug and n_q d_qk must be multiples of 128, n_k d_qk and n_v d_v multiples of 16 (of 128 beyond 64
 * sequences), d_qk 64 or 128 when rotating.
 */
size_t diffqkv_decode_frontend_workspace_bytes(const diffqkv_shape *shape, int32_t d_aug);
diffqkv_status diffqkv_decode_frontend(const void *h, const void *W_Q, const void *W_gate, const void *W_up,
                                       const void *W_down, const void *W_K, const void *W_V, int32_t d_model,
                                       int32_t d_aug, const float *cos, const float *sin, const diffqkv_cache *cache,
                                       const diffqkv_shape *shape, void *workspace, size_t workspace_bytes,
                                       void *q_out, int32_t *dev_status, void *stream);

/*
 * diffqkv_fold_k_up -- queries for a K cache that is stored at a smaller head width than the queries (Section 2:
 * when the Q and K head dimensions differ, Attend first transforms K to the query width through another feed-forward
 * layer; Observation 2 and its table: d_k = d_v / 2).  The layer is read as linear, without bias, one matrix per K
 * head.  Since <q_h, W[hk] k_j> = <W[hk]^T q_h, k_j>, widening every cached key is replaced by folding the layer
 * into the query once:
 *     q_out[t, h, :] = W_kup[hk]^T q[t, h, :],   hk = floor(h * n_k / n_q)
 *   q      [T, n_q, d_q] bf16      W_kup [n_k, d_q, d_k] bf16      q_out [T, n_q, d_k] bf16 (fp32 accumulation)
 * Call sequence for the half-width cache: diffqkv_fold_k_up, then diffqkv_decode / diffqkv_prefill /
 * diffqkv_decode_topk with shape.d_qk = d_k (64 with d_v = 128 runs on the TMA and tensor-core kernels) and the
 * same scale the full-width scores would use.  Runs on the tensor cores when d_q is a multiple of 16 up to 256, d_k
 * is 32, 64 or 128 and not above d_q, and the three pointers are 16-byte aligned; every other shape takes a plain
 * kernel, for which (n_q / n_k) * d_q may not exceed 3072 and d_q must be a multiple of 4 (DIFFQKV_ERR_UNSUPPORTED
 * otherwise).
 */
diffqkv_status diffqkv_fold_k_up(const void *q, const void *W_kup, int64_t T, int32_t n_q, int32_t n_k, int32_t d_q,
                                 int32_t d_k, void *q_out, void *stream);

/*
 * diffqkv_decode_topk -- decode with selective V cache fetching (paper Section "Selective V Cache Fetching"; its
 * table uses the 100 highest scores): every query head scores all cached tokens of its K head, keeps the `topk`
 * highest scores (equal scores: the earlier token), takes the softmax over the kept scores only (the paper does
 * not say whether the weights are renormalised; read as renormalised) and sums the kept V rows.  The K cache is
 * streamed once, of the V cache only topk rows per query head are read.  A sequence with at most topk tokens gives
 * exactly the full attention of diffqkv_decode.
 *   q, cache, out, lse, dev_status as in diffqkv_decode; bf16 only, d_qk 64 or 128, at most 32 query heads per
 *   K head, 1 <= topk <= 1024, d_v a multiple of 8 with 16-byte aligned V rows, pages of 16, 32, 64 or a multiple
 *   of 128 tokens; topk times the number of 32768-token pieces of max_seqlen may not exceed 8192
 *   (DIFFQKV_ERR_UNSUPPORTED otherwise)
 *   workspace  diffqkv_decode_topk_workspace_bytes(shape, cache->max_seqlen, topk) bytes, 256-byte aligned: the fp32
 *              scores [batch, n_q, max_seqlen rounded up to 128] and the largest score of every 16 consecutive tokens
 */
size_t diffqkv_decode_topk_workspace_bytes(const diffqkv_shape *shape, int32_t max_seqlen, int32_t topk);
diffqkv_status diffqkv_decode_topk(const void *q, const diffqkv_cache *cache, const diffqkv_shape *shape, int32_t topk,
                                   void *workspace, size_t workspace_bytes, void *out, float *lse,
                                   int32_t *dev_status, void *stream);
/*
 * diffqkv_decode_topk_ids -- the same, and also says which tokens were kept (for callers that audit the selection or
 * reuse it for a later step):
 *   kept_ids  int32 [batch, n_q, topk]: the cached positions of the tokens whose V rows entered the output of each
 *             query head, in no particular order, padded with -1 when the sequence has fewer than topk tokens; NULL
 *             makes the call identical to diffqkv_decode_topk
 */
diffqkv_status diffqkv_decode_topk_ids(const void *q, const diffqkv_cache *cache, const diffqkv_shape *shape,
                                       int32_t topk, void *workspace, size_t workspace_bytes, void *out, float *lse,
                                       int32_t *kept_ids, int32_t *dev_status, void *stream);

/* ------------------------------------------------------------------------------------------------------------------
 * Ragged batches over the paged cache: what an engine step with sequences at different stages needs (some decode one
 * token, some verify a few, some work off a long prompt in chunks).  The paper stops at one attention call; these
 * entry points are this library's own.  All of them describe the step by the same two arrays: the new rows of
 * sequence b are rows cu_q[b] .. cu_q[b + 1] - 1 of every ragged tensor (n_b = cu_q[b + 1] - cu_q[b], which may be 0),
 * and seqlens[b] = past_b is the number of tokens cached BEFORE the step (diffqkv_prefill's convention, not
 * diffqkv_decode's), so that one pair of arrays serves every layer:
 *     diffqkv_pages_reserve -> per layer: diffqkv_rope_append, diffqkv_extend -> the caller adds n_b to seqlens[b]
 *   cu_q     [batch + 1] int32, cu_q[0] = 0, not decreasing, cu_q[batch] <= total_q
 *   total_q  rows the ragged tensors hold; rows from cu_q[batch] on are not written and what they hold does not matter,
 *            so a step of fixed capacity can be captured into a graph and replayed with other lengths
 * A sequence whose rows do not fit (past_b + n_b > max_seqlen, a negative past_b, rows beyond total_q, an end before its
 * beginning) is reported as DIFFQKV_ERR_INDEX in *dev_status and skipped; rows and cache positions that are its alone stay
 * as they were.  Once cu_q decreases, sequences that still fit may be left out as well, and a row or cache position that it
 * gives to several holds any one's result.
 * ------------------------------------------------------------------------------------------------------------------ */

/*
 * diffqkv_extend -- causal attention of ragged chunks of new tokens over the cache (Section 2 formulation, head map of
 * Eq. (idx)).  Row i of sequence b sits at position past_b + i and sees tokens 0 .. past_b + i; the chunk's own K and V
 * rows are in the cache already (diffqkv_rope_append, diffqkv_cache_append or diffqkv_decode_frontend wrote them).
 *   q     [total_q, n_q, d_qk] shape.dtype
 *   out   [total_q, n_q, d_v]  shape.out_dtype         lse [total_q, n_q] fp32 natural log, or NULL
 *   shape.batch sequences; cache, scale, dev_status as in diffqkv_prefill
 *   workspace  diffqkv_extend_workspace_bytes(shape, total_q) bytes, 256-byte aligned; contents on entry are ignored.
 *              Two calls that may run at the same time (streams without an order, graphs replayed side by side) need
 *              a workspace each.
 * bf16 with (d_qk, d_v) = (128, 128), (64, 64) or (64, 128), a positive scale and pages of 8 to 64 tokens (a power of
 * two) or a multiple of 128 runs on the tensor cores, chunks of a few rows and long ones on a kernel each; everything else
 * diffqkv_decode accepts runs on fp32 FMAs.  Results do not depend on how sequences are batched beyond rounding (fp32
 * sums in another order, weights rounded to bf16 relative to another reference), and are bitwise reproducible from call
 * to call.  The launches do not depend on what the step holds: three on the tensor cores (two where so many query heads
 * share both heads that no chunk is short), one or two on FMAs.  A step known to have one row for every sequence is
 * faster through diffqkv_decode (whose seqlens count the new token).
 * Scores are formed in fp32 in units of log 2, so that one of more than 2.35e38 counts as infinite.  A row whose scores are
 * all -inf has out = 0 and lse = -inf; a NaN or +inf among them makes both NaN.
 * As in any tensor-core attention a weight of zero multiplies the V rows of later tokens of the same chunk; those rows
 * must be finite.  What lies behind the last cached token in its page may hold anything.
 */
size_t diffqkv_extend_workspace_bytes(const diffqkv_shape *shape, int32_t total_q);
diffqkv_status diffqkv_extend(const void *q, const int32_t *cu_q, int32_t total_q, const diffqkv_cache *cache,
                              const diffqkv_shape *shape, void *workspace, size_t workspace_bytes, void *out, float *lse,
                              int32_t *dev_status, void *stream);

/*
 * diffqkv_extend_window -- diffqkv_extend for a layer with a sliding window and a few first tokens that stay visible: row i
 * of sequence b, at position p = past_b + i, sees the tokens j <= p with j > p - window or j < sinks.
 *   window  >= 1: tokens of the window, the row's own among them       sinks  >= 0: first tokens that every row sees
 *   workspace  diffqkv_extend_window_workspace_bytes(shape, total_q) bytes, 256-byte aligned
 * Everything else as diffqkv_extend.  Work and traffic go by the tokens seen, not by the tokens cached.  Three launches on
 * the tensor cores, two where total_q is so small that no sequence can have many rows.  Pages that hold no token which a row
 * of the step sees are not read: they may have been given back, and their table entries may be -1.  (Positions go on
 * counting; diffqkv_pages_free gives back ends, not middles, so a caller who frees pages behind the window lowers their
 * counts and sets their entries itself; such a sequence is forked, freed and compacted like any other.)  A weight of zero
 * multiplies the V rows of tokens that another row of the same chunk sees; those must be finite, all others may hold
 * anything.
 * A window that reaches back over the whole cache (window + sinks >= max_seqlen) gives what diffqkv_extend gives beyond
 * rounding.  With a cu_q that decreases anywhere the whole step may be left out.
 */
size_t diffqkv_extend_window_workspace_bytes(const diffqkv_shape *shape, int32_t total_q);
diffqkv_status diffqkv_extend_window(const void *q, const int32_t *cu_q, int32_t total_q, int32_t window, int32_t sinks,
                                     const diffqkv_cache *cache, const diffqkv_shape *shape, void *workspace,
                                     size_t workspace_bytes, void *out, float *lse, int32_t *dev_status, void *stream);

/*
 * diffqkv_extend_shared -- diffqkv_extend for sequences that share their first tokens (samples of one prompt, requests behind
 * one instruction; diffqkv_pages_fork makes such sequences): the K and V of a shared prefix are read once for the rows of all
 * sequences of its group and joined with what each sequence has behind it,
 *     out = (2^a o_prefix + 2^b o_own) / (2^a + 2^b),   a, b the base-2 log-sum-exps of the two parts.
 * The result is that of diffqkv_extend beyond rounding.  The sequences of a group are neighbours in the batch.
 */
typedef struct {
  const int32_t *cu_seqs; /* [num_groups + 1] device, not decreasing: group g is the sequences cu_seqs[g] .. cu_seqs[g + 1] - 1 */
  const int32_t *lens;    /* [num_groups] device: tokens that the sequences of group g share, any number from 0 on               */
  int32_t num_groups;     /* at most 65535; sequences in front of the first group and behind the last share nothing              */
} diffqkv_prefixes;
/*
 *   prefixes   every sequence of a group that has rows in the step has at least lens[g] tokens cached, in its own pages (or
 *              slab) as for diffqkv_extend; those of all sequences of a group are the same, usually the same pages.  A shared
 *              prefix is read from the group's FIRST sequence, which may have no rows itself; where that one holds fewer than
 *              lens[g] tokens (it has been given up), and where sharing would save nothing (short prefixes, long chunks, one
 *              sequence alone with rows), every sequence reads its own.  A sequence whose group does not fit it (a prefix longer than its
 *              cache or than max_seqlen, or negative, an end of the group outside the batch, rows outside the group's) is
 *              reported as DIFFQKV_ERR_INDEX and skipped.
 *   workspace  diffqkv_extend_shared_workspace_bytes(shape, total_q) bytes, 256-byte aligned (it holds both parts of every
 *              row in fp32)
 * Everything else as diffqkv_extend.  Launches as diffqkv_extend_window; where diffqkv_extend runs on FMAs (fp32, page sizes and
 * heads that the tensor cores do not take) every sequence reads all of its own tokens.  With a cu_q or a cu_seqs that decreases
 * anywhere the whole step may be left out.  Two calls that may run at the same time need a workspace each.
 * It is for steps of many sequences with a few rows each behind a long prefix; steps of long chunks alone, which gain little or
 * nothing, usually take less time with diffqkv_extend.
 */
size_t diffqkv_extend_shared_workspace_bytes(const diffqkv_shape *shape, int32_t total_q);
diffqkv_status diffqkv_extend_shared(const void *q, const int32_t *cu_q, int32_t total_q, const diffqkv_prefixes *prefixes,
                                     const diffqkv_cache *cache, const diffqkv_shape *shape, void *workspace,
                                     size_t workspace_bytes, void *out, float *lse, int32_t *dev_status, void *stream);

/*
 * Rotary positions.  Channel pairs of the first rot_dim channels of every q and k head are turned by the angle
 * pos * inv_freq[i]; the other channels pass through:
 *     (y_a, y_b) = magnitude * (x_a cos - x_b sin, x_b cos + x_a sin),   pair i = (i, i + rot_dim / 2), or
 *     (2 i, 2 i + 1) when interleaved
 * The angle is formed and reduced to one turn in fp64 (in fp32 a position of 10^5 would already cost 8e-3 of a turn's
 * radian), the turn itself is fp32, each result is rounded once to the storage type.
 */
typedef struct {
  const double *inv_freq;   /* [rot_dim / 2] device, radians per position                                  */
  const int32_t *positions; /* [total_q] device, or NULL: row i of sequence b is at position past_b + i    */
  int32_t rot_dim;          /* 0 (no rotation) to d_qk, a multiple of 16 (bf16) or 8 (fp32)                */
  int32_t interleaved;      /* 0 = rotate-half pairs, 1 = neighbouring pairs                               */
  float magnitude;          /* multiplies the rotated channels; 1 except for diffqkv_rope_frequencies YARN */
} diffqkv_rope;

/*
 * diffqkv_rope_frequencies -- the table of inverse frequencies, on the HOST (nothing is launched), f_i = theta^(-2 i /
 * rot_dim) and its adaptations to contexts longer than the trained length L = original_length, factor s >= 1:
 *   PLAIN   f_i
 *   LINEAR  f_i / s (position interpolation)
 *   NTK     theta replaced by theta * s^(rot_dim / (rot_dim - 2))
 *   YARN    f_i (1 - g_i) + f_i / s * g_i with g_i = clamp((i - lo) / (hi - lo), 0, 1), lo = floor(c(fast)),
 *           hi = ceil(c(slow)), both kept within 0 .. rot_dim - 1, c(r) = rot_dim ln(L / (2 pi r)) / (2 ln theta);
 *           magnitude = 0.1 ln s + 1
 *   BANDS   wavelengths 2 pi / f_i below L / fast keep f_i, above L / slow take f_i / s, and in between
 *           (1 - t) f_i / s + t f_i with t = (L f_i / (2 pi) - slow) / (fast - slow)
 *   inv_freq  HOST [rot_dim / 2] fp64      magnitude  HOST, or NULL
 */
typedef enum {
  DIFFQKV_ROPE_PLAIN = 0,
  DIFFQKV_ROPE_LINEAR = 1,
  DIFFQKV_ROPE_NTK = 2,
  DIFFQKV_ROPE_YARN = 3,
  DIFFQKV_ROPE_BANDS = 4
} diffqkv_rope_scaling;
diffqkv_status diffqkv_rope_frequencies(int32_t rot_dim, double theta, diffqkv_rope_scaling scaling, double factor,
                                        double original_length, double fast, double slow, double *inv_freq,
                                        float *magnitude);

/*
 * diffqkv_rope_append -- rotates the q and k rows of a ragged step and writes k and v to positions past_b + i of the
 * cache, in one launch (diffqkv_cache_append for ragged chunks, with the rotation of the appendix attention listing).
 *   q      [total_q, n_q, d_qk], or NULL for keys and values alone      q_out  [total_q, n_q, d_qk] dense; may be q
 *   k_new  [total_q, n_k, d_qk]      v_new  [total_q, n_v, d_v]      all of shape.dtype, heads dense within a row
 *   *_stride_tok  elements between rows (slices of a fused projection); 0 = dense.  q_out == q needs a dense q.
 * The rotation moves with `positions`, the place in the cache does not.  Positions whose page id lies outside the
 * pool are skipped and reported as DIFFQKV_ERR_INDEX.
 */
diffqkv_status diffqkv_rope_append(const void *q, const void *k_new, const void *v_new, const int32_t *cu_q,
                                   int32_t total_q, int64_t q_stride_tok, int64_t k_stride_tok, int64_t v_stride_tok,
                                   const diffqkv_rope *rope, const diffqkv_cache *cache, const diffqkv_shape *shape,
                                   void *q_out, int32_t *dev_status, void *stream);

/*
 * diffqkv_norm_rope_append -- diffqkv_rope_append behind a root-mean-square norm of every q and k head, in the same launch:
 *     x <- x / sqrt(mean_c x_c^2 + eps) * (weight_offset + w_c)      over the d_qk channels of a head
 * and then the rotation, all in fp32, rounded once.  Squares are summed in fp32: a head's sum of squares has to stay below 3.4e38
 * (channels below 1.8e19 / sqrt(d_qk), 2e17 for 8192 of them) and, with eps = 0, its root mean square above 1e-18; with eps = 0 a
 * head of zeros is NaN.
 *   q_weight, k_weight   [d_qk], or one for each head ([n_q, d_qk], [n_k, d_qk]) with a head stride of d_qk; NULL = all zero
 *                        where weight_offset is not 0, all one where it is
 *   *_head_stride        elements between the weights of two heads: 0 (one for all heads) or a multiple of 16 bytes, >= d_qk;
 *                        not used beside a weight that is NULL
 * Everything else as diffqkv_rope_append (rot_dim 0 = norm and cache write alone).
 */
typedef struct {
  const void *q_weight, *k_weight;          /* device, 16-byte aligned                                     */
  int64_t q_head_stride, k_head_stride;
  diffqkv_dtype weight_dtype;               /* shape.dtype, or DIFFQKV_F32                                 */
  float eps;                                /* >= 0                                                        */
  float weight_offset;                      /* 0, or 1 for weights that are stored as their difference to 1 */
} diffqkv_qk_norm;
diffqkv_status diffqkv_norm_rope_append(const void *q, const void *k_new, const void *v_new, const int32_t *cu_q,
                                        int32_t total_q, int64_t q_stride_tok, int64_t k_stride_tok, int64_t v_stride_tok,
                                        const diffqkv_qk_norm *norm, const diffqkv_rope *rope, const diffqkv_cache *cache,
                                        const diffqkv_shape *shape, void *q_out, int32_t *dev_status, void *stream);

/*
 * Upkeep of the pages.  A page is a block of both pools (one id for K and V, as in diffqkv_cache).  The state is three
 * device arrays of the caller: the page table, the lengths, and the number of table entries that name each page.
 * Entry -1 (or any negative one) means no page; a sequence's pages fill its row from the front.  A page whose count is 0 is free, and free
 * pages are always handed out lowest id first, in the order of the sequences, so every call is deterministic.  Counts
 * may also be raised by the caller (a prefix that is kept pinned).  No call synchronises or tells the host anything:
 * a serving loop can run them inside a captured step.
 * Sequence ids outside [0, num_seqs) and page ids outside [0, num_pages) are reported as DIFFQKV_ERR_INDEX, skipped.
 * At most 65535 sequences and 2^20 pages; more are refused with DIFFQKV_ERR_UNSUPPORTED.
 */
typedef struct {
  int32_t *page_table; /* [num_seqs, max_pages_per_seq]                              */
  int32_t *seqlens;    /* [num_seqs] tokens cached                                   */
  int32_t *ref_counts; /* [num_pages] table entries (and pins) that name the page    */
  int32_t num_seqs, max_pages_per_seq, num_pages, page_size;
} diffqkv_pages;

/*
 * diffqkv_pages_free -- gives back the pages of n sequences behind their first keep_tokens[i] tokens (NULL: all of
 * them): entries become -1, counts go down by one, seqlens = min(seqlens, keep).  A sequence may be listed twice.
 */
diffqkv_status diffqkv_pages_free(const int32_t *seq_ids, const int32_t *keep_tokens, int32_t n,
                                  const diffqkv_pages *pages, int32_t *dev_status, void *stream);

/*
 * diffqkv_pages_fork -- children[i] becomes a copy of parents[i] that shares its pages (no token is copied): what the
 * child held is given back, its row names the pages of the parent's seqlens tokens, its length is the parent's.  All
 * parents are read as they were before the call, so a child may be a parent too (beams that change places) or its own.
 * A sequence that is listed as a child twice takes the first of its parents; the others are reported as
 * DIFFQKV_ERR_INDEX.
 *   workspace  diffqkv_pages_fork_workspace_bytes(pages, n) bytes, 256-byte aligned
 */
size_t diffqkv_pages_fork_workspace_bytes(const diffqkv_pages *pages, int32_t n);
diffqkv_status diffqkv_pages_fork(const int32_t *parents, const int32_t *children, int32_t n, const diffqkv_pages *pages,
                                  void *workspace, size_t workspace_bytes, int32_t *dev_status, void *stream);

/*
 * diffqkv_pages_reserve -- makes the cache writable for the step's rows: sequence b gets a page of its own for every
 * position past_b .. past_b + n_b - 1.  Missing pages are taken from the free ones; pages that another holder shares
 * (count > 1 at the start of the call) are replaced, and where past_b lies inside such a page its contents are copied
 * to the new one (copy on write).  If all holders of a page write in the same call each gets a copy.
 * A sequence gets all it needs or nothing: b is denied when the demands of sequences 0 .. b together exceed the free
 * pages (DIFFQKV_ERR_PAGES), or its rows do not fit or its table row is too short (DIFFQKV_ERR_INDEX).  The rows of a
 * denied sequence must not be written in this step: pages of its that others share are as they were, and missing ones are
 * missing.  A step that cannot ask the host (a captured one) gives diffqkv_rope_append and diffqkv_extend a seqlens array of
 * its own with -1 where granted is 0: they skip such a sequence and report it.
 *   cache, shape  the pools (pointers, strides, num_blocks = pages->num_pages); shape gives n_k, n_v, d_qk, d_v, dtype;
 *                 cache->page_table and cache->seqlens are not used; max_seqlen that of the calls which write the rows
 *                 (0 = the table rows' length alone).  total_q is not known here: rows beyond it are theirs to skip
 *   granted       [num_seqs] int32: 1 = its rows may be written, 0 = denied; or NULL
 *   workspace     diffqkv_pages_reserve_workspace_bytes(pages) bytes, 256-byte aligned
 */
size_t diffqkv_pages_reserve_workspace_bytes(const diffqkv_pages *pages);
diffqkv_status diffqkv_pages_reserve(const int32_t *cu_q, const diffqkv_pages *pages, const diffqkv_cache *cache,
                                     const diffqkv_shape *shape, int32_t *granted, void *workspace,
                                     size_t workspace_bytes, int32_t *dev_status, void *stream);

/*
 * diffqkv_pages_copy -- pages src_ids[i] of `src` become pages dst_ids[i] of `dst`, K and V (the same cache, or two
 * with equal page_size whose strides may differ: moving a sequence to another pool).  Within one cache no page may be
 * both a source and a destination, and no destination may be listed twice.  Tables and counts are not touched.
 */
diffqkv_status diffqkv_pages_copy(const int32_t *src_ids, const int32_t *dst_ids, int32_t n, const diffqkv_cache *src,
                                  const diffqkv_cache *dst, const diffqkv_shape *shape, int32_t *dev_status,
                                  void *stream);

/*
 * diffqkv_pages_compact -- moves the pages in use to the front of the pool: with `live` of them in use, the i-th lowest
 * page in use with an id >= live moves to the i-th lowest free id below live; everything else stays.  Afterwards
 * exactly the ids 0 .. live - 1 are in use.  Only the page table is told: a page held by a pin alone moves too, so a prefix
 * that is kept for later should be kept as a sequence (diffqkv_pages_fork to a spare row) where pools are compacted.
 *   table_out, refs_out  the new page table and counts; may be pages->page_table / ref_counts themselves.  Where they
 *                        are other buffers the old ones stay valid for readers already enqueued: a moved page keeps
 *                        its contents at its old id until that id is handed out again
 *   live                 one int32 that receives the number of pages in use, or NULL
 *   workspace            diffqkv_pages_compact_workspace_bytes(pages) bytes, 256-byte aligned
 */
size_t diffqkv_pages_compact_workspace_bytes(const diffqkv_pages *pages);
diffqkv_status diffqkv_pages_compact(const diffqkv_pages *pages, const diffqkv_cache *cache, const diffqkv_shape *shape,
                                     int32_t *table_out, int32_t *refs_out, int32_t *live, void *workspace,
                                     size_t workspace_bytes, int32_t *dev_status, void *stream);

/* Static, never-null description of a status value. */
const char *diffqkv_status_string(diffqkv_status status);

/*
 * Tuning hook (process-wide host state) for the TMA decode kernel's tail balance.  Every persistent block holds the
 * last few 64-token tiles of its share in a reserve that it and the other blocks working on the same (sequence, head
 * group) draw from one tile at a time, so that a block that runs ahead takes over tiles of one that runs behind.
 * Which block ends up with which tile depends on timing, so results can differ between runs in the last bits
 * (fp32 summation order); everything stays within the stated tolerances.
 *   tiles < 0  automatic (default): up to 8 tiles per block, at most a sixth of a block's share
 *   tiles = 0  no reserve: every tile has a fixed owner and results are bitwise reproducible from run to run
 *   tiles > 0  exactly that many (always leaving each segment one tile of its own); for tests
 * Workspace sizes do not depend on it.
 */
void diffqkv_set_tail_reserve(int32_t tiles);

#ifdef __cplusplus
}
#endif
#endif /* DIFFQKV_H_ */

// Shared device/host helpers of libdiffqkv (CUDA side only; the CPU oracle shares nothing with this).
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "diffqkv.h"

namespace diffqkv {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Host-side decode plan: the sequence axis is cut into chunks of `chunk` tokens (a multiple of
// kChunkQuantum); sequence b uses ceil(len_b / chunk) of the `splits` partial slots.
constexpr int kChunkQuantum = 64;
struct DecodePlan {
  int chunk;
  int splits;
};
DecodePlan plan_decode(const diffqkv_shape& shape, int max_seqlen, int num_splits);

struct CacheView {  // device copy of the addressing part of diffqkv_cache
  const void* k;
  const void* v;
  long long k_sb, k_sh, k_st;
  long long v_sb, v_sh, v_st;
  const int* seqlens;
  const int* page_table;
  int page_size, max_pages_per_seq, num_blocks, max_seqlen;
};

struct DecodeParams {
  const void* q;
  CacheView cache;
  int batch, n_q, n_k, n_v, d_qk, d_v;
  float scale_log2;  // scale * log2(e): scores are kept in the base-2 domain
  int chunk, splits;
  float* o_partial;    // [batch, n_q, splits, d_v]
  float* lse_partial;  // [batch, n_q, splits]   natural log
  int* dev_status;
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void store_out(float* p, float x) { *p = x; }
__device__ __forceinline__ void store_out(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// Device-side conditions are reported as bit (1 << diffqkv_status) so that several can coexist.
__device__ __forceinline__ void report(int* dev_status, int code) {
  if (dev_status) atomicOr(dev_status, 1 << code);
}

// Ragged steps: rows of sequence b (first row, number) and tokens cached before; false, with none of either, when they do
// not fit.
__device__ __forceinline__ bool ragged_rows(const int* cu_q, const int* seqlens, int b, int total_q, int max_seqlen, int& lo,
                                            int& n, int& past) {
  lo = cu_q[b];
  const int hi = cu_q[b + 1];
  past = seqlens[b];
  if (lo < 0 || hi < lo || hi > total_q || past < 0 || (long long)past + (hi - lo) > max_seqlen) {
    n = 0;
    past = 0;
    return false;
  }
  n = hi - lo;
  return true;
}
// The first sequence that fits and has row t between its ends, looked for by the whole block; -1 = none.  Not inlined: it is
// seldom called, and its registers are the caller's otherwise.
static __device__ __noinline__ int ragged_search(const int* cu_q, const int* seqlens, int batch, int total_q, int max_seqlen,
                                                 int t) {
  __shared__ int found_s;
  if (threadIdx.x == 0) found_s = batch;
  __syncthreads();
  for (int x = threadIdx.x; x < batch; x += blockDim.x) {
    int lo, n, past;
    if (ragged_rows(cu_q, seqlens, x, total_q, max_seqlen, lo, n, past) && lo <= t && t < lo + n) atomicMin(&found_s, x);
  }
  __syncthreads();
  return found_s < batch ? found_s : -1;
}
// The sequence that row t belongs to, with its rows, for a block of kThreads threads; -1 = none that fits.  With ends in order
// it is the number of ends at or below the row; only where that one does not have the row are all looked at, and `again` is
// called (for values of the caller's that then need not be kept meanwhile).  One block of a launch reports the sequences
// that do not fit (`report_all`).  Holds barriers.
template <int kThreads, typename F>
__device__ __forceinline__ int ragged_sequence_of(const int* cu_q, const int* seqlens, int batch, int total_q, int max_seqlen,
                                                  int t, bool report_all, int* dev_status, int& lo, int& n, int& past,
                                                  F again) {
  int b = 0;
  for (int b0 = 0; b0 < batch; b0 += kThreads) {
    const int x = b0 + (int)threadIdx.x;
    if (report_all && x < batch && !ragged_rows(cu_q, seqlens, x, total_q, max_seqlen, lo, n, past))
      report(dev_status, DIFFQKV_ERR_INDEX);
    b += __syncthreads_count(x < batch && cu_q[x + 1] <= t);
  }
  if (b >= batch) return -1;  // every end is at or below the row
  if (!ragged_rows(cu_q, seqlens, b, total_q, max_seqlen, lo, n, past) || t < lo || t >= lo + n) {
    b = ragged_search(cu_q, seqlens, batch, total_q, max_seqlen, t);
    if (b < 0) return -1;
    ragged_rows(cu_q, seqlens, b, total_q, max_seqlen, lo, n, past);
    again();
  }
  return b;
}

// Launchers (defined next to their kernels).
cudaError_t launch_decode_generic(const DecodeParams& p, diffqkv_dtype dtype, cudaStream_t stream);
cudaError_t launch_prefill_generic(const DecodeParams& p, diffqkv_dtype dtype, int q_len, void* out, int out_is_f32,
                                   float* lse, cudaStream_t stream);
cudaError_t launch_combine(const float* o_partial, const float* lse_partial, int rows, int d_v, int splits,
                           diffqkv_dtype out_dtype, void* out, float* lse, cudaStream_t stream);
void count_launch(int n = 1);
void set_decode_per_head_only(int on);  // test hook: the generic decode never takes the unit kernel

// Linear layers for at most kSkinnyMaxRows rows of x (weight-streaming kernel, linear_skinny.cu); same operands as the
// tensor-core GEMM of augq.cu: C[M, N] = A[M, K] . B0[N, K]^T, with B1 silu(A.B0^T) * (A.B1^T), with rope_cos/rope_sin
// the rotate-half rotary embedding per head of head_dim channels.
constexpr int kSkinnyMaxRows = 64;
void set_force_tensor_gemm(int on);
cudaError_t launch_qkv_skinny(const void* h, const void* W_Q, void* x, int d_q0, const void* W_K, const void* W_V,
                              long long M, int K, const float* rope_cos, const float* rope_sin, const CacheView& cache,
                              int n_k, int n_v, int d_qk, int d_v, int* dev_status, cudaStream_t stream);
// Everything a decode step computes from the hidden states h [batch, d_model]: q_out = rope(aug-Q(h)), and the new
// token's k = rope(h W_K^T), v = h W_V^T written into the cache at position seqlens[b] (augq.cu).
size_t decode_frontend_workspace_bytes(const diffqkv_shape& s, int d_aug);
cudaError_t launch_decode_frontend(const void* h, const void* W_Q, const void* W_gate, const void* W_up,
                                   const void* W_down, const void* W_K, const void* W_V, int d_model, int d_aug,
                                   const float* rope_cos, const float* rope_sin, const diffqkv_cache& c,
                                   const CacheView& view, const diffqkv_shape& s, void* workspace, void* q_out,
                                   int* dev_status, cudaStream_t stream);
bool linear_skinny_supported(long long M, int N, int K, bool dual, int head_dim, bool rotary);
cudaError_t launch_linear_skinny(const void* A, const void* B0, const void* B1, void* C, long long M, int N, int K,
                                 int* dev_status, cudaStream_t stream, const float* rope_cos, const float* rope_sin,
                                 int head_dim);
void profile_after_split(cudaStream_t stream);  // records the benchmark hook's second event, if armed

// TMA decode path (decode_tma.cu): persistent blocks over a flat (sequence, unit, tile) list.
struct TmaPlan {
  int U, kpu, vpu;   // query heads, K heads and V heads per unit
  int k_shift, v_shift;  // 2^shift neighbouring units read the same K (V) head (more than 8 query heads per head)
  int box_tok;       // tokens per TMA box
  int stages, grid, smem;
  long long slots;   // partial-result slots: grid + batch * units
  int reserve, reserve_auto;  // tail reserve per block in tiles (0 = none); auto: also at most a sixth of a block's share
  int cluster;       // 0, or the blocks per (sequence, unit) row that merge through each other's shared memory
};
bool tma_decode_supported(const diffqkv_shape& s, const diffqkv_cache& c, TmaPlan* plan);
size_t tma_decode_workspace_bytes(const diffqkv_shape& s, const TmaPlan& plan);
cudaError_t launch_decode_tma(const void* q, const diffqkv_cache& c, const diffqkv_shape& s, const TmaPlan& plan,
                              void* workspace, void* out, float* lse, int* dev_status, cudaStream_t stream);
void set_tma_max_blocks(int n);
void set_tma_tail_reserve(int n);
void set_tma_cluster_mode(int mode);  // -1 automatic, 0 never, 1 whenever the shape allows
void set_tma_debug_timeout(long long wait_limit_ns, long long skip_tile);

// Augmented-Q projection (augq.cu): three tcgen05 GEMMs, the gate/up pair fused with its silu-gate epilogue.
size_t augq_workspace_bytes(long long T, int d_q0, int d_aug);
cudaError_t launch_augq(const void* h, const void* W_Q, const void* W_gate, const void* W_up, const void* W_down,
                        long long T, int d_model, int d_q0, int d_aug, int d_out, void* workspace, void* q_out,
                        int* dev_status, cudaStream_t stream, const float* rope_cos = nullptr,
                        const float* rope_sin = nullptr, int head_dim = 0);
cudaError_t launch_project(const void* x, const void* W, long long T, int d_in, int d_out, void* y, int* dev_status,
                           cudaStream_t stream, const float* rope_cos, const float* rope_sin, int head_dim);


// Causal prefill (prefill.cu): cache update kernel, then tcgen05 attention over the cache.
bool prefill_supported(const diffqkv_shape& s, const diffqkv_cache& c, int* box_tok);
cudaError_t launch_cache_append(const void* k_new, const void* v_new, int q_len, const diffqkv_cache& c,
                                const diffqkv_shape& s, int* dev_status, cudaStream_t stream);
cudaError_t launch_prefill(const void* q, const void* k_new, const void* v_new, int q_len, const diffqkv_cache& c,
                           const diffqkv_shape& s, int box_tok, void* out, float* lse, int* dev_status,
                           cudaStream_t stream);


// Queries folded through the K feed-forward layer (kup.cu): q' = W_kup[hk]^T q per query head.
cudaError_t launch_fold_kup(const void* q, const void* W_kup, long long T, int n_q, int n_k, int d_q, int d_k,
                            void* q_out, cudaStream_t stream);

// Selective V fetching (decode_topk.cu): K-only score pass, then top-k selection and V gather per query head.
bool topk_decode_supported(const diffqkv_shape& s, const diffqkv_cache& c, int topk, int* box_tok);
size_t topk_decode_workspace_bytes(const diffqkv_shape& s, int max_seqlen, int topk);
void set_topk_general_only(int on);
cudaError_t launch_decode_topk(const void* q, const diffqkv_cache& c, const diffqkv_shape& s, int topk, int box_tok,
                               void* workspace, void* out, float* lse, int* dev_status, cudaStream_t stream,
                               int* kept_ids = nullptr);

// Ragged batches over the cache.  rope_append.cu: rotation of q and k and the cache write; host frequency tables.
cudaError_t launch_rope_append(const void* q, const void* k_new, const void* v_new, const int* cu_q, int total_q,
                               long long q_st, long long k_st, long long v_st, const diffqkv_rope& rope,
                               const CacheView& cache, const diffqkv_shape& s, void* q_out, int* dev_status,
                               cudaStream_t stream);
// norm_rope.cu: the same behind a norm of every head.
cudaError_t launch_norm_rope_append(const void* q, const void* k_new, const void* v_new, const int* cu_q, int total_q,
                                    long long q_st, long long k_st, long long v_st, const diffqkv_qk_norm& norm,
                                    const diffqkv_rope& rope, const CacheView& cache, const diffqkv_shape& s, void* q_out,
                                    int* dev_status, cudaStream_t stream);
bool rope_frequencies(int rot_dim, double theta, int scaling, double s, double L, double fast, double slow,
                      double* inv_freq, float* magnitude);
// Chunk attention: tensor cores (extend.cu, extend_thin.cu), tiles on FMAs (extend_simt.cu), one block per (row, query
// head) on FMAs (decode_generic.cu); each of the first two answers cudaErrorNotSupported where it does not apply.
// `range` (or null): rows that do not see all tokens before them.
struct ExtendRange {
  int window, sinks;  // a row sees tokens before `sinks` and those less than `window` before its own
  int groups;         // of sequences that share their first tokens; the window does not apply to these
  const int* cu_groups;
  const int* prefix_lens;
  int share;          // which of their prefixes are read once: 0 where that saves something, 1 all that can be, 2 none
};
size_t extend_workspace_bytes(const diffqkv_shape& s, int total_q, bool ranged);
size_t extend_groups_workspace_bytes(const diffqkv_shape& s, int total_q);  // on top of that
cudaError_t launch_extend(const void* q, const int* cu_q, int total_q, const diffqkv_cache& c, const diffqkv_shape& s,
                          const ExtendRange* range, void* workspace, void* out, float* lse, int* dev_status,
                          cudaStream_t stream);
size_t extend_simt_workspace_bytes(const diffqkv_shape& s, int total_q);
// These two take a window (range->groups = 0); a step with groups goes through them as one without, whose lengths
// launch_extend_lengths has set to -1 for the sequences that do not fit their group.
cudaError_t launch_extend_simt(const DecodeParams& d, const diffqkv_shape& s, const int* cu_q, int total_q,
                               const ExtendRange* range, void* workspace, void* out, float* lse, cudaStream_t stream);
cudaError_t launch_extend_generic(const DecodeParams& p, diffqkv_dtype dtype, const int* cu_q, int total_q,
                                  const ExtendRange* range, void* out, int out_is_f32, float* lse, cudaStream_t stream);
cudaError_t launch_extend_lengths(const int* cu_q, int total_q, const diffqkv_cache& c, int batch, const ExtendRange& range,
                                  int* seqlens, cudaStream_t stream);
// Page upkeep (pages.cu).
cudaError_t launch_pages_free(const int* seq_ids, const int* keep_tokens, int n, const diffqkv_pages& g, int* dev_status,
                              cudaStream_t stream);
size_t pages_fork_workspace_bytes(const diffqkv_pages& g, int n);
cudaError_t launch_pages_fork(const int* parents, const int* children, int n, const diffqkv_pages& g, void* workspace,
                              int* dev_status, cudaStream_t stream);
size_t pages_reserve_workspace_bytes(const diffqkv_pages& g);
cudaError_t launch_pages_reserve(const int* cu_q, const diffqkv_pages& g, const diffqkv_cache& c, const diffqkv_shape& s,
                                 int* granted, void* workspace, int* dev_status, cudaStream_t stream);
cudaError_t launch_pages_copy(const int* src_ids, const int* dst_ids, int n, const diffqkv_cache& from,
                              const diffqkv_cache& to, const diffqkv_shape& s, int* dev_status, cudaStream_t stream);
size_t pages_compact_workspace_bytes(const diffqkv_pages& g);
cudaError_t launch_pages_compact(const diffqkv_pages& g, const diffqkv_cache& c, const diffqkv_shape& s, int* table_out,
                                 int* refs_out, int* live, void* workspace, int* dev_status, cudaStream_t stream);

}  // namespace diffqkv

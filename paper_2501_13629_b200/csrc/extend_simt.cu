// Chunk attention on fp32 FMAs: the fp32 mode of diffqkv_extend, and bf16 calls that the tensor-core kernels do not take
// (other page sizes, scale <= 0), for heads of 64 or 128 channels; other dimensions stay with the kernel that has one
// block per row (decode_generic.cu).
//
// Mathematics as in extend.cu, in fp32 throughout.  A block takes 32 matrix rows (T = 32 / G tokens of the chunk times the
// G query heads that share K and V) and walks the cached tokens in tiles of 128.  Four rows belong to one warp for good:
// its lanes have four tokens each in the first product and kD / 32 channels each in the second, so that maxima and sums
// are warp shuffles, P goes through the warp's own shared memory, and the block meets only around the K and V tiles.
// Bound by shared-memory reads next to the FMAs: in the first product 64 FMAs a lane need four K vectors (rows padded by
// 16 bytes, no conflicts) and four broadcast Q vectors, 20 cycles of shared memory to 16 of FMA.
// V of a tile is copied (cp.async) while its scores are computed, K of the next tile during the second product.
// A long cache under few rows is cut into splits along the tokens, joined by a second kernel.  The host knows the cache's
// capacity and the number of rows, not the lengths: sequences that fill a small part of their capacity leave most of the
// splits, and of the blocks, without work.  Four sequences of 17-100 rows over up to 1k tokens, 16/2/4 heads of 64, fp32: 41 us and
// 4 us for the join (0.58 GFLOP, 8 us at the FMAs' rate; 2.2 instructions a cycle and SM); splits half as long 52 us, eight
// rows to each of four warps 46 us, packed FMAs in the first product no change.
#include <numeric>

#include "common.cuh"
#include "ptx.cuh"

namespace diffqkv {
namespace {

constexpr int kRows = 32, kTok = 128, kThreads = 256;
constexpr int kMaxSplits = 16;

struct SimtParams {
  const void* q;
  CacheView cache;
  const int* cu_q;
  int batch, total_q, n_q, G, T;
  int heads_per_k, heads_per_v;
  float scale_log2;
  int splits, split_tokens;  // tokens per split, a multiple of kTok
  void* out;
  int out_is_f32;
  float* lse;
  float* part_o;    // [total_q n_q][splits][d_v]
  float* part_lse;  // [total_q n_q][splits] base 2
  int* dev_status;
};

__device__ __forceinline__ bool rows_of(const SimtParams& p, int b, int& lo, int& n, int& past) {
  return ragged_rows(p.cu_q, p.cache.seqlens, b, p.total_q, p.cache.max_seqlen, lo, n, past);
}

// Where tokens k0 .. k0 + 127 lie: block and slot of each (block -1: not there), a thread per token.
__device__ __forceinline__ void place_tile(const SimtParams& p, int2* place, int b, int k0, int end) {
  if (threadIdx.x >= kTok) return;
  const int tok = k0 + threadIdx.x;
  int2 at = make_int2(-1, 0);
  if (tok < end) {
    at = make_int2(b, tok);
    if (p.cache.page_table) {
      at.x = p.cache.page_table[(long long)b * p.cache.max_pages_per_seq + tok / p.cache.page_size];
      at.y = tok % p.cache.page_size;
      if (at.x < 0 || at.x >= p.cache.num_blocks) {
        at.x = -1;
        report(p.dev_status, DIFFQKV_ERR_INDEX);
      }
    }
  }
  place[threadIdx.x] = at;
}

// Copies the tokens of a tile, one head, into [128][D + 4] floats.
template <typename T, int D>
__device__ __forceinline__ void copy_tile(float* dst, const void* pool, long long s_blk, long long s_tok, long long head_off,
                                          const int2* place) {
  constexpr int kPer = 16 / sizeof(T), kVecs = D / kPer;
#pragma unroll 4
  for (int e = threadIdx.x; e < kTok * kVecs; e += kThreads) {
    const int t = e / kVecs, c = (e - t * kVecs) * kPer;
    float* to = dst + t * (D + 4) + c;
    const int2 at = place[t];
    if (at.x < 0) {  // zeros: a weight of zero must not meet what lies behind the sequence
#pragma unroll
      for (int i = 0; i < kPer; i += 4) *reinterpret_cast<float4*>(to + i) = make_float4(0.f, 0.f, 0.f, 0.f);
      continue;
    }
    const T* from = reinterpret_cast<const T*>(pool) + at.x * s_blk + head_off + at.y * s_tok + c;
    if (sizeof(T) == 4) {
      ptx::cp_async_16(ptx::smem_u32(to), from);
    } else {
      const uint4 v = *reinterpret_cast<const uint4*>(from);
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; i += 2)
        *reinterpret_cast<float4*>(to + 2 * i) =
            make_float4(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u), __uint_as_float(w[i + 1] << 16),
                        __uint_as_float(w[i + 1] & 0xffff0000u));
    }
  }
}

template <typename T, int DQ, int DV>
__global__ void __launch_bounds__(kThreads) extend_simt_kernel(const SimtParams p) {
  constexpr int kC = DV / 32;  // channels of V per lane
  extern __shared__ float4 smem4[];
  float* q_s = reinterpret_cast<float*>(smem4);      // [32][DQ]
  float* k_s = q_s + kRows * DQ;                     // [128][DQ + 4]
  float* v_s = k_s + kTok * (DQ + 4);                // [128][DV + 4]
  float* p_s = v_s + kTok * (DV + 4);                // [32][128]
  __shared__ int seq_s, tile_s, scan_s[kThreads / 32];
  __shared__ int2 place_s[2][kTok];  // of this tile's and of the next one's tokens
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  // ---- block x takes the x-th row tile of all sequences
  if (tid == 0) seq_s = -1;
  int before = 0;
  const bool reports = blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0;  // the sequences that do not fit: sees them all
  for (int b0 = 0; b0 < p.batch; b0 += kThreads) {
    int lo, n = 0, past;
    const int b = b0 + tid;
    if (b < p.batch && !rows_of(p, b, lo, n, past) && reports) report(p.dev_status, DIFFQKV_ERR_INDEX);
    const int mine = b < p.batch ? (n + p.T - 1) / p.T : 0;
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    __syncthreads();
    if (lane == 31) scan_s[warp] = incl;
    __syncthreads();
    int base = before, all = 0;
    for (int w = 0; w < kThreads / 32; ++w) {
      if (w < warp) base += scan_s[w];
      all += scan_s[w];
    }
    const int at = base + incl - mine;
    if (mine > 0 && (int)blockIdx.x >= at && (int)blockIdx.x < at + mine) {
      seq_s = b;
      tile_s = blockIdx.x - at;
    }
    before += all;
    if ((int)blockIdx.x < before && !reports) break;
  }
  __syncthreads();
  const int b = seq_s;
  if (b < 0) return;
  int row_lo, n, past;
  rows_of(p, b, row_lo, n, past);
  const int tok0 = tile_s * p.T, head0 = blockIdx.y * p.G;
  const int rows = min(p.T, n - tok0) * p.G;
  const int hk = head0 / p.heads_per_k, hv = head0 / p.heads_per_v;  // Eq. (idx)
  const int last = past + min(n, tok0 + p.T);                        // tokens that the tile's last row sees
  const int t0 = blockIdx.z * p.split_tokens;
  const int t1 = p.splits > 1 ? min(last, t0 + p.split_tokens) : last;

  // ---- this block's rows of q, scaled to the base-2 domain
  for (int e = tid; e < kRows * DQ; e += kThreads) {
    const int r = e / DQ, c = e - r * DQ;
    float x = 0.f;
    if (r < rows) {
      const int tok = r / p.G;
      x = to_float(reinterpret_cast<const T*>(p.q)[((long long)(row_lo + tok0 + tok) * p.n_q + head0 + (r - tok * p.G)) * DQ + c]);
    }
    q_s[e] = x * p.scale_log2;
  }
  int pos[4];  // position of each of the warp's four rows; -1 = none
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = warp * 4 + i;
    pos[i] = r < rows ? past + tok0 + r / p.G : -1;
  }
  float m[4], l[4], acc[4][kC];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < kC; ++c) acc[i][c] = 0.f;
  }
  const CacheView& cv = p.cache;
  const long long k_head = (long long)hk * cv.k_sh, v_head = (long long)hv * cv.v_sh;
  int turn = 0;
  if (t0 < t1) {
    place_tile(p, place_s[0], b, t0, t1);
    __syncthreads();
    copy_tile<T, DQ>(k_s, cv.k, cv.k_sb, cv.k_st, k_head, place_s[0]);
    ptx::cp_async_commit();
  }
  const float* q_w = q_s + warp * 4 * DQ;
  float* p_w = p_s + warp * 4 * kTok;
  for (int k0 = t0; k0 < t1; k0 += kTok, turn ^= 1) {
    copy_tile<T, DV>(v_s, cv.v, cv.v_sb, cv.v_st, v_head, place_s[turn]);
    if (k0 + kTok < t1) place_tile(p, place_s[turn ^ 1], b, k0 + kTok, t1);
    ptx::cp_async_commit();
    ptx::cp_async_wait<1>();  // K of this tile
    __syncthreads();
    // ---- scores: rows warp * 4 + i, tokens lane + 32 j
    float s[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
    for (int c = 0; c < DQ; c += 4) {
      float4 a[4], x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4*>(q_w + i * DQ + c);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = *reinterpret_cast<const float4*>(k_s + (lane + 32 * j) * (DQ + 4) + c);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s[i][j] = fmaf(a[i].x, x[j].x, s[i][j]);
          s[i][j] = fmaf(a[i].y, x[j].y, s[i][j]);
          s[i][j] = fmaf(a[i].z, x[j].z, s[i][j]);
          s[i][j] = fmaf(a[i].w, x[j].w, s[i][j]);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float top = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int tok = k0 + lane + 32 * j;
        if (tok > pos[i] || tok >= t1) s[i][j] = -INFINITY;
        top = fmaxf(top, s[i][j]);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      const float next = fmaxf(m[i], top), ref = next == -INFINITY ? 0.f : next;
      const float alpha = exp2f(m[i] - ref);
      m[i] = next;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float w = exp2f(s[i][j] - ref);
        sum += w;
        p_w[i * kTok + lane + 32 * j] = w;
      }
      l[i] = l[i] * alpha + sum;  // per lane; over the lanes at the end
#pragma unroll
      for (int c = 0; c < kC; ++c) acc[i][c] *= alpha;
    }
    ptx::cp_async_wait<0>();  // V of this tile
    __syncthreads();          // everybody is through with K
    if (k0 + kTok < t1) {
      copy_tile<T, DQ>(k_s, cv.k, cv.k_sb, cv.k_st, k_head, place_s[turn ^ 1]);
      ptx::cp_async_commit();
    }
    // ---- O += P V: channels lane * kC ..
    const int used = min(kTok, t1 - k0);
#pragma unroll 2
    for (int t = 0; t < used; t += 4) {  // rows behind the last token are zeros
      float4 w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const float4*>(p_w + i * kTok + t);
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        float v[kC];
        const float* from = v_s + (t + y) * (DV + 4) + lane * kC;
        if (kC == 4) {
          const float4 x = *reinterpret_cast<const float4*>(from);
          v[0] = x.x; v[1] = x.y; v[2 % kC] = x.z; v[3 % kC] = x.w;
        } else {
          const float2 x = *reinterpret_cast<const float2*>(from);
          v[0] = x.x; v[1] = x.y;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float f = y == 0 ? w[i].x : y == 1 ? w[i].y : y == 2 ? w[i].z : w[i].w;
#pragma unroll
          for (int c = 0; c < kC; ++c) acc[i][c] = fmaf(f, v[c], acc[i][c]);
        }
      }
    }
    __syncthreads();  // V may be overwritten
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = warp * 4 + i;
    if (r >= rows) continue;  // the same for all lanes
    float sum = l[i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    const int tok = r / p.G;
    const long long row = (long long)(row_lo + tok0 + tok) * p.n_q + head0 + (r - tok * p.G);
    const float lse2 = sum != 0.f ? m[i] + log2f(sum) : -INFINITY;
    if (p.splits > 1) {
      const long long at = row * p.splits + blockIdx.z;
#pragma unroll
      for (int c = 0; c < kC; ++c) p.part_o[at * DV + lane * kC + c] = acc[i][c] * inv;
      if (lane == 0) p.part_lse[at] = lse2;
      continue;
    }
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      if (p.out_is_f32) reinterpret_cast<float*>(p.out)[row * DV + lane * kC + c] = acc[i][c] * inv;
      else store_out(reinterpret_cast<__nv_bfloat16*>(p.out) + row * DV + lane * kC + c, acc[i][c] * inv);
    }
    if (p.lse && lane == 0) p.lse[row] = lse2 * kLn2;
  }
}

// A warp per (row, head) of the rows that belong to the step; rows of sequences that do not fit are left alone.
template <int DV>
__global__ void __launch_bounds__(256) extend_join_kernel(const SimtParams p) {
  constexpr int kC = DV / 32;
  const int lane = threadIdx.x & 31;
  const int t = blockIdx.x, h = blockIdx.y * 8 + (threadIdx.x >> 5);
  int lo, n, past;
  if (ragged_sequence_of<256>(p.cu_q, p.cache.seqlens, p.batch, p.total_q, p.cache.max_seqlen, t, false, p.dev_status, lo, n,
                              past, [] {}) < 0 ||
      h >= p.n_q)
    return;
  const long long row = (long long)t * p.n_q + h;
  float top = -INFINITY, sum = 0.f, acc[kC];
#pragma unroll
  for (int c = 0; c < kC; ++c) acc[c] = 0.f;
  for (int i = 0; i < p.splits; ++i) top = fmaxf(top, p.part_lse[row * p.splits + i]);
  for (int i = 0; i < p.splits; ++i) {
    const float ls = p.part_lse[row * p.splits + i];
    if (ls == -INFINITY) continue;
    const float f = exp2f(ls - top);
    sum += f;
#pragma unroll
    for (int c = 0; c < kC; ++c) acc[c] = fmaf(f, p.part_o[(row * p.splits + i) * DV + lane * kC + c], acc[c]);
  }
  const float inv = sum != 0.f ? 1.f / sum : 0.f;
#pragma unroll
  for (int c = 0; c < kC; ++c) {
    if (p.out_is_f32) reinterpret_cast<float*>(p.out)[row * DV + lane * kC + c] = acc[c] * inv;
    else store_out(reinterpret_cast<__nv_bfloat16*>(p.out) + row * DV + lane * kC + c, acc[c] * inv);
  }
  if (p.lse && lane == 0) p.lse[row] = sum != 0.f ? (top + log2f(sum)) * kLn2 : -INFINITY;
}

int heads_per_tile(const diffqkv_shape& s) {
  int G = std::gcd(s.n_q / s.n_k, s.n_q / s.n_v);
  if (G > kRows) {
    int d = kRows;
    while (G % d != 0) --d;
    G = d;
  }
  return G;
}

bool dims_ok(const diffqkv_shape& s) { return (s.d_qk == 64 || s.d_qk == 128) && (s.d_v == 64 || s.d_v == 128); }

// Splits along the tokens: enough blocks for two a SM, of at least 256 tokens each; the partial rows of all splits stay
// within 32768.
int most_splits(const diffqkv_shape& s, int total_q) {
  const long long most = 32768 / ((long long)total_q * s.n_q);
  return most > kMaxSplits ? kMaxSplits : (int)most;
}
int split_count(const diffqkv_shape& s, int max_seqlen, int total_q) {
  const long long blocks = ((long long)total_q * s.n_q + kRows - 1) / kRows;
  long long want = (296 + blocks - 1) / blocks;
  if (want > max_seqlen / 256) want = max_seqlen / 256;
  if (want > most_splits(s, total_q)) want = most_splits(s, total_q);
  return want < 1 ? 1 : (int)want;
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

// The capacity of the cache is not known when the workspace is sized: room for the most splits.
size_t extend_simt_workspace_bytes(const diffqkv_shape& s, int total_q) {
  if (!dims_ok(s) || total_q == 0 || most_splits(s, total_q) < 2) return 0;
  const size_t parts = (size_t)total_q * s.n_q * most_splits(s, total_q);
  return up256(parts * sizeof(float)) + up256(parts * s.d_v * sizeof(float));
}

cudaError_t launch_extend_simt(const DecodeParams& d, const diffqkv_shape& s, const int* cu_q, int total_q, void* workspace,
                               void* out, float* lse, cudaStream_t stream) {
  if (!dims_ok(s)) return cudaErrorNotSupported;
  SimtParams p;
  p.q = d.q; p.cache = d.cache; p.cu_q = cu_q;
  p.batch = s.batch; p.total_q = total_q; p.n_q = s.n_q;
  p.G = heads_per_tile(s); p.T = kRows / p.G;
  p.heads_per_k = s.n_q / s.n_k; p.heads_per_v = s.n_q / s.n_v;
  p.scale_log2 = d.scale_log2;
  p.splits = split_count(s, d.cache.max_seqlen, total_q);
  p.split_tokens = ((d.cache.max_seqlen + p.splits - 1) / p.splits + kTok - 1) / kTok * kTok;
  p.out = out; p.out_is_f32 = s.out_dtype == DIFFQKV_F32; p.lse = lse;
  p.part_lse = static_cast<float*>(workspace);
  p.part_o = reinterpret_cast<float*>(static_cast<char*>(workspace) +
                                      up256((size_t)total_q * s.n_q * p.splits * sizeof(float)));
  p.dev_status = d.dev_status;
  const long long tiles = (long long)total_q / p.T + s.batch;
  const dim3 grid((unsigned)(tiles < total_q ? tiles : total_q), (unsigned)(s.n_q / p.G), (unsigned)p.splits);
  const size_t smem = sizeof(float) * ((size_t)kRows * s.d_qk + kTok * (s.d_qk + 4) + kTok * (s.d_v + 4) + kRows * kTok);
  void (*fn)(const SimtParams) = nullptr;
#define DIFFQKV_SIMT_CASE(DQ, DV)     \
  if (s.d_qk == DQ && s.d_v == DV)    \
    fn = s.dtype == DIFFQKV_F32 ? extend_simt_kernel<float, DQ, DV> : extend_simt_kernel<__nv_bfloat16, DQ, DV>;
  DIFFQKV_SIMT_CASE(64, 64) DIFFQKV_SIMT_CASE(64, 128) DIFFQKV_SIMT_CASE(128, 64) DIFFQKV_SIMT_CASE(128, 128)
#undef DIFFQKV_SIMT_CASE
  cudaError_t err = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (err != cudaSuccess) return err;
  fn<<<grid, kThreads, smem, stream>>>(p);
  count_launch();
  err = cudaGetLastError();
  if (err != cudaSuccess || p.splits == 1) return err;
  const dim3 join((unsigned)total_q, (unsigned)((s.n_q + 7) / 8));
  if (s.d_v == 64) extend_join_kernel<64><<<join, 256, 0, stream>>>(p);
  else extend_join_kernel<128><<<join, 256, 0, stream>>>(p);
  count_launch();
  return cudaGetLastError();
}

}  // namespace diffqkv

// Root-mean-square norms of query and key heads, rotary positions and the cache write of a ragged step in one launch
// (diffqkv_norm_rope_append).
//
// Mathematics: every head x of q and k becomes x * r * (offset + w), r = 1 / sqrt(mean x_c^2 + eps) over its d_qk channels,
// and its first rot_dim channels are then turned as in rope_append.cu, all in fp32 (bf16 between the two would cost another
// half step of 2^-8 of every channel), rounded once.
//
// Bound by memory like rope_append.cu, whose plan this follows: a block a row, its angles worked out once for all heads, first
// vectors read before the row's place is known.  A head belongs to a group of lanes of one warp, two 16-byte vectors to a
// lane (a channel and its partner; neighbours where pairs are neighbours or nothing turns), so that the sum of squares is
// a few shuffles and the head never leaves its registers.  Heads of more than 64 vectors are read a second time.
#include "common.cuh"
#include "rope.cuh"

namespace diffqkv {
namespace {

struct NormParams {
  const void* q_weight;
  const void* k_weight;
  long long q_wst, k_wst;  // elements between heads
  float eps, offset, inv_d;
  int lanes;               // of a head, a power of two
};

// One 16-byte vector's channels of a weight: W is T or float.
template <typename T, typename W>
__device__ __forceinline__ void open_weight(const W* w, float (&x)[Pack<T>::N]) {
  constexpr int M = Pack<W>::N;
#pragma unroll
  for (int i = 0; i < Pack<T>::N; i += M) {
    float y[M];
    Pack<W>::open(*reinterpret_cast<const uint4*>(w + i), y);
#pragma unroll
    for (int e = 0; e < M; ++e) x[i + e] = y[e];
  }
}

// kPairs: rotate-half.
template <typename T, typename W, bool kPairs>
__global__ void __launch_bounds__(kRopeThreads, 5) norm_rope_kernel(const RopeParams p, const NormParams m) {
  constexpr int N = Pack<T>::N;
  constexpr int kAhead = 3;  // heads read together
  extern __shared__ float2 turn_s[];  // [rot / 2] (cos, sin) * magnitude
  const int tid = threadIdx.x;
  const int t = blockIdx.x;  // row

  // A task is two vectors of a head; lane x of a head's lanes has tasks x, x + lanes, ...
  const int half = p.rot >> 1;
  const int rot_tasks = p.rot / (2 * N), rest = (p.d_qk - p.rot) / N, tasks = rot_tasks + (rest + 1) / 2;
  const int lanes = m.lanes, heads_at_once = kRopeThreads / lanes, first = tid / lanes, lane = tid - first * lanes;
  const int q_heads = p.q ? p.n_q : 0, heads = q_heads + p.n_k;
  const bool single = tasks <= lanes;
  struct Task {
    int c0, c1;  // first channels of its vectors; -1: none
    bool rotated;
  };
  auto task = [&](int x) -> Task {
    if (x < rot_tasks) return kPairs ? Task{x * N, x * N + half, true} : Task{2 * x * N, (2 * x + 1) * N, true};
    const int y = 2 * (x - rot_tasks);
    return {y < rest ? p.rot + y * N : -1, y + 1 < rest ? p.rot + (y + 1) * N : -1, false};
  };
  const T* q_row = reinterpret_cast<const T*>(p.q) + t * p.q_st;
  const T* k_row = reinterpret_cast<const T*>(p.k_new) + t * p.k_st;
  auto read = [&](int h, const Task& k, uint4 (&a)[2]) {
    a[0] = a[1] = make_uint4(0, 0, 0, 0);
    if (h >= heads) return;
    const T* src = h < q_heads ? q_row + h * p.d_qk : k_row + (h - q_heads) * p.d_qk;
    if (k.c0 >= 0) a[0] = *reinterpret_cast<const uint4*>(src + k.c0);
    if (k.c1 >= 0) a[1] = *reinterpret_cast<const uint4*>(src + k.c1);
  };
  const int vvec = p.d_v / N, v_at_once = kRopeThreads / vvec, v_first = tid / vvec, vc = (tid - v_first * vvec) * N;
  const int v_heads = v_first < v_at_once ? p.n_v : 0;
  const T* v_row = reinterpret_cast<const T*>(p.v_new) + t * p.v_st + vc;
  const Task mine = task(lane);
  uint4 ahead[kAhead][2], v_ahead;
  auto read_ahead = [&] {
#pragma unroll
    for (int y = 0; y < kAhead; ++y) read(first + y * heads_at_once, mine, ahead[y]);
    if (v_first < v_heads) v_ahead = *reinterpret_cast<const uint4*>(v_row + v_first * p.d_v);
  };
  read_ahead();

  // ---- the row's sequence and place
  int lo, n, past;
  const int b = ragged_sequence_of<kRopeThreads>(p.cu_q, p.cache.seqlens, p.batch, p.total_q, p.cache.max_seqlen, t, t == 0,
                                                 p.dev_status, lo, n, past, read_ahead);
  if (b < 0) return;  // behind the last sequence, or of one that does not fit
  const int tok = past + (t - lo);
  long long blk = b, slot = tok;
  bool place_ok = true;
  if (p.cache.page_table) {
    blk = p.cache.page_table[(long long)b * p.cache.max_pages_per_seq + tok / p.cache.page_size];
    slot = tok % p.cache.page_size;
    place_ok = blk >= 0 && blk < p.cache.num_blocks;
    if (!place_ok && tid == 0) report(p.dev_status, DIFFQKV_ERR_INDEX);
  }
  for (int i = tid; i < half; i += kRopeThreads) {
    const int pos = p.positions ? p.positions[t] : tok;
    float sn, cs;
    sincosf(reduced_angle(pos, p.inv_freq[i]), &sn, &cs);
    turn_s[i] = make_float2(cs * p.magnitude, sn * p.magnitude);
  }
  __syncthreads();
  if (place_ok) {
    T* v_out = reinterpret_cast<T*>(const_cast<void*>(p.cache.v)) + blk * p.cache.v_sb + slot * p.cache.v_st + vc;
    if (v_first < v_heads) *reinterpret_cast<uint4*>(v_out + v_first * p.cache.v_sh) = v_ahead;
    for (int h = v_first + v_at_once; h < v_heads; h += v_at_once)
      *reinterpret_cast<uint4*>(v_out + h * p.cache.v_sh) = *reinterpret_cast<const uint4*>(v_row + h * p.d_v);
  }
  T* q_out = reinterpret_cast<T*>(p.q_out) + (long long)t * p.n_q * p.d_qk;
  T* k_out = reinterpret_cast<T*>(const_cast<void*>(p.cache.k)) + blk * p.cache.k_sb + slot * p.cache.k_st;

  auto squares = [&](const uint4 (&raw)[2]) -> float {
    float s = 0.f;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      float a[N];
      Pack<T>::open(raw[y], a);
#pragma unroll
      for (int i = 0; i < N; ++i) s = fmaf(a[i], a[i], s);
    }
    return s;
  };
  auto over_lanes = [&](float s) -> float {  // the head's factor; every lane of the warp calls it
    for (int o = lanes >> 1; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return rsqrtf(fmaf(s, m.inv_d, m.eps));
  };
  auto finish = [&](int h, const Task& k, const float2 (&turn)[N], float r, const uint4 (&raw)[2]) {
    if (h >= heads || k.c0 < 0) return;
    const bool is_q = h < q_heads;
    if (!is_q && !place_ok) return;
    T* dst = is_q ? q_out + h * p.d_qk : k_out + (h - q_heads) * p.cache.k_sh;
    const W* weight = reinterpret_cast<const W*>(is_q ? m.q_weight : m.k_weight);
    if (weight) weight += is_q ? h * m.q_wst : (h - q_heads) * m.k_wst;
    float a[2][N];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      Pack<T>::open(raw[y], a[y]);
      float w[N];
      const int c = y == 0 ? k.c0 : k.c1;
      if (weight && c >= 0) {
        open_weight<T, W>(weight + c, w);
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] += m.offset;
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = m.offset != 0.f ? m.offset : 1.f;
      }
#pragma unroll
      for (int i = 0; i < N; ++i) a[y][i] = a[y][i] * r * w[i];
    }
    if (k.rotated) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float& u = kPairs ? a[0][i] : a[2 * i / N][2 * i % N];
        float& v = kPairs ? a[1][i] : a[2 * i / N][2 * i % N + 1];
        const float x = u, y = v;
        u = x * turn[i].x - y * turn[i].y;
        v = y * turn[i].x + x * turn[i].y;
      }
    }
    *reinterpret_cast<uint4*>(dst + k.c0) = Pack<T>::close(a[0]);
    if (k.c1 >= 0) *reinterpret_cast<uint4*>(dst + k.c1) = Pack<T>::close(a[1]);
  };
  auto turns_of = [&](const Task& k, float2 (&turn)[N]) {
    if (!k.rotated) return;
#pragma unroll
    for (int i = 0; i < N; ++i) turn[i] = turn_s[(kPairs ? k.c0 : k.c0 / 2) + i];
  };
  float2 turn[N];
  if (single) {
    turns_of(mine, turn);
    for (int h0 = 0;;) {  // the same for all threads: the warp's lanes meet in the sums
#pragma unroll
      for (int y = 0; y < kAhead; ++y)
        if (h0 + y * heads_at_once < heads) {
          const float r = over_lanes(squares(ahead[y]));
          finish(h0 + y * heads_at_once + first, mine, turn, r, ahead[y]);
        }
      h0 += kAhead * heads_at_once;
      if (h0 >= heads) break;
#pragma unroll
      for (int y = 0; y < kAhead; ++y) read(h0 + y * heads_at_once + first, mine, ahead[y]);
    }
    return;
  }
  for (int h0 = 0; h0 < heads; h0 += heads_at_once) {
    float s = 0.f;
    uint4 raw[2];
    for (int x = lane; x < tasks; x += lanes) {
      read(h0 + first, task(x), raw);
      s += squares(raw);
    }
    const float r = over_lanes(s);
    for (int x = lane; x < tasks; x += lanes) {
      const Task k = task(x);
      read(h0 + first, k, raw);
      turns_of(k, turn);
      finish(h0 + first, k, turn, r, raw);
    }
  }
}

template <typename T, typename W>
cudaError_t launch(const RopeParams& p, const NormParams& m, cudaStream_t stream) {
  const size_t smem = sizeof(float2) * (p.rot / 2 + 1);
  if (p.interleaved) norm_rope_kernel<T, W, false><<<(unsigned)p.total_q, kRopeThreads, smem, stream>>>(p, m);
  else norm_rope_kernel<T, W, true><<<(unsigned)p.total_q, kRopeThreads, smem, stream>>>(p, m);
  count_launch();
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_norm_rope_append(const void* q, const void* k_new, const void* v_new, const int* cu_q, int total_q,
                                    long long q_st, long long k_st, long long v_st, const diffqkv_qk_norm& norm,
                                    const diffqkv_rope& rope, const CacheView& cache, const diffqkv_shape& s, void* q_out,
                                    int* dev_status, cudaStream_t stream) {
  const RopeParams p = rope_params(q, k_new, v_new, cu_q, total_q, q_st, k_st, v_st, rope, cache, s, q_out, dev_status);
  const int n = s.dtype == DIFFQKV_BF16 ? 8 : 4;
  const int tasks = p.rot / (2 * n) + ((p.d_qk - p.rot) / n + 1) / 2;
  NormParams m;
  m.q_weight = norm.q_weight; m.k_weight = norm.k_weight;
  m.q_wst = norm.q_head_stride; m.k_wst = norm.k_head_stride;
  m.eps = norm.eps; m.offset = norm.weight_offset; m.inv_d = 1.f / (float)s.d_qk;
  for (m.lanes = 1; m.lanes < 32 && m.lanes < tasks;) m.lanes *= 2;
  if (s.dtype == DIFFQKV_F32) return launch<float, float>(p, m, stream);
  return norm.weight_dtype == DIFFQKV_F32 ? launch<__nv_bfloat16, float>(p, m, stream)
                                          : launch<__nv_bfloat16, __nv_bfloat16>(p, m, stream);
}

}  // namespace diffqkv

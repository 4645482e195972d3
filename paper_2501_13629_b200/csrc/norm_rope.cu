// Root-mean-square norms of query and key heads, rotary positions and the cache write of a ragged step in one launch
// (diffqkv_norm_rope_append).
//
// Mathematics: every head x of q and k becomes x * r * (offset + w), r = 1 / sqrt(mean x_c^2 + eps) over its d_qk channels,
// and its first rot_dim channels are then turned as in rope_append.cu, all in fp32 (bf16 between the two would cost another
// half step of 2^-8 of every channel), rounded once.  Weight and turn are one: with g = offset + w a pair (u, v) becomes
//     (r u) g_u cos - (r v) g_v sin,   (r v) g_v cos + (r u) g_u sin,
// four coefficients a pair, which the heads of a row share.
//
// Bound by memory like rope_append.cu, whose plan this follows: a block a row, its angles worked out once for all heads, first
// vectors read before the row's place is known.  A head belongs to a group of lanes of one warp, two 16-byte vectors to a
// lane (a channel and its partner; neighbours where pairs are neighbours or nothing turns), so that the sum of squares is
// a few shuffles and the head never leaves its registers.  The coefficients of a row, a thread a pair, lie in shared memory,
// where the lanes of a head read them without conflicts; weights and frequencies for them are read ahead too.
// 12k rows of 32/4/8 heads of 128 channels, bf16 (272 MB): 59 us, 4.6 TB/s, against 50 for rope_append; instructions are
// issued in three cycles of four.  With weight and turn applied one after the other to every head it was 72 us, with the
// coefficients in registers and a head after another 90-105, with several rows to a block, the next one's vectors read as
// registers fall free, 71-76, with 64 or 32 threads a row 60.  16 rows: 5.2 us.
// Heads of more than 64 vectors are read a second time.
#include "attn_math.cuh"
#include "common.cuh"
#include "ptx.cuh"
#include "rope.cuh"

namespace diffqkv {
namespace {

struct NormParams {
  const void* q_weight;
  const void* k_weight;
  long long q_wst, k_wst;  // elements between heads; 0: one for all of them, or none
  float eps, offset, inv_d;
  int lanes, lanes_log2;   // of a head, a power of two
  int tasks, rot_tasks, rest;  // of a head: those that turn and, in vectors, what does not
  int v_magic;             // thread / 2^16 rounded up over the vectors of a V head: its head
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

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// kPairs: rotate-half.  A task is two vectors of a head, seen as pairs: u from the first, v from the second; where neighbours
// turn together, u the even and v the odd channels of both.
template <typename T, bool kPairs>
struct Task {
  static constexpr int N = Pack<T>::N;
  int c0, c1;  // first channels of its vectors; -1: none
  bool rotated;
  __device__ void open(const uint4 (&raw)[2], uint64_t (&u)[N / 2], uint64_t (&v)[N / 2]) const {
    float a[2 * N];
    Pack<T>::open(raw[0], *reinterpret_cast<float(*)[N]>(a));
    Pack<T>::open(raw[1], *reinterpret_cast<float(*)[N]>(a + N));
    split(a, u, v);
  }
  static __device__ void split(const float (&a)[2 * N], uint64_t (&u)[N / 2], uint64_t (&v)[N / 2]) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      u[i] = kPairs ? pair(a[2 * i], a[2 * i + 1]) : pair(a[4 * i], a[4 * i + 2]);
      v[i] = kPairs ? pair(a[N + 2 * i], a[N + 2 * i + 1]) : pair(a[4 * i + 1], a[4 * i + 3]);
    }
  }
  static __device__ void join(const uint64_t (&u)[N / 2], const uint64_t (&v)[N / 2], uint4 (&raw)[2]) {
    float a[2 * N];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      unpair(u[i], a[kPairs ? 2 * i : 4 * i], a[kPairs ? 2 * i + 1 : 4 * i + 2]);
      unpair(v[i], a[kPairs ? N + 2 * i : 4 * i + 1], a[kPairs ? N + 2 * i + 1 : 4 * i + 3]);
    }
    raw[0] = Pack<T>::close(*reinterpret_cast<float(*)[N]>(a));
    raw[1] = Pack<T>::close(*reinterpret_cast<float(*)[N]>(a + N));
  }
};

template <typename T, typename W, bool kPairs>
__global__ void __launch_bounds__(kRopeThreads, 8) norm_rope_kernel(const RopeParams p, const NormParams m) {
  constexpr int N = Pack<T>::N;
  constexpr int kAhead = 3;  // heads read together
  using Task = Task<T, kPairs>;
  // (cos, sin) * magnitude [rot / 2], for heads of many tasks; or the coefficients of q's and of k's tasks, sixteen bytes of
  // every task behind one another: [2][N][tasks][4]
  extern __shared__ float4 smem4[];
  float2* turn_s = reinterpret_cast<float2*>(smem4);
  float* coef_s = reinterpret_cast<float*>(smem4);
  const int tid = threadIdx.x;
  const int t = blockIdx.x;  // row

  ptx::grid_dependency_wait();  // launched before the work in front of it has ended

  // lane x of a head's lanes has tasks x, x + lanes, ...
  const int half = p.rot >> 1, rot_tasks = m.rot_tasks, rest = m.rest, tasks = m.tasks;
  const int lanes = m.lanes, heads_at_once = kRopeThreads >> m.lanes_log2, first = tid >> m.lanes_log2, lane = tid & (lanes - 1);
  const int q_heads = p.q ? p.n_q : 0, heads = q_heads + p.n_k;
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
  const int vvec = p.d_v / N, v_at_once = kRopeThreads * m.v_magic >> 16, v_first = tid * m.v_magic >> 16, vc = (tid - v_first * vvec) * N;
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
  // Likewise what a thread's first pair of coefficients is made of: its place, weights and angle per position.
  struct Pair {
    float* dst;
    float gu, gv;
    double freq;
    bool rotated;
  };
  auto weights = [&](bool is_q) -> const W* { return reinterpret_cast<const W*>(is_q ? m.q_weight : m.k_weight); };
  auto weight_head = [&](bool is_q) -> long long { return is_q ? m.q_wst : m.k_wst; };
  const float no_weight = m.offset != 0.f ? m.offset : 1.f;
  auto pair_of = [&](int x) -> Pair {  // weights that every head has its own of are left to the heads
    const bool is_q = x < tasks * N;
    const int j = is_q ? x : x - tasks * N, at = j / N, i = j - at * N;
    const Task k = task(at);
    const int cu = kPairs ? k.c0 + i : k.c0 + 2 * i, cv = kPairs ? k.c1 + i : cu + 1;
    Pair r = {coef_s + (((is_q ? 0 : N) + i / 4) * tasks + at) * 4 + i % 4, 1.f, 1.f, 0.0, k.rotated};
    if (weight_head(is_q) == 0) {
      const W* weight = weights(is_q);  // (a last vector may have no second)
      r.gu = !weight ? no_weight : cu < p.d_qk ? to_float(weight[cu]) + m.offset : 0.f;
      r.gv = !weight ? no_weight : k.c1 >= 0 || (!kPairs && cv < p.d_qk) ? to_float(weight[cv]) + m.offset : 0.f;
    }
    if (k.rotated) r.freq = p.inv_freq[(kPairs ? k.c0 : k.c0 / 2) + i];
    return r;
  };
  const bool single = tasks <= lanes;
  Pair pair0 = {};
  if (single && tid < 2 * tasks * N) pair0 = pair_of(tid);

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
  const int pos = p.positions ? p.positions[t] : tok;
  auto turn = [&](double freq) -> float2 {
    float sn, cs;
    sincosf(reduced_angle(pos, freq), &sn, &cs);
    return make_float2(cs * p.magnitude, sn * p.magnitude);
  };
  if (single) {  // a thread a pair, of q's and of k's
    for (int x = tid; x < 2 * tasks * N; x += kRopeThreads) {
      if (x != tid) pair0 = pair_of(x);
      const float2 w = pair0.rotated ? turn(pair0.freq) : make_float2(1.f, 0.f);
      const int step = (N / 4) * tasks * 4;
      pair0.dst[0] = pair0.gu * w.x;
      pair0.dst[step] = pair0.gv * w.x;
      pair0.dst[2 * step] = pair0.gu * w.y;
      pair0.dst[3 * step] = -pair0.gv * w.y;
    }
  } else {
    for (int i = tid; i < half; i += kRopeThreads) turn_s[i] = turn(p.inv_freq[i]);
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

  auto squares = [&](const uint64_t (&u)[N / 2], const uint64_t (&v)[N / 2]) -> float {
    uint64_t s = 0;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) s = fma2(v[i], v[i], fma2(u[i], u[i], s));
    float x, y;
    unpair(s, x, y);
    return x + y;
  };
  auto over_lanes = [&](float s) -> float {  // the head's factor; every lane of the warp calls it
    for (int o = lanes >> 1; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return rsqrtf(fmaf(s, m.inv_d, m.eps));
  };
  auto own_weights = [&](const W* weight, const Task& k, uint64_t (&u)[N / 2], uint64_t (&v)[N / 2]) {  // of one head
    float g[2 * N];
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) g[i] = no_weight;
    if (weight) {
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int c = y == 0 ? k.c0 : k.c1;
        if (c < 0) continue;
        float w[N];
        open_weight<T, W>(weight + c, w);
#pragma unroll
        for (int i = 0; i < N; ++i) g[y * N + i] = w[i] + m.offset;
      }
    }
    uint64_t gu[N / 2], gv[N / 2];
    Task::split(g, gu, gv);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      u[i] = mul2(u[i], gu[i]);
      v[i] = mul2(v[i], gv[i]);
    }
  };
  auto place_of = [&](int h) -> T* { return h < q_heads ? q_out + h * p.d_qk : k_out + (h - q_heads) * p.cache.k_sh; };
  auto write = [&](int h, const Task& k, const uint64_t (&u)[N / 2], const uint64_t (&v)[N / 2]) {
    uint4 raw[2];
    Task::join(u, v, raw);
    T* dst = place_of(h);
    if (k.c0 >= 0) *reinterpret_cast<uint4*>(dst + k.c0) = raw[0];
    if (k.c1 >= 0) *reinterpret_cast<uint4*>(dst + k.c1) = raw[1];
  };

  if (single) {
    for (int h0 = 0;;) {  // the same for all threads: the warp's lanes meet in the sums
#pragma unroll
      for (int y = 0; y < kAhead; ++y) {
        if (h0 + y * heads_at_once >= heads) break;
        const int h = h0 + y * heads_at_once + first;
        uint64_t u[N / 2], v[N / 2];
        mine.open(ahead[y], u, v);
        const float r = over_lanes(squares(u, v));
        if (h >= heads || (h >= q_heads && !place_ok) || mine.c0 < 0) continue;
        const uint64_t r2 = pair(r, r);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
          u[i] = mul2(u[i], r2);
          v[i] = mul2(v[i], r2);
        }
        const bool is_q = h < q_heads;
        if (weight_head(is_q) != 0) own_weights(weights(is_q) + (is_q ? h : h - q_heads) * weight_head(is_q), mine, u, v);
        const ulonglong2* f = reinterpret_cast<const ulonglong2*>(coef_s) + (is_q ? 0 : N * tasks) + lane;
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {  // two packed pairs of each coefficient
          const ulonglong2 uc = f[i * tasks], vc2 = f[(N / 4 + i) * tasks];
          const uint64_t a0 = u[2 * i], b0 = v[2 * i], a1 = u[2 * i + 1], b1 = v[2 * i + 1];
          u[2 * i] = mul2(a0, uc.x);
          v[2 * i] = mul2(b0, vc2.x);
          u[2 * i + 1] = mul2(a1, uc.y);
          v[2 * i + 1] = mul2(b1, vc2.y);
          if (mine.rotated) {
            const ulonglong2 us = f[(2 * (N / 4) + i) * tasks], vs = f[(3 * (N / 4) + i) * tasks];
            u[2 * i] = fma2(b0, vs.x, u[2 * i]);
            v[2 * i] = fma2(a0, us.x, v[2 * i]);
            u[2 * i + 1] = fma2(b1, vs.y, u[2 * i + 1]);
            v[2 * i + 1] = fma2(a1, us.y, v[2 * i + 1]);
          }
        }
        write(h, mine, u, v);
      }
      h0 += kAhead * heads_at_once;
      if (h0 >= heads) break;
#pragma unroll
      for (int y = 0; y < kAhead; ++y) read(h0 + y * heads_at_once + first, mine, ahead[y]);
    }
    return;
  }
  for (int h0 = 0; h0 < heads; h0 += heads_at_once) {
    const int h = h0 + first;
    const bool is_q = h < q_heads;
    float s = 0.f;
    uint4 raw[2];
    uint64_t u[N / 2], v[N / 2];
    for (int x = lane; x < tasks; x += lanes) {
      const Task k = task(x);
      read(h, k, raw);
      k.open(raw, u, v);
      s += squares(u, v);
    }
    const float r = over_lanes(s);
    if (h >= heads || (!is_q && !place_ok)) continue;
    const uint64_t r2 = pair(r, r);
    const W* weight = weights(is_q);
    if (weight) weight += (is_q ? h : h - q_heads) * weight_head(is_q);
    for (int x = lane; x < tasks; x += lanes) {
      const Task k = task(x);
      read(h, k, raw);
      k.open(raw, u, v);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        u[i] = mul2(u[i], r2);
        v[i] = mul2(v[i], r2);
      }
      own_weights(weight, k, u, v);
      if (k.rotated) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
          const float2* w = turn_s + (kPairs ? k.c0 : k.c0 / 2) + 2 * i;
          const float2 w0 = w[0], w1 = w[1];
          const uint64_t a = u[i], b = v[i];
          u[i] = fma2(b, pair(-w0.y, -w1.y), mul2(a, pair(w0.x, w1.x)));
          v[i] = fma2(a, pair(w0.y, w1.y), mul2(b, pair(w0.x, w1.x)));
        }
      }
      write(h, k, u, v);
    }
  }
}

template <typename T, typename W>
cudaError_t launch(const RopeParams& p, const NormParams& m, cudaStream_t stream) {
  const size_t smem = m.tasks <= m.lanes ? sizeof(float4) * 2 * Pack<T>::N * m.tasks : sizeof(float2) * (p.rot / 2 + 1);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)p.total_q);
  cfg.blockDim = dim3(kRopeThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  const cudaError_t err = cudaLaunchKernelEx(&cfg, p.interleaved ? norm_rope_kernel<T, W, false> : norm_rope_kernel<T, W, true>, p, m);
  if (err == cudaSuccess) count_launch();
  return err;
}

}  // namespace

cudaError_t launch_norm_rope_append(const void* q, const void* k_new, const void* v_new, const int* cu_q, int total_q,
                                    long long q_st, long long k_st, long long v_st, const diffqkv_qk_norm& norm,
                                    const diffqkv_rope& rope, const CacheView& cache, const diffqkv_shape& s, void* q_out,
                                    int* dev_status, cudaStream_t stream) {
  const RopeParams p = rope_params(q, k_new, v_new, cu_q, total_q, q_st, k_st, v_st, rope, cache, s, q_out, dev_status);
  const int n = s.dtype == DIFFQKV_BF16 ? 8 : 4;
  NormParams m;
  m.rot_tasks = p.rot / (2 * n); m.rest = (p.d_qk - p.rot) / n; m.tasks = m.rot_tasks + (m.rest + 1) / 2;
  m.v_magic = (65536 + s.d_v / n - 1) / (s.d_v / n);
  m.q_weight = norm.q_weight; m.k_weight = norm.k_weight;
  // (a weight that is not there has no heads of its own: the heads' places are reckoned from its address)
  m.q_wst = norm.q_weight ? norm.q_head_stride : 0; m.k_wst = norm.k_weight ? norm.k_head_stride : 0;
  m.eps = norm.eps; m.offset = norm.weight_offset; m.inv_d = 1.f / (float)s.d_qk;
  m.lanes_log2 = 0;
  while (m.lanes_log2 < 5 && 1 << m.lanes_log2 < m.tasks) ++m.lanes_log2;
  m.lanes = 1 << m.lanes_log2;
  if (s.dtype == DIFFQKV_F32) return launch<float, float>(p, m, stream);
  return norm.weight_dtype == DIFFQKV_F32 ? launch<__nv_bfloat16, float>(p, m, stream)
                                          : launch<__nv_bfloat16, __nv_bfloat16>(p, m, stream);
}

}  // namespace diffqkv

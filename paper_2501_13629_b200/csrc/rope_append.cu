// Rotary positions for a ragged step, fused with the write of its K and V rows into the cache (diffqkv_rope_append),
// and the host-side frequency tables (diffqkv_rope_frequencies).
//
// Mathematics: channel pair (a, b) number i of the first rot_dim channels of a head is multiplied by
// magnitude * e^(i pos f_i).  The angle pos * f_i reaches 10^5 and more radians, where an fp32 value is spaced 8e-3
// apart, so it is formed in fp64, reduced to [-pi, pi] there (one multiplication by 1 / 2 pi, one rounding to the
// nearest turn, two fused steps with 2 pi split into a high and a low part) and only then handed to sincosf.
//
// Bound by memory: every element of q, k and v is read once and written once.  One block takes a row and computes its
// rot_dim / 2 angles once into shared memory for all n_q + n_k heads (36 heads share an angle with 32/4 heads: computed
// per element the fp64 steps and the sincos would cost more than the traffic).  Its threads move 16-byte vectors, for
// rotate-half pairs the two that hold a channel and its partner; a thread keeps its channels, so that their turns stay in
// registers, and goes from head to head.  The first vectors are read before the row's sequence is known.
// 10.9k rows of 32/4/8 heads of 128 channels, 64 of them turned, neighbouring pairs, bf16 (245 MB): 41 us, 6.0 TB/s;
// rotate-half 56 (over all channels 48).  256 threads took 52 us instead of 42 (half the vectors for the same addresses to
// work out, 3.2 instructions a cycle), without the reads ahead and with a quotient for every vector it was 56 us, with
// several rows to a block one after the other 60.  16 rows: 3.6 us, of which a launch is most.
#include <cmath>

#include "common.cuh"

namespace diffqkv {
namespace {

constexpr int kRopeThreads = 128;

struct RopeParams {
  const void* q;
  const void* k_new;
  const void* v_new;
  void* q_out;
  const int* cu_q;
  int total_q;
  long long q_st, k_st, v_st;  // elements between rows
  const double* inv_freq;
  const int* positions;
  int rot, interleaved;
  float magnitude;
  CacheView cache;
  int batch, n_q, n_k, n_v, d_qk, d_v;
  int* dev_status;
};

template <typename T>
struct Pack;  // 16 bytes of T as floats
template <>
struct Pack<float> {
  static constexpr int N = 4;
  static __device__ void open(const uint4& r, float (&x)[4]) {
    x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
  }
  static __device__ uint4 close(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
template <>
struct Pack<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ void open(const uint4& r, float (&x)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ uint4 close(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// pos * f reduced to [-pi, pi]; |pos f| < 2^31 turns.
__device__ __forceinline__ float reduced_angle(int pos, double f) {
  constexpr double kInvTwoPi = 0.15915494309189533577, kTwoPiHi = 6.2831853071795862, kTwoPiLo = 2.4492935982947064e-16;
  const double a = (double)pos * f;
  const double turns = rint(a * kInvTwoPi);
  return (float)fma(-turns, kTwoPiLo, fma(-turns, kTwoPiHi, a));
}

// kPairs: rotate-half, a vector and the one half a rotation further on together.
template <typename T, bool kPairs>
__global__ void __launch_bounds__(kRopeThreads, kPairs ? 6 : 8) rope_append_kernel(const RopeParams p) {
  constexpr int N = Pack<T>::N;
  constexpr int kVec = kPairs ? 2 : 1;       // vectors of a task
  constexpr int kAhead = kPairs ? 3 : 5;     // tasks read together
  constexpr int kTurns = kPairs ? N : N / 2;
  extern __shared__ float2 turn_s[];  // [rot / 2] (cos, sin) * magnitude
  const int tid = threadIdx.x;
  const int t = blockIdx.x;  // row

  // A thread keeps its channels and goes from head to head: q's, then k's; then the same for V's.  Of a head of very many
  // channels it has several tasks, one after the other.
  const int half = p.rot >> 1;
  const int rot_tasks = kPairs ? half / N : p.rot / N, tasks = rot_tasks + (p.d_qk - p.rot) / N;
  const int span = min(tasks, kRopeThreads), heads_at_once = kRopeThreads / span, first = tid / span;
  const int q_heads = p.q ? p.n_q : 0;
  const int heads = first < heads_at_once ? q_heads + p.n_k : 0;
  const int vvec = p.d_v / N, v_at_once = kRopeThreads / vvec, v_first = tid / vvec, vc = (tid - v_first * vvec) * N;
  const int v_heads = v_first < v_at_once ? p.n_v : 0;

  int x = tid - first * span;
  bool rotated = x < rot_tasks;
  int c0 = rotated ? x * N : p.rot + (x - rot_tasks) * N;  // first channel
  const T* q_row = reinterpret_cast<const T*>(p.q) + t * p.q_st;
  const T* k_row = reinterpret_cast<const T*>(p.k_new) + t * p.k_st;
  const T* v_row = reinterpret_cast<const T*>(p.v_new) + t * p.v_st + vc;
  auto read = [&](int h, uint4 (&a)[kVec]) {
    const T* src = (h < q_heads ? q_row + h * p.d_qk : k_row + (h - q_heads) * p.d_qk) + c0;
    a[0] = *reinterpret_cast<const uint4*>(src);
    if (kPairs && rotated) a[kVec - 1] = *reinterpret_cast<const uint4*>(src + half);
  };
  // The first vectors are on their way while the row's sequence, place and angles are found (reads that depend on one
  // another): they are rows of the caller's whether or not the step has a use for them.
  uint4 ahead[kAhead][kVec], v_ahead;
  auto read_ahead = [&] {
#pragma unroll
    for (int y = 0; y < kAhead; ++y)
      if (first + y * heads_at_once < heads) read(first + y * heads_at_once, ahead[y]);
    if (v_first < v_heads) v_ahead = *reinterpret_cast<const uint4*>(v_row + v_first * p.d_v);
  };
  read_ahead();

  // ---- the row's sequence
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
  float2 turn[kTurns];
  auto finish = [&](int h, uint4 (&raw)[kVec]) {
    T* dst = q_out + h * p.d_qk + c0;
    if (h >= q_heads) {
      if (!place_ok) return;
      dst = k_out + (h - q_heads) * p.cache.k_sh + c0;
    }
    if (rotated) {
      float a[N];
      Pack<T>::open(raw[0], a);
      if (kPairs) {
        float c[N];
        Pack<T>::open(raw[kVec - 1], c);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float2 w = turn[i % kTurns];
          const float u = a[i], v = c[i];
          a[i] = u * w.x - v * w.y;
          c[i] = v * w.x + u * w.y;
        }
        *reinterpret_cast<uint4*>(dst + half) = Pack<T>::close(c);
      } else {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
          const float2 w = turn[i / 2];
          const float u = a[i], v = a[i + 1];
          a[i] = u * w.x - v * w.y;
          a[i + 1] = v * w.x + u * w.y;
        }
      }
      raw[0] = Pack<T>::close(a);
    }
    *reinterpret_cast<uint4*>(dst) = raw[0];
  };
  for (;;) {
#pragma unroll
    for (int i = 0; i < kTurns; ++i)
      if (rotated) turn[i] = turn_s[x * kTurns + i];
    for (int h = first;;) {
#pragma unroll
      for (int y = 0; y < kAhead; ++y)
        if (h + y * heads_at_once < heads) finish(h + y * heads_at_once, ahead[y]);
      h += kAhead * heads_at_once;
      if (h >= heads) break;
#pragma unroll
      for (int y = 0; y < kAhead; ++y)
        if (h + y * heads_at_once < heads) read(h + y * heads_at_once, ahead[y]);
    }
    x += span;
    if (x >= tasks) break;
    rotated = x < rot_tasks;
    c0 = rotated ? x * N : p.rot + (x - rot_tasks) * N;
#pragma unroll
    for (int y = 0; y < kAhead; ++y)
      if (first + y * heads_at_once < heads) read(first + y * heads_at_once, ahead[y]);
  }
}

template <typename T>
cudaError_t launch(const RopeParams& p, cudaStream_t stream) {
  const size_t smem = sizeof(float2) * (p.rot / 2 + 1);
  if (p.interleaved) rope_append_kernel<T, false><<<(unsigned)p.total_q, kRopeThreads, smem, stream>>>(p);
  else rope_append_kernel<T, true><<<(unsigned)p.total_q, kRopeThreads, smem, stream>>>(p);
  count_launch();
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_rope_append(const void* q, const void* k_new, const void* v_new, const int* cu_q, int total_q,
                               long long q_st, long long k_st, long long v_st, const diffqkv_rope& rope,
                               const CacheView& cache, const diffqkv_shape& s, void* q_out, int* dev_status,
                               cudaStream_t stream) {
  RopeParams p;
  p.q = q; p.k_new = k_new; p.v_new = v_new; p.q_out = q_out; p.cu_q = cu_q; p.total_q = total_q;
  p.q_st = q_st ? q_st : (long long)s.n_q * s.d_qk;
  p.k_st = k_st ? k_st : (long long)s.n_k * s.d_qk;
  p.v_st = v_st ? v_st : (long long)s.n_v * s.d_v;
  p.inv_freq = rope.inv_freq; p.positions = rope.positions;
  p.rot = rope.rot_dim; p.interleaved = rope.interleaved != 0; p.magnitude = rope.magnitude;
  p.cache = cache;
  p.batch = s.batch; p.n_q = s.n_q; p.n_k = s.n_k; p.n_v = s.n_v; p.d_qk = s.d_qk; p.d_v = s.d_v;
  p.dev_status = dev_status;
  return s.dtype == DIFFQKV_BF16 ? launch<__nv_bfloat16>(p, stream) : launch<float>(p, stream);
}

bool rope_frequencies(int rot_dim, double theta, int scaling, double s, double L, double fast, double slow,
                      double* inv_freq, float* magnitude) {
  constexpr double kTwoPi = 6.28318530717958647692;
  if (rot_dim <= 0 || rot_dim % 2 != 0 || !(theta > 1.0) || !std::isfinite(theta) || !inv_freq) return false;
  if (scaling < DIFFQKV_ROPE_PLAIN || scaling > DIFFQKV_ROPE_BANDS) return false;
  if (scaling != DIFFQKV_ROPE_PLAIN && (!(s >= 1.0) || !std::isfinite(s))) return false;
  if (scaling == DIFFQKV_ROPE_NTK && rot_dim < 4) return false;  // the exponent rot / (rot - 2)
  const bool ranged = scaling == DIFFQKV_ROPE_YARN || scaling == DIFFQKV_ROPE_BANDS;
  if (ranged && (!(L > 0.0) || !(slow > 0.0) || !(fast > slow) || !std::isfinite(L) || !std::isfinite(fast))) return false;
  double base = theta, lo = 0.0, hi = 1.0;
  if (scaling == DIFFQKV_ROPE_NTK) base = theta * std::pow(s, (double)rot_dim / (rot_dim - 2));
  if (scaling == DIFFQKV_ROPE_YARN) {
    auto channel = [&](double turns) { return rot_dim * std::log(L / (kTwoPi * turns)) / (2.0 * std::log(theta)); };
    lo = std::fmax(std::floor(channel(fast)), 0.0);
    hi = std::fmin(std::ceil(channel(slow)), rot_dim - 1.0);
    if (hi <= lo) hi = lo + 1e-3;
  }
  for (int i = 0; i < rot_dim / 2; ++i) {
    const double f = std::pow(base, -2.0 * i / rot_dim);
    double y = f;
    if (scaling == DIFFQKV_ROPE_LINEAR) {
      y = f / s;
    } else if (scaling == DIFFQKV_ROPE_YARN) {
      const double g = std::fmin(std::fmax((i - lo) / (hi - lo), 0.0), 1.0);
      y = f * (1.0 - g) + f / s * g;
    } else if (scaling == DIFFQKV_ROPE_BANDS) {
      const double turns = L * f / kTwoPi;  // of the trained length
      if (turns < slow) y = f / s;
      else if (turns <= fast) {
        const double t = (turns - slow) / (fast - slow);
        y = (1.0 - t) * f / s + t * f;
      }
    }
    inv_freq[i] = y;
  }
  if (magnitude) *magnitude = scaling == DIFFQKV_ROPE_YARN ? (float)(0.1 * std::log(s) + 1.0) : 1.f;
  return true;
}

}  // namespace diffqkv

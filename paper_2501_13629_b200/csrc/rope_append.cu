// Rotary positions for a ragged step, fused with the write of its K and V rows into the cache (diffqkv_rope_append),
// and the host-side frequency tables (diffqkv_rope_frequencies).
//
// Mathematics: channel pair (a, b) number i of the first rot_dim channels of a head is multiplied by
// magnitude * e^(i pos f_i).  The angle pos * f_i reaches 10^5 and more radians, where an fp32 value is spaced 8e-3
// apart, so it is formed in fp64, reduced to [-pi, pi] there (one multiplication by 1 / 2 pi, one rounding to the
// nearest turn, two fused steps with 2 pi split into a high and a low part) and only then handed to sincosf.
//
// Bound by memory: every element of q, k and v is read once and written once.  One block takes kRows rows and computes
// their rot_dim / 2 angles once into shared memory for all n_q + n_k heads (36 heads share an angle with 32/4 heads:
// computed per element the fp64 steps and the sincos would cost more than the traffic).  Each thread then moves
// 16-byte vectors: for rotate-half pairs the two vectors that hold a channel and its partner, for neighbouring pairs
// one vector; unrotated channels and V rows are plain copies.
#include <cmath>

#include "common.cuh"

namespace diffqkv {
namespace {

constexpr int kRopeThreads = 256;

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

template <typename T, int kRows>
__global__ void __launch_bounds__(kRopeThreads) rope_append_kernel(const RopeParams p) {
  constexpr int N = Pack<T>::N;
  extern __shared__ float2 turn_s[];  // [kRows][rot / 2] (cos, sin) * magnitude
  __shared__ int seq_s[kRows];         // sequence of the row, -1 = not part of the step
  __shared__ int past_s[kRows], place_s[kRows];
  __shared__ int skip_s[kRows];
  const int tid = threadIdx.x;
  const int row0 = blockIdx.x * kRows;

  // ---- the row's sequence: the number of ends cu_q[1 ..] at or below the row, counted by the whole block
  if (tid < kRows) seq_s[tid] = 0;
  __syncthreads();
  {
    int count[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) count[r] = 0;
    for (int b = tid; b < p.batch; b += kRopeThreads) {
      const int end = p.cu_q[b + 1];
#pragma unroll
      for (int r = 0; r < kRows; ++r) count[r] += end <= row0 + r;
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const int c = __reduce_add_sync(0xffffffffu, count[r]);
      if ((tid & 31) == 0 && c) atomicAdd(&seq_s[r], c);
    }
  }
  __syncthreads();
  if (tid < kRows) {
    const int t = row0 + tid;
    int b = t < p.total_q ? seq_s[tid] : p.batch;
    int past = 0, place = 0;
    bool skip = true;
    if (b < p.batch) {
      const int lo = p.cu_q[b], hi = p.cu_q[b + 1];
      past = p.cache.seqlens[b];
      place = t - lo;
      skip = lo < 0 || place < 0 || t >= hi || hi > p.total_q || past < 0 || (long long)past + (hi - lo) > p.cache.max_seqlen;
      if (skip) report(p.dev_status, DIFFQKV_ERR_INDEX);
    }
    seq_s[tid] = b;
    past_s[tid] = past;
    place_s[tid] = place;
    skip_s[tid] = skip;
  }
  __syncthreads();
  const int half = p.rot >> 1;
  for (int e = tid; e < kRows * half; e += kRopeThreads) {
    const int r = e / half, i = e - r * half;
    if (skip_s[r]) continue;
    const int pos = p.positions ? p.positions[row0 + r] : past_s[r] + place_s[r];
    float sn, cs;
    sincosf(reduced_angle(pos, p.inv_freq[i]), &sn, &cs);
    turn_s[e] = make_float2(cs * p.magnitude, sn * p.magnitude);
  }
  __syncthreads();

  // ---- q and k heads: a task is one vector, or two that belong together (rotate-half)
  const int vec = p.d_qk / N;                                   // vectors of a head
  const int rot_vec = p.rot / N;                                // of them rotated
  const int half_vec = half / N;
  const int tasks = p.interleaved ? vec : half_vec + (vec - rot_vec);  // per head
  const int heads = (p.q ? p.n_q : 0) + p.n_k;
  const int vvec = p.d_v / N;
  const int per_row = heads * tasks, per_row_v = p.n_v * vvec;
#pragma unroll 1
  for (int r = 0; r < kRows; ++r) {
    if (skip_s[r]) continue;
    const long long t = row0 + r;
    const int b = seq_s[r], tok = past_s[r] + place_s[r];
    long long blk = b, slot = tok;
    bool place_ok = true;
    if (p.cache.page_table) {
      blk = p.cache.page_table[(long long)b * p.cache.max_pages_per_seq + tok / p.cache.page_size];
      slot = tok % p.cache.page_size;
      if (blk < 0 || blk >= p.cache.num_blocks) {
        place_ok = false;
        if (tid == 0) report(p.dev_status, DIFFQKV_ERR_INDEX);
      }
    }
    const float2* turn = turn_s + r * half;
    for (int e = tid; e < per_row + per_row_v; e += kRopeThreads) {
      if (e >= per_row) {  // a V vector
        const int head = (e - per_row) / vvec, c = (e - per_row) - head * vvec;
        if (place_ok) {
          const uint4 x = *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(p.v_new) + t * p.v_st +
                                                          (long long)head * p.d_v + c * N);
          *reinterpret_cast<uint4*>(reinterpret_cast<T*>(const_cast<void*>(p.cache.v)) + blk * p.cache.v_sb +
                                    head * p.cache.v_sh + slot * p.cache.v_st + c * N) = x;
        }
        continue;
      }
      int head = e / tasks;
      const int task = e - head * tasks;
      const T* src;
      T* dst;
      if (p.q && head < p.n_q) {
        src = reinterpret_cast<const T*>(p.q) + t * p.q_st + (long long)head * p.d_qk;
        dst = reinterpret_cast<T*>(p.q_out) + (t * p.n_q + head) * p.d_qk;
      } else {
        if (!place_ok) continue;
        if (p.q) head -= p.n_q;
        src = reinterpret_cast<const T*>(p.k_new) + t * p.k_st + (long long)head * p.d_qk;
        dst = reinterpret_cast<T*>(const_cast<void*>(p.cache.k)) + blk * p.cache.k_sb + head * p.cache.k_sh +
              slot * p.cache.k_st;
      }
      if (p.interleaved) {
        uint4 raw = *reinterpret_cast<const uint4*>(src + task * N);
        if (task < rot_vec) {
          float x[N];
          Pack<T>::open(raw, x);
#pragma unroll
          for (int i = 0; i < N; i += 2) {
            const float2 w = turn[(task * N + i) >> 1];
            const float a = x[i], c = x[i + 1];
            x[i] = a * w.x - c * w.y;
            x[i + 1] = c * w.x + a * w.y;
          }
          raw = Pack<T>::close(x);
        }
        *reinterpret_cast<uint4*>(dst + task * N) = raw;
      } else if (task < half_vec) {
        const uint4 ra = *reinterpret_cast<const uint4*>(src + task * N);
        const uint4 rb = *reinterpret_cast<const uint4*>(src + half + task * N);
        float a[N], c[N];
        Pack<T>::open(ra, a);
        Pack<T>::open(rb, c);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float2 w = turn[task * N + i];
          const float u = a[i], v = c[i];
          a[i] = u * w.x - v * w.y;
          c[i] = v * w.x + u * w.y;
        }
        *reinterpret_cast<uint4*>(dst + task * N) = Pack<T>::close(a);
        *reinterpret_cast<uint4*>(dst + half + task * N) = Pack<T>::close(c);
      } else {
        const int c = p.rot + (task - half_vec) * N;
        *reinterpret_cast<uint4*>(dst + c) = *reinterpret_cast<const uint4*>(src + c);
      }
    }
  }
}

template <typename T>
cudaError_t launch(const RopeParams& p, cudaStream_t stream) {
  constexpr int kRows = 1;
  const unsigned grid = (unsigned)((p.total_q + kRows - 1) / kRows);
  rope_append_kernel<T, kRows><<<grid, kRopeThreads, sizeof(float2) * kRows * (p.rot / 2 + 1), stream>>>(p);
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

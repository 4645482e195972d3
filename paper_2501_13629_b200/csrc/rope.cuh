// What the kernels that rotate a ragged step's rows and write them into the cache share (rope_append.cu, norm_rope.cu).
#pragma once

#include "common.cuh"

namespace diffqkv {

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

inline RopeParams rope_params(const void* q, const void* k_new, const void* v_new, const int* cu_q, int total_q,
                              long long q_st, long long k_st, long long v_st, const diffqkv_rope& rope,
                              const CacheView& cache, const diffqkv_shape& s, void* q_out, int* dev_status) {
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
  return p;
}

}  // namespace diffqkv

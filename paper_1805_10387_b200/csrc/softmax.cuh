// Softmax sums over rows of FP16 logits, and the words of a row, as the losses and the token scores use them.
#pragma once

#include "rows.cuh"

namespace softmax {

// ---- softmax statistics in powers of two ----
//
// exp(z) = 2^(z log2 e) (`scale`: log2 e over a temperature).  A partial sum over some of a row's logits is kept as s * 2^k with an INTEGER k near
// the largest z log2 e of its part: z log2 e - k is then one fused operation with one rounding, and
// partial sums are brought to a common k by exact powers of two.
struct Sum2 {
  int k;
  float s;
};
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kNothing = -(1 << 30);             // k of a part of -inf alone: below every other k
constexpr uint32_t kNegInf2 = 0xFC00FC00u;       // two FP16 -inf: what stands for words past the vocabulary

__device__ __forceinline__ float ex2(float x) {   // 2 units in the last place; 0 below the normal range
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Joins the sums of LANES neighbouring lanes; every lane gets the same bits.
template <int LANES>
__device__ __forceinline__ Sum2 join_lanes(Sum2 v) {
  int k;
  if constexpr (LANES == 32) {
    k = __reduce_max_sync(0xFFFFFFFFu, v.k);
  } else {
    k = v.k;
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) k = max(k, __shfl_xor_sync(0xFFFFFFFFu, k, o));
  }
  float s = v.s * ex2((float)(v.k - k));
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  return Sum2{k, s};
}

// A thread's largest word, vector by vector, and the k that goes with it.
__device__ __forceinline__ __half2 max8(__half2 m2, const uint4& z) {
  const uint32_t w[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) m2 = __hmax2(m2, *reinterpret_cast<const __half2*>(&w[j]));
  return m2;
}
struct Top {
  float k;
  bool infinite;
};
__device__ __forceinline__ Top top_of(__half2 m2) {
  const float2 m = __half22float2(m2);
  const float top = fmaxf(m.x, m.y);              // a NaN is lost here, and found again by the sum
  return Top{top == -INFINITY ? (float)kNothing : rintf(top * kLog2e), top == INFINITY};
}
__device__ __forceinline__ float sum8(const uint4& z, float k, float scale = kLog2e) {
  const uint32_t w[4] = {z.x, z.y, z.z, z.w};
  float s[2] = {0.0f, 0.0f};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
    s[0] += ex2(fmaf(f.x, scale, -k));
    s[1] += ex2(fmaf(f.y, scale, -k));
  }
  return s[0] + s[1];
}
// A logit of +inf leaves no distribution: inf - inf made the sum a NaN.
__device__ __forceinline__ Sum2 sum_of(Top t, float s) { return Sum2{t.infinite ? 0 : (int)t.k, s}; }
// The sum over a thread's words in one pass: k follows the first vector's largest word and is raised only
// when a word passes it by 2^64, so almost no vector pays for a change.
struct Running {
  float k = 0.0f, s = 0.0f;
  bool begun = false, infinite = false;
  __device__ __forceinline__ void add(const uint4& z, float scale = kLog2e) {
    const float2 m = __half22float2(max8(__half2half2(__ushort_as_half(0xFC00)), z));
    const float top = fmaxf(m.x, m.y);
    if (!begun || fmaf(top, scale, -k) > 64.0f) {
      const float up = top == -INFINITY ? (float)kNothing : rintf(top * scale);
      s = begun ? s * ex2(k - up) : 0.0f;
      k = up;
      begun = true;
      infinite |= top == INFINITY;
    }
    s += sum8(z, k, scale);
  }
  __device__ __forceinline__ Sum2 sum() const { return begun ? Sum2{infinite ? 0 : (int)k, s} : Sum2{kNothing, 0.0f}; }
};
// Sum over the words of C vectors of a thread.
template <int C>
__device__ __forceinline__ Sum2 thread_sum(const uint4 (&z)[C]) {
  __half2 m2 = __half2half2(__ushort_as_half(0xFC00));
#pragma unroll
  for (int c = 0; c < C; ++c) m2 = max8(m2, z[c]);
  const Top t = top_of(m2);
  float s = 0.0f;
#pragma unroll
  for (int c = 0; c < C; ++c) s += sum8(z[c], t.k);
  return sum_of(t, s);
}

__device__ __forceinline__ void store_words(uint16_t* dz, const uint4& q, int nv) {   // the first nv of eight words
  if (nv >= 8) {
    __stcs(reinterpret_cast<uint4*>(dz), q);
    return;
  }
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < nv) dz[j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
}
__device__ __forceinline__ bool nonfinite8(const uint4& q, int nv) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
  bool bad = false;
#pragma unroll
  for (int j = 0; j < 8; ++j) bad |= j < nv && rows::nonfinite16((uint16_t)(w[j / 2] >> (16 * (j & 1))));
  return bad;
}
// The first nv of eight words; -inf for the others.
__device__ __forceinline__ uint4 live8(uint4 q, int nv) {
  if (nv >= 8) return q;
  uint32_t* w = reinterpret_cast<uint32_t*>(&q);
#pragma unroll
  for (int j = 0; j < 4; ++j)
    w[j] = nv >= 2 * j + 2 ? w[j] : nv == 2 * j + 1 ? (w[j] & 0xFFFFu) | 0xFC000000u : kNegInf2;
  return q;
}
__device__ __forceinline__ uint4 no_words() { return make_uint4(kNegInf2, kNegInf2, kNegInf2, kNegInf2); }

}  // namespace softmax

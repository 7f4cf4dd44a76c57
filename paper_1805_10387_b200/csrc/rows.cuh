// Device helpers of the token-model kernels: FP16 words, reductions over a warp and a block, and
// the device-side record of a bad token id.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "common.h"

namespace rows {

__device__ __forceinline__ float h2f(uint16_t h) { return __half2float(__ushort_as_half(h)); }
__device__ __forceinline__ uint16_t f2h(float x) { return __half_as_ushort(__float2half_rn(x)); }
__device__ __forceinline__ bool nonfinite16(uint16_t h) { return (h & 0x7C00u) == 0x7C00u; }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}

// Sum over a block of WARPS full warps, the same value in every thread.  `sm` holds WARPS floats;
// the warps' sums are added in the order of the warps, so the result does not depend on timing.
template <int WARPS>
__device__ __forceinline__ float block_sum(float v, float* sm) {
  v = warp_sum(v);
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
  __syncthreads();
  float t = 0.0f;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) t += sm[w];
  __syncthreads();                       // sm may be written again
  return t;
}

// ---- rows split over groups of TPR threads (8 .. 1024, a power of two) ----
//
// Sum of N values over the threads of a group, the same in every thread of it.  Groups of at most 32
// threads stay inside a warp (every lane of the warp must call); larger ones exchange the warps'
// sums through `red` (red_floats for each group) and a barrier of their own.  Two calls in a
// row use the two halves of `red`: a warp that reaches the call after next has passed the next
// call's barrier, so everyone has read this call's values.
template <int TPR, int N>
constexpr int red_floats = TPR > 32 ? 2 * (TPR / 32) * N : 1;
template <int TPR, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float* red, int& parity) {
#pragma unroll
  for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
  if constexpr (TPR > 32) {
    constexpr int W = TPR / 32;
    const int warp = (threadIdx.x % TPR) >> 5;
    float* half = red + parity * W * N;
    parity ^= 1;
    if ((threadIdx.x & 31) == 0)
#pragma unroll
      for (int k = 0; k < N; ++k) half[warp * N + k] = v[k];
    asm volatile("bar.sync %0, %1;" ::"r"(1 + (int)threadIdx.x / TPR), "n"(TPR) : "memory");
#pragma unroll
    for (int k = 0; k < N; ++k) {
      float t = half[k];
#pragma unroll
      for (int w = 1; w < W; ++w) t += half[w * N + k];
      v[k] = t;
    }
  }
}

// Eight consecutive elements of a row as loaded: 16 bytes of FP16 or 32 of FP32.  `nv` (0 .. 8) of
// them lie inside the row; the others are made zero, whatever the padding holds.
template <class T> struct Raw8;
template <> struct Raw8<uint16_t> {
  uint4 q;
  __device__ __forceinline__ void load(const uint16_t* p, int nv) {
    q = nv > 0 ? __ldcs(reinterpret_cast<const uint4*>(p)) : make_uint4(0, 0, 0, 0);
    keep(nv);
  }
  __device__ __forceinline__ void load_cached(const uint16_t* p, int nv) {
    q = nv > 0 ? __ldg(reinterpret_cast<const uint4*>(p)) : make_uint4(0, 0, 0, 0);
    keep(nv);
  }
  __device__ __forceinline__ void keep(int nv) {
    if (nv >= 8) return;
    uint32_t* w = reinterpret_cast<uint32_t*>(&q);
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] &= nv >= 2 * j + 2 ? 0xFFFFFFFFu : nv == 2 * j + 1 ? 0x0000FFFFu : 0u;
  }
  __device__ __forceinline__ void floats(float (&f)[8]) const {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
      f[2 * j] = t.x;
      f[2 * j + 1] = t.y;
    }
  }
};
template <> struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p, int nv) {   // pitches are multiples of 4: no half past nv
    a = nv > 0 ? __ldcs(reinterpret_cast<const float4*>(p)) : make_float4(0, 0, 0, 0);
    b = nv > 4 ? __ldcs(reinterpret_cast<const float4*>(p) + 1) : make_float4(0, 0, 0, 0);
    keep(nv);
  }
  __device__ __forceinline__ void keep(int nv) {
    if (nv >= 8) return;
    float* f = reinterpret_cast<float*>(this);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = nv > j ? f[j] : 0.0f;
  }
  __device__ __forceinline__ void floats(float (&f)[8]) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
};
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  return make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
}
// Stores the first nv of eight elements.
__device__ __forceinline__ void store8(uint16_t* p, const float (&f)[8], int nv) {
  if (nv >= 8) {
    __stcs(reinterpret_cast<uint4*>(p), pack8(f));
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < nv) p[j] = f2h(f[j]);
}
__device__ __forceinline__ void store8(float* p, const float (&f)[8], int nv) {
  if (nv >= 8) {
    __stcs(reinterpret_cast<float4*>(p), make_float4(f[0], f[1], f[2], f[3]));
    __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(f[4], f[5], f[6], f[7]));
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < nv) p[j] = f[j];
}

// Token id i of a buffer of 4- or 8-byte integers.
template <class ID>
__device__ __forceinline__ int64_t load_id(const void* ids, int64_t i) {
  return (int64_t) reinterpret_cast<const ID*>(ids)[i];
}
__device__ __forceinline__ void record_bad_id(mp_dev_state* st) {
  if (st != nullptr) atomicCAS(&st->h.status, 0, (int)MP_ERR_INVALID_ARG);
}

}  // namespace rows

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
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
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
template <int WARPS>
__device__ __forceinline__ float block_max(float v, float* sm) {
  v = warp_max(v);
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
  __syncthreads();
  float t = sm[0];
#pragma unroll
  for (int w = 1; w < WARPS; ++w) t = fmaxf(t, sm[w]);
  __syncthreads();
  return t;
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

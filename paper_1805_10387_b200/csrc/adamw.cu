// AdamW over the tensors of a plan, states in 32 or in 8 bits, on the FP32 master.
//
// As in the Adam update beside it every operation is one individually rounded FP32 operation, so the
// result does not depend on what the compiler would contract.

#include <cuda_fp8.h>
#include <math.h>
#include <string.h>

#include <map>
#include <mutex>
#include <new>
#include <utility>
#include <vector>

#include "rows.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kBlock = MP_ADAMW_BLOCK;          // elements of one scale of the 8-bit states
constexpr float kTop = 448.0f;                  // largest E4M3 number
constexpr float kTiny = 0.001953125f;           // smallest E4M3 number above 0, 2^-9
constexpr float kNoScale = 7.888609052210118e-31f;   // 2^-100

struct Tensor {
  const uint16_t* g16;
  float* w32;
  void* m;
  void* v;
  uint16_t* w16;
  float* m_scale;
  float* v_scale;
  int64_t count;
  int64_t block_end;                            // blocks of this tensor and of those before it
  float decay;
};
struct Coef {
  float inv_s, b1, omb1, b2, omb2, decay, alpha, k2, eps;
};

// b^t by squaring, in FP64: an error of some 2 log2(t) units in the last place, and a fraction of pow's latency,
// which every block would wait for.
__device__ __forceinline__ double power(double b, int64_t t) {
  double r = 1.0;
  for (; t > 0; t >>= 1, b *= b)
    if (t & 1) r *= b;
  return r;
}
__device__ __forceinline__ Coef coefficients(const mp_dev_state* st, const mp_adamw_config& o) {
  const int64_t t = st->h.t + 1;
  const double c1 = 1.0 - power(o.beta1, t), c2 = 1.0 - power(o.beta2, t);
  Coef c;
  c.inv_s = __fdiv_rn(1.0f, st->h.scale);
  c.b1 = (float)o.beta1;
  c.omb1 = (float)(1.0 - o.beta1);
  c.b2 = (float)o.beta2;
  c.omb2 = (float)(1.0 - o.beta2);
  c.decay = (float)(o.lr * o.weight_decay);
  c.alpha = (float)(o.lr / c1);
  c.k2 = (float)(1.0 / sqrt(c2));
  c.eps = (float)o.eps;
  return c;
}

// One element: m and v in, m, v and r = sqrt(v) out; w is stepped.
__device__ __forceinline__ void step_one(float g16f, float& w, float& m, float& v, float& r, float decay, const Coef& c) {
  const float g = __fmul_rn(g16f, c.inv_s);
  m = __fadd_rn(__fmul_rn(c.b1, m), __fmul_rn(c.omb1, g));
  v = __fadd_rn(__fmul_rn(c.b2, v), __fmul_rn(c.omb2, __fmul_rn(g, g)));
  r = __fsqrt_rn(v);
  w = __fsub_rn(w, __fmul_rn(decay, w));
  w = __fsub_rn(w, __fmul_rn(c.alpha, __fdiv_rn(m, __fadd_rn(__fmul_rn(r, c.k2), c.eps))));
}

// Eight E4M3 numbers as loaded.
__device__ __forceinline__ void from_e4m3(uint2 q, float (&f)[8]) {
  const uint32_t w[2] = {q.x, q.y};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[j / 2] >> (16 * (j & 1))), __NV_E4M3);
    const float2 x = __half22float2(__half2(h));
    f[2 * j] = x.x;
    f[2 * j + 1] = x.y;
  }
}
__device__ __forceinline__ uint2 to_e4m3(const float (&f)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    w[j] = __nv_cvt_float2_to_fp8x2(make_float2(f[2 * j], f[2 * j + 1]), __NV_SATFINITE, __NV_E4M3);
  return make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
}
// The largest of a warp's non-negative values: their order is that of their bits.
__device__ __forceinline__ float warp_top(float v) {
  return __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(v)));
}

// The blocks of 256 elements that a thread block owns are one contiguous range; its warps take them in turn.
// `f` gets the tensor, the block's number in it and the elements of this lane (0 .. 8).
template <class F>
__device__ __forceinline__ void for_my_blocks(const Tensor* tensors, int n_tensors, int64_t n_blocks, F f) {
  const int64_t per = (n_blocks + gridDim.x - 1) / gridDim.x, begin = blockIdx.x * per;
  const int64_t end = begin + per < n_blocks ? begin + per : n_blocks;
  int64_t x = begin + (threadIdx.x >> 5);
  if (x >= end) return;
  int lo = 0;                                   // first tensor whose blocks end after x (the last one's end after all)
  for (int hi = n_tensors - 1; lo < hi;) {
    const int mid = (lo + hi) / 2;
    if (__ldg(&tensors[mid].block_end) > x) hi = mid;
    else lo = mid + 1;
  }
  for (; x < end; x += kThreads / 32) {
    while (__ldg(&tensors[lo].block_end) <= x) ++lo;
    const Tensor& T = tensors[lo];
    const int64_t b = x - (__ldg(&T.block_end) - (__ldg(&T.count) + kBlock - 1) / kBlock);
    const int64_t left = __ldg(&T.count) - b * kBlock - (threadIdx.x & 31) * 8;
    f(T, b, left >= 8 ? 8 : left < 0 ? 0 : (int)left);
  }
}

__global__ void __launch_bounds__(kThreads)
mp_adamw_check_kernel(const Tensor* tensors, int n_tensors, int64_t n_blocks, mp_dev_state* st) {
  bool bad = false;
  for_my_blocks(tensors, n_tensors, n_blocks, [&](const Tensor& T, int64_t b, int nv) {
    rows::Raw8<uint16_t> g;
    g.load(T.g16 + b * kBlock + (threadIdx.x & 31) * 8, nv);
    auto both = [](uint32_t v) { return (v & 0x7C00u) == 0x7C00u || (v & 0x7C000000u) == 0x7C000000u; };
    bad |= both(g.q.x) || both(g.q.y) || both(g.q.z) || both(g.q.w);
  });
  if (bad) atomicOr(&st->h.found_inf, 1);
}

// A lane takes 8 consecutive elements, so a warp takes a block of 256 that shares one scale and finds the
// block's largest magnitude among its own registers: the states are read and written once, in place.
template <int BITS>
__global__ void __launch_bounds__(kThreads)
mp_adamw_update_kernel(const Tensor* tensors, int n_tensors, int64_t n_blocks, const mp_dev_state* st, mp_adamw_config o,
                       const int* gemm_status) {
  if (st->h.found_inf != 0 || st->h.status != 0 || *gemm_status != 0) return;
  __shared__ Coef s_c;
  if (threadIdx.x == 0) s_c = coefficients(st, o);
  __syncthreads();
  const Coef c = s_c;
  for_my_blocks(tensors, n_tensors, n_blocks, [&](const Tensor& T, int64_t b, int nv) {
    const int64_t i = b * kBlock + (threadIdx.x & 31) * 8;
    rows::Raw8<uint16_t> gr;
    rows::Raw8<float> wr;
    float g[8], w[8], m[8], v[8], r[8];
    gr.load(T.g16 + i, nv);
    wr.load(T.w32 + i, nv);
    if constexpr (BITS == 32) {
      rows::Raw8<float> mr, vr;
      mr.load((const float*)T.m + i, nv);
      vr.load((const float*)T.v + i, nv);
      mr.floats(m);
      vr.floats(v);
    } else {
      uint2 mq = make_uint2(0, 0), vq = mq;
      if (nv > 0) {
        mq = __ldcs(reinterpret_cast<const uint2*>((const uint8_t*)T.m + i));
        vq = __ldcs(reinterpret_cast<const uint2*>((const uint8_t*)T.v + i));
      }
      const float ms = T.m_scale[b], vs = T.v_scale[b];
      from_e4m3(mq, m);
      from_e4m3(vq, r);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        m[j] = __fmul_rn(m[j], ms);
        r[j] = __fmul_rn(r[j], vs);
        v[j] = __fmul_rn(r[j], r[j]);
      }
    }
    gr.floats(g);
    wr.floats(w);
    const float decay = __fmul_rn(c.decay, T.decay);
#pragma unroll
    for (int j = 0; j < 8; ++j) step_one(g[j], w[j], m[j], v[j], r[j], decay, c);
    rows::store8(T.w32 + i, w, nv);
    rows::store8(T.w16 + i, w, nv);
    if constexpr (BITS == 32) {
      rows::store8((float*)T.m + i, m, nv);
      rows::store8((float*)T.v + i, v, nv);
    } else {
      // what lies past the tensor's end has no say in the scale and is not stored
      float tm = 0.0f, tr = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        tm = j < nv ? fmaxf(tm, fabsf(m[j])) : tm;
        tr = j < nv ? fmaxf(tr, r[j]) : tr;
      }
      tm = warp_top(tm);
      tr = warp_top(tr);
      const float im = tm < kNoScale ? 0.0f : __fdiv_rn(kTop, tm), ir = tr < kNoScale ? 0.0f : __fdiv_rn(kTop, tr);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        m[j] = __fmul_rn(m[j], im);
        r[j] = r[j] > 0.0f && ir > 0.0f ? fmaxf(__fmul_rn(r[j], ir), kTiny) : 0.0f;
      }
      const uint2 mq = to_e4m3(m), vq = to_e4m3(r);
      uint8_t *mp_ = (uint8_t*)T.m + i, *vp = (uint8_t*)T.v + i;
      if (nv == 8) {
        __stcs(reinterpret_cast<uint2*>(mp_), mq);
        __stcs(reinterpret_cast<uint2*>(vp), vq);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < nv) {
            mp_[j] = (uint8_t)((j < 4 ? mq.x : mq.y) >> (8 * (j & 3)));
            vp[j] = (uint8_t)((j < 4 ? vq.x : vq.y) >> (8 * (j & 3)));
          }
      }
      if ((threadIdx.x & 31) == 0) {
        T.m_scale[b] = tm < kNoScale ? 0.0f : __fdiv_rn(tm, kTop);
        T.v_scale[b] = tr < kNoScale ? 0.0f : __fdiv_rn(tr, kTop);
      }
    }
  });
}

// Blocks of `kernel` that are resident at once on the current device, asked once per device and kernel.
int resident_blocks(const void* kernel, int* out) {
  static std::mutex mu;
  static std::map<std::pair<int, const void*>, int> cache;
  int dev = 0;
  MP_CUDA_TRY(cudaGetDevice(&dev));
  std::lock_guard<std::mutex> lock(mu);
  int& have = cache[{dev, kernel}];
  if (have == 0) {
    int sms = 0, per = 0;
    MP_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    MP_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kernel, kThreads, 0));
    have = sms * (per < 1 ? 1 : per);
  }
  *out = have;
  return MP_OK;
}

}  // namespace

struct mp_adamw_plan {
  Tensor* d_tensors;
  int n_tensors;                                // with elements
  int64_t n_blocks;
  int bits;
};

extern "C" {

int mp_adamw_plan_create(int n, void* const* g16, void* const* w32, void* const* m, void* const* v,
                         void* const* w16, const int64_t* count, const float* decay, int state_bits,
                         float* const* m_scale, float* const* v_scale, mp_adamw_plan** out) {
  const char* name = "mp_adamw_plan_create";
  if (n <= 0 || !g16 || !w32 || !m || !v || !w16 || !count || !out)
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: null argument or n <= 0", name);
  if ((state_bits != 32 && state_bits != 8) || (state_bits == 8) != (m_scale != nullptr) ||
      (state_bits == 8) != (v_scale != nullptr))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: states have 32 bits, or 8 bits with scales", name);
  for (int i = 0; i < n; ++i) {
    if (count[i] < 0) return mp::set_error(MP_ERR_INVALID_ARG, "%s: count[%d] < 0", name, i);
    if (decay && !isfinite(decay[i])) return mp::set_error(MP_ERR_INVALID_ARG, "%s: decay[%d] is not finite", name, i);
    if (count[i] == 0) continue;
    if (!g16[i] || !w32[i] || !m[i] || !v[i] || !w16[i] || (state_bits == 8 && (!m_scale[i] || !v_scale[i])))
      return mp::set_error(MP_ERR_INVALID_ARG, "%s: tensor %d has a null buffer", name, i);
    if (!mp::aligned16(g16[i]) || !mp::aligned16(w32[i]) || !mp::aligned16(m[i]) || !mp::aligned16(v[i]) ||
        !mp::aligned16(w16[i]) ||
        (state_bits == 8 && (((uintptr_t)m_scale[i] | (uintptr_t)v_scale[i]) & 3)))
      return mp::set_error(MP_ERR_ALIGNMENT, "%s: tensor %d is not 16-byte aligned (scales: 4)", name, i);
  }
  if (int rc = mp::check_device()) return rc;
  mp_adamw_plan* p = new (std::nothrow) mp_adamw_plan();
  if (!p) return mp::set_error(MP_ERR_NOMEM, "%s: host allocation failed", name);
  p->bits = state_bits;
  try {
    std::vector<Tensor> ts;
    for (int i = 0; i < n; ++i) {                // a tensor without elements has no place in the table
      if (count[i] == 0) continue;
      p->n_blocks += (count[i] + kBlock - 1) / kBlock;
      ts.push_back(Tensor{(const uint16_t*)g16[i], (float*)w32[i], m[i], v[i], (uint16_t*)w16[i],
                          m_scale ? m_scale[i] : nullptr, v_scale ? v_scale[i] : nullptr, count[i], p->n_blocks,
                          decay ? decay[i] : 1.0f});
    }
    p->n_tensors = (int)ts.size();
    const size_t bytes = ts.size() * sizeof(Tensor);
    if (cudaMalloc(&p->d_tensors, bytes ? bytes : 1) != cudaSuccess) {
      mp_adamw_plan_destroy(p);
      return mp::set_error(MP_ERR_NOMEM, "%s: device allocation failed", name);
    }
    const cudaError_t e = bytes ? cudaMemcpy(p->d_tensors, ts.data(), bytes, cudaMemcpyHostToDevice) : cudaSuccess;
    if (e != cudaSuccess) {
      mp_adamw_plan_destroy(p);
      return mp::set_error(MP_ERR_CUDA, "%s: %s", name, cudaGetErrorString(e));
    }
  } catch (const std::bad_alloc&) {
    mp_adamw_plan_destroy(p);
    return mp::set_error(MP_ERR_NOMEM, "%s: host allocation failed", name);
  }
  *out = p;
  return MP_OK;
}

int mp_adamw_plan_destroy(mp_adamw_plan* p) {
  if (!p) return MP_OK;
  cudaFree(p->d_tensors);
  delete p;
  return MP_OK;
}

int mp_adamw_update(mp_adamw_plan* plan, mp_state* state, const mp_adamw_config* opt, int check_mode, void* stream) {
  if (!plan || !state || !opt) return mp::set_error(MP_ERR_INVALID_ARG, "mp_adamw_update: null argument");
  if (check_mode != 0 && check_mode != 1)
    return mp::set_error(MP_ERR_INVALID_ARG, "mp_adamw_update: check_mode must be 0 or 1");
  if (int rc = mp::check_device()) return rc;
  if (plan->n_blocks == 0) return MP_OK;
  cudaStream_t st = (cudaStream_t)stream;
  int* gemm_status = nullptr;
  if (int rc = mp::gemm_status_device_ptr(&gemm_status)) return rc;
  // one resident round of blocks; a block has work for each of its warps
  auto grid_of = [&](const void* kernel, int* grid) {
    if (int rc = resident_blocks(kernel, grid)) return rc;
    const int64_t want = (plan->n_blocks + kThreads / 32 - 1) / (kThreads / 32);
    if (want < *grid) *grid = (int)want;
    return (int)MP_OK;
  };
  int grid = 0;
  if (check_mode == 1) {
    if (int rc = grid_of((const void*)mp_adamw_check_kernel, &grid)) return rc;
    mp_adamw_check_kernel<<<grid, kThreads, 0, st>>>(plan->d_tensors, plan->n_tensors, plan->n_blocks, state->dev);
    mp::count_launch();
  }
  auto kernel = plan->bits == 32 ? mp_adamw_update_kernel<32> : mp_adamw_update_kernel<8>;
  if (int rc = grid_of((const void*)kernel, &grid)) return rc;
  kernel<<<grid, kThreads, 0, st>>>(plan->d_tensors, plan->n_tensors, plan->n_blocks, state->dev, *opt, gemm_status);
  mp::count_launch();
  MP_CUDA_TRY(cudaGetLastError());
  return MP_OK;
}

}  // extern "C"

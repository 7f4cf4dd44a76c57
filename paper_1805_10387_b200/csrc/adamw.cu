// AdamW over the tensors of a plan, states in 32 or in 8 bits, on the FP32 master.
//
// As in the Adam update beside it every operation is one individually rounded FP32 operation, so the
// result does not depend on what the compiler would contract.

#include <cuda_fp8.h>
#include <math.h>
#include <string.h>

#include <new>
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
  float decay;
};
struct Piece {
  int32_t tensor, block;                        // kBlock elements from block * kBlock on
};
struct Coef {
  float inv_s, b1, omb1, b2, omb2, decay, alpha, k2, eps;
};

__device__ __forceinline__ Coef coefficients(const mp_dev_state* st, const mp_adamw_config& o) {
  const double t = (double)(st->h.t + 1);
  const double c1 = 1.0 - pow(o.beta1, t), c2 = 1.0 - pow(o.beta2, t);
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

__device__ __forceinline__ float from_e4m3(uint8_t q) {
  const __half_raw h = __nv_cvt_fp8_to_halfraw(q, __NV_E4M3);
  return __half2float(__half(h));
}
__device__ __forceinline__ uint8_t to_e4m3(float x) {
  return __nv_cvt_float_to_fp8(x, __NV_SATFINITE, __NV_E4M3);
}

__global__ void __launch_bounds__(kThreads)
mp_adamw_check_kernel(const Tensor* tensors, const Piece* pieces, int64_t n_pieces, mp_dev_state* st) {
  bool bad = false;
  for (int64_t p = blockIdx.x; p < n_pieces; p += gridDim.x) {
    const Tensor& T = tensors[pieces[p].tensor];
    const int64_t i = (int64_t)pieces[p].block * kBlock + threadIdx.x;
    bad |= i < T.count && rows::nonfinite16(T.g16[i]);
  }
  if (bad) atomicOr(&st->h.found_inf, 1);
}

// One thread per element of a piece.
template <int BITS>
__global__ void __launch_bounds__(kThreads)
mp_adamw_update_kernel(const Tensor* tensors, const Piece* pieces, int64_t n_pieces, const mp_dev_state* st,
                       mp_adamw_config o, const int* gemm_status) {
  if (st->h.found_inf != 0 || st->h.status != 0 || *gemm_status != 0) return;
  __shared__ Coef s_c;
  __shared__ float red[kThreads / 32];
  if (threadIdx.x == 0) s_c = coefficients(st, o);
  __syncthreads();
  const Coef c = s_c;
  for (int64_t p = blockIdx.x; p < n_pieces; p += gridDim.x) {
    const Tensor& T = tensors[pieces[p].tensor];
    const int64_t b = pieces[p].block, i = b * kBlock + threadIdx.x;
    const bool in = i < T.count;
    float w = 0.0f, m = 0.0f, v = 0.0f, r = 0.0f;
    if (in) {
      w = T.w32[i];
      if (BITS == 32) {
        m = ((const float*)T.m)[i];
        v = ((const float*)T.v)[i];
      } else {
        m = __fmul_rn(from_e4m3(((const uint8_t*)T.m)[i]), T.m_scale[b]);
        r = __fmul_rn(from_e4m3(((const uint8_t*)T.v)[i]), T.v_scale[b]);
        v = __fmul_rn(r, r);
      }
      step_one(rows::h2f(T.g16[i]), w, m, v, r, __fmul_rn(c.decay, T.decay), c);
      T.w32[i] = w;
      T.w16[i] = rows::f2h(w);
    }
    if (BITS == 32) {
      if (in) {
        ((float*)T.m)[i] = m;
        ((float*)T.v)[i] = v;
      }
    } else {
      const float tm = rows::block_max<kThreads / 32>(fabsf(m), red), tr = rows::block_max<kThreads / 32>(r, red);
      const float im = tm < kNoScale ? 0.0f : __fdiv_rn(kTop, tm), ir = tr < kNoScale ? 0.0f : __fdiv_rn(kTop, tr);
      if (in) {
        ((uint8_t*)T.m)[i] = to_e4m3(__fmul_rn(m, im));
        ((uint8_t*)T.v)[i] = to_e4m3(r > 0.0f && ir > 0.0f ? fmaxf(__fmul_rn(r, ir), kTiny) : 0.0f);
      }
      if (threadIdx.x == 0) {
        T.m_scale[b] = tm < kNoScale ? 0.0f : __fdiv_rn(tm, kTop);
        T.v_scale[b] = tr < kNoScale ? 0.0f : __fdiv_rn(tr, kTop);
      }
    }
  }
}

}  // namespace

struct mp_adamw_plan {
  Tensor* d_tensors;
  Piece* d_pieces;
  int64_t n_pieces;
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
    if ((count[i] + kBlock - 1) / kBlock > INT32_MAX)
      return mp::set_error(MP_ERR_TOO_LARGE, "%s: tensor %d is too large", name, i);
  }
  if (int rc = mp::check_device()) return rc;
  mp_adamw_plan* p = new (std::nothrow) mp_adamw_plan();
  if (!p) return mp::set_error(MP_ERR_NOMEM, "%s: host allocation failed", name);
  p->bits = state_bits;
  try {
    std::vector<Tensor> ts(n);
    std::vector<Piece> ps;
    for (int i = 0; i < n; ++i) {
      ts[i] = Tensor{(const uint16_t*)g16[i], (float*)w32[i], m[i], v[i], (uint16_t*)w16[i],
                     m_scale ? m_scale[i] : nullptr, v_scale ? v_scale[i] : nullptr, count[i], decay ? decay[i] : 1.0f};
      for (int64_t b = 0; b < (count[i] + kBlock - 1) / kBlock; ++b) ps.push_back(Piece{i, (int32_t)b});
    }
    p->n_pieces = (int64_t)ps.size();
    if (cudaMalloc(&p->d_tensors, n * sizeof(Tensor)) != cudaSuccess ||
        cudaMalloc(&p->d_pieces, (ps.size() ? ps.size() : 1) * sizeof(Piece)) != cudaSuccess) {
      mp_adamw_plan_destroy(p);
      return mp::set_error(MP_ERR_NOMEM, "%s: device allocation failed", name);
    }
    cudaError_t e = cudaMemcpy(p->d_tensors, ts.data(), n * sizeof(Tensor), cudaMemcpyHostToDevice);
    if (e == cudaSuccess && !ps.empty())
      e = cudaMemcpy(p->d_pieces, ps.data(), ps.size() * sizeof(Piece), cudaMemcpyHostToDevice);
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
  cudaFree(p->d_pieces);
  delete p;
  return MP_OK;
}

int mp_adamw_update(mp_adamw_plan* plan, mp_state* state, const mp_adamw_config* opt, int check_mode, void* stream) {
  if (!plan || !state || !opt) return mp::set_error(MP_ERR_INVALID_ARG, "mp_adamw_update: null argument");
  if (check_mode != 0 && check_mode != 1)
    return mp::set_error(MP_ERR_INVALID_ARG, "mp_adamw_update: check_mode must be 0 or 1");
  if (int rc = mp::check_device()) return rc;
  if (plan->n_pieces == 0) return MP_OK;
  cudaStream_t st = (cudaStream_t)stream;
  int* gemm_status = nullptr;
  if (int rc = mp::gemm_status_device_ptr(&gemm_status)) return rc;
  const int grid = (int)(plan->n_pieces < 148 * 8 ? plan->n_pieces : 148 * 8);
  if (check_mode == 1) {
    mp_adamw_check_kernel<<<grid, kThreads, 0, st>>>(plan->d_tensors, plan->d_pieces, plan->n_pieces, state->dev);
    mp::count_launch();
  }
  if (plan->bits == 32)
    mp_adamw_update_kernel<32><<<grid, kThreads, 0, st>>>(plan->d_tensors, plan->d_pieces, plan->n_pieces, state->dev,
                                                          *opt, gemm_status);
  else
    mp_adamw_update_kernel<8><<<grid, kThreads, 0, st>>>(plan->d_tensors, plan->d_pieces, plan->n_pieces, state->dev,
                                                         *opt, gemm_status);
  mp::count_launch();
  MP_CUDA_TRY(cudaGetLastError());
  return MP_OK;
}

}  // extern "C"

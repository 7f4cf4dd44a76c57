// Norms before and after a block, with the block's gate and the residual scale, forward and backward.

#include "rows.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

__device__ __forceinline__ float load_x(const void* p, int x_bytes, int64_t i) {
  return x_bytes == 4 ? reinterpret_cast<const float*>(p)[i] : rows::h2f(reinterpret_cast<const uint16_t*>(p)[i]);
}
__device__ __forceinline__ void store_x(void* p, int x_bytes, int64_t i, float v) {
  if (x_bytes == 4) reinterpret_cast<float*>(p)[i] = v;
  else reinterpret_cast<uint16_t*>(p)[i] = rows::f2h(v);
}

// One block per row, the row's FP32 values in shared memory.
__global__ void __launch_bounds__(kThreads)
mp_block_norm_fwd_kernel(int kind, float eps, float res_scale, const void* x, int x_bytes, int64_t ldx,
                         const uint16_t* y, int64_t ldy, const uint16_t* g_post, const uint16_t* gate, int64_t ldgate,
                         void* x_out, int64_t ldxo, const uint16_t* g_pre, uint16_t* nn, int64_t ldn, float* stats,
                         int64_t M, int D) {
  extern __shared__ float row[];
  __shared__ float red[kWarps];
  for (int64_t m = blockIdx.x; m < M; m += gridDim.x) {
    float mean[2] = {0.0f, 0.0f}, root[2] = {0.0f, 0.0f};
    for (int which = y ? 0 : 1; which < 2; ++which) {
      if (which == 0)
        for (int c = threadIdx.x; c < D; c += kThreads) row[c] = rows::h2f(y[m * ldy + c]);
      else
        for (int c = threadIdx.x; c < D; c += kThreads) {
          float v = load_x(x, x_bytes, m * ldx + c);
          if (y) {
            float h = (row[c] - mean[0]) * root[0] * rows::h2f(g_post[c]);
            if (gate) h *= rows::h2f(gate[m * ldgate + c]);
            v = res_scale * v + h;
            store_x(x_out, x_bytes, m * ldxo + c, v);
          }
          row[c] = v;
        }
      if (kind == MP_NORM_LAYER) {
        float s = 0.0f;
        for (int c = threadIdx.x; c < D; c += kThreads) s += row[c];
        mean[which] = rows::block_sum<kWarps>(s, red) / (float)D;
      }
      float q = 0.0f;
      for (int c = threadIdx.x; c < D; c += kThreads) {
        const float v = row[c] - mean[which];
        q += v * v;
      }
      root[which] = rsqrtf(rows::block_sum<kWarps>(q, red) / (float)D + eps);
    }
    for (int c = threadIdx.x; c < D; c += kThreads)
      nn[m * ldn + c] = rows::f2h((row[c] - mean[1]) * root[1] * rows::h2f(g_pre[c]));
    if (stats && threadIdx.x == 0)
      reinterpret_cast<float4*>(stats)[m] = make_float4(mean[0], root[0], mean[1], root[1]);
    __syncthreads();
  }
}

// One block per slab of rows; the sums over the rows of its slab (dg_pre, dg_post, dgate) in
// shared memory, written as one partial row each.
__global__ void __launch_bounds__(kThreads)
mp_block_norm_bwd_kernel(int kind, float res_scale, const uint16_t* dn, int64_t lddn, const void* dx_out, int64_t lddxo,
                         const void* x_out, int x_bytes, int64_t ldxo, const uint16_t* y, int64_t ldy,
                         const uint16_t* g_post, const uint16_t* gate, int64_t ldgate, const uint16_t* g_pre,
                         const float* stats, void* dx, int64_t lddx, uint16_t* dy, int64_t lddy, uint16_t* dgate,
                         int64_t lddgate, int64_t M, int D, int64_t rows_per, float* partial) {
  extern __shared__ float sums[];                // dg_pre, dg_post, dgate
  __shared__ float red[kWarps];
  for (int c = threadIdx.x; c < 3 * D; c += kThreads) sums[c] = 0.0f;
  __syncthreads();
  const int64_t r0 = blockIdx.x * rows_per, r1 = r0 + rows_per < M ? r0 + rows_per : M;
  const float inv_d = 1.0f / (float)D;
  for (int64_t m = r0; m < r1; ++m) {
    const float4 st = reinterpret_cast<const float4*>(stats)[m];
    float a = 0.0f, b = 0.0f;
    for (int c = threadIdx.x; c < D; c += kThreads) {
      const float d = rows::h2f(dn[m * lddn + c]) * rows::h2f(g_pre[c]);
      a += d * ((load_x(x_out, x_bytes, m * ldxo + c) - st.z) * st.w);
      b += d;
    }
    a = rows::block_sum<kWarps>(a, red) * inv_d;
    b = kind == MP_NORM_LAYER ? rows::block_sum<kWarps>(b, red) * inv_d : 0.0f;
    auto gx_at = [&](int c, float& xhat, float& dnv) {
      xhat = (load_x(x_out, x_bytes, m * ldxo + c) - st.z) * st.w;
      dnv = rows::h2f(dn[m * lddn + c]);
      const float up = dx_out ? load_x(dx_out, x_bytes, m * lddxo + c) : 0.0f;
      return up + (dnv * rows::h2f(g_pre[c]) - xhat * a - b) * st.w;
    };
    float e = 0.0f, f = 0.0f;
    if (y) {
      for (int c = threadIdx.x; c < D; c += kThreads) {
        float xhat, dnv;
        float dh = gx_at(c, xhat, dnv) * rows::h2f(g_post[c]);
        if (gate) dh *= rows::h2f(gate[m * ldgate + c]);
        e += dh * ((rows::h2f(y[m * ldy + c]) - st.x) * st.y);
        f += dh;
      }
      e = rows::block_sum<kWarps>(e, red) * inv_d;
      f = kind == MP_NORM_LAYER ? rows::block_sum<kWarps>(f, red) * inv_d : 0.0f;
    }
    for (int c = threadIdx.x; c < D; c += kThreads) {
      float xhat, dnv;
      const float gx = gx_at(c, xhat, dnv);
      sums[c] += dnv * xhat;
      if (y) {
        const float yhat = (rows::h2f(y[m * ldy + c]) - st.x) * st.y, gp = rows::h2f(g_post[c]);
        float dh = gx;
        if (gate) {
          const float dg = gx * yhat * gp;
          dh *= rows::h2f(gate[m * ldgate + c]);
          if (ldgate == 0) sums[2 * D + c] += dg;
          else dgate[m * lddgate + c] = rows::f2h(dg);
        }
        sums[D + c] += dh * yhat;
        dy[m * lddy + c] = rows::f2h((dh * gp - yhat * e - f) * st.y);
      }
      store_x(dx, x_bytes, m * lddx + c, y ? res_scale * gx : gx);
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < 3 * D; c += kThreads) partial[(int64_t)blockIdx.x * 3 * D + c] = sums[c];
}

__global__ void __launch_bounds__(kThreads)
mp_block_norm_sum_kernel(const float* partial, int slabs, int D, uint16_t* dg_pre, uint16_t* dg_post, uint16_t* dgate,
                         mp_dev_state* st) {
  const int c = blockIdx.x * kThreads + threadIdx.x;
  if (c >= 3 * D) return;
  uint16_t* out = c < D ? dg_pre : c < 2 * D ? dg_post : dgate;
  if (!out) return;
  float t = 0.0f;
  for (int s = 0; s < slabs; ++s) t += partial[(int64_t)s * 3 * D + c];
  const uint16_t h = rows::f2h(t);
  out[c % D] = h;
  if (st && rows::nonfinite16(h)) atomicOr(&st->h.found_inf, 1);
}

constexpr int64_t kSlabs = 148;

int64_t slabs_for(int64_t M) { return M < kSlabs ? (M > 0 ? M : 1) : kSlabs; }

template <class K>
cudaError_t allow_smem(K kernel, size_t bytes) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

bool bad_ptr16(const void* p) { return p && !mp::aligned16(p); }

}  // namespace

extern "C" {

int mp_block_norm_fwd(int kind, float eps, float res_scale, const void* x, int x_bytes, int64_t ldx,
                      const void* y16, int64_t ldy, const void* g_post16, const void* gate16, int64_t ldgate,
                      void* x_out, int64_t ldxo, const void* g_pre16, void* n16, int64_t ldn, float* stats,
                      int64_t M, int64_t D, void* stream) {
  const char* name = "mp_block_norm_fwd";
  if ((kind != MP_NORM_RMS && kind != MP_NORM_LAYER) || (x_bytes != 2 && x_bytes != 4) || M < 0 || D <= 0 ||
      !(eps >= 0.0f) || ldx < D || ldn < D)
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: bad kind, size, pitch or eps", name);
  if (D > MP_NORM_MAX_D) return mp::set_error(MP_ERR_TOO_LARGE, "%s: D beyond %d", name, MP_NORM_MAX_D);
  if (!g_pre16 || (M > 0 && (!x || !n16))) return mp::set_error(MP_ERR_INVALID_ARG, "%s: null pointer", name);
  if (g_post16 ? ((M > 0 && (!y16 || !x_out)) || ldy < D || ldxo < D || (gate16 && ldgate != 0 && ldgate < D))
               : (y16 || x_out || gate16))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: g_post16 goes with y16 and x_out, without it there is no y16, "
                         "x_out or gate16", name);
  const int64_t xm = x_bytes == 4 ? 3 : 7;
  if ((ldx & xm) || (ldn & 7) || (y16 && ((ldy & 7) || (ldxo & xm))) || (gate16 && (ldgate & 7)) || bad_ptr16(x) ||
      bad_ptr16(y16) || bad_ptr16(g_post16) || bad_ptr16(gate16) || bad_ptr16(x_out) || bad_ptr16(g_pre16) ||
      bad_ptr16(n16) || bad_ptr16(stats))
    return mp::set_error(MP_ERR_ALIGNMENT, "%s: buffers must be 16-byte aligned, rows start on 16-byte boundaries", name);
  if (int rc = mp::check_device()) return rc;
  if (M == 0) return MP_OK;
  const int grid = (int)(M < 148 * 8 ? M : 148 * 8);
  const size_t smem = (size_t)D * sizeof(float);
  MP_CUDA_TRY(allow_smem(mp_block_norm_fwd_kernel, smem));
  mp_block_norm_fwd_kernel<<<grid, kThreads, smem, (cudaStream_t)stream>>>(
      kind, eps, res_scale, x, x_bytes, ldx, (const uint16_t*)y16, ldy, (const uint16_t*)g_post16,
      (const uint16_t*)gate16, ldgate, x_out, ldxo, (const uint16_t*)g_pre16, (uint16_t*)n16, ldn, stats, M, (int)D);
  mp::count_launch();
  MP_CUDA_TRY(cudaGetLastError());
  return MP_OK;
}

size_t mp_block_norm_bwd_workspace_bytes(int64_t M, int64_t D) {
  if (M < 0 || D <= 0 || D > MP_NORM_MAX_D) return 0;
  return (size_t)slabs_for(M) * 3 * (size_t)D * sizeof(float);
}

int mp_block_norm_bwd(int kind, float res_scale, const void* dn16, int64_t lddn, const void* dx_out,
                      int64_t lddxo, const void* x_out, int x_bytes, int64_t ldxo, const void* y16, int64_t ldy,
                      const void* g_post16, const void* gate16, int64_t ldgate, const void* g_pre16,
                      const float* stats, void* dx, int64_t lddx, void* dy16, int64_t lddy, void* dg_post16,
                      void* dgate16, int64_t lddgate, void* dg_pre16, int64_t M, int64_t D, mp_state* state,
                      void* workspace, size_t workspace_bytes, void* stream) {
  const char* name = "mp_block_norm_bwd";
  if ((kind != MP_NORM_RMS && kind != MP_NORM_LAYER) || (x_bytes != 2 && x_bytes != 4) || M < 0 || D <= 0 ||
      lddn < D || ldxo < D || lddx < D || (dx_out && lddxo < D))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: bad kind, size or pitch", name);
  if (D > MP_NORM_MAX_D) return mp::set_error(MP_ERR_TOO_LARGE, "%s: D beyond %d", name, MP_NORM_MAX_D);
  if (!g_pre16 || !dg_pre16 || (M > 0 && (!dn16 || !x_out || !stats || !dx)))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: null pointer", name);
  if (g_post16 ? ((M > 0 && (!y16 || !dy16)) || !dg_post16 || ldy < D || lddy < D ||
                  (gate16 != nullptr) != (dgate16 != nullptr) ||
                  (gate16 && ldgate != 0 && (ldgate < D || lddgate < D)))
               : (y16 || dy16 || dg_post16 || gate16 || dgate16))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: g_post16 goes with y16, dy16 and dg_post16, a gate with its gradient", name);
  const int64_t xm = x_bytes == 4 ? 3 : 7;
  if ((lddn & 7) || (ldxo & xm) || (lddx & xm) || (dx_out && (lddxo & xm)) || (y16 && ((ldy & 7) || (lddy & 7))) ||
      (gate16 && ((ldgate & 7) || (ldgate && (lddgate & 7)))) || bad_ptr16(dn16) || bad_ptr16(dx_out) ||
      bad_ptr16(x_out) || bad_ptr16(y16) || bad_ptr16(g_post16) || bad_ptr16(gate16) || bad_ptr16(g_pre16) ||
      bad_ptr16(stats) || bad_ptr16(dx) || bad_ptr16(dy16) || bad_ptr16(dg_post16) || bad_ptr16(dgate16) ||
      bad_ptr16(dg_pre16) || bad_ptr16(workspace))
    return mp::set_error(MP_ERR_ALIGNMENT, "%s: buffers must be 16-byte aligned, rows start on 16-byte boundaries", name);
  const size_t need = mp_block_norm_bwd_workspace_bytes(M, D);
  if (!workspace || workspace_bytes < need)
    return mp::set_error(MP_ERR_NOMEM, "%s: workspace of %zu bytes needed", name, need);
  if (int rc = mp::check_device()) return rc;
  const int64_t slabs = slabs_for(M), rows_per = (M + slabs - 1) / slabs;
  const size_t smem = (size_t)3 * D * sizeof(float);
  MP_CUDA_TRY(allow_smem(mp_block_norm_bwd_kernel, smem));
  mp_block_norm_bwd_kernel<<<(int)slabs, kThreads, smem, (cudaStream_t)stream>>>(
      kind, res_scale, (const uint16_t*)dn16, lddn, dx_out, lddxo, x_out, x_bytes, ldxo, (const uint16_t*)y16, ldy,
      (const uint16_t*)g_post16, (const uint16_t*)gate16, ldgate, (const uint16_t*)g_pre16, stats, dx, lddx,
      (uint16_t*)dy16, lddy, (uint16_t*)dgate16, lddgate, M, (int)D, rows_per, (float*)workspace);
  MP_CUDA_TRY(cudaGetLastError());
  mp_block_norm_sum_kernel<<<(int)((3 * D + kThreads - 1) / kThreads), kThreads, 0, (cudaStream_t)stream>>>(
      (const float*)workspace, (int)slabs, (int)D, (uint16_t*)dg_pre16, (uint16_t*)dg_post16,
      ldgate == 0 ? (uint16_t*)dgate16 : nullptr, state ? state->dev : nullptr);
  mp::count_launch(2);
  MP_CUDA_TRY(cudaGetLastError());
  return MP_OK;
}

}  // extern "C"

// Clipped policy loss with a KL term, forward and backward, and the token log-probabilities alone.

#include <math.h>

#include "rows.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

struct LossArgs {
  const uint16_t* z;
  int64_t ldl;
  const void* targets;
  const float *old_logp, *ref_logp, *advantage, *weight;
  int64_t N, V;
  float lo, hi, kl, grad_scale;
  uint16_t* dz;
  int64_t lddl;
  float *logp, *token_loss;
  mp_dev_state* st;
};

// Loss of one token and its derivative by the token's log-probability.
__device__ __forceinline__ void token_terms(const LossArgs& a, int64_t i, float lp, float& loss, float& dlp) {
  const float A = a.advantage[i];
  const float r = expf(lp - a.old_logp[i]);
  const float plain = r * A, clipped = fminf(fmaxf(r, 1.0f - a.lo), 1.0f + a.hi) * A;
  loss = plain <= clipped ? -plain : -clipped;
  dlp = plain <= clipped ? -plain : 0.0f;
  if (plain != plain) loss = dlp = plain;          // a NaN shows in the loss and the gradient
  if (a.ref_logp) {
    const float d = a.ref_logp[i] - lp, e = expm1f(d);
    loss += a.kl * (e - d);
    dlp -= a.kl * e;
  }
}

// One block per row, three passes over it.
template <class ID, bool LOSS>
__global__ void __launch_bounds__(kThreads) mp_policy_loss_kernel(const LossArgs a) {
  __shared__ float red[kWarps];
  const float S = a.st ? a.st->h.scale : 1.0f;
  for (int64_t i = blockIdx.x; i < a.N; i += gridDim.x) {
    const uint16_t* z = a.z + i * a.ldl;
    uint16_t* dz = a.dz ? a.dz + i * a.lddl : nullptr;
    const float w = a.weight ? a.weight[i] : 1.0f;
    if (w == 0.0f) {
      if (dz) for (int64_t j = threadIdx.x; j < a.V; j += kThreads) dz[j] = 0;
      if (threadIdx.x == 0) {
        a.logp[i] = 0.0f;
        if (LOSS) a.token_loss[i] = 0.0f;
      }
      continue;
    }
    float m = -INFINITY;
    for (int64_t j = threadIdx.x; j < a.V; j += kThreads) m = fmaxf(m, rows::h2f(z[j]));
    m = rows::block_max<kWarps>(m, red);
    if (isinf(m)) m = 0.0f;
    float s = 0.0f;
    for (int64_t j = threadIdx.x; j < a.V; j += kThreads) s += expf(rows::h2f(z[j]) - m);
    s = rows::block_sum<kWarps>(s, red);
    const int64_t t = rows::load_id<ID>(a.targets, i);
    const bool bad = t < 0 || t >= a.V;
    const float lp = bad ? NAN : (rows::h2f(z[t]) - m) - logf(s);
    float loss = 0.0f, dlp = 0.0f;
    if (LOSS) token_terms(a, i, lp, loss, dlp);
    if (threadIdx.x == 0) {
      if (bad) rows::record_bad_id(a.st);
      a.logp[i] = lp;
      if (LOSS) a.token_loss[i] = w * loss;
    }
    if (dz) {
      const float c = a.grad_scale * S * w * dlp, inv = 1.0f / s;
      __syncthreads();                               // z[t] is read before dz may overwrite it
      bool nonfinite = false;
      for (int64_t j = threadIdx.x; j < a.V; j += kThreads) {
        const uint16_t h = rows::f2h(c * ((j == t ? 1.0f : 0.0f) - expf(rows::h2f(z[j]) - m) * inv));
        dz[j] = h;
        nonfinite |= rows::nonfinite16(h);
      }
      if (nonfinite && a.st) atomicOr(&a.st->h.found_inf, 1);
    }
  }
}

// loss[0] = sum of the token losses, by one block in a fixed order.
__global__ void __launch_bounds__(kThreads) mp_loss_sum_kernel(const float* token_loss, int64_t N, float* loss) {
  __shared__ float red[kWarps];
  float s = 0.0f;
  for (int64_t i = threadIdx.x; i < N; i += kThreads) s += token_loss[i];
  s = rows::block_sum<kWarps>(s, red);
  if (threadIdx.x == 0) loss[0] = s;
}

int launch(const char* name, const LossArgs& a, int id_bytes, float* loss, bool with_loss, void* stream) {
  if (a.N < 0 || a.V <= 0 || a.ldl < a.V || (a.dz && a.lddl < a.V) || (id_bytes != 4 && id_bytes != 8))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: bad size, pitch or id width", name);
  if (a.N > 0 && (!a.z || !a.targets || !a.logp ||
                  (with_loss && (!a.old_logp || !a.advantage || !a.weight || !a.token_loss))))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: null pointer", name);
  const uintptr_t floats = (uintptr_t)a.old_logp | (uintptr_t)a.ref_logp | (uintptr_t)a.advantage |
                           (uintptr_t)a.weight | (uintptr_t)a.logp | (uintptr_t)a.token_loss | (uintptr_t)loss;
  if ((a.ldl & 7) || (a.dz && (a.lddl & 7)) || !mp::aligned16(a.z) || !mp::aligned16(a.dz) || (floats & 3) ||
      ((uintptr_t)a.targets & (uintptr_t)(id_bytes - 1)))
    return mp::set_error(MP_ERR_ALIGNMENT, "%s: logits must be 16-byte aligned with pitches that are multiples of 8, "
                         "ids and FP32 values aligned to their width", name);
  if (int rc = mp::check_device()) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  if (a.N > 0) {
    const int grid = (int)(a.N < 148 * 8 ? a.N : 148 * 8);
    if (with_loss) {
      if (id_bytes == 8) mp_policy_loss_kernel<int64_t, true><<<grid, kThreads, 0, st>>>(a);
      else mp_policy_loss_kernel<int32_t, true><<<grid, kThreads, 0, st>>>(a);
    } else {
      if (id_bytes == 8) mp_policy_loss_kernel<int64_t, false><<<grid, kThreads, 0, st>>>(a);
      else mp_policy_loss_kernel<int32_t, false><<<grid, kThreads, 0, st>>>(a);
    }
    mp::count_launch();
    MP_CUDA_TRY(cudaGetLastError());
  }
  if (loss) {
    mp_loss_sum_kernel<<<1, kThreads, 0, st>>>(a.token_loss, a.N, loss);
    mp::count_launch();
    MP_CUDA_TRY(cudaGetLastError());
  }
  return MP_OK;
}

}  // namespace

extern "C" {

int mp_policy_loss(const void* logits16, int64_t ldl, const void* targets, int id_bytes, const float* old_logp,
                   const float* ref_logp, const float* advantage, const float* weight, int64_t N, int64_t V,
                   const mp_policy_config* cfg, void* dlogits16, int64_t lddl, float* logp, float* token_loss,
                   float* loss, mp_state* state, void* stream) {
  if (!cfg) return mp::set_error(MP_ERR_INVALID_ARG, "mp_policy_loss: null configuration");
  if (!(cfg->clip_lo >= 0.0f) || !(cfg->clip_hi >= 0.0f) || !isfinite(cfg->kl_coef) || !isfinite(cfg->grad_scale))
    return mp::set_error(MP_ERR_INVALID_ARG, "mp_policy_loss: bad configuration");
  const LossArgs a{(const uint16_t*)logits16, ldl, targets, old_logp, ref_logp, advantage, weight, N, V,
                   cfg->clip_lo, cfg->clip_hi, cfg->kl_coef, cfg->grad_scale, (uint16_t*)dlogits16, lddl, logp,
                   token_loss, state ? state->dev : nullptr};
  return launch("mp_policy_loss", a, id_bytes, loss, true, stream);
}

int mp_token_logp(const void* logits16, int64_t ldl, const void* targets, int id_bytes, const float* weight,
                  int64_t N, int64_t V, float* logp, mp_state* state, void* stream) {
  const LossArgs a{(const uint16_t*)logits16, ldl, targets, nullptr, nullptr, nullptr, weight, N, V,
                   0.0f, 0.0f, 0.0f, 1.0f, nullptr, 0, logp, nullptr, state ? state->dev : nullptr};
  return launch("mp_token_logp", a, id_bytes, nullptr, false, stream);
}

}  // extern "C"

// Clipped policy loss with a KL term, forward and backward, and the token log-probabilities alone.
//
// The gradient needs the row's sum, so a row is read, held on the chip, and its gradient written: N V FP16 in, N V
// FP16 out, whatever lies between.  Two exponentials a word (16 results a clock and SM) and some 14 instructions stay
// below that: HBM bounds it from some 5000 words on.  Measured on B200s: 8192 x 32768, a tenth of the rows masked, 190 - 201 us
// (5.1 - 5.4 TB/s; a copy runs at 6.5); 1021 x 131071 98 - 101 us (4.5 - 4.6 TB/s).  Three passes over each row took 678 and
// 416 us.  Shorter rows are far from it: 40000 x 600 76 us where HBM would need 14, 20000 x 2000 56 (23), 20000 x 5000 86 (58).
// A block works on one row there, with two barriers and two joins a row, and nothing covers that.

#include <math.h>

#include "ptx.cuh"
#include "softmax.cuh"

namespace {

using namespace softmax;

struct LossArgs {
  const uint16_t* z;
  int64_t ldl;
  const void* targets;
  int id_bytes;
  const float *old_logp, *ref_logp, *advantage, *weight;
  int64_t N, V;
  float lo, hi, kl, grad_scale;
  uint16_t* dz;
  int64_t lddl;
  float *logp, *token_loss;
  mp_dev_state* st;
};

// Loss of one token and its derivative by the token's log-probability.
struct Token {
  float w, zt, old_logp, ref_logp, advantage;     // zt: the target's logit
  int target;                                     // -1: out of range
};
__device__ __forceinline__ int64_t target_of(const LossArgs& a, int64_t i) {
  return a.id_bytes == 8 ? rows::load_id<int64_t>(a.targets, i) : rows::load_id<int32_t>(a.targets, i);
}
// What row i has besides its logits; of a masked row (weight 0) and past the last one nothing is read.
__device__ __forceinline__ Token load_token(const LossArgs& a, int64_t i) {
  Token t{0.0f, 0.0f, 0.0f, 0.0f, 0.0f, -1};
  if (i >= a.N) return t;
  t.w = a.weight ? a.weight[i] : 1.0f;
  if (t.w == 0.0f) return t;
  const int64_t id = target_of(a, i);
  if (a.token_loss != nullptr) {
    t.old_logp = a.old_logp[i];
    t.advantage = a.advantage[i];
    if (a.ref_logp) t.ref_logp = a.ref_logp[i];
  }
  if (id >= 0 && id < a.V) {
    t.target = (int)id;
    t.zt = rows::h2f(a.z[i * a.ldl + id]);
  }
  return t;
}
__device__ __forceinline__ void token_terms(const LossArgs& a, const Token& t, float lp, float& loss, float& dlp) {
  const float A = t.advantage;
  const float x = lp - t.old_logp, r = expf(x);
  // a ratio past FP32 is finite all the same where its exponent is: 0 times it is 0, not a NaN
  const bool none = A == 0.0f && x < INFINITY;
  const float plain = none ? A : r * A, clipped = none ? A : fminf(fmaxf(r, 1.0f - a.lo), 1.0f + a.hi) * A;
  loss = plain <= clipped ? -plain : -clipped;
  dlp = plain <= clipped ? -plain : 0.0f;
  if (plain != plain) loss = dlp = plain;          // a NaN shows in the loss and the gradient
  if (a.ref_logp) {
    const float d = t.ref_logp - lp, e = expm1f(d);
    loss += a.kl * (e - d);
    dlp -= a.kl * e;
  }
}

// What a row's threads need to form its gradient: dz_j = cold 2^(z_j log2 e - k), and `hot` more at the
// target.  Every |dz_j| is at most |hot| (a probability is at most 1), so unless `check` is set nothing that
// is stored can be inf or NaN and nobody looks.
struct RowGrad {
  float k, hot, cold, at_target;
  int target, check;
};
// Finishes a row's sums: its outputs (by `writer`) and the factors of its gradient.
__device__ __forceinline__ RowGrad finish_row(const LossArgs& a, int64_t i, Sum2 v, const Token& t, float S, bool writer) {
  const float k = (float)v.k, up = fmaf(t.zt, kLog2e, -k);
  const float lp = t.target < 0 ? NAN : (up - log2f(v.s)) * kLn2;
  float loss = 0.0f, dlp = 0.0f;
  if (a.token_loss != nullptr) token_terms(a, t, lp, loss, dlp);
  if (writer) {
    if (t.target < 0) rows::record_bad_id(a.st);
    a.logp[i] = lp;
    if (a.token_loss != nullptr) a.token_loss[i] = t.w * loss;
  }
  const float c = a.grad_scale * S * t.w * dlp, cold = -c / v.s;
  return RowGrad{k, c, cold, fmaf(cold, ex2(up), c), t.target, !(fabsf(c) < 65000.0f) || !(fabsf(cold) <= 3.0e38f)};
}
__device__ __forceinline__ uint4 grad8(const uint4& z, const RowGrad& g) {
  const uint32_t w[4] = {z.x, z.y, z.z, z.w};
  float f[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
    f[2 * j] = g.cold * ex2(fmaf(x.x, kLog2e, -g.k));
    f[2 * j + 1] = g.cold * ex2(fmaf(x.y, kLog2e, -g.k));
  }
  return rows::pack8(f);
}
// The gradient of the nv live words of a vector, `dz` its place.
__device__ __forceinline__ bool put_grad(uint16_t* dz, const uint4& z, int nv, const RowGrad& g) {
  const uint4 q = grad8(z, g);
  store_words(dz, q, nv);
  return g.check ? nonfinite8(q, nv) : false;
}
// Then the target's word, by the thread that has just stored the vector with it.
__device__ __forceinline__ bool put_target(uint16_t* dz, const RowGrad& g) {
  const uint16_t h = rows::f2h(g.at_target);
  *dz = h;
  return rows::nonfinite16(h);
}
__device__ __forceinline__ void masked_outputs(const LossArgs& a, int64_t i) {
  a.logp[i] = 0.0f;
  if (a.token_loss != nullptr) a.token_loss[i] = 0.0f;
}
// ---- rows of up to 512 words: a group of TPR threads of a warp per row, the row in registers ----
constexpr int kGroupThreads = 256;
template <int TPR, int C>
__global__ void __launch_bounds__(kGroupThreads) mp_policy_loss_group_kernel(const LossArgs a) {
  static_assert(TPR <= 32, "a row's sums are joined inside a warp");
  constexpr int G = kGroupThreads / TPR;
  const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
  const int64_t i = (int64_t)blockIdx.x * G + group;
  const bool inside = i < a.N;
  if (TPR >= 32 && !inside) return;
  const Token tok = load_token(a, i);
  const bool live = tok.w != 0.0f;
  int nv[C];
  uint4 z[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int left = (int)a.V - (c * TPR + t) * 8;
    nv[c] = !inside || left < 0 ? 0 : left < 8 ? left : 8;
    z[c] = no_words();
    if (live && nv[c] > 0)
      z[c] = live8(__ldcs(reinterpret_cast<const uint4*>(a.z + i * a.ldl + (c * TPR + t) * 8)), nv[c]);
  }
  const float S = a.st ? a.st->h.scale : 1.0f;
  const Sum2 v = join_lanes<TPR>(thread_sum<C>(z));
  __syncwarp();                                    // every lane has read its token's logit before dz may take its place
  bool bad = false;
  if (live) {
    const RowGrad g = finish_row(a, i, v, tok, S, t == 0);
    if (a.dz != nullptr) {
      uint16_t* dz = a.dz + i * a.lddl;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = (c * TPR + t) * 8;
        if (nv[c] > 0) bad |= put_grad(dz + col, z[c], nv[c], g);
      }
      if (g.target >= 0 && (g.target / 8) % TPR == t) bad |= put_target(dz + g.target, g);
    }
  } else if (inside) {
    if (t == 0) masked_outputs(a, i);
    if (a.dz != nullptr)
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (nv[c] > 0) store_words(a.dz + i * a.lddl + (c * TPR + t) * 8, make_uint4(0, 0, 0, 0), nv[c]);
  }
  if (bad && a.st) atomicOr(&a.st->h.found_inf, 1);
}

// ---- rows of more than 512 words: CL blocks of a cluster per row, the row in their shared memory ----
//
// Persistent clusters, several blocks an SM: while one block sums a row or writes its gradient, the
// others' rows are on their way.  A block holds its part of a row, each thread its own vectors, which its own
// asynchronous copies bring into its own slots of shared memory; a slot is filled again with the
// next row's vector as soon as its gradient is formed.  One warp joins the partial sums and works out
// the token's loss and the factors of the gradient for all.  The blocks of a cluster hand their sums
// to each other's shared memory.
// Small blocks: with 128 threads and at most 32 KiB of a row (six to eight blocks an SM) the blocks drift
// apart and the loads of some cover the arithmetic of others.  8192 x 32768 with 128 threads and 32 KiB
// 189 us, 64 KiB 195, 16 KiB 223; 256 threads and 64 KiB 206; 512 threads 209; one block of 1024 threads
// with rows fetched two ahead 221.  (Rows in the registers of groups, as above for short ones, are slower from
// 512 words on: 20000 x 5000 229 us against 87, 40000 x 600 93 against 76.)
constexpr int kRowThreads = 128, kRowWarps = kRowThreads / 32;
constexpr int kPartWords = 16 * kRowThreads * 8;  // words of a row that a block takes if a cluster of 8 can
template <int CL>
__global__ void __launch_bounds__(kRowThreads, 8) mp_policy_loss_row_kernel(const LossArgs a) {
  extern __shared__ uint4 slots[];                // [vectors]
  __shared__ Sum2 s_part[2][kRowWarps];
  __shared__ Sum2 s_block[2][CL];
  __shared__ RowGrad s_grad[2];
  const int rank = CL > 1 ? (int)ptx::cluster_ctarank() : 0, lane = threadIdx.x & 31;
  const int64_t step = gridDim.x / CL, first = blockIdx.x / CL;
  const int V = (int)a.V, mine = rank * kRowThreads + (int)threadIdx.x;    // vector c of this thread: mine + c CL threads
  // this thread's whole vectors, and the words of one more that ends the row (most threads have none)
  const int rest = V / 8 - mine, whole = rest <= 0 ? 0 : (rest + CL * kRowThreads - 1) / (CL * kRowThreads);
  const int tail = rest >= 0 && rest % (CL * kRowThreads) == 0 ? V % 8 : 0;
  constexpr int kHop = CL * kRowThreads * 8;      // words from one vector of a thread to its next
  const uint32_t base = ptx::smem_u32(slots) + threadIdx.x * 16;
  const uint4* z = slots + threadIdx.x;
  const float S = a.st ? a.st->h.scale : 1.0f;
  auto weight_of = [&](int64_t i) { return i >= a.N ? 0.0f : a.weight ? __ldg(a.weight + i) : 1.0f; };
  auto copy = [&](const uint16_t* from, int c) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(base + c * kRowThreads * 16), "l"(from + c * kHop) : "memory");
  };
  auto fetch = [&](int64_t i) {
    const uint16_t* from = a.z + i * a.ldl + mine * 8;
    for (int c = 0; c < whole + (tail > 0); ++c) copy(from, c);
  };
  if constexpr (CL > 1) ptx::cluster_sync();      // every block of the cluster has started
  float w = weight_of(first);
  if (w != 0.0f) fetch(first);                    // a masked row is not read
  Token ahead{};                                  // first warp, lane l: what the l-th row from the last load on has
  int half = 0, turn = 0;
  bool bad = false;
  for (int64_t i = first; i < a.N; i += step, turn = (turn + 1) & 31) {
    // the loads of a token depend on one another (weight, target, its logit): 32 rows at a time
    if (threadIdx.x < 32 && turn == 0) ahead = load_token(a, i + lane * step);
    const float w_next = weight_of(i + step);
    const bool more = w_next != 0.0f;
    const uint16_t* from = a.z + (i + step) * a.ldl + mine * 8;
    uint16_t* dz = a.dz ? a.dz + i * a.lddl + mine * 8 : nullptr;
    if (w == 0.0f) {
      if (threadIdx.x == 0 && rank == 0) masked_outputs(a, i);
      if (dz != nullptr) {
        for (int c = 0; c < whole; ++c) __stcs(reinterpret_cast<uint4*>(dz + c * kHop), make_uint4(0, 0, 0, 0));
        if (tail > 0) store_words(dz + whole * kHop, make_uint4(0, 0, 0, 0), tail);
      }
      if (more) fetch(i + step);
      w = w_next;
      continue;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    Running r;
#pragma unroll 4
    for (int c = 0; c < whole; ++c) r.add(z[c * kRowThreads]);
    uint4 last = no_words();
    if (tail > 0) {
      last = live8(z[whole * kRowThreads], tail);
      r.add(last);
    }
    Sum2 v = join_lanes<32>(r.sum());
    if (lane == 0) s_part[half][threadIdx.x >> 5] = v;
    __syncthreads();
    if constexpr (CL > 1) {
      if (threadIdx.x < 32) {
        v = join_lanes<kRowWarps>(s_part[half][lane & (kRowWarps - 1)]);
        if (lane < CL) {                          // lane r hands this block's sum to block r
          const uint32_t to = ptx::map_to_cta(ptx::smem_u32(&s_block[half][rank]), lane);
          asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(to), "r"(v.k), "r"(__float_as_int(v.s)) : "memory");
        }
        __syncwarp();
      }
      ptx::cluster_sync();
    }
    if (threadIdx.x < 32) {
      if constexpr (CL > 1) v = join_lanes<CL>(s_block[half][lane & (CL - 1)]);
      else v = join_lanes<kRowWarps>(s_part[half][lane & (kRowWarps - 1)]);
      auto of = [&](float x) { return __shfl_sync(0xFFFFFFFFu, x, turn); };
      const Token t{w, of(ahead.zt), of(ahead.old_logp), of(ahead.ref_logp), of(ahead.advantage),
                    __shfl_sync(0xFFFFFFFFu, ahead.target, turn)};
      const RowGrad g = finish_row(a, i, v, t, S, lane == 0 && rank == 0);
      if (lane == 0) s_grad[half] = g;
    }
    if (dz != nullptr) {
      __syncthreads();
      const RowGrad g = s_grad[half];
      if (!g.check) {
#pragma unroll 4
        for (int c = 0; c < whole; ++c) {
          const uint4 q = grad8(z[c * kRowThreads], g);
          if (more) copy(from, c);                // the slot has been read
          __stcs(reinterpret_cast<uint4*>(dz + c * kHop), q);
        }
      } else {
        for (int c = 0; c < whole; ++c) {
          bad |= put_grad(dz + c * kHop, z[c * kRowThreads], 8, g);
          if (more) copy(from, c);
        }
      }
      if (tail > 0) {
        bad |= put_grad(dz + whole * kHop, last, tail, g);
        if (more) copy(from, whole);
      }
      if (g.target >= 0 && (g.target >> 3) % (CL * kRowThreads) == mine) bad |= put_target(a.dz + i * a.lddl + g.target, g);
    } else if (more) {
      fetch(i + step);
    }
    half ^= 1;                                    // a thread that gets back to this half has passed the next row's barrier
    w = w_next;
  }
  if (bad && a.st) atomicOr(&a.st->h.found_inf, 1);
}

// loss[0] = sum of the token losses, by one block in a fixed order.
constexpr int kSumThreads = 1024;
__global__ void __launch_bounds__(kSumThreads) mp_loss_sum_kernel(const float* token_loss, int64_t N, float* loss) {
  __shared__ float red[kSumThreads / 32];
  asm volatile("griddepcontrol.wait;" ::: "memory");   // the token losses are complete and visible
  float s = 0.0f;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < N; i += kSumThreads) s += token_loss[i];
  s = rows::block_sum<kSumThreads / 32>(s, red);
  if (threadIdx.x == 0) loss[0] = s;
}

template <int TPR, int C>
void group_launch(const LossArgs& a, cudaStream_t st) {
  constexpr int G = kGroupThreads / TPR;
  mp_policy_loss_group_kernel<TPR, C><<<(unsigned)((a.N + G - 1) / G), kGroupThreads, 0, st>>>(a);
}

// Persistent grid of whole clusters, as many as are resident at once (asked once per device, kernel and
// size of a block's part of a row).
template <int CL>
int row_launch(const LossArgs& a, cudaStream_t st) {
  static mp::PerDevice resident[MP_POLICY_MAX_V / 8 / (CL * kRowThreads) + 1];     // by layers
  const int64_t vecs = (a.V + 7) / 8, layers = (vecs + CL * kRowThreads - 1) / (CL * kRowThreads);
  const int smem = (int)layers * kRowThreads * 16;
  auto kernel = mp_policy_loss_row_kernel<CL>;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kRowThreads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = CL;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  int dev = 0, clusters = 0;
  MP_CUDA_TRY(cudaGetDevice(&dev));
  clusters = resident[layers].get(dev);
  if (clusters == 0) {
    MP_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MP_POLICY_MAX_V / 8 * 2));
    cfg.gridDim = dim3(CL * 148 * 16, 1, 1);
    MP_CUDA_TRY(cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg));
    if (clusters < 1) clusters = 1;
    resident[layers].set(dev, clusters);
  }
  if (a.N < clusters) clusters = (int)a.N;
  cfg.gridDim = dim3((unsigned)(clusters * CL), 1, 1);
  MP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, a));
  return MP_OK;
}

int dispatch(const LossArgs& a, cudaStream_t st) {
  if (a.V <= 32) group_launch<4, 1>(a, st);
  else if (a.V <= 128) group_launch<8, 2>(a, st);
  else if (a.V <= 512) group_launch<32, 2>(a, st);
  else if (a.V <= kPartWords) return row_launch<1>(a, st);
  else if (a.V <= 2 * kPartWords) return row_launch<2>(a, st);
  else if (a.V <= 4 * kPartWords) return row_launch<4>(a, st);
  else return row_launch<8>(a, st);
  return MP_OK;
}

int launch(const char* name, const LossArgs& a, float* loss, bool with_loss, void* stream) {
  const int id_bytes = a.id_bytes;
  if (a.N < 0 || a.V <= 0 || a.ldl < a.V || (a.dz && a.lddl < a.V) || (id_bytes != 4 && id_bytes != 8))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: bad size, pitch or id width", name);
  if (a.V > MP_POLICY_MAX_V) return mp::set_error(MP_ERR_TOO_LARGE, "%s: V beyond %d", name, MP_POLICY_MAX_V);
  if (a.N > 0 && (!a.z || !a.targets || !a.logp ||
                  (with_loss && (!a.old_logp || !a.advantage || !a.weight || !a.token_loss))))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: null pointer", name);
  const uintptr_t floats = (uintptr_t)a.old_logp | (uintptr_t)a.ref_logp | (uintptr_t)a.advantage |
                           (uintptr_t)a.weight | (uintptr_t)a.logp | (uintptr_t)a.token_loss | (uintptr_t)loss;
  if ((a.ldl & 7) || (a.dz && (a.lddl & 7)) || !mp::aligned16(a.z) || !mp::aligned16(a.dz) || (floats & 3) ||
      ((uintptr_t)a.targets & (uintptr_t)(id_bytes - 1)))
    return mp::set_error(MP_ERR_ALIGNMENT, "%s: logits must be 16-byte aligned with pitches that are multiples of 8, "
                         "ids and FP32 values aligned to their width", name);
  if (a.dz && a.dz == a.z && a.lddl != a.ldl)
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: a gradient in the logits' place needs their pitch", name);
  if (int rc = mp::check_device()) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  if (a.N > 0) {
    if (int rc = dispatch(a, st)) return rc;
    mp::count_launch();
    MP_CUDA_TRY(cudaGetLastError());
  }
  if (loss)
    if (int rc = mp::sum_token_loss(a.token_loss, a.N, loss, st)) return rc;
  return MP_OK;
}

}  // namespace

int mp::sum_token_loss(const float* token_loss, int64_t N, float* loss, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(1, 1, 1);
  cfg.blockDim = dim3(kSumThreads, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute attr;              // resident early, waits on the device for the token losses
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  MP_CUDA_TRY(cudaLaunchKernelEx(&cfg, mp_loss_sum_kernel, token_loss, N, loss));
  mp::count_launch();
  return MP_OK;
}

extern "C" {

int mp_policy_loss(const void* logits16, int64_t ldl, const void* targets, int id_bytes, const float* old_logp,
                   const float* ref_logp, const float* advantage, const float* weight, int64_t N, int64_t V,
                   const mp_policy_config* cfg, void* dlogits16, int64_t lddl, float* logp, float* token_loss,
                   float* loss, mp_state* state, void* stream) {
  if (!cfg) return mp::set_error(MP_ERR_INVALID_ARG, "mp_policy_loss: null configuration");
  if (!(cfg->clip_lo >= 0.0f) || !(cfg->clip_hi >= 0.0f) || !isfinite(cfg->kl_coef) || !isfinite(cfg->grad_scale))
    return mp::set_error(MP_ERR_INVALID_ARG, "mp_policy_loss: bad configuration");
  const float* ref = cfg->kl_coef != 0.0f ? ref_logp : nullptr;   // a factor of 0: no KL term, however far ref_logp is
  const LossArgs a{(const uint16_t*)logits16, ldl, targets, id_bytes, old_logp, ref, advantage, weight, N, V,
                   cfg->clip_lo, cfg->clip_hi, cfg->kl_coef, cfg->grad_scale, (uint16_t*)dlogits16, lddl, logp,
                   token_loss, state ? state->dev : nullptr};
  return launch("mp_policy_loss", a, loss, true, stream);
}

int mp_token_logp(const void* logits16, int64_t ldl, const void* targets, int id_bytes, const float* weight,
                  int64_t N, int64_t V, float* logp, mp_state* state, void* stream) {
  const LossArgs a{(const uint16_t*)logits16, ldl, targets, id_bytes, nullptr, nullptr, nullptr, weight, N, V,
                   0.0f, 0.0f, 0.0f, 1.0f, nullptr, 0, logp, nullptr, state ? state->dev : nullptr};
  return launch("mp_token_logp", a, nullptr, false, stream);
}

}  // extern "C"

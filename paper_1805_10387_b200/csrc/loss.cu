// Clipped policy loss with a KL term, forward and backward, and the token log-probabilities alone.

#include <math.h>

#include <map>
#include <mutex>

#include "ptx.cuh"
#include "rows.cuh"

namespace {

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

__device__ __forceinline__ int64_t target_of(const LossArgs& a, int64_t i) {
  return a.id_bytes == 8 ? rows::load_id<int64_t>(a.targets, i) : rows::load_id<int32_t>(a.targets, i);
}

// ---- softmax statistics in powers of two ----
//
// exp(z) = 2^(z log2 e).  A partial sum over some of a row's logits is kept as s * 2^k with an INTEGER k near
// the largest z log2 e of its part: z log2 e - k is then one fused operation with one rounding, and
// partial sums are brought to a common k by exact powers of two.
struct Sum2 {
  int k;
  float s;
};
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kNothing = -(1 << 20);             // k of a part of -inf alone: below every k that FP16 gives
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

// Sum over the words of C vectors of a thread.
template <int C>
__device__ __forceinline__ Sum2 thread_sum(const uint4 (&z)[C]) {
  __half2 m2 = __half2half2(__ushort_as_half(0xFC00));
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const uint32_t w[4] = {z[c].x, z[c].y, z[c].z, z[c].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) m2 = __hmax2(m2, *reinterpret_cast<const __half2*>(&w[j]));
  }
  const float2 m = __half22float2(m2);
  const float top = fmaxf(m.x, m.y);              // a NaN is lost here, and found again by the sum
  const float k = top == -INFINITY ? (float)kNothing : rintf(top * kLog2e);
  float s = 0.0f;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const uint32_t w[4] = {z[c].x, z[c].y, z[c].z, z[c].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
      s += ex2(fmaf(f.x, kLog2e, -k));
      s += ex2(fmaf(f.y, kLog2e, -k));
    }
  }
  // a logit of +inf leaves no distribution: inf - inf above made the sum a NaN
  return Sum2{top == INFINITY ? 0 : (int)k, s};
}

// What a row's threads need to form its gradient: dz_j = cold 2^(z_j log2 e - k), and `hot` more at the
// target.  Every |dz_j| is at most |hot| (a probability is at most 1), so unless `check` is set nothing that
// is stored can be inf or NaN and nobody looks.
struct RowGrad {
  float k, hot, cold, at_target;
  int check;
};
// Finishes a row's sums: its outputs (by `writer`) and the factors of its gradient.
__device__ __forceinline__ RowGrad finish_row(const LossArgs& a, int64_t i, Sum2 v, int64_t t, float zt, float w, float S,
                                              bool writer) {
  const bool bad = t < 0 || t >= a.V;
  const float k = (float)v.k, up = fmaf(zt, kLog2e, -k);
  const float lp = bad ? NAN : (up - log2f(v.s)) * kLn2;
  float loss = 0.0f, dlp = 0.0f;
  if (a.token_loss != nullptr) token_terms(a, i, lp, loss, dlp);
  if (writer) {
    if (bad) rows::record_bad_id(a.st);
    a.logp[i] = lp;
    if (a.token_loss != nullptr) a.token_loss[i] = w * loss;
  }
  const float c = a.grad_scale * S * w * dlp, cold = -c / v.s;
  return RowGrad{k, c, cold, fmaf(cold, ex2(up), c), !(fabsf(c) < 65000.0f) || !(fabsf(cold) <= 3.0e38f)};
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

// ---- rows of up to 8192 words: a group of TPR threads per row, the row in registers ----
constexpr int kGroupThreads = 256;
template <int TPR, int C>
__global__ void __launch_bounds__(kGroupThreads) mp_policy_loss_group_kernel(const LossArgs a) {
  constexpr int G = kGroupThreads / TPR, W = TPR / 32;
  __shared__ Sum2 s_part[G][W > 1 ? W : 1];
  const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
  const int64_t i = (int64_t)blockIdx.x * G + group;
  const bool inside = i < a.N;
  if (TPR >= 32 && !inside) return;
  const float w = !inside ? 0.0f : a.weight ? a.weight[i] : 1.0f;
  const bool live = w != 0.0f;
  int nv[C];
  uint4 z[C];
  int64_t target = -1;
  float zt = 0.0f;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int left = (int)a.V - (c * TPR + t) * 8;
    nv[c] = !inside || left < 0 ? 0 : left < 8 ? left : 8;
    z[c] = no_words();
    if (live && nv[c] > 0)
      z[c] = live8(__ldcs(reinterpret_cast<const uint4*>(a.z + i * a.ldl + (c * TPR + t) * 8)), nv[c]);
  }
  if (live) {
    target = target_of(a, i);
    if (target >= 0 && target < a.V) zt = rows::h2f(a.z[i * a.ldl + target]);
  }
  const float S = a.st ? a.st->h.scale : 1.0f;
  Sum2 v = join_lanes<(TPR < 32 ? TPR : 32)>(thread_sum<C>(z));
  if constexpr (W > 1) {
    if ((threadIdx.x & 31) == 0) s_part[group][t >> 5] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(TPR) : "memory");
    v = join_lanes<W>(s_part[group][threadIdx.x & (W - 1)]);
  } else {
    __syncwarp();                                  // every lane has read zt before dz may take its place
  }
  bool bad = false;
  if (live) {
    const RowGrad g = finish_row(a, i, v, target, zt, w, S, t == 0);
    if (a.dz != nullptr) {
      uint16_t* dz = a.dz + i * a.lddl;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = (c * TPR + t) * 8;
        if (nv[c] > 0) bad |= put_grad(dz + col, z[c], nv[c], g);
      }
      if (target >= 0 && target < a.V && (int)(target / 8) % TPR == t) bad |= put_target(dz + target, g);
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

// ---- rows of up to 262144 words: CL blocks of a cluster per row, the row in their shared memory ----
//
// Persistent clusters.  512 workers of a block hold up to 32768 words of a row, each thread its own vectors, which
// its own asynchronous copies bring into its own slots; three stages of slots, so that while row i is
// summed and row i - 1 gets its gradient, row i + 1 is on its way.  One more warp joins the partial
// sums of row i and works out the token's loss and the factors of the gradient while the workers
// are busy with the gradient of row i - 1; one block barrier a row is all that they share.  The
// blocks of a cluster hand their sums to each other's shared memory; the workers arrive at the
// cluster's barrier before a row's gradient and wait for it after.
// (Before: workers that held the row in registers and waited for its factors, two blocks an SM:
// 258 us for 8192 x 32768.)
constexpr int kWorkers = 512, kWorkerWarps = kWorkers / 32, kRowThreads = kWorkers + 32, kStages = 3;
template <int C, int CL>
__global__ void __launch_bounds__(kRowThreads, C > 4 ? 1 : 2) mp_policy_loss_row_kernel(const LossArgs a) {
  extern __shared__ uint4 slots[];                // [stage][C][workers]
  __shared__ Sum2 s_part[2][kWorkerWarps];
  __shared__ Sum2 s_block[2][CL];
  __shared__ RowGrad s_grad[2];
  const int rank = CL > 1 ? (int)ptx::cluster_ctarank() : 0, lane = threadIdx.x & 31;
  const int64_t step = gridDim.x / CL, first = blockIdx.x / CL;
  const int V = (int)a.V;
  auto weight_of = [&](int64_t i) { return i >= a.N ? 0.0f : a.weight ? __ldg(a.weight + i) : 1.0f; };
  auto arrive = [] { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); };
  auto wait = [] { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); };
  if constexpr (CL > 1) ptx::cluster_sync();      // every block of the cluster has started
  if (threadIdx.x >= kWorkers) {
    const float S = a.st ? a.st->h.scale : 1.0f;
    int half = 0;
    for (int64_t i = first; i - step < a.N; i += step, half ^= 1) {
      const float w = weight_of(i);
      int64_t target = 0;
      float zt = 0.0f;
      if (w != 0.0f) {
        target = target_of(a, i);
        if (target >= 0 && target < V) zt = rows::h2f(a.z[i * a.ldl + target]);
      }
      __syncthreads();                            // the workers' sums of row i are there
      Sum2 v{kNothing, 0.0f};
      if (w != 0.0f) v = join_lanes<kWorkerWarps>(s_part[half][lane & (kWorkerWarps - 1)]);
      if constexpr (CL > 1) {
        if (lane < CL) {                          // lane r hands this block's sum to block r
          const uint32_t to = ptx::map_to_cta(ptx::smem_u32(&s_block[half][rank]), lane);
          asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(to), "r"(v.k), "r"(__float_as_int(v.s)) : "memory");
        }
        __syncwarp();
        arrive();
        wait();
        v = join_lanes<CL>(s_block[half][lane & (CL - 1)]);
      }
      if (w != 0.0f) {
        const RowGrad g = finish_row(a, i, v, target, zt, w, S, lane == 0 && rank == 0);
        if (lane == 0) s_grad[half] = g;
      } else if (i < a.N && lane == 0 && rank == 0) {
        masked_outputs(a, i);
      }
    }
    return;
  }
  const int mine = rank * kWorkers + (int)threadIdx.x;    // vector c of this thread: mine + c CL workers
  const uint32_t base = ptx::smem_u32(slots) + threadIdx.x * 16;
  auto left_of = [&](int c) { return V - (mine + c * (CL * kWorkers)) * 8; };     // words from the vector's first on
  auto fetch = [&](int64_t i, float w, int stage) {       // w: the weight of row i; a masked row is not read
    if (w != 0.0f) {
      const uint16_t* z = a.z + i * a.ldl + mine * 8;
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (left_of(c) > 0)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(base + (stage * C + c) * kWorkers * 16),
                       "l"(z + c * (CL * kWorkers * 8)) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  float w_before = 0.0f, w = weight_of(first), w_next = weight_of(first + step);
  fetch(first, w, 0);
  int stage = 0, half = 0;
  bool bad = false;
  for (int64_t i = first; i - step < a.N; i += step, half ^= 1) {
    const float w_after = weight_of(i + 2 * step);
    const int next = stage == kStages - 1 ? 0 : stage + 1, before = stage == 0 ? kStages - 1 : stage - 1;
    fetch(i + step, w_next, next);                // that stage held row i - 2, whose gradient is stored
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    if (w != 0.0f) {
      uint4 z[C];
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int left = left_of(c);
        z[c] = left > 0 ? slots[(stage * C + c) * kWorkers + threadIdx.x] : no_words();
        if (left > 0 && left < 8) z[c] = live8(z[c], left);
      }
      const Sum2 v = join_lanes<32>(thread_sum<C>(z));
      if (lane == 0) s_part[half][threadIdx.x >> 5] = v;
    }
    __syncthreads();
    if constexpr (CL > 1) arrive();
    const int64_t b = i - step;                   // the row before gets its gradient
    if (b >= first && a.dz != nullptr) {
      uint16_t* dz = a.dz + b * a.lddl + mine * 8;
      if (w_before != 0.0f) {
        const RowGrad g = s_grad[half ^ 1];
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const int left = left_of(c);
          if (left > 0) bad |= put_grad(dz + c * (CL * kWorkers * 8), slots[(before * C + c) * kWorkers + threadIdx.x], left, g);
        }
        const int64_t target = target_of(a, b);
        if (target >= 0 && target < V && (int)(target >> 3) % (CL * kWorkers) == mine)
          bad |= put_target(a.dz + b * a.lddl + target, g);
      } else {
#pragma unroll
        for (int c = 0; c < C; ++c)
          if (left_of(c) > 0) store_words(dz + c * (CL * kWorkers * 8), make_uint4(0, 0, 0, 0), left_of(c));
      }
    }
    if constexpr (CL > 1) wait();
    stage = next;
    w_before = w;
    w = w_next;
    w_next = w_after;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  if (bad && a.st) atomicOr(&a.st->h.found_inf, 1);
}

// ---- longer rows: one block per row, two passes over it, the second mostly from L2 ----
constexpr int kLongThreads = 512, kLongWarps = kLongThreads / 32;
__global__ void __launch_bounds__(kLongThreads) mp_policy_loss_long_kernel(const LossArgs a) {
  __shared__ Sum2 s_part[kLongWarps];
  const float S = a.st ? a.st->h.scale : 1.0f;
  bool bad = false;
  for (int64_t i = blockIdx.x; i < a.N; i += gridDim.x) {
    const uint16_t* z = a.z + i * a.ldl;
    uint16_t* dz = a.dz ? a.dz + i * a.lddl : nullptr;
    const float w = a.weight ? a.weight[i] : 1.0f;
    auto left_of = [&](int64_t col) { return a.V - col < 8 ? (int)(a.V - col) : 8; };
    if (w == 0.0f) {
      if (dz)
        for (int64_t col = (int64_t)threadIdx.x * 8; col < a.V; col += kLongThreads * 8)
          store_words(dz + col, make_uint4(0, 0, 0, 0), left_of(col));
      if (threadIdx.x == 0) masked_outputs(a, i);
      continue;
    }
    const int64_t target = target_of(a, i);
    const bool good = target >= 0 && target < a.V;
    const float zt = good ? rows::h2f(z[target]) : 0.0f;
    Sum2 v{kNothing, 0.0f};
    for (int64_t col = (int64_t)threadIdx.x * 8; col < a.V; col += kLongThreads * 8) {
      const uint4 q[1] = {live8(*reinterpret_cast<const uint4*>(z + col), left_of(col))};
      const Sum2 x = thread_sum<1>(q);
      const int k = max(v.k, x.k);
      v = Sum2{k, v.s * ex2((float)(v.k - k)) + x.s * ex2((float)(x.k - k))};
    }
    v = join_lanes<32>(v);
    __syncthreads();                               // the part sums of the row before have been read
    if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = join_lanes<kLongWarps>(s_part[threadIdx.x & (kLongWarps - 1)]);
    const RowGrad g = finish_row(a, i, v, target, zt, w, S, threadIdx.x == 0);
    if (dz) {
      for (int64_t col = (int64_t)threadIdx.x * 8; col < a.V; col += kLongThreads * 8) {
        const int nv = left_of(col);
        bad |= put_grad(dz + col, live8(*reinterpret_cast<const uint4*>(z + col), nv), nv, g);
      }
      if (good && (int)((target >> 3) % kLongThreads) == (int)threadIdx.x) bad |= put_target(dz + target, g);
    }
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

// Persistent grid of whole clusters, as many as are resident at once (asked once per device and kernel).
template <int C, int CL>
int row_launch(const LossArgs& a, cudaStream_t st) {
  static std::mutex mu;
  static std::map<int, int> resident;             // clusters of this kernel per device
  const size_t smem = (size_t)kStages * C * kWorkers * 16;
  auto kernel = mp_policy_loss_row_kernel<C, CL>;
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
  {
    std::lock_guard<std::mutex> lock(mu);
    int& have = resident[dev];
    if (have == 0) {
      MP_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
      cfg.gridDim = dim3(CL * 148 * 2, 1, 1);
      MP_CUDA_TRY(cudaOccupancyMaxActiveClusters(&have, kernel, &cfg));
      if (have < 1) have = 1;
    }
    clusters = have;
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
  else if (a.V <= 2048) group_launch<32, 8>(a, st);
  else if (a.V <= 8192) group_launch<128, 8>(a, st);
  else if (a.V <= 16384) return row_launch<4, 1>(a, st);
  else if (a.V <= 32768) return row_launch<8, 1>(a, st);
  else if (a.V <= 65536) return row_launch<8, 2>(a, st);
  else if (a.V <= 131072) return row_launch<8, 4>(a, st);
  else if (a.V <= 262144) return row_launch<8, 8>(a, st);
  else mp_policy_loss_long_kernel<<<(unsigned)(a.N < 296 ? a.N : 296), kLongThreads, 0, st>>>(a);
  return MP_OK;
}

int launch(const char* name, const LossArgs& a, float* loss, bool with_loss, void* stream) {
  const int id_bytes = a.id_bytes;
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
    if (int rc = dispatch(a, st)) return rc;
    mp::count_launch();
    MP_CUDA_TRY(cudaGetLastError());
  }
  if (loss) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(1, 1, 1);
    cfg.blockDim = dim3(kSumThreads, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr;            // resident early, waits on the device for the token losses
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    MP_CUDA_TRY(cudaLaunchKernelEx(&cfg, mp_loss_sum_kernel, (const float*)a.token_loss, a.N, loss));
    mp::count_launch();
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
  const LossArgs a{(const uint16_t*)logits16, ldl, targets, id_bytes, old_logp, ref_logp, advantage, weight, N, V,
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

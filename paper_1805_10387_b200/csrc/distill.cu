// Distillation from a teacher's top entries, forward and backward: KL divergence of the student's softmax from the teacher's
// listed probabilities, with what the teacher does not list as one more outcome, or with the listed ones alone.
//
// Reads N V FP16, writes N V FP16: HBM bounds it.  A row stays in shared memory between its sum and its gradient, as in the
// policy loss.  The tail needs the softmax mass of the tokens that are NOT listed, which a difference of sums would lose
// where the list holds nearly everything; so the listed words are made -inf in shared memory and the sum over the
// row is that of the others, to full precision.  The listed words' gradients are written behind the row's, by the warp
// that keeps the list.  8192 x 32768, 20 entries: 210 us, where the bytes alone take 156; 1021 x 131071, 128 entries: 153
// us, the bytes 70: a row has four barriers, of the cluster one, and waits for the first warp's work on the list between two of
// them.  An entry's id is loaded two rows ahead and its logit one (266 us when both were loaded with their row).

#include <math.h>

#include "ptx.cuh"
#include "softmax.cuh"

namespace {

using namespace softmax;

struct DistillArgs {
  const uint16_t* z;
  int64_t ldl;
  const void* ids;
  int id_bytes;
  const float *tlogp, *weight;
  int64_t N, V;
  int K, tail;
  float scale, factor;                            // log2 e / temperature; grad_scale / temperature
  uint16_t* dz;
  int64_t lddl;
  float* token_loss;
  mp_dev_state* st;
};

constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr int kPartWords = 16 * kThreads * 8;     // words of a row that a block takes if a cluster of 8 can
constexpr int kWarpWords = 2048;                  // rows of up to so many words go to single warps

// The entries of a row, lane l's are l, l + 32, ..: by the first warp of a row's threads.
template <int E>
struct Entries {
  int id[E];                                      // -1: none; -2: not a token
  float a[E], z[E];                               // the teacher's log-probability, the student's logit
  __device__ __forceinline__ void load(const DistillArgs& g, int64_t i, bool on) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int k = e * 32 + (threadIdx.x & 31);
      id[e] = -1;
      a[e] = z[e] = -INFINITY;
      if (on && k < g.K) {
        const int64_t at = i * g.K + k;
        const int64_t t = g.id_bytes == 8 ? rows::load_id<int64_t>(g.ids, at) : rows::load_id<int32_t>(g.ids, at);
        a[e] = g.tlogp[at];
        id[e] = t == -1 ? -1 : t >= 0 && t < g.V ? (int)t : -2;
      }
    }
  }
  __device__ __forceinline__ void load_logits(const DistillArgs& g, int64_t i) {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (id[e] >= 0) z[e] = rows::h2f(g.z[i * g.ldl + id[e]]);
  }
};

// What the row's threads need: dz_j = cold 2^(z_j scale - k) for the words that are not listed.
struct Grad {
  float k, cold;
  int check;
};
// What the first warp keeps until the gradients are written.
template <int E>
struct Listed {
  float dz[E];
};

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
  return v;
}

// By a whole warp: the row's loss and the factors of its gradient, from the sum over the words that are not listed.
template <int kEach>
__device__ __forceinline__ Grad finish(const DistillArgs& g, int64_t i, Entries<kEach>& t, Sum2 rest, float w, float S,
                                       bool writer, Listed<kEach>& out) {
  // the listed words' sum, their probabilities under the teacher
  float top = -INFINITY, most = -INFINITY;
  bool bad = false, any = false;
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    bad |= t.id[e] == -2;
    any |= t.id[e] >= 0;
    if (t.id[e] >= 0) {
      top = fmaxf(top, t.z[e]);
      most = fmaxf(most, t.a[e]);
    }
  }
  bad = __any_sync(0xFFFFFFFFu, bad);
  any = __any_sync(0xFFFFFFFFu, any);
  top = warp_max(top);
  most = warp_max(most);
  const float kt = top == -INFINITY ? (float)kNothing : rintf(top * g.scale);
  float st = 0.0f, p[kEach], sum_p = 0.0f;
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    if (t.id[e] >= 0) st += ex2(fmaf(t.z[e], g.scale, -kt));
    // alone: probabilities of the list by itself, whatever constant the teacher's values carry
    p[e] = t.id[e] >= 0 ? expf(g.tail ? t.a[e] : t.a[e] - most) : 0.0f;
    sum_p += p[e];
  }
  st = rows::warp_sum(st);
  sum_p = rows::warp_sum(sum_p);
  float shift = 0.0f;                             // log p = a - shift
  if (!g.tail) {
    const float inv = any ? 1.0f / sum_p : 0.0f;
    shift = any ? most + logf(sum_p) : 0.0f;
#pragma unroll
    for (int e = 0; e < kEach; ++e) p[e] *= inv;
    sum_p = any ? 1.0f : 0.0f;
    if (most != most || most == -INFINITY) sum_p = any ? NAN : 0.0f;
  }
  // the whole row's sum 2^k (s), and the tail.  r = 1 - P and the student's 1 - Q lose bits where P and Q are small, and
  // there log1p keeps them; where Q is large the tail's own sum does
  const int k = max(rest.k, top == -INFINITY ? kNothing : top == INFINITY ? 0 : (int)kt);
  const float rest_up = ex2((float)(rest.k - k)), listed_s = st * ex2(kt - (float)k);
  const float s = rest.s * rest_up + listed_s;
  const float log2s = log2f(s);
  float mass = sum_p, lr = 0.0f, over = mass * rest_up / s;  // over: of the unlisted words' softmax, what their gradient takes
  if (g.tail && rest.s != 0.0f) {
    const float r = 1.0f - sum_p, Q = listed_s / s;
    if (!(r <= 0.0f)) {                           // a NaN goes on
      mass = sum_p + r;
      const float log_r = sum_p < 0.5f ? log1pf(-sum_p) : logf(r);
      const float log_q = Q < 0.5f ? log1pf(-Q) : ((float)(rest.k - k) + log2f(rest.s / s)) * kLn2;
      lr = r * (log_r - log_q);
      over = (Q < 0.5f ? sum_p - Q : rest.s * rest_up / s - r) / rest.s;
    }
  }
  if (bad) mass = NAN;
  const float G = g.factor * S * w;
  float loss = 0.0f;
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const float y = fmaf(t.z[e], g.scale, -(float)k) - log2s;           // log2 of the student's probability
    if (t.id[e] >= 0 && p[e] != 0.0f) loss += p[e] * ((t.a[e] - shift) - y * kLn2);
    out.dz[e] = G * fmaf(ex2(y), mass, -p[e]);
  }
  loss = rows::warp_sum(loss) + lr;
  if (mass != mass) loss = mass;
  if (s != s) loss = s;
  if ((threadIdx.x & 31) == 0) {
    if (bad) rows::record_bad_id(g.st);
    if (writer) g.token_loss[i] = w * loss;
  }
  const float cold = bad ? NAN : G * over;
  // every |dz_j| is at most 2 |G| mass: unless that is near FP16's end nobody looks at what is stored
  return Grad{(float)rest.k, cold, !(2.0f * fabsf(G) * mass < 65000.0f) || !(fabsf(cold) <= 3.0e38f)};
}

__device__ __forceinline__ uint4 cold8(const uint4& z, const Grad& g, float scale) {
  const uint32_t w[4] = {z.x, z.y, z.z, z.w};
  float f[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
    f[2 * j] = g.cold * ex2(fmaf(x.x, scale, -g.k));
    f[2 * j + 1] = g.cold * ex2(fmaf(x.y, scale, -g.k));
  }
  return rows::pack8(f);
}

// Makes a listed word of the row -inf; true when it was listed before.
__device__ __forceinline__ bool strike(uint16_t* word, bool finite) {
  uint32_t* at = reinterpret_cast<uint32_t*>(reinterpret_cast<uintptr_t>(word) & ~(uintptr_t)3);
  const int up = (reinterpret_cast<uintptr_t>(word) & 2) * 8;
  uint32_t old = *at, seen;
  do {
    seen = old;
    old = atomicCAS(at, seen, (seen & ~(0xFFFFu << up)) | (0xFC00u << up));
  } while (old != seen);
  return finite && ((seen >> up) & 0xFFFFu) == 0xFC00u;
}

// TEAM threads a row: a warp each (short rows), or a block, or CL blocks of a cluster.  The layout of a row over its
// threads and the refilling of its slots are the policy loss's.
// Blocks an SM: where several share a row six (1021 x 131071, 128 entries: 153 us, with seven 168), else seven, which 16384 words
// each leave room for; of warps eight, or five where a lane has four entries (20000 x 2000, 64 entries: 71 us, with eight 75).
template <int CL, int TEAM, int kEach>
__global__ void __launch_bounds__(kThreads, TEAM == 32 ? kEach > 1 ? 5 : 8 : CL > 1 ? 6 : 7) mp_distill_kernel(const DistillArgs g, int layers) {
  static_assert(TEAM == kThreads || (TEAM == 32 && CL == 1), "a warp, a block or a cluster for a row");
  constexpr int TEAMS = kThreads / TEAM;
  extern __shared__ uint4 all_slots[];            // [team][vectors]
  __shared__ Sum2 s_part[2][kWarps];
  __shared__ Sum2 s_block[2][CL];
  __shared__ Grad s_grad[2];
  const int rank = CL > 1 ? (int)ptx::cluster_ctarank() : 0, lane = threadIdx.x & 31;
  const int team = threadIdx.x / TEAM, t = threadIdx.x % TEAM;
  const bool first_warp = TEAM == 32 || threadIdx.x < 32;
  uint4* slots = all_slots + team * layers * TEAM;
  const int64_t step = (int64_t)(gridDim.x / CL) * TEAMS, first = (int64_t)(blockIdx.x / CL) * TEAMS + team;
  const int V = (int)g.V, mine = rank * TEAM + t;            // vector c of this thread: mine + c CL TEAM
  const int left = V / 8 - mine, whole = left <= 0 ? 0 : (left + CL * TEAM - 1) / (CL * TEAM);
  const int tail = left >= 0 && left % (CL * TEAM) == 0 ? V % 8 : 0;
  constexpr int kHop = CL * TEAM * 8;
  const uint32_t base = ptx::smem_u32(slots) + t * 16;
  const uint4* z = slots + t;
  const float S = g.st ? g.st->h.scale : 1.0f, scale = g.scale;
  auto sync = [&] {
    if constexpr (TEAM == 32) __syncwarp();
    else __syncthreads();
  };
  auto weight_of = [&](int64_t i) { return i >= g.N ? 0.0f : __ldg(g.weight + i); };
  auto copy = [&](const uint16_t* from, int c) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(base + c * TEAM * 16), "l"(from + c * kHop) : "memory");
  };
  auto fetch = [&](int64_t i) {
    const uint16_t* from = g.z + i * g.ldl + mine * 8;
    for (int c = 0; c < whole + (tail > 0); ++c) copy(from, c);
  };
  if constexpr (CL > 1) ptx::cluster_sync();
  float w = weight_of(first);
  if (w != 0.0f) fetch(first);
  // An entry's logit waits for its id: the ids are loaded two rows ahead, the logits one.
  Entries<kEach> e, ahead, later;
  float w_next = weight_of(first + step);
  if (first_warp) {
    ahead.load(g, first, w != 0.0f);
    ahead.load_logits(g, first);
    later.load(g, first + step, w_next != 0.0f);
  }
  Listed<kEach> listed;
  int64_t behind = -1;                            // the row whose listed words are still to be written
  int half = 0;
  bool bad = false;
  // by the first warp, when every thread has stored its part of the row: the listed words that are in this block's part
  auto write_listed = [&] {
#pragma unroll
    for (int k = 0; k < kEach; ++k)
      if (e.id[k] >= 0 && (CL == 1 || (e.id[k] >> 3) / TEAM % CL == rank)) {
        const uint16_t h = rows::f2h(listed.dz[k]);
        g.dz[behind * g.lddl + e.id[k]] = h;
        bad |= rows::nonfinite16(h);
      }
    behind = -1;
  };
  for (int64_t i = first; i < g.N; i += step) {
    const float w_later = weight_of(i + 2 * step);
    const bool more = w_next != 0.0f;
    auto advance = [&] {
      ahead = later;
      ahead.load_logits(g, i + step);
      later.load(g, i + 2 * step, w_later != 0.0f);
    };
    const uint16_t* from = g.z + (i + step) * g.ldl + mine * 8;
    uint16_t* dz = g.dz ? g.dz + i * g.lddl + mine * 8 : nullptr;
    if (w == 0.0f) {                              // a masked row is not read
      if (first_warp && lane == 0 && rank == 0) g.token_loss[i] = 0.0f;
      if (dz != nullptr) {
        for (int c = 0; c < whole; ++c) __stcs(reinterpret_cast<uint4*>(dz + c * kHop), make_uint4(0, 0, 0, 0));
        if (tail > 0) store_words(dz + whole * kHop, make_uint4(0, 0, 0, 0), tail);
      }
      if (more) fetch(i + step);
      if (first_warp) advance();
      w = w_next;
      w_next = w_later;
      continue;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    sync();                                       // the row has landed, and the row before is stored
    if (first_warp) {
      if (behind >= 0) write_listed();
      e = ahead;
#pragma unroll
      for (int k = 0; k < kEach; ++k)
        if (e.id[k] >= 0 && (CL == 1 || (e.id[k] >> 3) / TEAM % CL == rank)) {
          const int vec = e.id[k] >> 3, slot = vec / (CL * TEAM) * TEAM + vec % TEAM;
          if (strike(reinterpret_cast<uint16_t*>(slots + slot) + (e.id[k] & 7), e.z[k] != -INFINITY)) e.id[k] = -2;
        }
    }
    sync();
    if (first_warp) advance();
    Running r;
#pragma unroll 4
    for (int c = 0; c < whole; ++c) r.add(z[c * TEAM], scale);
    uint4 last = no_words();
    if (tail > 0) {
      last = live8(z[whole * TEAM], tail);
      r.add(last, scale);
    }
    Sum2 v = join_lanes<32>(r.sum());
    if constexpr (TEAM > 32) {
      if (lane == 0) s_part[half][threadIdx.x >> 5] = v;
      __syncthreads();
    }
    // a list with an id twice or out of range has no loss: a NaN in the sum reaches every block of the row
    if constexpr (CL > 1) {
      if (threadIdx.x < 32) {
        v = join_lanes<kWarps>(s_part[half][lane & (kWarps - 1)]);
        bool twice = false;
#pragma unroll
        for (int k = 0; k < kEach; ++k) twice |= e.id[k] == -2;
        if (__any_sync(0xFFFFFFFFu, twice)) v.s = NAN;
        if (lane < CL) {
          const uint32_t to = ptx::map_to_cta(ptx::smem_u32(&s_block[half][rank]), lane);
          asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(to), "r"(v.k), "r"(__float_as_int(v.s)) : "memory");
        }
        __syncwarp();
      }
      ptx::cluster_sync();
    }
    Grad gr;
    if (first_warp) {
      if constexpr (CL > 1) v = join_lanes<CL>(s_block[half][lane & (CL - 1)]);
      else if constexpr (TEAM > 32) v = join_lanes<kWarps>(s_part[half][lane & (kWarps - 1)]);
      gr = finish(g, i, e, v, w, S, rank == 0, listed);
      if (TEAM > 32 && lane == 0) s_grad[half] = gr;
      behind = dz != nullptr ? i : -1;
    }
    if (dz != nullptr) {
      if constexpr (TEAM > 32) {
        __syncthreads();
        gr = s_grad[half];
      }
#pragma unroll 4
      for (int c = 0; c < whole; ++c) {
        const uint4 q = cold8(z[c * TEAM], gr, scale);
        if (more) copy(from, c);                  // the slot has been read
        __stcs(reinterpret_cast<uint4*>(dz + c * kHop), q);
        if (gr.check) bad |= nonfinite8(q, 8);
      }
      if (tail > 0) {
        const uint4 q = cold8(last, gr, scale);
        if (more) copy(from, whole);
        store_words(dz + whole * kHop, q, tail);
        if (gr.check) bad |= nonfinite8(q, tail);
      }
    } else if (more) {
      fetch(i + step);
    }
    half ^= 1;
    w = w_next;
    w_next = w_later;
  }
  sync();
  if (first_warp && behind >= 0) write_listed();
  if (bad && g.st) atomicOr(&g.st->h.found_inf, 1);
}

template <int CL, int TEAM, int E>
int launch(const DistillArgs& g, cudaStream_t st) {
  constexpr int TEAMS = kThreads / TEAM;
  static mp::PerDevice resident[MP_POLICY_MAX_V / 8 / (CL * TEAM) + 1];            // by layers
  const int64_t vecs = (g.V + 7) / 8;
  const int layers = (int)((vecs + CL * TEAM - 1) / (CL * TEAM));
  auto kernel = mp_distill_kernel<CL, TEAM, E>;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = (size_t)layers * kThreads * 16;
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = CL;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  int dev = 0;
  MP_CUDA_TRY(cudaGetDevice(&dev));
  int clusters = resident[layers].get(dev);
  if (clusters == 0) {
    MP_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MP_POLICY_MAX_V / 8 * 2));
    cfg.gridDim = dim3(CL * 148 * 16, 1, 1);
    MP_CUDA_TRY(cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg));
    if (clusters < 1) clusters = 1;
    resident[layers].set(dev, clusters);
  }
  const int64_t need = (g.N + TEAMS - 1) / TEAMS;
  if (need < clusters) clusters = (int)need;
  cfg.gridDim = dim3((unsigned)(clusters * CL), 1, 1);
  MP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, g, layers));
  mp::count_launch();
  return MP_OK;
}

template <int E>                                  // entries of a lane
int by_width(const DistillArgs& g, cudaStream_t st) {
  return g.V <= kWarpWords ? launch<1, 32, E>(g, st)
         : g.V <= kPartWords ? launch<1, kThreads, E>(g, st)
         : g.V <= 2 * kPartWords ? launch<2, kThreads, E>(g, st)
         : g.V <= 4 * kPartWords ? launch<4, kThreads, E>(g, st) : launch<8, kThreads, E>(g, st);
}

}  // namespace

extern "C" int mp_distill_loss(const void* logits16, int64_t ldl, const void* ids, int id_bytes, const float* teacher_logp,
                               int64_t K, const float* weight, int64_t N, int64_t V, const mp_distill_config* cfg,
                               void* dlogits16, int64_t lddl, float* token_loss, float* loss, mp_state* state, void* stream) {
  const char* name = "mp_distill_loss";
  if (!cfg) return mp::set_error(MP_ERR_INVALID_ARG, "%s: null configuration", name);
  if (!(cfg->temperature >= MP_MIN_TEMPERATURE) || !(cfg->temperature <= MP_MAX_TEMPERATURE) || (cfg->tail != 0 && cfg->tail != 1) ||
      !isfinite(cfg->grad_scale))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: bad configuration", name);
  if (N < 0 || V <= 0 || K <= 0 || K > V || ldl < V || (dlogits16 && lddl < V) || (id_bytes != 4 && id_bytes != 8))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: bad size, pitch or id width", name);
  if (V > MP_POLICY_MAX_V || K > MP_DISTILL_MAX_K)
    return mp::set_error(MP_ERR_TOO_LARGE, "%s: V beyond %d or more than %d entries", name, MP_POLICY_MAX_V, MP_DISTILL_MAX_K);
  if (N > 0 && (!logits16 || !ids || !teacher_logp || !weight || !token_loss))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: null pointer", name);
  const uintptr_t floats = (uintptr_t)teacher_logp | (uintptr_t)weight | (uintptr_t)token_loss | (uintptr_t)loss;
  if ((ldl & 7) || (dlogits16 && (lddl & 7)) || !mp::aligned16(logits16) || !mp::aligned16(dlogits16) || (floats & 3) ||
      ((uintptr_t)ids & (uintptr_t)(id_bytes - 1)))
    return mp::set_error(MP_ERR_ALIGNMENT, "%s: logits must be 16-byte aligned with pitches that are multiples of 8, ids and "
                         "FP32 values aligned to their width", name);
  if (dlogits16 && dlogits16 == logits16 && lddl != ldl)
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: a gradient in the logits' place needs their pitch", name);
  if (int rc = mp::check_device()) return rc;
  const DistillArgs g{(const uint16_t*)logits16, ldl, ids, id_bytes, teacher_logp, weight, N, V, (int)K, cfg->tail,
                      kLog2e / cfg->temperature, cfg->grad_scale / cfg->temperature, (uint16_t*)dlogits16, lddl, token_loss,
                      state ? state->dev : nullptr};
  cudaStream_t st = (cudaStream_t)stream;
  if (N > 0) {
    const int rc = K <= 32 ? by_width<1>(g, st) : by_width<MP_DISTILL_MAX_K / 32>(g, st);
    if (rc) return rc;
  }
  return loss ? mp::sum_token_loss(token_loss, N, loss, st) : MP_OK;
}

// Scores of given tokens: log-probability, entropy of the distribution, and the top alternatives with theirs.
//
// One pass over the row, N V FP16 in and next to nothing out: HBM bounds it, the exponentials (one a word, 16 a clock and
// SM) come close.  The sums are those of the losses with one more, u = sum 2^y y for the entropy
// log2 s - u / s.  The largest logits are found in the same pass: the vectors' maxima of the first few thousand words give a
// value that at least k words reach, words that reach it are listed in shared memory as they stream by (a
// few hundred of a random row), and a warp picks the k largest of the list at the end.  Where the list would
// overflow, the bound is raised to its k-th entry; a row that defeats that too (rising order, thousands of equal
// logits) is counted through again, bit by bit of the FP16 pattern, exactly.  Entries are one whole number, value
// before id, so equal values go by the lower id whatever order they were listed in.

#include <math.h>

#include "ptx.cuh"
#include "softmax.cuh"

namespace {

using namespace softmax;

struct TopArgs {
  const uint16_t* z;
  int64_t ldl;
  const void* targets;
  int id_bytes;
  const float* weight;
  int64_t N, V;
  int k;
  float scale;                                    // log2 e / temperature
  float *logp, *entropy;
  int32_t* ids;
  float* tlogp;
  mp_dev_state* st;
};

// s 2^k = sum 2^(z scale), u = sum 2^y y with y = z scale - k.
struct Sums {
  int k;
  float s, u;
};
__device__ __forceinline__ void rebase(float& s, float& u, float d, float f) {     // y grows by d, f = 2^d
  u = f * fmaf(s, d, u);
  s *= f;
}
template <int LANES>
__device__ __forceinline__ Sums join(Sums v) {
  int k = v.k;
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) k = max(k, __shfl_xor_sync(0xFFFFFFFFu, k, o));
  const float d = (float)(v.k - k);
  rebase(v.s, v.u, d, ex2(d));
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) {
    v.s += __shfl_xor_sync(0xFFFFFFFFu, v.s, o);
    v.u += __shfl_xor_sync(0xFFFFFFFFu, v.u, o);
  }
  v.k = k;
  return v;
}
// A thread's sums.  k follows the largest word and lags by less than 2^8: the entropy is a difference of logarithms, and
// a k far off would cost it bits.
struct Stream {
  float k = 0.0f, s = 0.0f, u = 0.0f;
  bool begun = false, infinite = false;
  __device__ __forceinline__ void add(const uint4& z, float top, float scale) {
    if (!begun || fmaf(top, scale, -k) > 8.0f) {
      const float up = top == -INFINITY ? (float)kNothing : rintf(top * scale);
      if (begun) rebase(s, u, k - up, ex2(k - up));
      k = up;
      begun = true;
      infinite |= top == INFINITY;
    }
    const uint32_t w[4] = {z.x, z.y, z.z, z.w};
    float ss[2] = {0.0f, 0.0f}, uu[2] = {0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
      const float a = fmaf(f.x, scale, -k), b = fmaf(f.y, scale, -k);
      const float ea = ex2(a), eb = ex2(b);
      ss[0] += ea;
      ss[1] += eb;
      uu[0] = fmaf(ea, fmaxf(a, -200.0f), uu[0]);            // 0 times -inf is no summand
      uu[1] = fmaf(eb, fmaxf(b, -200.0f), uu[1]);
    }
    s += ss[0] + ss[1];
    u += uu[0] + uu[1];
  }
  __device__ __forceinline__ Sums sums() const { return begun ? Sums{infinite ? 0 : (int)k, s, u} : Sums{kNothing, 0.0f, 0.0f}; }
};

// ---- entries: 16 bits that order the values, then 20 that order the ids downwards ----
using Entry = unsigned long long;
constexpr uint32_t kLowKey = 0x03FF;              // of -inf; below are NaN patterns
__device__ __forceinline__ uint32_t key_of(uint16_t h) { return h == 0x8000 ? 0x8000u : h & 0x8000 ? 0xFFFFu & ~h : h | 0x8000u; }
__device__ __forceinline__ uint16_t value_of(uint32_t key) { return (uint16_t)(key & 0x8000 ? key & 0x7FFF : ~key); }
__device__ __forceinline__ __half bound_of(uint32_t key) { return __ushort_as_half(value_of(key < kLowKey ? kLowKey : key)); }
__device__ __forceinline__ Entry entry(uint16_t h, int id) { return (Entry)key_of(h) << 20 | (0xFFFFFu - (uint32_t)id); }
__device__ __forceinline__ float logit_of(Entry e) { return rows::h2f(value_of((uint32_t)(e >> 20))); }
__device__ __forceinline__ int id_of(Entry e) { return (int)(0xFFFFFu - (uint32_t)(e & 0xFFFFFu)); }

__device__ __forceinline__ float top8(const uint4& z) {
  const float2 m = __half22float2(max8(__half2half2(__ushort_as_half(0xFC00)), z));
  return fmaxf(m.x, m.y);
}
// Lists the words of a vector (its first at id `at`) that reach the bound.
__device__ __forceinline__ void list8(const uint4& z, int at, float bound, Entry* list, int cap, int* count) {
  const uint32_t w[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint16_t h = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
    if (rows::h2f(h) >= bound) {
      const int n = atomicAdd(count, 1);
      if (n < cap) list[n] = entry(h, at + j);
    }
  }
}
// By a whole warp: moves the k largest of `count` entries (all of them, if fewer) to `out`; returns how many.
__device__ __forceinline__ int pick(const Entry* list, int count, int k, Entry* out) {
  const int lane = threadIdx.x & 31;
  constexpr int R = 8;                            // entries a lane holds in registers
  Entry mine[R];
#pragma unroll
  for (int i = 0; i < R; ++i) mine[i] = i * 32 + lane < count ? list[i * 32 + lane] : 0;
  Entry t = 0;
  if (count > k) {
    for (int bit = 35; bit >= 0; --bit) {
      const Entry cand = t | (Entry)1 << bit;
      int n = 0;
#pragma unroll
      for (int i = 0; i < R; ++i) n += mine[i] >= cand;
      for (int i = R * 32 + lane; i < count; i += 32) n += list[i] >= cand;
      n = __reduce_add_sync(0xFFFFFFFFu, n);
      if (n >= k) t = cand;
      if (n == k) break;
    }
  }
  int have = 0;
  auto keep = [&](Entry e, bool on) {
    const uint32_t m = __ballot_sync(0xFFFFFFFFu, on && e >= t);
    if (on && e >= t) out[have + __popc(m & ((1u << lane) - 1))] = e;
    have += __popc(m);
  };
#pragma unroll
  for (int i = 0; i < R; ++i) keep(mine[i], i * 32 + lane < count);
  for (int i = R * 32; i < count; i += 32) {
    const bool on = i + lane < count;
    keep(on ? list[i + lane] : 0, on);
  }
  __syncwarp();
  return have;
}

// By a whole warp: a row's outputs, from its sums and its `have` picked entries.
__device__ __forceinline__ void put(const TopArgs& a, int64_t i, const Sums& v, const Entry* picked, int have) {
  const int lane = threadIdx.x & 31;
  const float log2s = log2f(v.s), k = (float)v.k;
  auto lp = [&](float z) { return (fmaf(z, a.scale, -k) - log2s) * kLn2; };
  for (int e = lane; e < a.k; e += 32) {
    if (e >= have) {                              // fewer numbers than k
      a.ids[i * a.k + e] = -1;
      a.tlogp[i * a.k + e] = NAN;
      continue;
    }
    const Entry mine = picked[e];
    int rank = 0;
    for (int o = 0; o < have; ++o) rank += picked[o] > mine;
    a.ids[i * a.k + rank] = id_of(mine);
    a.tlogp[i * a.k + rank] = lp(logit_of(mine));
  }
  if (lane == 0) {
    if (a.entropy != nullptr) {
      const float h = (log2s - v.u / v.s) * kLn2;
      a.entropy[i] = h < 0.0f ? 0.0f : h;
    }
    if (a.logp != nullptr) {
      const int64_t t = a.id_bytes == 8 ? rows::load_id<int64_t>(a.targets, i) : rows::load_id<int32_t>(a.targets, i);
      const bool good = t >= 0 && t < a.V;
      a.logp[i] = good ? lp(rows::h2f(a.z[i * a.ldl + t])) : NAN;
      if (!good) rows::record_bad_id(a.st);
    }
  }
}
__device__ __forceinline__ void put_masked(const TopArgs& a, int64_t i) {
  for (int e = threadIdx.x & 31; e < a.k; e += 32) {
    a.ids[i * a.k + e] = -1;
    a.tlogp[i * a.k + e] = 0.0f;
  }
  if ((threadIdx.x & 31) == 0) {
    if (a.entropy != nullptr) a.entropy[i] = 0.0f;
    if (a.logp != nullptr) a.logp[i] = 0.0f;
  }
}
// The largest key that at least `quota` of the values that `count(bound)` sees reach (kLowKey if there are fewer).
template <class F>
__device__ __forceinline__ uint32_t key_reached(int quota, F count) {
  uint32_t t = 0;
#pragma unroll 1
  for (int bit = 15; bit >= 0; --bit) {
    const uint32_t cand = t | 1u << bit;
    if (cand <= kLowKey || count(__half2float(bound_of(cand))) >= quota) t = cand;
  }
  return t;
}

// ---- rows of up to 1024 words: a warp each, the row in registers ----
constexpr int kWarpThreads = 128, kWarpRows = kWarpThreads / 32, kWarpWords = 1024;
template <int C>
__global__ void __launch_bounds__(kWarpThreads) mp_token_top_warp_kernel(const TopArgs a) {
  __shared__ Entry lists[kWarpRows][C * 256];
  __shared__ Entry picks[kWarpRows][MP_TOP_MAX_K];
  __shared__ int counts[kWarpRows];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t i = (int64_t)blockIdx.x * kWarpRows + warp;
  if (i >= a.N) return;
  if (a.weight != nullptr && a.weight[i] == 0.0f) {
    put_masked(a, i);
    return;
  }
  uint4 z[C];
  Stream sums;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int left = (int)a.V - (c * 32 + lane) * 8;
    z[c] = left > 0 ? live8(__ldcs(reinterpret_cast<const uint4*>(a.z + i * a.ldl + (c * 32 + lane) * 8)), left) : no_words();
  }
  if (lane == 0) counts[warp] = 0;
#pragma unroll
  for (int c = 0; c < C; ++c) sums.add(z[c], top8(z[c]), a.scale);
  const Sums v = join<32>(sums.sums());
  const uint32_t t = key_reached(a.k, [&](float bound) {
    int n = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const uint32_t w[4] = {z[c].x, z[c].y, z[c].z, z[c].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
        n += (f.x >= bound) + (f.y >= bound);
      }
    }
    return __reduce_add_sync(0xFFFFFFFFu, n);
  });
  __syncwarp();
  const float bound = __half2float(bound_of(t));
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = (c * 32 + lane) * 8, left = (int)a.V - at;
    if (left >= 8) {
      if (top8(z[c]) >= bound) list8(z[c], at, bound, lists[warp], C * 256, &counts[warp]);
    } else if (left > 0) {                        // the words past the row are -inf and no entries
      const uint32_t w[4] = {z[c].x, z[c].y, z[c].z, z[c].w};
      for (int j = 0; j < left; ++j) {
        const uint16_t h = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
        if (rows::h2f(h) >= bound) lists[warp][atomicAdd(&counts[warp], 1)] = entry(h, at + j);
      }
    }
  }
  __syncwarp();
  put(a, i, v, picks[warp], pick(lists[warp], counts[warp], a.k, picks[warp]));
}

// ---- longer rows: a block, or CL blocks of a cluster when there are few rows ----
constexpr int kThreads = 256, kWarps = kThreads / 32, kBatch = 4;       // vectors of a thread between two looks at the list
constexpr int kCap = 2048, kFull = 1024;          // entries of the list; how many make the bound rise

// The part of a row that a block has: vectors mine, mine + hop, ..
struct Part {
  const uint16_t* z;
  int V, vecs, mine, hop;
  __device__ __forceinline__ uint4 load(int vec) const {
    const int left = V - vec * 8;
    const uint4 q = __ldg(reinterpret_cast<const uint4*>(z) + vec);
    return left >= 8 ? q : live8(q, left);
  }
};
// Words of a vector that exist and reach the bound (a bound of -inf must not count what lies past the row).
__device__ __forceinline__ int reach8(const uint4& z, int left, float bound, bool above) {
  const uint32_t w[4] = {z.x, z.y, z.z, z.w};
  int n = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float f = rows::h2f((uint16_t)(w[j / 2] >> (16 * (j & 1))));
    n += j < left && (above ? f > bound : f >= bound);
  }
  return n;
}
__device__ __forceinline__ void list_part(const uint4& z, int vec, int V, float bound, Entry* list, int* count) {
  if (top8(z) < bound) return;
  if (V - vec * 8 >= 8) {
    list8(z, vec * 8, bound, list, kCap, count);
    return;
  }
  const uint32_t w[4] = {z.x, z.y, z.z, z.w};
  for (int j = 0; j < V - vec * 8; ++j) {
    const uint16_t h = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
    if (rows::h2f(h) >= bound) {
      const int n = atomicAdd(count, 1);
      if (n < kCap) list[n] = entry(h, vec * 8 + j);
    }
  }
}
// The part's k largest by counting: exact whatever the row, 16 reads of it.  By the whole block; `list` receives k entries or all.
__device__ __noinline__ void count_through(const Part& p, int k, Entry* list, int* count, int* scratch) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  auto block_sum = [&](int n) {
    n = __reduce_add_sync(0xFFFFFFFFu, n);
    __syncthreads();
    if (lane == 0) scratch[warp] = n;
    __syncthreads();
    int all = 0;
    for (int w = 0; w < kWarps; ++w) all += scratch[w];
    return all;
  };
  const uint32_t t = key_reached(k, [&](float bound) {
    int n = 0;
    for (int vec = p.mine; vec < p.vecs; vec += p.hop) n += reach8(p.load(vec), p.V - vec * 8, bound, false);
    return block_sum(n);
  });
  const float bound = __half2float(bound_of(t));
  __syncthreads();
  if (threadIdx.x == 0) *count = 0;
  __syncthreads();
  auto each = [&](const uint4& z, int vec, bool above, int& room) {      // lists at most `room` words, in order
    const uint32_t w[4] = {z.x, z.y, z.z, z.w};
    for (int j = 0; j < 8 && vec * 8 + j < p.V; ++j) {
      const uint16_t h = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
      const float f = rows::h2f(h);
      if ((above ? f > bound : f == bound) && room-- > 0) list[atomicAdd(count, 1)] = entry(h, vec * 8 + j);
    }
  };
  for (int vec = p.mine; vec < p.vecs; vec += p.hop) {       // fewer than k lie above the bound
    int room = 8;
    const uint4 z = p.load(vec);
    if (top8(z) > bound) each(z, vec, true, room);
  }
  __syncthreads();
  int need = k - *count;                          // of those at the bound the first ones
  const int first = p.mine - (int)threadIdx.x;
  for (int base = first; base < p.vecs && need > 0; base += p.hop) {
    const int vec = base + threadIdx.x;
    int n = 0;
    uint4 z = no_words();
    if (vec < p.vecs) {
      z = p.load(vec);
      n = reach8(z, p.V - vec * 8, bound, false) - reach8(z, p.V - vec * 8, bound, true);
    }
    int before = n;                               // ties in the vectors of this round up to this one
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xFFFFFFFFu, before, o);
      if (lane >= o) before += x;
    }
    __syncthreads();
    if (lane == 31) scratch[warp] = before;
    __syncthreads();
    int all = 0;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) before += scratch[w];
      all += scratch[w];
    }
    int room = need - (before - n);
    if (n > 0 && room > 0) each(z, vec, false, room);
    need -= all;
  }
  __syncthreads();
}

template <int CL>
__global__ void __launch_bounds__(kThreads) mp_token_top_row_kernel(const TopArgs a) {
  __shared__ Entry list[kCap];
  __shared__ Entry picks[CL * MP_TOP_MAX_K];      // of rank 0: CL > 1, what the blocks picked
  __shared__ Entry final_picks[CL > 1 ? MP_TOP_MAX_K : 1];
  __shared__ Sums part_sums[kWarps], block_sums[CL];
  __shared__ int block_have[CL];
  __shared__ int count, scratch[kWarps];
  __shared__ float warp_bound[kWarps];
  __shared__ uint32_t raised;
  const int rank = CL > 1 ? (int)ptx::cluster_ctarank() : 0, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t i = blockIdx.x / CL;
  if (a.weight != nullptr && a.weight[i] == 0.0f) {          // the same for all blocks of a row
    if (rank == 0 && warp == 0) put_masked(a, i);
    return;
  }
  if constexpr (CL > 1) ptx::cluster_sync();      // every block of the cluster has started
  const int V = (int)a.V, vecs = (V + 7) / 8;
  const Part p{a.z + i * a.ldl, V, vecs, rank * kThreads + (int)threadIdx.x, CL * kThreads};
  Stream sums;
  float bound = 0.0f;
  if (threadIdx.x == 0) count = 0;
  bool overflow = false, looked = false;
  for (int base = rank * kThreads; base < vecs; base += kBatch * p.hop) {
    uint4 z[kBatch];
    float top[kBatch];
#pragma unroll
    for (int c = 0; c < kBatch; ++c) {
      const int vec = base + c * p.hop + threadIdx.x;
      z[c] = vec < vecs ? p.load(vec) : no_words();
    }
#pragma unroll
    for (int c = 0; c < kBatch; ++c) top[c] = top8(z[c]);
    if (!looked) {
      // Each warp finds what its share of k vectors reaches: together at least k words reach the lowest of these.  Warps
      // that have no whole first layer of vectors do not take part.
      const int here = vecs - base, taking = here >= kThreads ? kWarps : here >= 32 ? here / 32 : 1;
      if (warp < taking) {
        const uint32_t t = key_reached((a.k + taking - 1) / taking, [&](float b) {
          int n = 0;
#pragma unroll
          for (int c = 0; c < kBatch; ++c) n += top[c] >= b;
          return __reduce_add_sync(0xFFFFFFFFu, n);
        });
        if (lane == 0) warp_bound[warp] = __half2float(bound_of(t));
      }
      __syncthreads();
      bound = warp_bound[0];
      for (int w = 1; w < taking; ++w) bound = fminf(bound, warp_bound[w]);
      looked = true;
    }
#pragma unroll
    for (int c = 0; c < kBatch; ++c) {
      const int vec = base + c * p.hop + threadIdx.x;
      if (vec < vecs) {
        sums.add(z[c], top[c], a.scale);
        if (!overflow) list_part(z[c], vec, V, bound, list, &count);
      }
    }
    if (base + kBatch * p.hop < vecs && !overflow) {
      // The list is looked at by all together: too long, and the bound rises to its k-th entry.
      if (__syncthreads_or(*(volatile int*)&count > kFull)) {
        overflow = count > kCap;
        __syncthreads();                          // everyone has read the count
        if (!overflow) {
          if (warp == 0) {
            const int have = pick(list, count, a.k, picks);
            Entry least = ~(Entry)0;
            for (int e = lane; e < have; e += 32) {
              least = picks[e] < least ? picks[e] : least;
              list[e] = picks[e];
            }
            const uint32_t key = __reduce_min_sync(0xFFFFFFFFu, (uint32_t)(least >> 20));
            if (lane == 0) {
              count = have;
              raised = key;
            }
          }
          __syncthreads();
          bound = __half2float(bound_of(raised));
        }
      }
    }
  }
  const Sums w = join<32>(sums.sums());
  if (lane == 0) part_sums[warp] = w;
  __syncthreads();
  if (overflow || count > kCap) count_through(p, a.k, list, &count, scratch);
  if constexpr (CL > 1) {
    if (warp == 0) {
      const Sums v = join<kWarps>(part_sums[lane & (kWarps - 1)]);
      Entry* mine = final_picks;                  // free until the blocks have met
      const int have = pick(list, count, a.k, mine);
      // hand them to rank 0
      const uint32_t to = ptx::map_to_cta(ptx::smem_u32(picks + rank * MP_TOP_MAX_K), 0);
      for (int e = lane; e < have; e += 32)
        asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(to + e * 8), "l"(mine[e]) : "memory");
      if (lane == 0) {
        const uint32_t s = ptx::map_to_cta(ptx::smem_u32(&block_sums[rank]), 0), h = ptx::map_to_cta(ptx::smem_u32(&block_have[rank]), 0);
        asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(s), "r"(v.k) : "memory");
        asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(s + 4), "r"(__float_as_int(v.s)) : "memory");
        asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(s + 8), "r"(__float_as_int(v.u)) : "memory");
        asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(h), "r"(have) : "memory");
      }
      __syncwarp();
    }
    ptx::cluster_sync();
    if (rank == 0 && warp == 0) {
      const Sums v = join<CL>(block_sums[lane & (CL - 1)]);
      int all = 0;                                // one list of what the blocks picked
      for (int r = 0; r < CL; ++r) {
        for (int e = lane; e < block_have[r]; e += 32) list[all + e] = picks[r * MP_TOP_MAX_K + e];
        all += block_have[r];
      }
      __syncwarp();
      const int have = pick(list, all, a.k, final_picks);
      put(a, i, v, final_picks, have);
    }
  } else {
    if (warp == 0) {
      const Sums v = join<kWarps>(part_sums[lane & (kWarps - 1)]);
      const int have = pick(list, count, a.k, picks);
      put(a, i, v, picks, have);
    }
  }
}

template <int C>
void warp_launch(const TopArgs& a, cudaStream_t st) {
  mp_token_top_warp_kernel<C><<<(unsigned)((a.N + kWarpRows - 1) / kWarpRows), kWarpThreads, 0, st>>>(a);
}

}  // namespace

extern "C" int mp_token_top(const void* logits16, int64_t ldl, const void* targets, int id_bytes, const float* weight,
                            int64_t N, int64_t V, int64_t k, float temperature, float* logp, float* entropy, int32_t* top_ids,
                            float* top_logp, mp_state* state, void* stream) {
  const char* name = "mp_token_top";
  if (N < 0 || V <= 0 || k <= 0 || k > V || ldl < V || (id_bytes != 4 && id_bytes != 8))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: bad size, pitch or id width", name);
  if (!(temperature >= MP_MIN_TEMPERATURE) || !(temperature <= MP_MAX_TEMPERATURE))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: the temperature must be %g .. %g", name, MP_MIN_TEMPERATURE, MP_MAX_TEMPERATURE);
  if (V > MP_POLICY_MAX_V || k > MP_TOP_MAX_K || N > 0x07FFFFFF)
    return mp::set_error(MP_ERR_TOO_LARGE, "%s: V beyond %d, k beyond %d or N beyond 2^27 - 1", name, MP_POLICY_MAX_V, MP_TOP_MAX_K);
  if (N > 0 && (!logits16 || !top_ids || !top_logp || !targets != !logp))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: null pointer (targets and logp: both or none)", name);
  const uintptr_t words = (uintptr_t)weight | (uintptr_t)logp | (uintptr_t)entropy | (uintptr_t)top_ids | (uintptr_t)top_logp;
  if ((ldl & 7) || !mp::aligned16(logits16) || (words & 3) || ((uintptr_t)targets & (uintptr_t)(id_bytes - 1)))
    return mp::set_error(MP_ERR_ALIGNMENT, "%s: logits must be 16-byte aligned with a pitch that is a multiple of 8, ids and "
                         "FP32 values aligned to their width", name);
  if (int rc = mp::check_device()) return rc;
  if (N == 0) return MP_OK;
  const TopArgs a{(const uint16_t*)logits16, ldl, targets, id_bytes, weight, N, V, (int)k, kLog2e / temperature, logp, entropy,
                  top_ids, top_logp, state ? state->dev : nullptr};
  cudaStream_t st = (cudaStream_t)stream;
  if (V <= 256) warp_launch<1>(a, st);
  else if (V <= 512) warp_launch<2>(a, st);
  else if (V <= kWarpWords) warp_launch<4>(a, st);
  else if (N > 148 || V <= 8 * kThreads * 8)
    mp_token_top_row_kernel<1><<<(unsigned)N, kThreads, 0, st>>>(a);
  else {                                          // fewer rows than SMs, each long enough for eight blocks
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(N * 8), 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 8;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    MP_CUDA_TRY(cudaLaunchKernelEx(&cfg, mp_token_top_row_kernel<8>, a));
  }
  mp::count_launch();
  MP_CUDA_TRY(cudaGetLastError());
  return MP_OK;
}

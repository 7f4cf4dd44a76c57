// Scores of given tokens: log-probability, entropy of the distribution, and the top alternatives with theirs.
//
// One read of the row, N V FP16 in and next to nothing out: HBM bounds it, the exponentials (one a word, 16 a clock and
// SM) come close.  The sums are those of the losses with one more, u = sum 2^y y for the entropy
// log2 s - u / s.  A row waits in shared memory (short ones: in a warp's registers) while three things are taken from it in
// turn: each thread's two best vectors, the sums, and the words that reach a bound.  The bound: a value that each warp's share
// of k lanes' maxima reach, and of these the lowest, so k words at least reach it; of a random row some dozens more do.  They are
// listed, and an entry's place is the number of larger ones.  Where the list would overflow (rising order, thousands
// of equal logits) the row is counted through bit by bit of the FP16 pattern, exactly.  Entries are one whole number,
// value before id, so equal values go by the lower id whatever order they were listed in.
//
// 8192 x 32768, 20 alternatives: 170 us where the bytes alone take 74 (393 in one pass without the row kept, whose list grew
// long before a good bound was known): a row's phases wait for one another, and the three blocks that fit an SM cover that in
// part.  128 alternatives take 340 us: of normal rows some 180 words are listed then, each compared with all, and in a quarter of the rows
// more than kOrdered, whose k largest one warp picks while the others wait.  Short rows are far from their bytes (40000 x 1000: 141 us with 20,
// 274 with 128, the bytes 13 and 18): sixteen rounds of counting, each over all words of a lane, and a list made word by word.

#include <math.h>

#include "ptx.cuh"
#include "softmax.cuh"

namespace {

using namespace softmax;
using rows::add2;
using rows::fma2;

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
// A thread's sums, with k near its largest word: the entropy is a difference of logarithms, and a k far off would cost it bits.
struct Tally {
  float k, s = 0.0f, u = 0.0f;
  bool infinite;
  __device__ __forceinline__ Tally(float top, float scale)
      : k(top == -INFINITY ? (float)kNothing : rintf(top * scale)), infinite(top == INFINITY) {}
  __device__ __forceinline__ void add(const uint4& z, float scale) {
    const uint32_t w[4] = {z.x, z.y, z.z, z.w};
    const float2 sc = make_float2(scale, scale), mk = make_float2(-k, -k);
    float2 ss = make_float2(0.0f, 0.0f), uu = ss;  // of the vector: long sums of small ones lose bits
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 y = fma2(__half22float2(*reinterpret_cast<const __half2*>(&w[j])), sc, mk);
      const float2 e = make_float2(ex2(y.x), ex2(y.y));
      ss = add2(ss, e);
      uu = fma2(e, make_float2(fmaxf(y.x, -200.0f), fmaxf(y.y, -200.0f)), uu);      // 0 times -inf is no summand
    }
    s += ss.x + ss.y;
    u += uu.x + uu.y;
  }
  __device__ __forceinline__ Sums sums() const { return Sums{infinite ? 0 : (int)k, s, u}; }
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
// Bits of the first `left` words of a vector that reach the bound.
__device__ __forceinline__ uint32_t reach8(const uint4& z, __half2 bound, int left) {
  const uint32_t w[4] = {z.x, z.y, z.z, z.w};
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t hit = __hge2_mask(*reinterpret_cast<const __half2*>(&w[j]), bound);
    m |= ((hit & 1) | (hit >> 16 & 2)) << (2 * j);
  }
  return left >= 8 ? m : m & ((1u << left) - 1);
}
// Lists the first `left` words of a vector (its first at id `at`) that reach the bound.
__device__ __forceinline__ void list8(const uint4& z, int at, int left, __half2 bound, Entry* list, int cap, int* count) {
  const uint32_t w[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t hit = __hge2_mask(*reinterpret_cast<const __half2*>(&w[j]), bound);
    if (hit == 0) continue;
    auto one = [&](int e) {
      const int n = atomicAdd(count, 1);
      if (n < cap) list[n] = entry((uint16_t)(w[j] >> (16 * e)), at + 2 * j + e);
    };
    if ((hit & 1) && 2 * j < left) one(0);
    if ((hit >> 16) && 2 * j + 1 < left) one(1);
  }
}
// By a whole warp: moves the k largest of `count` entries (all of them, if fewer) to `out`; returns how many.  R * 32 entries
// are held in registers, what is beyond is read again in every round.  At most MOST entries.
template <int MOST>
__device__ __noinline__ int pick(const Entry* list, int count, int k, Entry* out) {
  const int lane = threadIdx.x & 31;
  constexpr int R = 4;
  Entry mine[R];
#pragma unroll
  for (int i = 0; i < R; ++i) mine[i] = i * 32 + lane < count ? list[i * 32 + lane] : 0;
  Entry t = 0;
  if (count > k) {
    // The k-th value first, two bits a round (three bounds at once), from the first bit on in which the
    // values differ; then among those that equal it the k-th id.  Done when a bound leaves just k.
    uint32_t key[R], most = 0, least = ~0u;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      key[i] = (uint32_t)(mine[i] >> 20);
      most = max(most, key[i]);
      least = i * 32 + lane < count ? min(least, key[i]) : least;
    }
    for (int i = R * 32 + lane; i < count; i += 32) {
      const uint32_t x = (uint32_t)(list[i] >> 20);
      most = max(most, x);
      least = min(least, x);
    }
    most = __reduce_max_sync(0xFFFFFFFFu, most);
    least = __reduce_min_sync(0xFFFFFFFFu, least);
    int bit = (33 - __clz(most ^ least)) & ~1, n = count;    // even, all bits from here up are alike
    uint32_t v = most >> bit << bit;
    while (bit > 0 && n != k) {
      bit -= 2;
      const uint32_t c1 = v + (1u << bit), c2 = v + (2u << bit), c3 = v + (3u << bit);
      uint32_t here = 0, high = 0;                // three counts in a word, if 10 bits are enough for the last
      constexpr bool kOne = MOST <= 1023;
      auto add = [&](uint32_t x) {
        here += (x >= c1) + (x >= c2 ? 1u << 11 : 0);
        if (kOne) here += x >= c3 ? 1u << 22 : 0;
        else high += x >= c3;
      };
#pragma unroll
      for (int i = 0; i < R; ++i) add(key[i]);
      for (int i = R * 32 + lane; i < count; i += 32) add((uint32_t)(list[i] >> 20));
      here = __reduce_add_sync(0xFFFFFFFFu, here);
      const int n1 = here & 0x7FF, n2 = here >> 11 & 0x7FF, n3 = kOne ? here >> 22 : __reduce_add_sync(0xFFFFFFFFu, high);
      if (n3 >= k) { v = c3; n = n3; }
      else if (n2 >= k) { v = c2; n = n2; }
      else if (n1 >= k) { v = c1; n = n1; }
    }
    t = (Entry)v << 20;
    for (bit = 19; bit >= 0 && n != k; --bit) {
      const Entry cand = t | (Entry)1 << bit;
      int here = 0;
#pragma unroll
      for (int i = 0; i < R; ++i) here += mine[i] >= cand;
      for (int i = R * 32 + lane; i < count; i += 32) here += list[i] >= cand;
      here = __reduce_add_sync(0xFFFFFFFFu, here);
      if (here >= k) {
        t = cand;
        n = here;
      }
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

// A row's outputs: one of its entries, a place that no number is left for, and what goes with the row.
__device__ __forceinline__ float lp_of(const TopArgs& a, const Sums& v, float z) {
  return (fmaf(z, a.scale, -(float)v.k) - log2f(v.s)) * kLn2;
}
__device__ __forceinline__ void put_one(const TopArgs& a, int64_t i, const Sums& v, int place, Entry e) {
  a.ids[i * a.k + place] = id_of(e);
  a.tlogp[i * a.k + place] = lp_of(a, v, logit_of(e));
}
__device__ __forceinline__ void put_none(const TopArgs& a, int64_t i, int place) {
  a.ids[i * a.k + place] = -1;
  a.tlogp[i * a.k + place] = NAN;
}
__device__ __forceinline__ void put_row(const TopArgs& a, int64_t i, const Sums& v) {
  if (a.entropy != nullptr) {
    const float h = (log2f(v.s) - v.u / v.s) * kLn2;
    a.entropy[i] = h < 0.0f ? 0.0f : h;
  }
  if (a.logp != nullptr) {
    const int64_t t = a.id_bytes == 8 ? rows::load_id<int64_t>(a.targets, i) : rows::load_id<int32_t>(a.targets, i);
    const bool good = t >= 0 && t < a.V;
    a.logp[i] = good ? lp_of(a, v, rows::h2f(a.z[i * a.ldl + t])) : NAN;
    if (!good) rows::record_bad_id(a.st);
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

// ---- rows of up to 1024 words: a warp each, the row in registers (40000 x 1000, 20 alternatives: 141 us, a block each 283) ----
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
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int left = (int)a.V - (c * 32 + lane) * 8;
    z[c] = left > 0 ? live8(__ldcs(reinterpret_cast<const uint4*>(a.z + i * a.ldl + (c * 32 + lane) * 8)), left) : no_words();
  }
  if (lane == 0) counts[warp] = 0;
  float top = -INFINITY;
#pragma unroll
  for (int c = 0; c < C; ++c) top = fmaxf(top, top8(z[c]));
  Tally tally(top, a.scale);
#pragma unroll
  for (int c = 0; c < C; ++c) tally.add(z[c], a.scale);
  const Sums v = join<32>(tally.sums());
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
  const __half2 bound = __half2half2(bound_of(t));
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = (c * 32 + lane) * 8, left = (int)a.V - at;     // words past the row are no entries
    if (left > 0) list8(z[c], at, left, bound, lists[warp], C * 256, &counts[warp]);
  }
  __syncwarp();
  const int have = pick<C * 256>(lists[warp], counts[warp], a.k, picks[warp]);
  for (int e = lane; e < a.k; e += 32) {
    if (e >= have) {
      put_none(a, i, e);
      continue;
    }
    const Entry mine = picks[warp][e];
    int place = 0;
#pragma unroll 8
    for (int o = 0; o < have; ++o) place += picks[warp][o] > mine;
    put_one(a, i, v, place, mine);
  }
  if (lane == 0) put_row(a, i, v);
}

// ---- longer rows: a block for a row, or CL blocks of a cluster, the row in their shared memory ----
//
// Persistent blocks, whose threads bring their own vectors of the next row by asynchronous copies as soon as they are done with this
// one's, so each thread reads what it copied itself, and what covers a block's waits are the others on the SM.
constexpr int kPartWords = 32768;                 // words of a row that a block takes if a cluster of 8 can
constexpr int kCap = 1024;                        // entries of the list
constexpr int kOrdered = 192;                     // so many are ordered by comparing all with all; of more the k largest are picked

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
__device__ __forceinline__ int count8(const uint4& z, int left, float bound, bool above) {
  const uint32_t w[4] = {z.x, z.y, z.z, z.w};
  int n = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float f = rows::h2f((uint16_t)(w[j / 2] >> (16 * (j & 1))));
    n += j < left && (above ? f > bound : f >= bound);
  }
  return n;
}
// The part's k largest by counting: exact whatever the row, 16 reads of it.  By the whole block; `list` receives k entries or all.
template <int kThreads>
__device__ __noinline__ void count_through(const Part& p, int k, Entry* list, int* count, int* scratch) {
  constexpr int kWarps = kThreads / 32;
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
    for (int vec = p.mine; vec < p.vecs; vec += p.hop) n += count8(p.load(vec), p.V - vec * 8, bound, false);
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
      n = count8(z, p.V - vec * 8, bound, false) - count8(z, p.V - vec * 8, bound, true);
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

template <int CL, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads == 256 ? 3 : 8) mp_token_top_row_kernel(const TopArgs a) {
  constexpr int kWarps = kThreads / 32;
  extern __shared__ uint4 slots[];                // [vectors]
  __shared__ Entry list[kCap];
  __shared__ Entry gathered[2][CL > 1 ? CL * MP_TOP_MAX_K : 1];           // rank 0: what each block sorted
  __shared__ Sums part_sums[2][kWarps], block_sums[2][CL];
  __shared__ int block_have[2][CL], count[2], scratch[kWarps];
  __shared__ float bounds[CL * kWarps];           // of every warp of the row's blocks
  const int rank = CL > 1 ? (int)ptx::cluster_ctarank() : 0, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t step = gridDim.x / CL;
  const int V = (int)a.V, vecs = (V + 7) / 8, mine = rank * kThreads + (int)threadIdx.x;     // vector c: mine + c CL threads
  const int own = mine < vecs ? (vecs - mine + CL * kThreads - 1) / (CL * kThreads) : 0;
  const int layers = (vecs - rank * kThreads + CL * kThreads - 1) / (CL * kThreads);
  // every vector but perhaps the row's last is whole
  const int whole = own > 0 && (mine + (own - 1) * CL * kThreads) * 8 + 8 > V ? own - 1 : own, tail = own > whole ? V % 8 : 0;
  const uint32_t base = ptx::smem_u32(slots) + threadIdx.x * 16;
  uint4* z = slots + threadIdx.x;
  // Each warp's share of k: when every warp has a value that so many of its words reach, k words of the row reach the lowest
  // of these values.  Every thread has a vector at least: a row has more than 128 vectors for 128 threads, and for 256 in CL blocks
  // CL * 256 of them.
  const int share = (a.k + CL * kWarps - 1) / (CL * kWarps);
  auto weight_of = [&](int64_t i) { return i >= a.N ? 0.0f : a.weight ? __ldg(a.weight + i) : 1.0f; };
  auto fetch = [&](int64_t i) {
    const uint16_t* from = a.z + i * a.ldl + (int64_t)mine * 8;
#pragma unroll 4
    for (int c = 0; c < own; ++c)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(base + c * kThreads * 16), "l"(from + c * (CL * kThreads * 8)) : "memory");
  };
  if constexpr (CL > 1) ptx::cluster_sync();      // every block of the cluster has started
  int half = 0, turn = 0;
  float w = weight_of(blockIdx.x / CL);
  if (w != 0.0f) fetch(blockIdx.x / CL);          // a masked row is not read
  for (int64_t i = blockIdx.x / CL; i < a.N; i += step) {
    const float w_next = weight_of(i + step);
    if (w == 0.0f) {
      if (rank == 0 && warp == 0) put_masked(a, i);
      if (w_next != 0.0f) fetch(i + step);
      w = w_next;
      continue;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (tail > 0) z[whole * kThreads] = live8(z[whole * kThreads], tail);
    // the vectors with the largest and the second largest maxima, and the largest of the others'
    float top = -INFINITY, second = -INFINITY, third = -INFINITY;
    int in = 0, in2 = 0;
#pragma unroll 4
    for (int c = 0; c < own; ++c) {
      const float x = top8(z[c * kThreads]);
      const bool first = x > top;
      third = fmaxf(third, fminf(second, x));
      in2 = first ? in : x > second ? c : in2;
      second = fmaxf(second, fminf(top, x));
      in = first ? c : in;
      top = fmaxf(top, x);
    }
    Tally tally(top, a.scale);
#pragma unroll 4
    for (int c = 0; c < own; ++c) tally.add(z[c * kThreads], a.scale);
    const Sums part = join<32>(tally.sums());
    // the share-th largest of the lanes' maxima: a few by taking the largest away, more (and the second ones too) by comparing
    // all with all
    float mine_reaches;
    if (share <= 4) {
      const int bits = __float_as_int(top);
      int key = bits ^ (bits >> 31 & 0x7FFFFFFF), best = 0;  // ordered as the values are
      for (int s = 0; s < share; ++s) {
        best = __reduce_max_sync(0xFFFFFFFFu, key);
        const uint32_t has = __ballot_sync(0xFFFFFFFFu, key == best);
        if (lane == __ffs(has) - 1) key = (int)0x80000000;
      }
      mine_reaches = __int_as_float(best ^ (best >> 31 & 0x7FFFFFFF));
    } else {
      int above = 0, reach = 0, above2 = 0, reach2 = 0;
#pragma unroll 8
      for (int l = 0; l < 32; ++l) {
        const float x = __shfl_sync(0xFFFFFFFFu, top, l), y = __shfl_sync(0xFFFFFFFFu, second, l);
        above += (x > top) + (y > top);
        reach += (x >= top) + (y >= top);
        above2 += (x > second) + (y > second);
        reach2 += (x >= second) + (y >= second);
      }
      const uint32_t at = __ballot_sync(0xFFFFFFFFu, above < share && reach >= share);
      const uint32_t at2 = __ballot_sync(0xFFFFFFFFu, above2 < share && reach2 >= share);
      const float x = __shfl_sync(0xFFFFFFFFu, top, at ? __ffs(at) - 1 : 0), y = __shfl_sync(0xFFFFFFFFu, second, at2 ? __ffs(at2) - 1 : 0);
      mine_reaches = at ? x : y;
    }
    if (threadIdx.x == 0) count[turn] = 0;
    if (lane == 0) part_sums[turn][warp] = part;
    float bound;
    if constexpr (CL > 1) {
      if (lane < CL) {
        const uint32_t to = ptx::map_to_cta(ptx::smem_u32(&bounds[rank * kWarps + warp]), lane);
        asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(to), "r"(__float_as_int(mine_reaches)) : "memory");
      }
      __syncwarp();
      ptx::cluster_sync();
      bound = bounds[lane % (CL * kWarps)];
      if (CL * kWarps > 32) bound = fminf(bound, bounds[lane + 32 < CL * kWarps ? lane + 32 : lane]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) bound = fminf(bound, __shfl_xor_sync(0xFFFFFFFFu, bound, o));
    } else {
      if (lane == 0) bounds[warp] = mine_reaches;
      __syncthreads();
      bound = bounds[0];
      for (int x = 1; x < kWarps; ++x) bound = fminf(bound, bounds[x]);
    }
    // The few threads whose largest word reaches the bound list what does so in its vector; fewer have another such vector, and
    // hardly one a third.
    const __half2 two = __float2half2_rn(bound);             // an FP16 value
    auto list_vector = [&](int c, bool on) {                 // by a whole warp
      const int vec = mine + c * CL * kThreads;
      uint32_t hits = on ? reach8(z[c * kThreads], two, V - vec * 8) : 0;
      for (uint32_t any = __ballot_sync(0xFFFFFFFFu, hits); any; any = __ballot_sync(0xFFFFFFFFu, hits)) {
        int to = 0;
        if (lane == 0) to = atomicAdd(&count[turn], __popc(any));
        to = __shfl_sync(0xFFFFFFFFu, to, 0) + __popc(any & ((1u << lane) - 1));
        const int j = __ffs(hits) - 1;
        if (hits && to < kCap) list[to] = entry(reinterpret_cast<const uint16_t*>(z + c * kThreads)[j], vec * 8 + j);
        hits &= hits - 1;
      }
    };
    if (__any_sync(0xFFFFFFFFu, top >= bound)) list_vector(in, top >= bound && own > 0);
    if (__any_sync(0xFFFFFFFFu, second >= bound)) list_vector(in2, second >= bound && own > 1);
    if (__any_sync(0xFFFFFFFFu, third >= bound))
      for (int c = 0; c < layers; ++c) list_vector(c < own ? c : 0, c < own && c != in && c != in2 && third >= bound);
    __syncthreads();
    if (w_next != 0.0f) fetch(i + step);          // the slots have been read
    w = w_next;
    int n = count[turn];
    if (n > kCap) {
      const Part p{a.z + i * a.ldl, V, vecs, mine, CL * kThreads};
      count_through<kThreads>(p, a.k, list, &count[turn], scratch);
      n = count[turn];
    } else if (n > kOrdered) {
      if (warp == 0) pick<kCap>(list, n, a.k, list);
      __syncthreads();
      n = min(n, a.k);
    }
    const int have = min(n, a.k);
    Sums v{0, 0.0f, 0.0f};
    if (warp * 32 < max(n, 1)) v = join<kWarps>(part_sums[turn][lane & (kWarps - 1)]);
    turn ^= 1;                                    // a warp may be a row ahead
    for (int e = threadIdx.x; e - lane < n; e += kThreads) {
      // an entry's place: how many are larger
      const Entry mine_is = list[min(e, n - 1)];
      int place = 0;
#pragma unroll 8
      for (int o = 0; o < n; ++o) place += list[o] > mine_is;
      if (e >= n || place >= a.k) continue;
      if constexpr (CL == 1) {
        put_one(a, i, v, place, mine_is);
      } else {                                    // rank 0 gets it
        const uint32_t to = ptx::map_to_cta(ptx::smem_u32(gathered[half] + rank * MP_TOP_MAX_K + place), 0);
        asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(to), "l"(mine_is) : "memory");
      }
    }
    if constexpr (CL == 1) {
      if ((int)threadIdx.x >= have && (int)threadIdx.x < a.k) put_none(a, i, threadIdx.x);
      if (threadIdx.x == 0) put_row(a, i, v);
    }
    if constexpr (CL > 1) {
      if (threadIdx.x == 0) {
        const uint32_t s = ptx::map_to_cta(ptx::smem_u32(&block_sums[half][rank]), 0);
        const uint32_t h = ptx::map_to_cta(ptx::smem_u32(&block_have[half][rank]), 0);
        asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(s), "r"(v.k) : "memory");
        asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(s + 4), "r"(__float_as_int(v.s)) : "memory");
        asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(s + 8), "r"(__float_as_int(v.u)) : "memory");
        asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(h), "r"(have) : "memory");
      }
      ptx::cluster_sync();
      if (rank == 0) {
        v = join<CL>(block_sums[half][lane & (CL - 1)]);
        // an entry's place is its place in its own list and the number of larger ones in each of the others
        const int* in = block_have[half];
        int all = 0;
#pragma unroll
        for (int r = 0; r < CL; ++r) all += in[r];
        for (int x = threadIdx.x; x < CL * a.k; x += kThreads) {
          const int r = x / a.k, e = x - r * a.k;
          if (e >= in[r]) continue;
          const Entry entry = gathered[half][r * MP_TOP_MAX_K + e];
          int before[CL], to = 0;                 // (own list: finds itself)
#pragma unroll
          for (int o = 0; o < CL; ++o) before[o] = 0;
#pragma unroll
          for (int hop = MP_TOP_MAX_K; hop > 0; hop >>= 1)
#pragma unroll
            for (int o = 0; o < CL; ++o)
              if (before[o] + hop <= in[o] && gathered[half][o * MP_TOP_MAX_K + before[o] + hop - 1] > entry) before[o] += hop;
#pragma unroll
          for (int o = 0; o < CL; ++o) to += before[o];
          if (to < a.k) put_one(a, i, v, to, entry);
        }
        if ((int)threadIdx.x >= all && (int)threadIdx.x < a.k) put_none(a, i, threadIdx.x);
        if (threadIdx.x == 0) put_row(a, i, v);
      }
      half ^= 1;
    }
  }
}

// Persistent grid of whole clusters, as many as are resident at once (asked once per device, kernel and size of a part).
template <int CL, int kThreads>
int row_launch(const TopArgs& a, cudaStream_t st) {
  static mp::PerDevice resident[MP_POLICY_MAX_V / 8 / (CL * kThreads) + 2];        // by layers
  const int64_t vecs = (a.V + 7) / 8, layers = (vecs + CL * kThreads - 1) / (CL * kThreads);
  auto kernel = mp_token_top_row_kernel<CL, kThreads>;
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
  if (a.N < clusters) clusters = (int)a.N;
  cfg.gridDim = dim3((unsigned)(clusters * CL), 1, 1);
  MP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, a));
  return MP_OK;
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
  else {
    // A block takes up to kPartWords of a row.  Up to 16384 words blocks of 128 threads, of which twice as many fit an SM, do more
    // rows at once (16000 x 12000, 40 alternatives: 222 us against 323 with 256 threads; 8192 x 20000: 147 against 136).  Where the
    // rows leave SMs idle, two or four blocks share one if every thread has a vector of it then (16 x 32768, 128 alternatives:
    // four 10.3 us, two 12.4, one 16.5; 74 rows: 12.4, 12.4, 17.2; 148: 18.6, 14.5, 18.6; eight are slower than four at each).
    const int rc = V > 4 * kPartWords ? row_launch<8, 256>(a, st)
                   : V > 2 * kPartWords || (N <= 74 && V >= 4 * 256 * 8) ? row_launch<4, 256>(a, st)
                   : V > kPartWords || (N <= 148 && V >= 2 * 256 * 8) ? row_launch<2, 256>(a, st)
                   : V > 16384 ? row_launch<1, 256>(a, st) : row_launch<1, 128>(a, st);
    if (rc) return rc;
  }
  mp::count_launch();
  MP_CUDA_TRY(cudaGetLastError());
  return MP_OK;
}

// Attention over packed sequences, backward, from the forward pass's outputs and log-sums.
//
// With P = exp(scale S - lse), delta = rowsum(dO O):
//   dV = P^T dO,   dP = dO V^T,   dS = P (dP - delta),   dQ = scale dS K,   dK = scale dS^T Q.
// The probabilities are formed again from S, tile by tile.  dQ sums over the keys and dK, dV over the queries: two kinds of
// blocks form S and dP each for itself (7 products where 5 would do), because sums of both kinds in one
// would need floating-point atomics or partial sums in memory, and the same inputs must give the same bits.
//   keys' blocks: a tile of 128 keys of a key head; over the query heads that share it and their query tiles:
//     S^T = K Q^T, dP^T = V dO^T, P^T and dS^T into their places as FP16, dV += P^T dO, dK += dS^T Q.
//   queries' blocks: a tile of 128 queries of a head, over the key tiles: S = Q K^T, dP = dO V^T, dQ += dS K.
// Both kinds are one launch, the keys' blocks (the longer ones) first.
//
// What bounds it.  Heads of 128: the 7 products are 0.58 ms of the 0.87 that 8192 tokens, causal, 16 heads take (0.98 when the card
// runs it for seconds); the tensor core is busy 52 %, the rest goes to what the two kinds of product wait for, P and dS on
// their way through registers and shared memory.  Sixteen warps compute (eight, with two tiles of A, took 1.07 ms), and the next scores are formed
// while these are worked on, into a second place, from a third tile of A.  Two warps that issue products, which helped the
// forward pass, took 5 % longer here.  Heads of 64, 16 sequences of 512 on average, 16 heads: 185 .. 190 us, of which 15 go to the
// kernel ahead; a block has some four steps and an SM to itself, so nothing covers its place, first copies and last stores, and the last tile of
// a sequence costs a whole one (64 x 400, 25 heads: 980 us, ten times its operations).
//
// FP16 operands P and dS.  P, at most 1, is multiplied by 2^12, so that weights down to 2^-26 keep all their bits.
// |dS| is at most B = 2 max |dO_i| max |v_j| (row norms, Cauchy and Schwarz), so dS is formed times the power of two
// that takes B to 2^14 .. 2^15: it cannot overflow, and 2^-29 of B keeps all its bits, whatever the loss scale.  A
// kernel ahead of the two takes delta and the norms.

#include <math.h>

#include "attention.cuh"

namespace {

using namespace attn;

constexpr int kSlots = 32;                        // partial maxima of a head: one for each block of the first kernel
constexpr float kUp = 12.0f;                      // P is held times 2^kUp

struct BwdArgs {
  Shape s;
  const uint16_t *o, *dout, *v;
  int64_t ldo, lddo, ldv;
  const float* lse;
  uint16_t *dq, *dk, *dv;
  int64_t lddq, lddk, lddv;
  float *delta, *norms;                           // [heads][T]; [heads + kv_heads][kSlots]
  int slots;
  int key_blocks;                                 // blocks of the first kind
};

// delta of every row and head, and the largest squared norms of the rows of dO and v.  Blocks (slot, head or
// heads + key head); L lanes share a row's head, 8 elements each.
constexpr int kPrepThreads = 256;
template <int L>
__global__ void __launch_bounds__(kPrepThreads) mp_attention_prep_kernel(const BwdArgs a) {
  const Shape& s = a.s;
  ptx::launch_dependents();
  ptx::grid_dependency_wait();
  const int64_t from = max(offset_at(s, 0), (int64_t)0), to = min(offset_at(s, s.n_seq), s.T);
  const int head = blockIdx.y, col = (threadIdx.x % L) * 8;
  const bool queries = head < s.heads, inside = col < s.D;
  const int64_t c = (int64_t)(queries ? head : head - s.heads) * s.D + col;
  constexpr int R = kPrepThreads / L;
  float top = 0.0f;
  for (int64_t base = from + (int64_t)blockIdx.x * R; base < to; base += (int64_t)gridDim.x * R) {
    const int64_t i = base + threadIdx.x / L;
    float d[8], o[8], dot = 0.0f, sq = 0.0f;
    rows::Raw8<uint16_t> rd, ro;
    const bool on = inside && i < to;
    rd.load_cached(queries ? a.dout + i * a.lddo + c : a.v + i * a.ldv + c, on ? 8 : 0);
    ro.load_cached(a.o + i * a.ldo + c, on && queries ? 8 : 0);
    rd.floats(d);
    ro.floats(o);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      dot = fmaf(d[e], o[e], dot);
      sq = fmaf(d[e], d[e], sq);
    }
#pragma unroll
    for (int m = L / 2; m > 0; m >>= 1) {
      dot += __shfl_xor_sync(0xFFFFFFFFu, dot, m);
      sq += __shfl_xor_sync(0xFFFFFFFFu, sq, m);
    }
    if (queries && col == 0 && i < to) a.delta[(int64_t)head * s.T + i] = dot;
    top = sq > top || sq != sq ? sq : top;        // a NaN stays
  }
  __shared__ uint32_t most;
  if (threadIdx.x == 0) most = 0;
  __syncthreads();
  atomicMax(&most, __float_as_uint(top) & 0x7FFFFFFFu);      // squares: as whole numbers in the same order, NaN on top
  __syncthreads();
  if (threadIdx.x == 0) a.norms[head * kSlots + blockIdx.x] = __uint_as_float(most);
}

// The power of two that dS of key head kv is formed with: by a whole warp.
__device__ __forceinline__ float ds_exponent(const BwdArgs& a, int kv) {
  const int lane = threadIdx.x & 31, group = a.s.heads / a.s.kv_heads;
  float d = 0.0f, v = 0.0f;
  if (lane < a.slots) {
    for (int h = 0; h < group; ++h) {
      const float x = a.norms[(kv * group + h) * kSlots + lane];
      d = x > d || x != x ? x : d;
    }
    v = a.norms[(a.s.heads + kv) * kSlots + lane];
  }
  const uint32_t dm = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(d)), vm = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(v));
  if (dm >= 0x7F800000u || vm >= 0x7F800000u || dm == 0 || vm == 0) return 0.0f;    // inf and NaN go their way
  const float bound = 2.0f * sqrtf(__uint_as_float(dm)) * sqrtf(__uint_as_float(vm));
  return 15.0f - ceilf(log2f(bound) + 0.01f);
}

// Shared memory: two tiles that stay, rings of the tiles that pass (A: queries, or keys; B: gradients, or values), the queries'
// statistics, the barriers.  Nothing is declared apart, so that seven tiles of a head of 128 elements fit: a third place
// for A is what lets the next scores be formed while these are worked on.
template <int DP>
struct BwdLayout {
  static constexpr int kBoxes = DP / 64, kTileBytes = kBoxes * kBoxBytes;
  static constexpr int kA = DP == 64 ? 4 : 3, kB = DP == 64 ? 4 : 2, kStats = 2;
  static constexpr int kStatBytes = 2 * kTile * 4, kBarBytes = 512;
  static constexpr int kSmem = (2 + kA + kB) * kTileBytes + kStats * kStatBytes + kBarBytes;
};
static_assert(BwdLayout<128>::kSmem <= 232448, "of a block");
// Sixteen warps that compute (four a quarter of the columns, a row a thread), then one each for products, copies, row statistics.
constexpr int kCompute = 16, kProducts = 16, kCopies = 17, kStatistics = 18, kBwdThreads = 19 * 32;

struct BwdBars {
  uint64_t fixed_full, full_a[4], empty_a[4], full_b[4], empty_b[4], tail_full, stat_full[2], stat_empty[2];
  uint64_t s_full[2], s_free[2], dp_full, p_ready, ds_ready, done;
  uint32_t tmem;
};
static_assert(sizeof(BwdBars) <= BwdLayout<64>::kBarBytes, "room of the barriers");

template <int DP>
struct BwdSmem {
  using L = BwdLayout<DP>;
  uint8_t* base;
  __device__ __forceinline__ uint8_t* fixed(int i) const { return base + i * L::kTileBytes; }
  __device__ __forceinline__ uint8_t* a(int x) const { return base + (2 + x % L::kA) * L::kTileBytes; }
  __device__ __forceinline__ uint8_t* b(int x) const { return base + (2 + L::kA + x % L::kB) * L::kTileBytes; }
  __device__ __forceinline__ float* stats(int x) const {
    return reinterpret_cast<float*>(base + (2 + L::kA + L::kB) * L::kTileBytes + x % L::kStats * L::kStatBytes);
  }
  __device__ __forceinline__ BwdBars& bars() const {
    return *reinterpret_cast<BwdBars*>(base + (2 + L::kA + L::kB) * L::kTileBytes + L::kStats * L::kStatBytes);
  }
};

// The copies of n pairs of tiles; `tail(x)`: rows of pair x that exist.  A's rows that do not are cleared, B's if `clear_b`.
template <int DP, class Tail, class LoadA, class LoadB>
__device__ __forceinline__ bool copy_pairs(const BwdSmem<DP>& m, BwdBars& b, int n, bool clear_b, Tail tail, LoadA load_a, LoadB load_b) {
  using L = BwdLayout<DP>;
  const int lane = threadIdx.x & 31;
  bool ok = true;
  int x = 0, y = 0, tails = 0;
  auto one = [&](uint8_t* dst, uint64_t* full, bool cut, int valid, auto load) {
    uint64_t* bar = cut ? &b.tail_full : full;
    if (lane == 0) {
      ptx::mbar_arrive_expect_tx(bar, L::kTileBytes);
      load(dst, bar);
    }
    __syncwarp();
    if (cut) {
      ok = wait(&b.tail_full, tails++ & 1);
      clear_rows<L::kBoxes>(dst, valid);
      if (lane == 0) ptx::mbar_arrive(full);
    }
  };
  for (; x < n && ok; ++x) {
    const int valid = tail(x);
    ok = wait(&b.empty_a[x % L::kA], (x / L::kA & 1) ^ 1);
    if (!ok) break;
    one(m.a(x), &b.full_a[x % L::kA], valid < kTile, valid, [&](uint8_t* d, uint64_t* bar) { load_a(x, d, bar); });
    ok = ok && wait(&b.empty_b[x % L::kB], (x / L::kB & 1) ^ 1);
    if (!ok) break;
    one(m.b(x), &b.full_b[x % L::kB], clear_b && valid < kTile, valid, [&](uint8_t* d, uint64_t* bar) { load_b(x, d, bar); });
    y = x + 1;
  }
  // no copy is in flight into a block that has ended
  wait(&b.fixed_full, 0);
  for (int i = max(0, x - L::kA); i < x; ++i) wait(&b.full_a[i % L::kA], i / L::kA & 1);
  for (int i = max(0, y - L::kB); i < y; ++i) wait(&b.full_b[i % L::kB], i / L::kB & 1);
  return ok;
}

// 32 scores of a row to their place as FP16.
__device__ __forceinline__ void pack_store(uint32_t taddr, const float2 (&p)[16]) {
  uint32_t h[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) h[i] = rows::pack2(p[i].x, p[i].y);
  tmem_st_32x16(taddr, h);
}
// 32 columns of rows from tensor memory, times f, to the columns of a head from col0 on.
__device__ __forceinline__ void store_rows(uint32_t taddr, float f, uint16_t* out, bool on, int col0, int D) {
  uint32_t v[32];
  ptx::tmem_ld_32x32(taddr, v);
  ptx::tmem_ld_wait();
  if (!on) return;
#pragma unroll
  for (int e = 0; e < 32; e += 8) {
    float x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = __uint_as_float(v[e + k]) * f;
    if (col0 + e < D) *reinterpret_cast<uint4*>(out + col0 + e) = rows::pack8(x);
  }
}
__device__ __forceinline__ float2 pair_of(const uint32_t (&r)[32], int i) {
  return make_float2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1]));
}
// Zeros in place of the columns outside begin .. end - 1.
__device__ __forceinline__ void mask32(float2 (&p)[16], int begin, int end) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if (2 * i < begin || 2 * i >= end) p[i].x = 0.0f;
    if (2 * i + 1 < begin || 2 * i + 1 >= end) p[i].y = 0.0f;
  }
}

template <int DP>
__device__ __forceinline__ bool keys_block(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv,
                                           const CUtensorMap& mdo, const BwdArgs& a, const Place& at, int kv, const BwdSmem<DP>& m) {
  using L = BwdLayout<DP>;
  const Shape& s = a.s;
  BwdBars& b = m.bars();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = s.heads / s.kv_heads;
  const int k0 = (int)at.tile * kTile, len = (int)at.len, row0 = (int)at.start, nq = (len + kTile - 1) / kTile;
  const int i0 = s.causal ? (int)at.tile : 0;     // query tiles that see these keys
  const int64_t reach = k0 + kTile - 1 + (s.window > 0 ? s.window : (int64_t)len);   // first query past all their windows
  const int i1 = s.window > 0 && reach < len ? (int)((reach + kTile - 1) / kTile) : nq;
  const int per = i1 - i0, n = per * group;
  const uint32_t tmem = b.tmem;
  constexpr uint32_t kS = 0, kDP = 128, kSums = 256;         // then dV and dK
  bool ok = true;

  if (warp == kCopies) {
    if (lane == 0) {
      ptx::mbar_arrive_expect_tx(&b.fixed_full, 2 * L::kTileBytes);
      load_tile<L::kBoxes>(m.fixed(0), &mk, &b.fixed_full, kv, row0 + k0);
      load_tile<L::kBoxes>(m.fixed(1), &mv, &b.fixed_full, kv, row0 + k0);
    }
    // queries and gradients of the next sequence would be operands of both sums: cleared
    auto load = [&](const CUtensorMap& map, int x, uint8_t* d, uint64_t* bar) {
      load_tile<L::kBoxes>(d, &map, bar, kv * group + x / per, row0 + (i0 + x % per) * kTile);
    };
    ok = copy_pairs<DP>(m, b, n, true, [&](int x) { return len - (i0 + x % per) * kTile; },
                        [&](int x, uint8_t* d, uint64_t* bar) { load(mq, x, d, bar); },
                        [&](int x, uint8_t* d, uint64_t* bar) { load(mdo, x, d, bar); });
  } else if (warp == kStatistics) {
    const float f = ex2(ds_exponent(a, kv) - kUp);           // P holds 2^kUp of dS's factor
    for (int x = 0; x < n && ok; ++x) {
      const int head = kv * group + x / per, i = i0 + x % per;
      ok = wait(&b.stat_empty[x % L::kStats], (x / L::kStats & 1) ^ 1);
      if (!ok) break;
      float* dst = m.stats(x);
      const int64_t base = (int64_t)head * s.T + row0;
#pragma unroll
      for (int e = 0; e < kTile; e += 32) {
        const int q = i * kTile + e + lane;
        const bool on = q < len;                  // a query that is not there weighs nothing
        dst[e + lane] = on ? fmaf(a.lse[base + q], -kLog2e, kUp) : -INFINITY;
        dst[kTile + e + lane] = on ? -a.delta[base + q] * f : 0.0f;
      }
      arrive(&b.stat_full[x % L::kStats]);
    }
  } else if (warp == kProducts) {
    const int ksteps = (s.D + 15) / 16;
    const uint32_t idesc_s = ptx::idesc_f16_f32(kTile, kTile, false, false);
    const uint32_t idesc_o = ptx::idesc_f16_f32(kTile, ksteps * 16, false, true);
    const uint64_t dk = desc_k(ptx::smem_u32(m.fixed(0))), dv = desc_k(ptx::smem_u32(m.fixed(1)));
    auto scores = [&](int x) {
      product_ss<DP / 16>(tmem + kS, dk, desc_k(ptx::smem_u32(m.a(x))), idesc_s, ksteps);
      ptx::mma_commit(&b.s_full[0]);
    };
    auto dprob = [&](int x) {
      product_ss<DP / 16>(tmem + kDP, dv, desc_k(ptx::smem_u32(m.b(x))), idesc_s, ksteps);
      ptx::mma_commit(&b.dp_full);
    };
    ok = wait(&b.fixed_full, 0) && wait(&b.full_a[0], 0) && wait(&b.full_b[0], 0);
    ptx::tc_fence_after_sync();
    if (ok && ptx::elect_one()) {
      scores(0);
      dprob(0);
    }
    __syncwarp();
    for (int x = 0; x < n && ok; ++x) {
      if (x + 1 < n) ok = wait(&b.full_a[(x + 1) % L::kA], (x + 1) / L::kA & 1);
      ok = ok && wait(&b.p_ready, x & 1);
      if (!ok) break;
      ptx::tc_fence_after_sync();
      if (ptx::elect_one()) {
        product_ts<8, true>(tmem + kSums, tmem + kS, desc_mn(ptx::smem_u32(m.b(x))), idesc_o, 8, x > 0);
        if (x + 1 < n) scores(x + 1);             // in the place of that P
        ptx::mma_commit(&b.empty_b[x % L::kB]);
      }
      __syncwarp();
      if (x + 1 < n) ok = wait(&b.full_b[(x + 1) % L::kB], (x + 1) / L::kB & 1);
      ok = ok && wait(&b.ds_ready, x & 1);
      if (!ok) break;
      ptx::tc_fence_after_sync();
      if (ptx::elect_one()) {
        product_ts<8, true>(tmem + kSums + DP, tmem + kDP, desc_mn(ptx::smem_u32(m.a(x))), idesc_o, 8, x > 0);
        if (x + 1 < n) dprob(x + 1);
        else ptx::mma_commit(&b.done);
        ptx::mma_commit(&b.empty_a[x % L::kA]);
      }
      __syncwarp();
    }
  } else {
    const int quarter = warp >> 2, key = k0 + (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + kS + lanes + quarter * 32, td = tmem + kDP + lanes + quarter * 32;
    const float up = ds_exponent(a, kv), f = ex2(up - kUp);  // P holds 2^kUp of dS's factor
    const float2 c2 = make_float2(s.scale_log2, s.scale_log2), f2 = make_float2(f, f);
    for (int x = 0; x < n && ok; ++x) {
      const int q0 = (i0 + x % per) * kTile;
      ok = wait(&b.stat_full[x % L::kStats], x / L::kStats & 1) && wait(&b.s_full[0], x & 1);
      if (!ok) break;
      ptx::tc_fence_after_sync();
      uint32_t r[32];
      ptx::tmem_ld_32x32(ts, r);
      ptx::tmem_ld_wait();
      const float4* lse = reinterpret_cast<const float4*>(m.stats(x) + quarter * 32);
      const float4* delta = lse + kTile / 4;
      // queries that see this key: q - key in 0 .. window - 1
      const bool edge = s.causal && (q0 < k0 + kTile || (s.window > 0 && q0 + kTile > k0 + s.window));
      const int q = q0 + quarter * 32;
      const int begin = key - q, end = s.window > 0 ? (int)min(key - q + s.window, (int64_t)32) : 32;
      float2 p[16];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float4 l = lse[i];
        const float2 u = fma2(pair_of(r, 2 * i), c2, make_float2(l.x, l.y)), v = fma2(pair_of(r, 2 * i + 1), c2, make_float2(l.z, l.w));
        p[2 * i] = make_float2(ex2(u.x), ex2(u.y));
        p[2 * i + 1] = make_float2(ex2(v.x), ex2(v.y));
      }
      if (edge) mask32(p, begin, end);
      pack_store(ts, p);
      tmem_st_wait();
      ptx::tc_fence_before_sync();
      arrive(&b.p_ready);
      ok = wait(&b.dp_full, x & 1);
      if (!ok) break;
      ptx::tc_fence_after_sync();
      ptx::tmem_ld_32x32(td, r);
      ptx::tmem_ld_wait();
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float4 d = delta[i];
        p[2 * i] = mul2(p[2 * i], fma2(pair_of(r, 2 * i), f2, make_float2(d.x, d.y)));
        p[2 * i + 1] = mul2(p[2 * i + 1], fma2(pair_of(r, 2 * i + 1), f2, make_float2(d.z, d.w)));
      }
      if (edge) mask32(p, begin, end);            // 0 times what is not finite
      pack_store(td, p);
      tmem_st_wait();
      ptx::tc_fence_before_sync();
      arrive(&b.ds_ready);
      arrive(&b.stat_empty[x % L::kStats]);
    }
    if (ok) ok = wait(&b.done, 0);
    if (ok) {
      ptx::tc_fence_after_sync();
      const bool on = key < len;
      const int64_t row = at.start + key, col = (int64_t)kv * s.D;
#pragma unroll
      for (int u = quarter * 32; u < 2 * DP; u += 128) {     // dV's columns, then dK's
        const int col0 = u < DP ? u : u - DP;
        if (col0 >= s.D) continue;                // warp-uniform
        if (u < DP) store_rows(tmem + kSums + lanes + u, ex2(-kUp), a.dv + row * a.lddv + col, on, col0, s.D);
        else store_rows(tmem + kSums + lanes + u, s.scale * ex2(-up), a.dk + row * a.lddk + col, on, col0, s.D);
      }
    }
  }
  return ok;
}

template <int DP>
__device__ __forceinline__ bool queries_block(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv,
                                              const CUtensorMap& mdo, const BwdArgs& a, const Place& at, int head, const BwdSmem<DP>& m) {
  using L = BwdLayout<DP>;
  const Shape& s = a.s;
  BwdBars& b = m.bars();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, kv = head / (s.heads / s.kv_heads);
  const int tile = (int)(at.tiles - 1 - at.tile), q0 = tile * kTile, len = (int)at.len, row0 = (int)at.start;
  const int last = min(q0 + kTile, len);
  const int j0 = s.window > 0 && q0 + 1 > s.window ? (int)(q0 + 1 - s.window) / kTile : 0;
  const int j1 = ((s.causal ? last : len) + kTile - 1) / kTile, n = j1 - j0;
  const uint32_t tmem = b.tmem;
  constexpr uint32_t kS = 0, kDP = 256, kDQ = 384;           // two places for S
  bool ok = true;

  if (warp == kCopies) {
    if (lane == 0) {
      ptx::mbar_arrive_expect_tx(&b.fixed_full, 2 * L::kTileBytes);
      load_tile<L::kBoxes>(m.fixed(0), &mq, &b.fixed_full, head, row0 + q0);
      load_tile<L::kBoxes>(m.fixed(1), &mdo, &b.fixed_full, head, row0 + q0);
    }
    ok = copy_pairs<DP>(m, b, n, false, [&](int x) { return len - (j0 + x) * kTile; },
                        [&](int x, uint8_t* d, uint64_t* bar) { load_tile<L::kBoxes>(d, &mk, bar, kv, row0 + (j0 + x) * kTile); },
                        [&](int x, uint8_t* d, uint64_t* bar) { load_tile<L::kBoxes>(d, &mv, bar, kv, row0 + (j0 + x) * kTile); });
  } else if (warp == kProducts) {
    const int ksteps = (s.D + 15) / 16;
    const uint32_t idesc_s = ptx::idesc_f16_f32(kTile, kTile, false, false);
    const uint32_t idesc_o = ptx::idesc_f16_f32(kTile, ksteps * 16, false, true);
    const uint64_t dq = desc_k(ptx::smem_u32(m.fixed(0))), ddo = desc_k(ptx::smem_u32(m.fixed(1)));
    auto scores = [&](int x) {
      product_ss<DP / 16>(tmem + kS + (x & 1) * kTile, dq, desc_k(ptx::smem_u32(m.a(x))), idesc_s, ksteps);
      ptx::mma_commit(&b.s_full[x & 1]);
    };
    auto dprob = [&](int x) {
      product_ss<DP / 16>(tmem + kDP, ddo, desc_k(ptx::smem_u32(m.b(x))), idesc_s, ksteps);
      ptx::mma_commit(&b.dp_full);
      ptx::mma_commit(&b.empty_b[x % L::kB]);
    };
    ok = wait(&b.fixed_full, 0) && wait(&b.full_a[0], 0) && wait(&b.full_b[0], 0);
    ptx::tc_fence_after_sync();
    if (ok && ptx::elect_one()) {
      scores(0);
      dprob(0);
    }
    __syncwarp();
    for (int x = 0; x < n && ok; ++x) {
      if (x + 1 < n) {                            // the next tile's scores while this one's are worked on
        ok = wait(&b.full_a[(x + 1) % L::kA], (x + 1) / L::kA & 1) && wait(&b.s_free[(x + 1) & 1], ((x + 1) / 2 & 1) ^ 1);
        if (!ok) break;
        ptx::tc_fence_after_sync();
        if (ptx::elect_one()) scores(x + 1);
        __syncwarp();
        ok = wait(&b.full_b[(x + 1) % L::kB], (x + 1) / L::kB & 1);
      }
      ok = ok && wait(&b.ds_ready, x & 1);
      if (!ok) break;
      ptx::tc_fence_after_sync();
      if (ptx::elect_one()) {
        product_ts<8, true>(tmem + kDQ, tmem + kDP, desc_mn(ptx::smem_u32(m.a(x))), idesc_o, 8, x > 0);
        if (x + 1 < n) dprob(x + 1);
        else ptx::mma_commit(&b.done);
        ptx::mma_commit(&b.empty_a[x % L::kA]);
      }
      __syncwarp();
    }
  } else if (warp < kCompute) {
    const int quarter = warp >> 2, row = q0 + (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t td = tmem + kDP + lanes + quarter * 32;
    const float up = ds_exponent(a, kv), f = ex2(up - kUp);  // P holds 2^kUp of dS's factor
    const int64_t at_row = (int64_t)head * s.T + at.start + row;
    const bool on = row < len;
    const float lse = on ? fmaf(a.lse[at_row], -kLog2e, kUp) : 0.0f, delta = on ? -a.delta[at_row] * f : 0.0f;
    const float2 c2 = make_float2(s.scale_log2, s.scale_log2), lse2 = make_float2(lse, lse);
    const float2 f2 = make_float2(f, f), delta2 = make_float2(delta, delta);
    const int key1 = s.causal ? min(row + 1, len) : len;     // keys that this query sees
    const int key0 = s.window > 0 && row + 1 > s.window ? (int)(row + 1 - s.window) : 0;
    const int whole1 = s.causal ? min(q0 + 1, len) : len;
    const int whole0 = s.window > 0 && q0 + kTile > s.window ? (int)(q0 + kTile - s.window) : 0;
    for (int x = 0; x < n && ok; ++x) {
      ok = wait(&b.s_full[x & 1], x / 2 & 1);
      if (!ok) break;
      ptx::tc_fence_after_sync();
      uint32_t r[32];
      ptx::tmem_ld_32x32(tmem + kS + (x & 1) * kTile + lanes + quarter * 32, r);
      ptx::tmem_ld_wait();
      ptx::tc_fence_before_sync();
      arrive(&b.s_free[x & 1]);
      const int k0 = (j0 + x) * kTile;
      const bool edge = k0 + kTile > whole1 || k0 < whole0;
      float2 p[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float2 u = fma2(pair_of(r, i), c2, lse2);
        p[i] = make_float2(ex2(u.x), ex2(u.y));
      }
      ok = wait(&b.dp_full, x & 1);
      if (!ok) break;
      ptx::tc_fence_after_sync();
      ptx::tmem_ld_32x32(td, r);
      ptx::tmem_ld_wait();
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = mul2(p[i], fma2(pair_of(r, i), f2, delta2));
      if (edge) mask32(p, key0 - k0 - quarter * 32, key1 - k0 - quarter * 32);
      pack_store(td, p);
      tmem_st_wait();
      ptx::tc_fence_before_sync();
      arrive(&b.ds_ready);
    }
    if (ok) ok = wait(&b.done, 0);
    if (ok) {
      ptx::tc_fence_after_sync();
      const int col0 = quarter * 32;
      if (col0 < DP && col0 < s.D)
        store_rows(tmem + kDQ + lanes + col0, s.scale * ex2(-up), a.dq + (at.start + row) * a.lddq + (int64_t)head * s.D, on, col0, s.D);
    }
  }
  return ok;
}

template <int DP>
__global__ void __launch_bounds__(kBwdThreads, 1)
mp_attention_bwd_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                        const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdo, const BwdArgs a) {
  using L = BwdLayout<DP>;
  extern __shared__ __align__(1024) uint8_t smem[];          // (nothing else is in shared memory: it begins at a multiple of 1024)
  const BwdSmem<DP> m{smem};
  BwdBars& b = m.bars();
  const Shape& s = a.s;
  const int warp = threadIdx.x >> 5;
  ptx::grid_dependency_wait();
  const bool keys = (int)blockIdx.x < a.key_blocks;
  const int item = keys ? blockIdx.x : blockIdx.x - a.key_blocks, heads = keys ? s.kv_heads : s.heads;
  const Place at = place_of<kTile>(s, item / heads);
  if (blockIdx.x == 0 && warp == 0) check_offsets(s);
  if (at.tile >= at.tiles) return;
  if (threadIdx.x == 0) {
    ptx::mbar_init(&b.fixed_full, 1);
    ptx::mbar_init(&b.tail_full, 1);
    for (int i = 0; i < 4; ++i) {
      ptx::mbar_init(&b.full_a[i], 1);
      ptx::mbar_init(&b.empty_a[i], 1);
      ptx::mbar_init(&b.full_b[i], 1);
      ptx::mbar_init(&b.empty_b[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(&b.stat_full[i], 1);
      ptx::mbar_init(&b.stat_empty[i], kCompute);            // warps, as below
      ptx::mbar_init(&b.s_full[i], 1);
      ptx::mbar_init(&b.s_free[i], kCompute);
    }
    ptx::mbar_init(&b.dp_full, 1);
    ptx::mbar_init(&b.p_ready, kCompute);
    ptx::mbar_init(&b.ds_ready, kCompute);
    ptx::mbar_init(&b.done, 1);
    ptx::fence_mbar_init();
  }
  if (warp == kProducts) {
    ptx::tmem_alloc(&b.tmem, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  ptx::launch_dependents();                       // every block has its tensor memory, as in the forward pass
  const bool ok = keys ? keys_block<DP>(mq, mk, mv, mdo, a, at, item % heads, m)
                       : queries_block<DP>(mq, mk, mv, mdo, a, at, item % heads, m);
  if (!ok && (threadIdx.x & 31) == 0) report_timeout(s);
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (warp == kProducts) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(b.tmem, 512);
  }
}

void early(cudaLaunchConfig_t& cfg, cudaLaunchAttribute& attr) {      // may start under the kernel ahead, and waits for it
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
}

template <int L>
int prep_launch(const BwdArgs& a, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.slots, (unsigned)(a.s.heads + a.s.kv_heads), 1);
  cfg.blockDim = dim3(kPrepThreads, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute attr;
  early(cfg, attr);
  MP_CUDA_TRY(cudaLaunchKernelEx(&cfg, mp_attention_prep_kernel<L>, a));
  mp::count_launch();
  return MP_OK;
}

template <int DP>
int bwd_launch(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const CUtensorMap& mdo, const BwdArgs& a,
               int64_t blocks, cudaStream_t st) {
  static mp::PerDevice ready;
  int dev = 0;
  MP_CUDA_TRY(cudaGetDevice(&dev));
  auto kernel = mp_attention_bwd_kernel<DP>;
  if (!ready.get(dev)) {
    MP_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, BwdLayout<DP>::kSmem));
    ready.set(dev, 1);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks, 1, 1);
  cfg.blockDim = dim3(kBwdThreads, 1, 1);
  cfg.dynamicSmemBytes = BwdLayout<DP>::kSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr;
  early(cfg, attr);
  MP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, mq, mk, mv, mdo, a));
  mp::count_launch();
  return MP_OK;
}

}  // namespace

extern "C" {

size_t mp_attention_bwd_workspace_bytes(int64_t T, int64_t heads, int64_t kv_heads, int64_t D) {
  if (T < 0 || heads <= 0 || kv_heads <= 0 || heads % kv_heads || D <= 0 || D % 8 || D > MP_ATTENTION_MAX_D ||
      heads > 32767 || T > MP_ATTENTION_MAX_ROWS)
    return 0;
  return (size_t)(heads * T + (heads + kv_heads) * kSlots) * sizeof(float);
}

int mp_attention_bwd(const void* do16, int64_t lddo, const void* q16, int64_t ldq, const void* k16, int64_t ldk,
                     const void* v16, int64_t ldv, const void* o16, int64_t ldo, const float* lse, void* dq16, int64_t lddq,
                     void* dk16, int64_t lddk, void* dv16, int64_t lddv, const void* offsets, int id_bytes, int64_t n_seq,
                     int64_t T, int64_t heads, int64_t kv_heads, int64_t D, float scale, int causal, int64_t window,
                     mp_state* state, void* workspace, size_t workspace_bytes, void* stream) {
  const char* name = "mp_attention_bwd";
  BwdArgs a;
  if (int rc = check_call(name, a.s, offsets, id_bytes, n_seq, T, heads, kv_heads, D, scale, causal, window, state)) return rc;
  const struct { const void* p; int64_t ld, heads; } all[] = {
      {do16, lddo, heads}, {q16, ldq, heads}, {k16, ldk, kv_heads}, {v16, ldv, kv_heads},
      {o16, ldo, heads}, {dq16, lddq, heads}, {dk16, lddk, kv_heads}, {dv16, lddv, kv_heads}};
  for (const auto& m : all)
    if (int rc = check_matrix(name, m.p, m.ld, m.heads, D)) return rc;
  if ((uintptr_t)lse & 3) return mp::set_error(MP_ERR_ALIGNMENT, "%s: FP32 values must be aligned", name);
  if (T > 0 && n_seq > 0) {
    for (const auto& m : all)
      if (!m.p) return mp::set_error(MP_ERR_INVALID_ARG, "%s: null pointer", name);
    if (!lse) return mp::set_error(MP_ERR_INVALID_ARG, "%s: null pointer", name);
  }
  if (!mp::aligned16(workspace)) return mp::set_error(MP_ERR_ALIGNMENT, "%s: pointers must be 16-byte aligned", name);
  const size_t need = mp_attention_bwd_workspace_bytes(T, heads, kv_heads, D);
  if (need > 0 && T > 0 && n_seq > 0 && (!workspace || workspace_bytes < need))
    return mp::set_error(MP_ERR_NOMEM, "%s: workspace of %zu bytes needed, %zu given", name, need,
                         workspace ? workspace_bytes : (size_t)0);
  if (T > 0 && n_seq > 0)
    for (int i = 0; i < 8; ++i)                   // five inputs, three results
      for (int j = i < 5 ? 5 : i + 1; j < 8; ++j)
        if (all[i].p == all[j].p)
          return mp::set_error(MP_ERR_INVALID_ARG, "%s: a result may be neither an input nor another result", name);
  if (int rc = mp::check_device()) return rc;
  if (T == 0 || n_seq == 0) return MP_OK;
  if (int rc = mp::gemm_status_device_ptr(&a.s.status)) return rc;
  a.o = (const uint16_t*)o16;
  a.dout = (const uint16_t*)do16;
  a.v = (const uint16_t*)v16;
  a.ldo = ldo;
  a.lddo = lddo;
  a.ldv = ldv;
  a.lse = lse;
  a.dq = (uint16_t*)dq16;
  a.dk = (uint16_t*)dk16;
  a.dv = (uint16_t*)dv16;
  a.lddq = lddq;
  a.lddk = lddk;
  a.lddv = lddv;
  a.delta = (float*)workspace;
  a.norms = a.delta + heads * T;
  const int lanes = D <= 32 ? 4 : D <= 64 ? 8 : 16;
  const int64_t groups = (T * lanes + kPrepThreads - 1) / kPrepThreads;
  a.slots = groups < kSlots ? (int)groups : kSlots;
  CUtensorMap mq, mk, mv, mdo;
  if (int rc = make_map(&mq, Operand{q16, ldq, (int)heads}, T, (int)D)) return rc;
  if (int rc = make_map(&mk, Operand{k16, ldk, (int)kv_heads}, T, (int)D)) return rc;
  if (int rc = make_map(&mv, Operand{v16, ldv, (int)kv_heads}, T, (int)D)) return rc;
  if (int rc = make_map(&mdo, Operand{do16, lddo, (int)heads}, T, (int)D)) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  if (int rc = lanes == 4 ? prep_launch<4>(a, st) : lanes == 8 ? prep_launch<8>(a, st) : prep_launch<16>(a, st)) return rc;
  const int64_t tiles = T / kTile + n_seq;
  a.key_blocks = (int)(tiles * kv_heads);
  const int64_t blocks = tiles * (heads + kv_heads);
  return D <= 64 ? bwd_launch<64>(mq, mk, mv, mdo, a, blocks, st) : bwd_launch<128>(mq, mk, mv, mdo, a, blocks, st);
}

}  // extern "C"

// Attention over packed sequences, forward: O = softmax(scale Q K^T) V for each head, with the rows' log-sums.
//
// One pass over the keys with a running maximum and sum.  A tile of 128 queries meets 64 keys at a time: S = Q K^T in
// tensor memory, the exponentials, O += P V with P in the place of its S as FP16 (rounded once; the sum is taken from the
// unrounded FP32 values).  There are two places for S, so the tensor core forms the next
// scores while these go through the exponential.  Keys and values pass through a ring in shared memory.
// P = 2^(score - ref), with ref 7 below a maximum of the row that may lag: it is raised, and O multiplied, only where a score has passed
// that maximum by 8, so that almost no step pays for it.  So P stays below 2^15 and fits FP16, and a weight down to 2^-21 of its row's
// largest is rounded to half a step, 2^-11 of it; smaller ones are off by at most 2^-32 of the largest.  (With ref the maximum itself
// thousands of keys 18 nats below one other weighed nothing, while the sum counted them.)
// Scores of 2^22 and more (in powers of two), which FP32 holds in steps that count here, are rounded before ref is taken from them: the
// fused operation keeps what ref has lost in rounding, and P could pass FP16's range.  They have a copy of the steps apart (64 x 400:
// 236.7 us; a branch in the steps took 242).
//
// What bounds it.  For a head of 128 elements the special-function unit (16 results a clock and SM) and the products take as long,
// 16384 x 32 heads causal 1.0 and 1.3 ms; a step also waits for its scores and its P to change hands, 150 .. 200 clocks each
// time, which the other tile's work covers in part: 2.0 .. 2.1 ms (1060 TFLOP/s), 2.4 when the card runs it for seconds
// and meets its power limit.  Both units are busy just under half the time.  Sequences of 400 (64 of them, 25 heads of 64): a
// block has seven steps of 64 keys, and of its 20000 clocks 9000 go to finding its place, the first copies and the last stores.
// Taken back: one place for S and more blocks an SM (444 us against 263 there); 128 keys a step and two threads a row
// (273 against 248, though 16384 x 32 heads of 128 took 1.98 ms against 2.07); 32 keys a step and three blocks an SM (242
// against 265, but sequences of 16384 1080 against 963: a rule on the batch's lengths would make a row's bits depend on
// what else is in the batch, and they do not); part of the exponentials as polynomials (2.25 ms); one lane polling a
// barrier for its warp (1.51 ms against 1.30); the first copies issued ahead of the block's barrier (259 us against 255).

#include <math.h>

#include <atomic>

#include <cudaTypedefs.h>

#include "attention.cuh"

namespace {

using namespace attn;

struct FwdArgs {
  Shape s;
  uint16_t* o;
  int64_t ldo;
  float* lse;
};

// Heads of more than 64 elements: two tiles of queries a block share the keys and values, which would else ask L2 for 64 bytes a
// clock and SM.  Below that one tile a block and two blocks an SM, whose beginnings and ends cover one another.
template <int DP>
struct FwdLayout {
  static constexpr int kTiles = DP == 64 ? 1 : 2, kBlocks = DP == 64 ? 2 : 1;      // tiles a block, blocks an SM
  // Four warps a tile, a row a thread; then one a tile that issues its products (with one for both, the tensor core waited while
  // that warp waited for the other tile, four tenths of the time); then one for the copies.
  static constexpr int kThreads = kTiles * 160 + 32;
  static constexpr int kBoxes = DP / 64, kTileBytes = kBoxes * kBoxBytes;
  static constexpr int kStages = DP == 64 ? 5 : 4;
  static constexpr int kSmem = (kTiles + kStages) * kTileBytes + 1024;
  static constexpr int kColumns = DP == 64 ? 256 : 512;      // of tensor memory: S, with P in its place, then O, for each tile
};
constexpr int kStep = 64;                         // keys that a tile meets at once
constexpr float kLag = 8.0f, kUp = 7.0f, kLarge = 4194304.0f;         // in powers of two: see above

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// The rows of a warp, one a thread: what they see, their tile's barriers, and how far they have come.
struct Rows {
  uint32_t ts, to_o;                              // S and O
  int lo, hi;                                     // steps
  int key0, key1, whole0, whole1, end;            // keys: of the thread's query, and of the warp's
  float c;
  uint64_t *s_full, *p_ready, *o_done;
  float ref, sum;
  bool on, ok;                                    // the query exists; no wait has run out
};
// From step u on; returns the first step that is left, where the usual kind has met large scores before anything was made of them.
template <int DP, bool kAnySize>
__device__ __forceinline__ int row_steps(Rows& w, int u) {
  const float c = w.c;
  for (; u < w.hi && w.ok; ++u) {
    const int n = u - w.lo, k0 = u * kStep;
    const uint32_t at_s = w.ts + (n & 1) * kStep;
    w.ok = wait(&w.s_full[n & 1], n >> 1 & 1);
    if (!w.ok) break;
    ptx::tc_fence_after_sync();
    // pieces of 32 columns with keys that are seen
    const int pieces = max(0, min(2, (w.end - k0 + 31) / 32));
    uint32_t r[2][32];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (i < pieces) ptx::tmem_ld_32x32(at_s + i * 32, r[i]);
    ptx::tmem_ld_wait();
    if (k0 + kStep > w.whole1 || k0 < w.whole0) {
      const int stop = w.key1 - k0, begin = w.key0 - k0;
#pragma unroll
      for (int e = 0; e < kStep; ++e)
        if (e >= stop || e < begin) r[e / 32][e % 32] = 0xFF800000u;
    }
    float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (i < pieces)
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
          top[2 * i] = max3(top[2 * i], __uint_as_float(r[i][e]), __uint_as_float(r[i][e + 1]));
          top[2 * i + 1] = max3(top[2 * i + 1], __uint_as_float(r[i][e + 2]), __uint_as_float(r[i][e + 3]));
        }
    const float most = max3(fmaxf(top[0], top[1]), top[2], top[3]);
    // from -inf on: at the first step with a key that is seen
    const bool raise = (kAnySize ? __fmul_rn(most, c) - w.ref : fmaf(most, c, -w.ref)) > kUp + kLag;
    if (__any_sync(0xFFFFFFFFu, raise)) {
      const float next = raise ? (kAnySize ? __fmul_rn(most, c) - kUp : fmaf(most, c, -kUp)) : w.ref, f = raise ? ex2(w.ref - next) : 1.0f;
      if (!kAnySize && __any_sync(0xFFFFFFFFu, fabsf(next) >= kLarge && next > -INFINITY && w.on)) break;
      w.ref = next;
      w.sum *= f;
      if (n > 0) {                                // the products so far have this maximum's factor
        w.ok = wait(&w.o_done[(n - 1) & 1], n - 1 >> 1 & 1);
        ptx::tc_fence_after_sync();
#pragma unroll 1
        for (int i = 0; i < DP; i += 32) {
          uint32_t v[32];
          ptx::tmem_ld_32x32(w.to_o + i, v);
          ptx::tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * f);
          tmem_st_32x32(w.to_o + i, v);
        }
      }
    }
    const float shift = w.ref == -INFINITY ? 0.0f : -w.ref;
    const float2 c2 = make_float2(c, c), shift2 = make_float2(shift, shift);
    float2 part[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t p[16];
      if (i < pieces) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float2 z = make_float2(__uint_as_float(r[i][2 * e]), __uint_as_float(r[i][2 * e + 1]));
          // (packed, the product and the sum would be fused)
          const float2 x = kAnySize ? make_float2(__fadd_rn(__fmul_rn(z.x, c), shift), __fadd_rn(__fmul_rn(z.y, c), shift)) : fma2(z, c2, shift2);
          const float2 y = make_float2(ex2(x.x), ex2(x.y));
          part[e & 1] = add2(part[e & 1], y);
          p[e] = rows::pack2(y.x, y.y);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) p[e] = 0;
      }
      tmem_st_32x16(at_s + i * 16, p);
    }
    tmem_st_wait();
    ptx::tc_fence_before_sync();
    arrive(&w.p_ready[n & 1]);
    w.sum += (part[0].x + part[0].y) + (part[1].x + part[1].y);
  }
  return u;
}
template <int DP>
__device__ __noinline__ Rows large_row_steps(Rows w, int u) {
  row_steps<DP, true>(w, u);
  return w;
}
template <int DP>
__global__ void __launch_bounds__(FwdLayout<DP>::kThreads, FwdLayout<DP>::kBlocks)
mp_attention_fwd_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                        const __grid_constant__ CUtensorMap mv, const FwdArgs a) {
  using L = FwdLayout<DP>;
  constexpr int kTiles = L::kTiles, kProducts = kTiles * 4, kCopies = kProducts + kTiles;     // these warps' numbers
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* ring = smem + kTiles * L::kTileBytes;
  // of each place for S apart: a waiter is then never two phases from a barrier
  __shared__ uint64_t q_full, kv_full[L::kStages], kv_empty[L::kStages], tail_full, s_full[kTiles][2], p_ready[kTiles][2], o_done[kTiles][2];
  __shared__ uint32_t s_tmem;
  const Shape& s = a.s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  ptx::grid_dependency_wait();
  const int head = blockIdx.x % s.heads;
  const Place at = place_of<kTiles * kTile>(s, blockIdx.x / s.heads);
  if (blockIdx.x == 0 && warp == 0) check_offsets(s);
  if (at.tile >= at.tiles) return;
  if (threadIdx.x == 0) {
    ptx::mbar_init(&q_full, 1);
    ptx::mbar_init(&tail_full, 1);
    for (int i = 0; i < L::kStages; ++i) {
      ptx::mbar_init(&kv_full[i], 1);
      ptx::mbar_init(&kv_empty[i], kTiles);
    }
    for (int t = 0; t < kTiles; ++t) {
      for (int i = 0; i < 2; ++i) {
        ptx::mbar_init(&s_full[t][i], 1);
        ptx::mbar_init(&p_ready[t][i], 4);            // warps
        ptx::mbar_init(&o_done[t][i], 1);
      }
    }
    ptx::fence_mbar_init();
  }
  if (warp == kProducts) {
    ptx::tmem_alloc(&s_tmem, L::kColumns);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  // Only now may the next kernel's blocks come: one that takes tensor memory and then waits for this grid must not find an SM where
  // a block of this grid has still to take its own.
  ptx::launch_dependents();
  const uint32_t tmem = s_tmem;
  constexpr uint32_t kO = kTiles * kTile;
  // the long ones first: a causal query sees all keys before it
  const int q0 = (int)(at.tiles - 1 - at.tile) * kTiles * kTile, len = (int)at.len;
  // the steps of kStep keys that a tile of queries sees
  int u0[kTiles], u1[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int first = q0 + t * kTile, last = min(first + kTile, len);     // queries
    u0[t] = s.window > 0 && first + 1 > s.window ? (int)(first + 1 - s.window) / kStep : 0;
    u1[t] = first >= len ? u0[t] : ((s.causal ? last : len) + kStep - 1) / kStep;
  }
  const int from = u0[0], to = max(u1[0], u1[kTiles - 1]), j0 = from / 2, j1 = (to + 1) / 2;      // steps, and blocks of 128 keys
  bool ok = true;

  if (warp == kCopies) {
    const int kv = head / (s.heads / s.kv_heads), row0 = (int)at.start;
    const int tiles = kTiles == 2 && q0 + kTile < len ? 2 : 1;
    if (lane == 0) {
      ptx::mbar_arrive_expect_tx(&q_full, tiles * L::kTileBytes);
      for (int t = 0; t < tiles; ++t)
        load_tile<L::kBoxes>(smem + t * L::kTileBytes, &mq, &q_full, head, row0 + q0 + t * kTile);
    }
    int n = 0;
    for (int j = j0; j < j1 && ok; ++j) {
      const int valid = len - j * kTile;
      for (int v = 0; v < 2 && ok; ++v, ++n) {
        const int stage = n % L::kStages;
        if (!wait(&kv_empty[stage], (n / L::kStages & 1) ^ 1)) { ok = false; break; }
        uint8_t* dst = ring + stage * L::kTileBytes;
        const bool tail = v == 1 && valid < kTile;
        uint64_t* bar = tail ? &tail_full : &kv_full[stage];
        if (lane == 0) {
          ptx::mbar_arrive_expect_tx(bar, L::kTileBytes);
          load_tile<L::kBoxes>(dst, v ? &mv : &mk, bar, kv, row0 + j * kTile);
        }
        __syncwarp();
        if (tail) {                               // the last block alone
          ok = wait(&tail_full, 0);
          clear_rows<L::kBoxes>(dst, valid);
          if (lane == 0) ptx::mbar_arrive(&kv_full[stage]);
        }
      }
    }
    // no copy is in flight into a block that has ended
    wait(&q_full, 0);
    for (int i = max(0, n - L::kStages); i < n; ++i) wait(&kv_full[i % L::kStages], i / L::kStages & 1);
  } else if (warp >= kProducts) {
    const int t = warp - kProducts, lo = t ? u0[kTiles - 1] : u0[0], hi = t ? u1[kTiles - 1] : u1[0];
    const int ksteps = (s.D + 15) / 16;
    const uint32_t idesc_o = ptx::idesc_f16_f32(kTile, ksteps * 16, false, true);
    const uint32_t d_s = tmem + t * kTile, d_o = tmem + kO + t * DP;
    const uint64_t dq = desc_k(ptx::smem_u32(smem + t * L::kTileBytes));
    ok = wait(&q_full, 0);
    // Step u: O += P V of step u - 2, and S of step u in the place of that P.  A block of keys or values has two steps; the warp
    // lets go of those that only the other tile sees as well.
    for (int u = from; u < to + 2 && ok; ++u) {
      const int nk = 2 * ((u >> 1) - j0), nv = 2 * ((u - 2 >> 1) - j0) + 1;      // places in the order of copies
      const bool scores = u < to, values = u - 2 >= from;
      if (scores && (u == from || !(u & 1))) ok = wait(&kv_full[nk % L::kStages], nk / L::kStages & 1);
      if (ok && values && (u - 2 == from || !(u & 1))) ok = wait(&kv_full[nv % L::kStages], nv / L::kStages & 1);
      const int v = u - 2 - lo, place = (u - lo) & 1;
      if (ok && v >= 0 && u - 2 < hi) {
        ok = wait(&p_ready[t][place], v >> 1 & 1);
        ptx::tc_fence_after_sync();
        if (ok && ptx::elect_one()) {
          // the last step of a sequence is as wide as it has keys
          const int steps = (min(kStep, len - (u - 2) * kStep) + 15) / 16;
          const uint64_t dv = desc_mn(ptx::smem_u32(ring + nv % L::kStages * L::kTileBytes) + (u & 1) * kStep * 128);
          product_ts<kStep / 16, false>(d_o, d_s + place * kStep, dv, idesc_o, steps, v > 0);
          ptx::mma_commit(&o_done[t][place]);
        }
        __syncwarp();
      }
      if (ok && u >= lo && u < hi) {
        ptx::tc_fence_after_sync();
        if (ptx::elect_one()) {
          const int wide = (min(kStep, len - u * kStep) + 15) / 16 * 16;
          const uint64_t dk = desc_k(ptx::smem_u32(ring + nk % L::kStages * L::kTileBytes) + (u & 1) * kStep * 128);
          product_ss<DP / 16>(d_s + place * kStep, dq, dk, ptx::idesc_f16_f32(kTile, wide, false, false), ksteps);
          ptx::mma_commit(&s_full[t][place]);
        }
        __syncwarp();
      }
      if (ok && ptx::elect_one()) {
        if (values && ((u & 1) || u - 1 == to)) ptx::mma_commit(&kv_empty[nv % L::kStages]);
        if (scores && ((u & 1) || u + 1 == to)) ptx::mma_commit(&kv_empty[nk % L::kStages]);
      }
      __syncwarp();
    }
  } else {
    const int t = warp >> 2, row = q0 + t * kTile + (warp & 3) * 32 + lane;      // of the sequence
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + t * kTile + lanes, to_o = tmem + kO + t * DP + lanes;
    const int lo = t ? u0[kTiles - 1] : u0[0], hi = t ? u1[kTiles - 1] : u1[0];
    const bool some = row - lane < len;           // the warp has rows that exist
    // the keys that this query sees
    const int key1 = s.causal ? min(row + 1, len) : len;
    const int key0 = s.window > 0 && row + 1 > s.window ? (int)(row + 1 - s.window) : 0;
    // steps between these two are seen whole by every query of the warp; no query of it sees a key from `end` on
    const int first = row - lane;
    const int whole1 = s.causal ? min(first + 1, len) : len, end = s.causal ? min(first + 32, len) : len;
    const int whole0 = s.window > 0 && first + 32 > s.window ? (int)(first + 32 - s.window) : 0;
    Rows w{ts, to_o, lo, hi, key0, key1, whole0, whole1, end, s.scale_log2, s_full[t], p_ready[t], o_done[t], -INFINITY, 0.0f, row < len, true};
    if (some) {
      const int left = row_steps<DP, false>(w, lo);
      if (left < hi && w.ok) w = large_row_steps<DP>(w, left);
      ok = w.ok;
    } else {                                      // rows of what comes behind the sequence: whatever P holds stays in them
      for (int n = 0; n < hi - lo && ok; ++n) {
        ok = wait(&s_full[t][n & 1], n >> 1 & 1);
        if (ok) arrive(&p_ready[t][n & 1]);
      }
    }
    const float ref = w.ref, sum = w.sum;
    if (ok && some && hi > lo) {
      ok = wait(&o_done[t][(hi - 1 - lo) & 1], hi - 1 - lo >> 1 & 1);
      ptx::tc_fence_after_sync();
      const float inv = 1.0f / sum;
      uint16_t* o = a.o + (at.start + row) * a.ldo + (int64_t)head * s.D;
#pragma unroll 1
      for (int i = 0; i < s.D; i += 32) {
        uint32_t v[32];
        ptx::tmem_ld_32x32(to_o + i, v);
        ptx::tmem_ld_wait();
        if (ok && row < len) {
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
            float f[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) f[x] = __uint_as_float(v[e + x]) * inv;
            if (i + e < s.D) *reinterpret_cast<uint4*>(o + i + e) = rows::pack8(f);
          }
        }
      }
      if (ok && row < len) a.lse[(int64_t)head * s.T + at.start + row] = (ref + log2f(sum)) * kLn2;
    }
  }
  if (!ok && lane == 0) report_timeout(s);
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (warp == kProducts) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, L::kColumns);
  }
}

template <int DP>
int fwd_launch(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const FwdArgs& a, int64_t blocks,
               cudaStream_t st) {
  static mp::PerDevice ready;
  int dev = 0;
  MP_CUDA_TRY(cudaGetDevice(&dev));
  auto kernel = mp_attention_fwd_kernel<DP>;
  if (!ready.get(dev)) {
    MP_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, FwdLayout<DP>::kSmem));
    ready.set(dev, 1);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks, 1, 1);
  cfg.blockDim = dim3(FwdLayout<DP>::kThreads, 1, 1);
  cfg.dynamicSmemBytes = FwdLayout<DP>::kSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  MP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, mq, mk, mv, a));
  mp::count_launch();
  return MP_OK;
}

}  // namespace

namespace attn {

int make_map(CUtensorMap* map, const Operand& x, int64_t T, int D) {
  static std::atomic<PFN_cuTensorMapEncodeTiled_v12000> encode{nullptr};
  PFN_cuTensorMapEncodeTiled_v12000 fn = encode.load(std::memory_order_acquire);
  if (fn == nullptr) {                            // threads that both find it empty both ask
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    MP_CUDA_TRY(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found));
    if (found != cudaDriverEntryPointSuccess || !p)
      return mp::set_error(MP_ERR_CUDA, "cuTensorMapEncodeTiled is not available from this driver");
    fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
    encode.store(fn, std::memory_order_release);
  }
  const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)x.heads, (cuuint64_t)T};
  const cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)x.ld * 2};
  const cuuint32_t box[3] = {64, 1, kTile}, estr[3] = {1, 1, 1};
  const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(x.ptr), dims, strides, box, estr,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return mp::set_error(MP_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d", (int)r);
  return MP_OK;
}

int check_call(const char* name, Shape& s, const void* offsets, int id_bytes, int64_t n_seq, int64_t T, int64_t heads,
               int64_t kv_heads, int64_t D, float scale, int causal, int64_t window, mp_state* state) {
  if (n_seq < 0 || T < 0 || heads <= 0 || kv_heads <= 0 || heads % kv_heads || D <= 0 || D % 8 ||
      (id_bytes != 4 && id_bytes != 8))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: bad size, heads that the key heads do not divide, a head size that is "
                         "not a multiple of 8, or a bad width of the offsets", name);
  if (!(scale > 0.0f) || !isfinite(scale) || (causal != 0 && causal != 1) || window < 0 || (window > 0 && !causal))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: the scale must be positive and finite, causal 0 or 1, and a window "
                         "needs causal", name);
  if (D > MP_ATTENTION_MAX_D || heads > 32767 || T > MP_ATTENTION_MAX_ROWS || n_seq > MP_ATTENTION_MAX_ROWS ||
      (T / kTile + n_seq) * heads > 0x3FFFFFFF)
    return mp::set_error(MP_ERR_TOO_LARGE, "%s: a head of more than %d elements, more than %d rows, or too many tiles",
                         name, MP_ATTENTION_MAX_D, MP_ATTENTION_MAX_ROWS);
  if (T > 0 && n_seq > 0 && !offsets) return mp::set_error(MP_ERR_INVALID_ARG, "%s: null pointer", name);
  if ((uintptr_t)offsets & (uintptr_t)(id_bytes - 1))
    return mp::set_error(MP_ERR_ALIGNMENT, "%s: offsets must be aligned to their width", name);
  s.offsets = offsets;
  s.id_bytes = id_bytes;
  s.n_seq = (int)n_seq;
  s.T = T;
  s.heads = (int)heads;
  s.kv_heads = (int)kv_heads;
  s.D = (int)D;
  s.scale = scale;
  s.scale_log2 = scale * kLog2e;
  s.causal = causal;
  s.window = window < T ? window : 0;              // one that no query reaches past is none
  s.st = state ? state->dev : nullptr;
  s.status = nullptr;
  return MP_OK;
}

int check_matrix(const char* name, const void* p, int64_t ld, int64_t heads, int64_t D) {
  if (ld < heads * D) return mp::set_error(MP_ERR_INVALID_ARG, "%s: leading dimension smaller than the heads", name);
  if ((ld & 7) || !mp::aligned16(p))
    return mp::set_error(MP_ERR_ALIGNMENT, "%s: matrices must be 16-byte aligned with pitches that are multiples of 8", name);
  return MP_OK;
}

}  // namespace attn

extern "C" int mp_attention_fwd(const void* q16, int64_t ldq, const void* k16, int64_t ldk, const void* v16, int64_t ldv,
                                void* o16, int64_t ldo, float* lse, const void* offsets, int id_bytes, int64_t n_seq,
                                int64_t T, int64_t heads, int64_t kv_heads, int64_t D, float scale, int causal,
                                int64_t window, mp_state* state, void* stream) {
  const char* name = "mp_attention_fwd";
  FwdArgs a;
  if (int rc = check_call(name, a.s, offsets, id_bytes, n_seq, T, heads, kv_heads, D, scale, causal, window, state)) return rc;
  if (int rc = check_matrix(name, q16, ldq, heads, D)) return rc;
  if (int rc = check_matrix(name, k16, ldk, kv_heads, D)) return rc;
  if (int rc = check_matrix(name, v16, ldv, kv_heads, D)) return rc;
  if (int rc = check_matrix(name, o16, ldo, heads, D)) return rc;
  if ((uintptr_t)lse & 3) return mp::set_error(MP_ERR_ALIGNMENT, "%s: FP32 values must be aligned", name);
  if (T > 0 && n_seq > 0 && (!q16 || !k16 || !v16 || !o16 || !lse))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: null pointer", name);
  if (T > 0 && n_seq > 0 && (o16 == q16 || o16 == k16 || o16 == v16))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: the result may not be an input", name);
  if (int rc = mp::check_device()) return rc;
  if (T == 0 || n_seq == 0) return MP_OK;
  if (int rc = mp::gemm_status_device_ptr(&a.s.status)) return rc;
  a.o = (uint16_t*)o16;
  a.ldo = ldo;
  a.lse = lse;
  CUtensorMap mq, mk, mv;
  if (int rc = make_map(&mq, Operand{q16, ldq, (int)heads}, T, (int)D)) return rc;
  if (int rc = make_map(&mk, Operand{k16, ldk, (int)kv_heads}, T, (int)D)) return rc;
  if (int rc = make_map(&mv, Operand{v16, ldv, (int)kv_heads}, T, (int)D)) return rc;
  const int64_t blocks = (T / ((D <= 64 ? FwdLayout<64>::kTiles : FwdLayout<128>::kTiles) * kTile) + n_seq) * heads;
  return D <= 64 ? fwd_launch<64>(mq, mk, mv, a, blocks, (cudaStream_t)stream)
                 : fwd_launch<128>(mq, mk, mv, a, blocks, (cudaStream_t)stream);
}

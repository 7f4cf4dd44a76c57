// Attention over packed sequences, forward: O = softmax(scale Q K^T) V for each head, with the rows' log-sums.
//
// One pass over the keys with a running maximum and sum.  A block has two tiles of 128 queries of a head, whose two
// products S = Q K^T and O += P V alternate on the tensor core: while one tile's scores go through the exponential, the
// other's products run.  S and O stay in tensor memory, P takes the place of its S there as FP16 (rounded once, 2^-12 of
// the value; the sum is taken from the unrounded FP32 values), keys and values pass through a ring in shared memory.
// The running maximum may lag: it is raised, and O multiplied, only where a row's maximum has passed it by 2^8, so that
// almost no tile pays for it; P stays below 2^8 and its FP16 rounding is relative.

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

// TILES query tiles a block.  Heads of more than 64 elements: two tiles share the keys and values, which would else ask L2
// for 64 bytes a clock and SM; below that one tile a block and two blocks an SM, whose beginnings and ends cover one another.
template <int DP>
struct FwdLayout {
  static constexpr int kTiles = DP == 64 ? 1 : 2, kBlocks = DP == 64 ? 2 : 1;      // tiles a block, blocks an SM
  static constexpr int kThreads = kTiles * 256 + 64;         // eight warps a tile, half a row a thread; then products; copies
  static constexpr int kBoxes = DP / 64, kTileBytes = kBoxes * kBoxBytes;
  static constexpr int kStages = DP == 64 ? 5 : 4;
  static constexpr int kSmem = (kTiles + kStages) * kTileBytes + 1024;
  static constexpr int kColumns = DP == 64 ? 256 : 512;      // of tensor memory: S, with P in its place, then O, for each tile
};
constexpr float kLag = 8.0f;

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// 2^x for two values on the multiply-add pipe: whole and fractional part split by rounding, a polynomial of the fraction on
// [-1/2, 1/2] (least largest relative error, 2.6e-6; fitted to 2^f by weighted least squares), the whole part added to the exponent.
__device__ __forceinline__ float2 ex2_poly(float2 x) {
  const float2 magic = make_float2(12582912.0f, 12582912.0f);            // 1.5 * 2^23: the sum's low bits are the whole part
  x = make_float2(fmaxf(x.x, -126.0f), fmaxf(x.y, -126.0f));
  const float2 t = add2(x, magic), whole = add2(t, make_float2(-12582912.0f, -12582912.0f));
  const float2 f = fma2(whole, make_float2(-1.0f, -1.0f), x);
  float2 p = make_float2(0.009570101276040077f, 0.009570101276040077f);
  p = fma2(p, f, make_float2(0.05591785907745361f, 0.05591785907745361f));
  p = fma2(p, f, make_float2(0.240247443318367f, 0.240247443318367f));
  p = fma2(p, f, make_float2(0.6931217908859253f, 0.6931217908859253f));
  p = fma2(p, f, make_float2(0.9999992847442627f, 0.9999992847442627f));
  return make_float2(__int_as_float(__float_as_int(p.x) + (__float_as_int(t.x) << 23)),
                     __int_as_float(__float_as_int(p.y) + (__float_as_int(t.y) << 23)));
}

// Among the 256 threads of tile t: a barrier, and whether anyone says yes; a barrier alone.
__device__ __forceinline__ bool any_of_tile(int t, bool yes) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.or.pred q, %2, 256, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(any)
      : "r"((uint32_t)yes), "r"(1 + t)
      : "memory");
  return any != 0;
}
__device__ __forceinline__ void tile_sync(int t) { asm volatile("barrier.cta.sync %0, 256;" ::"r"(1 + t) : "memory"); }

template <int DP>
__global__ void __launch_bounds__(FwdLayout<DP>::kThreads, FwdLayout<DP>::kBlocks)
mp_attention_fwd_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                        const __grid_constant__ CUtensorMap mv, const FwdArgs a) {
  using L = FwdLayout<DP>;
  constexpr int kTiles = L::kTiles, kProducts = kTiles * 8, kCopies = kProducts + 1;      // these two warps' numbers
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* ring = smem + kTiles * L::kTileBytes;
  // p_ready: the first and the second 64 columns of P; row_of, sum_of: what the threads of a row tell one another
  __shared__ uint64_t q_full, kv_full[L::kStages], kv_empty[L::kStages], tail_full, s_full[kTiles], p_ready[kTiles][2], o_done[kTiles];
  __shared__ float row_of[kTiles][2][kTile], sum_of[kTiles][2][kTile];
  __shared__ uint32_t s_tmem;
  __shared__ volatile int failed[kTiles];
  const Shape& s = a.s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  ptx::launch_dependents();
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
      ptx::mbar_init(&kv_empty[i], 1);
    }
    for (int t = 0; t < kTiles; ++t) {
      ptx::mbar_init(&s_full[t], 1);
      ptx::mbar_init(&p_ready[t][0], kTile);
      ptx::mbar_init(&p_ready[t][1], kTile);
      ptx::mbar_init(&o_done[t], 1);
      failed[t] = 0;
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
  const uint32_t tmem = s_tmem;
  constexpr uint32_t kO = kTiles * kTile;
  // the long ones first: a causal query sees all keys before it
  const int q0 = (int)(at.tiles - 1 - at.tile) * kTiles * kTile, len = (int)at.len;
  // key blocks that a tile of queries sees
  int b0[kTiles], b1[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int first = q0 + t * kTile, last = min(first + kTile, len);     // queries
    b0[t] = s.window > 0 && first + 1 > s.window ? (int)(first + 1 - s.window) / kTile : 0;
    b1[t] = first >= len ? b0[t] : ((s.causal ? last : len) + kTile - 1) / kTile;
  }
  const int j0 = b0[0], j1 = max(b1[0], b1[kTiles - 1]);
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
  } else if (warp == kProducts) {
    const int ksteps = (s.D + 15) / 16;
    const uint32_t idesc_o = ptx::idesc_f16_f32(kTile, ksteps * 16, false, true);
    ok = wait(&q_full, 0);
    for (int j = j0; j <= j1 && ok; ++j) {
      const int nk = 2 * (j - j0), nv = nk - 1;   // their places in the order of copies
      if (j < j1) ok = wait(&kv_full[nk % L::kStages], nk / L::kStages & 1);
      if (ok && j > j0) ok = wait(&kv_full[nv % L::kStages], nv / L::kStages & 1);
      const uint32_t sk = ptx::smem_u32(ring + nk % L::kStages * L::kTileBytes);
      const uint32_t sv = ptx::smem_u32(ring + (nv < 0 ? 0 : nv % L::kStages) * L::kTileBytes);
      // the last block of a sequence is as wide as it has keys
      const int before = (min(kTile, len - (j - 1) * kTile) + 15) / 16, wide = (min(kTile, len - j * kTile) + 15) / 16 * 16;
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        if (ok && j > b0[t] && j <= b1[t]) {      // O += P V of the block before, in two halves
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            ok = ok && wait(&p_ready[t][h], (j - 1 - b0[t]) & 1);
            ptx::tc_fence_after_sync();
            if (ok && ptx::elect_one()) {
              if (h == 0) {
                product_ts<0, 4>(tmem + kO + t * DP, tmem + t * kTile, desc_mn(sv), idesc_o, before, j - 1 > b0[t]);
              } else {
                product_ts<4, 8>(tmem + kO + t * DP, tmem + t * kTile, desc_mn(sv), idesc_o, before, true);
                ptx::mma_commit(&o_done[t]);
              }
            }
            __syncwarp();
          }
        }
        if (ok && j >= b0[t] && j < b1[t]) {      // S of this one, in the place of that P
          ptx::tc_fence_after_sync();
          if (ptx::elect_one()) {
            product_ss<DP / 16>(tmem + t * kTile, desc_k(ptx::smem_u32(smem + t * L::kTileBytes)), desc_k(sk),
                                ptx::idesc_f16_f32(kTile, wide, false, false), ksteps);
            ptx::mma_commit(&s_full[t]);
          }
          __syncwarp();
        }
      }
      if (ok && ptx::elect_one()) {
        if (j > j0) ptx::mma_commit(&kv_empty[nv % L::kStages]);
        if (j < j1) ptx::mma_commit(&kv_empty[nk % L::kStages]);
      }
      __syncwarp();
    }
  } else {
    // Two threads have a row, 64 columns each: a tile's scores pass through twice as many warps in half the time, and it is this
    // time that the products of the tile wait for.
    const int t = warp >> 3, half = warp >> 2 & 1, in_tile = (warp & 3) * 32 + lane, row = q0 + t * kTile + in_tile;   // of the sequence
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + t * kTile + half * 64 + lanes, to = tmem + kO + t * DP + half * (DP / 2) + lanes;
    const int lo = t ? b0[kTiles - 1] : b0[0], hi = t ? b1[kTiles - 1] : b1[0];
    const float c = s.scale_log2;
    const bool some = row - lane < len;           // the warp has rows that exist
    // the keys that this query sees
    const int key1 = s.causal ? min(row + 1, len) : len;
    const int key0 = s.window > 0 && row + 1 > s.window ? (int)(row + 1 - s.window) : 0;
    // blocks between these two are seen whole by every query of the warp; no query of it sees a key from `end` on
    const int first = row - lane;
    const int whole1 = s.causal ? min(first + 1, len) : len, end = s.causal ? min(first + 32, len) : len;
    const int whole0 = s.window > 0 && first + 32 > s.window ? (int)(first + 32 - s.window) : 0;
    float m = -INFINITY, sum = 0.0f;
    for (int j = lo; j < hi; ++j) {
      ok = ok && wait(&s_full[t], (j - lo) & 1);
      ptx::tc_fence_after_sync();
      const int k0 = j * kTile + half * 64;       // this thread's first key
      // pieces of 32 columns with keys that are seen (rows of what comes behind the sequence: whatever P holds stays in them)
      const int pieces = !ok || !some ? 0 : max(0, min(2, (end - k0 + 31) / 32));
      const bool edge = k0 + 64 > whole1 || k0 < whole0;
      const int stop = key1 - k0, begin = key0 - k0;
      // The scores are read twice, for the maximum and for the weights: in registers all the while they would not leave room
      // for enough warps.
      uint32_t r[32];
      auto load = [&](int i) {
        ptx::tmem_ld_32x32(ts + i * 32, r);
        ptx::tmem_ld_wait();
        if (edge) {
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (i * 32 + e >= stop || i * 32 + e < begin) r[e] = 0xFF800000u;
        }
      };
      float now = -INFINITY, other = -INFINITY;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (i < pieces) {
          load(i);
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            now = max3(now, __uint_as_float(r[e]), __uint_as_float(r[e + 1]));
            other = max3(other, __uint_as_float(r[e + 2]), __uint_as_float(r[e + 3]));
          }
        }
      now = fmaxf(now, other) * c;
      // from -inf on: at the first block with a key that is seen.  (A wait that ran out comes this way too, to end all warps.)
      if (any_of_tile(t, now > m + kLag || !ok)) {
        row_of[t][half][in_tile] = now;
        if (!ok) failed[t] = 1;
        tile_sync(t);
        if (failed[t]) {
          ok = false;
          break;
        }
        now = fmaxf(now, row_of[t][half ^ 1][in_tile]);
        const bool raise = now > m + kLag;
        const float f = raise ? ex2(m - now) : 1.0f;
        m = raise ? now : m;
        sum *= f;
        if (j > lo && __any_sync(0xFFFFFFFFu, raise)) {      // the products so far have this maximum's factor
          ok = wait(&o_done[t], (j - 1 - lo) & 1);
          ptx::tc_fence_after_sync();
#pragma unroll 1
          for (int i = 0; i < DP / 2; i += 32) {
            uint32_t v[32];
            ptx::tmem_ld_32x32(to + i, v);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * f);
            tmem_st_32x32(to + i, v);
          }
        }
      }
      const float shift = m == -INFINITY ? 0.0f : -m;
      const float2 c2 = make_float2(c, c), shift2 = make_float2(shift, shift);
      float2 part = make_float2(0.0f, 0.0f);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t p[16];
        if (i < pieces) {
          load(i);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float2 x = fma2(make_float2(__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1])), c2, shift2);
            const float2 y = e % 8 == 7 ? ex2_poly(x) : make_float2(ex2(x.x), ex2(x.y));
            part = add2(part, y);
            p[e] = rows::pack2(y.x, y.y);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) p[e] = 0;
        }
        if (some) tmem_st_32x16(ts + i * 16, p);
      }
      tmem_st_wait();
      ptx::tc_fence_before_sync();
      ptx::mbar_arrive(&p_ready[t][half]);
      sum += part.x + part.y;
    }
    // (a warp whose wait ran out comes here as well: all of the tile's warps meet once more)
    sum_of[t][half][in_tile] = sum;
    if (!ok) failed[t] = 1;
    tile_sync(t);
    ok = ok && !failed[t];
    if (ok && some && hi > lo) {
      sum += sum_of[t][half ^ 1][in_tile];
      ok = wait(&o_done[t], (hi - 1 - lo) & 1);
      ptx::tc_fence_after_sync();
      const float inv = 1.0f / sum;
      uint16_t* o = a.o + (at.start + row) * a.ldo + (int64_t)head * s.D;
#pragma unroll
      for (int i = 0; i < DP / 2; i += 32) {
        const int col = half * (DP / 2) + i;
        if (col >= s.D) break;
        uint32_t v[32];
        ptx::tmem_ld_32x32(to + i, v);
        ptx::tmem_ld_wait();
        if (ok && row < len) {
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
            float f[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) f[x] = __uint_as_float(v[e + x]) * inv;
            if (col + e < s.D) *reinterpret_cast<uint4*>(o + col + e) = rows::pack8(f);
          }
        }
      }
      if (ok && row < len && half == 0) a.lse[(int64_t)head * s.T + at.start + row] = (m + log2f(sum)) * kLn2;
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

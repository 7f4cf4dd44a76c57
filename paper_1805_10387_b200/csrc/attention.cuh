// What the attention kernels share: where a block's tile lies in the packed sequences, tensor-memory accesses that
// the products do not have, operand descriptors of 128-row tiles, and the record of an expired wait.
#pragma once

#include <cuda.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "common.h"
#include "ptx.cuh"
#include "rows.cuh"

namespace attn {

using rows::add2;
using rows::fma2;
using rows::mul2;

constexpr int kTile = 128;                        // queries or keys of a tile: rows of an MMA, lanes of tensor memory
constexpr int kBoxBytes = kTile * 128;            // 128 rows x 64 FP16 columns, the unit that a copy brings
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Shape {
  const void* offsets;
  int id_bytes, n_seq;
  int64_t T;
  int heads, kv_heads, D;
  float scale, scale_log2;                        // of the scores, and times log2 e
  int causal;
  int64_t window;                                 // keys that a query sees, itself the last (0: all)
  mp_dev_state* st;
  int* status;                                    // the device-wide status word
};

// A tile of ROWS rows of a packed sequence.
struct Place {
  int64_t start;                                  // row of the sequence's first token
  int64_t len;                                    // its tokens
  int64_t tile, tiles;                            // this tile, tiles of the sequence; tile >= tiles: no work
};
__device__ __forceinline__ int64_t offset_at(const Shape& s, int64_t b) {
  return s.id_bytes == 8 ? rows::load_id<int64_t>(s.offsets, b) : rows::load_id<int32_t>(s.offsets, b);
}
// Work item v belongs to the last sequence b with offset[b] / ROWS + b <= v, and is its tile v - (offset[b] / ROWS + b): a
// sequence of n tokens has at most (offset[b + 1] / ROWS) - (offset[b] / ROWS) + 1 tiles, so no two sequences share an
// item, nobody needs the sum of the tiles before him, and T / ROWS + n_seq items cover all.  Found by a whole warp,
// 32 ways at a time (8192 sequences: three dependent loads).
template <int ROWS>
__device__ __forceinline__ Place place_of(const Shape& s, int64_t v) {
  const int lane = threadIdx.x & 31;
  int64_t lo = 0, hi = s.n_seq, from = offset_at(s, 0), to = 0;
  while (true) {
    const int64_t hop = (hi - lo + 31) / 32, b = lo + (lane + 1) * hop;
    const int64_t x = b <= hi ? offset_at(s, b) : 0;         // (offset[n_seq] ends the last sequence)
    const int n = __popc(__ballot_sync(0xFFFFFFFFu, b < hi && x / ROWS + b <= v));
    if (n > 0) from = __shfl_sync(0xFFFFFFFFu, x, n - 1);
    const int64_t next = lo + (n + 1) * hop;
    lo += n * hop;
    hi = next < hi ? next : hi;
    if (hop == 1) {                               // the next offset is the next lane's
      to = __shfl_sync(0xFFFFFFFFu, x, n);
      break;
    }
  }
  Place p{from, to - from, v - (from / ROWS + lo), 0};
  // an offset out of order or range gives no work (and is recorded by check_offsets)
  if (from >= 0 && to >= from && to <= s.T && p.tile >= 0) p.tiles = (p.len + ROWS - 1) / ROWS;
  else p.tile = 0;
  return p;
}
// One warp looks all offsets over.
__device__ __forceinline__ void check_offsets(const Shape& s) {
  bool bad = false;
  for (int64_t b = threadIdx.x & 31; b < s.n_seq; b += 32) {
    const int64_t from = offset_at(s, b), to = offset_at(s, b + 1);
    bad |= from < 0 || to < from || to > s.T;
  }
  if (bad) rows::record_bad_id(s.st);
}

// Bounded wait of a whole warp: the same answer in every lane.  (One lane that looks for all is slower: 8192 x 8192, 32 heads of 128,
// 1.51 ms against 1.30.)
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity) {
  return __all_sync(0xFFFFFFFFu, ptx::mbar_wait(bar, parity, ptx::kWaitNs));
}
__device__ __forceinline__ void arrive(uint64_t* bar) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) ptx::mbar_arrive(bar);
}
__device__ __forceinline__ void report_timeout(const Shape& s) {
  atomicCAS(s.status, 0, (int)MP_ERR_TIMEOUT);
  if (s.st != nullptr) atomicCAS(&s.st->h.status, 0, (int)MP_ERR_TIMEOUT);
}

__device__ __forceinline__ float ex2(float x) {   // 2 units in the last place; 0 below the normal range
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// ---- copies: 3-D maps [token][head][element] ----
__device__ __forceinline__ void load_box(void* dst, const CUtensorMap* map, uint64_t* bar, int col, int head, int row) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(ptx::smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(ptx::smem_u32(bar)), "r"(col), "r"(head), "r"(row)
      : "memory");
}
// 128 rows of one head from `row` on, BOXES x 64 columns (columns past the head are zeros).
template <int BOXES>
__device__ __forceinline__ void load_tile(uint8_t* dst, const CUtensorMap* map, uint64_t* bar, int head, int row) {
#pragma unroll
  for (int c = 0; c < BOXES; ++c) load_box(dst + c * kBoxBytes, map, bar, 64 * c, head, row);
}
// Zeros in place of the rows from `valid` on: rows of the next sequence, whose values must not matter (a weight of 0
// times an infinity is not 0).  By a whole warp, after the copy has landed; the caller hands the tile on.
template <int BOXES>
__device__ __forceinline__ void clear_rows(uint8_t* tile, int valid) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int c = 0; c < BOXES; ++c)
    for (int i = valid * 128 + lane * 16; i < kBoxBytes; i += 512)
      *reinterpret_cast<uint4*>(tile + c * kBoxBytes + i) = make_uint4(0, 0, 0, 0);
  ptx::fence_proxy_async_smem();
  __syncwarp();
}

// ---- operands in shared memory: boxes of 128 rows of 128 bytes, 128-byte swizzle ----
// Along the columns (the tile's rows are the operand's M or N), and along the rows (its columns are the operand's N); step ks
// of 16.  A descriptor is formed once for a tile; a step adds a constant to it, since its address is in units of 16 bytes.
__device__ __forceinline__ uint64_t desc_k(uint32_t tile) { return ptx::smem_desc_sw128(tile, 16, 1024); }
__device__ __forceinline__ uint64_t desc_mn(uint32_t tile) { return ptx::smem_desc_sw128(tile, kBoxBytes, 1024); }
__host__ __device__ constexpr uint64_t step_k(int ks) { return (uint64_t)((ks >> 2) * kBoxBytes + (ks & 3) * 32) >> 4; }
__host__ __device__ constexpr uint64_t step_mn(int ks) { return (uint64_t)(ks * 2048) >> 4; }

// D[tmem] (+)= A[tmem] B[smem]; A: FP16 pairs in 32-bit columns, 8 columns a step of 16.
__device__ __forceinline__ void mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                           uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// A product of two tiles: D (+)= sum over `steps` of 16, at most STEPS.  By one thread; unrolled, so that what an instruction
// needs is at hand when the tensor core is free: a loop that formed descriptors issued one in 130 cycles, and a step takes 64.
template <int STEPS>
__device__ __forceinline__ void product_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, int steps) {
#pragma unroll
  for (int k = 0; k < STEPS; ++k)
    if (k < steps) ptx::mma_f16_ss(d, a + step_k(k), b + step_k(k), idesc, k > 0);
}
// The same with A in tensor memory, along the rows of a tile.  QUARTERS: each 32 columns were written in the place of their
// scores by a warp of their own, so their 16 packed columns begin where the scores did; else all follow one another.
template <int STEPS, bool QUARTERS>
__device__ __forceinline__ void product_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, int steps, bool accumulate) {
#pragma unroll
  for (int k = 0; k < STEPS; ++k)
    if (k < steps) mma_f16_ts(d, a + (QUARTERS ? (k >> 1) * 32 + (k & 1) * 8 : 8 * k), b + step_mn(k), idesc, accumulate || k > 0);
}

// 32 lanes x 32 consecutive 32-bit columns from registers.
__device__ __forceinline__ void tmem_st_32x32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
      "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
      "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st_32x16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Host side.
struct Operand {
  const void* ptr;
  int64_t ld;
  int heads;
};
int make_map(CUtensorMap* map, const Operand& x, int64_t T, int D);
// Checks that the forward and the backward call have in common; fills `s`.
int check_call(const char* name, Shape& s, const void* offsets, int id_bytes, int64_t n_seq, int64_t T, int64_t heads,
               int64_t kv_heads, int64_t D, float scale, int causal, int64_t window, mp_state* state);
int check_matrix(const char* name, const void* p, int64_t ld, int64_t heads, int64_t D);

}  // namespace attn

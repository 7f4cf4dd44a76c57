// Norms before and after a block, with the block's gate and the residual scale, forward and backward.

#include "rows.cuh"

namespace {

// Rows of up to 8192 elements, forward and backward: persistent blocks of 512 threads.  A group of TPR
// threads, each with two vectors of 8 columns, walks the rows r, r + step, ...  Each thread fetches its own
// vectors of the next rows into its own slots of shared memory with asynchronous copies (zeros for what
// lies past the row), so the loads of the following rows are in flight while a row is worked on and no
// thread waits for another's copy; the row stays in registers and shared memory between the norms, so
// that everything is read once and written once.  What depends on the column alone (the gains, the
// gate vector) stays in the thread's registers over all rows.
// An element costs 8 B of HBM traffic forward and 12 B backward (FP16, shared gate), and some 20 and 50
// instructions.  Measured on B200s: forward 8192 x 1024 16.4 - 16.6 us (4.1 TB/s), 32768 x 1024 51 us (5.3 TB/s), backward
// 25600 x 1600 112 - 113 us (4.4 TB/s).  Backward fills neither HBM (two thirds) nor the issue slots (56 %): with 128 registers
// a thread an SM holds 16 warps, too few to cover the latency of the row's sums; a fifth of the lanes idle at a width of
// 1600.  Widths just above a power of two leave half idle (1032: 24 us forward, 1024: 16.5).  One row per block without prefetch took 70 and 2184 us, rows in registers of groups that come and
// go 22.6 us forward.  Tried for the backward pass and slower: 1024 threads with one vector each (150 us, spilled
// registers), 384 threads (125 us), the rows' addresses recomputed instead of kept (122 us).
constexpr int kRowThreads = 512, kC = 2;

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copy_wait(int stages) {     // all but the newest stages - 1 groups are complete
  if (stages == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else if (stages == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else asm volatile("cp.async.wait_group 3;" ::: "memory");
}

// One array of rows that a kernel reads: its vectors c of this thread lie in the slots slot + c * XS.
template <class T>
struct Stream {
  static constexpr int XS = sizeof(T) / 2;       // 16-byte slots of a vector
  const T* row;                                  // this thread's first column in the row to fetch next
  int64_t hop;                                   // elements from one of the group's rows to its next
  int slot;
  __device__ __forceinline__ Stream(const void* p, int64_t ld, int64_t first, int64_t step, int t, int& slots)
      : row(static_cast<const T*>(p) + first * ld + t * 8), hop(step * ld), slot(slots) {
    if (p != nullptr) slots += kC * XS;
  }
  // FP32: the 2 n halves of the vectors of n <= 32 neighbouring threads are copied in their order in memory, so
  // that an access of the warp touches whole sectors; a half lands in its owner's slot, wherever that is.
  // (Each thread copying both halves of its own vector fetched every sector twice.)
  template <int TPR>
  __device__ __forceinline__ void fetch(uint32_t stage, const int (&nv)[kC], int D, int t, bool inside) {
#pragma unroll
    for (int c = 0; c < kC; ++c)
      if constexpr (XS == 1) {
        copy16(stage + (slot + c) * (kRowThreads * 16), row + c * TPR * 8, inside && nv[c] > 0);
      } else {
        constexpr int n = TPR < 32 ? TPR : 32;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int piece = h * n + t % n, shift = piece / 2 - t % n, half = piece & 1;   // shift: to the owner
          copy16(stage + ((slot + c * 2 + half) * kRowThreads + shift) * 16, row + (c * TPR + shift) * 8 + half * 4,
                 inside && D > (c * TPR + t + shift) * 8 + half * 4);
        }
      }
    row += hop;
  }
  __device__ __forceinline__ void read(const uint4* stage, int c, int nv, float (&f)[8]) const {
    rows::Raw8<T> r;
    uint4* q = reinterpret_cast<uint4*>(&r);
#pragma unroll
    for (int h = 0; h < XS; ++h) q[h] = stage[(slot + c * XS + h) * kRowThreads];
    if (nv > 0 && nv < 8) r.keep(nv);            // a vector across the row's end: its padding may hold anything
    r.floats(f);
  }
};

// Stores a vector of the residual type at p.  FP32: two neighbouring threads exchange halves first, so that
// each store of the pair is 32 contiguous bytes.  Every thread of the warp calls; `live`: the row exists.
__device__ __forceinline__ void put(uint16_t* p, const float (&f)[8], int nv, int, bool live) {
  if (live && nv > 0) rows::store8(p, f, nv);
}
__device__ __forceinline__ void put(float* p, const float (&f)[8], int nv, int t, bool live) {
  const bool odd = t & 1;
  float o[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) o[j] = __shfl_xor_sync(0xFFFFFFFFu, odd ? f[j] : f[4 + j], 1);
  const bool both = __shfl_sync(0xFFFFFFFFu, nv, threadIdx.x | 1) == 8;      // then the even thread's is whole too
  if (!live) return;
  if (both) {
    __stcs(reinterpret_cast<float4*>(odd ? p - 4 : p), odd ? make_float4(o[0], o[1], o[2], o[3]) : make_float4(f[0], f[1], f[2], f[3]));
    __stcs(reinterpret_cast<float4*>(odd ? p + 4 : p + 8), odd ? make_float4(f[4], f[5], f[6], f[7]) : make_float4(o[0], o[1], o[2], o[3]));
  } else if (nv > 0) {
    rows::store8(p, f, nv);
  }
}

// ---------------------------------------------------------------- forward
struct FwdArgs {
  float eps, res_scale;
  const void* x; int64_t ldx;
  const uint16_t* y; int64_t ldy;
  const uint16_t *g_post, *gate; int64_t ldgate;
  void* x_out; int64_t ldxo;
  const uint16_t* g_pre;
  uint16_t* n; int64_t ldn;
  float* stats;
  int64_t M;
  int D;
  int stages;      // rows in flight per group, the one at work included (2 .. 4)
  int slots;       // 16-byte slots per thread and stage
};

// Sums of a vector's elements and of their squares about `mean`; of a vector across the row's end only what is inside.
__device__ __forceinline__ void add_squares(const float (&f)[8], float mean, int nv, float& q) {
  if (nv == 8) {
#pragma unroll
    for (int j = 0; j < 8; ++j) q = fmaf(f[j] - mean, f[j] - mean, q);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < nv) q = fmaf(f[j] - mean, f[j] - mean, q);
  }
}
template <int TPR, bool LAYER>
__device__ __forceinline__ float2 moments(const float (&f)[kC][8], const int (&nv)[kC], float inv_d, float eps, float* red,
                                          int& parity) {
  float mean = 0.0f;
  if constexpr (LAYER) {
    float s[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < kC; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) s[0] += f[c][j];     // zeros past the row's end
    rows::group_sum<TPR, 1>(s, red, parity);
    mean = s[0] * inv_d;
  }
  float q[1] = {0.0f};
#pragma unroll
  for (int c = 0; c < kC; ++c) {
    if constexpr (LAYER) {
      add_squares(f[c], mean, nv[c], q[0]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) q[0] = fmaf(f[c][j], f[c][j], q[0]);
    }
  }
  rows::group_sum<TPR, 1>(q, red, parity);
  return make_float2(mean, rsqrtf(fmaf(q[0], inv_d, eps)));
}

template <class XT, int TPR, bool LAYER>
__global__ void __launch_bounds__(kRowThreads, 1) mp_block_norm_fwd_kernel(const FwdArgs a) {
  constexpr int G = kRowThreads / TPR;
  extern __shared__ uint4 slots[];
  __shared__ float red_all[G][rows::red_floats<TPR, 1>];
  const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
  float* red = red_all[group];
  int parity = 0, used = 0;
  const bool has_y = a.g_post != nullptr, matrix = a.gate != nullptr && a.ldgate != 0;
  const float inv_d = 1.0f / (float)a.D;
  int nv[kC];
#pragma unroll
  for (int c = 0; c < kC; ++c) {
    const int left = a.D - (c * TPR + t) * 8;
    nv[c] = left < 0 ? 0 : left < 8 ? left : 8;
  }
  const int64_t step = (int64_t)gridDim.x * G, first = (int64_t)blockIdx.x * G + group;
  // the row that decides when the loop ends: that of the warp's first group, so that a warp stays whole
  const int64_t lead = TPR >= 32 ? first : (int64_t)blockIdx.x * G + (threadIdx.x & ~31) / TPR;
  Stream<XT> sx(a.x, a.ldx, first, step, t, used);
  Stream<uint16_t> sy(a.y, a.ldy, first, step, t, used), sg(matrix ? a.gate : nullptr, a.ldgate, first, step, t, used);
  const uint32_t base = static_cast<uint32_t>(__cvta_generic_to_shared(slots)) + threadIdx.x * 16;
  int64_t ahead = first;
  auto fetch = [&](int stage) {
    const bool inside = ahead < a.M;
    if (TPR < 32 || inside) {
      const uint32_t at = base + (uint32_t)(stage * a.slots) * (kRowThreads * 16);
      sx.template fetch<TPR>(at, nv, a.D, t, inside);
      if (has_y) sy.template fetch<TPR>(at, nv, a.D, t, inside);
      if (matrix) sg.template fetch<TPR>(at, nv, a.D, t, inside);
    }
    ahead += step;
    copy_commit();
  };
  for (int s = 0; s + 1 < a.stages; ++s) fetch(s);
  float q[kC][8], gq[kC][8];                     // g_post * gate (a gate matrix comes with the row), g_pre
#pragma unroll
  for (int c = 0; c < kC; ++c) {
    const int col = (c * TPR + t) * 8;
    rows::Raw8<uint16_t> r;
    r.load_cached(a.g_pre + col, nv[c]);
    r.floats(gq[c]);
    if (has_y) {
      float g[8];
      r.load_cached(a.g_post + col, nv[c]);
      r.floats(q[c]);
      if (a.gate != nullptr && !matrix) {
        r.load_cached(a.gate + col, nv[c]);
        r.floats(g);
#pragma unroll
        for (int j = 0; j < 8; ++j) q[c][j] *= g[j];
      }
    }
  }
  int stage = 0;
  int64_t m = first;
  for (int64_t lm = lead; lm < a.M; lm += step, m += step) {
    const bool live = TPR >= 32 || m < a.M;
    if (sizeof(XT) == 4) __syncwarp();           // everyone has read the slots of the row before this one
    fetch(stage == 0 ? a.stages - 1 : stage - 1);
    copy_wait(a.stages);
    if (sizeof(XT) == 4) __syncwarp();           // the others' copies into this thread's slots are complete too
    const uint4* mine = slots + threadIdx.x + (int64_t)stage * a.slots * kRowThreads;
    float xo[kC][8];
    float2 my = make_float2(0.0f, 0.0f);
    if (has_y) {
      float y[kC][8];
#pragma unroll
      for (int c = 0; c < kC; ++c) sy.read(mine, c, nv[c], y[c]);
      my = moments<TPR, LAYER>(y, nv, inv_d, a.eps, red, parity);
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        float g[8];
        sx.read(mine, c, nv[c], xo[c]);
        if (matrix) sg.read(mine, c, nv[c], g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float h = LAYER ? (y[c][j] - my.x) * my.y : y[c][j] * my.y;
          xo[c][j] = fmaf(h, matrix ? q[c][j] * g[j] : q[c][j], a.res_scale * xo[c][j]);
        }
        put(reinterpret_cast<XT*>(a.x_out) + m * a.ldxo + (c * TPR + t) * 8, xo[c], nv[c], t, live);
      }
    } else {
#pragma unroll
      for (int c = 0; c < kC; ++c) sx.read(mine, c, nv[c], xo[c]);
    }
    const float2 mx = moments<TPR, LAYER>(xo, nv, inv_d, a.eps, red, parity);
#pragma unroll
    for (int c = 0; c < kC; ++c) {
#pragma unroll
      for (int j = 0; j < 8; ++j) xo[c][j] = (LAYER ? xo[c][j] - mx.x : xo[c][j]) * mx.y * gq[c][j];
      if (live && nv[c] > 0) rows::store8(a.n + m * a.ldn + (c * TPR + t) * 8, xo[c], nv[c]);
    }
    if (a.stats != nullptr && t == 0 && live) reinterpret_cast<float4*>(a.stats)[m] = make_float4(my.x, my.y, mx.x, mx.y);
    stage = stage + 1 == a.stages ? 0 : stage + 1;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

// Longer rows: a block per row, the row in registers, one row after the other.
template <class XT, bool LAYER>
__global__ void __launch_bounds__(kRowThreads, 1) mp_block_norm_fwd_wide_kernel(const FwdArgs a) {
  constexpr int TPR = kRowThreads, C = 4;
  __shared__ float red[rows::red_floats<TPR, 1>];
  int parity = 0;
  const float inv_d = 1.0f / (float)a.D;
  auto moments_of = [&](const float (&f)[C][8]) {
    float mean = 0.0f;
    if constexpr (LAYER) {
      float s[1] = {0.0f};
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) s[0] += f[c][j];
      rows::group_sum<TPR, 1>(s, red, parity);
      mean = s[0] * inv_d;
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int left = a.D - (c * TPR + (int)threadIdx.x) * 8;
      add_squares(f[c], mean, left < 0 ? 0 : left < 8 ? left : 8, q[0]);
    }
    rows::group_sum<TPR, 1>(q, red, parity);
    return make_float2(mean, rsqrtf(fmaf(q[0], inv_d, a.eps)));
  };
  for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x) {
    float xo[C][8];
    float2 my = make_float2(0.0f, 0.0f);
    rows::Raw8<XT> xr;
    rows::Raw8<uint16_t> r;
    auto col_of = [&](int c) { return (c * TPR + (int)threadIdx.x) * 8; };
    auto nv_of = [&](int c) { const int left = a.D - col_of(c); return left < 0 ? 0 : left < 8 ? left : 8; };
#pragma unroll
    for (int c = 0; c < C; ++c) {
      xr.load(reinterpret_cast<const XT*>(a.x) + m * a.ldx + col_of(c), nv_of(c));
      xr.floats(xo[c]);
    }
    if (a.g_post != nullptr) {
      float y[C][8];
#pragma unroll
      for (int c = 0; c < C; ++c) {
        r.load(a.y + m * a.ldy + col_of(c), nv_of(c));
        r.floats(y[c]);
      }
      my = moments_of(y);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = col_of(c), nv = nv_of(c);
        if (nv == 0) continue;
        float g[8];
        r.load_cached(a.g_post + col, nv);
        r.floats(g);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[c][j] = (y[c][j] - my.x) * my.y * g[j];
        if (a.gate != nullptr) {
          r.load(a.gate + m * a.ldgate + col, nv);
          r.floats(g);
#pragma unroll
          for (int j = 0; j < 8; ++j) y[c][j] *= g[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) xo[c][j] = fmaf(a.res_scale, xo[c][j], y[c][j]);
        rows::store8(reinterpret_cast<XT*>(a.x_out) + m * a.ldxo + col, xo[c], nv);
      }
    }
    const float2 mx = moments_of(xo);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = col_of(c), nv = nv_of(c);
      if (nv == 0) continue;
      float g[8];
      r.load_cached(a.g_pre + col, nv);
      r.floats(g);
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] *= (xo[c][j] - mx.x) * mx.y;
      rows::store8(a.n + m * a.ldn + col, g, nv);
    }
    if (a.stats != nullptr && threadIdx.x == 0) reinterpret_cast<float4*>(a.stats)[m] = make_float4(my.x, my.y, mx.x, mx.y);
  }
}

// ---------------------------------------------------------------- backward
//
// The sums over the rows stay in the registers of the thread that owns the columns: two of them, since
// with a gate vector dg_post and dgate are the same sum S = sum gx yhat times a factor of the column
// (dg_post = gate S, dgate = g_post S), and with a gate matrix dgate is no sum.  At the end the groups of a block
// add theirs in order through shared memory and the block writes one partial row of each.
struct BwdArgs {
  int kind;
  float res_scale;
  const uint16_t* dn; int64_t lddn;
  const void* dx_out; int64_t lddxo;
  const void* x_out; int64_t ldxo;
  const uint16_t* y; int64_t ldy;
  const uint16_t *g_post, *gate; int64_t ldgate;
  const uint16_t* g_pre;
  const float* stats;
  void* dx; int64_t lddx;
  uint16_t* dy; int64_t lddy;
  uint16_t* dgate; int64_t lddgate;
  int64_t M;
  int D;
  float* partial;  // [block][2][D]
  int stages;      // rows in flight per group, the one at work included (2 .. 4)
  int slots;       // 16-byte slots per thread and stage
};

template <class XT, int TPR, bool LAYER, bool MATRIX>
__global__ void __launch_bounds__(kRowThreads, 1) mp_block_norm_bwd_kernel(const BwdArgs a) {
  constexpr int G = kRowThreads / TPR, N = LAYER ? 2 : 1;        // N: row sums that a norm's backward needs
  extern __shared__ uint4 slots[];
  __shared__ float red_all[G][rows::red_floats<TPR, N>];
  const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
  float* red = red_all[group];
  int parity = 0, used = 0;
  const bool has_y = a.g_post != nullptr, has_up = a.dx_out != nullptr;
  const float inv_d = 1.0f / (float)a.D, res = has_y ? a.res_scale : 1.0f;
  int nv[kC];
#pragma unroll
  for (int c = 0; c < kC; ++c) {
    const int left = a.D - (c * TPR + t) * 8;
    nv[c] = left < 0 ? 0 : left < 8 ? left : 8;
  }
  const int64_t step = (int64_t)gridDim.x * G, first = (int64_t)blockIdx.x * G + group;
  const int64_t lead = TPR >= 32 ? first : (int64_t)blockIdx.x * G + (threadIdx.x & ~31) / TPR;
  Stream<XT> sx(a.x_out, a.ldxo, first, step, t, used), su(a.dx_out, a.lddxo, first, step, t, used);
  Stream<uint16_t> sd(a.dn, a.lddn, first, step, t, used), sy(a.y, a.ldy, first, step, t, used),
      sg(MATRIX ? a.gate : nullptr, a.ldgate, first, step, t, used);
  const uint32_t base = static_cast<uint32_t>(__cvta_generic_to_shared(slots)) + threadIdx.x * 16;
  int64_t ahead = first;
  auto fetch = [&](int stage) {
    const bool inside = ahead < a.M;
    if (TPR < 32 || inside) {
      const uint32_t at = base + (uint32_t)(stage * a.slots) * (kRowThreads * 16);
      sx.template fetch<TPR>(at, nv, a.D, t, inside);
      if (has_up) su.template fetch<TPR>(at, nv, a.D, t, inside);
      sd.template fetch<TPR>(at, nv, a.D, t, inside);
      if (has_y) sy.template fetch<TPR>(at, nv, a.D, t, inside);
      if (MATRIX) sg.template fetch<TPR>(at, nv, a.D, t, inside);
    }
    ahead += step;
    copy_commit();
  };
  for (int s = 0; s + 1 < a.stages; ++s) fetch(s);
  float q[kC][8], gq[kC][8];                     // g_post * gate (a gate matrix comes with the row), g_pre
#pragma unroll
  for (int c = 0; c < kC; ++c) {
    const int col = (c * TPR + t) * 8;
    rows::Raw8<uint16_t> r;
    r.load_cached(a.g_pre + col, nv[c]);
    r.floats(gq[c]);
    if (has_y) {
      float g[8];
      r.load_cached(a.g_post + col, nv[c]);
      r.floats(q[c]);
      if (!MATRIX && a.gate != nullptr) {
        r.load_cached(a.gate + col, nv[c]);
        r.floats(g);
#pragma unroll
        for (int j = 0; j < 8; ++j) q[c][j] *= g[j];
      }
    }
  }
  float s_pre[kC][8] = {}, s_y[kC][8] = {};
  int stage = 0;
  int64_t m = first;
  for (int64_t lm = lead; lm < a.M; lm += step, m += step) {
    const bool live = TPR >= 32 || m < a.M;
    if (sizeof(XT) == 4) __syncwarp();           // everyone has read the slots of the row before this one
    fetch(stage == 0 ? a.stages - 1 : stage - 1);
    const float4 st = live ? __ldg(reinterpret_cast<const float4*>(a.stats) + m) : make_float4(0, 0, 0, 0);
    copy_wait(a.stages);
    if (sizeof(XT) == 4) __syncwarp();           // the others' copies into this thread's slots are complete too
    const uint4* mine = slots + threadIdx.x + (int64_t)stage * a.slots * kRowThreads;
    float gx[kC][8], hat[kC][8];
    float ab[N] = {};
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      float dn[8];
      sx.read(mine, c, nv[c], hat[c]);
      sd.read(mine, c, nv[c], dn);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        hat[c][j] = (LAYER ? hat[c][j] - st.z : hat[c][j]) * st.w;
        gx[c][j] = dn[j] * gq[c][j];
        s_pre[c][j] = fmaf(dn[j], hat[c][j], s_pre[c][j]);
        ab[0] = fmaf(gx[c][j], hat[c][j], ab[0]);
        if constexpr (LAYER) ab[1] += gx[c][j];
      }
    }
    rows::group_sum<TPR, N>(ab, red, parity);
    const float sa = ab[0] * inv_d;
    float sb = 0.0f;
    if constexpr (LAYER) sb = ab[1] * inv_d;
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      float up[8] = {};
      if (has_up) su.read(mine, c, nv[c], up);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        gx[c][j] = fmaf(fmaf(-hat[c][j], sa, LAYER ? gx[c][j] - sb : gx[c][j]), st.w, up[j]);
        up[j] = res * gx[c][j];
      }
      put(reinterpret_cast<XT*>(a.dx) + m * a.lddx + (c * TPR + t) * 8, up, nv[c], t, live);
    }
    if (has_y) {
      float ef[N] = {};
#pragma unroll
      for (int c = 0; c < kC; ++c) {             // hat: yhat from here on
        float g[8], dg[8];
        sy.read(mine, c, nv[c], hat[c]);
        if (MATRIX) sg.read(mine, c, nv[c], g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          hat[c][j] = (LAYER ? hat[c][j] - st.x : hat[c][j]) * st.y;
          float gy = gx[c][j] * hat[c][j];
          gx[c][j] *= MATRIX ? q[c][j] * g[j] : q[c][j];
          ef[0] = fmaf(gx[c][j], hat[c][j], ef[0]);
          if constexpr (LAYER) ef[1] += gx[c][j];
          if (MATRIX) {
            dg[j] = gy * q[c][j];
            gy *= g[j];
          }
          s_y[c][j] += gy;
        }
        if (MATRIX && live && nv[c] > 0) rows::store8(a.dgate + m * a.lddgate + (c * TPR + t) * 8, dg, nv[c]);
      }
      rows::group_sum<TPR, N>(ef, red, parity);
      const float se = ef[0] * inv_d;
      float sf = 0.0f;
      if constexpr (LAYER) sf = ef[1] * inv_d;
#pragma unroll
      for (int c = 0; c < kC; ++c) {
#pragma unroll
        for (int j = 0; j < 8; ++j) gx[c][j] = fmaf(-hat[c][j], se, LAYER ? gx[c][j] - sf : gx[c][j]) * st.y;
        if (live && nv[c] > 0) rows::store8(a.dy + m * a.lddy + (c * TPR + t) * 8, gx[c], nv[c]);
      }
    }
    stage = stage + 1 == a.stages ? 0 : stage + 1;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();                               // the slots become the groups' sums
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  float* sums = reinterpret_cast<float*>(slots);                 // [group][D rounded up to whole vectors]
  const int width = kC * TPR * 8;
  auto reduce = [&](float (&s)[kC][8], int which) {
#pragma unroll
    for (int c = 0; c < kC; ++c)
#pragma unroll
      for (int j = 0; j < 8; j += 4)
        *reinterpret_cast<float4*>(sums + group * width + (c * TPR + t) * 8 + j) =
            make_float4(s[c][j], s[c][j + 1], s[c][j + 2], s[c][j + 3]);
    __syncthreads();
    for (int col = threadIdx.x; col < a.D; col += kRowThreads) {
      float v = sums[col];
      for (int g = 1; g < G; ++g) v += sums[g * width + col];
      a.partial[((int64_t)blockIdx.x * 2 + which) * a.D + col] = v;
    }
    __syncthreads();
  };
  reduce(s_pre, 0);
  if (has_y) reduce(s_y, 1);
}

// Rows of more than 8192 elements: the sums over the rows no longer fit the registers of a block
// and take its shared memory instead; every row is read three times, the second and third time
// from L2.  2000 x 16384 takes 319 us (floor 60); the forward pass, a row in registers with nothing fetched ahead, 87 (40).
constexpr int kWide = 8192;
template <class XT>
__global__ void __launch_bounds__(kRowThreads, 1) mp_block_norm_bwd_wide_kernel(const BwdArgs a) {
  constexpr int TPR = kRowThreads;
  extern __shared__ float wide_sums[];           // the two sums over the rows
  __shared__ float red[rows::red_floats<TPR, 2>];
  int parity = 0;
  const bool has_y = a.g_post != nullptr, matrix = a.gate != nullptr && a.ldgate != 0, layer = a.kind == MP_NORM_LAYER;
  const float inv_d = 1.0f / (float)a.D;
  const XT* x_out = reinterpret_cast<const XT*>(a.x_out);
  const XT* dx_out = reinterpret_cast<const XT*>(a.dx_out);
  for (int c = threadIdx.x; c < 2 * a.D; c += TPR) wide_sums[c] = 0.0f;
  __syncthreads();
  for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x) {
    const float4 st = __ldg(reinterpret_cast<const float4*>(a.stats) + m);
    float sa = 0.0f, sb = 0.0f;
    auto front = [&](int col, int nv, float (&gx)[8], float (&xhat)[8], float (&dn)[8], bool whole) {
      rows::Raw8<XT> xr;
      rows::Raw8<uint16_t> r;
      float g[8], up[8] = {};
      xr.load(x_out + m * a.ldxo + col, nv);
      xr.floats(xhat);
      r.load(a.dn + m * a.lddn + col, nv);
      r.floats(dn);
      r.load_cached(a.g_pre + col, nv);
      r.floats(g);
      if (whole && dx_out != nullptr) {
        xr.load(dx_out + m * a.lddxo + col, nv);
        xr.floats(up);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        xhat[j] = (xhat[j] - st.z) * st.w;
        gx[j] = dn[j] * g[j];
        if (whole) gx[j] = fmaf(gx[j] - fmaf(xhat[j], sa, sb), st.w, up[j]);
      }
    };
    auto behind = [&](int col, int nv, float (&q)[8], float (&yhat)[8], float (&gp)[8], float (&g)[8]) {
      rows::Raw8<uint16_t> r;
      r.load(a.y + m * a.ldy + col, nv);
      r.floats(yhat);
      r.load_cached(a.g_post + col, nv);
      r.floats(gp);
      if (a.gate != nullptr) {
        r.load(a.gate + m * a.ldgate + col, nv);
        r.floats(g);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        yhat[j] = (yhat[j] - st.x) * st.y;
        if (a.gate == nullptr) g[j] = 1.0f;
        q[j] = g[j] * gp[j];
      }
    };
    float gx[8], xhat[8], dn[8], q[8], yhat[8], gp[8], g[8];
    float ab[2] = {0.0f, 0.0f}, ef[2] = {0.0f, 0.0f};
    for (int col = threadIdx.x * 8; col < a.D; col += TPR * 8) {
      front(col, min(8, a.D - col), gx, xhat, dn, false);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        ab[0] = fmaf(gx[j], xhat[j], ab[0]);
        ab[1] += gx[j];
      }
    }
    rows::group_sum<TPR, 2>(ab, red, parity);
    sa = ab[0] * inv_d;
    sb = layer ? ab[1] * inv_d : 0.0f;
    if (has_y) {
      for (int col = threadIdx.x * 8; col < a.D; col += TPR * 8) {
        front(col, min(8, a.D - col), gx, xhat, dn, true);
        behind(col, min(8, a.D - col), q, yhat, gp, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          ef[0] = fmaf(gx[j] * q[j], yhat[j], ef[0]);
          ef[1] = fmaf(gx[j], q[j], ef[1]);
        }
      }
      rows::group_sum<TPR, 2>(ef, red, parity);
    }
    const float se = ef[0] * inv_d, sf = layer ? ef[1] * inv_d : 0.0f;
    for (int col = threadIdx.x * 8; col < a.D; col += TPR * 8) {
      const int nv = min(8, a.D - col);
      front(col, nv, gx, xhat, dn, true);
      float* s = wide_sums + col;
      for (int j = 0; j < nv; ++j) s[j] = fmaf(dn[j], xhat[j], s[j]);
      if (has_y) {
        behind(col, nv, q, yhat, gp, g);
        float dy[8], dg[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          dg[j] = gx[j] * yhat[j] * gp[j];
          dy[j] = (gx[j] * q[j] - fmaf(yhat[j], se, sf)) * st.y;
        }
        for (int j = 0; j < nv; ++j) s[a.D + j] = fmaf(matrix ? gx[j] * g[j] : gx[j], yhat[j], s[a.D + j]);
        if (matrix) rows::store8(a.dgate + m * a.lddgate + col, dg, nv);
        rows::store8(a.dy + m * a.lddy + col, dy, nv);
#pragma unroll
        for (int j = 0; j < 8; ++j) gx[j] *= a.res_scale;
      }
      rows::store8(reinterpret_cast<XT*>(a.dx) + m * a.lddx + col, gx, nv);
    }
  }
  __syncthreads();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  for (int c = threadIdx.x; c < 2 * a.D; c += TPR) a.partial[(int64_t)blockIdx.x * 2 * a.D + c] = wide_sums[c];
}

// Adds the blocks' partial rows in order, rounds, stores and inspects.  A block owns 32 columns of one of
// the two sums; its 32 warps take the slabs in runs of at most five, all of them in flight at once.  gate: the gate
// vector, NULL without one; then the second sum gives dgate too.
constexpr int kSumThreads = 1024;
__global__ void __launch_bounds__(kSumThreads)
mp_block_norm_sum_kernel(const float* partial, int slabs, int D, const uint16_t* g_post, const uint16_t* gate,
                         uint16_t* dg_pre, uint16_t* dg_post, uint16_t* dgate, mp_dev_state* st) {
  __shared__ float sm[kSumThreads / 32][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, which = blockIdx.y;
  const int c = blockIdx.x * 32 + lane;
  const int per = (slabs + 31) / 32, s0 = warp * per, s1 = min(slabs, s0 + per);
  asm volatile("griddepcontrol.wait;" ::: "memory");   // the partial rows are complete and visible
  float v = 0.0f;
  if (c < D)
#pragma unroll 5
    for (int s = s0; s < s1; ++s) v += __ldcg(partial + ((int64_t)s * 2 + which) * D + c);
  sm[warp][lane] = v;
  __syncthreads();
  if (warp != 0) return;
  bool bad = false;
  if (c < D) {
    float v = sm[0][lane];
#pragma unroll
    for (int w = 1; w < kSumThreads / 32; ++w) v += sm[w][lane];
    auto put = [&](uint16_t* out, float x) {
      const uint16_t h = rows::f2h(x);
      out[c] = h;
      bad |= rows::nonfinite16(h);
    };
    if (which == 0) {
      put(dg_pre, v);
    } else if (gate == nullptr) {
      put(dg_post, v);
    } else {
      const float g = rows::h2f(gate[c]), p = rows::h2f(g_post[c]);
      put(dg_post, g * v);
      put(dgate, p * v);
    }
  }
  if (st != nullptr && __any_sync(0xFFFFFFFFu, bad) && lane == 0) atomicOr(&st->h.found_inf, 1);
}

constexpr int64_t kSms = 148;          // most blocks that the backward pass runs, and partial rows that it writes

// Threads per row, two vectors of 8 columns each.
int tpr_for(int64_t D) {
  int tpr = 8;
  while (tpr < 512 && (int64_t)tpr * 16 < D) tpr *= tpr == 8 ? 4 : 2;
  return tpr;
}
int64_t blocks_for(int64_t M, int64_t D) {
  const int64_t per = D > kWide ? 1 : kRowThreads / tpr_for(D);
  const int64_t blocks = (M + per - 1) / per;
  return blocks < 1 ? 1 : blocks < kSms ? blocks : kSms;
}

// Stages of `slots` 16-byte slots per thread that fit the shared memory, 2 to 4 (the slots of a stage are 14 at
// most, 112 KiB, so two always fit).
constexpr size_t kMostSmem = 224 << 10;
// Lets a kernel use that much dynamic shared memory; `allowed` is the kernel's own.
int allow_smem(const void* kernel, mp::PerDevice& allowed) {
  int dev = 0;
  MP_CUDA_TRY(cudaGetDevice(&dev));
  if (allowed.get(dev)) return MP_OK;
  MP_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem));
  allowed.set(dev, 1);
  return MP_OK;
}
size_t stages_for(int slots, int* stages) {
  const size_t stage = (size_t)slots * kRowThreads * 16;
  const int fit = (int)(kMostSmem / stage);
  *stages = fit > 4 ? 4 : fit;
  return *stages * stage;
}

template <class XT, int TPR>
int fwd_launch(FwdArgs a, bool layer, int blocks, cudaStream_t st) {
  static mp::PerDevice allowed[2];
  const int xs = sizeof(XT) / 2;
  a.slots = kC * (xs + (a.g_post ? 1 : 0) + (a.gate && a.ldgate ? 1 : 0));
  const size_t smem = stages_for(a.slots, &a.stages);
  auto kernel = layer ? mp_block_norm_fwd_kernel<XT, TPR, true> : mp_block_norm_fwd_kernel<XT, TPR, false>;
  if (int rc = allow_smem((const void*)kernel, allowed[layer])) return rc;
  kernel<<<blocks, kRowThreads, smem, st>>>(a);
  return MP_OK;
}
template <class XT>
int fwd_dispatch(const FwdArgs& a, bool layer, int blocks, cudaStream_t st) {
  if (a.D > kWide) {
    if (layer) mp_block_norm_fwd_wide_kernel<XT, true><<<blocks, kRowThreads, 0, st>>>(a);
    else mp_block_norm_fwd_wide_kernel<XT, false><<<blocks, kRowThreads, 0, st>>>(a);
    return MP_OK;
  }
  switch (tpr_for(a.D)) {
    case 8: return fwd_launch<XT, 8>(a, layer, blocks, st);
    case 32: return fwd_launch<XT, 32>(a, layer, blocks, st);
    case 64: return fwd_launch<XT, 64>(a, layer, blocks, st);
    case 128: return fwd_launch<XT, 128>(a, layer, blocks, st);
    case 256: return fwd_launch<XT, 256>(a, layer, blocks, st);
    default: return fwd_launch<XT, 512>(a, layer, blocks, st);
  }
}

template <class XT, int TPR>
int bwd_launch(BwdArgs a, int blocks, cudaStream_t st) {
  static mp::PerDevice allowed[4];
  const bool matrix = a.gate != nullptr && a.ldgate != 0, layer = a.kind == MP_NORM_LAYER;
  const int xs = sizeof(XT) / 2;
  a.slots = kC * (xs + (a.dx_out ? xs : 0) + 1 + (a.g_post ? 1 : 0) + (matrix ? 1 : 0));
  size_t smem = stages_for(a.slots, &a.stages);
  const size_t sums = (size_t)kRowThreads * kC * 8 * sizeof(float);
  if (smem < sums) smem = sums;
  auto kernel = layer ? matrix ? mp_block_norm_bwd_kernel<XT, TPR, true, true> : mp_block_norm_bwd_kernel<XT, TPR, true, false>
                      : matrix ? mp_block_norm_bwd_kernel<XT, TPR, false, true> : mp_block_norm_bwd_kernel<XT, TPR, false, false>;
  if (int rc = allow_smem((const void*)kernel, allowed[2 * layer + matrix])) return rc;
  kernel<<<blocks, kRowThreads, smem, st>>>(a);
  return MP_OK;
}
template <class XT>
int bwd_dispatch(const BwdArgs& a, int blocks, cudaStream_t st) {
  if (a.D > kWide) {
    static mp::PerDevice allowed;
    const size_t smem = (size_t)2 * a.D * sizeof(float);
    if (int rc = allow_smem((const void*)mp_block_norm_bwd_wide_kernel<XT>, allowed)) return rc;
    mp_block_norm_bwd_wide_kernel<XT><<<blocks, kRowThreads, smem, st>>>(a);
    return MP_OK;
  }
  switch (tpr_for(a.D)) {
    case 8: return bwd_launch<XT, 8>(a, blocks, st);
    case 32: return bwd_launch<XT, 32>(a, blocks, st);
    case 64: return bwd_launch<XT, 64>(a, blocks, st);
    case 128: return bwd_launch<XT, 128>(a, blocks, st);
    case 256: return bwd_launch<XT, 256>(a, blocks, st);
    default: return bwd_launch<XT, 512>(a, blocks, st);
  }
}

bool bad_ptr16(const void* p) { return p && !mp::aligned16(p); }

}  // namespace

extern "C" {

int mp_block_norm_fwd(int kind, float eps, float res_scale, const void* x, int x_bytes, int64_t ldx,
                      const void* y16, int64_t ldy, const void* g_post16, const void* gate16, int64_t ldgate,
                      void* x_out, int64_t ldxo, const void* g_pre16, void* n16, int64_t ldn, float* stats,
                      int64_t M, int64_t D, void* stream) {
  const char* name = "mp_block_norm_fwd";
  if ((kind != MP_NORM_RMS && kind != MP_NORM_LAYER) || (x_bytes != 2 && x_bytes != 4) || M < 0 || D <= 0 ||
      !(eps >= 0.0f) || ldx < D || ldn < D)
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: bad kind, size, pitch or eps", name);
  if (D > MP_NORM_MAX_D) return mp::set_error(MP_ERR_TOO_LARGE, "%s: D beyond %d", name, MP_NORM_MAX_D);
  if (!g_pre16 || (M > 0 && (!x || !n16))) return mp::set_error(MP_ERR_INVALID_ARG, "%s: null pointer", name);
  if (g_post16 ? ((M > 0 && (!y16 || !x_out)) || ldy < D || ldxo < D || (gate16 && ldgate != 0 && ldgate < D))
               : (y16 || x_out || gate16))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: g_post16 goes with y16 and x_out, without it there is no y16, "
                         "x_out or gate16", name);
  const int64_t xm = x_bytes == 4 ? 3 : 7;
  if ((ldx & xm) || (ldn & 7) || (y16 && ((ldy & 7) || (ldxo & xm))) || (gate16 && (ldgate & 7)) || bad_ptr16(x) ||
      bad_ptr16(y16) || bad_ptr16(g_post16) || bad_ptr16(gate16) || bad_ptr16(x_out) || bad_ptr16(g_pre16) ||
      bad_ptr16(n16) || bad_ptr16(stats))
    return mp::set_error(MP_ERR_ALIGNMENT, "%s: buffers must be 16-byte aligned, rows start on 16-byte boundaries", name);
  if ((x_out && x_out == x && ldxo != ldx) || (n16 && n16 == y16 && ldn != ldy))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: a result in an input's place needs its pitch", name);
  if (int rc = mp::check_device()) return rc;
  if (M == 0) return MP_OK;
  const FwdArgs a{eps, res_scale, x, ldx, (const uint16_t*)y16, ldy, (const uint16_t*)g_post16, (const uint16_t*)gate16,
                  ldgate, x_out, ldxo, (const uint16_t*)g_pre16, (uint16_t*)n16, ldn, stats, M, (int)D, 0, 0};
  const int blocks = (int)blocks_for(M, D);
  cudaStream_t st = (cudaStream_t)stream;
  const bool layer = kind == MP_NORM_LAYER;
  if (int rc = x_bytes == 4 ? fwd_dispatch<float>(a, layer, blocks, st) : fwd_dispatch<uint16_t>(a, layer, blocks, st))
    return rc;
  mp::count_launch();
  MP_CUDA_TRY(cudaGetLastError());
  return MP_OK;
}

size_t mp_block_norm_bwd_workspace_bytes(int64_t M, int64_t D) {
  if (M < 0 || D <= 0 || D > MP_NORM_MAX_D) return 0;
  return (size_t)blocks_for(M, D) * 2 * (size_t)D * sizeof(float);
}

int mp_block_norm_bwd(int kind, float res_scale, const void* dn16, int64_t lddn, const void* dx_out,
                      int64_t lddxo, const void* x_out, int x_bytes, int64_t ldxo, const void* y16, int64_t ldy,
                      const void* g_post16, const void* gate16, int64_t ldgate, const void* g_pre16,
                      const float* stats, void* dx, int64_t lddx, void* dy16, int64_t lddy, void* dg_post16,
                      void* dgate16, int64_t lddgate, void* dg_pre16, int64_t M, int64_t D, mp_state* state,
                      void* workspace, size_t workspace_bytes, void* stream) {
  const char* name = "mp_block_norm_bwd";
  if ((kind != MP_NORM_RMS && kind != MP_NORM_LAYER) || (x_bytes != 2 && x_bytes != 4) || M < 0 || D <= 0 ||
      lddn < D || ldxo < D || lddx < D || (dx_out && lddxo < D))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: bad kind, size or pitch", name);
  if (D > MP_NORM_MAX_D) return mp::set_error(MP_ERR_TOO_LARGE, "%s: D beyond %d", name, MP_NORM_MAX_D);
  if (!g_pre16 || !dg_pre16 || (M > 0 && (!dn16 || !x_out || !stats || !dx)))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: null pointer", name);
  if (g_post16 ? ((M > 0 && (!y16 || !dy16)) || !dg_post16 || ldy < D || lddy < D ||
                  (gate16 != nullptr) != (dgate16 != nullptr) ||
                  (gate16 && ldgate != 0 && (ldgate < D || lddgate < D)))
               : (y16 || dy16 || dg_post16 || gate16 || dgate16))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: g_post16 goes with y16, dy16 and dg_post16, a gate with its gradient", name);
  const int64_t xm = x_bytes == 4 ? 3 : 7;
  if ((lddn & 7) || (ldxo & xm) || (lddx & xm) || (dx_out && (lddxo & xm)) || (y16 && ((ldy & 7) || (lddy & 7))) ||
      (gate16 && ((ldgate & 7) || (ldgate && (lddgate & 7)))) || bad_ptr16(dn16) || bad_ptr16(dx_out) ||
      bad_ptr16(x_out) || bad_ptr16(y16) || bad_ptr16(g_post16) || bad_ptr16(gate16) || bad_ptr16(g_pre16) ||
      bad_ptr16(stats) || bad_ptr16(dx) || bad_ptr16(dy16) || bad_ptr16(dg_post16) || bad_ptr16(dgate16) ||
      bad_ptr16(dg_pre16) || bad_ptr16(workspace))
    return mp::set_error(MP_ERR_ALIGNMENT, "%s: buffers must be 16-byte aligned, rows start on 16-byte boundaries", name);
  if ((dx && ((dx == dx_out && lddx != lddxo) || (dx == x_out && lddx != ldxo))) || (dy16 && ((dy16 == dn16 && lddy != lddn) || (dy16 == y16 && lddy != ldy))) ||
      (dgate16 && dgate16 == gate16 && lddgate != ldgate))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: a result in an input's place needs its pitch", name);
  const size_t need = mp_block_norm_bwd_workspace_bytes(M, D);
  if (!workspace || workspace_bytes < need)
    return mp::set_error(MP_ERR_NOMEM, "%s: workspace of %zu bytes needed", name, need);
  if (int rc = mp::check_device()) return rc;
  const int blocks = (int)blocks_for(M, D);
  cudaStream_t st = (cudaStream_t)stream;
  const BwdArgs a{kind, res_scale, (const uint16_t*)dn16, lddn, dx_out, lddxo, x_out, ldxo, (const uint16_t*)y16, ldy,
                  (const uint16_t*)g_post16, (const uint16_t*)gate16, ldgate, (const uint16_t*)g_pre16, stats, dx, lddx,
                  (uint16_t*)dy16, lddy, (uint16_t*)dgate16, lddgate, M, (int)D, (float*)workspace, 0, 0};
  if (int rc = x_bytes == 4 ? bwd_dispatch<float>(a, blocks, st) : bwd_dispatch<uint16_t>(a, blocks, st)) return rc;
  MP_CUDA_TRY(cudaGetLastError());
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((D + 31) / 32), g_post16 ? 2 : 1, 1);
  cfg.blockDim = dim3(kSumThreads, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute attr;            // resident early, waits on the device for the partial rows
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  MP_CUDA_TRY(cudaLaunchKernelEx(&cfg, mp_block_norm_sum_kernel, (const float*)workspace, blocks, (int)D,
                                 (const uint16_t*)g_post16, ldgate == 0 ? (const uint16_t*)gate16 : nullptr,
                                 (uint16_t*)dg_pre16, (uint16_t*)dg_post16, (uint16_t*)dgate16,
                                 state ? state->dev : (mp_dev_state*)nullptr));
  mp::count_launch(2);
  MP_CUDA_TRY(cudaGetLastError());
  return MP_OK;
}

}  // extern "C"

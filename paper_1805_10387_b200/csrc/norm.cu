// Norms before and after a block, with the block's gate and the residual scale, forward and backward.

#include <map>
#include <mutex>
#include <utility>

#include "rows.cuh"

namespace {

// ---------------------------------------------------------------- forward
//
// A row belongs to a group of TPR threads, each with C vectors of 8 elements, so the row stays in
// registers between the two norms: x and y are read once and x_out and n written once.  8 B an element
// (FP16 residual, shared gate) against some 20 FP32 operations: HBM bounds it.
constexpr int kFwdThreads = 256;

template <class XT, int TPR, int C>
__global__ void __launch_bounds__(TPR > kFwdThreads ? TPR : kFwdThreads)
mp_block_norm_fwd_kernel(int kind, float eps, float res_scale, const XT* x, int64_t ldx, const uint16_t* y, int64_t ldy,
                         const uint16_t* g_post, const uint16_t* gate, int64_t ldgate, XT* x_out, int64_t ldxo,
                         const uint16_t* g_pre, uint16_t* nn, int64_t ldn, float* stats, int64_t M, int D) {
  constexpr int THREADS = TPR > kFwdThreads ? TPR : kFwdThreads, G = THREADS / TPR;
  __shared__ float red_all[G][32];
  const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
  float* red = red_all[group];
  int parity = 0;
  const int64_t m = (int64_t)blockIdx.x * G + group;
  // groups of part of a warp stay until the shuffles are over; larger groups may leave
  const bool live = m < M;
  if (TPR >= 32 && !live) return;
  const float inv_d = 1.0f / (float)D;
  int nv[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int left = D - (c * TPR + t) * 8;
    nv[c] = !live || left < 0 ? 0 : left < 8 ? left : 8;
  }
  rows::Raw8<XT> xr[C];
  rows::Raw8<uint16_t> yr[C];
#pragma unroll
  for (int c = 0; c < C; ++c) xr[c].load(x + m * ldx + (c * TPR + t) * 8, nv[c]);
  // mean and 1/sqrt of a row that `at` gives chunk by chunk
  auto moments = [&](auto at, float& mean, float& root) {
    float s[1] = {0.0f};
    mean = 0.0f;
    if (kind == MP_NORM_LAYER) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float f[8];
        at(c, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[0] += f[j];
      }
      rows::group_sum<TPR, 1>(s, red, parity);
      mean = s[0] * inv_d;
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float f[8];
      at(c, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float v = f[j] - mean;
        if (nv[c] == 8 || j < nv[c]) q[0] = fmaf(v, v, q[0]);
      }
    }
    rows::group_sum<TPR, 1>(q, red, parity);
    root = rsqrtf(fmaf(q[0], inv_d, eps));
  };
  float4 st = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  float xo[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) xr[c].floats(xo[c]);
  if (g_post != nullptr) {
#pragma unroll
    for (int c = 0; c < C; ++c) yr[c].load(y + m * ldy + (c * TPR + t) * 8, nv[c]);
    moments([&](int c, float (&f)[8]) { yr[c].floats(f); }, st.x, st.y);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (nv[c] == 0) continue;
      const int col = (c * TPR + t) * 8;
      rows::Raw8<uint16_t> gr;
      float f[8], gp[8];
      yr[c].floats(f);
      gr.load_cached(g_post + col, nv[c]);
      gr.floats(gp);
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = (f[j] - st.x) * st.y * gp[j];
      if (gate != nullptr) {
        if (ldgate == 0) gr.load_cached(gate + col, nv[c]);
        else gr.load(gate + m * ldgate + col, nv[c]);
        gr.floats(gp);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] *= gp[j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) xo[c][j] = fmaf(res_scale, xo[c][j], f[j]);
      rows::store8(x_out + m * ldxo + col, xo[c], nv[c]);
    }
  }
  moments([&](int c, float (&f)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = xo[c][j];
  }, st.z, st.w);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (nv[c] == 0) continue;
    const int col = (c * TPR + t) * 8;
    rows::Raw8<uint16_t> gr;
    float gq[8];
    gr.load_cached(g_pre + col, nv[c]);
    gr.floats(gq);
#pragma unroll
    for (int j = 0; j < 8; ++j) gq[j] *= (xo[c][j] - st.z) * st.w;
    rows::store8(nn + m * ldn + col, gq, nv[c]);
  }
  if (stats != nullptr && t == 0 && live) reinterpret_cast<float4*>(stats)[m] = st;
}

// ---------------------------------------------------------------- backward
//
// Persistent blocks of 512 threads; a group of TPR threads walks the rows r, r + step, ...  Each
// thread fetches its own vectors of the next rows (x_out, y, dn, dx_out, a gate matrix) into its
// own slots of shared memory with asynchronous copies, so the loads of the following rows are in
// flight while a row is worked on, and no thread waits for another's copy.  The sums over the rows
// (dg_pre, dg_post, dgate) stay in the registers of the thread that owns the columns; at the end
// the groups of a block add theirs in order through shared memory and the block writes one partial row.
constexpr int kBwdThreads = 512;

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copy_wait(int stages) {     // all but the newest stages - 1 groups are complete
  if (stages == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else if (stages == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else asm volatile("cp.async.wait_group 3;" ::: "memory");
}

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
  float* partial;
  int stages;      // rows in flight per group, the one at work included (2 .. 4)
  int slots;       // 16-byte slots per thread and stage
};

template <class XT, int TPR, int C>
__global__ void __launch_bounds__(kBwdThreads, 1) mp_block_norm_bwd_kernel(const BwdArgs a) {
  constexpr int G = kBwdThreads / TPR, XS = sizeof(XT) / 2;      // XS: slots of one vector of the residual type
  extern __shared__ uint4 slots[];
  __shared__ float red_all[G][2 * 16 * 2];
  const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
  float* red = red_all[group];
  int parity = 0;
  const bool has_y = a.g_post != nullptr, matrix = a.gate != nullptr && a.ldgate != 0, layer = a.kind == MP_NORM_LAYER;
  const float inv_d = 1.0f / (float)a.D;
  const XT* x_out = reinterpret_cast<const XT*>(a.x_out);
  const XT* dx_out = reinterpret_cast<const XT*>(a.dx_out);
  int nv[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int left = a.D - (c * TPR + t) * 8;
    nv[c] = left < 0 ? 0 : left < 8 ? left : 8;
  }
  const int64_t step = (int64_t)gridDim.x * G, first = (int64_t)blockIdx.x * G + group;
  // the row that decides when the loop ends: that of the warp's first group, so that a warp stays whole
  const int64_t lead = TPR >= 32 ? first : (int64_t)blockIdx.x * G + (threadIdx.x & ~31) / TPR;
  const uint32_t base = static_cast<uint32_t>(__cvta_generic_to_shared(slots)) + threadIdx.x * 16;
  // slot order of a vector c: x_out (XS), dx_out (XS), dn, y, gate; slot s of a stage lies at s * threads
  auto fetch = [&](int64_t m, int stage) {
    if (m < a.M) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = (c * TPR + t) * 8;
        uint32_t at = base + (uint32_t)(stage * a.slots + c * (a.slots / C)) * (kBwdThreads * 16);
        auto next = [&] { const uint32_t r = at; at += kBwdThreads * 16; return r; };
#pragma unroll
        for (int h = 0; h < XS; ++h) copy16(next(), x_out + m * a.ldxo + col + 4 * h, nv[c] > 4 * h);
        if (dx_out != nullptr)
#pragma unroll
          for (int h = 0; h < XS; ++h) copy16(next(), dx_out + m * a.lddxo + col + 4 * h, nv[c] > 4 * h);
        copy16(next(), a.dn + m * a.lddn + col, nv[c] > 0);
        if (has_y) copy16(next(), a.y + m * a.ldy + col, nv[c] > 0);
        if (matrix) copy16(next(), a.gate + m * a.ldgate + col, nv[c] > 0);
      }
    }
    copy_commit();
  };
  float s_pre[C][8] = {}, s_post[C][8] = {}, s_gate[C][8] = {};
  for (int s = 0; s + 1 < a.stages; ++s) fetch(first + s * step, s);
  int stage = 0;
  int64_t m = first;
  for (int64_t lm = lead; lm < a.M; lm += step, m += step) {
    const bool live = TPR >= 32 || m < a.M;
    // the slots of the row before this one are free: fetch into them
    fetch(m + (a.stages - 1) * step, stage == 0 ? a.stages - 1 : stage - 1);
    copy_wait(a.stages);
    const float4 st = live ? __ldg(reinterpret_cast<const float4*>(a.stats) + m) : make_float4(0, 0, 0, 0);
    int nvr[C];
#pragma unroll
    for (int c = 0; c < C; ++c) nvr[c] = live ? nv[c] : 0;
    float gx[C][8], xhat[C][8], dn[C][8];
    float ab[2] = {0.0f, 0.0f};
    const uint4* mine = slots + threadIdx.x + (int64_t)stage * a.slots * kBwdThreads;
    auto raw16 = [&](int c, int slot) {
      rows::Raw8<uint16_t> r;
      r.q = mine[(c * (a.slots / C) + slot) * kBwdThreads];
      r.keep(nvr[c]);
      return r;
    };
    auto rawx = [&](int c, int slot) {
      rows::Raw8<XT> r;
      uint4* q = reinterpret_cast<uint4*>(&r);
#pragma unroll
      for (int h = 0; h < XS; ++h) q[h] = mine[(c * (a.slots / C) + slot + h) * kBwdThreads];
      r.keep(nvr[c]);
      return r;
    };
    const int s_dn = dx_out != nullptr ? 2 * XS : XS;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float g[8];
      rows::Raw8<uint16_t> gr;
      rawx(c, 0).floats(xhat[c]);
      raw16(c, s_dn).floats(dn[c]);
      gr.load_cached(a.g_pre + (c * TPR + t) * 8, nv[c]);
      gr.floats(g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        xhat[c][j] = (xhat[c][j] - st.z) * st.w;
        const float d = dn[c][j] * g[j];
        gx[c][j] = d;
        ab[0] = fmaf(d, xhat[c][j], ab[0]);
        ab[1] += d;
      }
    }
    rows::group_sum<TPR, 2>(ab, red, parity);
    const float sa = ab[0] * inv_d, sb = layer ? ab[1] * inv_d : 0.0f;
    float ef[2] = {0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (nvr[c] == 0) continue;
      float up[8] = {};
      if (dx_out != nullptr) rawx(c, XS).floats(up);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        s_pre[c][j] = fmaf(dn[c][j], xhat[c][j], s_pre[c][j]);
        gx[c][j] = fmaf(gx[c][j] - fmaf(xhat[c][j], sa, sb), st.w, up[j]);
        up[j] = has_y ? a.res_scale * gx[c][j] : gx[c][j];
      }
      rows::store8(reinterpret_cast<XT*>(a.dx) + m * a.lddx + (c * TPR + t) * 8, up, nvr[c]);
    }
    if (has_y) {
      // from here on xhat holds yhat, and dn the product gate * g_post
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = (c * TPR + t) * 8;
        float g[8], gp[8];
        rows::Raw8<uint16_t> gr;
        raw16(c, s_dn + 1).floats(xhat[c]);
        gr.load_cached(a.g_post + col, nvr[c]);
        gr.floats(gp);
        if (a.gate != nullptr) {
          if (matrix) gr = raw16(c, s_dn + 2);
          else gr.load_cached(a.gate + col, nvr[c]);
          gr.floats(g);
          float dg[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            xhat[c][j] = (xhat[c][j] - st.x) * st.y;
            const float gy = gx[c][j] * xhat[c][j];
            dg[j] = gy * gp[j];
            s_post[c][j] = fmaf(gy, g[j], s_post[c][j]);
            dn[c][j] = g[j] * gp[j];
          }
          if (matrix) rows::store8(a.dgate + m * a.lddgate + col, dg, nvr[c]);
          else if (nvr[c] != 0)
#pragma unroll
            for (int j = 0; j < 8; ++j) s_gate[c][j] += dg[j];
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            xhat[c][j] = (xhat[c][j] - st.x) * st.y;
            s_post[c][j] = fmaf(gx[c][j], xhat[c][j], s_post[c][j]);
            dn[c][j] = gp[j];
          }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float d = gx[c][j] * dn[c][j];
          ef[0] = fmaf(d, xhat[c][j], ef[0]);
          ef[1] += d;
          gx[c][j] = d;
        }
      }
      rows::group_sum<TPR, 2>(ef, red, parity);
      const float se = ef[0] * inv_d, sf = layer ? ef[1] * inv_d : 0.0f;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        if (nvr[c] == 0) continue;
#pragma unroll
        for (int j = 0; j < 8; ++j) gx[c][j] = (gx[c][j] - fmaf(xhat[c][j], se, sf)) * st.y;
        rows::store8(a.dy + m * a.lddy + (c * TPR + t) * 8, gx[c], nvr[c]);
      }
    }
    stage = stage + 1 == a.stages ? 0 : stage + 1;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();                               // the slots become the groups' sums
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  float* sums = reinterpret_cast<float*>(slots);                 // [group][D rounded up to whole vectors]
  const int width = C * TPR * 8;
  auto reduce = [&](float (&s)[C][8], int which) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int j = 0; j < 8; j += 4)
        *reinterpret_cast<float4*>(sums + group * width + (c * TPR + t) * 8 + j) =
            make_float4(s[c][j], s[c][j + 1], s[c][j + 2], s[c][j + 3]);
    __syncthreads();
    for (int col = threadIdx.x; col < a.D; col += kBwdThreads) {
      float v = sums[col];
      for (int g = 1; g < G; ++g) v += sums[g * width + col];
      a.partial[((int64_t)blockIdx.x * 3 + which) * a.D + col] = v;
    }
    __syncthreads();
  };
  reduce(s_pre, 0);
  if (has_y) reduce(s_post, 1);
  if (has_y && a.gate != nullptr && !matrix) reduce(s_gate, 2);
}

// Rows of more than 8192 elements: the sums over the rows no longer fit the registers of a block
// and take its shared memory instead; every row is read three times, the second and third time
// from L2.
constexpr int kWide = 8192;
template <class XT>
__global__ void __launch_bounds__(kBwdThreads, 1) mp_block_norm_bwd_wide_kernel(const BwdArgs a) {
  constexpr int TPR = kBwdThreads;
  extern __shared__ float wide_sums[];           // dg_pre, dg_post, dgate
  __shared__ float red[2 * 16 * 2];
  int parity = 0;
  const bool has_y = a.g_post != nullptr, matrix = a.gate != nullptr && a.ldgate != 0, layer = a.kind == MP_NORM_LAYER;
  const float inv_d = 1.0f / (float)a.D;
  const XT* x_out = reinterpret_cast<const XT*>(a.x_out);
  const XT* dx_out = reinterpret_cast<const XT*>(a.dx_out);
  for (int c = threadIdx.x; c < 3 * a.D; c += TPR) wide_sums[c] = 0.0f;
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
        for (int j = 0; j < nv; ++j) s[a.D + j] = fmaf(gx[j] * g[j], yhat[j], s[a.D + j]);
        if (matrix) rows::store8(a.dgate + m * a.lddgate + col, dg, nv);
        else
          for (int j = 0; j < nv; ++j) s[2 * a.D + j] += dg[j];
        rows::store8(a.dy + m * a.lddy + col, dy, nv);
#pragma unroll
        for (int j = 0; j < 8; ++j) gx[j] *= a.res_scale;
      }
      rows::store8(reinterpret_cast<XT*>(a.dx) + m * a.lddx + col, gx, nv);
    }
  }
  __syncthreads();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  for (int c = threadIdx.x; c < 3 * a.D; c += TPR) a.partial[(int64_t)blockIdx.x * 3 * a.D + c] = wide_sums[c];
}

// Adds the blocks' partial rows in order, rounds, stores and inspects.  A block owns 32 columns of
// one of the three sums; its 8 warps take the slabs in eight runs, each with several loads in flight.
constexpr int kSumThreads = 256;
__global__ void __launch_bounds__(kSumThreads)
mp_block_norm_sum_kernel(const float* partial, int slabs, int D, uint16_t* dg_pre, uint16_t* dg_post, uint16_t* dgate,
                         mp_dev_state* st) {
  __shared__ float sm[kSumThreads / 32][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, which = blockIdx.y;
  uint16_t* out = which == 0 ? dg_pre : which == 1 ? dg_post : dgate;
  const int c = blockIdx.x * 32 + lane;
  const int per = (slabs + 7) / 8, s0 = warp * per, s1 = min(slabs, s0 + per);
  asm volatile("griddepcontrol.wait;" ::: "memory");   // the partial rows are complete and visible
  if (out == nullptr) return;
  float v = 0.0f;
  if (c < D)
#pragma unroll 8
    for (int s = s0; s < s1; ++s) v += partial[((int64_t)s * 3 + which) * D + c];
  sm[warp][lane] = v;
  __syncthreads();
  if (warp != 0) return;
  bool bad = false;
  if (c < D) {
    float v = sm[0][lane];
#pragma unroll
    for (int w = 1; w < kSumThreads / 32; ++w) v += sm[w][lane];
    const uint16_t h = rows::f2h(v);
    out[c] = h;
    bad = rows::nonfinite16(h);
  }
  if (st != nullptr && __any_sync(0xFFFFFFFFu, bad) && lane == 0) atomicOr(&st->h.found_inf, 1);
}

constexpr int64_t kSms = 148;          // most blocks that the backward pass runs, and partial rows that it writes

// Threads per row of the backward kernels (2 vectors each) and of the forward kernels (1 to 4).
int bwd_tpr(int64_t D) {
  int tpr = 8;
  while (tpr < 512 && (int64_t)tpr * 16 < D) tpr *= 2;
  return tpr;
}
int64_t bwd_blocks(int64_t M, int64_t D) {
  const int64_t per = D > kWide ? 1 : kBwdThreads / bwd_tpr(D);
  const int64_t blocks = (M + per - 1) / per;
  return blocks < 1 ? 1 : blocks < kSms ? blocks : kSms;
}

// Lets a kernel use `bytes` of dynamic shared memory; asked of the runtime once per device and kernel.
int allow_smem(const void* kernel, size_t bytes) {
  static std::mutex mu;
  static std::map<std::pair<int, const void*>, size_t> allowed;
  int dev = 0;
  MP_CUDA_TRY(cudaGetDevice(&dev));
  std::lock_guard<std::mutex> lock(mu);
  size_t& have = allowed[{dev, kernel}];
  if (have >= bytes) return MP_OK;
  MP_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
  have = bytes;
  return MP_OK;
}

struct FwdCall {
  int kind;
  float eps, res_scale;
  const void* x; int64_t ldx;
  const void* y; int64_t ldy;
  const void *g_post, *gate; int64_t ldgate;
  void* x_out; int64_t ldxo;
  const void* g_pre;
  void* n; int64_t ldn;
  float* stats;
  int64_t M, D;
};

template <class XT, int TPR, int C>
void fwd_launch(const FwdCall& f, cudaStream_t st) {
  constexpr int THREADS = TPR > kFwdThreads ? TPR : kFwdThreads, G = THREADS / TPR;
  mp_block_norm_fwd_kernel<XT, TPR, C><<<(unsigned)((f.M + G - 1) / G), THREADS, 0, st>>>(
      f.kind, f.eps, f.res_scale, (const XT*)f.x, f.ldx, (const uint16_t*)f.y, f.ldy, (const uint16_t*)f.g_post,
      (const uint16_t*)f.gate, f.ldgate, (XT*)f.x_out, f.ldxo, (const uint16_t*)f.g_pre, (uint16_t*)f.n, f.ldn,
      f.stats, f.M, (int)f.D);
}
template <class XT>
void fwd_dispatch(const FwdCall& f, cudaStream_t st) {
  if (f.D <= 128) fwd_launch<XT, 8, 2>(f, st);
  else if (f.D <= 256) fwd_launch<XT, 16, 2>(f, st);
  else if (f.D <= 512) fwd_launch<XT, 32, 2>(f, st);
  else if (f.D <= 1024) fwd_launch<XT, 32, 4>(f, st);
  else if (f.D <= 2048) fwd_launch<XT, 64, 4>(f, st);
  else if (f.D <= 4096) fwd_launch<XT, 128, 4>(f, st);
  else if (f.D <= 8192) fwd_launch<XT, 256, 4>(f, st);
  else fwd_launch<XT, 512, 4>(f, st);
}

template <class XT, int TPR>
int bwd_launch(BwdArgs a, int blocks, cudaStream_t st) {
  constexpr int C = 2;
  const bool has_y = a.g_post != nullptr, matrix = a.gate != nullptr && a.ldgate != 0;
  const int xs = sizeof(XT) / 2;
  a.slots = C * (xs + (a.dx_out ? xs : 0) + 1 + (has_y ? 1 : 0) + (matrix ? 1 : 0));
  const size_t stage = (size_t)a.slots * kBwdThreads * 16, most = 224 << 10;
  a.stages = (int)(most / stage);
  a.stages = a.stages > 4 ? 4 : a.stages;        // slots are 14 at most: 112 KiB a stage, so two always fit
  size_t smem = a.stages * stage;
  const size_t sums = (size_t)kBwdThreads * C * 8 * sizeof(float);
  if (smem < sums) smem = sums;
  auto kernel = mp_block_norm_bwd_kernel<XT, TPR, C>;
  if (int rc = allow_smem((const void*)kernel, most)) return rc;
  kernel<<<blocks, kBwdThreads, smem, st>>>(a);
  return MP_OK;
}
template <class XT>
int bwd_dispatch(const BwdArgs& a, int blocks, cudaStream_t st) {
  if (a.D > kWide) {
    const size_t smem = (size_t)3 * a.D * sizeof(float);
    if (int rc = allow_smem((const void*)mp_block_norm_bwd_wide_kernel<XT>, smem)) return rc;
    mp_block_norm_bwd_wide_kernel<XT><<<blocks, kBwdThreads, smem, st>>>(a);
    return MP_OK;
  }
  switch (bwd_tpr(a.D)) {
    case 8: return bwd_launch<XT, 8>(a, blocks, st);
    case 16: return bwd_launch<XT, 16>(a, blocks, st);
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
  if (int rc = mp::check_device()) return rc;
  if (M == 0) return MP_OK;
  const FwdCall f{kind, eps, res_scale, x, ldx, y16, ldy, g_post16, gate16, ldgate, x_out, ldxo, g_pre16, n16, ldn, stats, M, D};
  if (x_bytes == 4) fwd_dispatch<float>(f, (cudaStream_t)stream);
  else fwd_dispatch<uint16_t>(f, (cudaStream_t)stream);
  mp::count_launch();
  MP_CUDA_TRY(cudaGetLastError());
  return MP_OK;
}

size_t mp_block_norm_bwd_workspace_bytes(int64_t M, int64_t D) {
  if (M < 0 || D <= 0 || D > MP_NORM_MAX_D) return 0;
  return (size_t)bwd_blocks(M, D) * 3 * (size_t)D * sizeof(float);
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
  const size_t need = mp_block_norm_bwd_workspace_bytes(M, D);
  if (!workspace || workspace_bytes < need)
    return mp::set_error(MP_ERR_NOMEM, "%s: workspace of %zu bytes needed", name, need);
  if (int rc = mp::check_device()) return rc;
  const int blocks = (int)bwd_blocks(M, D);
  cudaStream_t st = (cudaStream_t)stream;
  const BwdArgs a{kind, res_scale, (const uint16_t*)dn16, lddn, dx_out, lddxo, x_out, ldxo, (const uint16_t*)y16, ldy,
                  (const uint16_t*)g_post16, (const uint16_t*)gate16, ldgate, (const uint16_t*)g_pre16, stats, dx, lddx,
                  (uint16_t*)dy16, lddy, (uint16_t*)dgate16, lddgate, M, (int)D, (float*)workspace, 0, 0};
  if (int rc = x_bytes == 4 ? bwd_dispatch<float>(a, blocks, st) : bwd_dispatch<uint16_t>(a, blocks, st)) return rc;
  MP_CUDA_TRY(cudaGetLastError());
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((D + 31) / 32), g_post16 ? 3 : 1, 1);
  cfg.blockDim = dim3(kSumThreads, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute attr;            // resident early, waits on the device for the partial rows
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  MP_CUDA_TRY(cudaLaunchKernelEx(&cfg, mp_block_norm_sum_kernel, (const float*)workspace, blocks, (int)D,
                                 (uint16_t*)dg_pre16, (uint16_t*)dg_post16, ldgate == 0 ? (uint16_t*)dgate16 : nullptr,
                                 state ? state->dev : (mp_dev_state*)nullptr));
  mp::count_launch(2);
  MP_CUDA_TRY(cudaGetLastError());
  return MP_OK;
}

}  // extern "C"

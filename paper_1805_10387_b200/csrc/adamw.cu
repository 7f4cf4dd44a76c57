// AdamW over the tensors of a plan, states in 32 or in 8 bits, on the FP32 master.
//
// As in the Adam update beside it every operation is one individually rounded FP32 operation, so the
// result does not depend on what the compiler would contract.  With 8-bit states, where the kernel moves
// 16 B a parameter and instructions weigh as much as memory, that holds for the moments alone: an E4M3 code
// may turn on their last bit.  The quotient of the step is taken from the hardware's approximation: off by about 2^-22
// of the step, so by a few units in the last place of the weight where the step is most of it (a weight at zero), and
// by less than half a unit where the step is a quarter of the weight or less.
//
// 28 B a parameter with 32-bit states, 16 B and two scales for each 256 parameters with 8-bit ones: HBM bounds both.
// Measured on B200s, 1e8 parameters: 32 bits 457 - 468 us (6.0 - 6.1 TB/s), 8 bits 324 - 350 us in one tensor or 500 (4.6 -
// 5.0 TB/s; leaving out the root, the quotient and the codes changes that by 2 %).  What was tried: asynchronous copies into
// shared memory two or three blocks ahead (32 bits 530, 8 bits 420 us), four blocks of threads an SM instead of
// three (8 bits 409), two (401).

#include <cuda_fp8.h>
#include <math.h>
#include <string.h>

#include <new>
#include <vector>

#include "rows.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kBlock = MP_ADAMW_BLOCK;          // elements of one scale of the 8-bit states
constexpr float kTop = 448.0f;                  // largest E4M3 number
constexpr float kTiny = 0.001953125f;           // smallest E4M3 number above 0, 2^-9
constexpr float kNoScale = 7.888609052210118e-31f;   // 2^-100

// A tensor of the plan.  Blocks of all tensors are numbered through, each tensor beginning at a multiple of
// kMostUnit; the addresses are those that the tensors' buffers would have if they began at block 0, so that
// block x lies at address + x * (bytes of a block).
constexpr int kMostUnit = 8;
struct alignas(16) Tensor {
  uint64_t g16, w32, m, v, w16, m_scale, v_scale;
  int64_t end;                                  // first block * 256 + elements
  int64_t block_end;                            // number of the first block after it
  float decay;
};
struct Coef {
  float inv_s, b1, omb1, b2, omb2, decay, alpha, k2, eps;
};

// b^t by squaring, in FP64: an error of some 2 log2(t) units in the last place, and a fraction of pow's latency,
// which every block would wait for.
__device__ __forceinline__ double power(double b, int64_t t) {
  double r = 1.0;
  for (; t > 0; t >>= 1, b *= b)
    if (t & 1) r *= b;
  return r;
}
__device__ __forceinline__ Coef coefficients(const mp_dev_state* st, const mp_adamw_config& o) {
  const int64_t t = st->h.t + 1;
  const double c1 = 1.0 - power(o.beta1, t), c2 = 1.0 - power(o.beta2, t);
  Coef c;
  c.inv_s = __fdiv_rn(1.0f, st->h.scale);
  c.b1 = (float)o.beta1;
  c.omb1 = (float)(1.0 - o.beta1);
  c.b2 = (float)o.beta2;
  c.omb2 = (float)(1.0 - o.beta2);
  c.decay = (float)(o.lr * o.weight_decay);
  c.alpha = (float)(o.lr / c1);
  c.k2 = (float)(1.0 / sqrt(c2));
  c.eps = (float)o.eps;
  return c;
}

__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// One element: m and v in, m, v and r = sqrt(v) out; w is stepped.  decay: lr weight_decay of the tensor.
template <int BITS>
__device__ __forceinline__ void step_one(float g16f, float& w, float& m, float& v, float& r, float decay, const Coef& c) {
  const float g = __fmul_rn(g16f, c.inv_s);
  m = __fadd_rn(__fmul_rn(c.b1, m), __fmul_rn(c.omb1, g));
  v = __fadd_rn(__fmul_rn(c.b2, v), __fmul_rn(c.omb2, __fmul_rn(g, g)));
  r = __fsqrt_rn(v);
  if constexpr (BITS == 32) {
    w = __fsub_rn(w, __fmul_rn(decay, w));
    w = __fsub_rn(w, __fmul_rn(c.alpha, __fdiv_rn(m, __fadd_rn(__fmul_rn(r, c.k2), c.eps))));
  } else {
    w = fmaf(-decay, w, w);
    w = fmaf(-c.alpha, m * rcp_approx(fmaf(r, c.k2, c.eps)), w);
  }
}

// Eight E4M3 numbers as loaded.
__device__ __forceinline__ void from_e4m3(uint2 q, float (&f)[8]) {
  const uint32_t w[2] = {q.x, q.y};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[j / 2] >> (16 * (j & 1))), __NV_E4M3);
    const float2 x = __half22float2(__half2(h));
    f[2 * j] = x.x;
    f[2 * j + 1] = x.y;
  }
}
__device__ __forceinline__ uint2 to_e4m3(const float (&f)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    w[j] = __nv_cvt_float2_to_fp8x2(make_float2(f[2 * j], f[2 * j + 1]), __NV_SATFINITE, __NV_E4M3);
  return make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
}
// The largest of a warp's non-negative values: their order is that of their bits.
__device__ __forceinline__ float warp_top(float v) {
  return __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(v)));
}

// A warp takes the units w, w + step, ... of the plan, w its number among the step warps of the grid, so that
// neighbouring warps stream neighbouring memory.  A unit is 1, 2, 4 or 8 neighbouring blocks: the 8-bit states'
// scales of a unit are one access of the warp.  (With one 4-byte access a block: 370 us instead of 329.)  A Cursor
// walks a warp's blocks.
struct Cursor {
  const Tensor* tensors;
  int64_t x, hop, n_blocks;                     // hop: from the end of one unit to the beginning of the warp's next
  int unit, at = 0, n_tensors;                  // at: the tensor that holds block x
  __device__ __forceinline__ Cursor(const Tensor* table, int n, int64_t blocks, int unit_blocks)
      : tensors(table), x(((int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * unit_blocks),
        hop(((int64_t)gridDim.x * (kThreads / 32) - 1) * unit_blocks), n_blocks(blocks), unit(unit_blocks), n_tensors(n) {
    if (more()) seek(0, n_tensors - 1);
    settle();
  }
  __device__ __forceinline__ bool more() const { return x < n_blocks; }
  __device__ __forceinline__ void next() {
    ++x;
    if ((x & (unit - 1)) == 0) x += hop;
    settle();
  }
  // finds the tensor, and passes over the numbers that no tensor fills
  __device__ __forceinline__ void settle() {
    while (more()) {
      if (__ldg(&tensors[at].block_end) <= x) forward();
      if (__ldg(&tensors[at].end) > x * kBlock) return;
      x = (x | (unit - 1)) + 1 + hop;
    }
  }
  __device__ __forceinline__ void forward() {   // most often one of the next 32 tensors
    const int lane = threadIdx.x & 31, hi = n_tensors - 1, probe = at + 1 + lane < hi ? at + 1 + lane : hi;
    const unsigned after = __ballot_sync(0xFFFFFFFFu, __ldg(&tensors[probe].block_end) > x);
    if (after) at = at + __ffs(after) < hi ? at + __ffs(after) : hi;
    else seek(at + 33, hi);
  }
  // the first tensor in lo .. hi whose blocks end after x (hi's do): 32 probes at a time
  __device__ __forceinline__ void seek(int lo, int hi) {
    const int lane = threadIdx.x & 31;
    for (;;) {
      const int stride = (hi - lo) / 32 + 1, probe = lo + lane * stride < hi ? lo + lane * stride : hi;
      const unsigned after = __ballot_sync(0xFFFFFFFFu, __ldg(&tensors[probe].block_end) > x);
      const int first = after ? __ffs(after) - 1 : 32;   // lane whose probe is the first that ends after x
      const int top = lo + first * stride;
      if (stride == 1) {
        at = top < hi ? top : hi;
        return;
      }
      hi = top < hi ? top : hi;
      if (first > 0) lo = lo + (first - 1) * stride + 1;
    }
  }
  // how many elements of the block lie inside the tensor
  __device__ __forceinline__ int inside(const Tensor& T) const {
    const int64_t left = __ldg(&T.end) - x * kBlock;
    return left < kBlock ? (int)left : kBlock;
  }
};
// A lane takes two quads of a block.  With 32-bit states they are 128 elements apart, so that each access of
// a warp is one contiguous piece; with 8-bit states they are neighbours, so that a lane's eight codes are one access.
// (1e8 parameters, asynchronous copies: 32 bits 663 us with neighbours, 530 so; 8 bits: no difference beyond 3 %.)
template <int BITS>
__device__ __forceinline__ int quad_at(int h) {
  const int lane = threadIdx.x & 31;
  return BITS == 32 ? lane * 4 + 128 * h : lane * 8 + 4 * h;
}
// Address of quad h (0, 1) of elements of `size` bytes in block x, and how many of its elements are inside.
template <class P, int BITS>
__device__ __forceinline__ P* lane_at(uint64_t base, int64_t x, int size, int h) {
  return reinterpret_cast<P*>(base + x * (kBlock * size) + quad_at<BITS>(h) * size);
}
template <int BITS>
__device__ __forceinline__ int quad(int inside, int h) {
  const int n = inside - quad_at<BITS>(h);
  return n < 0 ? 0 : n < 4 ? n : 4;
}

__global__ void __launch_bounds__(kThreads)
mp_adamw_check_kernel(const Tensor* tensors, int n_tensors, int64_t n_blocks, int unit, mp_dev_state* st) {
  bool bad = false;
  for (Cursor cur(tensors, n_tensors, n_blocks, unit); cur.more(); cur.next()) {
    const Tensor& T = cur.tensors[cur.at];
    const int inside = cur.inside(T);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint16_t* g = lane_at<const uint16_t, 32>(__ldg(&T.g16), cur.x, 2, h);
      const int nv = quad<32>(inside, h);
      auto both = [](uint32_t v) { return (v & 0x7C00u) == 0x7C00u || (v & 0x7C000000u) == 0x7C000000u; };
      if (nv == 4) {
        const uint2 q = __ldcs(reinterpret_cast<const uint2*>(g));
        bad |= both(q.x) || both(q.y);
      } else {
        for (int j = 0; j < nv; ++j) bad |= rows::nonfinite16(g[j]);
      }
    }
  }
  if (bad) atomicOr(&st->h.found_inf, 1);
}

// A warp takes a block of 256, which shares one scale, and finds the block's largest magnitude among its own
// registers: the states are read and written once, in place.  The loads of the warp's next block are
// issued before a block is worked on.
__device__ __forceinline__ float4 get4(const float* p, int nv) {      // zeros for what lies past the tensor's end
  if (nv == 4) return __ldcs(reinterpret_cast<const float4*>(p));
  return make_float4(nv > 0 ? p[0] : 0.0f, nv > 1 ? p[1] : 0.0f, nv > 2 ? p[2] : 0.0f, 0.0f);
}
__device__ __forceinline__ uint2 get4(const uint16_t* p, int nv) {
  if (nv == 4) return __ldcs(reinterpret_cast<const uint2*>(p));
  return make_uint2((nv > 0 ? p[0] : 0u) | (nv > 1 ? p[1] : 0u) << 16, nv > 2 ? p[2] : 0u);
}
__device__ __forceinline__ uint32_t get4(const uint8_t* p, int nv) {
  if (nv == 4) return __ldcs(reinterpret_cast<const uint32_t*>(p));
  return (nv > 0 ? p[0] : 0u) | (nv > 1 ? p[1] : 0u) << 8 | (nv > 2 ? p[2] : 0u) << 16;
}
// What a lane holds of a block's states.
template <int BITS> struct States;
template <> struct States<32> {
  float4 m[2], v[2];
  __device__ __forceinline__ void load(const Tensor& T, int64_t x, int inside, int) {
    const uint64_t pm = __ldg(&T.m), pv = __ldg(&T.v);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      m[h] = get4(lane_at<const float, 32>(pm, x, 4, h), quad<32>(inside, h));
      v[h] = get4(lane_at<const float, 32>(pv, x, 4, h), quad<32>(inside, h));
    }
  }
};
template <> struct States<8> {
  uint2 m, v;
  float ms = 0.0f, vs = 0.0f;                   // lane l: the scales of block l of the unit
  __device__ __forceinline__ void load(const Tensor& T, int64_t x, int inside, int unit) {
    const uint8_t *pm = lane_at<const uint8_t, 8>(__ldg(&T.m), x, 1, 0), *pv = lane_at<const uint8_t, 8>(__ldg(&T.v), x, 1, 0);
    if (inside >= kBlock) {
      m = __ldcs(reinterpret_cast<const uint2*>(pm));
      v = __ldcs(reinterpret_cast<const uint2*>(pv));
    } else {
      m = make_uint2(get4(pm, quad<8>(inside, 0)), get4(pm + 4, quad<8>(inside, 1)));
      v = make_uint2(get4(pv, quad<8>(inside, 0)), get4(pv + 4, quad<8>(inside, 1)));
    }
    const int lane = threadIdx.x & 31;
    if ((x & (unit - 1)) == 0 && lane < unit && (x + lane) * kBlock < __ldg(&T.end)) {
      ms = __ldcs(reinterpret_cast<const float*>(__ldg(&T.m_scale)) + x + lane);
      vs = __ldcs(reinterpret_cast<const float*>(__ldg(&T.v_scale)) + x + lane);
    }
  }
};
template <int BITS>
struct Held {
  uint2 g[2];
  float4 w[2];
  States<BITS> s;
  const Tensor* T;
  int64_t x;
  int inside;
  __device__ __forceinline__ void load(const Cursor& cur) {
    T = cur.tensors + cur.at;
    x = cur.x;
    inside = cur.inside(*T);
    const uint64_t pg = __ldg(&T->g16), pw = __ldg(&T->w32);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      g[h] = get4(lane_at<const uint16_t, BITS>(pg, x, 2, h), quad<BITS>(inside, h));
      w[h] = get4(lane_at<const float, BITS>(pw, x, 4, h), quad<BITS>(inside, h));
    }
    s.load(*T, x, inside, cur.unit);
  }
};
__device__ __forceinline__ void spread(const float4 (&q)[2], float (&f)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    f[4 * h] = q[h].x; f[4 * h + 1] = q[h].y; f[4 * h + 2] = q[h].z; f[4 * h + 3] = q[h].w;
  }
}
__device__ __forceinline__ void put4(float* p, const float* f, int nv) {
  if (nv == 4) __stcs(reinterpret_cast<float4*>(p), make_float4(f[0], f[1], f[2], f[3]));
  else
    for (int j = 0; j < nv; ++j) p[j] = f[j];
}
__device__ __forceinline__ void put4(uint16_t* p, const float* f, int nv) {
  if (nv == 4) __stcs(reinterpret_cast<uint2*>(p), make_uint2(rows::pack2(f[0], f[1]), rows::pack2(f[2], f[3])));
  else
    for (int j = 0; j < nv; ++j) p[j] = rows::f2h(f[j]);
}
__device__ __forceinline__ void put4(uint8_t* p, uint32_t q, int nv) {
  if (nv == 4) __stcs(reinterpret_cast<uint32_t*>(p), q);
  else
    for (int j = 0; j < nv; ++j) p[j] = (uint8_t)(q >> (8 * j));
}

template <int BITS>
__global__ void __launch_bounds__(kThreads, BITS == 32 ? 2 : 3)
mp_adamw_update_kernel(const Tensor* tensors, int n_tensors, int64_t n_blocks, int unit, const mp_dev_state* st,
                       mp_adamw_config o, const int* gemm_status) {
  if (st->h.found_inf != 0 || st->h.status != 0 || *gemm_status != 0) return;
  __shared__ Coef s_c;
  Cursor cur(tensors, n_tensors, n_blocks, unit);
  float new_ms = 0.0f, new_vs = 0.0f;           // lane l: of block l of the unit
  Held<BITS> next;
  if (cur.more()) next.load(cur);
  if (threadIdx.x == kThreads - 1) s_c = coefficients(st, o);
  __syncthreads();
  const Coef c = s_c;
  while (cur.more()) {
    const Held<BITS> held = next;
    cur.next();
    if (cur.more()) next.load(cur);
    const Tensor& T = *held.T;
    const int64_t x = held.x;
    const int inside = held.inside;
    float g[8], w[8], m[8], v[8], r[8];
    rows::Raw8<uint16_t> gr;
    gr.q = make_uint4(held.g[0].x, held.g[0].y, held.g[1].x, held.g[1].y);
    gr.floats(g);
    spread(held.w, w);
    if constexpr (BITS == 32) {
      spread(held.s.m, m);
      spread(held.s.v, v);
    } else {
      from_e4m3(held.s.m, m);
      from_e4m3(held.s.v, r);
      const float ms = __shfl_sync(0xFFFFFFFFu, held.s.ms, (int)x & (unit - 1));
      const float vs = __shfl_sync(0xFFFFFFFFu, held.s.vs, (int)x & (unit - 1));
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        m[j] = __fmul_rn(m[j], ms);
        r[j] = __fmul_rn(r[j], vs);
        v[j] = __fmul_rn(r[j], r[j]);
      }
    }
    const float decay = __fmul_rn(c.decay, __ldg(&T.decay));
#pragma unroll
    for (int j = 0; j < 8; ++j) step_one<BITS>(g[j], w[j], m[j], v[j], r[j], decay, c);
    uint2 mq = make_uint2(0, 0), vq = mq;
    if constexpr (BITS == 8) {
      float tm = 0.0f, tr = 0.0f;               // elements past the tensor's end are zero
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        tm = fmaxf(tm, fabsf(m[j]));
        tr = fmaxf(tr, r[j]);
      }
      tm = warp_top(tm);
      tr = warp_top(tr);
      const float im = tm < kNoScale ? 0.0f : __fmul_rn(__frcp_rn(tm), kTop);
      const float ir = tr < kNoScale ? 0.0f : __fmul_rn(__frcp_rn(tr), kTop);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        m[j] = __fmul_rn(m[j], im);
        r[j] = __fmul_rn(r[j], ir);
        r[j] = r[j] > 0.0f ? fmaxf(r[j], kTiny) : r[j];
      }
      mq = to_e4m3(m);
      vq = to_e4m3(r);
      const int lane = threadIdx.x & 31, of_unit = (int)x & (unit - 1);
      if (lane == of_unit) {
        new_ms = tm < kNoScale ? 0.0f : __fmul_rn(tm, 1.0f / kTop);
        new_vs = tr < kNoScale ? 0.0f : __fmul_rn(tr, 1.0f / kTop);
      }
      if ((of_unit == unit - 1 || (x + 1) * kBlock >= __ldg(&T.end)) && lane <= of_unit) {
        const int64_t first = x - of_unit;
        __stcs(reinterpret_cast<float*>(__ldg(&T.m_scale)) + first + lane, new_ms);
        __stcs(reinterpret_cast<float*>(__ldg(&T.v_scale)) + first + lane, new_vs);
      }
    }
    const uint64_t pw = __ldg(&T.w32), pw16 = __ldg(&T.w16), pm = __ldg(&T.m), pv = __ldg(&T.v);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int nv = quad<BITS>(inside, h);
      put4(lane_at<float, BITS>(pw, x, 4, h), w + 4 * h, nv);
      put4(lane_at<uint16_t, BITS>(pw16, x, 2, h), w + 4 * h, nv);
      if constexpr (BITS == 32) {
        put4(lane_at<float, BITS>(pm, x, 4, h), m + 4 * h, nv);
        put4(lane_at<float, BITS>(pv, x, 4, h), v + 4 * h, nv);
      } else if (inside < kBlock) {
        put4(lane_at<uint8_t, BITS>(pm, x, 1, h), h ? mq.y : mq.x, nv);
        put4(lane_at<uint8_t, BITS>(pv, x, 1, h), h ? vq.y : vq.x, nv);
      } else if (h == 0) {
        __stcs(lane_at<uint2, BITS>(pm, x, 1, 0), mq);
        __stcs(lane_at<uint2, BITS>(pv, x, 1, 0), vq);
      }
    }
  }
}

// Blocks of `kernel` that are resident at once on the current device; `known` is the kernel's own.
int resident_blocks(const void* kernel, mp::PerDevice& known, int* out) {
  int dev = 0;
  MP_CUDA_TRY(cudaGetDevice(&dev));
  *out = known.get(dev);
  if (*out == 0) {
    int sms = 0, per = 0;
    MP_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    MP_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kernel, kThreads, 0));
    *out = sms * (per < 1 ? 1 : per);
    known.set(dev, *out);
  }
  return MP_OK;
}

}  // namespace

struct mp_adamw_plan {
  Tensor* d_tensors;
  int n_tensors;                                // with elements
  int64_t n_blocks;
  int bits;
};

extern "C" {

int mp_adamw_plan_create(int n, void* const* g16, void* const* w32, void* const* m, void* const* v,
                         void* const* w16, const int64_t* count, const float* decay, int state_bits,
                         float* const* m_scale, float* const* v_scale, mp_adamw_plan** out) {
  const char* name = "mp_adamw_plan_create";
  if (n <= 0 || !g16 || !w32 || !m || !v || !w16 || !count || !out)
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: null argument or n <= 0", name);
  if ((state_bits != 32 && state_bits != 8) || (state_bits == 8) != (m_scale != nullptr) ||
      (state_bits == 8) != (v_scale != nullptr))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: states have 32 bits, or 8 bits with scales", name);
  for (int i = 0; i < n; ++i) {
    if (count[i] < 0) return mp::set_error(MP_ERR_INVALID_ARG, "%s: count[%d] < 0", name, i);
    if (decay && !isfinite(decay[i])) return mp::set_error(MP_ERR_INVALID_ARG, "%s: decay[%d] is not finite", name, i);
    if (count[i] == 0) continue;
    if (!g16[i] || !w32[i] || !m[i] || !v[i] || !w16[i] || (state_bits == 8 && (!m_scale[i] || !v_scale[i])))
      return mp::set_error(MP_ERR_INVALID_ARG, "%s: tensor %d has a null buffer", name, i);
    if (!mp::aligned16(g16[i]) || !mp::aligned16(w32[i]) || !mp::aligned16(m[i]) || !mp::aligned16(v[i]) ||
        !mp::aligned16(w16[i]) ||
        (state_bits == 8 && (((uintptr_t)m_scale[i] | (uintptr_t)v_scale[i]) & 3)))
      return mp::set_error(MP_ERR_ALIGNMENT, "%s: tensor %d is not 16-byte aligned (scales: 4)", name, i);
  }
  if (int rc = mp::check_device()) return rc;
  mp_adamw_plan* p = new (std::nothrow) mp_adamw_plan();
  if (!p) return mp::set_error(MP_ERR_NOMEM, "%s: host allocation failed", name);
  p->bits = state_bits;
  try {
    std::vector<Tensor> ts;
    for (int i = 0; i < n; ++i) {                // a tensor without elements has no place in the table
      if (count[i] == 0) continue;
      const int64_t first = p->n_blocks;
      p->n_blocks += (count[i] + kBlock * kMostUnit - 1) / (kBlock * kMostUnit) * kMostUnit;
      auto from_block_0 = [&](const void* q, int64_t block_bytes) { return (uint64_t)q - (uint64_t)(first * block_bytes); };
      const int64_t state = state_bits == 32 ? 4 * kBlock : kBlock;
      ts.push_back(Tensor{from_block_0(g16[i], 2 * kBlock), from_block_0(w32[i], 4 * kBlock), from_block_0(m[i], state),
                          from_block_0(v[i], state), from_block_0(w16[i], 2 * kBlock),
                          m_scale ? from_block_0(m_scale[i], 4) : 0, v_scale ? from_block_0(v_scale[i], 4) : 0,
                          first * kBlock + count[i], p->n_blocks, decay ? decay[i] : 1.0f});
    }
    p->n_tensors = (int)ts.size();
    const size_t bytes = ts.size() * sizeof(Tensor);
    if (cudaMalloc(&p->d_tensors, bytes ? bytes : 1) != cudaSuccess) {
      mp_adamw_plan_destroy(p);
      return mp::set_error(MP_ERR_NOMEM, "%s: device allocation failed", name);
    }
    cudaError_t e = bytes ? cudaMemcpy(p->d_tensors, ts.data(), bytes, cudaMemcpyHostToDevice) : cudaSuccess;
    if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);     // a pageable copy may return before it has arrived
    if (e != cudaSuccess) {
      mp_adamw_plan_destroy(p);
      return mp::set_error(MP_ERR_CUDA, "%s: %s", name, cudaGetErrorString(e));
    }
  } catch (const std::bad_alloc&) {
    mp_adamw_plan_destroy(p);
    return mp::set_error(MP_ERR_NOMEM, "%s: host allocation failed", name);
  }
  *out = p;
  return MP_OK;
}

int mp_adamw_plan_destroy(mp_adamw_plan* p) {
  if (!p) return MP_OK;
  cudaFree(p->d_tensors);
  delete p;
  return MP_OK;
}

int mp_adamw_update(mp_adamw_plan* plan, mp_state* state, const mp_adamw_config* opt, int check_mode, void* stream) {
  if (!plan || !state || !opt) return mp::set_error(MP_ERR_INVALID_ARG, "mp_adamw_update: null argument");
  if (check_mode != 0 && check_mode != 1)
    return mp::set_error(MP_ERR_INVALID_ARG, "mp_adamw_update: check_mode must be 0 or 1");
  if (int rc = mp::check_device()) return rc;
  if (plan->n_blocks == 0) return MP_OK;
  cudaStream_t st = (cudaStream_t)stream;
  int* gemm_status = nullptr;
  if (int rc = mp::gemm_status_device_ptr(&gemm_status)) return rc;
  // One resident round of blocks; units as large as leaves every warp four.
  static mp::PerDevice known[3];
  auto shape = [&](const void* kernel, mp::PerDevice& of_kernel, int most_unit, int* grid, int* unit) {
    if (int rc = resident_blocks(kernel, of_kernel, grid)) return rc;
    const int64_t warps = (int64_t)*grid * (kThreads / 32);
    *unit = most_unit;
    while (*unit > 1 && plan->n_blocks < 4 * warps * *unit) *unit /= 2;
    const int64_t want = (plan->n_blocks / *unit + kThreads / 32 - 1) / (kThreads / 32);
    if (want < *grid) *grid = (int)want;
    return (int)MP_OK;
  };
  int grid = 0, unit = 0;
  if (check_mode == 1) {
    if (int rc = shape((const void*)mp_adamw_check_kernel, known[0], 1, &grid, &unit)) return rc;
    mp_adamw_check_kernel<<<grid, kThreads, 0, st>>>(plan->d_tensors, plan->n_tensors, plan->n_blocks, unit, state->dev);
    mp::count_launch();
  }
  auto kernel = plan->bits == 32 ? mp_adamw_update_kernel<32> : mp_adamw_update_kernel<8>;
  if (int rc = shape((const void*)kernel, known[plan->bits == 32 ? 1 : 2], plan->bits == 32 ? 1 : kMostUnit, &grid, &unit)) return rc;
  kernel<<<grid, kThreads, 0, st>>>(plan->d_tensors, plan->n_tensors, plan->n_blocks, unit, state->dev, *opt, gemm_status);
  mp::count_launch();
  MP_CUDA_TRY(cudaGetLastError());
  return MP_OK;
}

}  // extern "C"

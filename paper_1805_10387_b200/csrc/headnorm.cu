// Norms of queries and keys for each head, with the position rotation in the same pass, forward and backward.
//
// A row of the projection's output is heads of D elements; each is divided by its root mean square, multiplied by a
// gain (one for the queries, one for the keys) and rotated pair by pair by the token's position.  One read and one
// write of the heads (backward: two reads and a write).  6387 tokens x 30 heads of 128: 28 us, where the bytes alone take
// 15; 8192 x 32 heads of 64 backward, with the gains' gradients: 37 us, the bytes 15.  What bounds it is issue: 6.7 of ten
// slots are used forward, 5.6 backward, where two blocks an SM are all that the gains' sums leave registers for.
// Angles formed by each lane for itself, in blocks of a few tokens each, took 35 us and 46; loads of the next round ahead of this
// one's work were no faster: other warps cover them.
// L lanes share a head, 8 elements each, so 32 / L heads are worked on by a warp at a time ("a round"); a warp keeps one
// token's angles for all its rounds, since all heads of a token turn alike: each lane forms a few, through shared memory every
// lane gets those of its columns.  Persistent blocks.
// Angles: a position times a frequency, in turns, is a 64-bit fixed-point product whose whole turns fall off the top: the
// fraction stays exact to 2^-53 of a turn times the position, where an FP32 product has lost a whole radian at 2^24.

#include <math.h>

#include "ptx.cuh"
#include "rows.cuh"

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kRounds = 4;                        // whose loads are in flight together
constexpr int kMaxBlocks = 148 * 2;               // of the backward kernel: as many as are resident; rows of its partial sums

struct HeadArgs {
  const uint16_t *x, *dy, *gq, *gk;
  int64_t ldx, lddy;
  const void* pos;
  int pos_bytes;
  const double* freqs;
  uint16_t* out;
  int64_t ldo;
  int64_t T;
  int hq, hk, D, rot, parts;
  float eps;
  float* part;                                    // [blocks][2][D]
};

// cos and sin for the 8 columns of a lane: of each column's pair, or (PAIRS) of its four pairs.
template <bool PAIRS>
struct Turn {
  static constexpr int N = PAIRS ? 4 : 8;
  float c[N], s[N];
  // From the token's angles at `table`, of which this lane's begin at `first`.
  __device__ __forceinline__ void load(const float2* table, int first) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float4 v = *reinterpret_cast<const float4*>(table + first + i);
      c[i] = v.x;
      s[i] = v.y;
      c[i + 1] = v.z;
      s[i + 1] = v.w;
    }
  }
  // Rotates a lane's 8 columns; `partner`: the lane with the other halves of its pairs, `sign`: -1 in the first halves.
  __device__ __forceinline__ void apply(float (&v)[8], int partner, float sign) const {
    if constexpr (PAIRS) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p = v[2 * i], q = v[2 * i + 1];
        v[2 * i] = fmaf(p, c[i], -(q * s[i]));
        v[2 * i + 1] = fmaf(p, s[i], q * c[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float w = __shfl_sync(0xFFFFFFFFu, v[i], partner);
        v[i] = fmaf(v[i], c[i], sign * (w * s[i]));
      }
    }
  }
};
constexpr int kAngles = MP_HEAD_MAX_D / 2 + 8;    // of a token, and 8 zero angles for columns that do not turn

__device__ __forceinline__ int64_t position(const HeadArgs& a, int64_t i) {
  if (a.rot == 0) return 0;
  return a.pos_bytes == 8 ? rows::load_id<int64_t>(a.pos, i) : rows::load_id<int32_t>(a.pos, i);
}
template <int L>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}
// A lane's 8 gains as stored (1 where there are none).
__device__ __forceinline__ uint4 gain8(const uint16_t* g, int col, bool on) {
  if (g == nullptr) return make_uint4(0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u);
  return on ? __ldg(reinterpret_cast<const uint4*>(g + col)) : make_uint4(0, 0, 0, 0);
}

// Work items: (token, part of its rounds); rounds 0 .. rq-1 are the queries', the others the keys'.
template <int L>
struct Rounds {
  static constexpr int G = 32 / L;
  int rq, all, first, end, hq, hk;
  __device__ __forceinline__ Rounds(const HeadArgs& a, int part) {
    hq = a.hq;
    hk = a.hk;
    rq = (a.hq + G - 1) / G;
    all = rq + (a.hk + G - 1) / G;
    first = (int)((int64_t)all * part / a.parts);
    end = (int)((int64_t)all * (part + 1) / a.parts);
  }
  // this lane's head in round r, or -1
  __device__ __forceinline__ int head(int r) const {
    const int sub = (threadIdx.x & 31) / L;
    if (r < rq) return r * G + sub < hq ? r * G + sub : -1;
    const int h = (r - rq) * G + sub;
    return h < hk ? hq + h : -1;
  }
};

// Blocks an SM: three forward (16384 x 40 heads of 128: 84 us; with four, which spill at 64 registers,
// 87), two backward.
template <bool BACK>
constexpr int kResident = BACK ? 2 : 3;
template <int L, bool PAIRS, bool BACK>
__global__ void __launch_bounds__(kThreads, kResident<BACK>) mp_head_norm_rope_kernel(const HeadArgs a) {
  constexpr int U = kRounds;
  __shared__ __align__(16) float2 tables[kWarps][kAngles];
  __shared__ uint64_t turns[MP_HEAD_MAX_D / 2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = lane % L, col = t * 8;
  const bool inside = col < a.D;
  ptx::launch_dependents();
  ptx::grid_dependency_wait();
  // the other member of a lane's pairs, where the halves of a head are rotated against one another
  const int hop = a.rot / 16, angles = a.rot / 2;
  const int partner = col >= a.rot ? lane : t < hop ? lane + hop : lane - hop;
  const float sign = t < hop ? -1.0f : 1.0f;
  const int mine = col >= a.rot ? MP_HEAD_MAX_D / 2 : PAIRS ? col / 2 : col >= angles ? col - angles : col;
  float2* table = tables[warp];
  if (lane < 8) table[MP_HEAD_MAX_D / 2 + lane] = make_float2(1.0f, 0.0f);
  // Turns of one position in 64-bit fixed point: times a position, whole turns fall off the top.
  for (int i = threadIdx.x; i < angles; i += kThreads) {
    double x = a.freqs[i] * 0.15915494309189535;
    x -= floor(x);
    turns[i] = __double2ull_rn(x * 18446744073709551616.0);
  }
  __syncthreads();
  const uint4 gain_q = gain8(a.gq, col, inside), gain_k = gain8(a.gk, col, inside);
  float sq[8], sk[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) sq[i] = sk[i] = 0.0f;
  const float inv_d = 1.0f / (float)a.D;
  const int64_t items = a.T * a.parts, stride = (int64_t)gridDim.x * kWarps;
  for (int64_t item = (int64_t)blockIdx.x * kWarps + warp; item < items; item += stride) {
    const int64_t token = item / a.parts;
    const Rounds<L> rounds(a, (int)(item - token * a.parts));
    rows::Raw8<uint16_t> rx[U], rd[BACK ? U : 1];
    auto load = [&](int r) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = r + u < rounds.end ? rounds.head(r + u) : -1;
        const int64_t c = (int64_t)h * a.D + col;
        const int n = h >= 0 && inside ? 8 : 0;
        rx[u].load(a.x + token * a.ldx + c, n);
        if constexpr (BACK) rd[u].load(a.dy + token * a.lddy + c, n);
      }
    };
    load(rounds.first);
    const uint64_t pos = (uint64_t)position(a, token);
    __syncwarp();                                 // the angles before have been read
    for (int i = lane; i < angles; i += 32) {
      const float x = (float)(int32_t)((turns[i] * pos) >> 32) * 0x1p-31f;       // half turns, -1 .. 1
      float2 cs;
      sincospif(BACK ? -x : x, &cs.y, &cs.x);
      table[i] = cs;
    }
    __syncwarp();
    Turn<PAIRS> turn;
    turn.load(table, mine);
    for (int r = rounds.first; r < rounds.end; r += U) {
      if (r > rounds.first) load(r);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (r + u >= rounds.end) break;           // warp-uniform
        const int h = rounds.head(r + u);
        const bool query = r + u < rounds.rq;
        float x[8], g[8], ss = 0.0f;
        rx[u].floats(x);
        rows::Raw8<uint16_t> gain;
        gain.q = query ? gain_q : gain_k;
        gain.floats(g);
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
        ss = head_sum<L>(ss);                     // every lane takes part
        float root = rsqrtf(fmaf(ss, inv_d, a.eps));
        if constexpr (BACK) root = h >= 0 ? root : 0.0f;     // zeros must stay so in the gains' sums, without an eps too
        if constexpr (!BACK) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] *= root * g[e];
          turn.apply(x, partner, sign);
        } else {
          float d[8], dot = 0.0f;
          rd[u].floats(d);
          turn.apply(d, partner, sign);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[e] *= root;
            const float w = d[e] * x[e];
            if (query) sq[e] += w;
            else sk[e] += w;
            d[e] *= g[e];
            dot = fmaf(d[e], x[e], dot);
          }
          dot = head_sum<L>(dot) * inv_d;
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = root * fmaf(-x[e], dot, d[e]);
        }
        if (h >= 0 && inside) rows::store8(a.out + token * a.ldo + (int64_t)h * a.D + col, x, 8);
      }
    }
  }
  if constexpr (BACK) {
    if (a.part == nullptr) return;
    // heads of a warp, then warps, in order
    __shared__ float sums[kWarps][2][L * 8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int o = L; o < 32; o <<= 1) {
        sq[e] += __shfl_xor_sync(0xFFFFFFFFu, sq[e], o);
        sk[e] += __shfl_xor_sync(0xFFFFFFFFu, sk[e], o);
      }
    if (lane < L)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sums[warp][0][col + e] = sq[e];
        sums[warp][1][col + e] = sk[e];
      }
    __syncthreads();
    for (int k = threadIdx.x; k < 2 * a.D; k += kThreads) {
      const int which = k >= a.D, c = k - which * a.D;
      float v = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) v += sums[w][which][c];
      a.part[(int64_t)blockIdx.x * 2 * a.D + k] = v;
    }
  }
}

// The gains' gradients: the blocks' sums, in order, rounded once.  A block has 32 columns, each summed by 8 threads.
__global__ void __launch_bounds__(256) mp_head_gain_kernel(const float* part, int blocks, int D, uint16_t* dgq, uint16_t* dgk,
                                                           mp_dev_state* st) {
  __shared__ float sums[8][32];
  ptx::grid_dependency_wait();
  const int k = blockIdx.x * 32 + threadIdx.x % 32, way = threadIdx.x / 32;
  const int a = (int)((int64_t)blocks * way / 8), b = (int)((int64_t)blocks * (way + 1) / 8);
  float v = 0.0f;
  if (k < 2 * D)
#pragma unroll 8
    for (int i = a; i < b; ++i) v += part[(int64_t)i * 2 * D + k];
  sums[way][threadIdx.x % 32] = v;
  __syncthreads();
  if (way > 0 || k >= 2 * D) return;
  v = 0.0f;
#pragma unroll
  for (int w = 0; w < 8; ++w) v += sums[w][threadIdx.x];
  const uint16_t h = rows::f2h(v);
  if (k < D) dgq[k] = h;
  else dgk[k - D] = h;
  if (rows::nonfinite16(h) && st) atomicOr(&st->h.found_inf, 1);
}

template <int L, bool PAIRS, bool BACK>
int launch(HeadArgs a, int* used, cudaStream_t st) {
  constexpr int G = 32 / L;
  const int rounds = (a.hq + G - 1) / G + (a.hk + G - 1) / G;
  // Tokens are cut into parts until every warp has some six of them, so that the last ones do not leave many idle, but not below the
  // rounds whose loads are in flight together; few tokens down to one round a warp, so that the loads of all heads start at once.
  const int64_t warps = (int64_t)148 * kResident<BACK> * kWarps, whole = (rounds + kRounds - 1) / kRounds;
  int64_t parts = (6 * warps + a.T - 1) / a.T;
  if (parts > whole) parts = a.T * whole >= warps ? whole : (warps + a.T - 1) / a.T;
  a.parts = (int)(parts > rounds ? rounds : parts);
  int64_t blocks = (a.T * a.parts + kWarps - 1) / kWarps;
  if (blocks > 148 * kResident<BACK>) blocks = 148 * kResident<BACK>;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks, 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  MP_CUDA_TRY(cudaLaunchKernelEx(&cfg, mp_head_norm_rope_kernel<L, PAIRS, BACK>, a));
  mp::count_launch();
  *used = (int)blocks;
  return MP_OK;
}
template <int L, bool BACK>
int by_pairs(const HeadArgs& a, bool pairs, int* used, cudaStream_t st) {
  return pairs ? launch<L, true, BACK>(a, used, st) : launch<L, false, BACK>(a, used, st);
}
template <bool BACK>
int dispatch(const HeadArgs& a, bool pairs, int* used, cudaStream_t st) {
  if (a.D <= 32) return by_pairs<4, BACK>(a, pairs, used, st);
  if (a.D <= 64) return by_pairs<8, BACK>(a, pairs, used, st);
  if (a.D <= 128) return by_pairs<16, BACK>(a, pairs, used, st);
  return by_pairs<32, BACK>(a, pairs, used, st);
}

int check(const char* name, const HeadArgs& a, int64_t hq, int64_t hk, int64_t D, int64_t rot, int pairs) {
  if (a.T < 0 || hq < 0 || hk < 0 || hq + hk <= 0 || D <= 0 || D % 8 || rot < 0 || rot > D || rot % 16 ||
      (pairs != 0 && pairs != 1) || !(a.eps >= 0.0f) || (rot > 0 && a.pos_bytes != 4 && a.pos_bytes != 8))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: bad size, a head size that is not a multiple of 8, a rotated part that is "
                         "not a multiple of 16, or a bad width of the positions", name);
  if (D > MP_HEAD_MAX_D || hq + hk > 65536) return mp::set_error(MP_ERR_TOO_LARGE, "%s: heads of more than %d elements, or more "
                                                                 "than 65536 heads", name, MP_HEAD_MAX_D);
  const int64_t width = (hq + hk) * D;
  if (a.ldx < width || a.ldo < width) return mp::set_error(MP_ERR_INVALID_ARG, "%s: leading dimension smaller than the heads", name);
  if (a.T > 0 && (!a.x || !a.out || (rot > 0 && (!a.pos || !a.freqs))))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: null pointer", name);
  if (((a.ldx | a.ldo) & 7) || !mp::aligned16(a.x) || !mp::aligned16(a.out) || !mp::aligned16(a.gq) || !mp::aligned16(a.gk) ||
      (rot > 0 && (((uintptr_t)a.pos & (uintptr_t)(a.pos_bytes - 1)) || ((uintptr_t)a.freqs & 7))))
    return mp::set_error(MP_ERR_ALIGNMENT, "%s: matrices and gains must be 16-byte aligned with pitches that are multiples of "
                         "8, positions and frequencies aligned to their width", name);
  if (a.out == a.x && a.ldo != a.ldx)
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: a result in an input's place needs its pitch", name);
  return MP_OK;
}

}  // namespace

extern "C" {

int mp_head_norm_rope_fwd(const void* x16, int64_t ldx, const void* gq16, const void* gk16, const void* positions,
                          int pos_bytes, const double* freqs, int64_t rot, int pairs, float eps, void* y16, int64_t ldy,
                          int64_t T, int64_t q_heads, int64_t k_heads, int64_t D, void* stream) {
  HeadArgs a = {};
  a.x = (const uint16_t*)x16; a.ldx = ldx; a.gq = (const uint16_t*)gq16; a.gk = (const uint16_t*)gk16;
  a.pos = positions; a.pos_bytes = pos_bytes; a.freqs = freqs; a.out = (uint16_t*)y16; a.ldo = ldy; a.T = T; a.eps = eps;
  if (int rc = check("mp_head_norm_rope_fwd", a, q_heads, k_heads, D, rot, pairs)) return rc;
  a.hq = (int)q_heads; a.hk = (int)k_heads; a.D = (int)D; a.rot = (int)rot;
  if (int rc = mp::check_device()) return rc;
  if (T == 0) return MP_OK;
  int used = 0;
  return dispatch<false>(a, pairs != 0, &used, (cudaStream_t)stream);
}

size_t mp_head_norm_rope_bwd_workspace_bytes(int64_t T, int64_t q_heads, int64_t k_heads, int64_t D) {
  if (T < 0 || q_heads < 0 || k_heads < 0 || q_heads + k_heads <= 0 || D <= 0 || D % 8 || D > MP_HEAD_MAX_D) return 0;
  return (size_t)kMaxBlocks * 2 * D * sizeof(float);
}

int mp_head_norm_rope_bwd(const void* dy16, int64_t lddy, const void* x16, int64_t ldx, const void* gq16, const void* gk16,
                          const void* positions, int pos_bytes, const double* freqs, int64_t rot, int pairs, float eps,
                          void* dx16, int64_t lddx, void* dgq16, void* dgk16, int64_t T, int64_t q_heads, int64_t k_heads,
                          int64_t D, mp_state* state, void* workspace, size_t workspace_bytes, void* stream) {
  const char* name = "mp_head_norm_rope_bwd";
  HeadArgs a = {};
  a.x = (const uint16_t*)x16; a.ldx = ldx; a.dy = (const uint16_t*)dy16; a.lddy = lddy;
  a.gq = (const uint16_t*)gq16; a.gk = (const uint16_t*)gk16;
  a.pos = positions; a.pos_bytes = pos_bytes; a.freqs = freqs; a.out = (uint16_t*)dx16; a.ldo = lddx; a.T = T; a.eps = eps;
  if (int rc = check(name, a, q_heads, k_heads, D, rot, pairs)) return rc;
  if (lddy < (q_heads + k_heads) * D) return mp::set_error(MP_ERR_INVALID_ARG, "%s: leading dimension smaller than the heads", name);
  if ((T > 0 && !dy16) || !gq16 != !dgq16 || !gk16 != !dgk16 || !gq16 != !gk16)
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: null pointer (gains and their gradients: all or none)", name);
  if ((lddy & 7) || !mp::aligned16(dy16) || !mp::aligned16(dgq16) || !mp::aligned16(dgk16) || !mp::aligned16(workspace))
    return mp::set_error(MP_ERR_ALIGNMENT, "%s: pointers must be 16-byte aligned, pitches multiples of 8", name);
  if (dx16 && dx16 == dy16 && lddx != lddy)
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: a result in an input's place needs its pitch", name);
  const size_t need = gq16 ? mp_head_norm_rope_bwd_workspace_bytes(T, q_heads, k_heads, D) : 0;
  if (need > 0 && (!workspace || workspace_bytes < need))
    return mp::set_error(MP_ERR_NOMEM, "%s: workspace of %zu bytes needed, %zu given", name, need,
                         workspace ? workspace_bytes : (size_t)0);
  a.hq = (int)q_heads; a.hk = (int)k_heads; a.D = (int)D; a.rot = (int)rot;
  a.part = need > 0 ? (float*)workspace : nullptr;
  if (int rc = mp::check_device()) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  int blocks = 0;
  if (T > 0)
    if (int rc = dispatch<true>(a, pairs != 0, &blocks, st)) return rc;
  if (a.part != nullptr) {                        // no tokens: zeros
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((2 * D + 31) / 32), 1, 1);
    cfg.blockDim = dim3(256, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    MP_CUDA_TRY(cudaLaunchKernelEx(&cfg, mp_head_gain_kernel, (const float*)a.part, blocks, (int)D, (uint16_t*)dgq16,
                                   (uint16_t*)dgk16, state ? state->dev : (mp_dev_state*)nullptr));
    mp::count_launch();
  }
  return MP_OK;
}

}  // extern "C"

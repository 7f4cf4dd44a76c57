// Embedding lookup with scaling, and its gradient by sorted tokens.

#include <climits>

#include "rows.cuh"

namespace {

constexpr int kThreads = 256;
constexpr uint16_t kNan16 = 0x7FFFu;

template <class ID>
__global__ void __launch_bounds__(kThreads)
mp_embedding_fwd_kernel(const void* ids, const uint16_t* W, int64_t ldw, uint16_t* Y, int64_t ldy, int64_t n,
                        int64_t V, int64_t D, int64_t pad_id, float scale, mp_dev_state* st) {
  for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
    const int64_t id = rows::load_id<ID>(ids, i);
    const bool pad = pad_id >= 0 && id == pad_id, bad = !pad && (id < 0 || id >= V);
    if (bad && threadIdx.x == 0) rows::record_bad_id(st);
    for (int64_t c = threadIdx.x; c < D; c += kThreads)
      Y[i * ldy + c] = pad ? (uint16_t)0 : bad ? kNan16 : rows::f2h(scale * rows::h2f(W[id * ldw + c]));
  }
}

// One block per table row: the block looks through all ids, 256 at a time, and lists the tokens
// of its row in ascending order; then every thread adds its columns over the list.
template <class ID>
__global__ void __launch_bounds__(kThreads)
mp_embedding_bwd_kernel(const void* ids, const uint16_t* dY, int64_t lddy, uint16_t* dW, int64_t ldw, int64_t n,
                        int64_t V, int64_t D, int64_t pad_id, float scale, mp_dev_state* st, float* acc_all) {
  __shared__ int64_t s_list[kThreads];
  __shared__ int s_count[kThreads / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float* acc = acc_all + (int64_t)blockIdx.x * D;
  for (int64_t v = blockIdx.x; v < V; v += gridDim.x) {
    for (int64_t c = threadIdx.x; c < D; c += kThreads) acc[c] = 0.0f;
    for (int64_t i0 = 0; i0 < n; i0 += kThreads) {
      const int64_t i = i0 + threadIdx.x;
      const int64_t id = i < n ? rows::load_id<ID>(ids, i) : -1;
      if (v == 0 && i < n && (id < 0 || id >= V) && !(pad_id >= 0 && id == pad_id)) rows::record_bad_id(st);
      const bool mine = i < n && id == v && !(pad_id >= 0 && id == pad_id);
      const unsigned mask = __ballot_sync(0xFFFFFFFFu, mine);
      if (lane == 0) s_count[warp] = __popc(mask);
      __syncthreads();
      int before = 0, total = 0;
      for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) before += s_count[w];
        total += s_count[w];
      }
      if (mine) s_list[before + __popc(mask & ((1u << lane) - 1))] = i;
      __syncthreads();
      if (total)
        for (int64_t c = threadIdx.x; c < D; c += kThreads) {
          float a = acc[c];
          for (int k = 0; k < total; ++k) a += rows::h2f(dY[s_list[k] * lddy + c]);
          acc[c] = a;
        }
      __syncthreads();
    }
    bool bad = false;
    for (int64_t c = threadIdx.x; c < D; c += kThreads) {
      const uint16_t h = rows::f2h(scale * acc[c]);
      dW[v * ldw + c] = h;
      bad |= rows::nonfinite16(h);
    }
    if (bad && st != nullptr) atomicOr(&st->h.found_inf, 1);
  }
}

constexpr int64_t kMaxBlocks = 148 * 8;

int check(const char* name, const void* ids, int id_bytes, const void* a16, int64_t lda, const void* b16,
          int64_t ldb, int64_t n, int64_t V, int64_t D) {
  if (n < 0 || V <= 0 || D <= 0 || lda < D || ldb < D || (id_bytes != 4 && id_bytes != 8))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: bad size, pitch or id width", name);
  if ((lda & 7) || (ldb & 7) || !mp::aligned16(a16) || !mp::aligned16(b16) ||
      (reinterpret_cast<uintptr_t>(ids) & (uintptr_t)(id_bytes - 1)))
    return mp::set_error(MP_ERR_ALIGNMENT, "%s: matrices must be 16-byte aligned with pitches that are multiples of 8, "
                         "ids aligned to their width", name);
  return MP_OK;
}

}  // namespace

extern "C" {

int mp_embedding_fwd(const void* ids, int id_bytes, const void* W16, int64_t ldw, void* Y16, int64_t ldy,
                     int64_t n, int64_t V, int64_t D, int64_t pad_id, float scale, mp_state* state,
                     void* stream) {
  if (n > 0 && (!ids || !W16 || !Y16)) return mp::set_error(MP_ERR_INVALID_ARG, "mp_embedding_fwd: null pointer");
  if (int rc = check("mp_embedding_fwd", ids, id_bytes, W16, ldw, Y16, ldy, n, V, D)) return rc;
  if (int rc = mp::check_device()) return rc;
  if (n == 0) return MP_OK;
  const int grid = (int)(n < kMaxBlocks ? n : kMaxBlocks);
  auto kernel = id_bytes == 8 ? mp_embedding_fwd_kernel<int64_t> : mp_embedding_fwd_kernel<int32_t>;
  kernel<<<grid, kThreads, 0, (cudaStream_t)stream>>>(ids, (const uint16_t*)W16, ldw, (uint16_t*)Y16, ldy, n, V, D,
                                                      pad_id, scale, state ? state->dev : nullptr);
  mp::count_launch();
  MP_CUDA_TRY(cudaGetLastError());
  return MP_OK;
}

size_t mp_embedding_bwd_workspace_bytes(int64_t n, int64_t V, int64_t D) {
  if (n < 0 || V <= 0 || D <= 0 || n >= INT_MAX || V >= INT_MAX) return 0;
  return (size_t)(V < kMaxBlocks ? V : kMaxBlocks) * (size_t)D * sizeof(float);
}

int mp_embedding_bwd(const void* ids, int id_bytes, const void* dY16, int64_t lddy, void* dW16, int64_t ldw,
                     int64_t n, int64_t V, int64_t D, int64_t pad_id, float scale, mp_state* state,
                     void* workspace, size_t workspace_bytes, void* stream) {
  if (!dW16 || (n > 0 && (!ids || !dY16)))
    return mp::set_error(MP_ERR_INVALID_ARG, "mp_embedding_bwd: null pointer");
  if (int rc = check("mp_embedding_bwd", ids, id_bytes, dY16, lddy, dW16, ldw, n, V, D)) return rc;
  if (n >= INT_MAX || V >= INT_MAX)
    return mp::set_error(MP_ERR_TOO_LARGE, "mp_embedding_bwd: n and V must be below 2^31 - 1");
  if (workspace && !mp::aligned16(workspace))
    return mp::set_error(MP_ERR_ALIGNMENT, "mp_embedding_bwd: workspace must be 16-byte aligned");
  const size_t need = mp_embedding_bwd_workspace_bytes(n, V, D);
  if (!workspace || workspace_bytes < need)
    return mp::set_error(MP_ERR_NOMEM, "mp_embedding_bwd: workspace of %zu bytes needed", need);
  if (int rc = mp::check_device()) return rc;
  const int grid = (int)(V < kMaxBlocks ? V : kMaxBlocks);
  auto kernel = id_bytes == 8 ? mp_embedding_bwd_kernel<int64_t> : mp_embedding_bwd_kernel<int32_t>;
  kernel<<<grid, kThreads, 0, (cudaStream_t)stream>>>(ids, (const uint16_t*)dY16, lddy, (uint16_t*)dW16, ldw, n, V, D,
                                                      pad_id, scale, state ? state->dev : nullptr, (float*)workspace);
  mp::count_launch();
  MP_CUDA_TRY(cudaGetLastError());
  return MP_OK;
}

}  // extern "C"

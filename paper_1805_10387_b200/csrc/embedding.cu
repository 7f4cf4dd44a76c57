// Embedding lookup with scaling, and its gradient by sorted tokens.

#include <climits>

#include "ptx.cuh"
#include "rows.cuh"

namespace {

// ---------------------------------------------------------------- lookup
//
// A warp's worth of work is 32 vectors of 8 elements in a row or in neighbouring rows: n D / 8 16-byte loads
// and stores with nothing but a multiplication between them.  Measured on a B200: 8192 x 1024 out of 32768 rows 8.3 us,
// 65536 x 1024 41 us (floors 5.1 and 31): a thread has one load in flight, behind that of its id.
constexpr int kFwdThreads = 256;
constexpr uint32_t kNan2 = 0x7FFF7FFFu;

__device__ __forceinline__ int64_t id_at(const void* ids, int id_bytes, int64_t i) {
  return id_bytes == 8 ? rows::load_id<int64_t>(ids, i) : rows::load_id<int32_t>(ids, i);
}
__device__ __forceinline__ void store_vec(uint16_t* p, const uint4& q, int nv) {   // the first nv of eight elements
  if (nv >= 8) {
    *reinterpret_cast<uint4*>(p) = q;
    return;
  }
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < nv) p[j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
}

__global__ void __launch_bounds__(kFwdThreads)
mp_embedding_fwd_kernel(const void* ids, int id_bytes, const uint16_t* W, int64_t ldw, uint16_t* Y, int64_t ldy,
                        int64_t n, int64_t V, int D, int64_t pad_id, float scale, mp_dev_state* st) {
  const int vecs = (D + 7) / 8;
  const int64_t total = n * vecs;
  for (int64_t x = (int64_t)blockIdx.x * kFwdThreads + threadIdx.x; x < total; x += (int64_t)gridDim.x * kFwdThreads) {
    const int64_t i = total <= UINT_MAX ? (uint32_t)x / (uint32_t)vecs : x / vecs;
    const int col = (int)(x - i * vecs) * 8, nv = D - col < 8 ? D - col : 8;
    const int64_t id = id_at(ids, id_bytes, i);
    uint4 q = make_uint4(0, 0, 0, 0);
    if (!(pad_id >= 0 && id == pad_id)) {
      if (id >= 0 && id < V) {
        rows::Raw8<uint16_t> r;
        r.load_cached(W + id * ldw + col, nv);
        float f[8];
        r.floats(f);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] *= scale;
        q = rows::pack8(f);
      } else {
        q = make_uint4(kNan2, kNan2, kNan2, kNan2);
        if (col == 0) rows::record_bad_id(st);
      }
    }
    store_vec(Y + i * ldy + col, q, nv);
  }
}

// ---------------------------------------------------------------- gradient
//
// 1. One cluster of 8 or 16 blocks sorts the tokens by id while the rest of the GPU writes zeros over dW, which
//    takes longer (most rows of a large table get no token of a batch).  The sort is a stable radix
//    sort of at most 8 bits a pass; each warp owns a run of tokens, counts its digits, and after a scan
//    over digits, blocks and warps places its tokens in order.  (A cluster of 16 for many tokens: 65536 of
//    them 71 us in all instead of 88; 8192 take 33 instead of 31.)
// 2. The sorted tokens are cut into tiles; a group of threads, one for each 8 columns, adds the rows of
//    dY over its tile and stores a row of dW whenever the id changes.  A run of one id that reaches
//    into the next tile is finished by the tile in which it begins; a run over three tiles or more leaves
//    one FP32 partial row in each tile.
// 3. The partial rows of such runs are added in order.
// dY is read once and dW written once (rows with tokens twice).  No floating-point atomics: the order of
// every sum follows from the ids alone.  Measured on a B200: 8192 x 1024 into 32768 rows 31 us (sort 11 with the zeros
// beside it, sums 8, join 5, and the gaps), 25600 x 1600 into 29 rows 37 us; HBM alone would need 13 each.  What
// is left is the latency of the sort's passes (about 5 us each: ids, counts, scan over the cluster, placement) and of
// three dependent kernels.  A block per table row that looked through all ids took 639 and 3051 us.  Tried without
// gain: fetching dY into L2 during the sort (the sums are not bound by HBM's latency), 16 rows in flight per
// thread instead of 8 (fewer blocks fit).
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kMostBits = 8, kHistPitch = (1 << kMostBits) + 1;   // odd pitch: a quad's four rows lie in four banks
constexpr int kTileRound = 128;                  // the sorted lists are filled up to a multiple of this and of every tile

struct SortArgs {
  const void* ids;
  int id_bytes;
  int n, n_round;                                // n_round: n rounded up to kTileRound
  int V;
  int64_t pad_id;
  int* key[2];                                   // ping-pong: pass p writes [p & 1]
  int* pos[2];
  int passes, bits;
  uint16_t* dW;
  int64_t ldw;
  int D;
  mp_dev_state* st;
};

__device__ __forceinline__ int sort_key(const SortArgs& a, int i) {   // tokens that count for nothing go last
  const int64_t id = id_at(a.ids, a.id_bytes, i);
  if (a.pad_id >= 0 && id == a.pad_id) return a.V;
  if (id >= 0 && id < a.V) return (int)id;
  rows::record_bad_id(a.st);
  return a.V;
}

__device__ void fill_zeros(const SortArgs& a, int64_t worker, int64_t workers) {
  const int vecs = (a.D + 7) / 8;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  if (a.ldw == a.D && a.D % 8 == 0) {
    uint4* p = reinterpret_cast<uint4*>(a.dW);
    const int64_t total = (int64_t)a.V * vecs;
    for (int64_t x = worker; x < total; x += workers) __stcs(p + x, zero);
    return;
  }
  const int64_t total = (int64_t)a.V * vecs;
  for (int64_t x = worker; x < total; x += workers) {
    const int64_t v = total <= UINT_MAX ? (uint32_t)x / (uint32_t)vecs : x / vecs;
    const int col = (int)(x - v * vecs) * 8;
    store_vec(a.dW + v * a.ldw + col, zero, a.D - col < 8 ? a.D - col : 8);
  }
}

// What follows the last token belongs to no row.
__device__ void pad_list(const SortArgs& a, int rank, int blocks) {
  for (int64_t i = (int64_t)a.n + rank * kSortThreads + threadIdx.x; i < a.n_round; i += blocks * kSortThreads)
    a.key[(a.passes & 1) ^ 1][i] = a.V;
}

// Few tokens need no passes: a token's place is the number of tokens before it in the order (id, position), so each
// block counts that for its share of the tokens against all of them, 8 segments of the list per token.  The
// whole gradient of 1000 x 512 into 8000 rows takes 16.5 us so, 22.6 with the passes; 500 tokens 14.4 and 19.7.
constexpr int kFewTokens = 1024;                 // with ids below kFewRows: id and position fit one word
constexpr int kFewRows = 1 << 21;
__device__ void rank_few(const SortArgs& a, int rank, int blocks) {
  __shared__ alignas(16) uint32_t s_word[kFewTokens];
  __shared__ int s_before[kFewTokens / 8];       // blocks is 8
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int i = threadIdx.x; i < kFewTokens; i += kSortThreads)       // past the last token: a word that is below none
    s_word[i] = i < a.n ? (uint32_t)sort_key(a, i) * kFewTokens + i : 0xFFFFFFFFu;
  if (threadIdx.x < kFewTokens / 8) s_before[threadIdx.x] = 0;
  __syncthreads();
  const int per = (a.n + blocks - 1) / blocks, first = rank * per, segment = warp & 7;
  const int mine = (warp >> 3) * 32 + lane, i = first + mine;        // 4 warps of tokens, 8 segments
  if (mine < per && i < a.n) {
    const uint32_t word = s_word[i];
    const uint4* list = reinterpret_cast<const uint4*>(s_word) + segment * (kFewTokens / 32);
    int before = 0;
#pragma unroll 8
    for (int x = 0; x < kFewTokens / 32; ++x) {
      const uint4 q = list[x];
      before += (q.x < word) + (q.y < word) + (q.z < word) + (q.w < word);
    }
    atomicAdd(s_before + mine, before);
  }
  __syncthreads();
  const int x = first + threadIdx.x;
  if ((int)threadIdx.x < per && x < a.n) {
    const int to = s_before[threadIdx.x], out = (a.passes & 1) ^ 1;
    a.key[out][to] = (int)(s_word[x] / kFewTokens);
    a.pos[out][to] = x;
  }
}

template <int kSortCluster>
__global__ void __launch_bounds__(kSortThreads, 1) mp_embedding_sort_kernel(const SortArgs a) {
  ptx::launch_dependents();                      // the sum kernel's blocks take the places of those that are done
  if (blockIdx.x >= kSortCluster) {              // the other clusters
    fill_zeros(a, (int64_t)(blockIdx.x - kSortCluster) * kSortThreads + threadIdx.x,
               (int64_t)(gridDim.x - kSortCluster) * kSortThreads);
    return;
  }
  if (kSortCluster == 8 && a.n <= kFewTokens && a.V < kFewRows) {
    rank_few(a, blockIdx.x, kSortCluster);
    pad_list(a, blockIdx.x, kSortCluster);
    return;
  }
  __shared__ int hist[kSortWarps][kHistPitch];   // [warp][digit]
  __shared__ int s_total[1 << kMostBits];        // of this block, by digit; the other blocks read it
  __shared__ int s_warp[kSortWarps];
  const int rank = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, mask = (1 << a.bits) - 1;
  int* mine = hist[warp];
  // runs of whole 32s, in order over blocks and warps; kStep tokens of a run are worked on at once, and a run
  // that is no longer stays in registers between counting and placing
  constexpr int kStep = 128, kU = kStep / 32;
  const int64_t run = (((int64_t)a.n + kSortCluster * kSortThreads - 1) / (kSortCluster * kSortThreads)) * 32;
  const int64_t begin = (rank * kSortWarps + warp) * run;
  const int64_t end = begin + run < a.n ? begin + run : a.n;
  for (int pass = 0; pass < a.passes; ++pass) {
    const int shift = pass * a.bits;
    const int* key_in = a.key[(pass & 1) ^ 1];
    const int* pos_in = a.pos[(pass & 1) ^ 1];
    int* key_out = a.key[pass & 1];
    int* pos_out = a.pos[pass & 1];
    int k[kU], p[kU];
    unsigned same[kU];                           // lanes with the same digit
    auto load = [&](int64_t i0, bool with_pos) {
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int64_t i = i0 + u * 32 + lane;
        k[u] = i >= end ? -1 : pass == 0 ? sort_key(a, (int)i) : __ldcg(key_in + i);
        p[u] = pass == 0 ? (int)i : i < end && with_pos ? __ldcg(pos_in + i) : 0;
      }
    };
    auto digit = [&](int key) { return key < 0 ? -1 : (key >> shift) & mask; };
    auto match = [&] {
#pragma unroll
      for (int u = 0; u < kU; ++u) {             // a vote a bit: cheaper than the hardware's match of whole values
        if (u * 32 >= run) break;
        same[u] = __ballot_sync(0xFFFFFFFFu, k[u] >= 0);
#pragma unroll
        for (int bit = 0; bit < kMostBits; ++bit) {
          if (bit >= a.bits) break;
          const bool on = k[u] >> (shift + bit) & 1;
          const unsigned votes = __ballot_sync(0xFFFFFFFFu, on);
          same[u] &= on ? votes : ~votes;
        }
      }
    };
    for (int j = threadIdx.x; j < kSortWarps * kHistPitch; j += kSortThreads) (&hist[0][0])[j] = 0;
    load(begin, run <= kStep);
    __syncthreads();
    // count
    for (int64_t i0 = begin; i0 < end; i0 += kStep) {
      if (i0 > begin) load(i0, false);
#pragma unroll
      for (int u = 0; u < kU; ++u)
        if (k[u] >= 0) atomicAdd(mine + digit(k[u]), 1);
    }
    __syncthreads();
    // scan: four threads per digit, eight warps' counts each
    const int dg = threadIdx.x >> 2, q = threadIdx.x & 3;
    int count[8], sum = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      count[i] = hist[q * 8 + i][dg];
      sum += count[i];
    }
    int upto = sum;                              // over this quad's threads up to this one
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      const int y = __shfl_up_sync(0xFFFFFFFFu, upto, o, 4);
      if (q >= o) upto += y;
    }
    if (q == 3) s_total[dg] = upto;
    ptx::cluster_sync();
    int all = 0, before = 0;                     // of this digit: over the cluster, and in lower blocks
    const uint32_t at = ptx::smem_u32(s_total + dg);
#pragma unroll
    for (int i = 0; i < kSortCluster / 4; ++i) {
      const int r = q * (kSortCluster / 4) + i;
      int x;
      asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(x) : "r"(ptx::map_to_cta(at, r)) : "memory");
      all += x;
      before += r < rank ? x : 0;
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      all += __shfl_xor_sync(0xFFFFFFFFu, all, o);
      before += __shfl_xor_sync(0xFFFFFFFFu, before, o);
    }
    int lower = all;                             // over this warp's eight digits up to this one
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xFFFFFFFFu, lower, o);
      if (lane >= o) lower += y;
    }
    if (lane == 31) s_warp[warp] = lower;
    __syncthreads();
    int warps = s_warp[lane];                    // over the warps up to this lane's
    const int own = warps;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xFFFFFFFFu, warps, o);
      if (lane >= o) warps += y;
    }
    int base = __shfl_sync(0xFFFFFFFFu, warps - own, warp) + lower - all + before + upto - sum;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      hist[q * 8 + i][dg] = base;
      base += count[i];
    }
    __syncthreads();
    // place: in order within a run, equal digits of 32 neighbours by their lanes
    for (int64_t i0 = begin; i0 < end; i0 += kStep) {
      if (run > kStep) load(i0, true);
      match();
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        if (u * 32 >= run) break;
        const int d = digit(k[u]);
        int to = 0;
        if (d >= 0) to = mine[d] + __popc(same[u] & ((1u << lane) - 1));
        __syncwarp();
        if (d >= 0) {
          if ((same[u] >> lane) == 1u) mine[d] = to + 1;
          __stcg(key_out + to, k[u]);
          __stcg(pos_out + to, p[u]);
        }
        __syncwarp();
      }
    }
    ptx::cluster_sync();                         // the pass's lists are complete; s_total may be written again
  }
  pad_list(a, rank, kSortCluster);
}

struct SumArgs {
  const int* key;
  const int* pos;
  int n_round, V, tile;                          // tile: sorted tokens per tile, a multiple of 8 that divides n_round
  const uint16_t* dY;
  int64_t lddy;
  uint16_t* dW;
  int64_t ldw;
  int D;
  float scale;
  float* part;                                   // [tile][2][D4]: a run from before the tile, a run that goes on
  int D4;                                        // D rounded up to 8
  mp_dev_state* st;
};

// Key of sorted position p; -1 before the first and past the last.
__device__ __forceinline__ int key_of(const SumArgs& a, int64_t p) { return p < 0 || p >= a.n_round ? -1 : __ldcg(a.key + p); }

__device__ __forceinline__ bool store_row(const SumArgs& a, int key, int col, const float (&acc)[8]) {
  float f[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = a.scale * acc[j];
  const int nv = a.D - col < 8 ? a.D - col : 8;
  const uint4 q = rows::pack8(f);
  store_vec(a.dW + (int64_t)key * a.ldw + col, q, nv);
  bool bad = false;
#pragma unroll
  for (int j = 0; j < 8; ++j) bad |= j < nv && !(fabsf(f[j]) < 65520.0f);      // what FP16 rounds to a finite number
  return bad;
}

constexpr int kSumThreads = 256, kMostGroups = 32;
__global__ void __launch_bounds__(kSumThreads, 3) mp_embedding_sum_kernel(const SumArgs a, int cols, int groups, int tiles, unsigned across) {
  // cols: vectors of 8 columns that a group of threads covers; across: blocks over the tiles.  The blocks over the columns
  // are numbered after them in x, since a grid's y ends at 65535 and a row may need more
  extern __shared__ int2 s_list[];               // (key, position) of the groups' tiles and of the tile after them
  const int group = threadIdx.x / cols, window = (groups + 1) * a.tile;
  const unsigned down = blockIdx.x / across, along = blockIdx.x - down * across;
  const int64_t t = (int64_t)along * groups + group, begin = (int64_t)along * groups * a.tile;
  const int col = (down * cols + threadIdx.x % cols) * 8;
  asm volatile("griddepcontrol.wait;" ::: "memory");   // the sorted lists and the zeros are complete
  ptx::launch_dependents();                      // the join kernel's blocks take the places of those that are done
  for (int x = threadIdx.x; x < window; x += blockDim.x) {
    const int64_t p = begin + x;
    s_list[x] = p < a.n_round ? make_int2(__ldcg(a.key + p), __ldcg(a.pos + p)) : make_int2(INT_MAX, 0);
  }
  const int64_t p0 = t * a.tile, p1 = p0 + a.tile;
  int after = 0, ahead = 0, before = 0;
  if (group < groups) {
    after = key_of(a, p1 + a.tile);
    ahead = key_of(a, p0 - 1);
    before = key_of(a, p0 - a.tile - 1);
  }
  __syncthreads();
  if (group >= groups || t >= tiles || col >= a.D) return;
  const int2* list = s_list + group * a.tile;
  const int first = list[0].x, last = list[a.tile - 1].x, next = list[a.tile].x;
  if (first >= a.V) return;
  // the run that comes from before: two tiles long, it belongs to the tile before; else it leaves a partial row
  const bool from_before = ahead == first;
  const bool skip_head = from_before && next != first && before != first;
  // the run that goes on, if it begins here: two tiles long, it is finished here
  const bool goes_on = next == last && last < a.V;
  const bool finish = goes_on && !(from_before && first == last) && after != last;
  float acc[8] = {};
  int cur = first;
  bool head = from_before, bad = false;
  auto emit = [&](bool open) {                   // open: the run goes on after what was added
    if (cur >= a.V || (head && skip_head)) return;
    if (!head && !open) {
      bad |= store_row(a, cur, col, acc);
      return;
    }
    float* to = a.part + (t * 2 + (head ? 0 : 1)) * a.D4 + col;
    reinterpret_cast<float4*>(to)[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    reinterpret_cast<float4*>(to)[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
  };
  const uint16_t* base = a.dY + col;
  const int stop = finish ? 2 * a.tile : a.tile;
  bool done = false;
  for (int p = 0; !done && p < stop; p += 8) {
    const bool beyond = p >= a.tile;
    uint4 v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int2 e = list[p + u];
      const bool wanted = e.x < a.V && (!beyond || e.x == last) && !(skip_head && e.x == first);
      v[u] = wanted ? __ldcs(reinterpret_cast<const uint4*>(base + (int64_t)e.y * a.lddy)) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int k = list[p + u].x;
      if (done) continue;
      if (k != cur) {
        if (beyond) {                            // the run that was to be finished ends
          done = true;
          continue;
        }
        emit(false);
        head = false;
        cur = k;
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = 0.0f;
      }
      float f[8];
      rows::Raw8<uint16_t> r;
      r.q = v[u];
      r.floats(f);
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += f[j];
    }
  }
  emit(finish ? false : goes_on);
  if (bad && a.st) atomicOr(&a.st->h.found_inf, 1);
}

// Runs over three tiles or more: the tile in which one begins left its part, every further tile its own.  A block
// looks through its share of the tiles for the beginnings of such runs; 4 groups of 64 threads (4
// columns each) add the parts of a run in 4 pieces, and the pieces in order.
// (Looking through the lists before the wait on the sum kernel would hide up to 2 us, but only what follows the wait is
// promised to see them.)
constexpr int kJoinThreads = 256, kJoinGroups = 4, kJoinLanes = kJoinThreads / kJoinGroups, kJoinCols = kJoinLanes * 4;
__global__ void __launch_bounds__(kJoinThreads) mp_embedding_join_kernel(const SumArgs a, int tiles) {
  __shared__ float4 sm[kJoinGroups][kJoinLanes];
  const unsigned down = blockIdx.x, along = blockIdx.y, across = gridDim.y;     // a row may need more blocks than y holds
  const int group = threadIdx.x / kJoinLanes, col = down * kJoinCols + (threadIdx.x % kJoinLanes) * 4;
  asm volatile("griddepcontrol.wait;" ::: "memory");   // the lists and the partial rows are complete and visible
  bool bad = false;
  for (int64_t t0 = along; t0 < tiles; t0 += (int64_t)across * kJoinThreads) {
    // thread x looks at tile t0 + x * blocks
    const int64_t t = t0 + (int64_t)threadIdx.x * across;
    bool begins = false;
    if (t < tiles) {
      const int64_t p0 = t * a.tile, p1 = p0 + a.tile;
      const int last = key_of(a, p1 - 1), next = key_of(a, p1), after = key_of(a, p1 + a.tile);
      const int first = key_of(a, p0), ahead = key_of(a, p0 - 1);
      begins = last < a.V && next == last && after == last && !(first == last && ahead == last);
    }
    __shared__ unsigned found[kJoinThreads / 32];
    const unsigned votes = __ballot_sync(0xFFFFFFFFu, begins);
    if ((threadIdx.x & 31) == 0) found[threadIdx.x >> 5] = votes;
    __syncthreads();
    for (int x = 0; x < kJoinThreads; ++x) {
      if (!(found[x >> 5] >> (x & 31) & 1)) {
        if (found[x >> 5] >> (x & 31) == 0) x |= 31;   // none in the rest of this word
        continue;
      }
      const int64_t b = t0 + (int64_t)x * across;
      const int key = key_of(a, (b + 1) * a.tile - 1);
      // further tiles whose first token is of this id
      int more = 0;
      for (;;) {
        const int here = __syncthreads_count(key_of(a, (b + 1 + more + threadIdx.x) * a.tile) == key);
        more += here;
        if (here < kJoinThreads) break;
      }
      const int parts = more + 1, per = (parts + kJoinGroups - 1) / kJoinGroups;
      const int from = group * per, to = from + per < parts ? from + per : parts;
      float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (col < a.D4)
#pragma unroll 8
        for (int i = from; i < to; ++i) {
          const float4 v = __ldcg(reinterpret_cast<const float4*>(a.part + ((b + i) * 2 + (i == 0 ? 1 : 0)) * a.D4 + col));
          s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
      sm[group][threadIdx.x % kJoinLanes] = s;
      __syncthreads();
      if (group == 0 && col < a.D) {
        for (int g = 1; g < kJoinGroups; ++g) {
          const float4 v = sm[g][threadIdx.x];
          s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        const float f[4] = {a.scale * s.x, a.scale * s.y, a.scale * s.z, a.scale * s.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (col + j < a.D) {
            const uint16_t h = rows::f2h(f[j]);
            a.dW[(int64_t)key * a.ldw + col + j] = h;
            bad |= rows::nonfinite16(h);
          }
      }
      __syncthreads();
    }
    __syncthreads();
  }
  if (bad && a.st) atomicOr(&a.st->h.found_inf, 1);
}

int check(const char* name, const void* ids, int id_bytes, const void* a16, int64_t lda, const void* b16,
          int64_t ldb, int64_t n, int64_t V, int64_t D) {
  if (n < 0 || V <= 0 || D <= 0 || lda < D || ldb < D || (id_bytes != 4 && id_bytes != 8))
    return mp::set_error(MP_ERR_INVALID_ARG, "%s: bad size, pitch or id width", name);
  if ((lda & 7) || (ldb & 7) || !mp::aligned16(a16) || !mp::aligned16(b16) ||
      (reinterpret_cast<uintptr_t>(ids) & (uintptr_t)(id_bytes - 1)))
    return mp::set_error(MP_ERR_ALIGNMENT, "%s: matrices must be 16-byte aligned with pitches that are multiples of 8, "
                         "ids aligned to their width", name);
  if (D > INT_MAX - 8) return mp::set_error(MP_ERR_TOO_LARGE, "%s: D must be below 2^31 - 8", name);
  return MP_OK;
}

// Launches the sort with as many clusters as are resident at once, asked once per device.  (A GPU's processing
// clusters hold whole clusters only: 16 of 8 blocks on a B200.  Two more would start when the first
// have left, and the zeros would take twice as long.)
template <int CL>
int sort_launch(const SortArgs& s, cudaStream_t st) {
  static mp::PerDevice resident;
  auto kernel = mp_embedding_sort_kernel<CL>;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(144, 1, 1);
  cfg.blockDim = dim3(kSortThreads, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = CL;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  int dev = 0, clusters = 0;
  MP_CUDA_TRY(cudaGetDevice(&dev));
  clusters = resident.get(dev);
  if (clusters == 0) {
    MP_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    MP_CUDA_TRY(cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg));
    if (clusters < 2) clusters = 2;              // the sort's and one that writes zeros
    resident.set(dev, clusters);
  }
  cfg.gridDim = dim3((unsigned)(clusters * CL), 1, 1);
  MP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, s));
  return MP_OK;
}
constexpr int64_t kManyTokens = 16384;           // from here on 16 blocks sort

int64_t round_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

// Sorted tokens per tile: about 8 16-byte loads for each of the threads that fit the GPU at once (148 SMs
// x 1024), so that a small batch spreads over all SMs and a large one leaves few partial rows; and at most some
// 2048 tiles, since the join kernel looks at each.
int64_t tile_for(int64_t n, int64_t D) {
  int64_t t = 16;
  while (t < kTileRound && (t * 148 * 1024 < n * ((D + 7) / 8) || t * 2048 < n)) t *= 2;
  return t;
}

// The workspace: two lists of keys, two of positions, the partial rows of the tiles.
size_t list_bytes(int64_t n) { return (size_t)round_up(n, kTileRound) * 4; }
size_t part_bytes(int64_t n, int64_t D) {
  return (size_t)(round_up(n, kTileRound) / tile_for(n, D)) * 2 * (size_t)round_up(D, 8) * sizeof(float);
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
  const int64_t blocks = (n * ((D + 7) / 8) + kFwdThreads - 1) / kFwdThreads, most = 148 * 8 * 4;
  mp_embedding_fwd_kernel<<<(unsigned)(blocks < most ? blocks : most), kFwdThreads, 0, (cudaStream_t)stream>>>(
      ids, id_bytes, (const uint16_t*)W16, ldw, (uint16_t*)Y16, ldy, n, V, (int)D, pad_id, scale,
      state ? state->dev : nullptr);
  mp::count_launch();
  MP_CUDA_TRY(cudaGetLastError());
  return MP_OK;
}

size_t mp_embedding_bwd_workspace_bytes(int64_t n, int64_t V, int64_t D) {
  if (n < 0 || V <= 0 || D <= 0 || n >= INT_MAX - kTileRound || V >= INT_MAX || D > INT_MAX - 8) return 0;
  return 4 * list_bytes(n) + part_bytes(n, D) + 16;
}

int mp_embedding_bwd(const void* ids, int id_bytes, const void* dY16, int64_t lddy, void* dW16, int64_t ldw,
                     int64_t n, int64_t V, int64_t D, int64_t pad_id, float scale, mp_state* state,
                     void* workspace, size_t workspace_bytes, void* stream) {
  if (!dW16 || (n > 0 && (!ids || !dY16)))
    return mp::set_error(MP_ERR_INVALID_ARG, "mp_embedding_bwd: null pointer");
  if (int rc = check("mp_embedding_bwd", ids, id_bytes, dY16, lddy, dW16, ldw, n, V, D)) return rc;
  if (n >= INT_MAX - kTileRound || V >= INT_MAX)
    return mp::set_error(MP_ERR_TOO_LARGE, "mp_embedding_bwd: n must be below 2^31 - %d and V below 2^31 - 1", kTileRound + 1);
  if (workspace && !mp::aligned16(workspace))
    return mp::set_error(MP_ERR_ALIGNMENT, "mp_embedding_bwd: workspace must be 16-byte aligned");
  const size_t need = mp_embedding_bwd_workspace_bytes(n, V, D);
  if (!workspace || workspace_bytes < need)
    return mp::set_error(MP_ERR_NOMEM, "mp_embedding_bwd: workspace of %zu bytes needed", need);
  if (int rc = mp::check_device()) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  mp_dev_state* dev = state ? state->dev : nullptr;
  char* ws = (char*)workspace;
  const size_t lb = list_bytes(n);
  SortArgs s{};
  s.ids = ids;
  s.id_bytes = id_bytes;
  s.n = (int)n;
  s.n_round = (int)round_up(n, kTileRound);
  s.V = (int)V;
  s.pad_id = pad_id;
  for (int i = 0; i < 2; ++i) {
    s.key[i] = (int*)(ws + 2 * i * lb);
    s.pos[i] = (int*)(ws + (2 * i + 1) * lb);
  }
  int bits = 1;                                  // of the largest key, V itself
  while (bits < 31 && ((int64_t)1 << bits) <= V) ++bits;
  s.passes = (bits + kMostBits - 1) / kMostBits;
  s.bits = (bits + s.passes - 1) / s.passes;
  s.dW = (uint16_t*)dW16;
  s.ldw = ldw;
  s.D = (int)D;
  s.st = dev;
  if (int rc = n < kManyTokens ? sort_launch<8>(s, st) : sort_launch<16>(s, st)) return rc;
  mp::count_launch();
  if (n == 0) return MP_OK;
  SumArgs m{};
  m.key = s.key[(s.passes & 1) ^ 1];
  m.pos = s.pos[(s.passes & 1) ^ 1];
  m.n_round = s.n_round;
  m.V = (int)V;
  m.tile = (int)tile_for(n, D);
  m.dY = (const uint16_t*)dY16;
  m.lddy = lddy;
  m.dW = (uint16_t*)dW16;
  m.ldw = ldw;
  m.D = (int)D;
  m.scale = scale;
  m.part = (float*)(ws + 4 * lb);
  m.D4 = (int)round_up(D, 8);
  m.st = dev;
  const int tiles = s.n_round / m.tile, vecs = m.D4 / 8, cols = vecs < kSumThreads ? vecs : kSumThreads;
  int groups = kSumThreads / cols;
  if (groups > kMostGroups) groups = kMostGroups;
  cudaLaunchConfig_t cfg = {};
  const unsigned across = (unsigned)((tiles + groups - 1) / groups);
  cfg.gridDim = dim3(across * (unsigned)((vecs + cols - 1) / cols), 1, 1);
  cfg.blockDim = dim3((unsigned)round_up(cols * groups, 32), 1, 1);
  cfg.dynamicSmemBytes = (size_t)(groups + 1) * m.tile * sizeof(int2);      // 33 KiB at most
  cfg.stream = st;
  cudaLaunchAttribute attr;            // resident early, waits on the device for the kernel before
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  MP_CUDA_TRY(cudaLaunchKernelEx(&cfg, mp_embedding_sum_kernel, m, cols, groups, tiles, across));
  mp::count_launch();
  if (tiles < 3) return MP_OK;         // no run over three tiles
  cfg.gridDim = dim3((unsigned)(((int64_t)m.D4 + kJoinCols - 1) / kJoinCols), (unsigned)(tiles < 148 ? tiles : 148), 1);
  cfg.blockDim = dim3(kJoinThreads, 1, 1);
  cfg.dynamicSmemBytes = 0;
  MP_CUDA_TRY(cudaLaunchKernelEx(&cfg, mp_embedding_join_kernel, m, tiles));
  mp::count_launch();
  return MP_OK;
}

}  // extern "C"

// dlm_kv_cache_evict, dlm_kv_cache_evict_q4: of every (layer, batch element, KV head) the rows of largest weight stay in the cache.
//
// Attention over the cache does not depend on the order of its rows (K rows carry their rotary positions), so what is kept is
// not pushed together: of the n = min(keep, length) rows to keep, those below n stay where they are, and the others move into the
// places of evicted rows below n.  No row is both read and written, so every row can move at the same time, and only
// n (1 - n / length) rows move where weights are in no order (half of what a compaction in order touches at n = length / 2).
//
// Two launches.  select: one block per (layer, batch element, KV head), the weights as ordered 32-bit integers in registers.
// The n-th largest is found two bits at a time from the top: 16 rounds of counting against three thresholds, each a warp
// reduction, an atomic per warp and a barrier -- no histogram, whose bins the weights of a softmax (a few exponents hold
// nearly all) would make collide.  Then ballots in index order number the holes and the rows to move.  move: a warp per 32
// places, 16-byte vectors, bound by HBM.
#include <math_constants.h>

#include "common.cuh"
#include "q4.cuh"

namespace {

constexpr int kPer = 16;             // weights per thread and tile
constexpr int kThreadsShort = 256, kThreadsLong = 1024;   // up to 4096 rows in one tile / 16384 a tile, any number of tiles
constexpr int kMaxTiles = 64;        // 1048576 rows
constexpr int kMoveThreads = 256;
constexpr int kMoveUnroll = 4;

struct EvictParams {
  const float* weight;               // may be weight_out, so not read through the read-only path
  float* weight_out;
  int32_t* kept_idx;
  const int32_t* cache_len;
  int batch, n_kv_heads, capacity, keep, protect_first, protect_last;
  int* status;
};

// Sums v over the block; `sums` is one of two slots used in turn and zero on entry, and the other is zeroed for the next call.
template <int kThreads>
__device__ __forceinline__ void block_sum3(int (&v)[3], int (*slots)[4], int turn) {
#pragma unroll
  for (int i = 0; i < 3; ++i) v[i] = __reduce_add_sync(0xffffffffu, v[i]);
  if ((threadIdx.x & 31) < 3) {
    const int mine = (threadIdx.x & 31) == 0 ? v[0] : (threadIdx.x & 31) == 1 ? v[1] : v[2];
    atomicAdd(&slots[turn % 3][threadIdx.x & 31], mine);
  }
  if (threadIdx.x < 4) slots[(turn + 1) % 3][threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 3; ++i) v[i] = slots[turn % 3][i];
}

// Exclusive prefix over the block's warps of a value that each warp has; `total` gets the sum.
template <int kThreads>
__device__ __forceinline__ int warp_prefix(int mine, int* buf, int& total) {
  constexpr int kWarps = kThreads / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  __syncthreads();
  if (lane == 0) buf[warp] = mine;
  __syncthreads();
  int x = lane < kWarps ? buf[lane] : 0, inc = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  total = __shfl_sync(0xffffffffu, inc, 31);
  return __shfl_sync(0xffffffffu, inc - x, warp);
}

// The weights of a cache that fits one tile are read once and stay in registers; longer ones are read again for every pass.
template <int kThreads>
__global__ void __launch_bounds__(kThreads) evict_select_kernel(const __grid_constant__ EvictParams p) {
  constexpr int kTile = kThreads * kPer;
  __shared__ int slots[3][4];
  __shared__ int prefix_buf[32];
  __shared__ int tile_equal[kMaxTiles], tile_holes[kMaxTiles];   // of the tiles before
  const int unit = blockIdx.x, b = (unit / p.n_kv_heads) % p.batch, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t below = (1u << lane) - 1u;   // the lanes before
  if (threadIdx.x < 12) slots[threadIdx.x / 4][threadIdx.x % 4] = 0;
  dlm_grid_dependency_wait();
  dlm_trigger_dependents();
  const int len = p.cache_len[b];
  int32_t* const kept = p.kept_idx + (size_t)unit * p.keep;
  if (len < 0 || len > p.capacity) {
    if (threadIdx.x == 0) dlm_set_status(p.status, DLM_ERR_CAPACITY);
    for (int i = threadIdx.x; i < p.keep; i += kThreads) kept[i] = -1;
    return;
  }
  const float* const w = p.weight + (size_t)unit * p.capacity;
  float* const w_out = p.weight_out ? p.weight_out + (size_t)unit * p.capacity : nullptr;
  const int n = min(p.keep, len), n_tiles = (len + kTile - 1) / kTile;
  // a warp's weights of a tile lie one after the other: element (e, lane) is row tile * kTile + warp * 32 * kPer + e * 32 + lane
  const int row0 = warp * 32 * kPer + lane;
  uint32_t key[kPer];
  auto load = [&](int tile) {
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int i = tile * kTile + row0 + e * 32;
      uint32_t k = 0;                                         // beyond the end: like NaN, below everything
      if (i < len) {
        const uint32_t u = __float_as_uint(w[i] + 0.f);       // -0 counts as 0
        k = (u & 0x7FFFFFFFu) > 0x7F800000u ? 0u : u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
        if (i < p.protect_first || i >= len - p.protect_last) k = 0xFFFFFFFFu;
      }
      key[e] = k;
    }
  };
  if (n_tiles <= 1) load(0);
  // the largest threshold that at least n keys reach (0, which all reach, to begin with)
  uint32_t threshold = 0;
  __syncthreads();
  if (n < len) {
    for (int round = 0; round < 16; ++round) {
      const int shift = 30 - 2 * round;
      const uint32_t t1 = threshold | (1u << shift), t2 = threshold | (2u << shift), t3 = threshold | (3u << shift);
      int c[3] = {0, 0, 0};
      for (int tile = 0; tile < n_tiles; ++tile) {
        if (n_tiles > 1) load(tile);
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          c[0] += key[e] >= t1;
          c[1] += key[e] >= t2;
          c[2] += key[e] >= t3;
        }
      }
      block_sum3<kThreads>(c, slots, round);
      threshold = c[2] >= n ? t3 : c[1] >= n ? t2 : c[0] >= n ? t1 : threshold;
    }
  }
  // how many keys at the threshold are kept: what those above leave of n, lowest rows first
  int above[3] = {0, 0, 0};
  for (int tile = 0; tile < n_tiles; ++tile) {
    if (n_tiles > 1) load(tile);
#pragma unroll
    for (int e = 0; e < kPer; ++e) above[0] += tile * kTile + row0 + e * 32 < len && key[e] > threshold;
  }
  block_sum3<kThreads>(above, slots, 16);
  const int at_threshold = n - above[0];
  // Which rows are kept (bit e of kept_mask), holes below n and rows to move numbered in index order: the k-th hole takes the k-th
  // row to move.  First the rows to move are listed, in the entries of kept_idx; then every place below n gets its entry.  A
  // hole's number is not above its index, so with the tiles taken from the last to the first, and reads before writes
  // within a tile, no entry of the list is replaced before it has been read.
  uint32_t kept_mask = 0;
  auto classify = [&](int tile, int equal_before) {   // returns the tile's keys at the threshold
    const int first = tile * kTile + row0;
    int eq = 0, total;
#pragma unroll
    for (int e = 0; e < kPer; ++e) eq += __popc(__ballot_sync(0xffffffffu, first + e * 32 < len && key[e] == threshold));
    int rank = equal_before + warp_prefix<kThreads>(eq, prefix_buf, total);
    kept_mask = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const bool in = first + e * 32 < len, equal = in && key[e] == threshold;
      const uint32_t ballot = __ballot_sync(0xffffffffu, equal);
      kept_mask |= (uint32_t)(in && (key[e] > threshold || (equal && rank + __popc(ballot & below) < at_threshold))) << e;
      rank += __popc(ballot);
    }
    return total;
  };
  int equal_before = 0, holes_before = 0, movers_before = 0;
  for (int tile = 0; tile < n_tiles; ++tile) {
    if (n_tiles > 1) load(tile);
    if (threadIdx.x == 0) {
      tile_equal[tile] = equal_before;
      tile_holes[tile] = holes_before;
    }
    equal_before += classify(tile, equal_before);
    const int first = tile * kTile + row0;
    int holes = 0, movers = 0, total;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int i = first + e * 32;
      const bool k = (kept_mask >> e) & 1u;
      holes += __popc(__ballot_sync(0xffffffffu, i < n && !k));
      movers += __popc(__ballot_sync(0xffffffffu, i >= n && k));
    }
    if (n_tiles > 1) {
      warp_prefix<kThreads>(holes, prefix_buf, total);
      holes_before += total;
    }
    int at = movers_before + warp_prefix<kThreads>(movers, prefix_buf, total);
    movers_before += total;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int i = first + e * 32;
      const bool mover = i >= n && ((kept_mask >> e) & 1u);
      const uint32_t ballot = __ballot_sync(0xffffffffu, mover);
      if (mover) kept[at + __popc(ballot & below)] = i;
      at += __popc(ballot);
    }
  }
  for (int tile = n_tiles - 1; tile >= 0; --tile) {
    if (tile * kTile >= n) continue;
    if (n_tiles > 1) {
      __syncthreads();   // tile_equal, and what the tile before has written
      load(tile);
      classify(tile, tile_equal[tile]);
    }
    const int first = tile * kTile + row0;
    int holes = 0, total;
#pragma unroll
    for (int e = 0; e < kPer; ++e) holes += __popc(__ballot_sync(0xffffffffu, first + e * 32 < n && !((kept_mask >> e) & 1u)));
    int at = (n_tiles > 1 ? tile_holes[tile] : 0) + warp_prefix<kThreads>(holes, prefix_buf, total);   // (its barriers: the list is written)
    int src[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int i = first + e * 32;
      const bool hole = i < n && !((kept_mask >> e) & 1u);
      const uint32_t ballot = __ballot_sync(0xffffffffu, hole);
      src[e] = hole ? kept[at + __popc(ballot & below)] : i;
      at += __popc(ballot);
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int i = first + e * 32;
      if (i < n) {
        kept[i] = src[e];
        if (w_out) w_out[i] = w[src[e]];   // src is i, or not below n: w_out may be w
      }
    }
  }
  __syncthreads();
  for (int i = n + threadIdx.x; i < p.keep; i += kThreads) kept[i] = -1;
  if (w_out)
    for (int i = n + threadIdx.x; i < len; i += kThreads) w_out[i] = 0.f;
}

// The rows to their places, and the new lengths.  A warp has 32 places of a unit; the rows that move are gathered to the front
// and taken as 16-byte vectors, a row's K and V one after the other.
struct MoveParams {
  uint4* k;
  uint4* v;
  uint8_t* k_scale;     // 4-bit cache, else NULL
  uint8_t* v_scale;
  int32_t* cache_len;
  const int32_t* kept_idx;
  int batch, capacity, keep, vec_per_row, scale_bytes;
  FastDiv by_chunks, by_row_pair;   // 32-place chunks of a unit; vectors of a row's K and V
  long long n_warps;
};

__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const __grid_constant__ MoveParams p) {
  __shared__ int2 moves[kMoveThreads / 32][32];   // (from, to)
  dlm_grid_dependency_wait();
  dlm_trigger_dependents();
  if (blockIdx.x == 0)
    for (int b = threadIdx.x; b < p.batch; b += kMoveThreads) {
      const int len = p.cache_len[b];
      if (len > p.keep && len <= p.capacity) p.cache_len[b] = p.keep;
    }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long id = (long long)blockIdx.x * (kMoveThreads / 32) + warp;
  if (id >= p.n_warps) return;
  int chunk;
  const int unit = p.by_chunks.divmod((int)id, chunk);
  const int to = chunk * 32 + lane;
  const int from = to < p.keep ? p.kept_idx[(size_t)unit * p.keep + to] : -1;
  const bool moves_on = from >= 0 && from != to;
  const uint32_t mask = __ballot_sync(0xffffffffu, moves_on);
  if (mask == 0) return;
  const size_t row0 = (size_t)unit * p.capacity;
  if (moves_on) moves[warp][__popc(mask & ((1u << lane) - 1u))] = make_int2(from, to);
  if (moves_on && p.k_scale) {
    if (p.scale_bytes == 4) {
      reinterpret_cast<uint32_t*>(p.k_scale)[row0 + to] = reinterpret_cast<const uint32_t*>(p.k_scale)[row0 + from];
      reinterpret_cast<uint32_t*>(p.v_scale)[row0 + to] = reinterpret_cast<const uint32_t*>(p.v_scale)[row0 + from];
    } else {
      reinterpret_cast<uint16_t*>(p.k_scale)[row0 + to] = reinterpret_cast<const uint16_t*>(p.k_scale)[row0 + from];
      reinterpret_cast<uint16_t*>(p.v_scale)[row0 + to] = reinterpret_cast<const uint16_t*>(p.v_scale)[row0 + from];
    }
  }
  __syncwarp();
  const int n_vec = __popc(mask) * 2 * p.vec_per_row;
  for (int base = lane; base < n_vec; base += 32 * kMoveUnroll) {
    uint4 x[kMoveUnroll];
    uint4* dst[kMoveUnroll];
#pragma unroll
    for (int u = 0; u < kMoveUnroll; ++u) {
      const int item = base + u * 32;
      dst[u] = nullptr;
      if (item < n_vec) {
        int vec;
        const int2 m = moves[warp][p.by_row_pair.divmod(item, vec)];
        uint4* t = p.k;
        if (vec >= p.vec_per_row) {
          vec -= p.vec_per_row;
          t = p.v;
        }
        x[u] = __ldcs(t + (row0 + m.x) * p.vec_per_row + vec);
        dst[u] = t + (row0 + m.y) * p.vec_per_row + vec;
      }
    }
#pragma unroll
    for (int u = 0; u < kMoveUnroll; ++u)
      if (dst[u]) *dst[u] = x[u];
  }
}

template <typename Cache>
int evict(dlm_ctx* ctx, const Cache* cache, uint8_t* k_scale, uint8_t* v_scale, int row_bytes, const float* weight, int keep,
          int protect_first, int protect_last, int32_t* kept_idx, float* weight_out, void* stream) {
  if (keep <= 0 || keep > cache->capacity || protect_first < 0 || protect_last < 0 || protect_first > keep || protect_last > keep - protect_first)
    return DLM_ERR_SHAPE;
  const long long units = (long long)cache->n_layers * cache->batch * cache->n_kv_heads, chunks = (keep + 31) / 32;
  if (units * chunks >= (1LL << 31) - kMoveThreads || (cache->capacity + kThreadsLong * kPer - 1) / (kThreadsLong * kPer) > kMaxTiles) return DLM_ERR_UNSUPPORTED;
  DLM_DEVICE_TRY(ctx);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  EvictParams e;
  e.weight = weight;
  e.weight_out = weight_out;
  e.kept_idx = kept_idx;
  e.cache_len = cache->cache_len;
  e.batch = cache->batch;
  e.n_kv_heads = cache->n_kv_heads;
  e.capacity = cache->capacity;
  e.keep = keep;
  e.protect_first = protect_first;
  e.protect_last = protect_last;
  e.status = &ctx->words->status;
  if (cache->capacity <= kThreadsShort * kPer)
    DLM_CUDA_TRY(dlm_launch(evict_select_kernel<kThreadsShort>, dim3((unsigned)units), dim3(kThreadsShort), 0, st, e));
  else
    DLM_CUDA_TRY(dlm_launch(evict_select_kernel<kThreadsLong>, dim3((unsigned)units), dim3(kThreadsLong), 0, st, e));
  MoveParams m;
  m.k = static_cast<uint4*>(cache->k);
  m.v = static_cast<uint4*>(cache->v);
  m.k_scale = k_scale;
  m.v_scale = v_scale;
  m.cache_len = cache->cache_len;
  m.kept_idx = kept_idx;
  m.batch = cache->batch;
  m.capacity = cache->capacity;
  m.keep = keep;
  m.vec_per_row = row_bytes / 16;
  m.scale_bytes = cache->head_dim / q4::kGroup;
  m.by_chunks = make_fast_div((int)chunks);
  m.by_row_pair = make_fast_div(2 * m.vec_per_row);
  m.n_warps = units * chunks;
  const unsigned blocks = (unsigned)((m.n_warps + kMoveThreads / 32 - 1) / (kMoveThreads / 32));
  DLM_CUDA_TRY(dlm_launch(evict_move_kernel, dim3(blocks), dim3(kMoveThreads), 0, st, m));
  return dlm_launch_ok(ctx, 2);
}

}  // namespace

extern "C" int dlm_kv_cache_evict(dlm_ctx* ctx, const dlm_kv_cache* cache, const float* weight, int keep, int protect_first,
                                  int protect_last, int32_t* kept_idx, float* weight_out, void* stream) {
  if (!ctx || !cache || !cache->k || !cache->v || !cache->cache_len || !weight || !kept_idx) return DLM_ERR_NULL;
  if (cache->n_layers <= 0 || cache->batch <= 0 || cache->n_kv_heads <= 0 || cache->capacity <= 0 || cache->head_dim <= 0) return DLM_ERR_SHAPE;
  if (cache->head_dim % 8 != 0 || (((uintptr_t)cache->k | (uintptr_t)cache->v) & 15)) return DLM_ERR_UNSUPPORTED;
  return evict(ctx, cache, nullptr, nullptr, cache->head_dim * 2, weight, keep, protect_first, protect_last, kept_idx, weight_out, stream);
}

extern "C" int dlm_kv_cache_evict_q4(dlm_ctx* ctx, const dlm_kv_cache_q4* cache, const float* weight, int keep, int protect_first,
                                     int protect_last, int32_t* kept_idx, float* weight_out, void* stream) {
  if (!ctx || !weight || !kept_idx) return DLM_ERR_NULL;
  const int rc = dlm_check_q4(cache);
  if (rc != DLM_OK) return rc;
  return evict(ctx, cache, static_cast<uint8_t*>(cache->k_scale), static_cast<uint8_t*>(cache->v_scale), cache->head_dim / 2, weight, keep,
               protect_first, protect_last, kept_idx, weight_out, stream);
}

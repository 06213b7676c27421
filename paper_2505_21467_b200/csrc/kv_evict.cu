// dlm_kv_cache_evict, dlm_kv_cache_evict_q4: of every (layer, batch element, KV head) the rows of largest weight stay in the cache.
//
// Attention over the cache does not depend on the order of its rows (K rows carry their rotary positions), so what is kept is
// not pushed together: of the n = min(keep, length) rows to keep, those below n stay where they are, and the others move into the
// places of evicted rows below n.  No row is both read and written, so every row can move at the same time, and only
// n (1 - n / length) rows move where weights are in no order (half of what a compaction in order touches at n = length / 2).
//
// Two launches.  select: one block per (layer, batch element, KV head), the weights as ordered 32-bit integers in registers, 8 a thread
// for as many threads as that takes, 16 beyond 8192 rows.  The n-th largest: a histogram with a bin per thread over the keys' range (and,
// while the bin that holds it has more than 256 keys, over that bin's), then the keys of that bin are ranked against each other (16
// rounds of counting against three thresholds instead: 36.9 us for 112 units of 16301 weights against 29.9, 51.5 us for 896 units of 1152 against 22.4).
// Then ballots in index order number the holes and the rows to move.  move: a warp per 32 places, 16-byte vectors.
//
// 112 units of 16301 4-bit rows, 8192 kept: 62 us (2.3 TB/s of what has to be read and written; by the profiler select 25 us, a chain of barriers
// on 112 SMs, and move 30 us); 896 units of 1152 bf16 rows, 700 kept: 63 us (3.4 TB/s, 0.53 of a copy's rate; 43 % of the issue slots).
#include <math_constants.h>

#include "common.cuh"
#include "q4.cuh"

namespace {

constexpr int kLongTile = 16384;     // rows of a tile where there are several: 1024 threads with 16 weights each
constexpr int kMaxTiles = 64;        // 1048576 rows
constexpr int kMoveThreads = 256;
constexpr int kMoveUnroll = 4;

struct RowParams {
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

struct EvictParams {
  const float* weight;               // may be weight_out, so not read through the read-only path
  float* weight_out;
  int32_t* kept_idx;
  const int32_t* cache_len;
  int batch, n_kv_heads, capacity, keep, protect_first, protect_last;
  int* status;
  unsigned int* ticket;
  RowParams rows;                    // the block moves its unit's rows itself (kMoves)
};

// One warp: the rows that 32 places of a unit (`from`: what lane's place `to` is to hold, -1 for nothing) get from elsewhere.  Those that move
// are gathered to the front and taken as 16-byte vectors, a row's K and V one after the other.
__device__ __forceinline__ void move_rows(const RowParams& p, size_t row0, int from, int to, int2* moves) {
  const int lane = threadIdx.x & 31;
  const bool moves_on = from >= 0 && from != to;
  const uint32_t mask = __ballot_sync(0xffffffffu, moves_on);
  if (mask == 0) return;
  if (moves_on) moves[__popc(mask & ((1u << lane) - 1u))] = make_int2(from, to);
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
        const int2 m = moves[p.by_row_pair.divmod(item, vec)];
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
  __syncwarp();
}

__device__ __forceinline__ void set_lengths(const RowParams& p) {
  for (int b = threadIdx.x; b < p.batch; b += blockDim.x) {
    const int len = p.cache_len[b];
    if (len > p.keep && len <= p.capacity) p.cache_len[b] = p.keep;
  }
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
// kMoves: the block moves its unit's rows too, and the last one to have read its length sets the new ones.
template <int kThreads, int kPer, bool kMoves>
__global__ void __launch_bounds__(kThreads) evict_select_kernel(const __grid_constant__ EvictParams p) {
  constexpr int kTile = kThreads * kPer;
  constexpr int kRanked = kThreads < 256 ? kThreads : 256;   // keys that are ranked against each other
  __shared__ int bins[kThreads];
  __shared__ int prefix_buf[32];
  __shared__ int tile_equal[kMaxTiles], tile_holes[kMaxTiles];   // of the tiles before
  __shared__ unsigned int range[2], ranked[kRanked];
  __shared__ unsigned int found_bin, found_key;
  __shared__ int found_above, found_count, n_ranked;
  __shared__ int moving[kTile / 2];              // one tile: the rows to move
  __shared__ int2 moves[kMoves ? kThreads / 32 : 1][32];
  __shared__ bool is_last;
  const int unit = blockIdx.x, b = (unit / p.n_kv_heads) % p.batch, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t below = (1u << lane) - 1u;      // the lanes before
  if (threadIdx.x < 2) range[threadIdx.x] = threadIdx.x ? 0u : 0xFFFFFFFFu;
  dlm_grid_dependency_wait();
  dlm_trigger_dependents();
  const int len = p.cache_len[b];
  int32_t* const kept = p.kept_idx + (size_t)unit * p.keep;
  if (kMoves) {
    __syncthreads();   // every thread has the length
    if (threadIdx.x == 0) {
      unsigned int t;
      asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(t) : "l"(p.ticket) : "memory");
      is_last = t == gridDim.x - 1;
    }
    __syncthreads();
    if (is_last) {
      set_lengths(p.rows);
      if (threadIdx.x == 0) *p.ticket = 0;
    }
  }
  if (len < 0 || len > p.capacity) {
    if (threadIdx.x == 0) dlm_set_status(p.status, DLM_ERR_CAPACITY);
    for (int i = threadIdx.x; i < p.keep; i += kThreads) kept[i] = -1;
    return;
  }
  const float* const w = p.weight + (size_t)unit * p.capacity;
  float* const w_out = p.weight_out ? p.weight_out + (size_t)unit * p.capacity : nullptr;
  const int n = min(p.keep, len), n_tiles = (len + kTile - 1) / kTile;
  int32_t* const list = n_tiles > 1 ? kept : moving;
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

  // `threshold`: the n-th largest key; n_above keys are above it, and of those at it the first n - n_above are kept (all, if `whole`)
  uint32_t threshold = 0;
  int n_above = 0;
  bool whole = true;
  const int n_protected = p.protect_first + p.protect_last;   // (fewer than len where anything is evicted)
  __syncthreads();
  if (n < len && n == n_protected) {
    threshold = 0xFFFFFFFFu;
  } else if (n < len) {
    uint32_t lo = 0xFFFFFFFFu, hi = 0;
    n_above = n_protected;
    for (int tile = 0; tile < n_tiles; ++tile) {
      if (n_tiles > 1) load(tile);
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        if (tile * kTile + row0 + e * 32 < len && key[e] != 0xFFFFFFFFu) {
          lo = min(lo, key[e]);
          hi = max(hi, key[e]);
        }
      }
    }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    if (lane == 0) {
      atomicMin(&range[0], lo);
      atomicMax(&range[1], hi);
    }
    __syncthreads();
    lo = range[0];
    hi = range[1];                                             // the key sought is in [lo, hi], n_above keys are above hi
    for (;;) {
      // bin i: keys lo + i * size .. ; the last bins may be empty
      const uint32_t size = (hi - lo) / kThreads + 1u;
      const float inv = 1.f / (float)size;
      bins[threadIdx.x] = 0;
      if (threadIdx.x == 0) n_ranked = 0;
      __syncthreads();
      // (a float quotient that is off by one only moves the border of two bins, alike for equal keys and in order: it is the
      // same function below)
      auto bin_of = [&](uint32_t k) { return min((int)((float)(k - lo) * inv), kThreads - 1); };
      for (int tile = 0; tile < n_tiles; ++tile) {
        if (n_tiles > 1) load(tile);
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          const bool in = tile * kTile + row0 + e * 32 < len && key[e] >= lo && key[e] <= hi;
          const int bin = in ? bin_of(key[e]) : -1;
          // keys that are all alike would add one after the other
          const int same = __shfl_sync(0xffffffffu, bin, 0);
          if (__all_sync(0xffffffffu, bin == same)) {
            if (lane == 0 && in) atomicAdd(&bins[bin], 32);
          } else if (in) {
            atomicAdd(&bins[bin], 1);
          }
        }
      }
      __syncthreads();
      // thread t has the t-th bin from the top
      const int mine = bins[kThreads - 1 - threadIdx.x];
      int inc = mine, total;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
      }
      const int above = n_above + warp_prefix<kThreads>(__shfl_sync(0xffffffffu, inc, 31), prefix_buf, total) + inc - mine;
      if (above < n && n <= above + mine) {
        found_bin = kThreads - 1 - threadIdx.x;
        found_above = above;
        found_count = mine;
      }
      __syncthreads();
      const int bin = (int)found_bin, count = found_count;
      n_above = found_above;
      if (size == 1u) {                                        // one value
        threshold = lo + bin;
        whole = n_above + count == n;
        break;
      }
      // the keys of the bin: ranked if they are few, else the smallest and largest of them are the next range
      uint32_t bin_lo = 0xFFFFFFFFu, bin_hi = 0;
      for (int tile = 0; tile < n_tiles; ++tile) {
        if (n_tiles > 1) load(tile);
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          if (tile * kTile + row0 + e * 32 < len && key[e] >= lo && key[e] <= hi && bin_of(key[e]) == bin) {
            if (count <= kRanked) ranked[atomicAdd(&n_ranked, 1)] = key[e];
            bin_lo = min(bin_lo, key[e]);
            bin_hi = max(bin_hi, key[e]);
          }
        }
      }
      if (count <= kRanked) {
        __syncthreads();
        if (threadIdx.x < count) {
          const uint32_t k = ranked[threadIdx.x];
          int greater = 0, equal = 0;
          for (int i = 0; i < count; ++i) {
            greater += ranked[i] > k;
            equal += ranked[i] == k;
          }
          if (n_above + greater < n && n <= n_above + greater + equal) {   // alike for all threads with this key
            found_key = k;
            found_above = n_above + greater;
            found_count = equal;
          }
        }
        __syncthreads();
        threshold = found_key;
        n_above = found_above;
        whole = n_above + found_count == n;
        break;
      }
      if (threadIdx.x < 2) range[threadIdx.x] = threadIdx.x ? 0u : 0xFFFFFFFFu;
      __syncthreads();
      bin_lo = __reduce_min_sync(0xffffffffu, bin_lo);
      bin_hi = __reduce_max_sync(0xffffffffu, bin_hi);
      if (lane == 0) {
        atomicMin(&range[0], bin_lo);
        atomicMax(&range[1], bin_hi);
      }
      __syncthreads();
      lo = range[0];
      hi = range[1];
    }
  }
  const int at_threshold = n - n_above;

  // Which rows are kept, 32 rows a word; holes below n and rows to move numbered in index order: the k-th hole takes the k-th row to
  // move.  First the rows to move are listed (several tiles: in the entries of kept_idx), then every place below n gets its entry.  A
  // hole's number is not above its index, so with the tiles taken from the last to the first, and reads before writes
  // within a tile, no entry of the list is replaced before it has been read.
  uint32_t kept_rows[kPer];
  auto classify = [&](int tile, int equal_before) {   // returns the tile's keys at the threshold
    int total = 0;
    if (whole) {
#pragma unroll
      for (int e = 0; e < kPer; ++e) kept_rows[e] = __ballot_sync(0xffffffffu, tile * kTile + row0 + e * 32 < len && key[e] >= threshold);
    } else {
      int eq = 0;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        kept_rows[e] = __ballot_sync(0xffffffffu, tile * kTile + row0 + e * 32 < len && key[e] == threshold);
        eq += __popc(kept_rows[e]);
      }
      int rank = equal_before + warp_prefix<kThreads>(eq, prefix_buf, total);
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const uint32_t equal = kept_rows[e];
        const bool k = tile * kTile + row0 + e * 32 < len &&
                       (key[e] > threshold || ((equal >> lane & 1u) && rank + __popc(equal & below) < at_threshold));
        kept_rows[e] = __ballot_sync(0xffffffffu, k);
        rank += __popc(equal);
      }
    }
    return total;
  };
  // the rows below n of the 32 that start at element e
  auto front = [&](int tile, int e) {
    const int rows = n - (tile * kTile + warp * 32 * kPer + e * 32);
    return rows <= 0 ? 0u : rows >= 32 ? 0xFFFFFFFFu : (1u << rows) - 1u;
  };
  int equal_before = 0, holes_before = 0, movers_before = 0;
  for (int tile = 0; tile < n_tiles; ++tile) {
    if (n_tiles > 1) load(tile);
    if (threadIdx.x == 0) {
      tile_equal[tile] = equal_before;
      tile_holes[tile] = holes_before;
    }
    equal_before += classify(tile, equal_before);
    int holes = 0, movers = 0, total;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      holes += __popc(~kept_rows[e] & front(tile, e));
      movers += __popc(kept_rows[e] & ~front(tile, e));
    }
    if (n_tiles > 1) {
      warp_prefix<kThreads>(holes, prefix_buf, total);
      holes_before += total;
    }
    int at = movers_before + warp_prefix<kThreads>(movers, prefix_buf, total);
    movers_before += total;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const uint32_t m = kept_rows[e] & ~front(tile, e);
      if (m >> lane & 1u) list[at + __popc(m & below)] = tile * kTile + row0 + e * 32;
      at += __popc(m);
    }
  }
  for (int tile = n_tiles - 1; tile >= 0; --tile) {
    if (tile * kTile >= n) continue;
    if (n_tiles > 1) {
      __syncthreads();   // tile_equal, and what the tile before has written
      load(tile);
      classify(tile, tile_equal[tile]);
    }
    int holes = 0, total;
#pragma unroll
    for (int e = 0; e < kPer; ++e) holes += __popc(~kept_rows[e] & front(tile, e));
    int at = (n_tiles > 1 ? tile_holes[tile] : 0) + warp_prefix<kThreads>(holes, prefix_buf, total);   // (its barriers: the list is written)
    int src[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const uint32_t h = ~kept_rows[e] & front(tile, e);
      src[e] = h >> lane & 1u ? list[at + __popc(h & below)] : tile * kTile + row0 + e * 32;
      at += __popc(h);
    }
    if (n_tiles > 1) __syncthreads();
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int i = tile * kTile + row0 + e * 32;
      if (i < n) {
        kept[i] = src[e];
        if (w_out && (w_out != w || src[e] != i)) w_out[i] = w[src[e]];   // src is i, or not below n: w_out may be w
      }
    }
  }
  __syncthreads();
  for (int i = n + threadIdx.x; i < p.keep; i += kThreads) kept[i] = -1;
  if (w_out)
    for (int i = n + threadIdx.x; i < len; i += kThreads) w_out[i] = 0.f;
  if (kMoves && n < len)
    for (int to = warp * 32 + lane; to - lane < n; to += kThreads)
      move_rows(p.rows, (size_t)unit * p.capacity, to < n ? kept[to] : -1, to, moves[warp]);
}

// The rows to their places, and the new lengths.
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const __grid_constant__ RowParams p) {
  __shared__ int2 moves[kMoveThreads / 32][32];   // (from, to)
  dlm_grid_dependency_wait();
  dlm_trigger_dependents();
  if (blockIdx.x == 0) set_lengths(p);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long id = (long long)blockIdx.x * (kMoveThreads / 32) + warp;
  if (id >= p.n_warps) return;
  int chunk;
  const int unit = p.by_chunks.divmod((int)id, chunk), to = chunk * 32 + lane;
  move_rows(p, (size_t)unit * p.capacity, to < p.keep ? p.kept_idx[(size_t)unit * p.keep + to] : -1, to, moves[warp]);
}

template <typename Cache>
int evict(dlm_ctx* ctx, const Cache* cache, uint8_t* k_scale, uint8_t* v_scale, int row_bytes, const float* weight, int keep,
          int protect_first, int protect_last, int32_t* kept_idx, float* weight_out, void* stream) {
  if (keep <= 0 || keep > cache->capacity || protect_first < 0 || protect_last < 0 || protect_first > keep || protect_last > keep - protect_first)
    return DLM_ERR_SHAPE;
  const long long units = (long long)cache->n_layers * cache->batch * cache->n_kv_heads, chunks = (keep + 31) / 32;
  if (units * chunks >= (1LL << 31) - kMoveThreads || (cache->capacity + kLongTile - 1) / kLongTile > kMaxTiles) return DLM_ERR_UNSUPPORTED;
  DLM_DEVICE_TRY(ctx);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  RowParams m;
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
  e.ticket = &ctx->words->commit_ticket;
  e.rows = m;
  // With a unit for every SM each block moves its rows itself (896 units of 1152 rows: 62.8 us, with a second launch 64.4); with fewer the moves are
  // spread over all SMs by a second launch (112 units of 16301 rows: 65.5, in one launch 66.0).
  const bool fused = units >= ctx->num_sms;
  const int cap = cache->capacity, which = cap <= 1024 ? 0 : cap <= 2048 ? 1 : cap <= 4096 ? 2 : cap <= 8192 ? 3 : 4;
  // as few threads as hold a whole cache, 8 weights each; the longest block with 16
  void (*const kernels[2][5])(const EvictParams) = {
      {evict_select_kernel<128, 8, false>, evict_select_kernel<256, 8, false>, evict_select_kernel<512, 8, false>,
       evict_select_kernel<1024, 8, false>, evict_select_kernel<1024, 16, false>},
      {evict_select_kernel<128, 8, true>, evict_select_kernel<256, 8, true>, evict_select_kernel<512, 8, true>,
       evict_select_kernel<1024, 8, true>, evict_select_kernel<1024, 16, true>}};
  const int threads[5] = {128, 256, 512, 1024, 1024};
  DLM_CUDA_TRY(dlm_launch(kernels[fused][which], dim3((unsigned)units), dim3(threads[which]), 0, st, e));
  if (fused) return dlm_launch_ok(ctx, 1);
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

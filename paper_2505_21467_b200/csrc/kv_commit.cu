// dlm_kv_cache_commit: row gather/scatter of fresh K/V into the device-resident cache
// (Sec. 3.2.1: saving K/V at initialisation, freezing a finished block); dlm_kv_cache_commit_q4, the same into a cache of 4
// bits, and dlm_kv_cache_read_q4, rows of that cache back as bf16.
//
// Pure data movement, bound by HBM.  One work item is one 16-byte vector of one K row and
// the matching vector of the V row; items are ordered [layer][batch][head][row][vector] so
// that consecutive threads touch consecutive addresses whenever the row indices are
// consecutive (refresh / append).  The item list is cut into equal contiguous ranges, one per
// block, and the grid is one resident wave, so every SM moves the same number of bytes; a
// thread keeps kUnroll independent 16-byte loads of K and of V in flight.  Item numbers are
// decoded with 32-bit reciprocals whenever the call has fewer than 2^31 items (64-bit divisions
// by run-time divisors cost more than the copy).  The last block to finish advances cache_len.
//
// Into 4 bits, 28 layers x 8 x 4 heads of 1024 rows: 155 us with the L2 cold, and 97 us back to bf16 (244 together in a row, 4.4 TB/s, 0.68 of a
// copy's rate); what is left is decoding item numbers and quantising (the first form, an item a vector, took 341).
#include "common.cuh"
#include "q4.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;
// 4-bit cache: an item is two vectors (8 values each) of a row, one from either half of it, so that decoding an item's number, as
// much work as quantising a vector, is shared by twice as many values; half as many items are in flight a thread.
constexpr int kUnrollQ4 = 2;

struct CommitParams {
  void* cache_k;         // 16-byte vectors; 4-bit cache: a 32-bit word for each vector of a source row, a scale byte for every fourth
  void* cache_v;
  uint8_t* k_scale;
  uint8_t* v_scale;
  int32_t* cache_len;
  const uint4* k_new;
  const uint4* v_new;
  const int32_t* src_idx;
  const int32_t* dst_pos;
  const int32_t* n_rows;
  int n_max, src_len, advance_len, layer_begin, n_layers_call, dst_mode;
  int batch, n_kv_heads, capacity;
  int vec_per_row;       // items of a row: its vectors of 16 bytes; 4-bit cache: half of them
  FastDiv by_vec, by_rows, by_heads, by_batch;   // vec_per_row, n_max, n_kv_heads, batch
  long long n_items;     // n_layers_call * batch * heads * n_max * vec_per_row
  long long per_block;   // items per block (a multiple of 32)
  int* status;
  unsigned int* ticket;
};

// n(b), validated; -1 if this batch element must be skipped entirely.
__device__ __forceinline__ int valid_rows(const CommitParams& p, int b, int len0) {
  const int n = p.n_rows ? p.n_rows[b] : p.n_max;
  if (n < 0 || n > p.n_max) return -1;
  const bool append = p.dst_pos == nullptr && p.dst_mode == DLM_DST_APPEND;
  if ((append || p.advance_len) && (len0 < 0 || (long long)len0 + n > p.capacity)) return -1;
  return n;
}

// Where one item comes from and goes to (vector indices), or to = -1: nothing to move.
struct Move {
  long long from, to;
  int vec;   // number of the item in its row
};

// Idx int: item numbers below 2^31, decoded with host-prepared reciprocals.
template <typename Idx>
__device__ __forceinline__ Move find_move(const CommitParams& p, Idx item) {
  Move mv = {0, -1, 0};
  int vec, r, h, b, lc;   // vector of the row, row, head, batch element, layer within the call
  if (sizeof(Idx) == 4) {
    lc = p.by_batch.divmod(p.by_heads.divmod(p.by_rows.divmod(p.by_vec.divmod((int)item, vec), r), h), b);
  } else {
    long long rest = (long long)item;
    vec = (int)(rest % p.vec_per_row);
    rest /= p.vec_per_row;
    r = (int)(rest % p.n_max);
    rest /= p.n_max;
    h = (int)(rest % p.n_kv_heads);
    rest /= p.n_kv_heads;
    b = (int)(rest % p.batch);
    lc = (int)(rest / p.batch);
  }
  // the index words are read before the row count is checked (their slots always exist), so the
  // three small loads are in flight together instead of one after the other
  const int len0 = p.cache_len[b];
  const long long src = p.src_idx ? p.src_idx[(long long)b * p.n_max + r] : r;
  const long long dst_given = p.dst_pos ? p.dst_pos[(long long)b * p.n_max + r] : 0;
  const int n = valid_rows(p, b, len0);
  if (n < 0) {
    if (r == 0 && vec == 0 && h == 0 && lc == 0) dlm_set_status(p.status, DLM_ERR_CAPACITY);
    return mv;
  }
  if (r >= n) return mv;
  const long long dst = p.dst_pos ? dst_given : (long long)len0 + (p.dst_mode == DLM_DST_WINDOW ? src : r);
  if (src < 0 || src >= p.src_len || dst < 0 || dst >= p.capacity) {
    if (vec == 0 && h == 0 && lc == 0) dlm_set_status(p.status, DLM_ERR_INDEX);
    return mv;
  }
  mv.vec = vec;
  mv.from = ((((long long)lc * p.batch + b) * p.n_kv_heads + h) * p.src_len + src) * p.vec_per_row + vec;
  mv.to = ((((long long)(lc + p.layer_begin) * p.batch + b) * p.n_kv_heads + h) * p.capacity + dst) * p.vec_per_row + vec;
  return mv;
}

// The last block to get here advances cache_len.  That needs every block to have read it, not to have stored its rows: whoever
// reads the rows is ordered behind the kernel.
__device__ __forceinline__ void advance_when_last(const CommitParams& p) {
  __shared__ bool is_last;
  __syncthreads();
  if (threadIdx.x == 0) {
    unsigned int t;
    asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(t) : "l"(p.ticket) : "memory");
    is_last = t == gridDim.x - 1;
  }
  __syncthreads();
  if (!is_last) return;
  for (int b = threadIdx.x; b < p.batch; b += kThreads) {
    const int len0 = p.cache_len[b];
    const int n = valid_rows(p, b, len0);
    if (n > 0) p.cache_len[b] = len0 + n;
  }
  if (threadIdx.x == 0) *p.ticket = 0;
}

// What an item brings: vectors of K and of V.
template <bool kQ4>
struct Item {
  uint4 k[kQ4 ? 2 : 1], v[kQ4 ? 2 : 1];
};
// 4 bits: number of an item's first vector (or of its word in the cache), given row * (items of a row) + item in the row
__device__ __forceinline__ long long first_vector(long long at, int vec) { return 2 * at - vec; }

template <bool kQ4>
__device__ __forceinline__ void load_item(const CommitParams& p, const Move& mv, Item<kQ4>& x) {
  if (mv.to < 0) {
    if (kQ4) x.k[0] = x.v[0] = x.k[kQ4 ? 1 : 0] = x.v[kQ4 ? 1 : 0] = make_uint4(0, 0, 0, 0);
    return;
  }
  const long long at = kQ4 ? first_vector(mv.from, mv.vec) : mv.from;
  x.k[0] = __ldcs(p.k_new + at);
  x.v[0] = __ldcs(p.v_new + at);
  if (kQ4) {
    x.k[kQ4 ? 1 : 0] = __ldcs(p.k_new + at + p.vec_per_row);
    x.v[kQ4 ? 1 : 0] = __ldcs(p.v_new + at + p.vec_per_row);
  }
}

// 4-bit cache: four neighbouring lanes have a group of 32 values, which lies in one row (a row's items are a multiple of four), so all four
// have a destination or none has; every lane of the warp calls this.
template <bool kQ4>
__device__ __forceinline__ void store_item(const CommitParams& p, const Move& mv, const Item<kQ4>& x) {
  if (kQ4) {
    const long long at = first_vector(mv.to, mv.vec);
#pragma unroll
    for (int h = 0; h < (kQ4 ? 2 : 1); ++h) {
      uint32_t kb, vb;
      const uint32_t kw = q4::encode8(x.k[h], kb), vw = q4::encode8(x.v[h], vb);
      if (mv.to < 0) continue;
      const long long to = at + h * p.vec_per_row;
      static_cast<uint32_t*>(p.cache_k)[to] = kw;
      static_cast<uint32_t*>(p.cache_v)[to] = vw;
      if ((mv.vec & 3) == 0) {
        p.k_scale[to >> 2] = (uint8_t)kb;
        p.v_scale[to >> 2] = (uint8_t)vb;
      }
    }
  } else if (mv.to >= 0) {
    static_cast<uint4*>(p.cache_k)[mv.to] = x.k[0];
    static_cast<uint4*>(p.cache_v)[mv.to] = x.v[0];
  }
}

template <typename Idx, bool kQ4>
__global__ void __launch_bounds__(kThreads, 4) kv_commit_kernel(const __grid_constant__ CommitParams p) {
  dlm_grid_dependency_wait();
  dlm_trigger_dependents();
  const Idx begin = (Idx)blockIdx.x * (Idx)p.per_block;
  const Idx end = (Idx)min((long long)begin + p.per_block, p.n_items);
  constexpr int kAtOnce = kQ4 ? kUnrollQ4 : kUnroll;
  // (4 bits: the lanes of a warp leave together)
  for (Idx base = begin + (Idx)threadIdx.x; kQ4 ? (base & ~(Idx)31) < end : base < end; base += (Idx)(kThreads * kAtOnce)) {
    Item<kQ4> x[kAtOnce];
    Move mv[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      mv[u] = {0, -1, 0};
      const Idx item = base + (Idx)(u * kThreads);
      if (item < end) mv[u] = find_move<Idx>(p, item);
      load_item<kQ4>(p, mv[u], x[u]);
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) store_item<kQ4>(p, mv[u], x[u]);
  }
  if (p.advance_len) advance_when_last(p);
}

// Calls too small for a resident wave: one item per thread.  They are a chain of round trips (index words, row, store; with
// advance_len also ticket and lengths, which go beside the row's): four items a thread put four decodings in front of the
// first load, and the ticket behind the stores (28 layers x 4 rows: 3.9 us; 8 x 32 rows with advance_len 3.9 us;
// now 1.9 and 1.8).
template <bool kQ4>
__global__ void __launch_bounds__(kThreads) kv_commit_small_kernel(const __grid_constant__ CommitParams p) {
  dlm_grid_dependency_wait();
  dlm_trigger_dependents();
  const int item = (int)blockIdx.x * kThreads + (int)threadIdx.x;
  Move mv = {0, -1, 0};
  if (item < (int)p.n_items) mv = find_move<int>(p, item);
  Item<kQ4> x;
  load_item<kQ4>(p, mv, x);
  if (p.advance_len) advance_when_last(p);
  store_item<kQ4>(p, mv, x);
}

// Rows of the 4-bit cache as bf16: one item is 2 x 8 values of a K row and of the V row, a 32-bit word and a scale byte each.  Bound by
// HBM like the commit; items, decoding and the words' coalescing are the commit's.
struct ReadParams {
  const uint32_t* k;
  const uint32_t* v;
  const uint8_t* k_scale;
  const uint8_t* v_scale;
  const int32_t* src_pos;
  const int32_t* n_rows;
  uint4* k_out;
  uint4* v_out;
  int n_max, layer_begin, batch, n_kv_heads, capacity, vec_per_row;
  FastDiv by_vec, by_rows, by_heads, by_batch;
  long long n_items;
  int* status;
};

template <typename Idx>
__global__ void __launch_bounds__(kThreads) kv_read_q4_kernel(const __grid_constant__ ReadParams p) {
  dlm_grid_dependency_wait();
  dlm_trigger_dependents();
  const Idx step = (Idx)gridDim.x * kThreads;
  for (Idx base = (Idx)blockIdx.x * kThreads + (Idx)threadIdx.x; base < (Idx)p.n_items; base += step * kUnrollQ4) {
    uint32_t kw[kUnrollQ4][2], vw[kUnrollQ4][2], kb[kUnrollQ4][2], vb[kUnrollQ4][2];
    long long to[kUnrollQ4];
    bool on[kUnrollQ4];
#pragma unroll
    for (int u = 0; u < kUnrollQ4; ++u) {
      const Idx item = base + (Idx)u * step;
      on[u] = item < (Idx)p.n_items;
      if (!on[u]) continue;
      int vec, r, h, b, lc;
      if (sizeof(Idx) == 4) {
        lc = p.by_batch.divmod(p.by_heads.divmod(p.by_rows.divmod(p.by_vec.divmod((int)item, vec), r), h), b);
      } else {
        long long rest = (long long)item;
        vec = (int)(rest % p.vec_per_row);
        rest /= p.vec_per_row;
        r = (int)(rest % p.n_max);
        rest /= p.n_max;
        h = (int)(rest % p.n_kv_heads);
        rest /= p.n_kv_heads;
        b = (int)(rest % p.batch);
        lc = (int)(rest / p.batch);
      }
      const int n = p.n_rows ? p.n_rows[b] : p.n_max;
      const int row = p.src_pos ? p.src_pos[(long long)b * p.n_max + r] : r;
      const bool first = vec == 0 && h == 0 && lc == 0;
      if (n < 0 || n > p.n_max) {
        if (first && r == 0) dlm_set_status(p.status, DLM_ERR_CAPACITY);
        on[u] = false;
      } else if (r >= n) {
        on[u] = false;
      } else if (row < 0 || row >= p.capacity) {
        if (first) dlm_set_status(p.status, DLM_ERR_INDEX);
        on[u] = false;
      }
      if (!on[u]) continue;
      const long long at = first_vector(((((long long)(lc + p.layer_begin) * p.batch + b) * p.n_kv_heads + h) * p.capacity + row) * p.vec_per_row + vec, vec);
      to[u] = first_vector((long long)item, vec);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        kw[u][i] = p.k[at + i * p.vec_per_row];
        vw[u][i] = p.v[at + i * p.vec_per_row];
        kb[u][i] = p.k_scale[(at + i * p.vec_per_row) >> 2];
        vb[u][i] = p.v_scale[(at + i * p.vec_per_row) >> 2];
      }
    }
#pragma unroll
    for (int u = 0; u < kUnrollQ4; ++u) {
      if (!on[u]) continue;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t w[4];
        q4::decode8(kw[u][i], q4::make_scale(kb[u][i]), w);
        __stcs(p.k_out + to[u] + i * p.vec_per_row, make_uint4(w[0], w[1], w[2], w[3]));
        q4::decode8(vw[u][i], q4::make_scale(vb[u][i]), w);
        __stcs(p.v_out + to[u] + i * p.vec_per_row, make_uint4(w[0], w[1], w[2], w[3]));
      }
    }
  }
}

// The arguments that the two commits share, checked; cache->k and ->v in vectors of 8 values.
template <bool kQ4, typename Cache>
int commit(dlm_ctx* ctx, const Cache* cache, uint8_t* k_scale, uint8_t* v_scale, const void* k_new, const void* v_new, int src_len,
           const int32_t* src_idx, const int32_t* dst_pos, int dst_mode, const int32_t* n_rows, int n_max, int advance_len,
           int layer_begin, int layer_end, void* stream) {
  if (cache->n_layers <= 0 || cache->batch <= 0 || cache->n_kv_heads <= 0 || cache->capacity <= 0 ||
      cache->head_dim <= 0 || src_len <= 0 || n_max <= 0 || (dst_mode != DLM_DST_APPEND && dst_mode != DLM_DST_WINDOW))
    return DLM_ERR_SHAPE;
  if (layer_begin < 0 || layer_end > cache->n_layers || layer_begin >= layer_end) return DLM_ERR_SHAPE;

  if (kQ4 ? cache->head_dim % q4::kGroup != 0 : (cache->head_dim * 2) % 16 != 0) return DLM_ERR_UNSUPPORTED;
  if (((uintptr_t)cache->k | (uintptr_t)cache->v | (uintptr_t)k_new | (uintptr_t)v_new) & 15) return DLM_ERR_UNSUPPORTED;
  DLM_DEVICE_TRY(ctx);

  CommitParams p;
  p.cache_k = cache->k;
  p.cache_v = cache->v;
  p.k_scale = k_scale;
  p.v_scale = v_scale;
  p.cache_len = cache->cache_len;
  p.k_new = static_cast<const uint4*>(k_new);
  p.v_new = static_cast<const uint4*>(v_new);
  p.src_idx = src_idx;
  p.dst_pos = dst_pos;
  p.n_rows = n_rows;
  p.n_max = n_max;
  p.src_len = src_len;
  p.advance_len = advance_len ? 1 : 0;
  p.dst_mode = dst_mode;
  p.layer_begin = layer_begin;
  p.n_layers_call = layer_end - layer_begin;
  p.batch = cache->batch;
  p.n_kv_heads = cache->n_kv_heads;
  p.capacity = cache->capacity;
  p.vec_per_row = cache->head_dim * 2 / 16 / (kQ4 ? 2 : 1);
  p.by_vec = make_fast_div(p.vec_per_row);
  p.by_rows = make_fast_div(n_max);
  p.by_heads = make_fast_div(cache->n_kv_heads);
  p.by_batch = make_fast_div(cache->batch);
  p.n_items = (long long)p.n_layers_call * p.batch * p.n_kv_heads * n_max * p.vec_per_row;
  p.status = &ctx->words->status;
  p.ticket = &ctx->words->commit_ticket;

  // one resident wave of equal contiguous ranges, or one item per thread where that is no more
  const bool narrow = p.n_items < (1LL << 31) - (long long)kThreads * kUnroll;
  int& per_sm = ctx->commit_blocks_per_sm[(kQ4 ? 2 : 0) + (narrow ? 0 : 1)];
  if (per_sm <= 0) {
    int n = 0;
    const cudaError_t e = narrow ? cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kv_commit_kernel<int, kQ4>, kThreads, 0)
                                 : cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kv_commit_kernel<long long, kQ4>, kThreads, 0);
    if (e != cudaSuccess || n <= 0) return DLM_ERR_CUDA;
    per_sm = n;
  }
  const long long max_blocks = (long long)ctx->num_sms * per_sm;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (p.n_items <= max_blocks * kThreads) {
    const unsigned int blocks = (unsigned int)((p.n_items + kThreads - 1) / kThreads);
    DLM_CUDA_TRY(dlm_launch(kv_commit_small_kernel<kQ4>, dim3(blocks), dim3(kThreads), 0, st, p));
    return dlm_launch_ok(ctx, 1);
  }
  const long long per_pass = (long long)kThreads * (kQ4 ? kUnrollQ4 : kUnroll);
  long long blocks = (p.n_items + per_pass - 1) / per_pass;
  if (blocks > max_blocks) blocks = max_blocks;
  p.per_block = ((p.n_items + blocks - 1) / blocks + 31) & ~31LL;
  blocks = (p.n_items + p.per_block - 1) / p.per_block;
  if (narrow)
    DLM_CUDA_TRY(dlm_launch(kv_commit_kernel<int, kQ4>, dim3((unsigned)blocks), dim3(kThreads), 0, st, p));
  else
    DLM_CUDA_TRY(dlm_launch(kv_commit_kernel<long long, kQ4>, dim3((unsigned)blocks), dim3(kThreads), 0, st, p));
  return dlm_launch_ok(ctx, 1);
}

}  // namespace

extern "C" int dlm_kv_cache_commit(dlm_ctx* ctx, const dlm_kv_cache* cache, const void* k_new,
                                   const void* v_new, int src_len, const int32_t* src_idx,
                                   const int32_t* dst_pos, int dst_mode, const int32_t* n_rows, int n_max,
                                   int advance_len, int layer_begin, int layer_end, void* stream) {
  if (!ctx || !cache || !cache->k || !cache->v || !cache->cache_len || !k_new || !v_new) return DLM_ERR_NULL;
  return commit<false>(ctx, cache, nullptr, nullptr, k_new, v_new, src_len, src_idx, dst_pos, dst_mode, n_rows, n_max, advance_len,
                       layer_begin, layer_end, stream);
}

extern "C" int dlm_kv_cache_commit_q4(dlm_ctx* ctx, const dlm_kv_cache_q4* cache, const void* k_new,
                                      const void* v_new, int src_len, const int32_t* src_idx,
                                      const int32_t* dst_pos, int dst_mode, const int32_t* n_rows, int n_max,
                                      int advance_len, int layer_begin, int layer_end, void* stream) {
  if (!ctx || !k_new || !v_new) return DLM_ERR_NULL;
  const int rc = dlm_check_q4(cache);
  if (rc != DLM_OK) return rc;
  return commit<true>(ctx, cache, static_cast<uint8_t*>(cache->k_scale), static_cast<uint8_t*>(cache->v_scale), k_new, v_new, src_len,
                      src_idx, dst_pos, dst_mode, n_rows, n_max, advance_len, layer_begin, layer_end, stream);
}

extern "C" int dlm_kv_cache_read_q4(dlm_ctx* ctx, const dlm_kv_cache_q4* cache, const int32_t* src_pos, const int32_t* n_rows,
                                    int n_max, int layer_begin, int layer_end, void* k_out, void* v_out, void* stream) {
  if (!ctx || !k_out || !v_out) return DLM_ERR_NULL;
  const int rc = dlm_check_q4(cache);
  if (rc != DLM_OK) return rc;
  if (n_max <= 0 || layer_begin < 0 || layer_end > cache->n_layers || layer_begin >= layer_end) return DLM_ERR_SHAPE;
  if (!src_pos && n_max > cache->capacity) return DLM_ERR_SHAPE;
  if (((uintptr_t)k_out | (uintptr_t)v_out) & 15) return DLM_ERR_UNSUPPORTED;
  DLM_DEVICE_TRY(ctx);
  ReadParams p;
  p.k = static_cast<const uint32_t*>(cache->k);
  p.v = static_cast<const uint32_t*>(cache->v);
  p.k_scale = static_cast<const uint8_t*>(cache->k_scale);
  p.v_scale = static_cast<const uint8_t*>(cache->v_scale);
  p.src_pos = src_pos;
  p.n_rows = n_rows;
  p.k_out = static_cast<uint4*>(k_out);
  p.v_out = static_cast<uint4*>(v_out);
  p.n_max = n_max;
  p.layer_begin = layer_begin;
  p.batch = cache->batch;
  p.n_kv_heads = cache->n_kv_heads;
  p.capacity = cache->capacity;
  p.vec_per_row = cache->head_dim / 16;
  p.by_vec = make_fast_div(p.vec_per_row);
  p.by_rows = make_fast_div(n_max);
  p.by_heads = make_fast_div(cache->n_kv_heads);
  p.by_batch = make_fast_div(cache->batch);
  p.n_items = (long long)(layer_end - layer_begin) * p.batch * p.n_kv_heads * n_max * p.vec_per_row;
  p.status = &ctx->words->status;
  long long blocks = (p.n_items + kThreads - 1) / kThreads;
  if (blocks > 8LL * ctx->num_sms) blocks = 8LL * ctx->num_sms;
  // item numbers run up to n_items + kUnroll - 1 steps of the grid
  const bool narrow = p.n_items + (kUnroll + 1) * blocks * kThreads < (1LL << 31);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (narrow)
    DLM_CUDA_TRY(dlm_launch(kv_read_q4_kernel<int>, dim3((unsigned)blocks), dim3(kThreads), 0, st, p));
  else
    DLM_CUDA_TRY(dlm_launch(kv_read_q4_kernel<long long>, dim3((unsigned)blocks), dim3(kThreads), 0, st, p));
  return dlm_launch_ok(ctx, 1);
}

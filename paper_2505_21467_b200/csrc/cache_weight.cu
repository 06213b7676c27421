// dlm_cache_weight_accumulate, dlm_cache_weight_accumulate_q4: the attention weight that each cached row gets from the query rows of its KV
// head, added to what it has collected.
//
// With the row's log sum known from the attention step, a weight is exp2(scale log2(e) <q, k> - lse log2(e)): no maximum, no second pass.
// The product is taken as S^T = K Q^T, keys as the rows of the tensor cores' tile: then a key is a TMEM lane, so a thread, and
// its sum over the query rows runs along the columns of that lane, in registers and in a fixed order, with no exchange between threads and
// no atomics.  Per (key, query) the tensor pipe needs 2 D flops and the thread one fused multiply-add, an exponential and an addition.
//
// Query rows that take no part are zeros with a logarithm far below all others, so their terms are 2^(0 - 3e38) = 0 with no test of any column.  A
// key that is not finite (bf16 cache) makes 0 * inf = NaN of them; a key whose sum is NaN is therefore summed once more without those columns.
//
// A step is a tile of 128 keys of a (layer, batch element, KV head) against 128 query rows; a tile meets all query rows of its KV head.
// Block = 32 warps (24 without decoders), one block per SM with a contiguous share of the tiles, dealt to four groups in turn.  What bounds a group
// is latency: a tile takes it a chain of waits, decoding, products, loads from TMEM and sums of 2000 - 4000 cycles, hence four of them.
//   warps 0-15       sums, four warps a group; a group has one K tile and 128 columns of TMEM (two score buffers of up to 64 query rows, else one)
//   8 more           4-bit cache: decoders of K tiles, two warps for a group
//   then             producer: K tiles by TMA (bf16) or bulk copies (4 bits), query rows by TMA
//   four             tcgen05.mma issuers of the groups (one lane each)
//   one              the query rows' logarithms, and zeros for query rows that take no part
// Query rows lie in two slots of 128: up to 256 stay there for all tiles of a unit, more go through for every four tiles.
//
// 28 layers x 4 KV heads of 16301 bf16 rows against 224 query rows: 168 us (2.9 TB/s of keys, 630 TFLOP/s; 165 without the test for NaN sums); 32 x 4 x 32 heads of 2048 4-bit rows
// against 64: 343 us (2.0 TB/s, 405 TFLOP/s; 64 % of the issue slots, 45 % of the integer pipe: decoding; exponentials 34 % of theirs, tensor pipe
// 17 %).  The latter took 368 us with two groups, and 451 with packed half tiles that belong to one group instead of a ring that all decoders read.
#include <cuda_bf16.h>
#include <math_constants.h>

#include "common.cuh"
#include "deal.cuh"
#include "q4_tiles.cuh"
#include "sm100_ptx.cuh"

namespace {

using namespace sm100;

constexpr int kKeys = 128;                // a tile
constexpr int kRows = 128;                // query rows of a step
constexpr int kMaxBatch = 1024;
constexpr int kMaxQCap = 4096;
constexpr int kMaxGrid = 256;
constexpr int kTmemCols = 512;
constexpr int kBarrierBytes = 512, kFlagBytes = 64;
constexpr int kGroupsOfTiles = 4, kSumWarps = 4 * kGroupsOfTiles;

template <int D, bool kQ4>
struct Shape {
  static constexpr int kDecodeWarps = kQ4 ? 8 : 0, kThreads = 32 * (kSumWarps + kDecodeWarps + 8);
  static constexpr int kPanels = D / 64;
  static constexpr int kPanel = 128 * 128;           // bytes of a K tile's panel: 128 rows of 64 values
  static constexpr int kTile = kPanels * kPanel;
  static constexpr int KS = kGroupsOfTiles;          // K tiles
  static constexpr int kPackedStage = q4::Packed<D, kKeys>::kBytes;
};
constexpr int kMaxPacked = 8;                        // packed K tiles: as many as there is room for
constexpr int kLogBytes = 2 * kRows * 4;
constexpr float kLeftOut = -3.402823466e38f;         // in place of minus the logarithm of a query row that takes no part

struct Params {
  const int32_t* cache_len;
  const int32_t* q_len;
  const uint8_t *k, *k_scale;   // 4-bit cache
  const float* lse;
  const float* collected;       // may be `weight`
  float* weight;
  float decay;
  int nl, layer_begin, batch, n_kv_heads, n_q_heads, group, capacity, q_cap;
  int rows_total, n_qc;         // query rows of a KV head, chunks of 128 of them
  int q_box, k_box;             // rows of the TMA boxes
  uint32_t q_panel;             // bytes of a query slot's panel: as many rows as a chunk has, in whole groups of 16
  int n_packed;                 // packed stages
  FastDiv by_kv_heads, by_q_cap;
  float scale_log2;
  int* status;
};

struct Segment {
  int layer, b, kvh, Lc, Lq;
  int begin, end;   // tiles of the unit
};

struct Walk {
  const Params& p;
  const Lengths& s;
  const Deal& d;
  int at, end;
  __device__ __forceinline__ Walk(const Params& p_, const Lengths& s_, const Deal& d_, int cta) : p(p_), s(s_), d(d_) {
    at = cta < d.n ? d.lo(cta) : 0;
    end = cta < d.n ? d.lo(cta + 1) : 0;
  }
  __device__ __forceinline__ bool next(Segment& g) {
    if (at >= end) return false;
    int rest;
    const int grp = d.group_of(at, rest);
    g.b = element_of(s, p.batch, rest);
    g.layer = p.by_kv_heads.divmod(grp, g.kvh);
    g.Lc = s.lc[g.b];
    g.Lq = s.lq[g.b];
    const int unit = grp * d.sum + s.prefix[g.b];
    g.begin = at - unit;
    g.end = min(s.prefix[g.b + 1] - s.prefix[g.b], end - unit);
    at = unit + g.end;
    return true;
  }
};

struct Ring {   // the next use of a ring of n stages: which stage, and the parity of its barrier's phase
  uint32_t stage = 0, parity = 0;
  __device__ __forceinline__ void advance(uint32_t n) {
    if (++stage == n) {
      stage = 0;
      parity ^= 1u;
    }
  }
};

// The sum over n16 query rows (columns of TMEM from `from` on, logarithms at log_at) without those that take no part; what they hold is not
// looked at.  The others' terms are added in the same order as in the kernel, so a sum that is a number comes out with the same bits.
__device__ __noinline__ float sum_of_those_that_take_part(uint32_t from, uint32_t log_at, int n16, float scale_log2) {
  float a[4] = {};
#pragma unroll 1
  for (int i0 = 0; i0 < n16; i0 += 16) {
    uint32_t v[16];
    tmem_ld16(from + i0, v);
    tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const float4 l = ld_shared_f4(log_at + (i0 + i) * 4);
      const float minus_log[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (minus_log[c] != kLeftOut) a[c] += ex2_approx(fmaf(__uint_as_float(v[i + c]), scale_log2, minus_log[c]));
    }
  }
  return (a[0] + a[1]) + (a[2] + a[3]);
}

// Tiles begin + w, begin + w + 4, .. of a segment belong to group w of the warps.  Every role enumerates the loads of query rows alike: events,
// event e in slot e & 1.  Up to two chunks: one event each for a segment; more: one each for four tiles.
//
// A wait for a barrier's phase works only when the phase before is over, so whoever waits on a barrier either has to arrive for its next
// phase or waits behind something that does: hence stages that belong to one group, and events that each role takes, also where it has
// no tile.
//
// kNoWait = true is the instantiation that a test selects to run the give-up path: every wait on work still to come tests its barrier once.
template <int D, bool kQ4, bool kNoWait>
__global__ void __launch_bounds__(Shape<D, kQ4>::kThreads, 1)
cache_weight_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ Params p) {
  using G = Shape<D, kQ4>;
  using Pk = q4::Packed<D, kKeys>;
  constexpr int KS = G::KS, kControl = kSumWarps + G::kDecodeWarps;
  constexpr uint64_t kLimit = kNoWait ? 0ull : kWaitLimitNs;
  const uint32_t PS = (uint32_t)p.n_packed, q_slot = G::kPanels * p.q_panel;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_pad = (1024u - (smem_u32(smem_raw) & 1023u)) & 1023u;
  const uint32_t sm_k = smem_u32(smem_raw) + smem_pad, sm_q = sm_k + KS * G::kTile, sm_p = sm_q + 2 * q_slot;
  const uint32_t sm_log = sm_p + (kQ4 ? PS * G::kPackedStage : 0), sm_bar = sm_log + kLogBytes;
  float* const logs = reinterpret_cast<float*>(smem_raw + smem_pad + (sm_log - sm_k));
  int* const flags = reinterpret_cast<int*>(smem_raw + smem_pad + (sm_bar - sm_k) + kBarrierBytes);
  volatile int* const abort_ptr = flags;
  volatile int* const never_ptr = flags + 1;
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(flags + 2);
  const Lengths len(flags + kFlagBytes / 4, p.batch);

  const uint32_t bar_k_full = sm_bar, bar_k_empty = bar_k_full + 8 * KS, bar_p_full = bar_k_empty + 8 * KS, bar_p_empty = bar_p_full + 8 * kMaxPacked;
  const uint32_t bar_q_tx = bar_p_empty + 8 * kMaxPacked, bar_q_ready = bar_q_tx + 16, bar_q_empty = bar_q_ready + 16;   // [slot]
  const uint32_t bar_s_ready = bar_q_empty + 16, bar_s_empty = bar_s_ready + 64, bar_drain = bar_s_empty + 64;   // [group][buffer], [group]

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    *abort_ptr = 0; *never_ptr = 0;
    for (int i = 0; i < KS; ++i) {
      mbar_init(bar_k_full + 8 * i, kQ4 ? G::kDecodeWarps / kGroupsOfTiles : 1);
      mbar_init(bar_k_empty + 8 * i, 1);
    }
    for (int i = 0; kQ4 && i < kMaxPacked; ++i) {
      mbar_init(bar_p_full + 8 * i, 1);
      mbar_init(bar_p_empty + 8 * i, G::kDecodeWarps);
    }

    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_q_tx + 8 * i, 1);
      mbar_init(bar_q_ready + 8 * i, 1);
      mbar_init(bar_q_empty + 8 * i, kSumWarps + kGroupsOfTiles);   // and the issuers
    }
    for (int i = 0; i < 2 * kGroupsOfTiles; ++i) {
      mbar_init(bar_s_ready + 8 * i, 1);
      mbar_init(bar_s_empty + 8 * i, 4);
    }
    for (int i = 0; i < kGroupsOfTiles; ++i) mbar_init(bar_drain + 8 * i, 1);
    mbar_fence_init();
    fence_proxy_async_smem();
  }
  if (warp == kControl + 1) {
    tmem_alloc(smem_u32(tmem_slot), kTmemCols);
    tmem_relinquish();
  }
  if (warp == kControl && lane == 0) {
    prefetch_tensormap(&tm_q);
    if (!kQ4) prefetch_tensormap(&tm_k);
  }
  dlm_grid_dependency_wait();
  dlm_trigger_dependents();
  if (warp == 0)
    read_lengths(p.cache_len, p.q_len, p.batch, p.capacity, p.q_cap, p.status, len, nullptr, [](int Lc, int) { return (Lc + kKeys - 1) / kKeys; });
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  const Deal deal(len.prefix[p.batch], p.nl * p.n_kv_heads, (int)gridDim.x, 1);
  const bool resident = p.n_qc <= 2;
  // score buffers of a group and their columns
  const uint32_t n_buf = p.rows_total <= 64 ? 2 : 1, buf_cols = p.rows_total <= 64 ? 64 : 128;
  auto chunk_rows = [&](int c) { return min(kRows, p.rows_total - c * kRows); };
  Walk walk(p, len, deal, blockIdx.x);
  Segment g = {};
  bool ok = true;

  if (warp == kControl) {
    // ================================================================= producer
    uint32_t kt = 0, ev = 0;   // packed tiles and events so far; tiles of the groups (bf16)
    Ring ps;
    uint32_t tiles[kGroupsOfTiles] = {};
    auto wait = [&](uint32_t bar, uint32_t parity) { return mbar_wait_warp(bar, parity, abort_ptr, kLimit); };
    auto load_q = [&](int c) {
      const uint32_t s = ev & 1;
      if (ev >= 2 && !wait(bar_q_empty + 8 * s, ((ev >> 1) - 1) & 1)) return false;
      if (lane == 0) {
        mbar_expect_tx(bar_q_tx + 8 * s, (uint32_t)p.q_box * 128u * G::kPanels);   // a box counts in full
        const int z = (g.layer * p.batch + g.b) * p.n_kv_heads + g.kvh;
        for (int pn = 0; pn < G::kPanels; ++pn) tma_load_3d(sm_q + s * q_slot + pn * p.q_panel, &tm_q, bar_q_tx + 8 * s, pn * 64, c * kRows, z);
      }
      __syncwarp();
      ++ev;
      return true;
    };
    auto load_k = [&](int t, int w) {
      const int z = ((g.layer + p.layer_begin) * p.batch + g.b) * p.n_kv_heads + g.kvh;
      if (kQ4) {
        const uint32_t s = ps.stage, bar = bar_p_full + 8 * s;
        if (kt >= PS && !wait(bar_p_empty + 8 * s, ps.parity ^ 1u)) return false;
        const int rows = min(kKeys, g.Lc - t * kKeys);
        if (lane == 0) mbar_expect_tx(bar, Pk::bytes(rows));
        __syncwarp();
        if (lane < 2) Pk::copy_part(sm_p + s * G::kPackedStage, p.k, p.k_scale, lane, (size_t)z * p.capacity + (size_t)t * kKeys, rows, bar);
        __syncwarp();
        ++kt;
        ps.advance(PS);
      } else {
        const uint32_t s = w, bar = bar_k_full + 8 * s;
        if (tiles[w] > 0 && !wait(bar_k_empty + 8 * s, (tiles[w] - 1) & 1)) return false;
        if (lane == 0) mbar_expect_tx(bar, (uint32_t)p.k_box * 128u * G::kPanels);
        __syncwarp();
        if (lane < G::kPanels) tma_load_3d(sm_k + s * G::kTile + lane * G::kPanel, &tm_k, bar, lane * 64, t * kKeys, z);
        __syncwarp();
        ++tiles[w];
      }
      return true;
    };
    while (ok && walk.next(g)) {
      if (resident)
        for (int c = 0; c < p.n_qc && ok; ++c) ok = load_q(c);
      for (int t = g.begin; t < g.end && ok; t += kGroupsOfTiles) {
#pragma unroll
        for (int w = 0; w < kGroupsOfTiles; ++w)
          if (ok && t + w < g.end) ok = load_k(t + w, w);
        if (!resident)
          for (int c = 0; c < p.n_qc && ok; ++c) ok = load_q(c);
      }
    }
    // no copy lands after the block has released its shared memory
    if (kQ4) {
      for (uint32_t i = kt > PS ? kt - PS : 0; i < kt; ++i) mbar_wait(bar_p_full + 8 * (i % PS), (i / PS) & 1, never_ptr);
    } else {
#pragma unroll
      for (int w = 0; w < kGroupsOfTiles; ++w)
        if (tiles[w] > 0) mbar_wait(bar_k_full + 8 * w, (tiles[w] - 1) & 1, never_ptr);
    }
    for (uint32_t i = ev > 2 ? ev - 2 : 0; i < ev; ++i) mbar_wait(bar_q_tx + 8 * (i & 1), (i >> 1) & 1, never_ptr);
  } else if (warp > kControl && warp <= kControl + kGroupsOfTiles) {
    if (elect_one_sync()) {
      // ================================================================= MMA issuers, one for each group of warps
      const int w = warp - kControl - 1;
      auto wait = [&](uint32_t bar, uint32_t parity) { return mbar_wait_limit(bar, parity, abort_ptr, kLimit); };
      uint32_t kt = 0, ev = 0, st = 0;   // the group's tiles, events, the group's steps so far
      const uint64_t desc_k0 = make_smem_desc_sw128(sm_k, 16, 1024), desc_q0 = make_smem_desc_sw128(sm_q, 16, 1024);
      auto take_event = [&](uint32_t e) { return wait(bar_q_ready + 8 * (e & 1), (e >> 1) & 1); };
      while (ok && walk.next(g)) {
        for (int t = g.begin + w; t - w < g.end && ok; t += kGroupsOfTiles) {
          const bool mine = t < g.end;
          if (mine) ok = wait(bar_k_full + 8 * w, kt & 1);
          for (int c = 0; c < p.n_qc && ok && (mine || !resident); ++c) {
            const uint32_t e = ev + c;
            ok = take_event(e);
            if (ok && mine) {
              const uint32_t b = st % n_buf, use = st / n_buf, buf = 16 * w + 8 * b;
              ok = use == 0 || wait(bar_s_empty + buf, (use - 1) & 1);
              if (!ok) break;
              tc_fence_after_sync();
              const uint32_t idesc = make_idesc_bf16(128, (uint32_t)((chunk_rows(c) + 15) & ~15), 0);
              const uint64_t dk = desc_offset(desc_k0, w * G::kTile), dq = desc_offset(desc_q0, (e & 1) * q_slot);
              const uint32_t d = tmem + w * 128 + b * buf_cols;
#pragma unroll
              for (int k = 0; k < D / 16; ++k) {
                const uint32_t a = ((k >> 2) * G::kPanel + (k & 3) * 32) >> 4, b_off = ((k >> 2) * p.q_panel + (k & 3) * 32) >> 4;
                mma_ss_lo<false>(d, (uint32_t)dk + a, (uint32_t)dq + b_off, (uint32_t)(dk >> 32), idesc, k > 0 ? 1u : 0u);
              }
              tc_commit(bar_s_ready + buf);
              ++st;
            }
            if (ok && !resident) mbar_arrive(bar_q_empty + 8 * (e & 1));   // (the slot is not free before the group's warps have summed this step)
          }
          if (ok && mine) {
            tc_commit(bar_k_empty + 8 * w);
            ++kt;
          }
          if (!resident) ev += p.n_qc;
        }
        if (resident) {
          for (int c = 0; c < p.n_qc && ok; ++c) {
            ok = take_event(ev + c);
            if (ok) mbar_arrive(bar_q_empty + 8 * ((ev + c) & 1));
          }
          ev += p.n_qc;
        }
      }
      tc_commit(bar_drain + 8 * w);
      mbar_wait(bar_drain + 8 * w, 0, never_ptr);
    }
  } else if (warp == kControl + kGroupsOfTiles + 1) {
    // ================================================================= query rows: logarithms, zeros
    uint32_t ev = 0;
    while (ok && walk.next(g)) {
      const int events = resident ? p.n_qc : p.n_qc * ((g.end - g.begin + kGroupsOfTiles - 1) / kGroupsOfTiles);
      const float* const lse = p.lse + (((size_t)g.layer * p.batch + g.b) * p.n_q_heads + (size_t)g.kvh * p.group) * p.q_cap;
      for (int i = 0, c = 0; i < events && ok; ++i, ++ev, c = c + 1 == p.n_qc ? 0 : c + 1) {
        const uint32_t s = ev & 1;
        const int n16 = (chunk_rows(c) + 15) & ~15;
        float x[kRows / 32];
        bool out[kRows / 32];
#pragma unroll
        for (int j = 0; j < kRows / 32; ++j) {
          const int r = j * 32 + lane, r_kv = c * kRows + r;
          const bool in = r_kv < p.rows_total && r_kv - p.by_q_cap.div(r_kv) * p.q_cap < g.Lq;
          x[j] = in ? lse[r_kv] : -CUDART_INF_F;
          out[j] = x[j] == -CUDART_INF_F;
        }
        // the copy into the slot shows that the slot's logarithms have been used too
        ok = mbar_wait_warp(bar_q_tx + 8 * s, (ev >> 1) & 1, abort_ptr, kLimit);
        if (!ok) break;
#pragma unroll
        for (int j = 0; j < kRows / 32; ++j) {
          const int r = j * 32 + lane;
          logs[s * kRows + r] = out[j] ? kLeftOut : x[j] * -1.4426950408889634f;
          // a row that takes no part: zeros, whatever it holds
          for (uint32_t todo = __ballot_sync(0xffffffffu, out[j] && r < n16); todo != 0; todo &= todo - 1)
            if (lane < D / 8) q4::clear_piece<D>(sm_q + s * q_slot, p.q_panel, (j * 32 + __ffs(todo) - 1) * (D / 8) + lane);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_q_ready + 8 * s);
      }
    }
  } else if (warp >= kSumWarps && warp < kControl) {
    if constexpr (kQ4) {
      // ================================================================= decoders, two warps for a group's tiles
      constexpr int kTeam = G::kDecodeWarps / kGroupsOfTiles * 32;
      const q4::Decoder<D, kKeys, kTeam> decoder(tid & (kTeam - 1), G::kPanel);
      const int w = (warp - kSumWarps) / (G::kDecodeWarps / kGroupsOfTiles);
      uint32_t n = 0;   // the group's tiles
      Ring ps;
      while (ok && walk.next(g)) {
        for (int t = g.begin; t < g.end && ok; ++t, ps.advance(PS)) {
          const uint32_t s = ps.stage, packed = sm_p + s * G::kPackedStage;
          ok = mbar_wait_warp(bar_p_full + 8 * s, ps.parity, abort_ptr, kLimit);
          if (!ok) break;
          if (((t - g.begin) & (kGroupsOfTiles - 1)) != w) {
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_p_empty + 8 * s);
            continue;
          }
          const uint32_t tile = sm_k + w * G::kTile;
          if (n > 0) ok = mbar_wait_warp(bar_k_empty + 8 * w, (n - 1) & 1, abort_ptr, kLimit);
          if (!ok) break;
          decoder.run(packed, tile, min(kKeys, g.Lc - t * kKeys));
          ++n;
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(bar_p_empty + 8 * s);
            mbar_arrive(bar_k_full + 8 * w);
          }
        }
      }
    }
  } else if (warp < kSumWarps) {
    // ================================================================= sums: thread = key of the tile = TMEM lane
    const int w = warp >> 2, key = (warp & 3) * 32 + lane;
    const uint32_t t_s = tmem + ((uint32_t)((warp & 3) * 32) << 16) + w * 128;
    const uint64_t scale2 = pack2(p.scale_log2, p.scale_log2);
    uint32_t ev = 0, st = 0;   // events, the group's steps
    while (ok && walk.next(g)) {
      const size_t row0 = (((size_t)(g.layer + p.layer_begin) * p.batch + g.b) * p.n_kv_heads + g.kvh) * p.capacity;
      // what the group's next tile has collected so far, asked for a tile ahead: a load from memory takes longer than a tile
      auto collected_of = [&](int t) {
        const int j = t * kKeys + key;
        return t < g.end && j < g.Lc && p.collected && p.decay != 0.f ? p.collected[row0 + j] : 0.f;
      };
      float ahead = collected_of(g.begin + w);
      for (int t0 = g.begin; t0 < g.end && ok; t0 += kGroupsOfTiles) {
        const int t = t0 + w;
        if (t < g.end) {
          float total = 0.f;
          const int j = t * kKeys + key;
          const float before = ahead;
          ahead = collected_of(t + kGroupsOfTiles);
          for (int c = 0; c < p.n_qc && ok; ++c, ++st) {
            const uint32_t e = ev + c, b = st % n_buf, use = st / n_buf, buf = 16 * w + 8 * b;
            const int n16 = (chunk_rows(c) + 15) & ~15;
            ok = mbar_wait_warp(bar_s_ready + buf, use & 1, abort_ptr, kLimit);   // (behind q_ready, whose logarithms are read here)
            if (ok) ok = mbar_wait_warp(bar_q_ready + 8 * (e & 1), (e >> 1) & 1, abort_ptr, kLimit);
            if (!ok) break;
            tc_fence_after_sync();
            const uint32_t from = t_s + b * buf_cols, log_at = sm_log + (e & 1) * kRows * 4;
            uint64_t a01 = 0, a23 = 0;   // pairs of sums
            auto add = [&](const uint32_t* v, int i0, int n) {
#pragma unroll
              for (int i = 0; i < 32; i += 4) {
                if (i >= n) break;
                const float4 l = ld_shared_f4(log_at + (i0 + i) * 4);
                float x0, x1, x2, x3;
                unpack2(fma2(pack2(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), scale2, pack2(l.x, l.y)), x0, x1);
                unpack2(fma2(pack2(__uint_as_float(v[i + 2]), __uint_as_float(v[i + 3])), scale2, pack2(l.z, l.w)), x2, x3);
                a01 = add2(a01, pack2(ex2_approx(x0), ex2_approx(x1)));
                a23 = add2(a23, pack2(ex2_approx(x2), ex2_approx(x3)));
              }
            };
            uint32_t v[32];
            int i = 0;
#pragma unroll 1
            for (; i + 32 <= n16; i += 32) {
              tmem_ld32(from + i, v);
              tmem_ld_wait();
              add(v, i, 32);
            }
            if (i < n16) {
              tmem_ld16(from + i, v);
              tmem_ld_wait();
              add(v, i, 16);
            }
            float a0, a1, a2, a3;
            unpack2(a01, a0, a1);
            unpack2(a23, a2, a3);
            float sum = (a0 + a1) + (a2 + a3);
            if (!kQ4 && __any_sync(0xffffffffu, sum != sum && j < g.Lc)) sum = sum_of_those_that_take_part(from, log_at, n16, p.scale_log2);   // rare
            total += sum;
            __syncwarp();
            if (lane == 0) {
              tc_fence_before_sync();
              mbar_arrive(bar_s_empty + buf);
              if (!resident) mbar_arrive(bar_q_empty + 8 * (e & 1));
            }
          }
          if (!ok) break;
          if (j < g.Lc) p.weight[row0 + j] = fmaf(p.decay, before, total);
        } else if (!resident) {   // no tile for the group: the query rows are not needed here
          for (int c = 0; c < p.n_qc && ok; ++c) {
            ok = mbar_wait_warp(bar_q_ready + 8 * ((ev + c) & 1), ((ev + c) >> 1) & 1, abort_ptr, kLimit);
            __syncwarp();
            if (ok && lane == 0) mbar_arrive(bar_q_empty + 8 * ((ev + c) & 1));
          }
        }
        if (!resident) ev += p.n_qc;
      }
      if (resident) {
        for (int c = 0; c < p.n_qc && ok; ++c) {
          ok = mbar_wait_warp(bar_q_ready + 8 * ((ev + c) & 1), ((ev + c) >> 1) & 1, abort_ptr, kLimit);
          __syncwarp();
          if (ok && lane == 0) mbar_arrive(bar_q_empty + 8 * ((ev + c) & 1));
        }
        ev += p.n_qc;
      }
    }
  }
  // ---- teardown
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  if (tid == 0 && (*abort_ptr || *never_ptr)) dlm_set_status(p.status, DLM_ERR_TIMEOUT);
  if (warp == kControl + 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, kTmemCols);
    __syncwarp();
  }
}

using Kernel = void (*)(const CUtensorMap, const CUtensorMap, const Params);

template <bool kQ4, typename Cache>
int accumulate(dlm_ctx* ctx, const Cache* cache, const uint8_t* k_scale, int layer_begin, int layer_end, const void* q, const float* lse,
               int n_q_heads, int q_cap, const int32_t* q_len, float softmax_scale, int cache_len_hint, const float* collected, float decay,
               float* weight, void* stream) {
  if (n_q_heads <= 0 || q_cap <= 0 || layer_begin < 0 || layer_end > cache->n_layers || layer_begin >= layer_end) return DLM_ERR_SHAPE;
  const int D = cache->head_dim;
  if ((D != 64 && D != 128) || n_q_heads % cache->n_kv_heads != 0 || decay != decay) return DLM_ERR_UNSUPPORTED;
  const int group = n_q_heads / cache->n_kv_heads, nl = layer_end - layer_begin;
  if (q_cap > kMaxQCap || (long long)group * q_cap > (1 << 20) || cache->batch > kMaxBatch) return DLM_ERR_UNSUPPORTED;
  if (((uintptr_t)q | (uintptr_t)cache->k) & 15) return DLM_ERR_UNSUPPORTED;
  const long long units = (long long)nl * cache->batch * cache->n_kv_heads, tiles = (cache->capacity + kKeys - 1) / kKeys;
  if (units * tiles >= (1LL << 30)) return DLM_ERR_UNSUPPORTED;   // items are counted in 32 bits
  DLM_DEVICE_TRY(ctx);
  const bool no_wait = ctx->wait_limit_ns == 0;
  const Kernel kern = D == 128 ? (no_wait ? cache_weight_kernel<128, kQ4, true> : cache_weight_kernel<128, kQ4, false>)
                               : (no_wait ? cache_weight_kernel<64, kQ4, true> : cache_weight_kernel<64, kQ4, false>);
  const int threads = Shape<128, kQ4>::kThreads;
  const int which = (D == 128 ? 0 : 1) + (kQ4 ? 2 : 0) + (no_wait ? 4 : 0);
  if (ctx->weight_smem_limit[which] == 0) {
    DLM_CUDA_TRY(cudaFuncSetAttribute(reinterpret_cast<const void*>(kern), cudaFuncAttributeMaxDynamicSharedMemorySize, ctx->max_smem_optin));
    ctx->weight_smem_limit[which] = ctx->max_smem_optin;
  }
  Params p;
  p.cache_len = cache->cache_len;
  p.q_len = q_len;
  p.k = static_cast<const uint8_t*>(cache->k);
  p.k_scale = k_scale;
  p.lse = lse;
  p.collected = collected;
  p.weight = weight;
  p.decay = collected ? decay : 0.f;
  p.nl = nl;
  p.layer_begin = layer_begin;
  p.batch = cache->batch;
  p.n_kv_heads = cache->n_kv_heads;
  p.n_q_heads = n_q_heads;
  p.group = group;
  p.capacity = cache->capacity;
  p.q_cap = q_cap;
  p.rows_total = group * q_cap;
  p.n_qc = (p.rows_total + kRows - 1) / kRows;
  p.q_box = p.rows_total < kRows ? p.rows_total : kRows;
  p.k_box = cache->capacity < kKeys ? cache->capacity : kKeys;
  p.q_panel = (uint32_t)((p.q_box + 15) & ~15) * 128u;
  const int tile = D == 128 ? Shape<128, kQ4>::kTile : Shape<64, kQ4>::kTile;
  const int packed = D == 128 ? Shape<128, kQ4>::kPackedStage : Shape<64, kQ4>::kPackedStage;
  const int fixed = 1024 + Shape<128, kQ4>::KS * tile + 2 * (D / 64) * (int)p.q_panel + kLogBytes + kBarrierBytes + kFlagBytes +
                    4 * length_ints(cache->batch);
  p.n_packed = kQ4 ? (ctx->max_smem_optin - fixed) / packed : 0;
  if (p.n_packed > kMaxPacked) p.n_packed = kMaxPacked;
  const int smem = fixed + p.n_packed * packed;
  if (smem > ctx->max_smem_optin || (kQ4 && p.n_packed < 2)) return DLM_ERR_UNSUPPORTED;
  p.by_kv_heads = make_fast_div(p.n_kv_heads);
  p.by_q_cap = make_fast_div(q_cap);
  p.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)D)) * 1.4426950408889634f;
  p.status = &ctx->words->status;
  CUtensorMap tm_q, tm_k;
  int rc = encode_rows_map(ctx, &tm_q, q, D, p.rows_total, (long long)nl * cache->batch * cache->n_kv_heads, p.q_box);
  tm_k = tm_q;
  if (!kQ4 && rc == DLM_OK)
    rc = encode_rows_map(ctx, &tm_k, cache->k, D, cache->capacity, (long long)cache->n_layers * cache->batch * cache->n_kv_heads, p.k_box);
  if (rc != DLM_OK) return rc;
  const int sms = ctx->num_sms < kMaxGrid ? ctx->num_sms : kMaxGrid, expected = cache_len_hint > 0 && cache_len_hint < cache->capacity ? cache_len_hint : cache->capacity;
  const long long most = units * ((expected + kKeys - 1) / kKeys);   // blocks that find work if the cache is as long as expected
  const int grid = most < sms ? (int)most : sms;
  DLM_CUDA_TRY(dlm_launch(kern, dim3(grid), dim3(threads), (size_t)smem, static_cast<cudaStream_t>(stream), tm_q, tm_k, p));
  return dlm_launch_ok(ctx, 1);
}

}  // namespace

extern "C" int dlm_cache_weight_accumulate(dlm_ctx* ctx, const dlm_kv_cache* cache, int layer_begin, int layer_end, const void* q,
                                           const float* lse, int n_q_heads, int q_cap, const int32_t* q_len, float softmax_scale,
                                           int cache_len_hint, const float* collected, float decay, float* weight, void* stream) {
  if (!ctx || !cache || !cache->k || !cache->cache_len || !q || !lse || !weight) return DLM_ERR_NULL;
  if (cache->n_layers <= 0 || cache->batch <= 0 || cache->n_kv_heads <= 0 || cache->capacity <= 0) return DLM_ERR_SHAPE;
  return accumulate<false>(ctx, cache, nullptr, layer_begin, layer_end, q, lse, n_q_heads, q_cap, q_len, softmax_scale, cache_len_hint, collected,
                           decay, weight, stream);
}

extern "C" int dlm_cache_weight_accumulate_q4(dlm_ctx* ctx, const dlm_kv_cache_q4* cache, int layer_begin, int layer_end, const void* q,
                                              const float* lse, int n_q_heads, int q_cap, const int32_t* q_len, float softmax_scale,
                                              int cache_len_hint, const float* collected, float decay, float* weight, void* stream) {
  if (!ctx || !q || !lse || !weight) return DLM_ERR_NULL;
  const int bad = dlm_check_q4(cache);
  if (bad != DLM_OK) return bad;
  return accumulate<true>(ctx, cache, static_cast<const uint8_t*>(cache->k_scale), layer_begin, layer_end, q, lse, n_q_heads, q_cap, q_len,
                          softmax_scale, cache_len_hint, collected, decay, weight, stream);
}

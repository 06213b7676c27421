// dlm_freecache_attn_step_q4: attention of the active window over [4-bit cache rows ; fresh bf16 rows].
//
// The arithmetic is dlm_freecache_attn_step's: scores S = Q K^T in fp32, an online softmax with base-2 exponentials, O += P V with P in
// bf16 (the products' operand type; sums of P in fp32, before the rounding) and O in fp32, everything on the tensor cores with S, P and O in TMEM.  A value of the cache has 7 significant bits, so the
// bf16 tile that the products read holds it exactly; what is quantised is what was committed, nothing on the way.
//
// One unit is (layer, batch element, KV head, chunk of up to 256 query rows); its keys are taken in steps of 64, first the cache's,
// then the fresh ones.  Up to 32 query rows a KV head are a kernel of their own (attn_q4_few.cuh); above 128 a block has two M tiles of 128 query
// rows that share every step, else one M tile, whose steps two chains of warps take in turn, each with an O, maxima and sums of its own that
// are joined at the end.  What bounds a chain is latency (a step's softmax takes its warps 1800 cycles), so both forms have two.  Block = 16 or 20 warps:
//   warps 0-3, 4-7   softmax of chain 0, 1 (thread = query row = TMEM lane)
//   4 or 8 more      decoders: packed K and V steps to bf16 operand tiles, a group of 32 values a thread at a time; two or four of their lanes
//                    have fresh rows copied straight into operand tiles (TMA)
//   then             producer: bulk copies of packed steps (a step's rows lie one after the other), TMA of Q
//   two              tcgen05.mma issuers of chain 0, 1 (one lane each)
//
// Every (unit, step) pair is one item of a global list and block c takes a contiguous share of it, at least `min_share` items: whole
// units are finished by the block; a share's first and last unit may be a part, whose unnormalised O, maximum and sum go to the
// workspace.  A second, small launch joins the parts in block order (the result does not depend on timing), so that no block waits for
// another.
//
// One layer of 32 x 7 query rows over 1024 cached ones: 15.9 us (20.5 in the first form, 17.5 before the joining launch looked for its
// parts early; shares of at least 1, 2, 3, 4 and 6 steps took 18.9, 19.0, 19.7, 20.3 and 22.9 in between).  28 layers over 16301 rows: 267 us, 0.48 of the tensor peak, the softmax warps' chain: per step 1470
// of 2236 cycles.  32 layers x 4 x 32 heads over 2048 rows, 64 query rows (half of the M tile): 750 us, 1.9 TB/s of the cache; 49 % of the issue
// slots and 34 % of the tensor pipe are in use, and without any decoding, exponentials or products the waits alone took 490.  (16 decoding warps for
// one M tile: 691 us with a cold cache instead of 663, 779 in a row with other inputs instead of 748.)
#include <cuda_bf16.h>
#include <math_constants.h>

#include "attn_softmax.cuh"
#include "common.cuh"
#include "deal.cuh"
#include "q4_tiles.cuh"

namespace {

constexpr int kStep = 64;                 // keys
constexpr int kMaxBatch = 1024;
constexpr int kMaxQCap = 4096;
constexpr int kMaxGrid = 256;
constexpr int kTmemCols = 512;
constexpr int kBarrierBytes = 512, kFlagBytes = 64;

template <int D, int NMT>
struct Shape {
  static constexpr bool kSplit = NMT == 1;                   // the chains share an M tile and split the steps
  static constexpr int kDecodeWarps = kSplit ? 8 : 4, kTeamWarps = kDecodeWarps / 4, kControl = 8 + kDecodeWarps, kThreads = 32 * (kControl + 4);
  // registers a thread: at launch all of the SM's, then by role
  static constexpr int kRegsLaunch = kSplit ? 96 : 128, kRegsSoftmax = kSplit ? 136 : 168, kRegsDecode = kSplit ? 72 : 104, kRegsControl = kSplit ? 64 : 72;
  static_assert(8 * kRegsSoftmax + kDecodeWarps * kRegsDecode + 4 * kRegsControl <= (kControl + 4) * kRegsLaunch, "register split");
  static constexpr int kPanels = D / 64;
  static constexpr int kQPanel = 128 * 128;                  // bytes: 128 rows of 64 values
  static constexpr int kQTile = kPanels * kQPanel;
  static constexpr int kPanel = kStep * 128;
  static constexpr int kTile = kPanels * kPanel;             // a step of K or V
  static constexpr int kPackedStage = 2 * q4::Packed<D, kStep>::kBytes;
  // Steps are dealt in turn to two lines (split: the chains), each with operand tiles, packed stages and decoders of its own
  static constexpr int kDepthK = 2, kDepthV = kSplit ? 2 : 1, kDepthP = 3;
  static constexpr int KS = 2 * kDepthK, VS = 2 * kDepthV, PS = 2 * kDepthP;
  static constexpr int kTiles = NMT * kQTile + (KS + VS) * kTile + PS * kPackedStage;
  static constexpr int kFoldBytes = kSplit ? 2 * 128 * 8 : 0;   // (maximum, sum) of every row and chain
  static constexpr uint32_t kColO = 0, kColS = 2 * D;        // O of chain c at c * D, its scores at 2 D + c * 128 (P in their place)
};

struct Params {
  const int32_t* cache_len;
  const int32_t* q_len;
  const uint8_t *k, *v, *k_scale, *v_scale;
  __nv_bfloat16* out;
  float* lse;
  float4* ws_o;     // [slot][D / 4][rows_pad]: a part's O, four columns of a row a vector (few query rows: [slot][rows_pad][D / 4])
  float2* ws_ml;    // [slot][rows_pad]: its running maximum (log2 units) and sum
  int nl, layer_begin, batch, n_kv_heads, n_q_heads, group, capacity, q_cap;
  int rows_total;   // group * q_cap: query rows of a KV head
  int n_rc, chunk, rows, rows_pad;   // row chunks, rows of a full chunk (128 or 256), rows of a unit, those in whole warps
  int fresh_box;    // rows of a TMA box of fresh K / V
  int min_share;
  int all_lengths;  // few query rows: whether shared memory holds more of the lengths than the prefix
  FastDiv by_batch, by_rc, by_kv_heads, by_q_cap;
  float scale_log2;
  int* status;
};

// Everything that counts steps is told their size: 64 keys, or 128 in the kernel for few query rows.
template <int kKeys>
__device__ __forceinline__ int steps_of(int Lc, int Lq) { return Lq <= 0 ? 0 : (Lc + kKeys - 1) / kKeys + (Lq + kKeys - 1) / kKeys; }

template <int kKeys>
__device__ __forceinline__ void read_lengths(const Params& p, const Lengths& s, volatile int* any_empty) {
  read_lengths(p.cache_len, p.q_len, p.batch, p.capacity, p.q_cap, p.status, s, any_empty, steps_of<kKeys>);
}
__device__ __forceinline__ Deal deal_of(const Params& p, const Lengths& s, int grid) {
  return Deal(s.prefix[p.batch], p.nl * p.n_kv_heads * p.n_rc, grid, p.min_share);
}

struct Segment {
  int layer, b, kvh, rc;      // layer of the call
  int Lc, Lq, n_c;            // lengths, steps of the cache
  int unit_begin;             // item
  int begin, end;             // steps of the unit
  int slot;                   // where a part goes, -1: the unit is whole
};

// The unit that an item belongs to (not its part).
template <int kKeys>
__device__ __forceinline__ void find_unit(const Params& p, const Lengths& s, const Deal& d, int item, Segment& g) {
  int rest;
  const int grp = d.group_of(item, rest);
  g.b = element_of(s, p.batch, rest);
  g.layer = p.by_kv_heads.divmod(p.by_rc.divmod(grp, g.rc), g.kvh);
  if (kKeys == kStep || s.lc) {
    g.Lc = s.lc[g.b];
    g.Lq = s.lq[g.b];
  } else {
    g.Lc = max(0, min(p.cache_len[g.b], p.capacity));
    g.Lq = p.q_len ? max(0, min(p.q_len[g.b], p.q_cap)) : p.q_cap;
  }
  g.n_c = (g.Lc + kKeys - 1) / kKeys;
  g.unit_begin = grp * d.sum + s.prefix[g.b];
}

// Walks the segments of a block, alike in every role.
template <int kKeys = kStep>
struct Walk {
  const Params& p;
  const Lengths& s;
  const Deal& d;
  int at, first, end;
  __device__ __forceinline__ Walk(const Params& p_, const Lengths& s_, const Deal& d_, int cta) : p(p_), s(s_), d(d_) {
    at = first = cta < d.n ? d.lo(cta) : 0;
    end = cta < d.n ? d.lo(cta + 1) : 0;
  }
  __device__ __forceinline__ bool next(Segment& g) {
    if (at >= end) return false;
    find_unit<kKeys>(p, s, d, at, g);
    const int steps = s.prefix[g.b + 1] - s.prefix[g.b];
    g.begin = at - g.unit_begin;
    g.end = min(steps, end - g.unit_begin);
    g.slot = g.begin == 0 && g.end == steps ? -1 : at == first ? 2 * (int)blockIdx.x : 2 * (int)blockIdx.x + 1;
    at = g.unit_begin + g.end;
    return true;
  }
};

template <int kKeys = kStep>
__device__ __forceinline__ int step_keys(const Segment& g, int t) {
  return t < g.n_c ? min(kKeys, g.Lc - t * kKeys) : min(kKeys, g.Lq - (t - g.n_c) * kKeys);
}

#include "attn_q4_few.cuh"

template <int D, int NMT, bool kNoWait>
__global__ void __launch_bounds__(Shape<D, NMT>::kThreads, 1)
q4_attention_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_kn,
                    const __grid_constant__ CUtensorMap tm_vn, const __grid_constant__ Params p) {
  using G = Shape<D, NMT>;
  using Pk = q4::Packed<D, kStep>;
  constexpr uint64_t kLimit = kNoWait ? 0ull : kWaitLimitNs;
  constexpr int KS = G::KS, VS = G::VS, PS = G::PS, kControl = G::kControl;
  constexpr bool kSplit = G::kSplit;
  constexpr int kStride = kSplit ? 2 : 1;   // of a chain's steps; its first is step c of a segment where they are split
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_pad = (1024u - (smem_u32(smem_raw) & 1023u)) & 1023u;
  const uint32_t sm_q = smem_u32(smem_raw) + smem_pad;
  const uint32_t sm_k = sm_q + NMT * G::kQTile, sm_v = sm_k + KS * G::kTile, sm_p = sm_v + VS * G::kTile, sm_bar = sm_p + PS * G::kPackedStage;
  float2* const fold = reinterpret_cast<float2*>(smem_raw + smem_pad + G::kTiles + kBarrierBytes);   // [chain][row]
  int* const flags = reinterpret_cast<int*>(smem_raw + smem_pad + G::kTiles + kBarrierBytes + G::kFoldBytes);
  volatile int* const abort_ptr = flags;        // raised by the first wait that gives up
  volatile int* const never_ptr = flags + 1;    // for waits that must not be cut short by an abort; raised by one that runs out
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(flags + 2);
  volatile int* const any_empty = flags + 3;
  const Lengths len(flags + kFlagBytes / 4, p.batch);

  const uint32_t bar_q_full = sm_bar, bar_q_empty = sm_bar + 8, bar_drain = sm_bar + 16;              // drain [2]
  const uint32_t bar_s_ready = sm_bar + 32, bar_p_ready = sm_bar + 64, bar_pv_done = sm_bar + 96;     // [M tile][buffer]
  const uint32_t bar_k_full = sm_bar + 128, bar_k_empty = bar_k_full + 8 * KS, bar_v_full = bar_k_empty + 8 * KS, bar_v_empty = bar_v_full + 8 * VS;
  const uint32_t bar_kf = bar_v_empty + 8 * VS, bar_vf = bar_kf + 16;                                 // [line]: fresh rows copied
  const uint32_t bar_p_full = bar_vf + 16, bar_p_empty = bar_p_full + 8 * PS, bar_fold = bar_p_empty + 8 * PS;   // fold [2]
  static_assert(128 + 8 * (2 * KS + 2 * VS + 4 + 2 * PS + 2) <= kBarrierBytes, "barriers");

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // warps whose 32 query rows exist, of each chain
  auto live_warps = [&](int c) { return (max(32, min(128, p.rows - (kSplit ? 0 : 128 * c))) + 31) / 32; };

  if (tid == 0) {
    *abort_ptr = 0; *never_ptr = 0; *any_empty = 0;
    mbar_init(bar_q_full, 1);
    mbar_init(bar_q_empty, 2);
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_drain + 8 * i, 1);
      mbar_init(bar_fold + 8 * i, (uint32_t)(2 * live_warps(0)));
      for (int u = 0; u < 2; ++u) {
        mbar_init(bar_s_ready + 16 * i + 8 * u, 1);
        mbar_init(bar_p_ready + 16 * i + 8 * u, (uint32_t)live_warps(i));
        mbar_init(bar_pv_done + 16 * i + 8 * u, 1);
      }
    }
    for (int i = 0; i < KS; ++i) {
      mbar_init(bar_k_full + 8 * i, G::kTeamWarps);
      mbar_init(bar_k_empty + 8 * i, NMT);
    }
    for (int i = 0; i < VS; ++i) {
      mbar_init(bar_v_full + 8 * i, G::kTeamWarps);
      mbar_init(bar_v_empty + 8 * i, NMT);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_kf + 8 * i, 1);
      mbar_init(bar_vf + 8 * i, 1);
    }
    for (int i = 0; i < PS; ++i) {
      mbar_init(bar_p_full + 8 * i, 1);
      mbar_init(bar_p_empty + 8 * i, 2 * G::kTeamWarps);   // K and V
    }
    mbar_fence_init();
    fence_proxy_async_smem();
  }
  if (warp == kControl + 1) {
    tmem_alloc(smem_u32(tmem_slot), kTmemCols);
    tmem_relinquish();
  }
  if (warp == kControl && lane == 0) {
    prefetch_tensormap(&tm_q);
    prefetch_tensormap(&tm_kn);
    prefetch_tensormap(&tm_vn);
  }
  dlm_grid_dependency_wait();
  dlm_trigger_dependents();
  if (warp == 0) read_lengths<kStep>(p, len, any_empty);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  const Deal deal = deal_of(p, len, (int)gridDim.x);

  if (warp >= kControl) {
    setmaxnreg_dec<G::kRegsControl>();
    if (warp == kControl) {
      // ================================================================= producer
      Walk<> walk(p, len, deal, blockIdx.x);
      Segment g = {};
      uint32_t st = 0, n_q = 0, copied[2] = {0, 0};   // steps, Q tiles, packed steps of the lines so far
      bool ok = true, q_due = false;
      auto issue_q = [&]() {
        q_due = false;
        if (n_q > 0 && !mbar_wait_warp(bar_q_empty, (n_q - 1) & 1, abort_ptr, kLimit)) return false;
        const int z = (g.layer * p.batch + g.b) * p.n_kv_heads + g.kvh, mt = lane / G::kPanels, pn = lane % G::kPanels;
        if (lane == 0) mbar_expect_tx(bar_q_full, (uint32_t)(NMT * min(128, p.rows)) * 128u * G::kPanels);   // a box counts in full
        __syncwarp();
        if (mt < NMT) tma_load_3d(sm_q + mt * G::kQTile + pn * G::kQPanel, &tm_q, bar_q_full, pn * 64, g.rc * p.chunk + mt * 128, z);
        __syncwarp();
        ++n_q;
        return true;
      };
      // Q is copied as soon as the unit before has done with its own, and at the latest where this warp would wait for the
      // steps that need it
      auto wait = [&](uint32_t bar, uint32_t parity) {
        if (q_due && (n_q == 0 || mbar_test_wait_warp(bar_q_empty, (n_q - 1) & 1) || !mbar_test_wait_warp(bar, parity)) && !issue_q()) return false;
        return mbar_wait_warp(bar, parity, abort_ptr, kLimit);
      };
      while (ok && walk.next(g)) {
        q_due = true;
        if (n_q == 0) ok = issue_q();
        const size_t head = ((size_t)(g.layer + p.layer_begin) * p.batch + g.b) * p.n_kv_heads + g.kvh;
        for (int t = g.begin; t < min(g.end, g.n_c) && ok; ++t) {
          const uint32_t i = t - g.begin, x = (kSplit ? i : st + i) & 1, n = x ? copied[1] : copied[0];
          const uint32_t s = x * G::kDepthP + n % G::kDepthP, bar = bar_p_full + 8 * s;
          if (n >= (uint32_t)G::kDepthP) ok = wait(bar_p_empty + 8 * s, (n / G::kDepthP - 1) & 1);
          if (!ok) break;
          const int rows = step_keys(g, t);
          if (lane == 0) mbar_expect_tx(bar, 2 * Pk::bytes(rows));
          __syncwarp();
          if (lane < 4)   // values and scales of K and of V
            Pk::copy_part(sm_p + s * G::kPackedStage + (lane >> 1) * Pk::kBytes, lane < 2 ? p.k : p.v, lane < 2 ? p.k_scale : p.v_scale, lane & 1,
                          head * p.capacity + (size_t)t * kStep, rows, bar);
          __syncwarp();
          if (x) ++copied[1]; else ++copied[0];
        }
        st += g.end - g.begin;
        if (ok && q_due) ok = issue_q();
      }
      // no copy lands after the block has released its shared memory
      for (uint32_t x = 0; x < 2; ++x) {
        const uint32_t n = x ? copied[1] : copied[0];
        for (uint32_t i = n > (uint32_t)G::kDepthP ? n - G::kDepthP : 0; i < n; ++i)
          mbar_wait(bar_p_full + 8 * (x * G::kDepthP + i % G::kDepthP), (i / G::kDepthP) & 1, never_ptr);
      }
      if (n_q > 0) mbar_wait(bar_q_full, (n_q - 1) & 1, never_ptr);
    } else if ((warp == kControl + 1 || warp == kControl + 2) && elect_one_sync()) {
      // ================================================================= MMA issuers, one lane each
      const int c = warp - kControl - 1;
      auto wait = [&](uint32_t bar, uint32_t parity) { return mbar_wait_limit(bar, parity, abort_ptr, kLimit); };
      Walk<> walk(p, len, deal, blockIdx.x);
      Segment g = {};
      uint32_t st = 0, pt = 0, seg = 0;   // the chain's steps whose scores / whose P V product have been issued
      bool ok = true;
      const uint32_t idesc_pv = make_idesc_bf16(128, D, 1);
      const uint64_t desc_q = make_smem_desc_sw128(sm_q + (kSplit ? 0 : c) * G::kQTile, 16, 1024);
      const uint64_t desc_k0 = make_smem_desc_sw128(sm_k, 16, 1024);
      const uint64_t desc_v0 = make_smem_desc_sw128(sm_v, G::kPanel, 1024);
      const uint32_t t_o = tmem + G::kColO + c * D, t_s = tmem + G::kColS + c * 128;
      // operand tile of the chain's n-th step, and the use of it that this is
      auto stage = [&](uint32_t n, uint32_t ring) { return kSplit ? 2 * c + (n & 1) : n % ring; };
      auto use = [&](uint32_t n, uint32_t ring) { return kSplit ? n >> 1 : n / ring; };
      while (ok && walk.next(g)) {
        ok = wait(bar_q_full, seg & 1);
        if (!ok) break;
        const int first = g.begin + (kSplit ? c : 0);
        int ts = first;
        if (ts >= g.end) mbar_arrive(bar_q_empty);   // no step of the segment for this chain
        // scores of the next step that has none yet, into buffer st & 1
        auto issue_s = [&]() -> bool {
          if (ts >= g.end) return true;
          const uint32_t ks = stage(st, KS);
          if (!wait(bar_k_full + 8 * ks, use(st, KS) & 1)) return false;
          tc_fence_after_sync();
          const uint32_t idesc = make_idesc_bf16(128, (uint32_t)((step_keys(g, ts) + 15) & ~15), 0);
          const uint64_t dk = desc_offset(desc_k0, ks * G::kTile);
          const uint32_t d = t_s + (st & 1) * kStep;
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint32_t a = ((k >> 2) * G::kQPanel + (k & 3) * 32) >> 4, b = ((k >> 2) * G::kPanel + (k & 3) * 32) >> 4;
            mma_ss_lo<false>(d, (uint32_t)desc_q + a, (uint32_t)dk + b, (uint32_t)(desc_q >> 32), idesc, k > 0 ? 1u : 0u);
          }
          tc_commit(bar_s_ready + 16 * c + 8 * (st & 1));
          tc_commit(bar_k_empty + 8 * ks);
          ++st;
          ts += kStride;
          if (ts >= g.end) tc_commit(bar_q_empty);   // Q is not read again in this segment
          return true;
        };
        ok = issue_s() && issue_s();
        for (int t = first; t < g.end && ok; t += kStride, ++pt) {
          const uint32_t vs = stage(pt, VS), buf = pt & 1;
          ok = wait(bar_v_full + 8 * vs, use(pt, VS) & 1) && wait(bar_p_ready + 16 * c + 8 * buf, (pt >> 1) & 1);
          if (!ok) break;
          tc_fence_after_sync();
          const int n16 = (step_keys(g, t) + 15) & ~15;
          const uint64_t dv = desc_offset(desc_v0, vs * G::kTile);
          const uint32_t a = t_s + buf * kStep;
          if (t == first) mma_ts<false>(t_o, a, dv, idesc_pv); else mma_ts<true>(t_o, a, dv, idesc_pv);
          if (n16 == kStep) {
#pragma unroll
            for (int i = 1; i < kStep / 16; ++i) mma_ts<true>(t_o, a + i * 8, desc_offset(dv, i * 2048), idesc_pv);
          } else {
            for (int i = 1; i < n16 / 16; ++i) mma_ts<true>(t_o, a + i * 8, desc_offset(dv, i * 2048), idesc_pv);
          }
          tc_commit(bar_pv_done + 16 * c + 8 * buf);
          tc_commit(bar_v_empty + 8 * vs);
          ok = issue_s();   // the buffer just consumed takes the step after next
        }
        ++seg;
      }
      // every MMA issued by this lane has finished before TMEM and shared memory are released
      tc_commit(bar_drain + 8 * c);
      mbar_wait(bar_drain + 8 * c, 0, never_ptr);
    }
  } else if (warp >= 8) {
    // ================================================================= decoders: K of line 0, K of line 1, V of line 0, V of line 1
    // (a tile costs a warp a chain of waits, loads, conversions, stores, a fence and an arrival, most of it latency: the teams' run side by
    // side, and what a team waits on is its own, so that it need not follow the others' steps)
    setmaxnreg_dec<G::kRegsDecode>();
    constexpr int kThreadsOfTeam = G::kTeamWarps * 32;
    const int team = (warp - 8) / G::kTeamWarps, me = tid & (kThreadsOfTeam - 1);
    const bool is_k = team < 2;
    const uint32_t x = team & 1, depth = is_k ? G::kDepthK : G::kDepthV, part = is_k ? 0 : Pk::kBytes, packed0 = sm_p + x * G::kDepthP * G::kPackedStage;
    // operand tile i of the line: split, the line's tiles lie together; else the lines' alternate
    const uint32_t first_tile = kSplit ? x * depth : x, tile_step = kSplit ? 1 : 2;
    const uint32_t tiles = (is_k ? sm_k : sm_v) + first_tile * G::kTile;
    const uint32_t bar_full = (is_k ? bar_k_full : bar_v_full) + 8 * first_tile, bar_empty = (is_k ? bar_k_empty : bar_v_empty) + 8 * first_tile;
    const uint32_t bar_fresh = (is_k ? bar_kf : bar_vf) + 8 * x, bar_packed = bar_p_full + 8 * x * G::kDepthP, bar_read = bar_p_empty + 8 * x * G::kDepthP;
    const q4::Decoder<D, kStep, kThreadsOfTeam> decoder(me, G::kPanel);
    auto wait = [&](uint32_t bar, uint32_t parity) { return mbar_wait_warp(bar, parity, abort_ptr, kLimit); };
    Walk<> walk(p, len, deal, blockIdx.x);
    Segment g = {};
    uint32_t st = 0, n = 0, ps = 0, fs = 0;   // steps; the line's steps, packed ones and fresh ones
    bool ok = true, asked = false;
    while (ok && walk.next(g)) {
      for (int t = g.begin + (int)((kSplit ? x : x ^ st) & 1); t < g.end && ok; t += 2, ++n) {
        const uint32_t i = tile_step * (depth == 2 ? n & 1 : 0), use = depth == 2 ? n >> 1 : n, tile = tiles + i * G::kTile;
        const int keys = step_keys(g, t), n16 = (keys + 15) & ~15;
        if (use > 0) ok = wait(bar_empty + 8 * i, (use - 1) & 1);
        if (!ok) break;
        if (t < g.n_c) {
          const uint32_t q = ps % G::kDepthP;
          ok = wait(bar_packed + 8 * q, (ps / G::kDepthP) & 1);
          if (!ok) break;
          decoder.run(packed0 + q * G::kPackedStage + part, tile, keys);
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_read + 8 * q);
          ++ps;
        } else {
          if (me == 0) {
            mbar_expect_tx(bar_fresh, (uint32_t)p.fresh_box * 128u * G::kPanels);
            for (int pn = 0; pn < G::kPanels; ++pn)
              tma_load_3d(tile + pn * G::kPanel, is_k ? &tm_kn : &tm_vn, bar_fresh, pn * 64, (t - g.n_c) * kStep, (g.layer * p.batch + g.b) * p.n_kv_heads + g.kvh);
          }
          asked = true;
          __syncwarp();
          ok = wait(bar_fresh, fs & 1);
          if (!ok) break;
          asked = false;
          ++fs;
        }
        // V rows from `keys` to the next multiple of 16 meet P = 0: clear them, so that a NaN left there cannot reach O
        if (!is_k)
          for (int j = keys * (D / 8) + me; j < n16 * (D / 8); j += kThreadsOfTeam) q4::clear_piece<D>(tile, G::kPanel, j);
        // what was stored to the tile is visible to the tensor cores before it is announced
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_full + 8 * i);
      }
      st += g.end - g.begin;
    }
    // a copy that was given up lands before the block has released its shared memory
    if (asked && me == 0) mbar_wait(bar_fresh, fs & 1, never_ptr);
  } else {
    // ================================================================= softmax warps (those that own real rows)
    setmaxnreg_inc<G::kRegsSoftmax>();
    const int c = warp >> 2, row = (warp & 3) * 32 + lane, r_unit = kSplit ? row : c * 128 + row;
    if ((warp & 3) < live_warps(c)) {
      const uint32_t t_lane = (uint32_t)((warp & 3) * 32) << 16;
      const uint32_t t_s = tmem + t_lane + G::kColS + c * 128, t_o = tmem + t_lane + G::kColO + c * D;
      auto wait = [&](uint32_t bar, uint32_t parity) { return mbar_wait_warp(bar, parity, abort_ptr, kLimit); };
      auto out_row = [&](int layer, int b, int kvh, int rc) {
        return (((size_t)layer * p.batch + b) * p.n_q_heads + (size_t)kvh * p.group) * p.q_cap + rc * p.chunk + r_unit;
      };
      if (*any_empty && (!kSplit || c == 0)) {
        // units without any key (inactive batch elements) appear in no share: their rows are zero
        const int n_units = p.nl * p.n_kv_heads * p.n_rc * p.batch;
        for (int unit = blockIdx.x; unit < n_units; unit += gridDim.x) {
          int b, rc, kvh;
          const int layer = p.by_kv_heads.divmod(p.by_rc.divmod(p.by_batch.divmod(unit, b), rc), kvh);
          if (len.prefix[b + 1] != len.prefix[b] || r_unit >= p.rows || rc * p.chunk + r_unit >= p.rows_total) continue;
          const size_t r = out_row(layer, b, kvh, rc);
#pragma unroll
          for (int i = 0; i < D / 8; ++i) reinterpret_cast<uint4*>(p.out + r * D)[i] = make_uint4(0, 0, 0, 0);
          if (p.lse) p.lse[r] = -CUDART_INF_F;
        }
      }
      Walk<> walk(p, len, deal, blockIdx.x);
      Segment g = {};
      uint32_t st = 0, seg = 0;   // the chain's steps; segments
      bool ok = true;
      while (ok && walk.next(g)) {
        float m_used = -CUDART_INF_F, l_run = 0.f;
        const int r_kv = g.rc * p.chunk + r_unit;
        const bool real = r_unit < p.rows && r_kv < p.rows_total, active = real && r_kv - p.by_q_cap.div(r_kv) * p.q_cap < g.Lq;
        const int first = g.begin + (kSplit ? c : 0);
        for (int t = first; t < g.end; t += kStride, ++st) {
          const uint32_t buf = st & 1, before = 16 * c + 8 * ((st - 1) & 1), parity = ((st - 1) >> 1) & 1;
          ok = wait(bar_s_ready + 16 * c + 8 * buf, (st >> 1) & 1);
          if (!ok) break;
          tc_fence_after_sync();
          const int keys = step_keys(g, t);
          if (keys == kStep)
            ok = softmax_half_full<D, true>(t_s + buf * kStep, t_o, t == first, p.scale_log2, m_used, l_run, bar_pv_done + before, parity, abort_ptr, active);
          else
            ok = softmax_half_ragged<D, true>(t_s + buf * kStep, t_o, keys, t == first, p.scale_log2, m_used, l_run, bar_pv_done + before, parity, abort_ptr, active);
          if (!ok) break;
          __syncwarp();
          if (lane == 0) {
            tc_fence_before_sync();
            mbar_arrive(bar_p_ready + 16 * c + 8 * buf);
          }
        }
        // ---- O is complete once the last P V product has finished
        if (ok && first < g.end) ok = wait(bar_pv_done + 16 * c + 8 * ((st - 1) & 1), ((st - 1) >> 1) & 1);
        if (!ok) break;
        tc_fence_after_sync();
        // split: both chains' threads of a row learn of each other's maximum and sum, then each has half of the columns
        float w0 = 1.f, w1 = 0.f;
        bool both = false;
        if (kSplit) {
          fold[c * 128 + row] = make_float2(m_used, l_run);
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_fold);
          ok = wait(bar_fold, seg & 1);
          if (!ok) break;
          tc_fence_after_sync();
          const float2 a = fold[row], b = fold[128 + row];
          both = g.end - g.begin > 1;
          m_used = both ? fmaxf(a.x, b.x) : a.x;
          w0 = both ? ex2_approx(a.x - m_used) : 1.f;
          w1 = both ? ex2_approx(b.x - m_used) : 0.f;
          l_run = both ? fmaf(w0, a.y, w1 * b.y) : a.y;
        }
        constexpr int kCols = kSplit ? D / 2 : D;   // that this thread joins and stores, from c0 on
        const int c0 = kSplit ? c * kCols : 0;
        const uint32_t t_first = kSplit ? t_o - c * D : t_o;
        uint32_t v[32];
        auto read_o = [&](int col) {
          tmem_ld32(t_first + col, v);
          if (kSplit && both) {
            uint32_t u[32];
            tmem_ld32(t_first + D + col, u);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(fmaf(w1, __uint_as_float(u[j]), w0 * __uint_as_float(v[j])));
          } else {
            tmem_ld_wait();
          }
        };
        if (g.slot < 0) {
          const float inv = active ? 1.f / l_run : 0.f;
          const size_t r = out_row(g.layer, g.b, g.kvh, g.rc);
#pragma unroll 1
          for (int col = c0; col < c0 + kCols; col += 32) {
            read_o(col);
            if (!real) continue;
            uint4* o = reinterpret_cast<uint4*>(p.out + r * D + col);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t h[4];
#pragma unroll
              for (int j = 0; j < 4; ++j)
                h[j] = active ? pack_bf16(__uint_as_float(v[i * 8 + 2 * j]) * inv, __uint_as_float(v[i * 8 + 2 * j + 1]) * inv) : 0u;
              o[i] = make_uint4(h[0], h[1], h[2], h[3]);
            }
          }
          if (real && p.lse && c0 == 0) p.lse[r] = active ? (m_used + lg2_approx(l_run)) * 0.6931471805599453f : -CUDART_INF_F;
        } else {
          float4* po = p.ws_o + (size_t)g.slot * (D / 4) * p.rows_pad + r_unit;
#pragma unroll 1
          for (int col = c0; col < c0 + kCols; col += 32) {
            read_o(col);
#pragma unroll
            for (int j = 0; j < 8; ++j)
              __stcg(po + (size_t)(col / 4 + j) * p.rows_pad, make_float4(__uint_as_float(v[4 * j]), __uint_as_float(v[4 * j + 1]),
                                                                          __uint_as_float(v[4 * j + 2]), __uint_as_float(v[4 * j + 3])));
          }
          if (c0 == 0) __stcg(p.ws_ml + (size_t)g.slot * p.rows_pad + r_unit, make_float2(m_used, l_run));
        }
        tc_fence_before_sync();   // O has been read: the next segment's first product overwrites it once this thread's P is announced
        if (kSplit) {             // ... and the other chain's O and `fold`, once both have read them
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_fold + 8);
          ok = wait(bar_fold + 8, seg & 1);
          tc_fence_after_sync();
        }
        ++seg;
      }
    }
  }
  // ---- teardown: nothing of this block is in flight any more
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

// Joins the parts of split units.  Every boundary between two shares that lies inside a unit belongs to that unit; the first of them does
// the work for all its parts.  Block = (boundary, 32 rows); a warp has 8 columns, a lane a row.
//
// What is to be joined follows from the lengths, and is found while the parts are still computed (one layer: 17.5 us without this).  Nothing
// promises that lengths read before the wait are those that the attention kernel read, so they are read again behind it, next to the parts; where
// any differs, everything is done once more with the new ones.  Until then no result is stored, and parts are only read within the workspace:
// lengths are clamped, so any give slots of this grid.
template <int D, bool kFew>
__global__ void __launch_bounds__(D * 4, 2) q4_attention_join_kernel(const __grid_constant__ Params p, int grid) {
  extern __shared__ int join_smem[];
  const Lengths len(join_smem, p.batch);
  constexpr int kKeys = kFew ? few::kKeys : kStep;
  constexpr int kAtOnce = 4;
  const int row = blockIdx.y * 32 + (threadIdx.x & 31), c8 = threadIdx.x >> 5, c = blockIdx.x + 1;
  bool joins;      // the block has a unit to join, and this thread a row of it
  Segment g = {};
  float m, l, o[8];
#pragma unroll 1
  for (bool early = true;; early = false) {
    if (threadIdx.x < 32) read_lengths(p.cache_len, p.q_len, p.batch, p.capacity, p.q_cap, nullptr, len, nullptr, steps_of<kKeys>);   // (recorded by the kernel before)
    __syncthreads();
    const Deal d = deal_of(p, len, grid);
    joins = c < d.n;
    int c_first = 0, c_last = 0, first_slot = 0;
    if (joins) {
      const int boundary = d.lo(c);
      find_unit<kKeys>(p, len, d, boundary, g);
      joins = g.unit_begin != boundary && d.lo(c - 1) <= g.unit_begin;   // inside a unit, and its first
      const int unit_end = g.unit_begin + len.prefix[g.b + 1] - len.prefix[g.b];
      c_first = c - 1;
      c_last = d.owner(unit_end - 1);
      // the part of block b: its first segment if the part starts where its share does, as all but the first part do, else its second
      first_slot = 2 * c_first + (d.lo(c_first) >= g.unit_begin ? 0 : 1);
    }
    joins = joins && row < p.rows && g.rc * p.chunk + row < p.rows_total;
    int now_c = 0, now_q = 0;
    if (early) {
      dlm_grid_dependency_wait();
      dlm_trigger_dependents();
      if (threadIdx.x < p.batch) {
        now_c = clamped_length(p.cache_len, threadIdx.x, p.capacity);
        now_q = clamped_length(p.q_len, threadIdx.x, p.q_cap);
      }
    }
    m = -CUDART_INF_F;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = 0.f;
#pragma unroll 1
    for (int b0 = c_first; joins && b0 <= c_last; b0 += kAtOnce) {
      float2 ml[kAtOnce];
      float4 x[kAtOnce], y[kAtOnce];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        ml[j] = make_float2(-CUDART_INF_F, 0.f);
        x[j] = y[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (b0 + j <= c_last) {
          const size_t s = (size_t)(b0 + j == c_first ? first_slot : 2 * (b0 + j));
          const float4* po = kFew ? p.ws_o + (s * p.rows_pad + row) * (D / 4) + 2 * c8 : p.ws_o + (s * (D / 4) + 2 * c8) * p.rows_pad + row;
          ml[j] = __ldcg(p.ws_ml + s * p.rows_pad + row);
          x[j] = __ldcg(po);
          y[j] = __ldcg(po + (kFew ? 1 : p.rows_pad));
        }
      }
      float m_new = m;
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) m_new = fmaxf(m_new, ml[j].x);
      const float old = ex2_approx(m - m_new);   // the first time 2^-inf = 0
      l *= old;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] *= old;
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const float w = ex2_approx(ml[j].x - m_new);
        l = fmaf(w, ml[j].y, l);
        o[0] = fmaf(w, x[j].x, o[0]); o[1] = fmaf(w, x[j].y, o[1]); o[2] = fmaf(w, x[j].z, o[2]); o[3] = fmaf(w, x[j].w, o[3]);
        o[4] = fmaf(w, y[j].x, o[4]); o[5] = fmaf(w, y[j].y, o[5]); o[6] = fmaf(w, y[j].z, o[6]); o[7] = fmaf(w, y[j].w, o[7]);
      }
      m = m_new;
    }
    if (!early) break;
    bool changed = threadIdx.x < p.batch && (now_c != len.lc[threadIdx.x] || now_q != len.lq[threadIdx.x]);
    for (int b = threadIdx.x + D * 4; b < p.batch; b += D * 4)
      changed |= clamped_length(p.cache_len, b, p.capacity) != len.lc[b] || clamped_length(p.q_len, b, p.q_cap) != len.lq[b];
    if (!__syncthreads_or(changed)) break;
  }
  if (!joins) return;
  const int r_kv = g.rc * p.chunk + row;
  const bool active = r_kv - p.by_q_cap.div(r_kv) * p.q_cap < g.Lq;
  const size_t out = (((size_t)g.layer * p.batch + g.b) * p.n_q_heads + (size_t)g.kvh * p.group) * p.q_cap + r_kv;
  const float inv = 1.f / l;
  uint32_t h[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) h[j] = active ? pack_bf16(o[2 * j] * inv, o[2 * j + 1] * inv) : 0u;
  *reinterpret_cast<uint4*>(p.out + out * D + c8 * 8) = make_uint4(h[0], h[1], h[2], h[3]);
  if (c8 == 0 && p.lse) p.lse[out] = active ? (m + lg2_approx(l)) * 0.6931471805599453f : -CUDART_INF_F;
}

// The kernels: few query rows a KV head (up to 16, up to 32), one M tile (up to 128), two; D 128 and 64; the last, with waits that do not wait.
using Kernel = void (*)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const Params);
constexpr int kKinds = 4;
template <int D, bool kNoWait>
Kernel kernel_of(int kind) {
  switch (kind) {
    case 0: return few::q4_attention_few_kernel<D, 16, kNoWait>;
    case 1: return few::q4_attention_few_kernel<D, 32, kNoWait>;
    case 2: return q4_attention_kernel<D, 1, kNoWait>;
    default: return q4_attention_kernel<D, 2, kNoWait>;
  }
}
template <int D>
int tile_bytes(int kind) {
  switch (kind) {
    case 0: return few::Shape<D, 16>::kTiles + few::Shape<D, 16>::kExchange;
    case 1: return few::Shape<D, 32>::kTiles + few::Shape<D, 32>::kExchange;
    case 2: return Shape<D, 1>::kTiles + Shape<D, 1>::kFoldBytes;
    default: return Shape<D, 2>::kTiles;
  }
}

struct Workspace {
  size_t o_bytes, ml_bytes;
};
// Whether a call of these sizes is taken: query rows are counted in 32 bits, and shared memory holds the lengths of so many sequences.
bool sizes_taken(int n_q_heads, int n_kv_heads, int q_cap, int batch) {
  return n_q_heads % n_kv_heads == 0 && q_cap <= kMaxQCap && (long long)(n_q_heads / n_kv_heads) * q_cap <= (1 << 20) && batch <= kMaxBatch;
}
Workspace workspace_of(const dlm_ctx* ctx, int head_dim, int rows_total) {
  const size_t slots = 2 * (size_t)(ctx->num_sms < kMaxGrid ? ctx->num_sms : kMaxGrid), pad = (size_t)((rows_total < 256 ? rows_total : 256) + 31) / 32 * 32;
  return {slots * pad * head_dim * sizeof(float), slots * pad * 2 * sizeof(float)};
}

}  // namespace

extern "C" size_t dlm_attn_workspace_bytes_q4(const dlm_ctx* ctx, const dlm_kv_cache_q4* cache, int n_layers_in_call,
                                              int n_q_heads, int q_cap) {
  if (!ctx || !cache || n_layers_in_call <= 0 || n_q_heads <= 0 || q_cap <= 0 || cache->n_kv_heads <= 0 || cache->batch <= 0 ||
      (cache->head_dim != 64 && cache->head_dim != 128) || !sizes_taken(n_q_heads, cache->n_kv_heads, q_cap, cache->batch))
    return 0;
  const Workspace w = workspace_of(ctx, cache->head_dim, n_q_heads / cache->n_kv_heads * q_cap);
  return w.o_bytes + w.ml_bytes;
}

extern "C" int dlm_freecache_attn_step_q4(dlm_ctx* ctx, const dlm_kv_cache_q4* cache, int layer_begin, int layer_end, const void* q,
                                          const void* k_new, const void* v_new, int n_q_heads, int q_cap, const int32_t* q_len,
                                          float softmax_scale, int cache_len_hint, void* out, float* lse, void* workspace,
                                          size_t workspace_bytes, void* stream) {
  if (!ctx || !q || !k_new || !v_new || !out) return DLM_ERR_NULL;
  const int bad = dlm_check_q4(cache);
  if (bad != DLM_OK) return bad;
  if (n_q_heads <= 0 || q_cap <= 0 || layer_begin < 0 || layer_end > cache->n_layers || layer_begin >= layer_end) return DLM_ERR_SHAPE;
  if (!sizes_taken(n_q_heads, cache->n_kv_heads, q_cap, cache->batch)) return DLM_ERR_UNSUPPORTED;
  const int D = cache->head_dim, group = n_q_heads / cache->n_kv_heads, nl = layer_end - layer_begin;
  if (((uintptr_t)q | (uintptr_t)k_new | (uintptr_t)v_new | (uintptr_t)out) & 15) return DLM_ERR_UNSUPPORTED;
  const int rows_total = group * q_cap, kind = rows_total <= 16 ? 0 : rows_total <= 32 ? 1 : rows_total <= 128 ? 2 : 3;
  const bool is_few = kind < 2;
  const int chunk = kind == 3 ? 256 : 128, n_rc = (rows_total + chunk - 1) / chunk;
  const long long units = (long long)nl * cache->batch * cache->n_kv_heads * n_rc;
  const int step = is_few ? few::kKeys : kStep;
  const long long steps = (cache->capacity + step - 1) / step + (q_cap + step - 1) / step;
  if (units * steps >= (1LL << 30)) return DLM_ERR_UNSUPPORTED;   // items are counted in 32 bits
  DLM_DEVICE_TRY(ctx);
  const Workspace ws = workspace_of(ctx, D, rows_total);
  if (!workspace || workspace_bytes < ws.o_bytes + ws.ml_bytes || ((uintptr_t)workspace & 255)) return DLM_ERR_WORKSPACE;
  const bool no_wait = ctx->wait_limit_ns == 0;
  const Kernel kern = D == 128 ? (no_wait ? kernel_of<128, true>(kind) : kernel_of<128, false>(kind))
                               : (no_wait ? kernel_of<64, true>(kind) : kernel_of<64, false>(kind));
  const int which = kind + (D == 128 ? 0 : kKinds) + (no_wait ? 2 * kKinds : 0);
  if (ctx->q4_smem_limit[which] == 0) {
    cudaFuncAttributes a;
    DLM_CUDA_TRY(cudaFuncGetAttributes(&a, reinterpret_cast<const void*>(kern)));
    const int regs = is_few ? few::kRegsLaunch : kind == 2 ? Shape<64, 1>::kRegsLaunch : Shape<64, 2>::kRegsLaunch;
    if (a.numRegs != regs) return DLM_ERR_UNSUPPORTED;   // the register split would wait for ever
    const int limit = ctx->max_smem_optin - (int)a.sharedSizeBytes;
    DLM_CUDA_TRY(cudaFuncSetAttribute(reinterpret_cast<const void*>(kern), cudaFuncAttributeMaxDynamicSharedMemorySize, limit));
    ctx->q4_smem_limit[which] = limit;
  }
  const int without_lengths = 1024 + (D == 128 ? tile_bytes<128>(kind) : tile_bytes<64>(kind)) + kBarrierBytes + kFlagBytes;
  // (heads of 128, few query rows: there is room for all lengths of 399 sequences, for the prefix alone of 1024)
  const bool all_lengths = !is_few || without_lengths + 4 * length_ints(cache->batch) <= ctx->q4_smem_limit[which];
  const int smem = without_lengths + 4 * length_ints(cache->batch, all_lengths);
  if (smem > ctx->q4_smem_limit[which]) return DLM_ERR_UNSUPPORTED;
  Params p;
  p.all_lengths = all_lengths;
  p.n_rc = n_rc;
  p.cache_len = cache->cache_len;
  p.q_len = q_len;
  p.k = static_cast<const uint8_t*>(cache->k);
  p.v = static_cast<const uint8_t*>(cache->v);
  p.k_scale = static_cast<const uint8_t*>(cache->k_scale);
  p.v_scale = static_cast<const uint8_t*>(cache->v_scale);
  p.out = static_cast<__nv_bfloat16*>(out);
  p.lse = lse;
  p.ws_o = static_cast<float4*>(workspace);
  p.ws_ml = reinterpret_cast<float2*>(static_cast<uint8_t*>(workspace) + ws.o_bytes);
  p.nl = nl;
  p.layer_begin = layer_begin;
  p.batch = cache->batch;
  p.n_kv_heads = cache->n_kv_heads;
  p.n_q_heads = n_q_heads;
  p.group = group;
  p.capacity = cache->capacity;
  p.q_cap = q_cap;
  p.rows_total = rows_total;
  p.chunk = chunk;
  p.rows = rows_total < chunk ? rows_total : chunk;
  p.rows_pad = (p.rows + 31) & ~31;
  p.fresh_box = q_cap < step ? q_cap : step;
  p.min_share = 2;
  p.by_batch = make_fast_div(p.batch);
  p.by_rc = make_fast_div(p.n_rc);
  p.by_kv_heads = make_fast_div(p.n_kv_heads);
  p.by_q_cap = make_fast_div(q_cap);
  p.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)D)) * 1.4426950408889634f;
  p.status = &ctx->words->status;
  CUtensorMap tm_q, tm_kn, tm_vn;
  const long long slabs = (long long)nl * cache->batch * cache->n_kv_heads;
  int rc = encode_rows_map(ctx, &tm_q, q, D, rows_total, slabs, p.rows < 128 ? p.rows : 128);
  if (rc == DLM_OK) rc = encode_rows_map(ctx, &tm_kn, k_new, D, q_cap, slabs, p.fresh_box);
  if (rc == DLM_OK) rc = encode_rows_map(ctx, &tm_vn, v_new, D, q_cap, slabs, p.fresh_box);
  if (rc != DLM_OK) return rc;
  // blocks that find work if the cache is as long as expected (else fewer blocks have more)
  const int expected = cache_len_hint > 0 && cache_len_hint < cache->capacity ? cache_len_hint : cache->capacity;
  const long long most = (units * ((expected + step - 1) / step + (q_cap + step - 1) / step) + p.min_share - 1) / p.min_share;
  const int sms = ctx->num_sms < kMaxGrid ? ctx->num_sms : kMaxGrid, grid = most < sms ? (int)most : sms;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  DLM_CUDA_TRY(dlm_launch(kern, dim3(grid), dim3(is_few ? few::kThreads : kind == 2 ? Shape<64, 1>::kThreads : Shape<64, 2>::kThreads), (size_t)smem, st, tm_q, tm_kn, tm_vn, p));
  if (grid == 1) return dlm_launch_ok(ctx, 1);
  const dim3 join((unsigned)(grid - 1), (unsigned)(p.rows_pad / 32));
  const size_t join_smem = 4 * (size_t)length_ints(cache->batch);
  void (*const join_kern)(const Params, int) = D == 128 ? (is_few ? q4_attention_join_kernel<128, true> : q4_attention_join_kernel<128, false>)
                                                        : (is_few ? q4_attention_join_kernel<64, true> : q4_attention_join_kernel<64, false>);
  DLM_CUDA_TRY(dlm_launch(join_kern, join, dim3(D * 4), join_smem, st, p, grid));
  return dlm_launch_ok(ctx, 2);
}

// Attention over the 4-bit cache for up to 32 query rows a KV head (single tokens, small windows of multi-head models).  Included by
// attn_step_q4.cu, whose parameters, units, segments and joining of parts it shares.
//
// With the query rows as the tensor cores' 128 rows, most of a product would be padding, and so few warps would have a row that a
// step's softmax, a chain of one warp, took 1800 cycles.  Here the keys are those rows: S^T = K Q^T has a key a TMEM lane, so each of
// 128 threads has a key and works along the query rows; O^T = V^T P^T has a value column a lane.  What a softmax needs across keys is
// then across threads, and is avoided: P = 2^(s - m) for a reference m per query row that need not be its maximum.  P is bf16 and
// sums are fp32, whose range is that of 2^127, so the reference is the score of the first key of a group's first tile, kept for the rest
// of the segment unless some score exceeds it by 30 (then every thread of the group learns of it before P is used, m becomes the tile's largest
// score, and the sums and O^T are moved to it).  A first score that is not finite is no reference: the lowest number stands in for it, which any
// finite score then replaces.  Sums are per thread and added up once, at the end of the segment, in a fixed order.
//
// P is rounded to bf16, by at most 2^-8 of itself, since the products take it so; the sums add it unrounded.  An output is off by at most
// 2^-8 sum p |v| from this, about what its own rounding to bf16 costs.
//
// 8 sequences of 3630 to 4001 rows, 32 heads, one query row each: 71 us, 1.9 TB/s of the cache, bound by decoding (98 us with query rows as the
// products' rows and two chains, 192 with one); of 1 to 4001 rows evenly: 46 us, 1.5 TB/s.  For 64 query rows the same form takes 781 us where two chains
// take 750, and for one small layer 19 instead of 8.6.
// Those are scores that seldom exceed a part's first by 30.  Keys twice, 4, 8 and 32 times as large: 79, 87, 92 and 108 us; references that move in every
// tile 154, NaN in every tile 168 (32 query rows: 90, and 131, 135, 212, 299, 305 and 317).
//
// Steps ("tiles") of 128 keys, dealt in turn to two groups of four warps, each with an O^T, references and sums of its own.  Block = 28 warps:
//   warps 0-3, 4-7    the groups
//   warps 8-23        decoders: K of even tiles (counted over the block's life), K of odd ones, V of even, V of odd; one lane of each has fresh
//                     rows copied.  A warp alone issues an instruction in five cycles, so a tile takes four warps about 1100 to decode.
//   warp  24          producer
//   warps 25, 26      issuers of S^T and of O^T (one lane each), in the tiles' order
//   warp  27          zeros for query rows that take no part, whose contents would call for other references
namespace few {

constexpr int kThreads = 896;
constexpr int kKeys = 128;
constexpr int kRegsLaunch = 72, kRegsGroup = 96, kRegsDecode = 64, kRegsControl = 56;
static_assert(2 * kRegsGroup + 4 * kRegsDecode + kRegsControl <= 7 * kRegsLaunch, "register split");
constexpr uint32_t kTooLarge = (127u + 30u) << 7;   // bf16 of 2^30: P of a segment's keys times values up to 2^80 sums up in fp32
constexpr float kLowest = -3.402823466e38f;

// Numbers as unsigned integers in the same order; 0 is none of them.
__device__ __forceinline__ uint32_t to_ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t o) { return __uint_as_float(o >> 31 ? o & 0x7FFFFFFFu : ~o); }

template <int D, int N>
struct Shape {
  static constexpr int kPanels = D / 64;
  static constexpr int kPanel = kKeys * 128;                    // bytes of a panel of a K or V tile: 128 rows of 64 values
  static constexpr int kTile = kPanels * kPanel;
  static constexpr int kQPanel = N * 128, kQTile = kPanels * kQPanel;
  static constexpr int kPTile = kKeys * 128;                    // P of a group's tile: a key's N values in a row of 128 bytes
  static constexpr int kPackedStage = 2 * q4::Packed<D, 64>::kBytes;   // half a tile
  // packed stages of either line (the even tiles and the odd ones have tiles, packed stages and decoders of their own)
  static constexpr int KS = 2, VS = 2, kDepthP = D == 128 ? 3 : 6, PS = 2 * kDepthP;
  // (P behind V: with heads of 64 the products read a second panel behind a V tile, whose rows of O^T nobody reads)
  static constexpr int kTiles = (KS + VS) * kTile + 2 * kPTile + kQTile + PS * kPackedStage;
  // floats: minus the references [2][N], parts of sums [2][4][N], weights of the groups [2][N], next references [2][N]
  static constexpr int kExchange = 4 * (2 + 8 + 2 + 2) * N;
  static constexpr uint32_t kColS = 0, kColO = 256;             // S^T: [group][buffer] of 64 columns; O^T: [group] of 64
};

// Sums of N per-lane values over the warp's lanes: v[0] of each lane is the sum of column column_of(lane).
template <int N>
__device__ __forceinline__ void reduce_columns(float (&v)[N]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int off = 16, half = N / 2; off >= 1; off >>= 1, half >>= 1) {
    if (half >= 1) {
      const bool up = lane & off;
#pragma unroll
      for (int k = 0; k < (half >= 1 ? half : 1); ++k) {
        const float send = up ? v[k] : v[k + half], keep = up ? v[k + half] : v[k];
        v[k] = keep + __shfl_xor_sync(0xffffffffu, send, off);
      }
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], off);
    }
  }
}
template <int N>
__device__ __forceinline__ int column_of(int lane) {
  return N == 32 ? lane : lane >> 1;
}

template <int D, int N, bool kNoWait>
__global__ void __launch_bounds__(kThreads, 1)
q4_attention_few_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_kn,
                        const __grid_constant__ CUtensorMap tm_vn, const __grid_constant__ Params p) {
  using G = Shape<D, N>;
  using Pk = q4::Packed<D, 64>;
  constexpr uint64_t kLimit = kNoWait ? 0ull : kWaitLimitNs;
  constexpr int KS = G::KS, VS = G::VS, PS = G::PS;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_pad = (1024u - (smem_u32(smem_raw) & 1023u)) & 1023u;
  const uint32_t sm_k = smem_u32(smem_raw) + smem_pad, sm_v = sm_k + KS * G::kTile, sm_pt = sm_v + VS * G::kTile, sm_q = sm_pt + 2 * G::kPTile;
  const uint32_t sm_p = sm_q + G::kQTile, sm_x = sm_p + PS * G::kPackedStage, sm_bar = sm_x + G::kExchange;
  float* const xch = reinterpret_cast<float*>(smem_raw + smem_pad + G::kTiles);
  float* const minus_m = xch;              // [group][N], log2 units
  float* const sums = xch + 2 * N;         // [group][warp][N]
  float* const share = xch + 10 * N;       // [group][N]: what O^T of the group is multiplied with
  uint32_t* const next_m = reinterpret_cast<uint32_t*>(xch + 12 * N);   // [group][N]: the largest score above the reference (to_ordered; 0: none)
  int* const flags = reinterpret_cast<int*>(smem_raw + smem_pad + G::kTiles + G::kExchange + kBarrierBytes);
  volatile int* const abort_ptr = flags;
  volatile int* const never_ptr = flags + 1;
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(flags + 2);
  volatile int* const any_empty = flags + 3;
  volatile uint32_t* const too_large = reinterpret_cast<volatile uint32_t*>(flags + 4);   // [group]: the group's last tile (counted from 1) with such a score
  const Lengths len(flags + kFlagBytes / 4, p.batch, p.all_lengths);

  const uint32_t bar_q_full = sm_bar, bar_q_empty = sm_bar + 8, bar_drain = sm_bar + 16, bar_fold = sm_bar + 32;   // [1], [1], [2], [3]
  const uint32_t bar_s_ready = sm_bar + 56, bar_s_empty = bar_s_ready + 32;                       // [group][buffer]
  const uint32_t bar_pt_full = bar_s_empty + 32, bar_pv_done = bar_pt_full + 16, bar_vote = bar_pv_done + 16, bar_ref = bar_vote + 16;   // [group]
  const uint32_t bar_slow = bar_ref + 16;                                                         // [group]
  const uint32_t bar_k_full = bar_slow + 16, bar_k_empty = bar_k_full + 16, bar_v_full = bar_k_empty + 16, bar_v_empty = bar_v_full + 16;
  const uint32_t bar_kf = bar_v_empty + 16, bar_vf = bar_kf + 16, bar_p_full = bar_vf + 16, bar_p_empty = bar_p_full + 8 * PS;
  const uint32_t bar_q_ready = bar_p_empty + 8 * PS;
  static_assert(56 + 64 + 5 * 16 + 6 * 16 + 16 * PS + 8 <= kBarrierBytes, "barriers");

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    *abort_ptr = 0; *never_ptr = 0; *any_empty = 0;
    too_large[0] = too_large[1] = 0;
    mbar_init(bar_q_full, 1);
    mbar_init(bar_q_ready, 1);
    mbar_init(bar_q_empty, 1);
    for (int i = 0; i < 3; ++i) mbar_init(bar_fold + 8 * i, 8);
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_drain + 8 * i, 1);
      mbar_init(bar_pt_full + 8 * i, 4);
      mbar_init(bar_pv_done + 8 * i, 1);
      mbar_init(bar_vote + 8 * i, 4);
      mbar_init(bar_ref + 8 * i, 1);
      mbar_init(bar_slow + 8 * i, 4);
      mbar_init(bar_k_full + 8 * i, 4);
      mbar_init(bar_k_empty + 8 * i, 1);
      mbar_init(bar_v_full + 8 * i, 4);
      mbar_init(bar_v_empty + 8 * i, 1);
      mbar_init(bar_kf + 8 * i, 1);
      mbar_init(bar_vf + 8 * i, 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar_s_ready + 8 * i, 1);
      mbar_init(bar_s_empty + 8 * i, 4);
    }
    for (int i = 0; i < PS; ++i) {
      mbar_init(bar_p_full + 8 * i, 1);
      mbar_init(bar_p_empty + 8 * i, 8);
    }
    mbar_fence_init();
    fence_proxy_async_smem();
  }
  if (tid < 2 * N) next_m[tid] = 0;
  if (warp == 25) {
    tmem_alloc(smem_u32(tmem_slot), kTmemCols);
    tmem_relinquish();
  }
  if (warp == 24 && lane == 0) {
    prefetch_tensormap(&tm_q);
    prefetch_tensormap(&tm_kn);
    prefetch_tensormap(&tm_vn);
  }
  dlm_grid_dependency_wait();
  dlm_trigger_dependents();
  if (warp == 0) read_lengths<kKeys>(p, len, any_empty);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  const Deal deal = deal_of(p, len, (int)gridDim.x);
  Walk<kKeys> walk(p, len, deal, blockIdx.x);
  Segment g = {};
  bool ok = true;
  auto wait = [&](uint32_t bar, uint32_t parity) { return mbar_wait_warp(bar, parity, abort_ptr, kLimit); };

  if (warp >= 24) {
    setmaxnreg_dec<kRegsControl>();
    if (warp == 24) {
      // ================================================================= producer
      uint32_t st = 0, n_q = 0, copied[2] = {0, 0};   // tiles, Q, packed stages of the lines
      while (ok && walk.next(g)) {
        const size_t head = ((size_t)(g.layer + p.layer_begin) * p.batch + g.b) * p.n_kv_heads + g.kvh;
        bool q_due = true;
        auto issue_q = [&]() {
          q_due = false;
          if (n_q > 0 && !wait(bar_q_empty, (n_q - 1) & 1)) return false;
          if (lane == 0) mbar_expect_tx(bar_q_full, (uint32_t)p.rows * 128u * G::kPanels);
          __syncwarp();
          if (lane < G::kPanels)
            tma_load_3d(sm_q + lane * G::kQPanel, &tm_q, bar_q_full, lane * 64, 0, (g.layer * p.batch + g.b) * p.n_kv_heads + g.kvh);
          __syncwarp();
          ++n_q;
          return true;
        };
        if (n_q == 0) ok = issue_q();
        for (int t = g.begin; t < min(g.end, g.n_c) && ok; ++t) {
          const uint32_t x = (st + (t - g.begin)) & 1;
          const int keys = step_keys<kKeys>(g, t);
          for (int from = 0; from < keys && ok; from += 64) {
            const uint32_t n = x ? copied[1] : copied[0], s = x * G::kDepthP + n % G::kDepthP, bar = bar_p_full + 8 * s;
            if (n >= (uint32_t)G::kDepthP) {
              const uint32_t parity = (n / G::kDepthP - 1) & 1;
              // Q as soon as the unit before has done with its own, and at the latest where this warp would wait for tiles that need it
              if (q_due && (mbar_test_wait_warp(bar_q_empty, (n_q - 1) & 1) || !mbar_test_wait_warp(bar_p_empty + 8 * s, parity))) ok = issue_q();
              ok = ok && wait(bar_p_empty + 8 * s, parity);
            }
            if (!ok) break;
            const int rows = min(64, keys - from);
            if (lane == 0) mbar_expect_tx(bar, 2 * Pk::bytes(rows));
            __syncwarp();
            if (lane < 4)
              Pk::copy_part(sm_p + s * G::kPackedStage + (lane >> 1) * Pk::kBytes, lane < 2 ? p.k : p.v, lane < 2 ? p.k_scale : p.v_scale, lane & 1,
                            head * p.capacity + (size_t)t * kKeys + from, rows, bar);
            __syncwarp();
            if (x) ++copied[1]; else ++copied[0];
          }
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
    } else if (warp == 25 && elect_one_sync()) {
      // ================================================================= issuer of S^T
      auto wait1 = [&](uint32_t bar, uint32_t parity) { return mbar_wait_limit(bar, parity, abort_ptr, kLimit); };
      const uint64_t desc_k0 = make_smem_desc_sw128(sm_k, 16, 1024), desc_q = make_smem_desc_sw128(sm_q, 16, 1024);
      const uint32_t idesc = make_idesc_bf16(128, N, 0);
      uint32_t st = 0, seg = 0, own[2] = {0, 0};   // tiles, segments, tiles of the groups
      while (ok && walk.next(g)) {
        ok = wait1(bar_q_ready, seg & 1);
        for (int t = g.begin; t < g.end && ok; ++t, ++st) {
          const uint32_t w = (t - g.begin) & 1, s = st & 1, n = w ? own[1]++ : own[0]++, buf = 16 * w + 8 * (n & 1);
          ok = wait1(bar_k_full + 8 * s, (st >> 1) & 1) && (n < 2 || wait1(bar_s_empty + buf, ((n >> 1) - 1) & 1));
          if (!ok) break;
          tc_fence_after_sync();
          const uint64_t dk = desc_offset(desc_k0, s * G::kTile);
          const uint32_t d = tmem + G::kColS + w * 128 + (n & 1) * 64;
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint32_t a = ((k >> 2) * G::kPanel + (k & 3) * 32) >> 4, b = ((k >> 2) * G::kQPanel + (k & 3) * 32) >> 4;
            mma_ss_lo<false>(d, (uint32_t)dk + a, (uint32_t)desc_q + b, (uint32_t)(dk >> 32), idesc, k > 0 ? 1u : 0u);
          }
          tc_commit(bar_s_ready + buf);
          tc_commit(bar_k_empty + 8 * s);
          if (t + 1 == g.end) tc_commit(bar_q_empty);
        }
        ++seg;
      }
      tc_commit(bar_drain);
      mbar_wait(bar_drain, 0, never_ptr);
    } else if (warp == 26 && elect_one_sync()) {
      // ================================================================= issuer of O^T
      auto wait1 = [&](uint32_t bar, uint32_t parity) { return mbar_wait_limit(bar, parity, abort_ptr, kLimit); };
      const uint64_t desc_v0 = make_smem_desc_sw128(sm_v, G::kPanel, 1024), desc_p0 = make_smem_desc_sw128(sm_pt, 16, 1024);
      const uint32_t idesc = make_idesc_bf16(128, N, 1) | (1u << 15);   // both operands have the keys along their rows
      uint32_t st = 0, own[2] = {0, 0};
      while (ok && walk.next(g)) {
        for (int t = g.begin; t < g.end && ok; ++t, ++st) {
          const uint32_t w = (t - g.begin) & 1, s = st & 1, n = w ? own[1]++ : own[0]++;
          ok = wait1(bar_v_full + 8 * s, (st >> 1) & 1) && wait1(bar_pt_full + 8 * w, n & 1);
          if (!ok) break;
          tc_fence_after_sync();
          const uint32_t dv = (uint32_t)desc_offset(desc_v0, s * G::kTile), dp = (uint32_t)desc_offset(desc_p0, w * G::kPTile);
          const uint32_t d = tmem + G::kColO + w * 64, steps = (step_keys<kKeys>(g, t) + 15) / 16;
          for (uint32_t k = 0; k < steps; ++k)
            mma_ss_lo<false>(d, dv + k * (2048 >> 4), dp + k * (2048 >> 4), (uint32_t)(desc_v0 >> 32), idesc, k > 0 || t - g.begin >= 2 ? 1u : 0u);
          tc_commit(bar_pv_done + 8 * w);
          tc_commit(bar_v_empty + 8 * s);
        }
      }
      tc_commit(bar_drain + 8);
      mbar_wait(bar_drain + 8, 0, never_ptr);
    } else if (warp == 27) {
      // ================================================================= query rows
      for (uint32_t seg = 0; ok && walk.next(g); ++seg) {
        ok = wait(bar_q_full, seg & 1);
        if (!ok) break;
        if (seg == 0 || g.Lq < p.q_cap)      // (no copy reaches the rows behind the last)
          for (int r = 0; r < N; ++r)
            if ((r >= p.rows || r - p.by_q_cap.div(r) * p.q_cap >= g.Lq) && lane < D / 8) q4::clear_piece<D>(sm_q, G::kQPanel, r * (D / 8) + lane);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_q_ready);
      }
    }
  } else if (warp >= 8) {
    // ================================================================= decoders
    setmaxnreg_dec<kRegsDecode>();
    const bool is_k = warp < 16;
    const int me = tid & 127;
    const uint32_t odd = (warp >> 2) & 1, part = is_k ? 0 : Pk::kBytes, tile = (is_k ? sm_k : sm_v) + odd * G::kTile;
    const uint32_t bar_full = (is_k ? bar_k_full : bar_v_full) + 8 * odd, bar_empty = (is_k ? bar_k_empty : bar_v_empty) + 8 * odd;
    const uint32_t bar_fresh = (is_k ? bar_kf : bar_vf) + 8 * odd;
    const q4::Decoder<D, 64, 128> decoder(me, G::kPanel);
    uint32_t st = 0, n = 0, ps = 0, fs = 0;   // tiles; the line's tiles, packed stages and fresh tiles
    bool asked = false;
    while (ok && walk.next(g)) {
      for (int t = g.begin + (int)((odd ^ st) & 1); t < g.end && ok; t += 2, ++n) {
        if (n > 0) ok = wait(bar_empty, (n - 1) & 1);
        if (!ok) break;
        const int keys = step_keys<kKeys>(g, t), n16 = (keys + 15) & ~15;
        if (t < g.n_c) {
          for (int from = 0; from < keys && ok; from += 64, ++ps) {
            const uint32_t q = odd * G::kDepthP + ps % G::kDepthP;
            ok = wait(bar_p_full + 8 * q, (ps / G::kDepthP) & 1);
            if (!ok) break;
            decoder.run(sm_p + q * G::kPackedStage + part, tile + from * 128, min(64, keys - from));
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_p_empty + 8 * q);
          }
          if (!ok) break;
        } else {
          if (me == 0) {
            mbar_expect_tx(bar_fresh, (uint32_t)p.fresh_box * 128u * G::kPanels);
            for (int pn = 0; pn < G::kPanels; ++pn)
              tma_load_3d(tile + pn * G::kPanel, is_k ? &tm_kn : &tm_vn, bar_fresh, pn * 64, 0, (g.layer * p.batch + g.b) * p.n_kv_heads + g.kvh);
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
          for (int i = keys * (D / 8) + me; i < n16 * (D / 8); i += 128) q4::clear_piece<D>(tile, G::kPanel, i);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_full);
      }
      st += g.end - g.begin;
    }
    // a copy that was given up lands before the block has released its shared memory
    if (asked && me == 0) mbar_wait(bar_fresh, fs & 1, never_ptr);
  } else {
    // ================================================================= the groups
    setmaxnreg_inc<kRegsGroup>();
    const int w = warp >> 2, key = tid & 127;                      // key of the tile; value column of O^T
    const uint32_t t_lane = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t sm_m = sm_x + w * N * 4, pt_row = sm_pt + w * G::kPTile + key * 128;
    const uint64_t scale2 = pack2(p.scale_log2, p.scale_log2);
    if (*any_empty) {
      // units without any key (inactive batch elements) appear in no share: their rows are zero
      const int n_units = p.nl * p.n_kv_heads * p.batch;
      for (int unit = blockIdx.x; unit < n_units; unit += gridDim.x) {
        int b, kvh;
        const int layer = p.by_kv_heads.divmod(p.by_batch.divmod(unit, b), kvh);
        if (len.prefix[b + 1] != len.prefix[b]) continue;
        const size_t r0 = (((size_t)layer * p.batch + b) * p.n_q_heads + (size_t)kvh * p.group) * p.q_cap;
        for (int i = tid; i < p.rows * (D / 8); i += 256) reinterpret_cast<uint4*>(p.out + r0 * D)[i] = make_uint4(0, 0, 0, 0);
        if (p.lse && tid < p.rows) p.lse[r0 + tid] = -CUDART_INF_F;
      }
    }
    uint32_t n_own = 0, seg = 0, refs = 0, slow = 0;               // the group's tiles, segments, segments with a tile of the group, slow turns
    while (ok && walk.next(g)) {
      uint64_t l2[N / 2];                                          // sums of the thread's keys, pairs of query rows
#pragma unroll
      for (int i = 0; i < N / 2; ++i) l2[i] = 0;
      const uint32_t n_first = n_own;
      for (int t = g.begin + w; t < g.end && ok; t += 2, ++n_own) {
        const uint32_t b = n_own & 1, buf = 16 * w + 8 * b, t_s = tmem + t_lane + G::kColS + w * 128 + b * 64;
        const int keys = step_keys<kKeys>(g, t);
        const bool valid = key < keys;
        ok = wait(bar_s_ready + buf, (n_own >> 1) & 1);
        if (!ok) break;
        tc_fence_after_sync();
        uint32_t v[16];
        if (n_own == n_first) {
          // the references: the first key's scores
          if ((warp & 3) == 0) {
#pragma unroll 1
            for (int c = 0; c < N; c += 16) {
              tmem_ld16(t_s + c, v);
              tmem_ld_wait();
              if (lane == 0) {
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                  const float m = __fmul_ru(__uint_as_float(v[j]), p.scale_log2);   // (up: scaled_maximum)
                  minus_m[w * N + c + j] = fabsf(m) <= -kLowest ? -m : -kLowest;
                }
              }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_ref + 8 * w);
          }
          ok = wait(bar_ref + 8 * w, refs & 1);
          if (!ok) break;
          ++refs;
        }
        if (n_own > 0) ok = wait(bar_pv_done + 8 * w, (n_own - 1) & 1);   // P of the group's last tile has been read
        if (!ok) break;
        uint32_t most = 0;                                         // of the bf16 P, by halves
        // 16 query rows: exponents (with the references in use), P to shared memory, sums if `first`
        auto columns = [&](int c, bool first, uint64_t* l) {
          tmem_ld16(t_s + c, v);
          tmem_ld_wait();
          uint32_t h[8];
#pragma unroll
          for (int j = 0; j < 16; j += 4) {
            const float4 m = ld_shared_f4(sm_m + (c + j) * 4);
            float x[4];
            unpack2(fma2(pack2(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), scale2, pack2(m.x, m.y)), x[0], x[1]);
            unpack2(fma2(pack2(__uint_as_float(v[j + 2]), __uint_as_float(v[j + 3])), scale2, pack2(m.z, m.w)), x[2], x[3]);
            float q[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) q[k] = valid ? ex2_approx(x[k]) : 0.f;
            if (first) {
              l[j / 2] = add2(l[j / 2], pack2(q[0], q[1]));
              l[j / 2 + 1] = add2(l[j / 2 + 1], pack2(q[2], q[3]));
            }
            h[j / 2] = pack_bf16(q[0], q[1]);
            h[j / 2 + 1] = pack_bf16(q[2], q[3]);
            most = __vmaxu2(most, __vmaxu2(h[j / 2], h[j / 2 + 1]));
          }
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t piece = (uint32_t)(c / 8 + i) ^ (uint32_t)(key & 7);
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(pt_row + piece * 16u), "r"(h[4 * i]), "r"(h[4 * i + 1]), "r"(h[4 * i + 2]), "r"(h[4 * i + 3]) : "memory");
          }
        };
#pragma unroll
        for (int c = 0; c < N; c += 16) columns(c, true, l2 + c / 2);
        // does a score exceed its reference by too much?  (a NaN does)
        const bool large = __any_sync(0xffffffffu, max(most & 0xFFFFu, most >> 16) > kTooLarge);
        if (lane == 0) {
          if (large) too_large[w] = n_own + 1;
          mbar_arrive(bar_vote + 8 * w);
        }
        ok = wait(bar_vote + 8 * w, n_own & 1);
        if (!ok) break;
        if (too_large[w] == n_own + 1) {
          // ---- rare: the tile's maxima become the references, for the query rows where they are larger
          auto scores = [&](int c, float (&x)[8]) {
            uint32_t one[8];
            tmem_ld8(t_s + c, one);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(one[j]);
          };
          // (differences of two references are as good as the references; a score is only ever taken against one of them, in one rounding)
          auto minus_next = [&](int i) { return next_m[i] ? -from_ordered(next_m[i]) : minus_m[i]; };
          auto meet = [&]() {
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_slow + 8 * w);
            return wait(bar_slow + 8 * w, slow++ & 1);
          };
          float x[8];
#pragma unroll 1
          for (int c = 0; c < N; c += 8) {
            scores(c, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const bool above = valid && fmaf(x[j], p.scale_log2, minus_m[w * N + c + j]) > 0.f;
              const uint32_t top = __reduce_max_sync(0xffffffffu, above ? to_ordered(__fmul_ru(x[j], p.scale_log2)) : 0u);
              if (lane == 0 && top > 0) atomicMax(&next_m[w * N + c + j], top);
            }
          }
          ok = meet();
          if (!ok) break;
#pragma unroll
          for (int c = 0; c < N; c += 8) {
            scores(c, x);
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
              float l[2];
              unpack2(l2[(c + j) / 2], l[0], l[1]);
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const int i = w * N + c + j + k;
                const float next = minus_next(i);
                // (a sum with a term above 2^100 is that term, as far as fp32 holds it)
                l[k] = valid && fmaf(x[j + k], p.scale_log2, minus_m[i]) > 100.f ? ex2_approx(fmaf(x[j + k], p.scale_log2, next)) : l[k] * ex2_approx(next - minus_m[i]);
              }
              l2[(c + j) / 2] = pack2(l[0], l[1]);
            }
          }
          if (n_own > n_first) {                                   // the group's products so far are complete (pv_done above)
            tc_fence_after_sync();
            const uint32_t t_o = tmem + t_lane + G::kColO + w * 64;
#pragma unroll 1
            for (int c = 0; c < N; c += 16) {
              tmem_ld16(t_o + c, v);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 16; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * ex2_approx(minus_next(w * N + c + j) - minus_m[w * N + c + j]));
              tmem_st16(t_o + c, v);
            }
            tmem_st_wait();
          }
          ok = meet();
          if (!ok) break;
          if (key < N) {
            minus_m[w * N + key] = minus_next(w * N + key);
            next_m[w * N + key] = 0;
          }
          ok = meet();
          if (!ok) break;
#pragma unroll 1
          for (int c = 0; c < N; c += 16) columns(c, false, l2);
        }
        // ---- P is there, the scores are free
        fence_proxy_async_smem();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bar_s_empty + buf);
          mbar_arrive(bar_pt_full + 8 * w);
        }
      }
      if (!ok) break;
      // ---- the end of the segment: sums over the keys, then the two groups together
      const bool mine = n_own > n_first;
      if (mine) {
        ok = wait(bar_pv_done + 8 * w, (n_own - 1) & 1);
        if (!ok) break;
        tc_fence_after_sync();
      }
      {
        float l[N];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) unpack2(l2[i], l[2 * i], l[2 * i + 1]);
        reduce_columns<N>(l);
        float* const to = sums + (w * 4 + (warp & 3)) * N + column_of<N>(lane);
        to[0] = l[0];
      }
      // (fences on both sides: behind it a group reads the other's O^T, of whose products only that group has waited for; and the last one lets
      // the next segment's products overwrite what both have read)
      auto meet = [&](int i) {
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_fold + 8 * i);
        if (!wait(bar_fold + 8 * i, seg & 1)) return false;
        tc_fence_after_sync();
        return true;
      };
      ok = meet(0);
      if (!ok) break;
      const bool both = g.end - g.begin > 1;                       // the second group has a tile
      const size_t r0 = (((size_t)g.layer * p.batch + g.b) * p.n_q_heads + (size_t)g.kvh * p.group) * p.q_cap;
      if (tid < N) {                                               // thread = query row
        float l0 = 0.f, l1 = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          l0 += sums[i * N + tid];
          l1 += sums[(4 + i) * N + tid];
        }
        const float m0 = -minus_m[tid], m1 = both ? -minus_m[N + tid] : -CUDART_INF_F, m = fmaxf(m0, m1);
        const float w0 = ex2_approx(m0 - m), w1 = both ? ex2_approx(m1 - m) : 0.f, l = both ? fmaf(w0, l0, w1 * l1) : l0;
        const bool active = tid < p.rows && tid - p.by_q_cap.div(tid) * p.q_cap < g.Lq;
        const float inv = g.slot < 0 ? (active ? 1.f / l : 0.f) : 1.f;
        share[tid] = w0 * inv;
        share[N + tid] = w1 * inv;
        if (g.slot < 0) {
          if (tid < p.rows && p.lse) p.lse[r0 + tid] = active ? (m + lg2_approx(l)) * 0.6931471805599453f : -CUDART_INF_F;
        } else if (tid < p.rows) {
          __stcg(p.ws_ml + (size_t)g.slot * p.rows_pad + tid, make_float2(m, l));
        }
      }
      ok = meet(1);
      if (!ok) break;
      // each group half of the query rows; thread = value column
      const uint32_t t_o = tmem + t_lane + G::kColO;
      float* const part_o = reinterpret_cast<float*>(p.ws_o) + ((size_t)max(g.slot, 0) * p.rows_pad) * D + key;
#pragma unroll 1
      for (int c = w * (N / 2); c < (w + 1) * (N / 2) && c < p.rows; c += 8) {
        uint32_t x[8], y[8];
        tmem_ld8(t_o + c, x);
        if (both) tmem_ld8(t_o + 64 + c, y);
        tmem_ld_wait();
        if (D == 64 && key >= 64) continue;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int r = c + j;
          if (r >= p.rows) break;
          float o = share[r] * __uint_as_float(x[j]);
          if (both) o = fmaf(share[N + r], __uint_as_float(y[j]), o);
          if (g.slot < 0) {
            const bool active = r - p.by_q_cap.div(r) * p.q_cap < g.Lq;
            p.out[(r0 + r) * D + key] = __float2bfloat16_rn(active ? o : 0.f);
          } else {
            __stcg(part_o + (size_t)r * D, o);
          }
        }
      }
      ok = meet(2);                                                // O^T, the references and sums have been read
      ++seg;
    }
  }
  // ---- teardown: nothing of this block is in flight any more
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  if (tid == 0 && (*abort_ptr || *never_ptr)) dlm_set_status(p.status, DLM_ERR_TIMEOUT);
  if (warp == 25) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, kTmemCols);
    __syncwarp();
  }
}

}  // namespace few

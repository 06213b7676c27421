// The online softmax of the attention kernels: scores in TMEM to P in TMEM, 64 keys of a query row per thread at a time.
#pragma once

#include <cuda_bf16.h>
#include <math_constants.h>
#include <stdint.h>

#include "sm100_ptx.cuh"

namespace {

using namespace sm100;

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Softmax of one half-step for the query row held by this thread (S row in TMEM -> P row in TMEM).
// O is rescaled only when the scores have outgrown the maximum in use by a lot: until then P is
// formed against the older, smaller maximum and may exceed 1 by a few powers of two, which bf16
// and the fp32 accumulators hold just as well; the final division by the row sum, taken against
// the same maximum, cancels it.  Ragged half-steps compare maxima (kRescaleThreshold, log2 units);
// full ones look at the row sum (kSumLimit).
// (real = false: nobody reads the thread's row, which may hold anything; it does not take the warp through a rescaling.)
// kFloor: for scores of any size.  A half-step of nothing but -infinity leaves the lowest number as the maximum and 0 as the sum (else both are NaN
// from there on), and the maximum is rounded up, so that scores below -2^30, which are further than 1 apart, give no 2^(s - m) above 1.
constexpr float kLowestMaximum = -3.402823466e38f;
template <bool kFloor>
__device__ __forceinline__ float scaled_maximum(float mx, float scale_log2) {
  return kFloor ? fmaxf(__fmul_ru(mx, scale_log2), kLowestMaximum) : mx * scale_log2;
}
constexpr float kRescaleThreshold = 8.0f;

// Rare path shared by both kinds of half-step: some row of the warp outgrew its maximum by more
// than the threshold, so the warp's O rows in TMEM are rescaled (rows that did not grow keep
// factor 1).  The P V product of the previous half-step may still be running: wait for it first.
template <int D>
__device__ __noinline__ bool rescale_o(uint32_t t_o, bool grow, float m_new, float& m_used, float& l_run,
                                       uint32_t bar_pv_done, uint32_t parity, volatile int* abort_ptr) {
  const bool ok = __all_sync(0xffffffffu, mbar_wait(bar_pv_done, parity, abort_ptr)) != 0;
  if (!ok) return false;
  tc_fence_after_sync();
  const float alpha = grow ? ex2_approx(m_used - m_new) : 1.0f;
  uint32_t v[32];
#pragma unroll 1
  for (int c = 0; c < D / 32; ++c) {
    tmem_ld32(t_o + c * 32, v);
    tmem_ld_wait();
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * alpha);
    tmem_st32(t_o + c * 32, v);
  }
  tmem_st_wait();
  l_run *= alpha;
  if (grow) m_used = m_new;
  return true;
}

// Full half-step (64 valid keys): the score row sits in registers, so TMEM is read once and with a
// single wait.  Only the first half-step of a segment takes the row maximum before the
// exponentials; later ones form P against the maximum in use and look at the row sum afterwards:
// a sum above kSumLimit means some score outgrew that maximum by a lot, and only then (rare)
// is the maximum taken, O rescaled and P formed again.  The maximum pass, half-rate ALU work
// that both softmax groups of an SMSP would do at the same time, is gone from the steady state.
constexpr float kSumLimit = 1024.0f;   // 64 keys: some P is then above 16, and none was above 1024 before

template <int D>
__device__ __forceinline__ float row_max64(const uint32_t (&s)[64]) {
  float mx[8];   // independent chains: the maximum is latency-bound otherwise
#pragma unroll
  for (int c = 0; c < 8; ++c) mx[c] = __uint_as_float(s[c]);
#pragma unroll
  for (int j = 8; j < 64; j += 8) {
#pragma unroll
    for (int c = 0; c < 8; ++c) mx[c] = fmaxf(mx[c], __uint_as_float(s[j + c]));
  }
  return fmaxf(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), fmaxf(fmaxf(mx[4], mx[5]), fmaxf(mx[6], mx[7])));
}

// P = 2^(s * scale - m) for 32 scores, packed to bf16 pairs and written to 16 TMEM columns at t_p;
// adds to the two partial row sums, unrounded.  (P in bf16 is what the product with V takes beside bf16 values: off by at most
// 2^-8 of itself, an output by at most 2^-8 sum p |v|, about what rounding the output costs.)  (Variants measured in the kernel and found no faster at the
// configs' shapes: all 32 exponentials issued before the sums, and packing by integer add and byte
// permute instead of the conversion instruction, which shares the SFU's pipe.)
__device__ __forceinline__ void exp32_store(const uint32_t* s, float scale_log2, float m_used, uint32_t t_p, float& l0,
                                            float& l1) {
  uint32_t pk[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const float p0 = ex2_approx(fmaf(__uint_as_float(s[2 * j]), scale_log2, -m_used));
    const float p1 = ex2_approx(fmaf(__uint_as_float(s[2 * j + 1]), scale_log2, -m_used));
    l0 += p0;
    l1 += p1;
    pk[j] = pack_bf16(p0, p1);
  }
  tmem_st16(t_p, pk);
}

// The same for 64 scores (32 TMEM columns at t_p); returns the row sum.
__device__ __forceinline__ float exp64_store(const uint32_t (&s)[64], float scale_log2, float m_used, uint32_t t_p) {
  float l0 = 0.f, l1 = 0.f;
  exp32_store(s, scale_log2, m_used, t_p, l0, l1);
  exp32_store(s + 32, scale_log2, m_used, t_p + 16, l0, l1);
  return l0 + l1;
}

template <int D, bool kFloor = false>
__device__ __forceinline__ bool softmax_half_full(uint32_t t_s, uint32_t t_o, bool first, float scale_log2,
                                                  float& m_used, float& l_run, uint32_t bar_pv_done,
                                                  uint32_t pv_parity, volatile int* abort_ptr, bool real = true) {
  uint32_t s[64];
  tmem_ld32(t_s, s);
  tmem_ld32(t_s + 32, s + 32);
  tmem_ld_wait();
  if (first) {
    m_used = scaled_maximum<kFloor>(row_max64<D>(s), scale_log2);
    l_run = 0.f;
  }
  float l_half = exp64_store(s, scale_log2, m_used, t_s);
  if (!first) {
    const bool grow = real && !(l_half <= kSumLimit);   // also catches a NaN sum
    if (__any_sync(0xffffffffu, grow)) {
      const float m_new = scaled_maximum<kFloor>(row_max64<D>(s), scale_log2);
      tmem_st_wait();   // the P just written is replaced below
      if (!rescale_o<D>(t_o, grow, m_new, m_used, l_run, bar_pv_done, pv_parity, abort_ptr)) return false;
      l_half = exp64_store(s, scale_log2, m_used, t_s);
    }
  }
  l_run += l_half;
  tmem_st_wait();
  return true;
}

// Ragged half-step (fewer than 64 valid keys: the end of the cache rows, or the fresh rows): 32
// columns at a time, keys at or beyond `valid` masked out.
template <int D, bool kFloor = false>
__device__ __noinline__ bool softmax_half_ragged(uint32_t t_s, uint32_t t_o, int valid, bool first, float scale_log2,
                                                 float& m_used, float& l_run, uint32_t bar_pv_done,
                                                 uint32_t pv_parity, volatile int* abort_ptr, bool real = true) {
  const int n_chunks = (valid + 31) >> 5;
  uint32_t v[32];
  float mx = -CUDART_INF_F;
  for (int c = 0; c < n_chunks; ++c) {
    tmem_ld32(t_s + c * 32, v);
    tmem_ld_wait();
#pragma unroll
    for (int j = 0; j < 32; ++j)
      if (c * 32 + j < valid) mx = fmaxf(mx, __uint_as_float(v[j]));
  }
  const float m_new = scaled_maximum<kFloor>(mx, scale_log2);
  if (first) {
    m_used = m_new;
    l_run = 0.f;
  } else {
    const bool grow = real && m_new > m_used + kRescaleThreshold;
    if (__any_sync(0xffffffffu, grow)) {
      if (!rescale_o<D>(t_o, grow, m_new, m_used, l_run, bar_pv_done, pv_parity, abort_ptr)) return false;
    }
  }
  float l_add = 0.f;
  for (int c = 0; c < n_chunks; ++c) {
    tmem_ld32(t_s + c * 32, v);
    tmem_ld_wait();
    uint32_t pk[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      float p0 = ex2_approx(fmaf(__uint_as_float(v[2 * j]), scale_log2, -m_used));
      float p1 = ex2_approx(fmaf(__uint_as_float(v[2 * j + 1]), scale_log2, -m_used));
      if (c * 32 + 2 * j >= valid) p0 = 0.f;
      if (c * 32 + 2 * j + 1 >= valid) p1 = 0.f;
      l_add += p0 + p1;
      pk[j] = pack_bf16(p0, p1);
    }
    tmem_st16(t_s + c * 16, pk);
  }
  l_run += l_add;
  tmem_st_wait();
  return true;
}

}  // namespace

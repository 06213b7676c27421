// How the work of a call on a cache is dealt to the blocks of a persistent grid.  A unit is (layer of the call, KV head, row chunk, batch element),
// numbered in this order, and takes a number of steps that its batch element's lengths decide, which are known on the device only.
// Every (unit, step) pair is one item of a global list; block c of n takes a contiguous share of it.
#pragma once

#include "common.cuh"

namespace {

struct Lengths {   // in shared memory, by batch element
  int* prefix;     // [batch + 1] steps of the elements before
  int* lc;         // [batch] cached rows; NULL: not kept (no room), whoever needs them reads them again
  int* lq;         // [batch] active rows
  __device__ __forceinline__ Lengths(int* at, int batch, bool all = true)
      : prefix(at), lc(all ? at + batch + 1 : nullptr), lq(all ? at + 2 * batch + 1 : nullptr) {}
};
inline int length_ints(int batch, bool all = true) { return all ? 3 * batch + 1 : batch + 1; }

__device__ __forceinline__ int clamped_length(const int32_t* len, int b, int most) { return len ? max(0, min(__ldcg(len + b), most)) : most; }

// One warp: lengths (clamped, and recorded where out of range, unless `status` is NULL) and the prefix of steps_of(cached rows, active rows).
template <typename Steps>
__device__ __forceinline__ void read_lengths(const int32_t* cache_len, const int32_t* q_len, int batch, int capacity, int q_cap, int* status,
                                             const Lengths& s, volatile int* any_empty, Steps steps_of) {
  const int lane = threadIdx.x & 31;
  int acc = 0;
  for (int b0 = 0; b0 < batch; b0 += 32) {
    const int b = b0 + lane;
    int steps = 0;
    if (b < batch) {
      int Lc = __ldcg(cache_len + b), Lq = q_len ? __ldcg(q_len + b) : q_cap;
      if (Lc < 0 || Lc > capacity || Lq < 0 || Lq > q_cap) {
        if (status) dlm_set_status(status, DLM_ERR_CAPACITY);
        Lc = max(0, min(Lc, capacity));
        Lq = max(0, min(Lq, q_cap));
      }
      steps = steps_of(Lc, Lq);
      if (s.lc) {
        s.lc[b] = Lc;
        s.lq[b] = Lq;
      }
    }
    int inc = steps;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += v;
    }
    if (b < batch) s.prefix[b] = acc + inc - steps;
    if (any_empty && b < batch && steps == 0) *any_empty = 1;
    acc += __shfl_sync(0xffffffffu, inc, 31);
  }
  if (lane == 0) s.prefix[batch] = acc;
}

// Block c of n has items [lo(c), lo(c + 1)).
struct Deal {
  int sum, total, n, share, rem;   // steps of a (layer, KV head, row chunk) over the batch; items (the host keeps them below 2^30)
  __device__ __forceinline__ Deal(int sum_, int groups, int grid, int min_share) {
    sum = sum_;
    total = sum * groups;
    n = max(1, min(grid, total / min_share));
    share = total / n;
    rem = total - share * n;
  }
  __device__ __forceinline__ int lo(int c) const { return share * c + (rem * c) / n; }
  // the block that has an item
  __device__ __forceinline__ int owner(int item) const {
    int c = min(n - 1, (int)(__fdividef((float)item, (float)max(total, 1)) * (float)n));   // to within a block or two
    while (lo(c) > item) --c;
    while (lo(c + 1) <= item) ++c;
    return c;
  }
  // the (layer, KV head, row chunk) of an item, numbered, and its item within: the divisor is made of lengths, so not known on the host:
  // a float estimate, exact division where it is off
  __device__ __forceinline__ int group_of(int item, int& rest) const {
    int grp = (int)__fdividef((float)item, (float)sum);
    rest = item - grp * sum;
    if (rest < 0 || rest >= sum) {
      grp = item / sum;
      rest = item - grp * sum;
    }
    return grp;
  }
};

// The batch element that has step `rest` of a group: the last one whose prefix is not above it.
__device__ __forceinline__ int element_of(const Lengths& s, int batch, int rest) {
  int lo = 0, hi = batch - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s.prefix[mid] <= rest) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// bf16 tensor viewed as [slabs][rows][D]; box = 64 elements x box_rows rows x 1 slab, 128-byte swizzle.
inline int encode_rows_map(dlm_ctx* ctx, CUtensorMap* map, const void* base, int D, long long rows, long long slabs, int box_rows) {
  const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)rows, (cuuint64_t)slabs};
  const cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)rows * D * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
  return dlm_tensor_map(ctx, map, base, 3, dims, strides, box) ? DLM_OK : DLM_ERR_CUDA;
}

}  // namespace

// Tiles of a 4-bit cache in shared memory: as they are copied in, and decoded to the bf16 operand tiles of the tensor cores.
#pragma once

#include "q4.cuh"
#include "sm100_ptx.cuh"

namespace q4 {

// kRows consecutive rows of K or of V as copied: [kRows][D / 2] bytes of values, [kRows][D / 32] scale bytes.
template <int D, int kRows>
struct Packed {
  static constexpr int kRowBytes = D / 2, kRowScales = D / kGroup;
  static constexpr int kData = kRows * kRowBytes, kBytes = kData + kRows * kRowScales;
  // bytes that a copy of `rows` rows brings: whole 16-byte pieces of scales (rows up to the next multiple of 8, which the capacity is)
  __device__ static __forceinline__ uint32_t scale_bytes(int rows) { return (uint32_t)((rows * kRowScales + 15) & ~15); }
  __device__ static __forceinline__ uint32_t bytes(int rows) { return (uint32_t)(rows * kRowBytes) + scale_bytes(rows); }
  // One of the two copies that this takes, by one lane: a lane needs 200 - 300 cycles to issue a copy, so they are issued side by side.
  __device__ static __forceinline__ void copy_part(uint32_t dst, const uint8_t* data, const uint8_t* scale, bool scales, size_t row, int rows, uint32_t bar) {
    sm100::bulk_load(dst + (scales ? kData : 0), (scales ? scale : data) + row * (scales ? kRowScales : kRowBytes),
                     scales ? scale_bytes(rows) : (uint32_t)(rows * kRowBytes), bar);
  }
};

// Decodes a packed tile of kRows rows into an operand tile -- rows of 128 bytes (64 values) with 128-byte swizzle, a panel of 64 columns
// `panel_bytes` after the other -- with a team of kTeam threads, a group of 32 values at a time.  Task i is group i % (D / 32) of row
// i / (D / 32), so that a warp reads consecutive 16-byte pieces and consecutive bytes.  Eight lanes have two rows of four groups (D = 128) or four
// rows of two: with the two panels' 16-byte pieces taken in another order they store to eight different pieces of 128 bytes.
// A thread's tasks are a multiple of 8 rows apart, so all it needs to know of them is made once (Decoder) and a task takes about 62 instructions.
template <int D, int kRows, int kTeam>
struct Decoder {
  static constexpr int kGroups = D / kGroup, kTasks = kRows * kGroups / kTeam;
  static constexpr int kRowStep = kTeam / kGroups;          // rows between a thread's tasks
  static_assert(kRowStep % 8 == 0 && kTeam % kGroups == 0 && (kRows * kGroups) % kTeam == 0, "tasks");
  int row0, from16, from1;
  uint32_t to[4];         // of the four pieces of a group, in the order of the words below
  bool other;
  __device__ __forceinline__ Decoder(int me, uint32_t panel_bytes) {
    row0 = me / kGroups;
    const int grp = me % kGroups;
    from16 = me * 16;
    from1 = Packed<D, kRows>::kData + me;
    other = D == 128 && (grp & 2);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      to[j] = (uint32_t)(grp >> 1) * panel_bytes + (uint32_t)row0 * 128u + (((uint32_t)((grp & 1) * 4 + (other ? j ^ 2 : j)) ^ (uint32_t)(row0 & 7)) << 4);
  }
  // rows of the tile from `rows` on are left as they are
  __device__ __forceinline__ void run(uint32_t packed, uint32_t tile, int rows) const {
    constexpr int kBatch = kTasks < 2 ? kTasks : 2;
    // (a short loop: unrolled, it and the code of the other roles drive each other out of the instruction caches)
#pragma unroll 1
    for (int t = 0; t < kTasks; t += kBatch) {
      uint32_t w[kBatch][4], b[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const uint32_t at = packed + (uint32_t)(t + i) * kTeam * 16u;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[i][0]), "=r"(w[i][1]), "=r"(w[i][2]), "=r"(w[i][3]) : "r"(at + from16) : "memory");
        asm volatile("ld.shared.u8 %0, [%1];" : "=r"(b[i]) : "r"(packed + (uint32_t)(t + i) * kTeam + from1) : "memory");
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        if (row0 + (t + i) * kRowStep >= rows) continue;
        const Scale sc = make_scale(b[i]);
        const uint32_t base = tile + (uint32_t)((t + i) * kRowStep) * 128u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t v[4];
          decode8(D == 128 && other ? w[i][j ^ 2] : w[i][j], sc, v);
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(base + to[j]), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
        }
      }
    }
  }
};

// Clears 16-byte piece i of row i / (D / 8) of an operand tile.
template <int D>
__device__ __forceinline__ void clear_piece(uint32_t tile, uint32_t panel_bytes, int i) {
  const int row = i / (D / 8), c = i % (D / 8);
  const uint32_t a = tile + (uint32_t)(c >> 3) * panel_bytes + (uint32_t)row * 128u + (uint32_t)(c & 7) * 16u;
  asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(a), "r"(0u) : "memory");
}

}  // namespace q4

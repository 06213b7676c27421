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

// One group of 32 values and its scale, taken from a packed tile: task i is group i % (D / 32) of row i / (D / 32), so that a warp reads
// consecutive 16-byte pieces and consecutive bytes.
struct Group32 {
  uint32_t w[4];
  uint32_t scale;
};
template <int D, int kRows>
__device__ __forceinline__ Group32 read_group(uint32_t packed, int i) {
  Group32 g;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(g.w[0]), "=r"(g.w[1]), "=r"(g.w[2]), "=r"(g.w[3]) : "r"(packed + i * 16) : "memory");
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(g.scale) : "r"(packed + Packed<D, kRows>::kData + i) : "memory");
  return g;
}

// Decodes it into an operand tile: rows of 128 bytes (64 values) with 128-byte swizzle, a panel of 64 columns `panel_bytes` after the other.
// Eight lanes have two rows of four groups (D = 128) or four rows of two: with the two panels' 16-byte pieces taken in another order
// they store to eight different pieces of 128 bytes.
template <int D>
__device__ __forceinline__ void write_group(uint32_t tile, uint32_t panel_bytes, int i, const Group32& g) {
  constexpr int kGroups = D / kGroup;
  const int row = i / kGroups, grp = i % kGroups;
  const uint32_t base = tile + (uint32_t)(grp >> 1) * panel_bytes + (uint32_t)row * 128u;
  const Scale sc = make_scale(g.scale);
  const int other = D == 128 ? (grp & 2) : 0;
  const uint32_t w[4] = {other ? g.w[2] : g.w[0], other ? g.w[3] : g.w[1], other ? g.w[0] : g.w[2], other ? g.w[1] : g.w[3]};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t v[4];
    decode8(w[j], sc, v);
    const uint32_t piece = (uint32_t)((grp & 1) * 4 + (j ^ other)) ^ (uint32_t)(row & 7);
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(base + piece * 16u), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
  }
}

// Clears 16-byte piece i of row i / (D / 8) of an operand tile.
template <int D>
__device__ __forceinline__ void clear_piece(uint32_t tile, uint32_t panel_bytes, int i) {
  const int row = i / (D / 8), c = i % (D / 8);
  const uint32_t a = tile + (uint32_t)(c >> 3) * panel_bytes + (uint32_t)row * 128u + (uint32_t)(c & 7) * 16u;
  asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(a), "r"(0u) : "memory");
}

}  // namespace q4

// What the attention kernels share: the layout of K and V tiles in LDS, exchanges between lane groups, row sums.
#pragma once
#include "dev_common.hpp"

namespace httm {

// V tile in LDS: 64 rows of 128 bytes, written by global->LDS loads like the K tile; the 16-byte
// chunk c of row r sits at chunk position c ^ (2 * ((r >> 1) & 3)), so that the eight rows which half a
// transposing read touches (32 bytes each, same channels) fall into eight different 32-byte bank groups.
__device__ __forceinline__ int v_swizzle(int row) { return ((row >> 1) & 3) << 1; }

// K tile in LDS: 64 rows of 128 bytes, unpadded (it is written by global->LDS loads, 1 KB per
// wave instruction); the 16-byte chunk c of row r sits at chunk position c ^ ((r >> 1) & 7), which
// makes the operand reads of 16 consecutive rows hit 16 distinct bank groups.
__device__ __forceinline__ int k_swizzle(int row) { return (row >> 1) & 7; }

typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x16 __attribute__((ext_vector_type(16)));
// One half of a pair of query tiles' P^T: the B operand of a 16x16x32 MFMA
__device__ __forceinline__ bf16x8 p_half(const u32x8& p, int j) {
  return __builtin_bit_cast(bf16x8, j ? __builtin_shufflevector(p, p, 4, 5, 6, 7) : __builtin_shufflevector(p, p, 0, 1, 2, 3));
}

// A constant in a register of its own, here and now: the compiler moves constants that an instruction cannot hold
// in front of the loop over a share's segments, where they take registers through the whole tile.
__device__ __forceinline__ uint32_t local(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Row sums on the matrix cores.  A sum does not need the zeros of a structured-sparse A
// operand: v_smfmac_f32_16x16x64_bf16 takes 64 dense k per instruction in the time the dense
// 16x16x32 takes 32 (18 against 16 cycles in a register-only loop), and the two k of every four that a row
// of A drops are taken by another row.  Its B operand are the eight P^T registers of two query tiles
// (query l%16 of both): the first tile's values are the k below 32 and the second one's the others,
// which are multiplied by lanes 0..31 and lanes 32..63 of A.  So rows 0 and 4 of A hold ones in lanes below
// 32 and rows 8 and 12 in the others; rows 0 and 8 keep the k 0, 1 of every four (index 0x4), rows 4 and 12
// the k 2, 3 (0xE).  D[0][n] + D[4][n] is the sum of query n of the first tile, D[8][n] + D[12][n] that of
// the second: register 0 of the four lane groups (row_sums()), so that one comparison per pair looks at
// every row.  A step's 32 products take 512 matrix-core cycles; its
// row sums take 36 instead of the 64 of four dense 16x16x32.  Stage 3 is bound by those cycles and the
// power they draw: 16 heads x 16384 x 16384 878 -> 860 us.
__device__ __forceinline__ bf16x8 row_sum_operand(int lane) {
  const int m = lane & 15;
  const uint32_t w = (m & 3) == 0 && (m >> 3) == (lane >> 5) ? local(0x3F803F80u) : 0u;
  return __builtin_bit_cast(bf16x8, u32x4{w, w, w, w});
}
__device__ __forceinline__ int row_sum_index(int lane) { return (int)((lane & 4) ? local(0xEEEEEEEEu) : local(0x44444444u)); }
// Exchange between neighbouring lane groups of 16 (halves of the wave): both lanes of a pair receive {x of the lower
// one, x of the upper one}.
struct LanePair {
  float a, b;
};
__device__ __forceinline__ LanePair swap16(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t lo = r[0], hi = r[1];
  return {__uint_as_float(lo), __uint_as_float(hi)};
}
__device__ __forceinline__ LanePair swap32(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const uint32_t lo = r[0], hi = r[1];
  return {__uint_as_float(lo), __uint_as_float(hi)};
}
// The sums of query column l16 of a pair's two query tiles from its register 0, in all lanes.
__device__ __forceinline__ LanePair row_sums(float l0) {
  const LanePair h = swap16(l0);
  return swap32(h.a + h.b);
}

__device__ __forceinline__ f32x4 mfma16(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

typedef short s16x4 __attribute__((ext_vector_type(4)));

}  // namespace httm

// 4-bit expert matrices: the layout shared by the kernels that write and read it.
//
// Codes: per matrix, row tiles of 16 rows; per row tile, blocks of 64 inputs of 512 bytes: lane
// (g, q) = (lane / 4, lane % 4) of a warp has 16 bytes, four words:
//   word 2h + s   row g + 8s, inputs 32h + 8q .. + 7 of the block
// so a warp's 16-byte loads are whole lines, and a word is a lane's share of the A operand of
// two 16 x 8 x 16 MMAs (with the inputs of each 32 taken in an order of their own, the same for
// both operands: x is then read 16 bytes at a time). In a word, input 2i is the nibble at bit 4i
// and input 2i + 1 the one at bit 16 + 4i: a shift and a mask leave a pair of them in the low
// bits of two 16-bit halves. A nibble is the code + 8.
// Scales: per matrix and row tile, per g, the groups' scale pairs (row g, row g + 8) of bf16,
// the groups padded to a multiple of four with zeros.
// Rows behind n_out have scales of zero, inputs behind n_in codes of zero.
#pragma once

#include "dmoe_internal.cuh"

namespace dmoe {

struct Q4Shape {
  int N, K, group;
  int row_tiles, k_tiles, groups, groups_pad;
  __host__ __device__ size_t code_bytes() const { return (size_t)row_tiles * k_tiles * 512; }
  __host__ __device__ size_t scale_bytes() const { return (size_t)row_tiles * 8 * groups_pad * 4; }
};

inline Q4Shape q4_shape(const dmoe_q4_desc& d) {
  Q4Shape s;
  s.N = d.n_out;
  s.K = d.n_in;
  s.group = d.group;
  s.row_tiles = (d.n_out + 15) / 16;
  s.k_tiles = (d.n_in + 63) / 64;
  s.groups = d.n_in / d.group;
  s.groups_pad = (s.groups + 3) / 4 * 4;
  return s;
}

// Pair i of a word's inputs (2i, 2i + 1) as bf16 codes: 128 + nibble is exact in bf16's eight
// bits, and so is the difference from 136.
__device__ __forceinline__ __nv_bfloat162 q4_pair(uint32_t word, int i) {
  const uint32_t u = ((word >> (4 * i)) & 0x000F000Fu) | 0x43004300u;
  return __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&u), __float2bfloat162_rn(136.f));
}

// The same times the scale (five significant bits times three: exact).
__device__ __forceinline__ uint32_t q4_value_pair(uint32_t word, int i, __nv_bfloat162 scale) {
  const __nv_bfloat162 v = __hmul2(q4_pair(word, i), scale);
  return *reinterpret_cast<const uint32_t*>(&v);
}

}  // namespace dmoe

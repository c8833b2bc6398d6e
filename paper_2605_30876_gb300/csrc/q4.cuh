// 4-bit expert matrices: the layout shared by the kernels that write and read it.
//
// Codes: per matrix, row tiles of 16 rows; per row tile, blocks of 64 inputs of 512 bytes: lane
// (g, q) = (lane / 4, lane % 4) of a warp has 16 bytes, four words:
//   word 2h + s   row g + 8s, inputs 32h + 8q .. + 7 of the block
// so a warp's 16-byte loads are whole lines, and a word is a lane's share of the A operand of
// two 16 x 8 x 16 MMAs (with the inputs of each 32 taken in an order of their own, the same for
// both operands: x is then read 16 bytes at a time). In a word, input 2i is the nibble at bit 4i + 3
// and input 2i + 1 the one at bit 4i + 19, counted around the word's end: a rotation and a mask
// leave a pair of them in the upper mantissa bits of two bf16 halves. A nibble is the code + 8.
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

__device__ __forceinline__ uint32_t q4_pack_word(const int (&code)[8]) {
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w |= (uint32_t)(code[2 * i] + 8) << (4 * i) | (uint32_t)(code[2 * i + 1] + 8) << (16 + 4 * i);
  return __funnelshift_l(w, w, 3);
}

// A row's scale as the two operands of the values' FMA: s and -24 s, in both halves.
struct Q4Scale {
  __nv_bfloat162 s, b;
};
__device__ __forceinline__ Q4Scale q4_scale_pair(uint32_t bits) {
  Q4Scale r;
  const uint32_t two = __byte_perm(bits, bits, 0x1010);
  r.s = *reinterpret_cast<const __nv_bfloat162*>(&two);
  r.b = __hmul2(r.s, __float2bfloat162_rn(-24.f));
  return r;
}

// Pair i of a word's inputs, 2i and 2i + 1, as bf16 values. The nibble in the upper four mantissa
// bits of 16 makes 16 + nibble; times s, less 24 s, it is s (nibble - 8). Every step is exact: 24 s
// has 5 + 2 significant bits, the value 5 + 3, and bf16 holds eight; the FMA rounds once. With the
// nibble in the lower bits (128 + nibble) the offset would be 136 s, 5 + 5 bits, and a
// subtraction of its own were needed.
__device__ __forceinline__ uint32_t q4_value_pair(uint32_t word, int i, const Q4Scale& s) {
  const uint32_t r = i == 0 ? word : i == 3 ? __funnelshift_r(word, word, 12) : word >> (4 * i);
  const uint32_t u = (r & 0x00780078u) | 0x41804180u;
  const __nv_bfloat162 v = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&u), s.s, s.b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

}  // namespace dmoe

// 4-bit expert matrices: the layout shared by the kernels that write and read it.
//
// Codes: per matrix, tiles of 128 rows (the last one of as many as are left, in sixteens); per tile,
// blocks of 64 inputs: first every row's inputs 0 .. 31 of the block, 16 bytes a row, then every
// row's 32 .. 63. A warp whose lanes have 32 neighbouring rows reads whole lines, and a lane
// has a row's inputs: what a lane of tensor memory takes. Word w of the 16 bytes has inputs 8w ..
// 8w + 7. In a word, input 2i is the nibble at bit 4i + 3 and input 2i + 1 the one at bit 4i + 19,
// counted around the word's end: a rotation and a mask leave a pair of them in the upper mantissa
// bits of two bf16 halves. A nibble is the code + 8.
// Scales: bf16, per row its groups, padded with zeros to a multiple of eight (16 bytes).
// Rows behind n_out have scales of zero, inputs behind n_in codes of zero.
#pragma once

#include "dmoe_internal.cuh"

namespace dmoe {

struct Q4Shape {
  int N, K, group;
  int rows, k_tiles, groups, groups_pad;   // rows: n_out in whole sixteens
  __host__ __device__ size_t code_bytes() const { return (size_t)rows * k_tiles * 32; }
  __host__ __device__ size_t scale_bytes() const { return (size_t)rows * groups_pad * 2; }
  // rows of the 128-row tile that has row n
  __host__ __device__ int tile_rows(int n) const {
    const int left = rows - n / 128 * 128;
    return left < 128 ? left : 128;
  }
  // byte offset of row n's 16 bytes of block kt, half h, in its matrix
  __host__ __device__ size_t code_at(int n, int kt, int h) const {
    const int tile = n / 128 * 128;
    return (size_t)tile * k_tiles * 32 + ((size_t)kt * 2 + h) * tile_rows(n) * 16 + (n - tile) * 16;
  }
};

inline Q4Shape q4_shape(const dmoe_q4_desc& d) {
  Q4Shape s;
  s.N = d.n_out;
  s.K = d.n_in;
  s.group = d.group;
  s.rows = (d.n_out + 15) / 16 * 16;
  s.k_tiles = (d.n_in + 63) / 64;
  s.groups = d.n_in / d.group;
  s.groups_pad = (s.groups + 7) / 8 * 8;
  return s;
}

__device__ __forceinline__ uint32_t q4_pack_word(const int (&code)[8]) {
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w |= (uint32_t)(code[2 * i] + 8) << (4 * i) | (uint32_t)(code[2 * i + 1] + 8) << (16 + 4 * i);
  return __funnelshift_l(w, w, 3);
}

// A scale as the two operands of the values' FMA: s and -24 s, in both halves.
struct Q4Scale {
  __nv_bfloat162 s, b;
};
__device__ __forceinline__ Q4Scale q4_scale_pair(uint32_t bits) {   // (the lower half's)
  Q4Scale r;
  const uint32_t two = __byte_perm(bits, 0u, 0x1010);
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

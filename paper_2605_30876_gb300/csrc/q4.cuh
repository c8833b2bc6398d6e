// 4-bit expert matrices: the layout shared by the kernels that write and read it.
//
// A matrix is cut into tiles of 32 rows, a tile into blocks of 128 inputs: 2048 bytes of codes, for a
// warp whose lanes have the rows. In them every row's inputs 0 .. 31 come first, 16 bytes a row, then
// every row's 32 .. 63, and so on. Word w of the 16 bytes has inputs 8w .. 8w + 7: input 2i of them is
// the nibble at bit 4i + 3 and input 2i + 1 the one at bit 4i + 19, counted around the word's end:
// a rotation and a mask leave a pair of them in the upper mantissa bits of two bf16 halves. A nibble
// is the code + 8.
// Scales: bf16, per tile and block every row's groups of the block (4, 2 or 1).
// Rows behind n_out and inputs behind n_in have codes and scales of zero.
#pragma once

#include "dmoe_internal.cuh"

namespace dmoe {

constexpr int kMaxQ4Experts = 512;   // (256 routed experts and a shared one are one set)
constexpr int kQ4Rows = 32, kQ4Inputs = 128, kQ4CodeBytes = kQ4Rows * kQ4Inputs / 2;

struct Q4Shape {
  int N, K, group;
  int tiles, blocks;   // of a matrix, and of a tile
  int groups;          // of a row in a block
  __host__ __device__ size_t code_bytes() const { return (size_t)tiles * blocks * kQ4CodeBytes; }
  __host__ __device__ int scale_block() const { return kQ4Rows * groups * 2; }   // bytes
  __host__ __device__ size_t scale_bytes() const { return (size_t)tiles * blocks * scale_block(); }
};

inline Q4Shape q4_shape(const dmoe_q4_desc& d) {
  Q4Shape s;
  s.N = d.n_out;
  s.K = d.n_in;
  s.group = d.group;
  s.tiles = (d.n_out + kQ4Rows - 1) / kQ4Rows;
  s.blocks = (d.n_in + kQ4Inputs - 1) / kQ4Inputs;
  s.groups = kQ4Inputs / d.group;
  return s;
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
// The mask and the exponent bits of a pair are held in registers by the caller (an instruction takes one
// immediate: given both, the compiler makes two of the AND and the OR).
struct Q4Bits {
  uint32_t mask, sixteen;
  __device__ __forceinline__ Q4Bits() {
    asm volatile("mov.u32 %0, 0x00780078;" : "=r"(mask));
    asm volatile("mov.u32 %0, 0x41804180;" : "=r"(sixteen));
  }
};
__device__ __forceinline__ uint32_t q4_value_pair(uint32_t word, int i, const Q4Scale& s,
                                                  const Q4Bits& bits) {
  const uint32_t r = i == 0 ? word : i == 3 ? __funnelshift_r(word, word, 12) : word >> (4 * i);
  uint32_t u;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(u) : "r"(r), "r"(bits.mask), "r"(bits.sixteen));   // and, or
  const __nv_bfloat162 v = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&u), s.s, s.b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

}  // namespace dmoe

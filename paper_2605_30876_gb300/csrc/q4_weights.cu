// bf16 weights to 4-bit codes and group scales, and back. One warp takes 16 rows x 128 inputs
// (whole groups of every size): 4 KB of weights. 268 M weights (256 matrices of 512 x 2048, groups of
// 64): quantising 133 us, the values back 100 us (both 232 us, cold, with 200 us of bytes at 6.8 TB/s).
// Quantising is bound by its instructions (issue slots 84 % busy, DRAM about three quarters), the way
// back by the bytes (DRAM 79 %).
#include "q4.cuh"

namespace dmoe {
namespace {

constexpr int kQ4Threads = 256;

struct Q4Block {   // a warp's 16 x 128 weights
  int e, nt, kb;
  bool ok;
};
__device__ __forceinline__ Q4Block q4_block(const Q4Shape& s, int n_experts) {
  int64_t i = (int64_t)blockIdx.x * (kQ4Threads / 32) + (threadIdx.x >> 5);
  Q4Block b;
  b.kb = (int)(i % s.blocks);
  i /= s.blocks;
  b.nt = (int)(i % (2 * s.tiles));
  i /= 2 * s.tiles;
  b.e = (int)i;
  b.ok = i < n_experts;
  return b;
}

// a / 7 to five significant bits, for a bf16 a of 2^-100 and more. A quotient of eight significant bits
// by 7 is a tie of two such numbers or 2^-9 of itself and more away from one; the product with 1 / 7,
// off by less than 2^-22, is brought back to a tie by a first rounding to 17 bits.
__device__ __forceinline__ float q4_scale(float a) {
  uint32_t u = __float_as_uint(a * (1.f / 7.f));
  u = (u + 0x40u) & ~0x7Fu;
  u = (u + 0x3FFFFu + (u >> 19 & 1u)) & ~0x7FFFFu;
  return __uint_as_float(u);
}

// rint(w / s) + 8 in the lower four bits, from inv = 1 / s within 2^-21. The quotient of eight significant
// bits by five is a tie of two integers or 2^-9 and more away from one, and w * inv is off by less
// than 2^-20: the sum with 384, rounded to 2^-15, brings a tie back to it and passes no other one.
// The second sum rounds to an integer, ties to even. A zero inv gives 8, the code of zero. (With
// divisions for each weight and scale, 268 M weights and back took 335 us.)
__device__ __forceinline__ uint32_t q4_nibble(float w, float inv) {
  return __float_as_uint(__fadd_rn(__fmaf_rn(w, inv, 384.f), 12582912.f + 8.f - 384.f));
}

__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) { return __vmaxu2(a, b); }

__global__ void __launch_bounds__(kQ4Threads)
q4_quantize_kernel(Q4Shape s, int n_experts, const uint4* __restrict__ w, uint8_t* __restrict__ codes,
                   uint16_t* __restrict__ scales) {
  pdl_wait();
  pdl_launch_dependents();
  const Q4Block b = q4_block(s, n_experts);
  if (!b.ok) return;
  const int lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  uint4 v[2][4];       // rows g and g + 8; 32 inputs each
  uint32_t top[2][4];  // the largest magnitude, as the bits of a bf16
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int n = b.nt * 16 + g + 8 * r, k = b.kb * 128 + c * 32 + q * 8;
      v[r][c] = n < s.N && k < s.K
                    ? __ldcs(w + (((size_t)b.e * s.N + n) * s.K + k) / 8) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint32_t m = 0x7FFF7FFFu;
      uint32_t t = max2(max2(v[r][c].x & m, v[r][c].y & m), max2(v[r][c].z & m, v[r][c].w & m));
      t = max2(t, __shfl_xor_sync(0xffffffffu, t, 1));
      t = max2(t, __shfl_xor_sync(0xffffffffu, t, 2));
      top[r][c] = max(t & 0xFFFFu, t >> 16);
    }
  const int per = s.group / 32;   // 32-input chunks per group: 1, 2 or 4
  float scale[2][4], inv[2][4];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    if (per >= 2) {
      top[r][0] = max(top[r][0], top[r][1]);
      top[r][2] = max(top[r][2], top[r][3]);
    }
    if (per == 4) top[r][0] = max(top[r][0], top[r][2]);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      if (c % per != 0) {   // the same group as chunk 0, or chunk 2
        const bool two = c == 3 && per == 2;
        scale[r][c] = two ? scale[r][2] : scale[r][0];
        inv[r][c] = two ? inv[r][2] : inv[r][0];
        continue;
      }
      const float a = __uint_as_float(top[r][c] << 16);
      // (the values' FMA holds 24 s: finite for a < 2^120)
      const bool nan = top[r][c] >= (120u + 127u) << 7, zero = a < 0x1p-100f;
      scale[r][c] = nan ? __int_as_float(0x7FC00000) : zero ? 0.f : q4_scale(a);
      inv[r][c] = nan || zero ? 0.f : __fdividef(1.f, scale[r][c]);
    }
  }
  uint32_t word[2][4];
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint32_t raw[4] = {v[r][c].x, v[r][c].y, v[r][c].z, v[r][c].w};
      uint32_t nibble[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        nibble[2 * i] = q4_nibble(__uint_as_float(raw[i] << 16), inv[r][c]);
        nibble[2 * i + 1] = q4_nibble(__uint_as_float(raw[i] & 0xFFFF0000u), inv[r][c]);
      }
      word[r][c] = q4_pack_word(nibble);
    }
  const size_t block = ((size_t)b.e * s.tiles + b.nt / 2) * s.blocks + b.kb;
  const int row = b.nt % 2 * 16 + g;   // of the tile, and the one 8 behind it
  uint8_t* to = codes + block * kQ4CodeBytes + row * 16 + 4 * q;
  uint16_t* sc = scales + (block * kQ4Rows + row) * s.groups;
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      *reinterpret_cast<uint32_t*>(to + c * kQ4Rows * 16 + r * 8 * 16) = word[r][c];
      if (q == c && c % per == 0)
        sc[r * 8 * s.groups + c / per] = (uint16_t)(__float_as_uint(scale[r][c]) >> 16);
    }
}

__global__ void __launch_bounds__(kQ4Threads)
q4_dequantize_kernel(Q4Shape s, int n_experts, const uint8_t* __restrict__ codes,
                     const uint16_t* __restrict__ scales, uint4* __restrict__ w) {
  pdl_wait();
  pdl_launch_dependents();
  const Q4Block b = q4_block(s, n_experts);
  if (!b.ok) return;
  const int lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const size_t block = ((size_t)b.e * s.tiles + b.nt / 2) * s.blocks + b.kb;
  const int row = b.nt % 2 * 16 + g;
  const uint8_t* from = codes + block * kQ4CodeBytes + row * 16 + 4 * q;
  const uint16_t* sc = scales + (block * kQ4Rows + row) * s.groups;
  const Q4Bits pair_bits;
  uint32_t word[2][4], bits[2][4];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
#pragma unroll
    for (int c = 0; c < 4; ++c)
      word[r][c] = __ldcs(reinterpret_cast<const uint32_t*>(from + c * kQ4Rows * 16 + r * 8 * 16));
    const uint16_t* own = sc + r * 8 * s.groups;
    uint32_t lo, hi;
    if (s.groups == 4) {
      const uint2 p = __ldg(reinterpret_cast<const uint2*>(own));
      lo = p.x;
      hi = p.y;
    } else if (s.groups == 2) {
      const uint32_t p = __ldg(reinterpret_cast<const uint32_t*>(own));
      lo = __byte_perm(p, 0u, 0x1010);
      hi = __byte_perm(p, 0u, 0x3232);
    } else {
      lo = hi = __ldg(own) * 0x10001u;
    }
    bits[r][0] = lo;
    bits[r][1] = lo >> 16;
    bits[r][2] = hi;
    bits[r][3] = hi >> 16;
  }
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int n = b.nt * 16 + g + 8 * r, k = b.kb * 128 + c * 32 + q * 8;
      const Q4Scale v = q4_scale_pair(bits[r][c]);
      if (n < s.N && k < s.K)
        __stcs(w + (((size_t)b.e * s.N + n) * s.K + k) / 8,
               make_uint4(q4_value_pair(word[r][c], 0, v, pair_bits), q4_value_pair(word[r][c], 1, v, pair_bits),
                          q4_value_pair(word[r][c], 2, v, pair_bits), q4_value_pair(word[r][c], 3, v, pair_bits)));
    }
}

unsigned q4_ctas(const Q4Shape& s, int n_experts) {
  const int64_t warps = (int64_t)n_experts * 2 * s.tiles * s.blocks;
  return (unsigned)((warps + kQ4Threads / 32 - 1) / (kQ4Threads / 32));
}

}  // namespace

cudaError_t launch_q4_quantize(const dmoe_q4_desc& d, const void* w, void* codes, void* scales,
                               cudaStream_t s) {
  const Q4Shape sh = q4_shape(d);
  return launch_ex(q4_quantize_kernel, dim3(q4_ctas(sh, d.n_experts)), dim3(kQ4Threads), 0, s, true,
                   sh, d.n_experts, static_cast<const uint4*>(w), static_cast<uint8_t*>(codes),
                   static_cast<uint16_t*>(scales));
}

cudaError_t launch_q4_dequantize(const dmoe_q4_desc& d, const void* codes, const void* scales,
                                 void* w, cudaStream_t s) {
  const Q4Shape sh = q4_shape(d);
  return launch_ex(q4_dequantize_kernel, dim3(q4_ctas(sh, d.n_experts)), dim3(kQ4Threads), 0, s,
                   true, sh, d.n_experts, static_cast<const uint8_t*>(codes),
                   static_cast<const uint16_t*>(scales), static_cast<uint4*>(w));
}

}  // namespace dmoe

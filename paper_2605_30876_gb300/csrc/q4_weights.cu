// bf16 weights to 4-bit codes and group scales, and back. One warp takes 16 rows x 128 inputs
// (whole groups of every size): 4 KB of weights. Bound by the bytes: 268 M weights (256 matrices of
// 512 x 2048, groups of 64) are quantised in 104 us and brought back in 98.5 (DRAM 76 and 80 % busy;
// both in a row 200 us, what their bytes take at 6.8 TB/s). Quantising is close to its instructions,
// too (issue slots 66 %): each lane finds the scale of a quarter of the rows' groups.
#include "q4.cuh"

namespace dmoe {
namespace {

constexpr int kQ4Threads = 256;

struct Q4Block {   // a warp's 16 x 128 weights
  int e, nt, kb;
  bool ok;
};
// (At most 2^28 warps, and 32-bit divisions: with 64-bit ones quantising took 3 us more.)
__device__ __forceinline__ Q4Block q4_block(const Q4Shape& s, int n_experts) {
  const uint32_t i = blockIdx.x * (kQ4Threads / 32) + (threadIdx.x >> 5), blocks = s.blocks,
                 tiles = 2 * s.tiles, j = i / blocks, e = j / tiles;
  Q4Block b;
  b.kb = (int)(i - j * blocks);
  b.nt = (int)(j - e * tiles);
  b.e = (int)e;
  b.ok = b.e < n_experts;
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

// rint(w / s) + 8 in the lower bits, for a pair of weights, from inv = 1 / s within 2^-21. The quotient of
// eight significant bits by five is a tie of two integers or 2^-9 and more away from one, and w * inv
// is off by less than 2^-20: the sum with 384, rounded to 2^-15, brings a tie back to it and passes
// no other one. The second sum rounds to an integer, ties to even: kNibble's bits and 1 .. 15 more
// (a zero inv gives 8, the code of zero). With divisions for each weight and scale, 268 M weights
// and back took 335 us; with sums of one weight at a time, their lower bits masked, shifted and
// joined, 232 (144 of them quantising, bound by the ALUs).
constexpr uint32_t kNibble = 0x4B400000u;   // 1.5 * 2^23
__device__ __forceinline__ uint2 q4_nibble_pair(uint32_t two_bf16, float inv) {
  uint2 r;
  asm("{\n\t"
      ".reg .b64 w, i, s, m;\n\t"
      "mov.b64 w, {%2, %3};\n\t"
      "mov.b64 i, {%4, %4};\n\t"
      "mov.b64 s, {%5, %5};\n\t"
      "mov.b64 m, {%6, %6};\n\t"
      "fma.rn.f32x2 w, w, i, s;\n\t"
      "add.rn.f32x2 w, w, m;\n\t"
      "mov.b64 {%0, %1}, w;\n\t"
      "}"
      : "=r"(r.x), "=r"(r.y)
      : "r"(two_bf16 << 16), "r"(two_bf16 & 0xFFFF0000u), "r"(__float_as_uint(inv)),
        "r"(__float_as_uint(384.f)), "r"(__float_as_uint(12582912.f + 8.f - 384.f)));
  return r;
}
// Four such pairs as a word of codes. The products shift the nibbles to their places, and the sum starts
// from minus what kNibble's bits come to there. (A NaN fills its word; its group's values are NaNs.)
__device__ __forceinline__ uint32_t q4_word(const uint4& w, float inv) {
  const uint32_t two[4] = {w.x, w.y, w.z, w.w};
  uint32_t sum = 0u - kNibble * 0x11111111u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint2 n = q4_nibble_pair(two[i], inv);
    sum += n.x * (1u << 4 * i);
    sum += n.y * (1u << (16 + 4 * i));
  }
  return __funnelshift_l(sum, sum, 3);
}

// the larger magnitudes of eight weights' four pairs
__device__ __forceinline__ uint32_t max8(const uint4& w) {
  const uint32_t m = 0x7FFF7FFFu;
  return __vmaxu2(__vmaxu2(w.x & m, w.y & m), __vmaxu2(w.z & m, w.w & m));
}

// of both halves, with what the lane kLane away sends
template <int kLane>
__device__ __forceinline__ uint32_t max_with(uint32_t mine, uint32_t sent) {
  return __vmaxu2(mine, __shfl_xor_sync(0xffffffffu, sent, kLane));
}

__global__ void __launch_bounds__(kQ4Threads)
q4_quantize_kernel(Q4Shape s, int n_experts, const uint4* __restrict__ w, uint8_t* __restrict__ codes,
                   uint16_t* __restrict__ scales) {
  pdl_wait();
  pdl_launch_dependents();
  const Q4Block b = q4_block(s, n_experts);
  if (!b.ok) return;
  const int lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  uint4 v[2][4];       // rows g and g + 8; 32 inputs each
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int n = b.nt * 16 + g + 8 * r, k = b.kb * 128 + c * 32 + q * 8;
      v[r][c] = n < s.N && k < s.K
                    ? __ldcs(w + (((size_t)b.e * s.N + n) * s.K + k) / 8) : make_uint4(0, 0, 0, 0);
    }
  // the largest magnitudes of the 32 inputs, as the bits of two bf16 (row g's the lower)
  uint32_t top[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const uint32_t low = max8(v[0][c]), high = max8(v[1][c]);
    top[c] = __vmaxu2(__byte_perm(low, high, 0x5410), __byte_perm(low, high, 0x7632));
  }
  // over the four lanes of the rows: lane q gets those of chunk q, then of its group
  const bool upper = (q & 2) != 0, odd = (q & 1) != 0;
  const uint32_t even = max_with<2>(upper ? top[2] : top[0], upper ? top[0] : top[2]),
                 other = max_with<2>(upper ? top[3] : top[1], upper ? top[1] : top[3]);
  uint32_t mine = max_with<1>(odd ? other : even, odd ? even : other);
  const int per = s.group / 32;   // 32-input chunks per group: 1, 2 or 4
  if (per >= 2) mine = max_with<1>(mine, mine);
  if (per == 4) mine = max_with<2>(mine, mine);
  float scale[2], inv[2];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const float a = __uint_as_float(r == 0 ? mine << 16 : mine & 0xFFFF0000u);
    // (the values' FMA holds 24 s: finite for a < 2^120)
    const bool nan = !(a < 0x1p120f), zero = a < 0x1p-100f;
    scale[r] = nan ? __int_as_float(0x7FC00000) : zero ? 0.f : q4_scale(a);
    inv[r] = nan || zero ? 0.f : __fdividef(1.f, scale[r]);
  }
  const size_t block = ((size_t)b.e * s.tiles + b.nt / 2) * s.blocks + b.kb;
  const int row = b.nt % 2 * 16 + g;   // of the tile, and the one 8 behind it
  uint8_t* to = codes + block * kQ4CodeBytes + row * 16 + 4 * q;
  uint16_t* sc = scales + (block * kQ4Rows + row) * s.groups;
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    if (q % per == 0)
      sc[r * 8 * s.groups + q / per] = (uint16_t)(__float_as_uint(scale[r]) >> 16);
#pragma unroll
    for (int c = 0; c < 4; ++c)
      *reinterpret_cast<uint32_t*>(to + c * kQ4Rows * 16 + r * 8 * 16) =
          q4_word(v[r][c], __shfl_sync(0xffffffffu, inv[r], lane - q + c));
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

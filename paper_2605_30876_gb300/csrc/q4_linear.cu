// Products of sorted rows with their experts' 4-bit matrices, plain or gate and up with SwiGLU.
#include "q4.cuh"
#include "silu.cuh"

namespace dmoe {
namespace {

constexpr int kMmaWarps = 8;
constexpr int kMmaThreads = kMmaWarps * 32;

__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0,
                                          uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ __nv_bfloat162 both(uint32_t bits) {
  const uint32_t two = bits << 16 | bits;
  return *reinterpret_cast<const __nv_bfloat162*>(&two);
}

// 16 outputs of NT * 8 rows of one group: the warps take every kMmaWarps-th block of 64 inputs,
// their sums are added up in the order of the warps.
template <int NT, int MATS>
__device__ __forceinline__ void q4_rows(const Q4Args& a, const Q4Shape& s, int e, int nt, int r0,
                                        int r1, float* red) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
  const uint4* xrow[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int r = r0 + t * 8 + g;
    int64_t src = -1;
    if (r < r1) src = a.rows != nullptr ? __ldg(a.rows + r) : r;
    if (a.rows != nullptr && src >= 0) src /= a.k;
    xrow[t] = src >= 0 && src < a.T_x ? reinterpret_cast<const uint4*>(a.x + src * a.ldx) : nullptr;
  }
  float acc[MATS][NT][4] = {};
  const size_t tile = (size_t)e * s.row_tiles + nt;
#pragma unroll 4
  for (int kt = warp; kt < s.k_tiles; kt += kMmaWarps) {
    uint4 c[MATS];
    uint32_t sc[MATS][2];
#pragma unroll
    for (int m = 0; m < MATS; ++m) {
      c[m] = __ldg(static_cast<const uint4*>(a.codes[m]) + (tile * s.k_tiles + kt) * 32 + lane);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int gi = (kt * 64 + h * 32) / s.group;
        sc[m][h] = gi < s.groups ? __ldg(static_cast<const uint32_t*>(a.scales[m]) +
                                         (tile * 8 + g) * s.groups_pad + gi) : 0u;
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = kt * 64 + h * 32 + q * 8;
      uint4 b[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t)
        b[t] = xrow[t] != nullptr && k < s.K ? __ldg(xrow[t] + k / 8) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int m = 0; m < MATS; ++m) {
        const uint32_t lo = h == 0 ? c[m].x : c[m].z, hi = h == 0 ? c[m].y : c[m].w;
        const __nv_bfloat162 slo = both(sc[m][h] & 0xFFFFu), shi = both(sc[m][h] >> 16);
        const uint32_t a0[4] = {q4_value_pair(lo, 0, slo), q4_value_pair(hi, 0, shi),
                                q4_value_pair(lo, 1, slo), q4_value_pair(hi, 1, shi)};
        const uint32_t a1[4] = {q4_value_pair(lo, 2, slo), q4_value_pair(hi, 2, shi),
                                q4_value_pair(lo, 3, slo), q4_value_pair(hi, 3, shi)};
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          mma_16816(acc[m][t], a0, b[t].x, b[t].y);
          mma_16816(acc[m][t], a1, b[t].z, b[t].w);
        }
      }
    }
  }
  // red[warp][m][row of the pass][output of the tile]
  constexpr int kPer = MATS * NT * 8 * 16;
#pragma unroll
  for (int m = 0; m < MATS; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int n = g + (i >> 1) * 8, r = t * 8 + q * 2 + (i & 1);
        red[warp * kPer + (m * NT * 8 + r) * 16 + n] = acc[m][t][i];
      }
  __syncthreads();
  for (int i = tid; i < NT * 8 * 16; i += kMmaThreads) {
    const int r = r0 + i / 16, n = nt * 16 + i % 16;
    float v[MATS];
#pragma unroll
    for (int m = 0; m < MATS; ++m) {
      v[m] = red[m * NT * 8 * 16 + i];
      for (int w = 1; w < kMmaWarps; ++w) v[m] += red[w * kPer + m * NT * 8 * 16 + i];
    }
    if (r < r1 && n < s.N) {
      const float o = MATS == 2 ? silu_divide(v[0]) * v[MATS - 1] : v[0];
      if (a.y_fp32) static_cast<float*>(a.y)[r * a.ldy + n] = o;
      else static_cast<__nv_bfloat16*>(a.y)[r * a.ldy + n] = __float2bfloat16_rn(o);
    }
  }
  __syncthreads();
}

template <int MATS>
__global__ void __launch_bounds__(kMmaThreads)
q4_mma_kernel(Q4Args a, Q4Shape s) {
  extern __shared__ float red[];
  pdl_wait();
  pdl_launch_dependents();
  const int u = blockIdx.y, R = (int)a.R;
  int r0 = 0, r1 = R;
  if (a.offsets != nullptr) {
    r0 = max(__ldg(a.offsets + u), 0);
    r1 = min(__ldg(a.offsets + u + 1), R);
  }
  if (r0 >= r1) return;
  const int e = a.expert_ids != nullptr ? __ldg(a.expert_ids + u) : u;
  if (e < 0 || e >= a.n_experts) return;
  for (int nt = blockIdx.x; nt < s.row_tiles; nt += gridDim.x)
    for (int r = r0; r < r1; r += 32) {
      if (r1 - r <= 8) q4_rows<1, MATS>(a, s, e, nt, r, r1, red);
      else if (r1 - r <= 16) q4_rows<2, MATS>(a, s, e, nt, r, r1, red);
      else q4_rows<4, MATS>(a, s, e, nt, r, r1, red);
    }
}

}  // namespace

cudaError_t launch_q4_linear(const Q4Args& a, const dmoe_q4_desc& d, cudaStream_t st) {
  const Q4Shape s = q4_shape(d);
  const bool gated = a.codes[1] != nullptr;
  const int mats = gated ? 2 : 1;
  const size_t smem = sizeof(float) * kMmaWarps * mats * 32 * 16;
  const dim3 grid(s.row_tiles, a.n_groups);
  return launch_ex(gated ? q4_mma_kernel<2> : q4_mma_kernel<1>, grid, dim3(kMmaThreads), smem, st,
                   true, a, s);
}

}  // namespace dmoe

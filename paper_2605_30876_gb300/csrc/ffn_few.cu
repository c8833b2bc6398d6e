// The feed-forward block of the experts for few rows: what counts is to have the weights of the experts in
// use on their way at once, from all SMs. Two launches (gate and up with SwiGLU, then down) of many
// small CTAs; mma.sync.m16n8k16 with 16 rows of weights as A and eight token rows as B, both straight
// from global memory into the fragments. A lane's fragment takes pairs of k from four places; any
// order of k gives the same sum as long as A and B agree, so a lane takes eight neighbours (16 bytes)
// of a 32-long piece of K for two MMAs.
// The eight warps of a CTA share the sum over K (kKS ways) or the rows (8 / kKS ways); the parts meet in
// shared memory and are added in the order of the warps. The second launch has its first weights on
// their way before it waits for the first one's h.
#include <cuda_fp16.h>

#include <algorithm>

#include "dmoe_internal.cuh"

namespace dmoe {
namespace {

constexpr int kFewThreads = 256;
constexpr int kFewWarps = kFewThreads / 32;

struct FewParams {
  const int32_t* offsets;
  const int32_t* expert_ids;
  int n_groups, n_experts;
  int R;
  int M, K;                  // rows of a weight matrix, length of the sums
  const void* w[2];          // gate and up, or down and null
  const void* b;             // [R, K] rows
  int64_t ldb;
  void* out;                 // h or y
  int64_t ldo;
  void* pre;                 // up: gate and up products, or null
  int zero_rest;
};

template <bool kHalf>
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                          uint32_t b0, uint32_t b1) {
  if constexpr (kHalf)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <bool kHalf>
__device__ __forceinline__ void store_16(void* p, int64_t at, float v) {
  if constexpr (kHalf) static_cast<__half*>(p)[at] = __float2half_rn(v);
  else static_cast<__nv_bfloat16*>(p)[at] = __float2bfloat16_rn(v);
}

__device__ __forceinline__ int few_rows(const FewParams& p, int g, int* row0) {
  int lo = 0, hi = p.R;
  if (p.offsets != nullptr) {
    lo = min(max(__ldg(p.offsets + g), 0), p.R);
    hi = min(max(__ldg(p.offsets + g + 1), 0), p.R);
  }
  *row0 = lo;
  return max(hi - lo, 0);
}
__device__ __forceinline__ int few_expert(const FewParams& p, int g) {
  const int e = p.expert_ids != nullptr ? __ldg(p.expert_ids + g) : g;
  return e >= 0 && e < p.n_experts ? e : -1;
}

// kUp: a 16-row tile is eight rows of gate and the same eight of up, so that a lane holds both of an
// element. kMT tiles a warp, kNT times eight token rows at once, kSteps pieces of K in flight.
template <bool kUp, bool kHalf, int kMT, int kNT, int kKS, int kSteps>
__global__ void __launch_bounds__(kFewThreads, kMT == 1 ? 3 : 2)
ffn_few_kernel(const FewParams p) {
  constexpr int kMW = kFewWarps / kKS;          // warps side by side in M
  constexpr int kTile = kUp ? 8 : 16;           // rows of M in a tile
  constexpr int kRows = kMW * kMT * kTile;      // ... of a CTA
  constexpr int kCols = kNT * 8;
  constexpr int kMaxG = kMaxFfnExperts;
  extern __shared__ float4 s_acc[];             // [warp][tile][n tile][lane]
  __shared__ int s_first[kMaxG + 1];            // row chunks before a group
  __shared__ int s_sum[kFewWarps];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int ks = warp % kKS, mw = warp / kKS, g8 = lane >> 2, q = lane & 3;
  // (the second launch: the offsets were there before the first one released it)
  if (kUp) {
    pdl_wait();
    pdl_launch_dependents();
  }

  // chunks of up to kCols rows of every group, counted
  int mine[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int g = 2 * tid + j;
    int row0;
    if (g < p.n_groups && few_expert(p, g) >= 0) mine[j] = (few_rows(p, g, &row0) + kCols - 1) / kCols;
  }
  int sum = mine[0] + mine[1];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += v;
  }
  if (lane == 31) s_sum[warp] = sum;
  __syncthreads();
  int before = sum - mine[0] - mine[1], chunks = 0;
#pragma unroll
  for (int w = 0; w < kFewWarps; ++w) {
    if (w < warp) before += s_sum[w];
    chunks += s_sum[w];
  }
  s_first[2 * tid] = before;
  s_first[2 * tid + 1] = before + mine[0];
  if (tid == 0) s_first[kMaxG] = chunks;
  __syncthreads();

  const int m_units = (p.M + kRows - 1) / kRows, steps = (p.K + 31) / 32;
  const int per = (steps + kKS - 1) / kKS, k_begin = ks * per, k_end = min(steps, k_begin + per);
  bool waited = kUp;
  for (int u = blockIdx.x; u < chunks * m_units; u += gridDim.x) {
    const int chunk = u / m_units, m0 = (u - chunk * m_units) * kRows + mw * kMT * kTile;
    int lo = 0, hi = kMaxG - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_first[mid] <= chunk) lo = mid; else hi = mid - 1;
    }
    int row0;
    const int cnt = few_rows(p, lo, &row0), e = few_expert(p, lo);
    const int at = (chunk - s_first[lo]) * kCols, rows = min(kCols, cnt - at);
    row0 += at;
    // this lane's rows of weights: g8 and g8 + 8 of every tile
    const uint4* wr[kMT][2];
    bool there[kMT][2];
#pragma unroll
    for (int m = 0; m < kMT; ++m)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r = m0 + m * kTile + g8 + (kUp ? 0 : 8 * j);
        there[m][j] = r < p.M;
        wr[m][j] = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.w[kUp ? j : 0]) +
                                                  ((int64_t)e * p.M + (r < p.M ? r : 0)) * p.K) + q;
      }
    const uint4* br[kNT];
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
      const int r = min(n * 8 + g8, rows - 1);     // (past the last row: its columns are not used)
      br[n] = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.b) + (int64_t)(row0 + r) * p.ldb) + q;
    }
    float acc[kMT][kNT][4];
#pragma unroll
    for (int m = 0; m < kMT; ++m)
#pragma unroll
      for (int n = 0; n < kNT; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[m][n][j] = 0.f;
    for (int k = k_begin; k < k_end; k += kSteps) {
      uint4 a[kSteps][kMT][2], b[kSteps][kNT];
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const bool in = k + s < k_end && (k + s) * 32 + q * 8 < p.K;
#pragma unroll
        for (int m = 0; m < kMT; ++m)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            a[s][m][j] = in && there[m][j] ? __ldcs(wr[m][j] + (k + s) * 4) : make_uint4(0, 0, 0, 0);
      }
      if (!waited) {            // the first launch's h
        pdl_wait();
        pdl_launch_dependents();
        waited = true;
      }
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const bool in = k + s < k_end && (k + s) * 32 + q * 8 < p.K;
#pragma unroll
        for (int n = 0; n < kNT; ++n)
          b[s][n] = in && n * 8 < rows ? *(br[n] + (k + s) * 4) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int n = 0; n < kNT; ++n) {
          if (n > 0 && n * 8 >= rows) break;
#pragma unroll
          for (int m = 0; m < kMT; ++m) {
            const uint4 &x = a[s][m][0], &y = a[s][m][1];
            mma_16816<kHalf>(acc[m][n], x.x, y.x, x.y, y.y, b[s][n].x, b[s][n].y);
            mma_16816<kHalf>(acc[m][n], x.z, y.z, x.w, y.w, b[s][n].z, b[s][n].w);
          }
        }
    }
    // the warps' parts of the sum meet
    if (kKS > 1) {
      __syncthreads();          // (the unit before has been read)
#pragma unroll
      for (int m = 0; m < kMT; ++m)
#pragma unroll
        for (int n = 0; n < kNT; ++n)
          s_acc[((warp * kMT + m) * kNT + n) * 32 + lane] =
              make_float4(acc[m][n][0], acc[m][n][1], acc[m][n][2], acc[m][n][3]);
      __syncthreads();
    }
    // (tile, n tile) pairs of this warp's rows go round the warps that share them
#pragma unroll
    for (int i = 0; i < (kMT * kNT + kKS - 1) / kKS; ++i) {
      const int t = i * kKS + ks, m = t / kNT, n = t % kNT;
      if (t >= kMT * kNT || n * 8 >= rows) continue;
      float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < kKS; ++k) {
        const float4 f = s_acc[(((mw * kKS + k) * kMT + m) * kNT + n) * 32 + lane];
        v[0] += f.x;
        v[1] += f.y;
        v[2] += f.z;
        v[3] += f.w;
      }
      // rows g8 and g8 + 8 of the tile, columns (token rows) 2 q and 2 q + 1
      const int r = m0 + m * kTile + g8, c = n * 8 + 2 * q;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (c + j >= rows) continue;
        const int64_t row = row0 + c + j;
        if constexpr (kUp) {
          if (r < p.M) {
            store_16<kHalf>(p.out, row * p.ldo + r, v[j] / (1.f + __expf(-v[j])) * v[2 + j]);
            if (p.pre != nullptr) {
              store_16<kHalf>(p.pre, row * 2 * p.M + r, v[j]);
              store_16<kHalf>(p.pre, row * 2 * p.M + p.M + r, v[2 + j]);
            }
          }
        } else {
          if (r < p.M) store_16<kHalf>(p.out, row * p.ldo + r, v[j]);
          if (r + 8 < p.M) store_16<kHalf>(p.out, row * p.ldo + r + 8, v[2 + j]);
        }
      }
    }
  }
  if (!kUp && p.zero_rest) {    // rows in no group, a warp each
    for (int r = blockIdx.x * kFewWarps + warp; r < p.R; r += gridDim.x * kFewWarps) {
      bool owned = false;
      for (int g = lane; g < p.n_groups; g += 32) {
        int row0;
        const int cnt = few_rows(p, g, &row0);
        owned |= r >= row0 && r < row0 + cnt && few_expert(p, g) >= 0;
      }
      if (__any_sync(0xffffffffu, owned)) continue;
      uint4* row = reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + (int64_t)r * p.ldo);
      for (int c = lane; c < p.M / 8; c += 32) row[c] = make_uint4(0, 0, 0, 0);
    }
  }
  if (!waited) pdl_wait();      // (a CTA without units: nothing behind this launch starts before the first)
}

template <bool kUp, bool kHalf, int kMT, int kNT, int kKS, int kSteps>
cudaError_t launch_few(const FewParams& p, cudaStream_t s) {
  constexpr int rows = kFewWarps / kKS * kMT * (kUp ? 8 : 16);
  const int64_t units = (int64_t)std::min(p.R, p.n_groups + p.R / (kNT * 8)) * ((p.M + rows - 1) / rows);
  const int ctas = (int)std::min<int64_t>(units, 152 * (kMT == 1 ? 3 : 2));
  const size_t smem = sizeof(float4) * kFewWarps * kMT * kNT * 32;
  return launch_ex(ffn_few_kernel<kUp, kHalf, kMT, kNT, kKS, kSteps>, dim3(ctas), dim3(kFewThreads), smem, s,
                   true, p);
}

template <bool kHalf>
cudaError_t few(const FfnArgs& a, cudaStream_t s) {
  FewParams p{};
  p.offsets = a.offsets;
  p.expert_ids = a.expert_ids;
  p.n_groups = a.n_groups;
  p.n_experts = a.n_experts;
  p.R = (int)a.R;
  p.M = a.I;
  p.K = a.d;
  p.w[0] = a.w_gate;
  p.w[1] = a.w_up;
  p.b = a.x;
  p.ldb = a.ldx;
  p.out = a.h;
  p.ldo = a.I;
  p.pre = a.pre;
  cudaError_t e = a.R <= 8 ? launch_few<true, kHalf, 1, 1, 8, 8>(p, s) : launch_few<true, kHalf, 2, 4, 8, 2>(p, s);
  if (e != cudaSuccess) return e;
  p.M = a.d;
  p.K = a.I;
  p.w[0] = a.w_down;
  p.w[1] = nullptr;
  p.b = a.h;
  p.ldb = a.I;
  p.out = a.y;
  p.ldo = a.ldy;
  p.pre = nullptr;
  p.zero_rest = a.zero_rest ? 1 : 0;
  return a.R <= 8 ? launch_few<false, kHalf, 1, 1, 2, 8>(p, s) : launch_few<false, kHalf, 2, 4, 4, 2>(p, s);
}

}  // namespace

cudaError_t launch_expert_ffn_few(const FfnArgs& a, cudaStream_t s) {
  return a.dtype == DMOE_FP16 ? few<true>(a, s) : few<false>(a, s);
}

}  // namespace dmoe

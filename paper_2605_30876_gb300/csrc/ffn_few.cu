// The feed-forward block of the experts for few rows: what counts is to have the weights of the experts in
// use on their way at once, from all SMs. Two launches (gate and up with SwiGLU, then down) of many
// small CTAs; mma.sync.m16n8k16 with 16 rows of weights as A and eight token rows as B, both straight
// from global memory into the fragments. A lane's fragment takes pairs of k from four places; any
// order of k gives the same sum as long as A and B agree, so a lane takes eight neighbours (16 bytes)
// of a 32-long piece of K for two MMAs. (tcgen05 has nothing to win here: the weights'
// bytes are the bound, and its launches, with tensor memory and barriers to set up and 64 SMs at work,
// take 23.9 us where these take 14.2, for one token's eight experts of 2048 x 512; 50 MB at the copy rate are
// 7.4.)
// The eight warps of a CTA share the sum over K (kKS ways) or the rows (8 / kKS ways); the parts meet in
// shared memory and are added in the order of the warps. The second launch has its first weights on
// their way before it waits for the first one's h.
#include <cuda_fp16.h>

#include <algorithm>

#include "dmoe_internal.cuh"

namespace dmoe {
namespace {

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

// weights, read once: past L1
__device__ __forceinline__ uint4 load_stream(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

template <bool kHalf>
__device__ __forceinline__ void store_16(void* p, int64_t at, float v) {
  if constexpr (kHalf) static_cast<__half*>(p)[at] = __float2half_rn(v);
  else static_cast<__nv_bfloat16*>(p)[at] = __float2bfloat16_rn(v);
}

// g and u for the gradients: cut to the type's finite range, as the form for more rows does
template <bool kHalf>
__device__ __forceinline__ void store_16_finite(void* p, int64_t at, float v) {
  uint16_t w;
  if constexpr (kHalf) asm("cvt.rn.satfinite.f16.f32 %0, %1;" : "=h"(w) : "f"(v));
  else asm("cvt.rn.satfinite.bf16.f32 %0, %1;" : "=h"(w) : "f"(v));
  static_cast<uint16_t*>(p)[at] = w;
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
// element. A unit is kMT tiles a warp and up to 32 token rows of a group.
// - Up to eight token rows (single tokens, a batch routed token by token): a warp's part of them lies in
//   shared memory, in a place of its own, and weights are read kAhead pieces of K (32 each) ahead, into
//   the next unit, too: 256 experts of one row each come at 0.99 of the copy rate.
// - More of them (a block of tokens through its experts): the registers hold the sums of 32, and two
//   pieces of K are read at a time, token rows too (from L2, with the warps of the other rows).
constexpr int kFewCols = 32;
constexpr int few_pitch(int per) { return per * 64 + 16; }   // bytes of a row's part, off by a bank group
template <bool kUp, bool kHalf, int kMT, int kKS>
__global__ void __launch_bounds__(256, 2)
ffn_few_kernel(const FewParams p) {
  constexpr int kWarps = 8, kNT = kFewCols / 8, kAhead = kMT == 1 ? 8 : 4;
  constexpr int kMW = kWarps / kKS;             // warps side by side in M
  constexpr int kTile = kUp ? 8 : 16;           // rows of M in a tile
  constexpr int kRows = kMW * kMT * kTile;      // ... of a CTA
  constexpr int kCols = kFewCols;
  constexpr int kMaxG = kMaxFfnExperts;
  extern __shared__ float4 smem[];
  float4* s_acc = smem;                         // [warp][tile][n tile][lane]
  const int acc_nt = p.R <= 8 ? 1 : kNT;
  uint8_t* s_rows = reinterpret_cast<uint8_t*>(smem + kWarps * kMT * acc_nt * 32);   // [warp][row][part]
  __shared__ int s_first[2][kMaxG];             // chunks of rows before a group: groups of up to eight
  __shared__ int2 s_sum[kWarps];                // rows, and the others
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int ks = warp % kKS, mw = warp / kKS, g8 = lane >> 2, q = lane & 3;
  // (the second launch: the offsets were there before the first one released it)
  if (kUp) {
    pdl_wait();
    pdl_launch_dependents();
  }

  constexpr int kOwn = kMaxG / (kWarps * 32);
  int2 mine[kOwn], sum = make_int2(0, 0);
#pragma unroll
  for (int j = 0; j < kOwn; ++j) {
    const int g = kOwn * tid + j;
    int row0;
    const int cnt = g < p.n_groups && few_expert(p, g) >= 0 ? few_rows(p, g, &row0) : 0;
    mine[j] = make_int2(cnt > 0 && cnt <= 8 ? 1 : 0, cnt > 8 ? (cnt + kCols - 1) / kCols : 0);
    sum.x += mine[j].x;
    sum.y += mine[j].y;
  }
  const int2 own = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, sum.x, o), y = __shfl_up_sync(0xffffffffu, sum.y, o);
    if (lane >= o) {
      sum.x += x;
      sum.y += y;
    }
  }
  if (lane == 31) s_sum[warp] = sum;
  __syncthreads();
  int2 before = make_int2(sum.x - own.x, sum.y - own.y), chunks = make_int2(0, 0);
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const int2 v = s_sum[w];
    if (w < warp) {
      before.x += v.x;
      before.y += v.y;
    }
    chunks.x += v.x;
    chunks.y += v.y;
  }
#pragma unroll
  for (int j = 0; j < kOwn; ++j) {
    s_first[0][kOwn * tid + j] = before.x;
    s_first[1][kOwn * tid + j] = before.y;
    before.x += mine[j].x;
    before.y += mine[j].y;
  }
  __syncthreads();

  const int m_units = (p.M + kRows - 1) / kRows, steps = (p.K + 31) / 32;
  const int per = (steps + kKS - 1) / kKS, k_begin = min(ks * per, steps), k_steps = min(steps, k_begin + per) - k_begin;

  struct At {
    const uint4* w[2];       // this lane's first rows of weights, at the warp's first piece of K
    uint32_t there;          // bits: rows that exist
    int row0, rows, m0;
  };
  auto locate = [&](int u, int kind) -> At {
    At at;
    const int chunk = u / m_units;
    at.m0 = (u - chunk * m_units) * kRows + mw * kMT * kTile;
    int lo = 0, hi = kMaxG - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_first[kind][mid] <= chunk) lo = mid; else hi = mid - 1;
    }
    const int cnt = few_rows(p, lo, &at.row0), skip = (chunk - s_first[kind][lo]) * kCols;
    const int64_t e = few_expert(p, lo);
    at.rows = min(kCols, cnt - skip);
    at.row0 += skip;
    at.there = 0;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = at.m0 + g8 + (kUp ? 0 : 8 * j);
#pragma unroll
      for (int m = 0; m < kMT; ++m)
        if (r + m * kTile < p.M) at.there |= 1u << (2 * m + j);
      at.w[j] = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.w[kUp ? j : 0]) +
                                               (e * p.M + min(r, p.M - 1)) * p.K) + k_begin * 4 + q;
    }
    return at;
  };
  const int tile_stride = kTile * p.K / 8;      // 16-byte words from a tile's rows to the next one's
  auto load_weights = [&](const At& at, int k, uint4 (&a)[kMT][2]) {
    const bool in = k < k_steps && (k_begin + k) * 32 + q * 8 < p.K;
#pragma unroll
    for (int m = 0; m < kMT; ++m)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        a[m][j] = in && (at.there >> (2 * m + j) & 1u) ? load_stream(at.w[j] + m * tile_stride + k * 4)
                                                       : make_uint4(0, 0, 0, 0);
  };
  // a warp's sums of tile m, columns 8 n .. 8 n + 7
  auto sums_at = [&](int w, int m, int n) -> float4* { return s_acc + ((w * kMT + m) * acc_nt + n) * 32 + lane; };
  // all of them are there: (tile, n tile) pairs of this warp's rows go round the warps that share them
  auto finish = [&](const At& now, int n_tiles) {
    for (int t = ks; t < kMT * n_tiles; t += kKS) {
      const int m = t % kMT, n = t / kMT;
      float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < kKS; ++k) {
        const float4 f = *sums_at(mw * kKS + k, m, n);
        v[0] += f.x;
        v[1] += f.y;
        v[2] += f.z;
        v[3] += f.w;
      }
      // rows g8 and g8 + 8 of the tile, columns (token rows) 2 q and 2 q + 1
      const int r = now.m0 + m * kTile + g8, c = n * 8 + 2 * q;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (c + j >= now.rows) continue;
        const int64_t row = now.row0 + c + j;
        if constexpr (kUp) {
          if (r < p.M) {
            store_16<kHalf>(p.out, row * p.ldo + r, v[j] / (1.f + __expf(-v[j])) * v[2 + j]);
            if (p.pre != nullptr) {
              store_16_finite<kHalf>(p.pre, row * 2 * p.M + r, v[j]);
              store_16_finite<kHalf>(p.pre, row * 2 * p.M + p.M + r, v[2 + j]);
            }
          }
        } else {
          if (r < p.M) store_16<kHalf>(p.out, row * p.ldo + r, v[j]);
          if (r + 8 < p.M) store_16<kHalf>(p.out, row * p.ldo + r + 8, v[2 + j]);
        }
      }
    }
  };

  // ---------------- groups of up to eight rows
  const int narrow = chunks.x * m_units, wide = chunks.y * m_units;
  {
    const int pitch = few_pitch(per);
    uint8_t* const my_rows = s_rows + warp * 8 * pitch;
    // the warp's part of the token rows: 16-byte words, four lanes to a piece of K
    auto fetch_rows = [&](const At& at) {
      const int words = k_steps * 4, all = words * at.rows;
      for (int i = lane; i < all; i += 32) {
        const int r = i / words, c = i - r * words;
        const bool in = k_begin * 32 + c * 8 < p.K;
        const uint32_t to = (uint32_t)__cvta_generic_to_shared(my_rows + r * pitch + c * 16);
        const uint16_t* from = static_cast<const uint16_t*>(p.b) + (int64_t)(at.row0 + r) * p.ldb +
                               (in ? k_begin * 32 + c * 8 : 0);
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(in ? 16 : 0)
                     : "memory");
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    uint4 ring[kAhead][kMT][2];
    int u = blockIdx.x;
    At at;
    if (u < narrow) {
      at = locate(u, 0);
#pragma unroll
      for (int s = 0; s < kAhead; ++s) load_weights(at, s, ring[s]);
    }
    if (!kUp) {              // the first launch's h
      pdl_wait();
      pdl_launch_dependents();
    }
    if (u < narrow) fetch_rows(at);
    while (u < narrow) {
      const At now = at;
      float acc[kMT][4];
#pragma unroll
      for (int m = 0; m < kMT; ++m)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[m][j] = 0.f;
      asm volatile("cp.async.wait_all;" ::: "memory");
      __syncwarp();
      // (past the last row: what the place held; its columns are not used)
      const uint8_t* from = my_rows + g8 * pitch + q * 16;
      for (int k0 = 0; k0 < k_steps; k0 += kAhead) {
#pragma unroll
        for (int s = 0; s < kAhead; ++s) {
          if (k0 + s >= k_steps) break;
          const uint4 b = *reinterpret_cast<const uint4*>(from + (k0 + s) * 64);
#pragma unroll
          for (int m = 0; m < kMT; ++m) {
            const uint4 &x = ring[s][m][0], &y = ring[s][m][1];
            mma_16816<kHalf>(acc[m], x.x, y.x, x.y, y.y, b.x, b.y);
            mma_16816<kHalf>(acc[m], x.z, y.z, x.w, y.w, b.z, b.w);
          }
          load_weights(now, k0 + s + kAhead, ring[s]);
        }
      }
      // the next unit's weights and rows are on their way while this one's sums meet
      u += gridDim.x;
      if (u < narrow) {
        at = locate(u, 0);
#pragma unroll
        for (int s = 0; s < kAhead; ++s) load_weights(at, s, ring[s]);
        __syncwarp();
        fetch_rows(at);
      }
#pragma unroll
      for (int m = 0; m < kMT; ++m)
        *sums_at(warp, m, 0) = make_float4(acc[m][0], acc[m][1], acc[m][2], acc[m][3]);
      __syncthreads();
      finish(now, 1);
      __syncthreads();       // the sums have been read
    }
  }
  // ---------------- groups of more, 32 rows at a time (the CTAs that had fewer units begin)
  for (int u = (int)((blockIdx.x + gridDim.x - narrow % gridDim.x) % gridDim.x); u < wide; u += gridDim.x) {
    const At now = locate(u, 1);
    const uint4* br[kNT];
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
      const int r = min(n * 8 + g8, now.rows - 1);     // (as above)
      br[n] = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.b) + (int64_t)(now.row0 + r) * p.ldb) +
              k_begin * 4 + q;
    }
    float acc[kMT][kNT][4];
#pragma unroll
    for (int m = 0; m < kMT; ++m)
#pragma unroll
      for (int n = 0; n < kNT; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[m][n][j] = 0.f;
    for (int k = 0; k < k_steps; k += 2) {
      uint4 a[2][kMT][2], b[2][kNT];
#pragma unroll
      for (int s = 0; s < 2; ++s) load_weights(now, k + s, a[s]);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const bool in = k + s < k_steps && (k_begin + k + s) * 32 + q * 8 < p.K;
#pragma unroll
        for (int n = 0; n < kNT; ++n)
          b[s][n] = in && n * 8 < now.rows ? *(br[n] + (k + s) * 4) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int n = 0; n < kNT; ++n) {
          if (n * 8 >= now.rows) break;
#pragma unroll
          for (int m = 0; m < kMT; ++m) {
            const uint4 &x = a[s][m][0], &y = a[s][m][1];
            mma_16816<kHalf>(acc[m][n], x.x, y.x, x.y, y.y, b[s][n].x, b[s][n].y);
            mma_16816<kHalf>(acc[m][n], x.z, y.z, x.w, y.w, b[s][n].z, b[s][n].w);
          }
        }
    }
#pragma unroll
    for (int m = 0; m < kMT; ++m)
#pragma unroll
      for (int n = 0; n < kNT; ++n)
        if (n * 8 < now.rows)
          *sums_at(warp, m, n) = make_float4(acc[m][n][0], acc[m][n][1], acc[m][n][2], acc[m][n][3]);
    __syncthreads();
    finish(now, (now.rows + 7) / 8);
    __syncthreads();
  }
  if (!kUp && p.zero_rest) {    // rows in no group, a warp each
    for (int r = blockIdx.x * kWarps + warp; r < p.R; r += gridDim.x * kWarps) {
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
}

// What shared memory takes is missing from L1, through which the weights in flight come (two CTAs of 98 KB
// each: 4 experts of 4096 x 2048, a row or two each, 60 us; of 75 KB: 38).
constexpr size_t kFewSmem = 80 * 1024;
constexpr size_t few_smem(int64_t R, int tiles, int per) {
  return sizeof(float4) * 8 * tiles * (R <= 8 ? 1 : kFewCols / 8) * 32 + (size_t)8 * 8 * few_pitch(per);
}

// Ways a sum over K is cut, at least, and the pieces of K that are a warp's then.
constexpr int few_ks(int K) { return K > 1024 ? 8 : K > 512 ? 4 : K > 256 ? 2 : 1; }
constexpr int few_per(int K, int ks) { return ((K + 31) / 32 + ks - 1) / ks; }

// Units of a launch, at most
template <bool kUp>
int64_t few_units(const FewParams& p, int tiles, int ks) {
  const int rows = 8 / ks * tiles * (kUp ? 8 : 16);
  return (int64_t)std::min(p.R, p.n_groups + p.R / kFewCols) * ((p.M + rows - 1) / rows);
}

template <bool kUp, bool kHalf, int kMT, int kKS>
cudaError_t launch_form(const FewParams& p, cudaStream_t s) {
  const int ctas = (int)std::min<int64_t>(few_units<kUp>(p, kMT, kKS), 152 * 2);
  const size_t smem = few_smem(p.R, kMT, few_per(p.K, kKS));
  auto* kernel = ffn_few_kernel<kUp, kHalf, kMT, kKS>;
  static std::atomic<uint32_t> done;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  const uint32_t bit = dev < 32 ? 1u << dev : 0u;
  if (e == cudaSuccess && (done.load(std::memory_order_relaxed) & bit) == 0u) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kFewSmem);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  }
  if (e != cudaSuccess) return e;
  return launch_ex(kernel, dim3(ctas), dim3(256), smem, s, true, p);
}

// The sums over K are cut into as many parts as leave a warp eight pieces of each, and into more where there are
// fewer than 100 units for the SMs; a warp takes two tiles where that leaves two CTAs per SM their units.
// Us in a graph: 191 experts of 168 x 1632, a row each, cut eight ways 140, four (or two) 77, once 66; eight of
// 2048 x 512, down's sums of 512 cut four ways 15.1, two 14.2; one of 512 x 512 and 64 rows, two ways 11.3, eight
// 7.7; of 64 such eight in use, up cut two ways (128 units) 7.1, four 8.2.
template <bool kUp, bool kHalf, int kKS>
cudaError_t launch_cut(const FewParams& p, cudaStream_t s) {
  if (few_units<kUp>(p, 2, kKS) < 304) return launch_form<kUp, kHalf, 1, kKS>(p, s);
  return launch_form<kUp, kHalf, 2, kKS>(p, s);
}
template <bool kUp, bool kHalf>
cudaError_t launch_few(const FewParams& p, cudaStream_t s) {
  int ks = few_ks(p.K);
  while (ks < 8 && 32 * ks < p.K && few_units<kUp>(p, 1, ks) < 100) ks *= 2;
  switch (ks) {
    case 8: return launch_cut<kUp, kHalf, 8>(p, s);
    case 4: return launch_cut<kUp, kHalf, 4>(p, s);
    case 2: return launch_cut<kUp, kHalf, 2>(p, s);
    default: return launch_cut<kUp, kHalf, 1>(p, s);
  }
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
  const cudaError_t e = launch_few<true, kHalf>(p, s);
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
  return launch_few<false, kHalf>(p, s);
}

}  // namespace

// Which of the two forms a call takes. The number of experts in use is not known to the host; what counts is
// how many rows there are, how large the weights are (a group's come once for 32 rows), and that
// shared memory leaves room in L1. Us in a graph, weights of several calls in turn, tcgen05 / this form:
//   one expert of 2048 x 512: 8 rows 14.8 / 7.4, 128 rows 17.5 / 15.3, 256 rows 21.4 / 20.6; of 4096 x 4096:
//   8 rows 32.8 / 28.6; of 2048 x 2048: 32 rows 22.0 / 16.4; of 512 x 512: 512 rows 14.3 / 13.5
//   4 experts of 4096 x 2048: 8 rows 43.8 / 39.4, 16 rows 42 / 63 (room in L1)
//   8 of 2048 x 512: 8 rows 23.9 / 14.2, 64 rows 23.7 / 15.4, 256 rows 25.9 / 23.1 if each has 32 (a block routed as
//   one), but 25.9 / 29.2 if they have 13 to 61 (two chunks for some, one for others)
//   128 of 1024 x 512: 128 rows 70.3 / 71.7; 256 of 2048 x 512: 128 rows 128.9 / 131.6; 191 of 168 x 1632:
//   191 rows 84.5 / 65.9; 75 of 72 x 2480: 75 rows 48.3 / 24.1
bool expert_ffn_few_ok(const FfnArgs& a) {
  auto fits = [&](int K) { return few_smem(a.R, 2, few_per(K, few_ks(K))) <= kFewSmem; };
  return (a.R <= 8 || (a.R <= 512 && a.R * a.d * a.I <= (int64_t)1 << 27)) && fits(a.d) && fits(a.I);
}

cudaError_t launch_expert_ffn_few(const FfnArgs& a, cudaStream_t s) {
  return a.dtype == DMOE_FP16 ? few<true>(a, s) : few<false>(a, s);
}

}  // namespace dmoe

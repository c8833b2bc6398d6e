// Products of sorted rows with their experts' 4-bit matrices, plain or gate and up with SwiGLU.
//
// q4_mma_kernel: few rows per group, as a decoding step has. The weights' bytes are the bound: a
// warp takes two tiles of 16 outputs (gate and up, or neighbours), reads their codes straight into
// the A fragments of mma.sync (no shared memory, no shuffles: the layout is made for it), and
// multiplies them by 8, 16 or 32 rows of x. Where there are fewer tiles than warps, several
// warps of a CTA share a tile pair's inputs and add their sums up in shared memory, in order.
#include "q4.cuh"
#include "silu.cuh"

namespace dmoe {
namespace {

constexpr int kMmaWarps = 8;
constexpr int kMmaThreads = kMmaWarps * 32;

__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0,
                                          uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void store_y(const Q4Args& a, int64_t r, int n, float v) {
  if (a.y_fp32) static_cast<float*>(a.y)[r * a.ldy + n] = v;
  else static_cast<__nv_bfloat16*>(a.y)[r * a.ldy + n] = __float2bfloat16_rn(v);
}

// The groups that have rows and an expert, in order.
struct Q4Groups {
  int n;
  int e[kMaxExperts], r0[kMaxExperts], r1[kMaxExperts];
};
__device__ __forceinline__ void q4_groups(const Q4Args& a, Q4Groups& s, int* wcount) {
  const int u = threadIdx.x, lane = u & 31, warp = u >> 5, R = (int)a.R;
  static_assert(kMmaThreads >= kMaxExperts, "a thread per group");
  int e = u, r0 = 0, r1 = 0;
  if (u < a.n_groups) {
    r1 = R;
    if (a.offsets != nullptr) {
      r0 = max(__ldg(a.offsets + u), 0);
      r1 = min(__ldg(a.offsets + u + 1), R);
    }
    if (a.expert_ids != nullptr) e = __ldg(a.expert_ids + u);
  }
  const bool live = r0 < r1 && e >= 0 && e < a.n_experts;
  const uint32_t m = __ballot_sync(0xffffffffu, live);
  if (lane == 0) wcount[warp] = __popc(m);
  __syncthreads();
  int at = __popc(m & ((1u << lane) - 1u)), all = 0;
  for (int w = 0; w < kMmaWarps; ++w) {
    if (w < warp) at += wcount[w];
    all += wcount[w];
  }
  if (live) {
    s.e[at] = e;
    s.r0[at] = r0;
    s.r1[at] = r1;
  }
  if (u == 0) s.n = all;
  __syncthreads();
}

// A warp's steps through its work: units (tile pairs) u0, u0 + stride, ... of the CTA, each in passes of
// NT * 8 rows of its group, each over the warp's blocks of 64 inputs. Two cursors go the same way,
// one that starts copies and, behind it, one that multiplies.
struct Q4Plan {
  int64_t units;
  int pairs, share, per, pass_rows;
};
template <bool kGated>
struct Q4Cursor {
  int64_t u0;
  int p, longest;    // row of the pass within the group; rows of the CTA's longest group now
  int r0, r1;        // rows of this warp's group (r0 == r1: no unit)
  int pair, e;
  bool done;
  __device__ __forceinline__ void enter(const Q4Plan& pl, const Q4Groups& gs, int warp) {
    p = 0;
    done = u0 >= pl.units;
    r0 = r1 = longest = 0;
    if (done) return;
    const int64_t unit = u0 + warp / pl.share;
    if (unit < pl.units) {
      const int gi = (int)(unit / pl.pairs);
      pair = (int)(unit % pl.pairs);
      e = gs.e[gi];
      r0 = gs.r0[gi];
      r1 = gs.r1[gi];
    }
    longest = r1 - r0;
    if (pl.share > 1)
      for (int j = 0; j < pl.per; ++j)
        if (u0 + j < pl.units) {
          const int og = (int)((u0 + j) / pl.pairs);
          longest = max(longest, gs.r1[og] - gs.r0[og]);
        }
  }
  // the next pass, or the next unit's first
  __device__ __forceinline__ void next(const Q4Plan& pl, const Q4Groups& gs, int warp) {
    p += pl.pass_rows;
    if (p < longest) return;
    u0 += (int64_t)gridDim.x * pl.per;
    enter(pl, gs, warp);
  }
  __device__ __forceinline__ bool live() const { return r0 + p < r1; }
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
template <int N>
__device__ __forceinline__ void copy_small(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(N) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// The ring of a warp: a stage is a block's codes (2 x 512 bytes), scale pairs (2 x 256) and, up to 16
// rows a pass, rows of x (2 NT x 512). Every lane reads what it copied itself: no barriers. The
// CTA's shared memory is the rings and the warps' sums (two CTAs per SM: 4, 3 or 5 stages).
constexpr int kMmaSmem = 100 * 1024;
template <int NT>
struct Q4Ring {
  static constexpr bool kX = NT <= 2;   // (at 32 rows x is read directly: the stages would be too few)
  static constexpr int stage = 1536 + (kX ? 2 * NT * 512 : 0);
  static constexpr int red = kMmaWarps * NT * 8 * 32 * (int)sizeof(float);
  static constexpr int stages = (kMmaSmem - red) / kMmaWarps / stage;
};

template <int NT>
__device__ __forceinline__ const uint4* x_row(const Q4Args& a, int r, int r1, int q) {
  int64_t src = -1;
  if (r < r1) {
    src = r;
    if (a.rows != nullptr) {
      const int i = __ldg(a.rows + r);
      src = i >= 0 ? i / a.k : -1;
    }
  }
  return src >= 0 && src < a.T_x ? reinterpret_cast<const uint4*>(a.x + src * a.ldx) + q : nullptr;
}

// The copying cursor: the current pass's addresses, advanced block by block.
template <int NT, bool kGated, bool kG32>
struct Q4Copier {
  Q4Cursor<kGated> c;
  const uint4* codes[2];
  const uint32_t* scales[2];
  const uint4* xrow[NT];
  int kt, slot;
  __device__ __forceinline__ void enter_pass(const Q4Args& a, const Q4Shape& s, int first) {
    const int lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    kt = first;
    if (c.done || !c.live()) return;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      int nt = kGated ? c.pair : c.pair * 2 + m;
      nt = nt < s.row_tiles ? nt : s.row_tiles - 1;   // (the twin of an odd last tile: its outputs
                                                      // are behind n_out and not stored)
      const size_t tile = (size_t)c.e * s.row_tiles + nt;
      codes[m] = static_cast<const uint4*>(a.codes[kGated ? m : 0]) + tile * s.k_tiles * 32 + lane;
      scales[m] = static_cast<const uint32_t*>(a.scales[kGated ? m : 0]) + (tile * 8 + g) * s.groups_pad;
    }
    if (Q4Ring<NT>::kX)
#pragma unroll
      for (int t = 0; t < NT; ++t) xrow[t] = x_row<NT>(a, c.r0 + c.p + t * 8 + g, c.r1, q);
  }
  // starts the next block's copies, if there is one; always one group of copies
  __device__ __forceinline__ void copy(const Q4Args& a, const Q4Shape& s, const Q4Plan& pl,
                                       const Q4Groups& gs, int warp, int first, uint32_t ring) {
    while (!c.done && (!c.live() || kt >= s.k_tiles)) {
      c.next(pl, gs, warp);
      enter_pass(a, s, first);
    }
    if (!c.done) {
      const int lane = threadIdx.x & 31;
      const uint32_t dst = ring + slot * Q4Ring<NT>::stage;
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        copy16(dst + m * 512 + lane * 16, codes[m] + (size_t)kt * 32, 16);
        if (kG32) copy_small<8>(dst + 1024 + m * 256 + lane * 8, scales[m] + 2 * kt);   // (padded)
        else copy_small<4>(dst + 1024 + m * 256 + lane * 8, scales[m] + (s.group == 64 ? kt : kt >> 1));
      }
      if (Q4Ring<NT>::kX)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const bool ok = xrow[t] != nullptr && kt * 64 + h * 32 < s.K;   // (n_in is whole halves)
            copy16(dst + 1536 + (h * NT + t) * 512 + lane * 16,
                   ok ? static_cast<const void*>(xrow[t] + kt * 8 + h * 4) : codes[0], ok ? 16 : 0);
          }
      kt += pl.share;
      slot = slot + 1 == Q4Ring<NT>::stages ? 0 : slot + 1;
    }
    copies_commit();
  }
};

template <int NT, bool kG32>
__device__ __forceinline__ void mma_block(const uint8_t* st, const uint4 (&x)[2][NT],
                                          float (&acc)[2][NT][4]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const uint4 c = *reinterpret_cast<const uint4*>(st + m * 512 + lane * 16);
    const uint2 sc = *reinterpret_cast<const uint2*>(st + 1024 + m * 256 + lane * 8);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t lo = h == 0 ? c.x : c.z, hi = h == 0 ? c.y : c.w;
      const uint32_t bits = kG32 && h == 1 ? sc.y : sc.x;
      const Q4Scale slo = q4_scale_pair(bits), shi = q4_scale_pair(bits >> 16);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t a[4] = {q4_value_pair(lo, 2 * j, slo), q4_value_pair(hi, 2 * j, shi),
                               q4_value_pair(lo, 2 * j + 1, slo), q4_value_pair(hi, 2 * j + 1, shi)};
#pragma unroll
        for (int t = 0; t < NT; ++t)
          mma_16816(acc[m][t], a, j == 0 ? x[h][t].x : x[h][t].z, j == 0 ? x[h][t].y : x[h][t].w);
      }
    }
  }
}

// Outputs of a tile pair: acc[m][t][i] is output g + 8 (i / 2) of tile m, row 8 t + 2 q + i % 2.
// `share` warps of the CTA have parts of the sums; the CTA calls this together if share > 1.
template <int NT, bool kGated>
__device__ __forceinline__ void unit_outputs(const Q4Args& a, const Q4Shape& s, int pair, bool live,
                                             int r0, int r1, int share,
                                             const float (&acc)[2][NT][4], float* red) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
  if (share == 1) {
    if (!live) return;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = r0 + t * 8 + q * 2 + (i & 1), n = g + (i >> 1) * 8;
        if (r >= r1) continue;
        if (kGated) {
          if (pair * 16 + n < s.N) store_y(a, r, pair * 16 + n, silu_divide(acc[0][t][i]) * acc[1][t][i]);
        } else {
#pragma unroll
          for (int m = 0; m < 2; ++m)
            if (pair * 32 + m * 16 + n < s.N) store_y(a, r, pair * 32 + m * 16 + n, acc[m][t][i]);
        }
      }
    return;
  }
  // red[warp][row of the pass][output of the pair]
  constexpr int kPer = NT * 8 * 32;
  if (live) {
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          red[warp * kPer + (t * 8 + q * 2 + (i & 1)) * 32 + m * 16 + g + (i >> 1) * 8] = acc[m][t][i];
  }
  __syncthreads();
  if (live) {
    // the sharing warps take the pair's rows in turn; a lane has one output of the pair
    const int w0 = warp / share * share;
    for (int j = warp - w0; j < NT * 8; j += share) {
      float v = 0.f;
      for (int w = 0; w < share; ++w) v += red[(w0 + w) * kPer + j * 32 + lane];
      const float up = __shfl_down_sync(0xffffffffu, v, 16);
      const int r = r0 + j;
      if (r >= r1) continue;
      if (kGated) {
        if (lane < 16 && pair * 16 + lane < s.N) store_y(a, r, pair * 16 + lane, silu_divide(v) * up);
      } else {
        if (pair * 32 + lane < s.N) store_y(a, r, pair * 32 + lane, v);
      }
    }
  }
  __syncthreads();
}

template <int NT, bool kGated, bool kG32>
__device__ __forceinline__ void run_units(const Q4Args& a, const Q4Shape& s, Q4Plan pl,
                                          const Q4Groups& gs, uint8_t* smem) {
  using Ring = Q4Ring<NT>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  float* red = reinterpret_cast<float*>(smem);
  uint8_t* ring = smem + Ring::red + warp * (Ring::stages * Ring::stage);
  const uint32_t ring_addr = (uint32_t)__cvta_generic_to_shared(ring);
  const int first = warp % pl.share;
  pl.pass_rows = NT * 8;
  Q4Copier<NT, kGated, kG32> cp;
  cp.c.u0 = (int64_t)blockIdx.x * pl.per;
  cp.c.enter(pl, gs, warp);
  cp.slot = 0;
  cp.enter_pass(a, s, first);
  Q4Cursor<kGated> c = cp.c;
#pragma unroll 1
  for (int i = 0; i < Ring::stages - 1; ++i) cp.copy(a, s, pl, gs, warp, first, ring_addr);
  int slot = 0;
  for (; !c.done; c.next(pl, gs, warp)) {
    float acc[2][NT][4];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[m][t][i] = 0.f;
    const int from = c.r0 + c.p;
    if (c.live()) {
      const uint4* xrow[NT];
      if (!Ring::kX)
#pragma unroll
        for (int t = 0; t < NT; ++t) xrow[t] = x_row<NT>(a, from + t * 8 + g, c.r1, q);
#pragma unroll 1
      for (int kt = first; kt < s.k_tiles; kt += pl.share) {
        uint4 x[2][NT];
        if (!Ring::kX)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int t = 0; t < NT; ++t)
              x[h][t] = xrow[t] != nullptr && kt * 64 + h * 32 < s.K
                            ? __ldg(xrow[t] + kt * 8 + h * 4) : make_uint4(0, 0, 0, 0);
        cp.copy(a, s, pl, gs, warp, first, ring_addr);
        copies_wait<Ring::stages - 1>();
        const uint8_t* st = ring + slot * Ring::stage;
        if (Ring::kX)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int t = 0; t < NT; ++t)
              x[h][t] = *reinterpret_cast<const uint4*>(st + 1536 + (h * NT + t) * 512 + lane * 16);
        mma_block<NT, kG32>(st, x, acc);
        slot = slot + 1 == Ring::stages ? 0 : slot + 1;
      }
    }
    unit_outputs<NT, kGated>(a, s, c.pair, c.live(), from, c.r1, pl.share, acc, red);
  }
  copies_wait<0>();
}

template <bool kGated, bool kG32>
__global__ void __launch_bounds__(kMmaThreads, 2)
q4_mma_kernel(Q4Args a, Q4Shape s) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ Q4Groups groups;
  __shared__ int wcount[kMmaWarps];
  pdl_wait();
  pdl_launch_dependents();
  q4_groups(a, groups, wcount);
  Q4Plan pl;
  pl.pairs = kGated ? s.row_tiles : (s.row_tiles + 1) / 2;
  pl.units = (int64_t)groups.n * pl.pairs;
  // Warps that share a tile pair's inputs: as many as give the least blocks per warp, where two
  // blocks' time goes into an iteration's end.
  int64_t best = -1;
#pragma unroll
  for (int c = 1; c <= kMmaWarps; c *= 2) {
    const int64_t slots = (int64_t)gridDim.x * (kMmaWarps / c);
    const int64_t cost = (pl.units + slots - 1) / slots * ((s.k_tiles + c - 1) / c + 2);
    if (best < 0 || cost < best) {
      best = cost;
      pl.share = c;
    }
  }
  pl.per = kMmaWarps / pl.share;
  int most = 0;
  for (int i = 0; i < groups.n; ++i) most = max(most, groups.r1[i] - groups.r0[i]);
  if (most <= 8) run_units<1, kGated, kG32>(a, s, pl, groups, smem);
  else if (most <= 16) run_units<2, kGated, kG32>(a, s, pl, groups, smem);
  else run_units<4, kGated, kG32>(a, s, pl, groups, smem);
}

}  // namespace

cudaError_t launch_q4_linear(const Q4Args& a, const dmoe_q4_desc& d, cudaStream_t st) {
  const Q4Shape s = q4_shape(d);
  const bool gated = a.codes[1] != nullptr;
  const int64_t pairs = gated ? s.row_tiles : (s.row_tiles + 1) / 2;
  // at most a unit per CTA and group that can have rows
  const int64_t groups = a.n_groups < a.R ? a.n_groups : a.R;
  int64_t ctas = 2 * (int64_t)device_sm_count();
  if (pairs * groups < ctas) ctas = pairs * groups;
  auto* kernel = s.group == 32 ? (gated ? q4_mma_kernel<true, true> : q4_mma_kernel<false, true>)
                               : (gated ? q4_mma_kernel<true, false> : q4_mma_kernel<false, false>);
  static std::atomic<uint32_t> ready{0};   // a bit per device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  const uint32_t bit = dev < 32 ? 1u << dev : 0u;
  if (e == cudaSuccess && (ready.load(std::memory_order_acquire) & bit) == 0u) {
    for (auto* k : {q4_mma_kernel<true, true>, q4_mma_kernel<false, true>, q4_mma_kernel<true, false>,
                    q4_mma_kernel<false, false>})
      if (e == cudaSuccess)
        e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kMmaSmem);
    if (e == cudaSuccess) ready.fetch_or(bit, std::memory_order_release);
  }
  if (e != cudaSuccess) return e;
  return launch_ex(kernel, dim3((unsigned)ctas), dim3(kMmaThreads), kMmaSmem, st, true, a, s);
}

}  // namespace dmoe

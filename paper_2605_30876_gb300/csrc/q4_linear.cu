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
// NT * 8 rows of its group, each over the warp's chunks of 256 inputs. Two cursors go the same
// way, one that starts copies and, behind it, one that multiplies.
constexpr int kChunk = 4;   // blocks of 64 inputs
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

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// The ring of a warp: a stage is a chunk's codes (2 matrices x 4 x 512 bytes) and scale pairs (2 x
// 128 bytes, twice that in groups of 32). No other warp reads it.
template <bool kG32>
struct Q4Ring {
  static constexpr int words = kG32 ? 2 : 1;   // 16-byte pieces of scale pairs per chunk
  static constexpr int stage = 2 * kChunk * 512 + 2 * words * 128;
  static constexpr int stages = 2;
  static constexpr int bytes = kMmaWarps * stages * stage;
};
constexpr int kRedTiles = 2;   // tiles of 8 rows whose sums are exchanged at a time
template <int NT>
constexpr int q4_red_bytes() {
  return kMmaWarps * (NT < kRedTiles ? NT : kRedTiles) * 8 * 32 * (int)sizeof(float);
}

__device__ uint4 q4_zero_row[kMaxDModel / 8];   // stands in for sources that are not there

// the row of x of sorted row r, from input 8 q on; behind the group's last row, that one's (its
// products are not stored)
__device__ __forceinline__ const uint4* x_row(const Q4Args& a, int r, int r1, int q) {
  r = min(r, r1 - 1);
  int64_t src = r;
  if (a.rows != nullptr) {
    const int i = __ldg(a.rows + r);
    src = i >= 0 ? i / a.k : -1;
  }
  return (src >= 0 && src < a.T_x ? reinterpret_cast<const uint4*>(a.x + src * a.ldx) : q4_zero_row) + q;
}

// The copying cursor: the current unit's addresses, advanced chunk by chunk.
template <bool kGated, bool kG32>
struct Q4Copier {
  using Ring = Q4Ring<kG32>;
  Q4Cursor<kGated> c;
  const uint4* codes[2];
  const uint32_t* scales[2];
  int ch, slot;
  __device__ __forceinline__ void enter_pass(const Q4Args& a, const Q4Shape& s, int first) {
    const int lane = threadIdx.x & 31;
    ch = first;
    if (c.done || !c.live()) return;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      int nt = kGated ? c.pair : c.pair * 2 + m;
      nt = nt < s.row_tiles ? nt : s.row_tiles - 1;   // (the twin of an odd last tile: its outputs
                                                      // are behind n_out and not stored)
      const size_t tile = (size_t)c.e * s.row_tiles + nt;
      codes[m] = static_cast<const uint4*>(a.codes[kGated ? m : 0]) + tile * s.k_tiles * 32 + lane;
      scales[m] = static_cast<const uint32_t*>(a.scales[kGated ? m : 0]) +
                  (tile * 8 + (lane >> 2)) * s.groups_pad;
    }
  }
  // starts the next chunk's copies, if there is one; always one group of copies
  __device__ __forceinline__ void copy(const Q4Args& a, const Q4Shape& s, const Q4Plan& pl,
                                       const Q4Groups& gs, int warp, int first, int chunks,
                                       uint32_t ring) {
    while (!c.done && (!c.live() || ch >= chunks)) {
      c.next(pl, gs, warp);
      enter_pass(a, s, first);
    }
    if (!c.done) {
      const int lane = threadIdx.x & 31;
      const uint32_t dst = ring + slot * Ring::stage;
      const int kt = ch * kChunk;
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const uint4* src = codes[m] + kt * 32;
#pragma unroll
        for (int i = 0; i < kChunk; ++i)
          if (kt + i < s.k_tiles) copy16(dst + lane * 16 + (m * kChunk + i) * 512, src + i * 32);
        const int gi = kG32 ? ch * 8 : s.group == 64 ? ch * 4 : (ch * 2) & ~3;
#pragma unroll
        for (int w = 0; w < Ring::words; ++w)
          if ((lane & 3) == 0 && gi + 4 * w < s.groups_pad)
            copy16(dst + 2 * kChunk * 512 + (m * Ring::words + w) * 128 + lane * 4, scales[m] + gi + 4 * w);
      }
      ch += pl.share;
      slot = slot + 1 == Ring::stages ? 0 : slot + 1;
    }
    copies_commit();
  }
};

// One block of 64 inputs: st is the lane's place in the block's codes
template <int NT>
__device__ __forceinline__ void mma_block(const uint8_t* st, const uint32_t (&bits)[2][2],
                                          const uint4 (&x)[2][NT], float (&acc)[2][NT][4]) {
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const uint4 c = *reinterpret_cast<const uint4*>(st + m * kChunk * 512);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t lo = h == 0 ? c.x : c.z, hi = h == 0 ? c.y : c.w;
      const Q4Scale slo = q4_scale_pair(bits[m][h]), shi = q4_scale_pair(bits[m][h] >> 16);
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

// A chunk: kFull has all its blocks and all of their inputs.
template <int NT, bool kG32, bool kFull>
__device__ __forceinline__ void mma_chunk(const Q4Shape& s, int ch, const uint8_t* st,
                                          const uint4* const (&xrow)[NT], float (&acc)[2][NT][4]) {
  const int lane = threadIdx.x & 31;
  uint4 sc[2][Q4Ring<kG32>::words];
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int w = 0; w < Q4Ring<kG32>::words; ++w)
      sc[m][w] = *reinterpret_cast<const uint4*>(st + 2 * kChunk * 512 +
                                                 (m * Q4Ring<kG32>::words + w) * 128 + (lane >> 2) * 16);
  const bool g128 = s.group == 128, odd = ch & 1;
#pragma unroll
  for (int i = 0; i < kChunk; ++i) {
    const int kt = ch * kChunk + i;
    if (!kFull && kt >= s.k_tiles) break;
    uint4 x[2][NT];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int t = 0; t < NT; ++t)
        x[h][t] = kFull || kt * 64 + h * 32 < s.K   // (n_in is whole halves)
                      ? __ldg(xrow[t] + kt * 8 + h * 4) : make_uint4(0, 0, 0, 0);
    uint32_t bits[2][2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const uint32_t v[4] = {sc[m][0].x, sc[m][0].y, sc[m][0].z, sc[m][0].w};
      if (kG32) {
        const uint4 o = sc[m][Q4Ring<kG32>::words - 1];
        const uint32_t w[4] = {o.x, o.y, o.z, o.w};
        bits[m][0] = i < 2 ? v[2 * i & 3] : w[2 * i & 3];
        bits[m][1] = i < 2 ? v[(2 * i + 1) & 3] : w[(2 * i + 1) & 3];
      } else {
        bits[m][0] = bits[m][1] = g128 ? (odd ? v[2 + i / 2] : v[i / 2]) : v[i];
      }
    }
    mma_block<NT>(st + i * 512 + lane * 16, bits, x, acc);
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
  // red[warp][row of the part][output of the pair]
  constexpr int kTiles = NT < kRedTiles ? NT : kRedTiles, kPer = kTiles * 8 * 32;
#pragma unroll
  for (int t0 = 0; t0 < NT; t0 += kTiles) {
    if (live) {
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            red[warp * kPer + (t * 8 + q * 2 + (i & 1)) * 32 + m * 16 + g + (i >> 1) * 8] =
                acc[m][t0 + t][i];
    }
    __syncthreads();
    if (live) {
      // the sharing warps take the part's rows in turn; a lane has one output of the pair
      const int w0 = warp / share * share;
      for (int j = warp - w0; j < kTiles * 8; j += share) {
        float v = 0.f;
        for (int w = 0; w < share; ++w) v += red[(w0 + w) * kPer + j * 32 + lane];
        const float up = __shfl_down_sync(0xffffffffu, v, 16);
        const int r = r0 + t0 * 8 + j;
        if (r >= r1) continue;
        if (kGated) {
          if (lane < 16 && pair * 16 + lane < s.N)
            store_y(a, r, pair * 16 + lane, silu_divide(v) * up);
        } else {
          if (pair * 32 + lane < s.N) store_y(a, r, pair * 32 + lane, v);
        }
      }
    }
    __syncthreads();
  }
}

template <int NT, bool kGated, bool kG32>
__device__ __forceinline__ void run_units(const Q4Args& a, const Q4Shape& s, Q4Plan pl,
                                          const Q4Groups& gs, uint8_t* smem) {
  using Ring = Q4Ring<kG32>;
  const int warp = threadIdx.x >> 5, g = (threadIdx.x & 31) >> 2, q = threadIdx.x & 3;
  uint8_t* ring = smem + warp * (Ring::stages * Ring::stage);
  const uint32_t ring_addr = (uint32_t)__cvta_generic_to_shared(ring);
  float* red = reinterpret_cast<float*>(smem + Ring::bytes);
  const int first = warp % pl.share, chunks = (s.k_tiles + kChunk - 1) / kChunk;
  const int full = s.K / (64 * kChunk);
  pl.pass_rows = NT * 8;
  Q4Copier<kGated, kG32> cp;
  cp.c.u0 = (int64_t)blockIdx.x * pl.per;
  cp.c.enter(pl, gs, warp);
  cp.slot = 0;
  cp.enter_pass(a, s, first);
  Q4Cursor<kGated> c = cp.c;
#pragma unroll 1
  for (int i = 0; i < Ring::stages - 1; ++i) cp.copy(a, s, pl, gs, warp, first, chunks, ring_addr);
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
#pragma unroll
      for (int t = 0; t < NT; ++t) xrow[t] = x_row(a, from + t * 8 + g, c.r1, q);
#pragma unroll 1
      for (int ch = first; ch < chunks; ch += pl.share) {
        cp.copy(a, s, pl, gs, warp, first, chunks, ring_addr);
        copies_wait<Ring::stages - 1>();
        __syncwarp();   // (scale pairs are read by the lanes beside the copying one)
        const uint8_t* st = ring + slot * Ring::stage;
        if (ch < full) mma_chunk<NT, kG32, true>(s, ch, st, xrow, acc);
        else mma_chunk<NT, kG32, false>(s, ch, st, xrow, acc);
        __syncwarp();
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
  // Warps that share a tile pair's inputs: as many as give the least chunks per warp, where half a
  // chunk's time goes into an iteration's end.
  const int chunks = (s.k_tiles + kChunk - 1) / kChunk;
  int64_t best = -1;
#pragma unroll
  for (int c = 1; c <= kMmaWarps; c *= 2) {
    const int64_t slots = (int64_t)gridDim.x * (kMmaWarps / c);
    const int64_t cost = (pl.units + slots - 1) / slots * (2 * ((chunks + c - 1) / c) + 1);
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
        e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 Q4Ring<true>::bytes + q4_red_bytes<4>());
    if (e == cudaSuccess) ready.fetch_or(bit, std::memory_order_release);
  }
  if (e != cudaSuccess) return e;
  // (a group has no more rows than there are: the sums' space for passes of 8, 16 or 32)
  const size_t smem = (s.group == 32 ? Q4Ring<true>::bytes : Q4Ring<false>::bytes) +
                      (a.R <= 8 ? q4_red_bytes<1>() : a.R <= 16 ? q4_red_bytes<2>() : q4_red_bytes<4>());
  return launch_ex(kernel, dim3((unsigned)ctas), dim3(kMmaThreads), smem, st, true, a, s);
}

}  // namespace dmoe

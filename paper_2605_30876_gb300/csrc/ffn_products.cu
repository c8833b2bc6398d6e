// The gated feed-forward block of the experts on rows sorted by expert, and its gradients:
//   g = Wg x, u = Wu x, h = silu(g) * u, y = Wd h
//   dh = Wd^T dy, dg = dh u s (1 + g (1 - s)), du = dh g s   (s = sigmoid(g))
//   dx = Wg^T dg + Wu^T du, dWg = dg^T x, dWu = du^T x, dWd = dy^T h
// Five products, one kernel form of each (kMode):
//   kUp    D[i, r]  = Wg x, Wu x      epilogue: SwiGLU -> h (and g, u for the gradients)
//   kDown  D[c, r]  = Wd h            epilogue: y
//   kGradH D[i, r]  = Wd^T dy         epilogue: dg, du from g, u (dh stays in tensor memory, fp32)
//   kGradX D[c, r]  = Wg^T dg + Wu^T du, one sum over both
//   kGradW D[n, c]  = out^T in        over the rows of an expert
// In the first four the weights are the MMA's M operand and the rows of a group its N: a group of
// few rows wastes no tensor work on the other side and its weights stream once. Wd and Wg / Wu are
// read as they lie, along the reduction (kUp, kDown: K-major) or across it (kGradH, kGradX:
// MN-major, the tensor cores' transposed operand); so are both operands of kGradW. Nothing is
// transposed in memory. kGradW's three gradients are one launch (a small training step takes 5 us less than
// with two).
//
// Two CTAs of neighbouring SMs (a cluster) share an MMA of M = 256 (cta_group::2): each holds 128 of
// the M rows and half of the N columns. A persistent pair per two SMs takes units (group, 256 rows
// of M, up to 256 columns of N) in turn; they are found on the device from the offsets, so that no
// call waits for the host. Warp 0 issues the TMA loads, warp 1 of the first CTA the MMAs; the warps from
// 2 on (sixteen, in kGradW eight) run the epilogue from one of two accumulators in tensor memory while
// the other fills; the one behind them decodes units ahead. The last warp: in kGradW it clears what a stage
// holds behind an expert's last row (the rows there are another expert's, and 0 * inf would not be 0);
// in kDown and kGradX it writes the zeros of rows in no group, where they are wanted.
// Where there are fewer units than half of the pairs, up to four pairs (a cluster) share a unit's sum (split):
// each takes a part of the reduction and, at the end, a part of the columns, for which it reads the other
// pairs' sums from their shared memory and adds them in the order of the pairs.
// Sums are fp32 throughout. g, u, dg, du and h are rounded to the rows' type between products: they
// are the next product's operands, and the tensor cores take 16 bits (two operands for each, high and low
// part, would be twice the work). In bf16, 59000 rows: y and dWd are off by 0.0023 of their size so, dx, dWg and dWu by
// 0.0031, and by 0.0017, the rounding of the result, with g, u and h in fp32.
// Waits are bounded, record a timeout and unwind.
//
// What bounds it, in bf16 with inputs larger than L2: 1024 rows for each of 64 experts of 2048 x 1024 take
// 510 us forward (1.62 PFLOP/s, 0.85 of a large library product's rate) and 1080 backward (1.53): the
// tensor pipe, epilogues at the ends. 230 rows each of 256 experts of 2048 x 512: 414 (5.6 TB/s) and
// 792 us (5.4 TB/s): weights and rows from HBM, with MMAs of N < 256, which take 60 ns from N = 32 to 160,
// close behind. Small calls: 5 us a launch before the first bytes and after the last.
#include <cuda_fp16.h>

#include <algorithm>
#include <climits>
#include <mutex>

#include "dmoe_internal.cuh"
#include "silu.cuh"
#include "sm100_ptx.cuh"

namespace dmoe {
namespace {

constexpr int kCluster = 2;
constexpr int kTileABytes = 128 * 128;      // 128 rows (or 2 x 64 columns) x 64 of K
constexpr int kMaxStages = 8;
constexpr int kQueue = 4;
constexpr int kLevels = 4;                  // heights of the boxes of rows
constexpr int kMaxGroups = kMaxFfnExperts;
constexpr int kNMax = 256;
// A wait lasts as long as a unit at most: microseconds, but for the weights' gradients of very many rows, 317 ns for 64
// of them (with 1 s for all waits 203 M rows of one expert ran out of time). They have a second, and 1 us for 64 rows.
constexpr uint64_t kWaitNs = 1000000000ull;
constexpr uint64_t kStageNs = 1000;

enum Mode { kUp, kDown, kGradH, kGradX, kGradW };

__device__ DevErrRecord ffn_fault;

// A box costs the SM's copy engine about 100 cycles besides its rows, and with six boxes of 2 to 8 KB for
// 128 of K a stage took 0.5 us whatever its MMAs took: whole stages come in as few boxes as can be, through
// maps in which 64 neighbours of the fast dimension are one of their own (`whole`). What is cut by the
// end of a matrix comes in boxes of 64 (`cut`), filled up with zeros.
struct Maps {
  CUtensorMap a[2], a_cut[2];             // weights, or (kGradW) the output side's rows
  CUtensorMap b[kLevels], b_cut[kLevels]; // rows in boxes of level_rows
  CUtensorMap out[3];                     // kGradW: the gradients
};

struct Params {
  const int32_t* offsets;
  const int32_t* expert_ids;
  int n_groups, n_experts;
  int64_t R;
  int n_max;                // columns of a unit, at most (kGradW: of N)
  int M;                    // valid rows of D: I or d
  int K;                    // length of a part's reduction
  int parts;                // kGradX: sums over gate and up
  int m_tiles;
  // kGradW: the gradients of gate and up, M x N each, then that of down (either may be missing), in tiles
  int M_down, N, N_down;
  int n_tiles, m_tiles_down, n_tiles_down;
  int up_units, per_group;  // of a group: of gate and up together, and all
  int level_rows[kLevels];
  int stages;
  void* out;                // h, y, dpre or dx
  int64_t ldo;
  void* pre;                // kUp: written (or null); kGradH: read
  int I;
  int hold;
  int zero_rest;            // kDown, kGradX
  int after_x;              // kGradW: the launch before is kGradX's
  int split;                // pairs of a cluster, which share a unit (then the only one of theirs)
};

// A commit costs the issuing thread about as much as two MMAs, so slots of the ring are given back
// after eight MMAs: a stage is two steps of K = 64. An expert's rows are few, and an end inside a
// stage costs loads: kGradW's stages are one step, given back two at a time.
template <int kMode> constexpr int sub_steps() { return kMode == kGradW ? 1 : 2; }
template <int kMode> constexpr int per_commit() { return kMode == kGradW ? 2 : 1; }
// The launch before is one of the same call. It was released when its own wait had returned, with all work before the
// call complete: what the call was given (the weights, the offsets) is read before this launch's wait (a token's
// eight experts 14.8 us, 17.9 with all reads behind it; a small training step 129 and 139). What another launch
// of the call made is read behind it: rows of B, and all that kGradW reads. kGradX, before kGradW, writes nothing that
// kGradW reads and has waited for kGradH, but that kGradH's dpre is visible to a third launch is promised by that
// launch's own wait alone. (Without it kGradW began where kGradX's units had run out: 126 us instead of 129.)
template <int kMode> constexpr bool early() { return kMode == kDown || kMode == kGradX; }
// Warps of the epilogue: sixteen take half as long as eight with a launch's last tile (a small training
// step of 6186 rows 143 us with eight, 133 with sixteen), but kGradW's words in shared memory would take
// the place of stages.
template <int kMode> constexpr int epi_warps() { return kMode == kGradW ? 8 : 16; }
template <int kMode> constexpr int threads() { return (4 + epi_warps<kMode>()) * 32; }
template <int kMode> constexpr bool a_mn() { return kMode >= kGradH; }
template <int kMode> constexpr bool b_mn() { return kMode == kGradW; }
constexpr int kPitch = 80;      // of a column's 32 rows of D in shared memory, off by a bank group
template <int kMode> constexpr int epi_bytes() {
  return epi_warps<kMode>() * (kMode == kGradW ? 4096 : kMode == kUp ? 1024 + 8 * kPitch : 16 * kPitch);
}

template <bool kHalf>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  if constexpr (kHalf) {
    const __half2 b = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&b);
  } else {
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&b);
  }
}
// g and u for the gradients: what the type cannot hold becomes its largest value (and NaN stays NaN). A gate of
// -70000 is an exact 0 in h, and with -inf in its place dg and du were 0 * inf in fp16, as they were for rows with dy = 0.
template <bool kHalf>
__device__ __forceinline__ uint32_t pack2_finite(float lo, float hi) {
  uint32_t w;
  if constexpr (kHalf) asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  else asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}
template <bool kHalf>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  if constexpr (kHalf) return __half22float2(*reinterpret_cast<const __half2*>(&w));
  return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w));
}

// AND over the epilogue's threads (named barrier 1)
template <int kThreads>
__device__ __forceinline__ bool epilogue_all(bool v) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "bar.red.and.pred q, 1, %2, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)v), "n"(kThreads)
      : "memory");
  return r != 0;
}

__host__ __device__ inline int round_up(int v, int to) { return (v + to - 1) / to * to; }

// rows of group g, cut to [0, R]
__device__ __forceinline__ void group_rows(const Params& p, int g, int64_t* row0, int* count) {
  int64_t lo = 0, hi = p.R;
  if (p.offsets != nullptr) {
    lo = __ldg(p.offsets + g);
    hi = __ldg(p.offsets + g + 1);
    lo = lo < 0 ? 0 : lo > p.R ? p.R : lo;
    hi = hi < 0 ? 0 : hi > p.R ? p.R : hi;
  }
  *row0 = lo;
  *count = hi > lo ? (int)(hi - lo) : 0;
}
__device__ __forceinline__ int group_expert(const Params& p, int g) {
  const int e = p.expert_ids != nullptr ? __ldg(p.expert_ids + g) : g;
  return e >= 0 && e < p.n_experts ? e : -1;
}

struct Unit {
  int row, rows, e;   // first row and their number (kGradW: of the sum); e < 0: the end
  int part, m, n;     // kGradW: gate, up or down; column tile
};

template <int kMode, bool kHalf, bool kSplit>
__global__ void __launch_bounds__(threads<kMode>(), 1)
ffn_products_kernel(const __grid_constant__ Maps tm, const Params p) {
  constexpr int kSub = sub_steps<kMode>(), kPer = per_commit<kMode>();
  constexpr int kEpiWarps = epi_warps<kMode>(), kPlanWarp = 2 + kEpiWarps, kFixWarp = 3 + kEpiWarps;
  constexpr int kStep = kEpiWarps * 4;       // columns that the groups of four warps take at once, 16 each
  constexpr bool kAmn = a_mn<kMode>(), kBmn = b_mn<kMode>();
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (ptx::smem_addr(smem_raw) & 1023u)) & 1023u);
  const uint32_t b_sub = (uint32_t)p.level_rows[0] * 128u;   // bytes of one K = 64 step of B
  const uint32_t stage_bytes = kSub * (kTileABytes + b_sub);
  uint8_t* s_epi = smem + (uint32_t)p.stages * stage_bytes;
  uint64_t* full = reinterpret_cast<uint64_t*>(s_epi + epi_bytes<kMode>());
  uint64_t* empty = full + kMaxStages;
  uint64_t* tail = empty + kMaxStages;       // kGradW: this CTA's part of a group's last stage
  uint64_t* acc_full = tail + kMaxStages;
  uint64_t* acc_empty = acc_full + 2;
  uint64_t* drain = acc_empty + 2;
  uint64_t* held = drain + 1;
  uint64_t* d_full = held + 1;
  uint64_t* d_empty = d_full + kQueue;
  int* s_unit = reinterpret_cast<int*>(d_empty + kQueue);   // [kQueue][4]
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(s_unit + 4 * kQueue);
  volatile int* s_abort = reinterpret_cast<int*>(s_tmem + 1);
  // (not kGradW) [kMaxGroups + 1] units before a group, and its first row and rows
  int* s_first = reinterpret_cast<int*>(s_tmem + 2);
  int2* s_rows = reinterpret_cast<int2*>(s_first + kMaxGroups + 2);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int pair = (int)ptx::cluster_ctarank() >> 1, rank = (int)ptx::cluster_ctarank() & 1, base = 2 * pair;
  const int S = kSplit ? p.split : 1;
  const int cl = S == 1 ? (int)blockIdx.x >> 1 : (int)blockIdx.x / (2 * S);
  const int ncl = S == 1 ? (int)gridDim.x >> 1 : (int)gridDim.x / (2 * S);
  // stages of a sum (not kGradW): all parts', or those of this pair
  const int part_stages = (p.K + 127) / 128, all_stages = p.parts * part_stages;
  const int stage0 = S == 1 ? 0 : all_stages * pair / S;
  const int row_stages = S == 1 ? all_stages : all_stages * (pair + 1) / S - stage0;
  int joined = 0;                        // the cluster's barrier within a shared sum was passed

  if (tid == 0) {
    for (int s = 0; s < kMaxStages; ++s) {
      // kGradW: the first CTA's producer, and for each CTA the producer, or the clearing warp of a
      // group's last stage
      ptx::mbar_init(&full[s], kMode == kGradW ? 1 + kCluster : 1);
      ptx::mbar_init(&empty[s], 1);
      ptx::mbar_init(&tail[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(&acc_full[a], 1);
      ptx::mbar_init(&acc_empty[a], kCluster * kEpiWarps);
    }
    ptx::mbar_init(drain, 1);
    ptx::mbar_init(held, 1);
    for (int i = 0; i < kQueue; ++i) {
      ptx::mbar_init(&d_full[i], 1);
      // the producer, the epilogue's warps, and the MMAs' (first CTA) and the clearing warp
      ptx::mbar_init(&d_empty[i], 1 + kEpiWarps + (rank == 0 ? 1 : 0) + (kMode == kGradW ? 1 : 0));
    }
    ptx::fence_mbarrier_init();
    *s_abort = 0;
    if (kMode != kGradW && (kAmn ? p.M : p.K) >= 128) ptx::prefetch_tensormap(&tm.a[0]);
    if (kMode != kGradW && p.K >= 128) ptx::prefetch_tensormap(&tm.b[0]);
  }
  if (warp == 1) {
    ptx::tmem_alloc2(s_tmem, 512);
    ptx::tmem_relinquish2();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_arrive();   // the barriers of both CTAs are set up
  ptx::cluster_wait();
  ptx::tc_fence_after();
  const uint32_t tmem_base = *s_tmem;
  if (!early<kMode>() && !(kMode == kGradW && p.after_x)) {
    pdl_wait();
    pdl_launch_dependents();
  }

  auto wait_for = [&](auto try_wait, int value) -> bool {
    if (try_wait()) return true;
    const uint64_t t0 = ptx::globaltimer_ns();
    const uint64_t limit = kWaitNs + (kMode == kGradW ? (uint64_t)p.R / 64 * kStageNs : 0);
    for (uint32_t i = 1;; ++i) {
      if (try_wait()) return true;
      if ((i & 63u) == 0u) {
        if (*s_abort) return false;
        if (ptx::globaltimer_ns() - t0 > limit) {
          record_error(&ffn_fault, kErrTimeout, kAtFfn, value);
          *s_abort = 1;
          return false;
        }
      }
    }
  };
  auto wait = [&](uint64_t* bar, uint32_t parity, int value) -> bool {
    return wait_for([&] { return ptx::mbar_try_wait(bar, parity); }, value);
  };
  // The pair's i-th unit for a thread, or (warp_wide) a warp. A wait that failed gives an end.
  auto unit_at = [&](int i, bool warp_wide) -> Unit {
    const int q = i % kQueue;
    bool got = wait(&d_full[q], (uint32_t)(i / kQueue) & 1u, i);
    if (warp_wide) got = __all_sync(0xffffffffu, got);
    Unit un{0, 0, -1, 0, 0, 0};
    if (got) {
      const int4 v = *reinterpret_cast<const int4*>(s_unit + 4 * q);
      un.row = v.x;
      un.rows = v.y;
      un.e = v.z;
      un.part = v.w >> 16;
      un.m = (v.w >> 8) & 0xff;
      un.n = v.w & 0xff;
    }
    if (warp_wide) __syncwarp();
    if (got && (!warp_wide || lane == 0)) ptx::mbar_arrive(&d_empty[q]);
    return un;
  };
  // columns of D: N of the unit's MMAs, a multiple of 32; half of them are each CTA's
  auto rows_m = [&](const Unit& un) -> int { return kMode == kGradW && un.part == 2 ? p.M_down : p.M; };
  auto cols_n = [&](const Unit& un) -> int { return un.part == 2 ? p.N_down : p.N; };   // kGradW
  auto columns = [&](const Unit& un) -> int {
    if (kMode == kGradW) return min(round_up(cols_n(un) - un.n * kNMax, 32), kNMax);
    return round_up(un.rows, 32);
  };
  // stages of a unit: 64 rows (kGradW), or 128 of K of each part
  auto stages_of = [&](const Unit& un) -> int {
    if (kMode == kGradW) return (un.rows + 63) / 64;
    return row_stages;
  };
  // the lowest box of rows that holds a CTA's half of the columns
  auto level_of = [&](int half, int* rows) -> int {
    int lv = 0;
    *rows = p.level_rows[0];
#pragma unroll
    for (int l = 1; l < kLevels; ++l)
      if (p.level_rows[l] >= half) { lv = l; *rows = p.level_rows[l]; }
    return lv;
  };

  if (warp == 0) {
    // ================= TMA producer: this CTA's rows of A and its half of B's
    if (lane == 0) {
      const uint64_t once = ptx::policy_evict_first(), again = ptx::policy_evict_normal();
      const uint32_t full0 = ptx::peer_smem(full, base);
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      const int part0 = stage0 >= part_stages ? 1 : 0, first_k = (stage0 - part0 * part_stages) * 128;
      if (kMode == kGradW && p.after_x) {
        pdl_wait();
        pdl_launch_dependents();
      }
      for (int i = 0; ok; ++i) {
        const Unit un = unit_at(i, false);
        if (un.e < 0) break;
        const int stages = stages_of(un), half = columns(un) / 2;
        const int m0 = kMode == kUp ? un.m * 128 + rank * 64 : un.m * 256 + rank * 128;
        int rows;
        const int lv = level_of(half, &rows);
        const int b_row = un.row + rank * half;
        // a stage's weights: 128 of K from k on
        auto load_a = [&](uint8_t* a, uint32_t bar, int part, int k) {
          if constexpr (kMode == kUp || kMode == kDown) {
            // K-major. Whole: eight rows over both 64 of K, then the next eight
            const int row8 = (un.e * p.M + m0) >> 3;
            if (k + 128 <= p.K) {
              ptx::tma_load_4d_pair(a, &tm.a[0], bar, 0, 0, k >> 6, row8, once);
              if (kMode == kUp) ptx::tma_load_4d_pair(a + kTileABytes, &tm.a[1], bar, 0, 0, k >> 6, row8, once);
            } else {
              for (int s = 0; s < 2 && k + 64 * s < p.K; ++s) {
                uint8_t* as = a + s * kTileABytes;
                ptx::tma_load_3d_pair(as, &tm.a_cut[0], bar, k + 64 * s, m0, un.e, once);
                if (kMode == kUp) ptx::tma_load_3d_pair(as + 8192, &tm.a_cut[1], bar, k + 64 * s, m0, un.e, once);
              }
            }
          } else {
            // MN-major: 128 rows of K of 64 columns, then of the next 64
            if (m0 + 128 <= p.M) {
              ptx::tma_load_4d_pair(a, &tm.a[part], bar, 0, k, m0 >> 6, un.e, once);
            } else {
              ptx::tma_load_3d_pair(a, &tm.a_cut[part], bar, m0, k, un.e, once);
              ptx::tma_load_3d_pair(a + kTileABytes, &tm.a_cut[part], bar, m0 + 64, k, un.e, once);
            }
          }
        };
        auto stage_tx = [&](int k) -> uint32_t {
          const uint32_t subs = k + 64 < p.K ? 2 : 1;
          return subs * (uint32_t)rows * 128u + (kAmn ? 2u : subs) * kTileABytes;
        };
        int part = part0, k0 = first_k;
        auto next = [&](int& part_, int& k) {
          k += 128;
          if (k >= p.K) { k = 0; ++part_; }
        };
        int ahead = 0;                 // stages whose weights were asked for before the wait
        if (early<kMode>() && i == 0) {
          int part_ = part0, k = first_k;
          for (; ahead < stages && ahead < p.stages; ++ahead, next(part_, k)) {
            if (rank == 0) ptx::mbar_arrive_expect_tx(&full[ahead], kCluster * stage_tx(k));
            load_a(smem + (uint32_t)ahead * stage_bytes, full0 + 8u * (uint32_t)ahead, part_, k);
          }
          pdl_wait();
          pdl_launch_dependents();
        }
        for (int c = 0; c < stages; ++c) {
          const bool a_there = ahead > 0;
          if (a_there) --ahead;
          if (stage % kPer == 0 && !a_there && !wait(&empty[stage / kPer], phase ^ 1u, i)) {
            ok = false;
            break;
          }
          uint8_t* a = smem + (uint32_t)stage * stage_bytes;
          uint8_t* b = a + kSub * kTileABytes;
          const uint32_t bar = full0 + 8u * (uint32_t)stage;
          if constexpr (kMode == kGradW) {
            // the last stage, if it is to be cleared, completes on this CTA's own barrier, and the
            // clearing warp arrives for this CTA
            const int r = un.row + c * 64, n0 = un.n * kNMax + rank * half;
            const int b_boxes = (half + 63) / 64;
            const uint32_t bytes = kTileABytes + (uint32_t)b_boxes * 8192u;
            const bool ends = (un.rows & 15) != 0 && c == stages - 1;
            const uint32_t to = ends ? ptx::peer_smem(&tail[stage], base + rank) : bar;
            if (ends) ptx::mbar_arrive_expect_tx(&tail[stage], bytes);
            if (rank == 0) ptx::mbar_arrive_expect_tx(&full[stage], ends ? 0 : kCluster * bytes);
            if (!ends) ptx::mbar_arrive_pair(bar);
            const int job = un.part >> 1, part = un.part & 1;   // (down: part 0 of its own rows)
            if (m0 + 128 <= rows_m(un)) {
              ptx::tma_load_4d_pair(a, &tm.a[job], to, 0, r, m0 >> 6, part, again);
            } else {
              for (int j = 0; j < 2; ++j)
                ptx::tma_load_3d_pair(a + j * 8192, &tm.a_cut[job], to, m0 + 64 * j, part, r, again);
            }
            if (half == 128 && n0 + 128 <= cols_n(un)) {
              ptx::tma_load_4d_pair(b, &tm.b[job], to, 0, r, n0 >> 6, 0, again);
            } else {
              for (int j = 0; j < b_boxes; ++j)
                ptx::tma_load_3d_pair(b + j * 8192, &tm.b_cut[job], to, n0 + 64 * j, 0, r, again);
            }
          } else {
            if (!a_there) {
              if (rank == 0) ptx::mbar_arrive_expect_tx(&full[stage], kCluster * stage_tx(k0));
              load_a(a, bar, part, k0);
            }
            if (k0 + 128 <= p.K) {
              ptx::tma_load_4d_pair(b, &tm.b[lv], bar, 0, b_row, k0 >> 6, part, again);
            } else {
              for (int s = 0; s < 2 && k0 + 64 * s < p.K; ++s)
                ptx::tma_load_3d_pair(b + s * rows * 128, &tm.b_cut[lv], bar, k0 + 64 * s, part, b_row, again);
            }
            next(part, k0);
          }
          if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
      }
      if (early<kMode>()) pdl_wait();   // (a pair without units ends no earlier than the launch before)
      // the issuer's last commit arrives in this CTA, too
      wait(drain, 0, -1);
    }
  } else if (warp == kPlanWarp) {
    // ================= units: counted per group, then decoded ahead of their use
    const int per_group = p.per_group;   // kGradW
    int units = p.n_groups * per_group;
    // (several groups: n_max is kNMax, or no less than the call's rows. A division by a variable for each
    // of them would be half a microsecond)
    auto tiles_of = [&](int cnt) -> int { return p.n_max == kNMax ? (cnt + kNMax - 1) / kNMax : cnt > 0 ? 1 : 0; };
    int one = 0;                     // tiles of rows of the only group
    if (kMode != kGradW) {
      // a lane counts 16 groups in a row (their offsets are all asked for at once)
      constexpr int kOwn = kMaxGroups / 32;
      int own[kOwn], sum = 0;
#pragma unroll
      for (int j = 0; j < kOwn; ++j) {
        const int g = lane * kOwn + j;
        int64_t row0 = 0;
        int cnt = 0;
        if (g < p.n_groups) {
          group_rows(p, g, &row0, &cnt);
          if (group_expert(p, g) < 0) cnt = 0;
          s_rows[g] = make_int2((int)row0, cnt);
        }
        if (p.n_groups > 1) {
          own[j] = tiles_of(cnt) * p.m_tiles;
        } else {
          if (j == 0) one = (cnt + p.n_max - 1) / p.n_max;
          own[j] = j == 0 ? one * p.m_tiles : 0;
        }
        sum += own[j];
      }
      int before = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += v;
      }
      units = __shfl_sync(0xffffffffu, before, 31);
      before -= sum;
#pragma unroll
      for (int j = 0; j < kOwn; ++j) {
        s_first[lane * kOwn + j] = before;
        before += own[j];
      }
      __syncwarp();
    }
    if (lane == 0) {
      int64_t row_ahead = 0;         // kGradW: the rows of the unit after this one, on their way
      int cnt_ahead = 0;
      if (kMode == kGradW && cl < units) group_rows(p, cl / per_group, &row_ahead, &cnt_ahead);
      for (int i = 0;; ++i) {
        const int u = cl + i * ncl;
        int4 v = make_int4(0, 0, -1, 0);
        if (u < units) {
          if (kMode == kGradW) {
            const int g = u / per_group, local = u - g * per_group;
            const bool down = local >= p.up_units;
            const int in_job = down ? local - p.up_units : local, nt = down ? p.n_tiles_down : p.n_tiles;
            const int mt = down ? p.m_tiles_down : p.m_tiles, n = in_job % nt, mp = in_job / nt;
            int skip = 0, cnt = cnt_ahead;
            if (S > 1) {             // this pair's rows
              const int per = round_up((cnt + S - 1) / S, 64);
              skip = min(pair * per, cnt);
              cnt = min(per, cnt - skip);
            }
            v = make_int4((int)row_ahead + skip, cnt, g, (down ? 2 : mp / mt) << 16 | (mp % mt) << 8 | n);
            if (u + ncl < units) group_rows(p, (u + ncl) / per_group, &row_ahead, &cnt_ahead);
          } else {
            int lo = 0, hi = p.n_groups - 1;
            while (lo < hi) {
              const int mid = (lo + hi + 1) >> 1;
              if (s_first[mid] <= u) lo = mid; else hi = mid - 1;
            }
            const int row0 = s_rows[lo].x, cnt = s_rows[lo].y, local = u - s_first[lo];
            // the tiles of a group next to one another share its weights; they are of one size
            const int nt = p.n_groups > 1 ? tiles_of(cnt) : one;
            const int m = local / nt, n = local - m * nt;
            const int tile = round_up((cnt + nt - 1) / nt, 32);
            v = make_int4(row0 + n * tile, min(tile, cnt - n * tile),
                          p.expert_ids != nullptr ? group_expert(p, lo) : lo, m << 8);
          }
        }
        const int q = i % kQueue;
        if (i >= kQueue && !wait(&d_empty[q], ((uint32_t)(i / kQueue) & 1u) ^ 1u, i)) break;
        *reinterpret_cast<int4*>(s_unit + 4 * q) = v;
        ptx::mbar_arrive(&d_full[q]);
        if (v.z < 0) break;
      }
    }
  } else if (warp == 1) {
    // ================= MMA issuer: the first CTA's, for both
    if (rank == 0 && lane == 0) {
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      const uint32_t ring = ptx::smem_addr(smem);
      bool in = false;        // the next stage was seen full: tested while MMAs are queued, as the
                              // pipe takes one or two ahead and this thread's pauses are its own
      bool ok = p.hold == 0 || wait(held, 0, -2);
      for (int i = 0; ok; ++i) {
        const Unit un = unit_at(i, false);
        if (un.e < 0) break;
        const int stages = stages_of(un), n = columns(un);
        if (stages == 0) continue;
        const uint32_t idesc = ptx::idesc_16bit(256, (uint32_t)n, !kHalf, kAmn, kBmn);
        const uint32_t d0 = tmem_base + (uint32_t)acc * kNMax;
        const int K = kMode == kGradW ? un.rows : p.K;
        int rows;
        level_of(n / 2, &rows);
        ok = wait(&acc_empty[acc], acc_phase ^ 1u, i);
        ptx::tc_fence_after();
        int left = K;                           // of the part's sum
        if (kMode != kGradW) left -= (stage0 >= part_stages ? stage0 - part_stages : stage0) * 128;
        for (int c = 0; ok && c < stages; ++c) {
          ok = in || wait(&full[stage], phase, i);
          if (!ok) break;
          // (the clearing warps' words, those of the other CTA as well)
          if (kMode == kGradW && left < 64 && (left & 15) != 0) ptx::fence_acquire_cluster_smem();
          ptx::tc_fence_after();
          const uint32_t a = ring + (uint32_t)stage * stage_bytes, b = a + kSub * kTileABytes;
          const bool last = stage % kPer == kPer - 1;
          uint64_t* const done = &empty[stage / kPer];
          if (++stage == p.stages) { stage = 0; phase ^= 1u; }
          const bool whole = left >= 128;       // (kUp, kDown: how the weights lie)
#pragma unroll
          for (int s = 0; s < kSub; ++s) {
            if (s > 0 && left <= 64 * s) break;
            const uint32_t as = a + (kMode == kGradW ? 0u : kAmn ? s * 8192u : s * (whole ? 1024u : kTileABytes));
            const uint32_t bs = b + s * (uint32_t)rows * 128u;
            const int l = left - 64 * s;
            auto mma = [&](int kk) {
              const uint64_t ad = kAmn ? ptx::sdesc_mn_sw128(as + kk * 2048, kMode == kGradW ? 8192 : 16384)
                                       : ptx::sdesc_k_sw128(as + kk * 32, whole ? 2048u : 1024u);
              const uint64_t bd = kBmn ? ptx::sdesc_mn_sw128(bs + kk * 2048, 8192) : ptx::sdesc_k_sw128(bs + kk * 32);
              ptx::mma_bf16_pair(d0, ad, bd, idesc, (c > 0 || s > 0 || kk > 0) ? 1u : 0u);
            };
            mma(0);
            if (l > 16) mma(1);
            if (s == 0) in = ptx::mbar_test_wait(&full[stage], phase);
            if (l > 32) mma(2);
            if (l > 48) mma(3);
          }
          left -= 64 * kSub;
          if (left <= 0) left = K;
          if (last) ptx::mma_commit_pair(done, base);
        }
        if (!ok) break;
        ptx::mma_commit_pair(&acc_full[acc], base);
        acc ^= 1;
        if (acc == 0) acc_phase ^= 1u;
      }
      // no MMA is running when tensor memory is released
      ptx::mma_commit_pair(drain, base);
      const uint64_t t0 = ptx::globaltimer_ns();
      while (!ptx::mbar_try_wait(drain, 0) && ptx::globaltimer_ns() - t0 < kWaitNs) {
      }
    }
  } else if (warp == kFixWarp) {
    if constexpr (kMode == kGradW) {
      // ================= zeros in the rows of K behind the group's last row, up to the 16 of its last
      // MMA, in both operands of this CTA (a row of K is 128 bytes of each block of 64 columns; the
      // swizzle stays within it)
      // (Fences that also order global memory cost a microsecond a group: the gradient of 256 experts'
      // 2048 x 512 from 230 rows each took 190 us with them, 141 without, as from 240 rows, which need
      // no clearing.)
      const uint32_t full0 = ptx::peer_smem(full, base);
      int stage = 0;
      uint32_t phases = 0;      // of tail, a bit each
      bool ok = true;
      for (int i = 0; ok; ++i) {
        const Unit un = unit_at(i, true);
        if (un.e < 0) break;
        const int stages = stages_of(un), blocks = 2 + (columns(un) / 2 + 63) / 64;
        const int at = (stage + stages - 1) % p.stages;
        stage = (stage + stages) % p.stages;
        if ((un.rows & 15) == 0) continue;
        ok = __all_sync(0xffffffffu, wait(&tail[at], (phases >> at) & 1u, i));
        if (!ok) break;
        const int from = un.rows & 63, per_block = (16 - (from & 15)) * 8;
        uint8_t* a = smem + (uint32_t)at * stage_bytes + from * 128;
        for (int j = lane; j < blocks * per_block; j += 32) {
          const int blk = j / per_block, o = j - blk * per_block;
          *reinterpret_cast<uint4*>(a + blk * 8192 + o * 16) = make_uint4(0, 0, 0, 0);
        }
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive_cluster_smem(full0 + 8u * (uint32_t)at);
        phases ^= 1u << at;
      }
    } else if ((kMode == kDown || kMode == kGradX) && p.zero_rest) {
      // ================= zeros in the rows in no group, 64 rows at a time
      uint16_t* out = static_cast<uint16_t*>(p.out);
      for (int64_t r0 = (int64_t)blockIdx.x * 64; r0 < p.R; r0 += (int64_t)gridDim.x * 64) {
        uint64_t owned = 0;
        for (int g = lane; g < p.n_groups; g += 32) {
          int64_t lo;
          int cnt;
          group_rows(p, g, &lo, &cnt);
          const int64_t hi = lo + cnt;
          if (cnt == 0 || lo >= r0 + 64 || hi <= r0 || group_expert(p, g) < 0) continue;
          const int b = lo > r0 ? (int)(lo - r0) : 0, e = hi < r0 + 64 ? (int)(hi - r0) : 64;
          owned |= (~0ull >> (64 - (e - b))) << b;
        }
        owned = (uint64_t)__reduce_or_sync(0xffffffffu, (uint32_t)(owned >> 32)) << 32 |
                __reduce_or_sync(0xffffffffu, (uint32_t)owned);
        for (int j = 0; j < 64 && r0 + j < p.R; ++j) {
          if (owned >> j & 1) continue;
          uint4* row = reinterpret_cast<uint4*>(out + (r0 + j) * p.ldo);
          for (int c = lane; c < p.M / 8; c += 32) row[c] = make_uint4(0, 0, 0, 0);
        }
      }
    }
  } else {
    // ================= epilogue: warps from 2 on, TMEM lanes 32 * (warp % 4) ..; groups of four
    // warps take alternate slices of the columns
    const int q = warp & 3, cg = (warp - 2) >> 2;
    const uint32_t lane_off = (uint32_t)(q * 32) << 16;
    const uint32_t acc_empty0 = ptx::peer_smem(acc_empty, base);
    int acc = 0;
    uint32_t acc_phase = 0;
    for (int i = 0;; ++i) {
      const Unit un = unit_at(i, true);
      const bool sums = kMode != kGradW || un.rows > 0;
      // Rows of D become words of a token's row by stmatrix: 16 columns' (tokens') 64 bytes each in shared memory,
      // which four lanes store, 16 bytes each.
      const int feature = un.m * 256 + rank * 128 + q * 32 + 8 * (lane & 3);     // (not kUp)
      uint8_t* mine = s_epi + (warp - 2) * 16 * kPitch;
      const uint32_t blocks = ptx::smem_addr(mine) + (8 * (lane >> 4) + (lane & 7)) * kPitch + (lane & 8) * 2;
      uint4* const words = reinterpret_cast<uint4*>(mine + (lane >> 2) * kPitch + (lane & 3) * 16);
      constexpr int kEight = 8 * kPitch / 16;       // to the words eight tokens on
      // kGradH: g and u of the next slice of columns, asked for before this one's sums are there (the
      // backward pass of 59000 rows over 256 experts of 2048 x 512 took 833 us when they were asked for in turn, 789 so)
      uint4 gw[2], uw[2];
      auto ask_pre = [&](int c0) {
        const uint16_t* pre = static_cast<const uint16_t*>(p.pre) + (int64_t)un.row * 2 * p.I + feature;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int t = c0 + 8 * s + (lane >> 2);
          const bool in = t < un.rows && feature < p.I;
          const uint16_t* from = pre + (int64_t)t * 2 * p.I;
          gw[s] = in ? __ldg(reinterpret_cast<const uint4*>(from)) : make_uint4(0, 0, 0, 0);
          uw[s] = in ? __ldg(reinterpret_cast<const uint4*>(from + p.I)) : make_uint4(0, 0, 0, 0);
        }
      };
      if (kMode == kGradH && un.e >= 0 && S == 1) ask_pre(16 * cg);
      // (a warp whose wait failed leaves with the others)
      if (!epilogue_all<kEpiWarps * 32>(un.e >= 0 && (!sums || wait(&acc_full[acc], acc_phase, i)))) break;
      ptx::tc_fence_after();
      const uint32_t tbase = tmem_base + lane_off + (uint32_t)acc * kNMax;
      // 16 columns as 8 x 8 blocks (kGradW: a lane's row)
      auto load16 = [&](int c0, float (&v)[16]) {
        if constexpr (kMode != kGradW) ptx::tmem_ld16_blocks(tbase + c0, v);
        else ptx::tmem_ld16(tbase + c0, v);
        ptx::tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 16; ++j) asm volatile("" : "+f"(v[j]));
      };
      // this pair's columns: all, or a part of them
      int lo = 0, hi = kMode == kGradW ? columns(un) : un.rows, slice = 0;
      if (S > 1) {
        // The other pairs' columns, as [16 columns][4 of a lane's values][lane], in the place of the ring (its
        // MMAs are done).
        const int n = columns(un);
        slice = round_up((n + S - 1) / S, kMode == kGradW ? 64 : 16);
        for (int c0 = 16 * cg; c0 < n; c0 += kStep) {
          if (c0 >= pair * slice && c0 < (pair + 1) * slice) continue;
          float v[16];
          if (sums) load16(c0, v);
          float4* to = reinterpret_cast<float4*>(smem) + c0 / 4 * 128 + q * 32 + lane;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            to[j * 128] = sums ? make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3])
                               : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        ptx::cluster_arrive();
        ptx::cluster_wait();
        joined = 1;
        lo = min(pair * slice, hi);
        hi = min(lo + slice, hi);
        if (kMode == kGradH) ask_pre(lo + 16 * cg);
      }
      const int nvalid = hi;
      // 16 columns of the sum
      auto sum16 = [&](int c0, float (&v)[16]) {
        if (S == 1 || sums) {
          load16(c0, v);
        } else {
#pragma unroll
          for (int j = 0; j < 16; ++j) v[j] = 0.f;
        }
        if (S > 1) {
          const float4* mine = reinterpret_cast<const float4*>(smem) + c0 / 4 * 128 + q * 32 + lane;
          float t[16];
          for (int s = 0; s < S; ++s) {
            float4 f[4];
            const uint32_t from = ptx::peer_smem(mine, 2 * s + rank);
#pragma unroll
            for (int j = 0; j < 4; ++j)
              f[j] = s == pair ? make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3])
                               : ptx::ld_cluster_f32x4(from + j * 2048);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              t[4 * j] = s == 0 ? f[j].x : t[4 * j] + f[j].x;
              t[4 * j + 1] = s == 0 ? f[j].y : t[4 * j + 1] + f[j].y;
              t[4 * j + 2] = s == 0 ? f[j].z : t[4 * j + 2] + f[j].z;
              t[4 * j + 3] = s == 0 ? f[j].w : t[4 * j + 3] + f[j].w;
            }
          }
#pragma unroll
          for (int j = 0; j < 16; ++j) v[j] = t[j];
        }
      };
      if constexpr (kMode == kUp) {
        // TMEM lanes 0-63: g of 64 i, lanes 64-127: u of the same. Of 16 columns the warps of g
        // keep the first eight and give the others to the warps of u, through shared memory.
        const bool is_gate = q < 2;
        const int f = un.m * 128 + rank * 64 + (q & 1) * 32 + 8 * (lane & 3);
        float4* box = reinterpret_cast<float4*>(s_epi) + (cg * 2 + (q & 1)) * 128;
        const int bar_id = 2 + cg * 2 + (q & 1);
        uint8_t* own = s_epi + kEpiWarps * 1024 + (warp - 2) * 8 * kPitch;
        const uint32_t put = ptx::smem_addr(own) + (lane & 7) * kPitch + (lane >> 3) * 16;
        const uint4* take_words = reinterpret_cast<const uint4*>(own + (lane >> 2) * kPitch + (lane & 3) * 16);
        const int64_t row = un.row + (is_gate ? 0 : 8) + (lane >> 2);      // (and c0)
        uint16_t* h = static_cast<uint16_t*>(p.out) + row * p.I + f;
        uint16_t* pre = static_cast<uint16_t*>(p.pre) + row * 2 * p.I + f;
        for (int c0 = lo + 16 * cg; c0 < nvalid; c0 += kStep) {
          float v[16];
          sum16(c0, v);
          // [from gate / from up][two float4][lane]
          float4* give = box + (is_gate ? 0 : 64) + lane;
          const float4* take = box + (is_gate ? 64 : 0) + lane;
#pragma unroll
          for (int j = 0; j < 2; ++j)
            give[32 * j] = is_gate ? make_float4(v[8 * j + 4], v[8 * j + 5], v[8 * j + 6], v[8 * j + 7])
                                   : make_float4(v[8 * j], v[8 * j + 1], v[8 * j + 2], v[8 * j + 3]);
          ptx::named_bar_sync(bar_id, 64);
          const float4 o0 = take[0], o1 = take[32];
          ptx::named_bar_sync(bar_id, 64);       // (the words have been read)
          const float o[8] = {o0.x, o0.y, o0.z, o0.w, o1.x, o1.y, o1.z, o1.w};
          float g[8], u[8], hv[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int at = 8 * (j >> 2) + (j & 3);
            g[j] = is_gate ? v[at] : o[j];
            u[j] = is_gate ? o[j] : v[at + 4];
            hv[j] = g[j];
          }
          silu_all(hv);
#pragma unroll
          for (int j = 0; j < 8; ++j) hv[j] *= u[j];
          const bool in = c0 + (is_gate ? 0 : 8) + (lane >> 2) < nvalid && f < p.I;
          auto store = [&](const float (&w)[8], uint16_t* to, auto pack) {
            __syncwarp();                        // (the words before have been read)
            ptx::stmatrix4_trans(put, pack(w[0], w[1]), pack(w[2], w[3]), pack(w[4], w[5]), pack(w[6], w[7]));
            __syncwarp();
            const uint4 words8 = *take_words;
            if (in) *reinterpret_cast<uint4*>(to) = words8;
          };
          store(hv, h + (int64_t)c0 * p.I, pack2<kHalf>);
          if (p.pre != nullptr) {
            store(g, pre + (int64_t)c0 * 2 * p.I, pack2_finite<kHalf>);
            store(u, pre + (int64_t)c0 * 2 * p.I + p.I, pack2_finite<kHalf>);
          }
        }
      } else if constexpr (kMode == kGradH) {
        uint16_t* dpre = static_cast<uint16_t*>(p.out) + ((int64_t)un.row + (lane >> 2)) * 2 * p.I + feature;
        for (int c0 = lo + 16 * cg; c0 < nvalid; c0 += kStep) {
          uint32_t g2[2][4], u2[2][4];           // [h][2 c + r] of the blocks
          auto spread = [&](const uint4 (&w)[2], uint32_t (&o)[2][4]) {
            __syncwarp();                        // (the words before have been read)
            words[0] = w[0];
            words[kEight] = w[1];
            __syncwarp();
            ptx::ldmatrix4_trans(blocks, o[0]);
            ptx::ldmatrix4_trans(blocks + 32, o[1]);
          };
          spread(gw, g2);
          spread(uw, u2);
          if (c0 + kStep < nvalid) ask_pre(c0 + kStep);
          float v[16];
          sum16(c0, v);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float2 gj = unpack2<kHalf>(g2[h][j]), uj = unpack2<kHalf>(u2[h][j]);
              const float g[2] = {gj.x, gj.y}, u[2] = {uj.x, uj.y};
              float dg[2], du[2];
#pragma unroll
              for (int b = 0; b < 2; ++b) {
                const float dh = v[8 * h + 2 * j + b], s = __fdividef(1.f, 1.f + __expf(-g[b]));
                dg[b] = dh * u[b] * s * (1.f + g[b] * (1.f - s));
                du[b] = dh * g[b] * s;
              }
              g2[h][j] = pack2<kHalf>(dg[0], dg[1]);
              u2[h][j] = pack2<kHalf>(du[0], du[1]);
            }
          auto store = [&](const uint32_t (&w)[2][4], uint16_t* to) {
            __syncwarp();
#pragma unroll
            for (int h = 0; h < 2; ++h) ptx::stmatrix4_trans(blocks + 32 * h, w[h][0], w[h][1], w[h][2], w[h][3]);
            __syncwarp();
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              const uint4 word = words[s * kEight];
              if (c0 + 8 * s + (lane >> 2) < nvalid && feature < p.I)
                *reinterpret_cast<uint4*>(to + (int64_t)(c0 + 8 * s) * 2 * p.I) = word;
            }
          };
          store(g2, dpre);
          store(u2, dpre + p.I);
        }
      } else if constexpr (kMode == kGradW) {
        // 64 columns of this warp's 32 rows at a time: through shared memory (128-byte swizzle), one
        // bulk store each. What lies outside of the matrix is cut by its map.
        const int row = un.m * 256 + rank * 128 + q * 32;
        uint8_t* mine = s_epi + (warp - 2) * 4096;
        const CUtensorMap* out = &tm.out[un.part];
        const int M = rows_m(un), N = cols_n(un);
        for (int c0 = lo + 64 * cg; c0 < nvalid; c0 += 128) {
          float v[2][32];
          if (S > 1) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              float t[16];
              sum16(c0 + 16 * j, t);
#pragma unroll
              for (int i16 = 0; i16 < 16; ++i16) v[j >> 1][16 * (j & 1) + i16] = t[i16];
            }
          } else if (sums) {
            ptx::tmem_ld32(tbase + c0, v[0]);
            ptx::tmem_ld32(tbase + c0 + 32, v[1]);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) asm volatile("" : "+f"(v[0][j]), "+f"(v[1][j]));
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[0][j] = v[1][j] = 0.f;
          }
          if (lane == 0) ptx::bulk_commit_wait_read();   // the store before has read its words
          __syncwarp();
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float* f = &v[j >> 2][8 * (j & 3)];
            *reinterpret_cast<uint4*>(mine + lane * 128 + ((j ^ (lane & 7)) * 16)) =
                make_uint4(pack2<kHalf>(f[0], f[1]), pack2<kHalf>(f[2], f[3]),
                           pack2<kHalf>(f[4], f[5]), pack2<kHalf>(f[6], f[7]));
          }
          ptx::fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0 && row < M && un.n * kNMax + c0 < N)
            ptx::tma_store_3d(out, mine, un.n * kNMax + c0, row, un.e);
        }
      } else {
        uint16_t* out = static_cast<uint16_t*>(p.out) + (int64_t)(un.row + (lane >> 2)) * p.ldo + feature;
        if (un.m * 256 + rank * 128 + q * 32 < p.M) {   // (the same for the warp)
          for (int c0 = lo + 16 * cg; c0 < nvalid; c0 += kStep) {
            float v[16];
            sum16(c0, v);
            __syncwarp();                               // (the words before have been read)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              ptx::stmatrix4_trans(blocks + 32 * h, pack2<kHalf>(v[8 * h], v[8 * h + 1]),
                                   pack2<kHalf>(v[8 * h + 2], v[8 * h + 3]), pack2<kHalf>(v[8 * h + 4], v[8 * h + 5]),
                                   pack2<kHalf>(v[8 * h + 6], v[8 * h + 7]));
            __syncwarp();
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              const uint4 w = words[s * kEight];
              if (c0 + 8 * s + (lane >> 2) < nvalid && feature < p.M)
                *reinterpret_cast<uint4*>(out + (c0 + 8 * s) * p.ldo) = w;
            }
          }
        }
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (sums) {
        if (lane == 0) ptx::mbar_arrive_pair(acc_empty0 + 8u * (uint32_t)acc);
        acc ^= 1;
        if (acc == 0) acc_phase ^= 1u;
      }
    }
    if (kMode == kGradW && lane == 0) ptx::bulk_commit_wait_all();
  }

  // (the barrier of a shared sum, for the warps that have no part in it, and where a wait failed)
  __syncwarp();
  if (S > 1 && joined == 0) {
    ptx::cluster_arrive();
    ptx::cluster_wait();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  // neither CTA leaves while the other may still signal its barriers or read its tiles
  ptx::cluster_arrive();
  ptx::cluster_wait();
  if (warp == 1) {
    __syncwarp();
    ptx::tmem_dealloc2(tmem_base, 512);
  }
  // After a wait that failed, copies into this CTA's shared memory may not have been waited for: it
  // stays until they have long landed.
  if (*s_abort) {
    const uint64_t t0 = ptx::globaltimer_ns();
    while (ptx::globaltimer_ns() - t0 < kWaitNs / 10) __nanosleep(1000);
  }
}

// ------------------------------------------------------------------ host side
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                  const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &ptr, 12000, cudaEnableDefault,
                                         &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeTiledFn>(ptr);
  });
  return fn;
}

// A map of 16-bit elements with n.size() dimensions (the fastest first), strides in elements from the second
// on, in boxes of 64 x box.
bool make_map(CUtensorMap* m, bool half, const void* base, std::initializer_list<uint64_t> n,
              std::initializer_list<uint64_t> ld, std::initializer_list<uint32_t> box) {
  EncodeTiledFn enc = encode_fn();
  if (enc == nullptr) return false;
  cuuint64_t dims[4], strides[3];
  cuuint32_t b[4] = {64, 1, 1, 1};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  std::copy(n.begin(), n.end(), dims);
  std::transform(ld.begin(), ld.end(), strides, [](uint64_t v) { return 2 * v; });
  std::copy(box.begin(), box.end(), b + 1);
  auto encode = [&] {
    return enc(m, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
               (cuuint32_t)n.size(), const_cast<void*>(base), dims, strides, b, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  if (encode()) return true;
  // The driver's call wants a context; a thread that has made no runtime call that needs one (the
  // thread in which autograd runs a backward pass) has none yet: setting its device makes it current.
  int dev = 0;
  return cudaGetDevice(&dev) == cudaSuccess && cudaSetDevice(dev) == cudaSuccess && encode();
}

struct Rows {          // [R][parts][K], rows ld apart
  const void* p;
  int64_t ld;
  int parts, K;
};

cudaError_t smem_limit(int* limit) {
  static std::atomic<int> known[32];
  int dev = 0, v = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  v = dev < 32 ? known[dev].load(std::memory_order_relaxed) : 0;
  if (v == 0) {
    e = cudaDeviceGetAttribute(&v, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev);
    if (e == cudaSuccess && dev < 32) known[dev].store(v, std::memory_order_relaxed);
  }
  *limit = v;
  return e;
}

template <int kMode, bool kHalf, bool kSplit>
cudaError_t raise_limit(int limit) {
  static std::atomic<uint32_t> done;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  const uint32_t bit = dev < 32 ? 1u << dev : 0u;
  if (e != cudaSuccess || (done.load(std::memory_order_relaxed) & bit) != 0u) return e;
  e = cudaFuncSetAttribute(ffn_products_kernel<kMode, kHalf, kSplit>,
                           cudaFuncAttributeMaxDynamicSharedMemorySize, limit);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

Params base_params(const FfnArgs& a) {
  Params p{};
  p.offsets = a.offsets;
  p.expert_ids = a.expert_ids;
  p.n_groups = a.n_groups;
  p.n_experts = a.n_experts;
  p.R = a.R;
  p.I = a.I;
  p.parts = 1;
  p.split = 1;
  p.hold = a.hold;
  p.zero_rest = a.zero_rest ? 1 : 0;
  return p;
}

// behind the ring: the epilogue's words, barriers, units, alignment
template <int kMode>
constexpr size_t fixed_smem() {
  return 1024 + epi_bytes<kMode>() + 8 * (3 * kMaxStages + 6 + 2 * kQueue) + 16 * kQueue + 8 +
         (kMode == kGradW ? 0 : 4 * (kMaxGroups + 2) + 8 * kMaxGroups);
}

// The rest of the launch: stages, grid. `units`: at most so many.
template <int kMode, bool kHalf, bool kSplit>
cudaError_t launch_form(Maps& m, Params& p, int64_t units, cudaStream_t s) {
  int limit = 0;
  cudaError_t e = smem_limit(&limit);
  if (e == cudaSuccess) e = raise_limit<kMode, kHalf, kSplit>(limit);
  if (e != cudaSuccess) return e;
  constexpr size_t fixed = fixed_smem<kMode>();
  const size_t stage = (size_t)sub_steps<kMode>() * (kTileABytes + (size_t)p.level_rows[0] * 128);
  p.stages = (int)std::min<size_t>(kMaxStages, ((size_t)limit - fixed) / stage);
  p.stages -= p.stages % per_commit<kMode>();
  if (p.stages < 2) return cudaErrorInvalidConfiguration;
  const int cluster = kCluster * p.split;      // (a cluster has one unit at most where it is more than a pair)
  const int most = p.split > 1 ? INT_MAX / cluster : device_sm_count() / kCluster;
  const int clusters = (int)std::min<int64_t>(most, std::max<int64_t>(units, 1));
  return launch_cluster(ffn_products_kernel<kMode, kHalf, kSplit>, dim3(clusters * cluster), dim3(threads<kMode>()),
                        fixed + p.stages * stage, s, cluster, true, m, p);
}
template <int kMode, bool kHalf>
cudaError_t launch(Maps& m, Params& p, int64_t units, cudaStream_t s) {
  return p.split > 1 ? launch_form<kMode, kHalf, true>(m, p, units, s)
                     : launch_form<kMode, kHalf, false>(m, p, units, s);
}

// Pairs that share a unit's sum of `stages` x 128: as many as there are for all units at once, with 512 of the sum
// or more for each. (Larger clusters do not fill the machine: 36 of four CTAs are resident at most, 23 of six,
// 15 of eight.) Us in a graph, a pair a unit / so: 64 rows of 4096 x 4096 forward 41 / 32, backward 85 / 60; 300 of
// 8192 x 1024 52 / 33, 73 / 52; 50000 of 512 x 1024 backward 449 / 330; 1024 of 512 x 512 backward 25.9 / 24.6.
int pairs_of_unit(int64_t units, int stages) {
  return units <= 15 && stages >= 16 ? 4 : units <= 23 && stages >= 12 ? 3 : units <= 36 && stages >= 8 ? 2 : 1;
}

// A product of weights with the groups' rows (all but kGradW).
template <int kMode, bool kHalf>
cudaError_t rows_product(const FfnArgs& a, const void* w0, const void* w1, const Rows& b, void* out,
                         int64_t ldo, cudaStream_t s) {
  Params p = base_params(a);
  Maps m{};
  p.parts = b.parts;
  p.K = b.K;
  p.M = kMode == kUp || kMode == kGradH ? a.I : a.d;
  const int per_m = kMode == kUp ? 128 : 256;
  p.m_tiles = (p.M + per_m - 1) / per_m;
  p.out = out;
  p.ldo = ldo;
  p.pre = kMode == kUp || kMode == kGradH ? a.pre : nullptr;
  p.n_max = (int)std::min<int64_t>(kNMax, (a.R + 31) / 32 * 32);
  // One group: the columns of a unit for which the pairs' turns take the least, when an MMA of up to
  // 160 columns takes as long as one of 160. (A dense block of 2031 rows, 2048 x 2744: gate and up in
  // 22 x 8 units of 256 are three turns of 76 pairs, and so are 22 x 10 of 224. Its backward pass takes 120 us
  // so, 127 with units of 256.)
  if (a.n_groups == 1 && a.R > kNMax) {
    const int pairs = device_sm_count() / kCluster;
    int64_t best = INT64_MAX;
    for (int n = kNMax; n >= 160; n -= 32) {
      const int64_t turns = ((a.R + n - 1) / n * p.m_tiles + pairs - 1) / pairs, cost = turns * (n + 32);
      if (cost < best) {
        best = cost;
        p.n_max = n;
      }
    }
  }
  // (only the maps that are used: each costs the host time)
  const uint64_t M = p.M, K = p.K, E = a.n_experts, R = a.R, parts = p.parts, ld = b.ld;
  const bool whole = p.K >= 128, cut = p.K % 128 != 0;
  bool ok = true;
  for (int i = 0; i < 2; ++i) {
    const void* w = i == 0 ? w0 : w1;
    if (w == nullptr) continue;
    if (a_mn<kMode>()) {       // w [E][K][M]
      if (M >= 128)
        ok = ok && make_map(&m.a[i], kHalf, w, {64, K, M / 64, E}, {M, 64, K * M}, {128, 2, 1});
      if (M % 256 != 0)
        ok = ok && make_map(&m.a_cut[i], kHalf, w, {M, K, E}, {M, K * M}, {128, 1});
    } else {                   // w [E][M][K]
      const uint32_t rows = kMode == kDown ? 128 : 64;
      if (whole)
        ok = ok && make_map(&m.a[i], kHalf, w, {64, 8, K / 64, E * M / 8}, {K, 64, 8 * K}, {8, 2, rows / 8});
      if (cut) ok = ok && make_map(&m.a_cut[i], kHalf, w, {K, M, E}, {K, M * K}, {rows, 1});
    }
  }
  int level = 0;
  for (int h = p.n_max / 2; level < kLevels; ++level) {
    if (level == 0 || h < p.level_rows[level - 1]) {
      p.level_rows[level] = h;
      if (whole)
        ok = ok && make_map(&m.b[level], kHalf, b.p, {64, R, K / 64, parts}, {ld, 64, K}, {(uint32_t)h, 2, 1});
      if (cut) ok = ok && make_map(&m.b_cut[level], kHalf, b.p, {K, parts, R}, {K, ld}, {1, (uint32_t)h});
    }
    h = std::max(16, (h / 2 + 15) / 16 * 16);
  }
  if (!ok) return cudaErrorInvalidValue;
  // as many as there can be, and if groups overlap: a cluster of several pairs takes one unit, no more
  const int64_t most = a.n_groups * ((a.R + p.n_max - 1) / p.n_max) * p.m_tiles;
  p.split = pairs_of_unit(most, p.parts * ((p.K + 127) / 128));
  const int64_t units = (a.R / p.n_max + std::min<int64_t>(a.n_groups, a.R)) * p.m_tiles;
  return launch<kMode, kHalf>(m, p, p.split > 1 ? most : units, s);
}

// Gradients of weights: sums over the groups' rows of out [R][parts][M] and in [R][N].
template <bool kHalf>
cudaError_t weights_products(const FfnArgs& a, const Rows& dpre, const Rows& x, const Rows& dy, const Rows& h,
                             cudaStream_t s) {
  Params p = base_params(a);
  Maps m{};
  p.level_rows[0] = 128;     // (a half of B: 64 rows of K of 128 columns)
  const bool up = a.dw_gate != nullptr, down = a.dw_down != nullptr;
  p.after_x = a.dx != nullptr ? 1 : 0;
  bool ok = true;
  auto maps = [&](int job, const Rows& out, const Rows& in, std::initializer_list<void*> dws) {
    const uint64_t M = out.K, N = in.K, R = a.R, parts = out.parts, lda = out.ld, ldb = in.ld;
    if (M >= 128) ok = ok && make_map(&m.a[job], kHalf, out.p, {64, R, M / 64, parts}, {lda, 64, M}, {64, 2, 1});
    if (M % 256 != 0) ok = ok && make_map(&m.a_cut[job], kHalf, out.p, {M, parts, R}, {M, lda}, {1, 64});
    if (N >= 128) ok = ok && make_map(&m.b[job], kHalf, in.p, {64, R, N / 64, 1}, {ldb, 64, N}, {64, 2, 1});
    if (N % 256 != 0) ok = ok && make_map(&m.b_cut[job], kHalf, in.p, {N, 1, R}, {N, ldb}, {1, 64});
    int i = 2 * job;
    for (void* dw : dws)
      ok = ok && make_map(&m.out[i++], kHalf, dw, {N, M, (uint64_t)a.n_experts}, {N, M * N}, {32, 1});
  };
  if (up) {
    maps(0, dpre, x, {a.dw_gate, a.dw_up});
    p.M = a.I;
    p.N = a.d;
    p.m_tiles = (p.M + 255) / 256;
    p.n_tiles = (p.N + kNMax - 1) / kNMax;
    p.up_units = 2 * p.m_tiles * p.n_tiles;
  }
  p.per_group = p.up_units;
  if (down) {
    maps(1, dy, h, {a.dw_down});
    p.M_down = a.d;
    p.N_down = a.I;
    p.m_tiles_down = (p.M_down + 255) / 256;
    p.n_tiles_down = (p.N_down + kNMax - 1) / kNMax;
    p.per_group += p.m_tiles_down * p.n_tiles_down;
  }
  if (!ok) return cudaErrorInvalidValue;
  const int64_t units = (int64_t)a.n_groups * p.per_group;
  p.split = pairs_of_unit(units, (int)(a.R / a.n_groups / 128));
  return launch<kGradW, kHalf>(m, p, units, s);
}

template <bool kHalf>
cudaError_t forward(const FfnArgs& a, cudaStream_t s) {
  cudaError_t e = rows_product<kUp, kHalf>(a, a.w_gate, a.w_up, {a.x, a.ldx, 1, a.d}, a.h, a.I, s);
  if (e == cudaSuccess)
    e = rows_product<kDown, kHalf>(a, a.w_down, nullptr, {a.h, a.I, 1, a.I}, a.y, a.ldy, s);
  return e;
}

template <bool kHalf>
cudaError_t backward(const FfnArgs& a, cudaStream_t s) {
  const Rows x{a.x, a.ldx, 1, a.d}, dy{a.dy, a.lddy, 1, a.d}, h{a.h, a.I, 1, a.I};
  const Rows dpre{a.dpre, 2 * a.I, 2, a.I};
  cudaError_t e = cudaSuccess;
  if (a.dx != nullptr || a.dw_gate != nullptr)
    e = rows_product<kGradH, kHalf>(a, a.w_down, nullptr, dy, a.dpre, 2 * a.I, s);
  if (e == cudaSuccess && a.dx != nullptr)
    e = rows_product<kGradX, kHalf>(a, a.w_gate, a.w_up, dpre, a.dx, a.lddx, s);
  if (e == cudaSuccess && (a.dw_gate != nullptr || a.dw_down != nullptr))
    e = weights_products<kHalf>(a, dpre, x, dy, h, s);
  return e;
}

}  // namespace

cudaError_t launch_expert_ffn(const FfnArgs& a, cudaStream_t s) {
  if (expert_ffn_few_ok(a)) return launch_expert_ffn_few(a, s);
  return a.dtype == DMOE_FP16 ? forward<true>(a, s) : forward<false>(a, s);
}
cudaError_t launch_expert_ffn_backward(const FfnArgs& a, cudaStream_t s) {
  return a.dtype == DMOE_FP16 ? backward<true>(a, s) : backward<false>(a, s);
}
cudaError_t ffn_fault_address(void** p) { return cudaGetSymbolAddress(p, ffn_fault); }

}  // namespace dmoe

// Products of sorted rows with their experts' 4-bit matrices, plain or gate and up with SwiGLU:
// y^T = W x^T, per unit of 128 outputs (or 64 gate and 64 up outputs) and at most 128 rows of a group.
//
// A persistent CTA per SM, in roles:
//   dequantising warps (two sets of four, in turn): a lane has a row of W. Its codes come by
//       asynchronous copies into a ring of its own, become bf16 values by one exact FMA per pair
//       and go to tensor memory: the A operand of the MMAs. Through shared memory they would take
//       four times the codes' bytes twice, and a 4 KB block of codes has 184 cycles of its share of
//       HBM's rate, in which shared memory moves 23 KB.
//   loading warps: the rows of x that the group names, 64 inputs at a time, into shared memory (B)
//   an issuing thread: tcgen05.mma, M = 128 outputs, N = the unit's rows in sixteens
//   epilogue warps: sums from tensor memory, SwiGLU, y
// Few rows: the weights' bytes are the bound, and the arithmetic on the codes is close to it (32
// pairs a row and block, 2.75 operations each). Many rows: the tensor pipe.
// Every wait has a limit of one second. One that runs out is recorded (dmoe_q4_device_error) and ends
// its role; the others' waits run out after it, and the CTA gives its tensor memory back.
#include "q4.cuh"
#include "silu.cuh"
#include "sm100_ptx.cuh"

namespace dmoe {
namespace {

constexpr int kThreads = 512;
constexpr int kEpiWarps = 4, kDeqWarps = 8, kMmaWarp = kEpiWarps + kDeqWarps;
constexpr int kLoadThreads = kThreads - 32 * (kMmaWarp + 1);   // 96
constexpr int kUnitRows = 128;             // rows of a group per unit, at most
constexpr int kASlots = 8;                 // blocks of A in tensor memory, 32 columns each
constexpr int kBRing = 128 * 1024;         // bytes of the ring of x blocks
constexpr int kBSlotsMax = 16;
constexpr int kLoadLag = 6;                // blocks of x whose copies are in flight
constexpr int kCodeSlots = 6;              // blocks of codes per set in flight
constexpr int kAcc0 = kASlots * 32;        // first column of the sums: two buffers of 128
constexpr uint64_t kWaitNs = 1000000000ull;

__device__ DevErrRecord q4_fault;               // of every call on the device
__device__ uint4 q4_zero_row[kMaxDModel / 8];   // stands in for sources that are not there

// The groups that have rows and an expert, in order, and their first units.
struct Groups {
  int n, units;
  int widest;   // rows of the widest unit, in sixteens
  int e[kMaxExperts], r0[kMaxExperts], r1[kMaxExperts], first[kMaxExperts];
};

struct Smem {
  uint8_t b[kBRing];                                       // 1024-byte aligned
  uint4 codes[2][kCodeSlots][2][128];                      // [set][slot][half][row]
  uint4 scales[2][kCodeSlots][128];                        // eight groups of a row
  float swap[2][2][64][9];                                 // ups and gates between epilogue warps
  Groups groups;
  uint64_t a_full[kASlots], a_empty[kASlots];
  uint64_t b_full[kBSlotsMax], b_empty[kBSlotsMax];
  uint64_t d_full[2], d_empty[2], drain;
  uint32_t tmem;
  int wcount[kThreads / 32];
};

__device__ __forceinline__ void find_groups(const Q4Args& a, int m_tiles, Smem& sm) {
  Groups& s = sm.groups;
  const int u = threadIdx.x, lane = u & 31, warp = u >> 5, R = (int)a.R;
  static_assert(kThreads >= kMaxExperts, "a thread per group");
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
  const int tiles = live ? (r1 - r0 + kUnitRows - 1) / kUnitRows : 0;
  const uint32_t m = __ballot_sync(0xffffffffu, live);
  int units = tiles * m_tiles, before = units;   // inclusive sum over the warp
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, before, o);
    if (lane >= o) before += v;
  }
  if (u == 0) s.widest = 16;
  if (lane == 31) {
    sm.wcount[warp] = before;
    if (warp < kMaxExperts / 32) s.first[warp] = __popc(m);   // (for the moment)
  }
  __syncthreads();
  int at = __popc(m & ((1u << lane) - 1u)), n = 0, all = 0;
  for (int w = 0; w < kMaxExperts / 32; ++w) {
    if (w < warp) {
      at += s.first[w];
      before += sm.wcount[w];
    }
    n += s.first[w];
    all += sm.wcount[w];
  }
  __syncthreads();
  if (live) {
    s.e[at] = e;
    s.r0[at] = r0;
    s.r1[at] = r1;
    s.first[at] = before - units;
    const int per = (r1 - r0 + tiles - 1) / tiles;
    atomicMax(&s.widest, (per + 15) / 16 * 16);
  }
  if (u == 0) {
    s.n = n;
    s.units = all;
  }
  __syncthreads();
}

struct Unit {
  int e, mt;      // expert, tile of outputs
  int r0, n;      // rows
};
__device__ __forceinline__ Unit find_unit(const Groups& s, int m_tiles, int unit) {
  int lo = 0, hi = s.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (s.first[mid] <= unit) lo = mid;
    else hi = mid - 1;
  }
  const int local = unit - s.first[lo], part = local / m_tiles;
  const int rows = s.r1[lo] - s.r0[lo], parts = (rows + kUnitRows - 1) / kUnitRows;
  const int per = (rows + parts - 1) / parts;
  Unit u;
  u.e = s.e[lo];
  u.mt = local - part * m_tiles;
  u.r0 = s.r0[lo] + part * per;
  u.n = min(per, s.r1[lo] - u.r0);
  return u;
}

__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, int where) {
  if (ptx::mbar_wait(bar, parity, kWaitNs)) return true;
  record_error(&q4_fault, kErrTimeout, kAtQ4, where);
  return false;
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, uint32_t bytes = 16) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// ------------------------------------------------------------------ dequantising
// Copies run ahead of the values by kCodeSlots - 1 blocks of the set, over the ends of units.
template <bool kGated>
struct CodeCursor {
  int unit, kt, base;   // base: blocks of the units before this one
  int piece;            // of eight groups' scales, of the block before
  const uint8_t* codes; // of this row
  const uint8_t* scales;
  size_t step, half;    // bytes from block to block, and from half to half
  bool row;             // this row is there
  __device__ __forceinline__ void enter(const Q4Args& a, const Q4Shape& s, const Groups& gs,
                                        int m_tiles, int set, int lane_row) {
    kt = set ^ (base & 1);
    piece = -1;
    if (unit >= gs.units) return;
    const Unit u = find_unit(gs, m_tiles, unit);
    const int m = kGated ? lane_row >> 6 : 0;
    const int n = kGated ? u.mt * 64 + (lane_row & 63) : u.mt * 128 + lane_row;
    row = n < s.rows;
    if (!row) return;
    codes = static_cast<const uint8_t*>(a.codes[m]) + u.e * s.code_bytes() + s.code_at(n, 0, 0);
    half = (size_t)s.tile_rows(n) * 16;
    step = 2 * half;
    scales = static_cast<const uint8_t*>(a.scales[m]) + ((size_t)u.e * s.rows + n) * s.groups_pad * 2;
  }
};

template <bool kGated>
__device__ __forceinline__ void dequantise(const Q4Args& a, const Q4Shape& s, int m_tiles, Smem& sm,
                                           uint32_t tmem) {
  const int warp = threadIdx.x / 32 - kEpiWarps, set = warp >> 2;
  const int lane_row = (threadIdx.x & 127);   // (warps 4-7 and 8-11: lanes 0 .. 127 of either set)
  const Groups& gs = sm.groups;
  const int per_piece = s.group == 32 ? 2 : s.group == 64 ? 3 : 4;   // log2 of blocks per piece
  const uint32_t codes_at = ptx::smem_addr(&sm.codes[set][0][0][lane_row]);
  const uint32_t scales_at = ptx::smem_addr(&sm.scales[set][0][lane_row]);
  CodeCursor<kGated> c;
  c.unit = blockIdx.x;
  c.base = 0;
  c.enter(a, s, gs, m_tiles, set, lane_row);
  int copy_slot = 0, copy_piece = 0;
  auto copy = [&]() {
    while (c.unit < gs.units && c.kt >= s.k_tiles) {
      c.base += s.k_tiles;
      c.unit += gridDim.x;
      c.enter(a, s, gs, m_tiles, set, lane_row);
    }
    if (c.unit < gs.units) {
      const int piece = c.kt >> per_piece;
      if (c.row) {
        const uint8_t* src = c.codes + c.kt * c.step;
        copy16(codes_at + copy_slot * sizeof(sm.codes[0][0]), src);
        copy16(codes_at + copy_slot * sizeof(sm.codes[0][0]) + sizeof(sm.codes[0][0][0]), src + c.half);
        if (piece != c.piece) copy16(scales_at + copy_piece * sizeof(sm.scales[0][0]), c.scales + piece * 16);
      }
      if (piece != c.piece) copy_piece = copy_piece + 1 == kCodeSlots ? 0 : copy_piece + 1;
      c.piece = piece;
      copy_slot = copy_slot + 1 == kCodeSlots ? 0 : copy_slot + 1;
      c.kt += 2;
    }
    copies_commit();
  };
  for (int i = 0; i < kCodeSlots - 1; ++i) copy();
  int base = 0, slot = 0, next_piece = 0;
  bool ok = true;
  for (int unit = blockIdx.x; ok && unit < gs.units; unit += gridDim.x, base += s.k_tiles) {
    int piece = -1;
    uint4 sc = make_uint4(0, 0, 0, 0);
    for (int kt = set ^ (base & 1); kt < s.k_tiles; kt += 2) {
      copy();
      copies_wait<kCodeSlots - 1>();
      if (kt >> per_piece != piece) {
        piece = kt >> per_piece;
        sc = sm.scales[set][next_piece][lane_row];
        next_piece = next_piece + 1 == kCodeSlots ? 0 : next_piece + 1;
      }
      const uint4 c0 = sm.codes[set][slot][0][lane_row], c1 = sm.codes[set][slot][1][lane_row];
      slot = slot + 1 == kCodeSlots ? 0 : slot + 1;
      // the block's scales: one, or one per half
      const int at = s.group == 32 ? (kt & 3) * 2 : s.group == 64 ? kt & 7 : (kt >> 1) & 7;
      const uint32_t lo = at & 2 ? sc.y : sc.x, hi = at & 2 ? sc.w : sc.z;
      const uint32_t pair = at & 4 ? hi : lo;
      const Q4Scale s0 = q4_scale_pair(at & 1 ? pair >> 16 : pair);
      const Q4Scale s1 = s.group == 32 ? q4_scale_pair(pair >> 16) : s0;
      const uint32_t w[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
      uint32_t v[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = q4_value_pair(w[i / 4], i & 3, i < 16 ? s0 : s1);
      const int block = base + kt, as = block % kASlots;
      ok = wait(&sm.a_empty[as], ((block / kASlots) & 1) ^ 1, 1);
      if (!__all_sync(0xffffffffu, ok)) {
        ok = false;
        break;
      }
      ptx::tc_fence_after();
      ptx::tmem_st32(tmem + as * 32 + ((uint32_t)(warp & 3) << 21), v);
      ptx::tmem_st_wait();
      ptx::tc_fence_before();
      __syncwarp();
      if ((threadIdx.x & 31) == 0) ptx::mbar_arrive(&sm.a_full[as]);
    }
  }
  copies_wait<0>();
}

// ------------------------------------------------------------------ loading x
__device__ __forceinline__ void load_x(const Q4Args& a, const Q4Shape& s, int m_tiles, Smem& sm,
                                       int b_slots, int b_bytes) {
  const int tid = threadIdx.x - (kThreads - kLoadThreads), chunk = tid & 7, row0 = tid >> 3;
  constexpr int kStep = kLoadThreads / 8, kMine = (kUnitRows + kStep - 1) / kStep;   // 12, 11
  const Groups& gs = sm.groups;
  const uint32_t ring = ptx::smem_addr(sm.b);
  int block = 0;
  bool ok = true;
  auto done = [&](int b) {   // this thread's part of block b is there, for the tensor pipe to see
    ptx::fence_proxy_async_smem();
    ptx::mbar_arrive(&sm.b_full[b % b_slots]);
  };
  for (int unit = blockIdx.x; ok && unit < gs.units; unit += gridDim.x) {
    const Unit u = find_unit(gs, m_tiles, unit);
    const __nv_bfloat16* src[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int r = row0 + i * kStep;
      src[i] = nullptr;
      if (r < u.n) {
        int64_t t = u.r0 + r;
        if (a.rows != nullptr) {
          const int p = __ldg(a.rows + u.r0 + r);
          t = p >= 0 ? p / a.k : -1;
        }
        src[i] = t >= 0 && t < a.T_x ? a.x + t * a.ldx + chunk * 8
                                     : reinterpret_cast<const __nv_bfloat16*>(q4_zero_row) + chunk * 8;
      }
    }
    for (int kt = 0; kt < s.k_tiles; ++kt, ++block) {
      const int bs = block % b_slots;
      ok = wait(&sm.b_empty[bs], ((block / b_slots) & 1) ^ 1, 2);
      if (!ok) break;
      const uint32_t bytes = kt * 64 + chunk * 8 < s.K ? 16u : 0u;   // (zeros behind n_in)
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int r = row0 + i * kStep;
        if (src[i] != nullptr)
          copy16(ring + bs * b_bytes + r * 128 + ((chunk ^ (r & 7)) << 4),
                 bytes ? src[i] + kt * 64 : src[i], bytes);
      }
      copies_commit();
      if (block >= kLoadLag) {
        copies_wait<kLoadLag>();
        done(block - kLoadLag);
      }
    }
  }
  copies_wait<0>();
  if (ok)
    for (int b = block < kLoadLag ? 0 : block - kLoadLag; b < block; ++b) done(b);
}

// ------------------------------------------------------------------ issuing the MMAs
__device__ __forceinline__ void issue(const Q4Shape& s, int m_tiles, Smem& sm, uint32_t tmem,
                                      int b_slots, int b_bytes) {
  const Groups& gs = sm.groups;
  const uint32_t ring = ptx::smem_addr(sm.b);
  int block = 0, turn = 0;
  bool ok = true;
  for (int unit = blockIdx.x; ok && unit < gs.units; unit += gridDim.x, ++turn) {
    const Unit u = find_unit(gs, m_tiles, unit);
    const uint32_t idesc = ptx::idesc_bf16(128, (u.n + 15) / 16 * 16);
    const int buf = turn & 1;
    ok = wait(&sm.d_empty[buf], ((turn >> 1) & 1) ^ 1, 3);
    for (int kt = 0; ok && kt < s.k_tiles; ++kt, ++block) {
      const int as = block % kASlots, bs = block % b_slots;
      ok = wait(&sm.b_full[bs], (block / b_slots) & 1, 4) && wait(&sm.a_full[as], (block / kASlots) & 1, 5);
      if (!ok) break;
      ptx::tc_fence_after();
#pragma unroll
      for (int j = 0; j < 4; ++j)
        ptx::mma_bf16_ta(tmem + kAcc0 + buf * 128, tmem + as * 32 + j * 8,
                         ptx::sdesc_k_sw128(ring + bs * b_bytes + j * 32), idesc, (kt | j) != 0);
      ptx::mma_commit(&sm.a_empty[as]);
      ptx::mma_commit(&sm.b_empty[bs]);
    }
    if (ok) ptx::mma_commit(&sm.d_full[buf]);
  }
  // everything issued has been done before the CTA gives its memory back
  ptx::mma_commit(&sm.drain);
  wait(&sm.drain, 0, 6);
}

// ------------------------------------------------------------------ epilogue
__device__ __forceinline__ void store_y(const Q4Args& a, int64_t r, int n, float v) {
  if (a.y_fp32) static_cast<float*>(a.y)[r * a.ldy + n] = v;
  else static_cast<__nv_bfloat16*>(a.y)[r * a.ldy + n] = __float2bfloat16_rn(v);
}

template <bool kGated>
__device__ __forceinline__ void epilogue(const Q4Args& a, const Q4Shape& s, int m_tiles, Smem& sm,
                                         uint32_t tmem) {
  const int warp = threadIdx.x >> 5, row = threadIdx.x;   // lane of tensor memory
  const Groups& gs = sm.groups;
  int turn = 0, swap = 0;
  for (int unit = blockIdx.x; unit < gs.units; unit += gridDim.x, ++turn) {
    const Unit u = find_unit(gs, m_tiles, unit);
    const int buf = turn & 1;
    if (!ptx::epi_all(wait(&sm.d_full[buf], (turn >> 1) & 1, 7))) break;
    ptx::tc_fence_after();
    const uint32_t from = tmem + kAcc0 + buf * 128 + ((uint32_t)warp << 21);
    const int n = kGated ? u.mt * 64 + (row & 63) : u.mt * 128 + row;
    for (int c0 = 0; c0 < u.n; c0 += 16) {
      float v[16];
      ptx::tmem_ld16(from + c0, v);
      ptx::tmem_ld_wait();
      if (kGated) {
        // lanes 0 .. 63 are gates, 64 .. 127 ups: the gates' lanes do eight rows, the ups' the others
        const int up = row >> 6, first = up * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) sm.swap[swap][up][row & 63][j] = up ? v[j] : v[8 + j];
        ptx::named_bar_sync(1, 32 * kEpiWarps);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float other = sm.swap[swap][up ^ 1][row & 63][j], mine = up ? v[8 + j] : v[j];
          if (c0 + first + j < u.n && n < s.N)
            store_y(a, u.r0 + c0 + first + j, n,
                    up ? silu_divide(other) * mine : silu_divide(mine) * other);
        }
        swap ^= 1;
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (c0 + j < u.n && n < s.N) store_y(a, u.r0 + c0 + j, n, v[j]);
      }
    }
    ptx::tc_fence_before();
    ptx::mbar_arrive(&sm.d_empty[buf]);
  }
}

template <bool kGated>
__global__ void __launch_bounds__(kThreads, 1)
q4_kernel(const __grid_constant__ Q4Args a, const __grid_constant__ Q4Shape s) {
  extern __shared__ __align__(1024) uint8_t raw[];
  Smem& sm = *reinterpret_cast<Smem*>(raw);
  const int warp = threadIdx.x >> 5;
  if (warp == kMmaWarp) {
    ptx::tmem_alloc(&sm.tmem, 512);
    ptx::tmem_relinquish();
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < kASlots; ++i) {
      ptx::mbar_init(&sm.a_full[i], kDeqWarps / 2);
      ptx::mbar_init(&sm.a_empty[i], 1);
    }
    for (int i = 0; i < kBSlotsMax; ++i) {
      ptx::mbar_init(&sm.b_full[i], kLoadThreads);
      ptx::mbar_init(&sm.b_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(&sm.d_full[i], 1);
      ptx::mbar_init(&sm.d_empty[i], 32 * kEpiWarps);
    }
    ptx::mbar_init(&sm.drain, 1);
    ptx::fence_mbarrier_init();
  }
  ptx::tc_fence_before();
  pdl_wait();
  pdl_launch_dependents();
  const int m_tiles = kGated ? (s.N + 63) / 64 : (s.N + 127) / 128;
  find_groups(a, m_tiles, sm);   // (synchronises the CTA)
  ptx::tc_fence_after();
  const uint32_t tmem = sm.tmem;
  const int b_bytes = sm.groups.widest * 128;
  const int b_slots = min(kBSlotsMax, kBRing / b_bytes);
  if (warp < kEpiWarps) epilogue<kGated>(a, s, m_tiles, sm, tmem);
  else if (warp < kMmaWarp) dequantise<kGated>(a, s, m_tiles, sm, tmem);
  else if (warp > kMmaWarp) load_x(a, s, m_tiles, sm, b_slots, b_bytes);
  else if ((threadIdx.x & 31) == 0) issue(s, m_tiles, sm, tmem, b_slots, b_bytes);
  __syncwarp();
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) ptx::tmem_dealloc(tmem, 512);
}

}  // namespace

cudaError_t launch_q4_linear(const Q4Args& a, const dmoe_q4_desc& d, cudaStream_t st) {
  const Q4Shape s = q4_shape(d);
  const bool gated = a.codes[1] != nullptr;
  static std::atomic<uint32_t> ready{0};   // a bit per device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  const uint32_t bit = dev < 32 ? 1u << dev : 0u;
  if (e == cudaSuccess && (ready.load(std::memory_order_acquire) & bit) == 0u) {
    for (auto* k : {q4_kernel<false>, q4_kernel<true>})
      if (e == cudaSuccess)
        e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(Smem));
    if (e == cudaSuccess) ready.fetch_or(bit, std::memory_order_release);
  }
  if (e != cudaSuccess) return e;
  // at most as many CTAs as units there can be
  const int64_t groups = a.n_groups < a.R ? a.n_groups : a.R;
  const int64_t units = (groups + a.R / kUnitRows) * (gated ? (s.N + 63) / 64 : (s.N + 127) / 128);
  const int sms = device_sm_count();
  return launch_ex(gated ? q4_kernel<true> : q4_kernel<false>, dim3((unsigned)(units < sms ? units : sms)),
                   dim3(kThreads), sizeof(Smem), st, true, a, s);
}

cudaError_t q4_fault_address(void** p) { return cudaGetSymbolAddress(p, q4_fault); }

}  // namespace dmoe

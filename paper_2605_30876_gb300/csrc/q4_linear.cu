// Products of sorted rows with their experts' 4-bit matrices, plain or gate and up with SwiGLU:
// y^T = W x^T, per unit of 128 outputs (or 64 gate and 64 up outputs) and at most 128 rows of a group.
//
// A persistent CTA per SM, in roles, by stages of 128 inputs:
//   dequantising warps (four sets of four, a stage each in turn): a lane has a row of W. A bulk copy
//       brings the codes of a warp's 32 rows; they become bf16 values by one exact FMA per pair
//       and go to tensor memory: the A operand of the MMAs. Through shared memory they would take
//       four times the codes' bytes twice, and 8 KB of codes have 368 cycles of an SM's share of
//       HBM's rate, in which shared memory moves 46 KB.
//   loading warps: the rows of x that the group names, a stage each in turn, by copies of 16 bytes
//       into shared memory (B). Between the copies and the tensor pipe's reads is a fence of 200
//       cycles and more, so several stages are under way. (TMA gathers of four rows need no fence,
//       but took 80 cycles each: for 64 rows 2500 cycles a stage.)
//   an issuing warp: tcgen05.mma, M = 128 outputs, N = the unit's rows in sixteens
//   epilogue warps: sums from tensor memory, SwiGLU, y
// Few rows: the weights' bytes are the bound, and the instructions per code are close to it: 64 pairs
// a lane and stage at 2.75, of the 368 that each scheduler issues in that time. Many rows: the
// tensor pipe, and the copies of x.
// Every wait has a limit of one second. One that runs out is recorded (dmoe_q4_device_error) and ends
// its role; the others' waits run out after it, and the CTA gives its tensor memory back.
#include "q4.cuh"
#include "silu.cuh"
#include "sm100_ptx.cuh"

namespace dmoe {
namespace {

constexpr int kEpiWarps = 4, kSets = 4, kDeqWarps = 4 * kSets, kLoadWarps = 4;
constexpr int kLoadWarp = kEpiWarps + kDeqWarps, kMmaWarp = kLoadWarp + kLoadWarps;
constexpr int kThreads = 32 * (kMmaWarp + 1);
constexpr int kUnitRows = 128;             // rows of a group per unit, at most
constexpr int kASlots = kSets;             // stages of A in tensor memory, 64 columns each
constexpr int kBRing = 96 * 1024;          // bytes of the ring of x's stages
constexpr int kBSlotsMax = 8;
constexpr int kCodeSlots = 3;              // blocks of codes per warp, one of them in use
constexpr int kAcc0 = kASlots * 64;        // first column of the sums: two buffers of 128
constexpr uint64_t kWaitNs = 1000000000ull;
constexpr int kSched = 256;                // units of a CTA that are looked up once, together

__device__ DevErrRecord q4_fault;          // of every call on the device

// The groups that have rows and an expert, in order, and their first units.
struct Groups {
  int n, units;
  int widest;   // rows of the widest unit, in sixteens
  int e[kMaxExperts], r0[kMaxExperts], r1[kMaxExperts], first[kMaxExperts];
};

struct __align__(16) Unit {
  int e, mt;      // expert, tile of outputs
  int r0, n;      // rows
};

struct CodeSlot {
  uint4 codes[4][kQ4Rows];       // [32 inputs][row]
  uint16_t scales[kQ4Rows * 4];  // [row][group]
};

struct Smem {
  uint8_t b[kBRing];                         // 1024-byte aligned
  CodeSlot code[kDeqWarps][kCodeSlots];
  float swap[2][2][64][9];                   // ups and gates between epilogue warps
  Unit sched[kSched];                        // the CTA's units, in its order
  Groups groups;
  uint64_t code_full[kDeqWarps][kCodeSlots];
  uint64_t a_full[kASlots], a_empty[kASlots];
  uint64_t b_full[kBSlotsMax], b_empty[kBSlotsMax];
  uint64_t d_full[2], d_empty[2], drain;
  uint32_t tmem;
  int wcount[kThreads / 32];
};

__device__ __forceinline__ void find_groups(const Q4Args& a, int m_tiles, Smem& sm) {
  Groups& s = sm.groups;
  const int u = threadIdx.x, lane = u & 31, warp = u >> 5, R = (int)a.R;
  static_assert(kThreads >= kMaxExperts && kThreads >= kSched, "a thread per group, and per unit");
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

// the i-th unit of this CTA, which is there
__device__ __forceinline__ Unit unit_at(const Smem& sm, int m_tiles, int i) {
  return i < kSched ? sm.sched[i] : find_unit(sm.groups, m_tiles, blockIdx.x + i * gridDim.x);
}
__device__ __forceinline__ int units_of_cta(const Groups& s) {
  return s.units > (int)blockIdx.x ? (s.units - (int)blockIdx.x - 1) / (int)gridDim.x + 1 : 0;
}

// Waits with pauses, or, for the issuing warp (kPause 0), without.
template <int kPause>
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, int where) {
  if (ptx::mbar_wait_paused(bar, parity, kWaitNs, kPause)) return true;
  record_error(&q4_fault, kErrTimeout, kAtQ4, where);
  return false;
}

// A slot of a ring and the parity of its turn, one step on.
struct Slot {
  int i = 0;
  uint32_t turn = 0;
  __device__ __forceinline__ void next(int n) {
    if (++i == n) {
      i = 0;
      turn ^= 1u;
    }
  }
};

// ------------------------------------------------------------------ dequantising
template <bool kGated>
__device__ __forceinline__ void dequantise(const Q4Args& a, const Q4Shape& s, int m_tiles, Smem& sm,
                                           uint32_t tmem) {
  const int warp = threadIdx.x / 32 - kEpiWarps, set = warp >> 2, lane = threadIdx.x & 31;
  const int units = units_of_cta(sm.groups), scale_block = s.scale_block();
  CodeSlot* const ring = sm.code[warp];
  uint64_t* const full = sm.code_full[warp];

  // The copies run ahead of the values by kCodeSlots - 1 blocks of this warp, over the ends of units.
  // base: stages of the units before; the set takes the stages whose number is set mod kSets.
  int unit = 0, base = 0, st = set, copied = 0;
  const uint8_t *codes = nullptr, *scales = nullptr;
  bool there = false;   // the warp's rows of this unit are in the matrix
  auto enter = [&]() {
    if (unit >= units) return;
    const Unit u = unit_at(sm, m_tiles, unit);
    const int m = kGated ? (warp & 3) >> 1 : 0;
    const int tile = kGated ? u.mt * 2 + (warp & 1) : u.mt * 4 + (warp & 3);
    there = tile < s.tiles;
    const size_t block = ((size_t)u.e * s.tiles + tile) * s.blocks + st;
    codes = static_cast<const uint8_t*>(a.codes[m]) + block * kQ4CodeBytes;
    scales = static_cast<const uint8_t*>(a.scales[m]) + block * scale_block;
  };
  Slot to;
  auto copy = [&]() {
    while (st >= s.blocks && unit < units) {
      base += s.blocks;
      ++unit;
      st = (set - base) & (kSets - 1);
      if (st < s.blocks) enter();
    }
    if (unit >= units) return;
    if (lane == 0) {
      ptx::mbar_arrive_expect_tx(&full[to.i], there ? kQ4CodeBytes + scale_block : 0);
      if (there) {
        ptx::bulk_load(ring[to.i].codes, codes, kQ4CodeBytes, &full[to.i]);
        ptx::bulk_load(ring[to.i].scales, scales, scale_block, &full[to.i]);
      }
    }
    codes += kSets * kQ4CodeBytes;
    scales += kSets * scale_block;
    st += kSets;
    ++copied;
    to.next(kCodeSlots);
  };
  if (st < s.blocks) enter();
  for (int i = 0; i < kCodeSlots - 1; ++i) copy();

  const uint32_t at = tmem + set * 64 + ((uint32_t)(warp & 3) << 21);   // (A's slot is the set's)
  Slot from;
  uint32_t a_turn = 1;
  int done = 0;
  for (;; ++done) {
    copy();
    if (done == copied) break;   // (copies are ahead until there are none)
    if (!__all_sync(0xffffffffu, wait<0>(&full[from.i], from.turn, 8))) break;
    const CodeSlot& slot = ring[from.i];
    // the scales of the stage's four 32 inputs
    uint32_t s01, s23;
    if (s.groups == 4) {
      const uint2 v = reinterpret_cast<const uint2*>(slot.scales)[lane];
      s01 = v.x;
      s23 = v.y;
    } else if (s.groups == 2) {
      const uint32_t v = reinterpret_cast<const uint32_t*>(slot.scales)[lane];
      s01 = __byte_perm(v, 0u, 0x1010);
      s23 = __byte_perm(v, 0u, 0x3232);
    } else {
      s01 = s23 = slot.scales[lane] * 0x10001u;
    }
    if (!__all_sync(0xffffffffu, wait<20>(&sm.a_empty[set], a_turn, 1))) break;
    ptx::tc_fence_after();
#pragma unroll 1
    for (int h = 0; h < 4; h += 2) {
      const uint32_t pair = h == 0 ? s01 : s23;
      const Q4Scale s0 = q4_scale_pair(pair), s1 = q4_scale_pair(pair >> 16);
      const uint4 c0 = slot.codes[h][lane], c1 = slot.codes[h + 1][lane];
      const uint32_t w[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
      uint32_t v[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = q4_value_pair(w[i / 4], i & 3, i < 16 ? s0 : s1);
      ptx::tmem_st32(at + h * 16, v);
    }
    ptx::tmem_st_wait();
    ptx::tc_fence_before();
    __syncwarp();   // (the slot has been read, too)
    if (lane == 0) ptx::mbar_arrive(&sm.a_full[set]);
    a_turn ^= 1u;
    from.next(kCodeSlots);
  }
  // no copy is left in flight behind a wait that ran out
  for (; done < copied; ++done, from.next(kCodeSlots))
    if (!ptx::mbar_wait_paused(&full[from.i], from.turn, kWaitNs, 0)) break;
}

// ------------------------------------------------------------------ loading x
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// The source row of sorted row r, or -1.
__device__ __forceinline__ int source(const Q4Args& a, int r) {
  if (a.rows == nullptr) return r;
  const int p = __ldg(a.rows + r), t = p >= 0 ? p / a.k : -1;
  return t < a.T_x ? t : -1;
}

// The ring's slots: 8, or as many as there is room for. A slot's stages are one warp's, so that no warp
// waits for a slot two turns ahead of another: with 8 slots, a warp has two.
__device__ __forceinline__ int b_slots_of(int widest) { return widest <= 48 ? 8 : widest <= 96 ? 4 : 3; }
static_assert(8 * 48 * 256 <= kBRing && 4 * 96 * 256 <= kBRing && 3 * 128 * 256 <= kBRing &&
                  kLoadWarps == 4, "ring of x");

__device__ __forceinline__ void load_x(const Q4Args& a, const Q4Shape& s, int m_tiles, Smem& sm) {
  const int warp = threadIdx.x / 32 - kLoadWarp, lane = threadIdx.x & 31;
  const int chunk = lane & 7, sub = lane >> 3;   // 16 bytes of a row's 128, row of four
  const int units = units_of_cta(sm.groups), block_bytes = sm.groups.widest * 128;
  const int slots = b_slots_of(sm.groups.widest), warps = slots < kLoadWarps ? slots : kLoadWarps;
  const bool lag = slots > kLoadWarps;   // a stage's copies are waited for after the next one's start
  const uint32_t ring = ptx::smem_addr(sm.b);
  if (warp >= warps) return;
  int first = warp, slot = warp, pending = -1;   // this warp's next stage, counted from the unit's start
  uint32_t turn = 1;
  auto publish = [&](int i) {   // this warp's stage in slot i, for the tensor pipe to see
    ptx::fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(&sm.b_full[i]);
  };
  for (int unit = 0; unit < units; ++unit, first -= s.blocks) {
    if (first >= s.blocks) continue;
    const Unit u = unit_at(sm, m_tiles, unit);
    int src[kUnitRows / 32];                     // of rows lane, lane + 32, ...
#pragma unroll
    for (int j = 0; j < kUnitRows / 32; ++j)
      src[j] = 32 * j < u.n ? max(source(a, u.r0 + min(32 * j + lane, u.n - 1)), 0) : 0;
    for (; first < s.blocks; first += warps) {
      if (!__all_sync(0xffffffffu, wait<20>(&sm.b_empty[slot], turn, 2))) {
        copies_wait<0>();
        return;
      }
      // (row r's 16-byte piece c is at r * 128 + (c ^ r % 8) * 16)
      const uint32_t dst = ring + slot * 2 * block_bytes;
      const int k = first * 128 + chunk * 8;
      const __nv_bfloat16* x = a.x + k;
      const uint32_t in0 = k < s.K ? 16u : 0u, in1 = k + 64 < s.K ? 16u : 0u;   // (zeros behind n_in)
#pragma unroll
      for (int j = 0; j < kUnitRows / 32; ++j) {
        const int n = min(u.n - 32 * j, 32);
#pragma unroll 1
        for (int i = 0; i < n; i += 4) {
          const int r = i + sub;
          const int64_t at = __shfl_sync(0xffffffffu, src[j], r) * a.ldx;
          if (r < n) {
            const uint32_t to = dst + (32 * j + r) * 128 + ((chunk ^ (r & 7)) << 4);
            copy16(to, in0 ? x + at : a.x, in0);
            copy16(to + block_bytes, in1 ? x + at + 64 : a.x, in1);
          }
        }
      }
      copies_commit();
      if (!lag) {
        copies_wait<0>();
        publish(slot);
      } else {
        copies_wait<1>();
        if (pending >= 0) publish(pending);
        pending = slot;
      }
      slot += warps;
      if (slot >= slots) {
        slot = warp;
        turn ^= 1u;
      }
    }
  }
  copies_wait<0>();
  if (pending >= 0) publish(pending);
}

// ------------------------------------------------------------------ issuing the MMAs
__device__ __forceinline__ void issue(const Q4Shape& s, int m_tiles, Smem& sm, uint32_t tmem) {
  const int units = units_of_cta(sm.groups), block_bytes = sm.groups.widest * 128;
  const int slots = b_slots_of(sm.groups.widest);
  const uint64_t ring = ptx::sdesc_k_sw128(ptx::smem_addr(sm.b));
  const uint32_t block16 = block_bytes >> 4;   // (a descriptor's address is in units of 16 bytes)
  Slot as, bs, ds;
  bool ok = true;
  for (int turn = 0; ok && turn < units; ++turn, ds.next(2)) {
    const Unit u = unit_at(sm, m_tiles, turn);
    const uint32_t idesc = ptx::idesc_bf16(128, (u.n + 15) / 16 * 16);
    const uint32_t d = tmem + kAcc0 + ds.i * 128;
    ok = __all_sync(0xffffffffu, wait<0>(&sm.d_empty[ds.i], ds.turn ^ 1u, 3));
    for (int st = 0; ok && st < s.blocks; ++st) {
      ok = wait<0>(&sm.b_full[bs.i], bs.turn, 4) && wait<0>(&sm.a_full[as.i], as.turn, 5);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      ptx::tc_fence_after();
      if (ptx::elect_one()) {
        const uint64_t b0 = ring + bs.i * 2 * block16;
        const uint32_t a0 = tmem + as.i * 64;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          ptx::mma_bf16_ta(d, a0 + j * 8, b0 + (j & 4 ? block16 : 0u) + (j & 3) * 2, idesc, (st | j) != 0);
        ptx::mma_commit(&sm.a_empty[as.i]);
        ptx::mma_commit(&sm.b_empty[bs.i]);
        if (st == s.blocks - 1) ptx::mma_commit(&sm.d_full[ds.i]);
      }
      __syncwarp();
      as.next(kASlots);
      bs.next(slots);
    }
  }
  // everything issued has been done before the CTA gives its memory back
  if (ptx::elect_one()) ptx::mma_commit(&sm.drain);
  wait<0>(&sm.drain, 0, 6);
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
  const int units = units_of_cta(sm.groups);
  int swap = 0;
  for (int turn = 0; turn < units; ++turn) {
    const Unit u = unit_at(sm, m_tiles, turn);
    const int buf = turn & 1;
    uint32_t missing[4] = {0, 0, 0, 0};   // rows without a source: zeros
    if (a.rows != nullptr) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = 32 * j + (row & 31);
        missing[j] = __ballot_sync(0xffffffffu, r < u.n && source(a, u.r0 + r) < 0);
      }
    }
    if (!ptx::epi_all(wait<100>(&sm.d_full[buf], (turn >> 1) & 1, 7))) break;
    ptx::tc_fence_after();
    const uint32_t from = tmem + kAcc0 + buf * 128 + ((uint32_t)warp << 21);
    const int n = kGated ? u.mt * 64 + (row & 63) : u.mt * 128 + row;
    for (int c0 = 0; c0 < u.n; c0 += 16) {
      float v[16];
      ptx::tmem_ld16(from + c0, v);
      ptx::tmem_ld_wait();
      const uint32_t miss = c0 < 64 ? (c0 < 32 ? missing[0] : missing[1])
                                    : (c0 < 96 ? missing[2] : missing[3]);
      if (miss >> (c0 & 16) & 0xFFFFu) {
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (miss >> ((c0 & 16) + j) & 1u) v[j] = 0.f;
      }
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
    for (int i = 0; i < kDeqWarps * kCodeSlots; ++i) ptx::mbar_init(&sm.code_full[0][0] + i, 1);
    for (int i = 0; i < kASlots; ++i) {
      ptx::mbar_init(&sm.a_full[i], 4);
      ptx::mbar_init(&sm.a_empty[i], 1);
    }
    for (int i = 0; i < kBSlotsMax; ++i) {
      ptx::mbar_init(&sm.b_full[i], 1);
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
  if ((int)threadIdx.x < min(kSched, units_of_cta(sm.groups)))
    sm.sched[threadIdx.x] = find_unit(sm.groups, m_tiles, blockIdx.x + threadIdx.x * gridDim.x);
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = sm.tmem;
  if (warp < kEpiWarps) epilogue<kGated>(a, s, m_tiles, sm, tmem);
  else if (warp < kLoadWarp) dequantise<kGated>(a, s, m_tiles, sm, tmem);
  else if (warp == kMmaWarp) issue(s, m_tiles, sm, tmem);
  else load_x(a, s, m_tiles, sm);
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

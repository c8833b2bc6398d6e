// Products of sorted rows with their experts' 4-bit matrices, plain or gate and up with SwiGLU:
// y^T = W x^T, per unit of 128 outputs (or 64 gate and 64 up outputs) and at most 64 or 96 rows of a
// group.
//
// A persistent CTA per SM, in roles, by stages of 128 inputs:
//   dequantising warps (four sets of four, a stage each in turn): a lane has a row of W. Its codes come
//       by asynchronous copies (bulk copies, one per warp and stage, were slower); they become bf16
//       values by one exact FMA per pair and go to tensor memory: the A operand of the MMAs. Through
//       shared memory they would take four times the codes' bytes twice, and 8 KB of codes have
//       368 cycles of an SM's share of HBM's rate, in which shared memory moves 46 KB.
//   loading warps: the rows of x that the group names, a stage each in turn, by copies of 16 bytes
//       into shared memory (B). Between the copies and the tensor pipe's reads is a fence of 200
//       cycles and more, so several stages are under way. (TMA gathers of four rows need no fence,
//       but took 80 cycles each: for 64 rows 2500 cycles a stage.)
//   two issuing warps: tcgen05.mma, M = 128 outputs, N = the unit's rows in sixteens
//   epilogue warps: sums from tensor memory, SwiGLU, y
//
// Few rows: the weights' bytes are the bound, and the instructions per code are close to it (64 pairs a
// lane and stage at 2.75 instructions, of the 368 that a scheduler issues in an SM's share of the
// time). Measured with cold weights in a graph, floors at 6.8 TB/s: 256 rows for 104 experts,
// 512 x 2048, 21.0 us (62 MB, 9.2 us): issue slots 58 % busy, the ALUs 44 %, DRAM 34 %; one row
// times 8192 x 8192 17.0 us (5.3 us); 2048 rows for 220 of 256 experts, gate and up of 2048 x 512,
// 60 us (36.6 us: 4.2 TB/s). Of the time for one token's eight experts (10.6 us) the launch, the
// look-up of groups and rows and the first bytes' way from HBM are about half.
// Many rows: a stage's values take 440 cycles, and with its MMAs 610 (not all of either overlaps); the
// copies of x, 24 KB of every SM's from L2 in a stage of 96 rows, bring that to 830. 2048 rows times
// 4096 x 4096 74 us (930 TFLOP/s), 2048 x 8 rows for 256 experts, gate and up of 2048 x 512,
// 116.5 us (590 TFLOP/s; 64 rows an expert).
//
// With long sums the CTAs run in pairs (clusters of two). Where there are at most half as many units as
// CTAs, a pair shares a unit, half of the stages each, and the first CTA adds the second one's sums to
// its own. Alone and in pairs, us, cold weights in a graph:
//   outputs x K     8192 x 2048   x 2944       x 4096       x 8192       2048 x 2048   x 2944
//   1 row            9.6  9.9   11.2 11.1   13.2 12.6   20.3 16.0        8.8  8.8   10.4  9.6
//   64 rows         12.2 12.7   15.0 14.5   17.8 16.5   28.0 22.0       11.7 11.5   14.2 12.9
//   96 rows         12.2 14.7   14.6 16.8   17.1 18.8   26.4 25.2       11.4 10.9   13.7 12.1
// The pairs' launch, barriers and exchange take 1 to 2 us (0.5 to 1 where they share nothing), the
// exchange more with more rows. So pairs are for kPairStages stages and more, and at most half as many
// tiles as SMs; that gives away 0.8 to 1.6 us with few tiles just below it, and 1.7 with 96 rows
// and 64 tiles above it.
// Every wait has a limit of one second. One that runs out is recorded (dmoe_q4_device_error) and ends
// its role; the others' waits run out after it, and the CTA gives its tensor memory back.
#include "q4.cuh"
#include "silu.cuh"
#include "sm100_ptx.cuh"

namespace dmoe {
namespace {

constexpr int kEpiWarps = 4, kSets = 4, kDeqWarps = 4 * kSets, kLoadWarps = 8, kMmaWarps = 2;
constexpr int kLoadWarp = kEpiWarps + kDeqWarps, kMmaWarp = kLoadWarp + kLoadWarps;
constexpr int kThreads = 32 * (kMmaWarp + kMmaWarps);
// Rows of a group per unit, at most: a launch has one of the two limits. With the smaller one a stage
// takes two thirds to four fifths of the time; which one is better goes by the CTAs' turns
// (unit_limit).
constexpr int kUnitRows = 96, kSmallUnitRows = 64;
// The ring of stages: A in tensor memory, 64 columns a slot, and B in shared memory. A slot is a set's
// and two loading warps', and one pair of barriers serves both operands: an issuing warp's waits
// and commits take as long as the MMAs of few rows (100 to 150 cycles each). There are two issuing
// warps for the same reason, with the even and the odd stages of a unit and sums of their own,
// which the epilogue adds (even plus odd whichever warp has which: the same sums wherever a unit is;
// units of the other limit, of one issuing warp, and shared ones have other partial sums).
constexpr int kSlots = 4;
constexpr int kCodeSlots = 3;              // blocks of codes per warp, one of them in use
constexpr int kAcc0 = kSlots * 64;         // first column of the sums
static_assert(kSets == kSlots && kLoadWarps == 2 * kSlots, "a set and two loading warps per slot");
constexpr uint64_t kWaitNs = 1000000000ull;
constexpr int kSources = 1024;             // sorted rows whose sources are looked up once, together
constexpr int kPairStages = 24;
constexpr int kSched = 128;                // units of a CTA that are looked up once, together

__device__ DevErrRecord q4_fault;          // of every call on the device

// The groups that have rows and an expert, in order, and their first units.
struct Groups {
  int n;
  int limit;    // rows of a unit, at most
  int e[kMaxQ4Experts], r0[kMaxQ4Experts], r1[kMaxQ4Experts], first[kMaxQ4Experts];
};

// What this CTA does: its units, and of their stages those from `first` on.
struct Work {
  int units, first, blocks;
  int rank;      // in a pair that shares its unit: 0 or 1; else -1
};

struct __align__(16) Unit {
  int e, mt;      // expert, tile of outputs
  int r0, n;      // rows
};

// The source row of sorted row r, or -1: with its index divided, and from the table.
__device__ __forceinline__ int find_source(const Q4Args& a, int r) {
  const int p = __ldg(a.rows + r), t = p >= 0 ? p / a.k : -1;
  return t < a.T_x ? t : -1;
}

struct CodeSlot {
  uint4 codes[4][kQ4Rows];       // [32 inputs][row]
  uint16_t scales[kQ4Rows * 4];  // [row][group]
};

struct Smem {
  uint8_t b[kSlots][2][kUnitRows * 128];     // [slot][64 inputs], 1024-byte aligned
  CodeSlot code[kDeqWarps][kCodeSlots];
  float swap[2][16][66];                     // gates and ups of 16 rows, between the epilogue warps
  Unit sched[kSched];                        // the CTA's units, in its order
  Groups groups;
  uint64_t full[kSlots], empty[kSlots];      // of the ring's stages
  uint64_t d_full[2], d_empty[2], drain[kMmaWarps];
  uint64_t pair_ready, pair_full;            // the first CTA has room for the second's sums; has them
  uint32_t tmem;
  int4 warp_groups[kMaxQ4Experts / 32];      // of 32 groups: those with rows; rows; units by either limit
  int source[kSources];                      // row of x of the first sorted rows, or -1
};
static_assert(sizeof(Smem) <= 227 * 1024, "shared memory of a CTA");

__device__ __forceinline__ int source(const Q4Args& a, const Smem& sm, int r) {
  return a.rows == nullptr ? r : r < kSources ? sm.source[r] : find_source(a, r);
}

// Where there are at most half as many units as CTAs, a pair of CTAs shares one.
__device__ __forceinline__ bool share_units(int units, int ctas, bool paired) {
  return paired && units <= ctas / 2;
}
// The limit of a launch, from the units that there are with either (of `rows` rows and tiles in all): a
// stage of n rows takes about as long as (100 + n) / 0.44 ns, so the limit is the one whose turns
// (halves, in pairs) times that are less. (The two constants are fitted to these: 256 rows times 8192 x
// 8192, two turns with either, 51 us with 64 and 55 with 96; 2048 rows times 4096 x 4096, seven and
// five turns, 86 and 74.)
__device__ __forceinline__ float unit_cost(float rows, int units, int ctas, bool paired) {
  const uint32_t halves = share_units(units, ctas, paired) ? 1u : 2u * ((uint32_t)(units - 1) / (uint32_t)ctas + 1u);
  return (float)halves * (100.f + __fdividef(rows, (float)units));
}
__device__ __forceinline__ int unit_limit(float rows, int small_units, int large_units, int ctas,
                                          bool paired) {
  return small_units == large_units ||
                 unit_cost(rows, small_units, ctas, paired) <= unit_cost(rows, large_units, ctas, paired)
             ? kSmallUnitRows : kUnitRows;
}

// a matrix's tiles of a unit's outputs
__host__ __device__ __forceinline__ int unit_tiles(const Q4Shape& s, bool gated) {
  return gated ? (s.N + 63) / 64 : (s.N + 127) / 128;
}

// A group's rows are cut into parts of about the same size, each a unit per tile of outputs.
__device__ __forceinline__ Unit make_unit(int e, int r0, int r1, int parts, int m_tiles, int local) {
  const int part = local / m_tiles, per = (r1 - r0 + parts - 1) / parts;
  Unit u;
  u.e = e;
  u.mt = local - part * m_tiles;
  u.r0 = r0 + part * per;
  u.n = min(per, r1 - u.r0);
  return u;
}

// The groups with rows and an expert, this CTA's work, and its first units. Every thread has a group, and
// writes down those of its units that are this CTA's. (The caller synchronises the CTA after it.)
__device__ __forceinline__ Work find_work(const Q4Args& a, int m_tiles, int blocks, bool paired, Smem& sm) {
  Groups& s = sm.groups;
  const int u = threadIdx.x, lane = u & 31, warp = u >> 5, R = (int)a.R;
  static_assert(kThreads >= kMaxQ4Experts, "a thread per group");
  constexpr int kWarps = kMaxQ4Experts / 32;
  int e = u, r0 = 0, r1 = 0;
  if (u < a.n_groups) {
    r1 = R;
    if (a.offsets != nullptr) {
      r0 = __ldg(a.offsets + u);
      r1 = __ldg(a.offsets + u + 1);
    }
    if (a.expert_ids != nullptr) e = __ldg(a.expert_ids + u);
  }
  if (a.rows != nullptr)   // (while those loads are under way)
    for (int r = u; r < min(R, kSources); r += kThreads) sm.source[r] = find_source(a, r);
  r0 = max(r0, 0);
  r1 = min(r1, R);
  const bool live = r0 < r1 && e >= 0 && e < a.n_experts;
  const int size = live ? r1 - r0 : 0;
  const uint32_t m = __ballot_sync(0xffffffffu, live);
  // (the sums of the units over the groups fit: checked on the host)
  const int small_units = (size + kSmallUnitRows - 1) / kSmallUnitRows * m_tiles;
  const int large_units = (size + kUnitRows - 1) / kUnitRows * m_tiles;
  const int warp_small = __reduce_add_sync(0xffffffffu, small_units);
  const int warp_large = __reduce_add_sync(0xffffffffu, large_units);
  const int warp_rows = __reduce_add_sync(0xffffffffu, size);
  if (lane == 0 && warp < kWarps)
    sm.warp_groups[warp] = make_int4(__popc(m), warp_rows, warp_small, warp_large);
  __syncthreads();
  const int4 v = sm.warp_groups[lane & (kWarps - 1)];   // every warp adds them up
  const uint32_t all_lanes = 0xffffffffu;
  static_assert(kWarps <= 32 && (kWarps & (kWarps - 1)) == 0, "a lane per warp of groups");
  const bool counts = lane < kWarps, before = counts && lane < warp;
  const int all_small = __reduce_add_sync(all_lanes, counts ? v.z : 0);
  const int all_large = __reduce_add_sync(all_lanes, counts ? v.w : 0);
  const int rows = __reduce_add_sync(all_lanes, counts ? v.y : 0);
  const int limit = unit_limit((float)rows * (float)m_tiles, all_small, all_large, gridDim.x, paired);
  const bool small = limit == kSmallUnitRows;
  const int all = small ? all_small : all_large, units = small ? small_units : large_units;
  const int parts = (size + limit - 1) / limit;
  const int n = __reduce_add_sync(all_lanes, counts ? v.x : 0);
  const int at = __reduce_add_sync(all_lanes, before ? v.x : 0) + __popc(m & ((1u << lane) - 1u));
  int end = units;   // inclusive sum over the groups
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int k = __shfl_up_sync(all_lanes, end, o);
    if (lane >= o) end += k;
  }
  end += __reduce_add_sync(all_lanes, before ? small ? v.z : v.w : 0);
  Work w;
  const int ctas = gridDim.x, cta = blockIdx.x;
  int first = cta;   // this CTA's first unit; the others are `ctas` apart
  if (share_units(all, ctas, paired)) {
    w.rank = cta & 1;   // (CTAs 2p and 2p + 1 are a cluster)
    first = cta / 2;
    w.units = first < all ? 1 : 0;
    w.first = w.rank == 0 ? 0 : (blocks + 1) / 2;
    w.blocks = w.rank == 0 ? (blocks + 1) / 2 : blocks / 2;
  } else {
    w.rank = -1;
    w.units = all > cta ? (all - cta - 1) / ctas + 1 : 0;
    w.first = 0;
    w.blocks = blocks;
  }
  if (live) {
    const int begin = end - units;
    s.e[at] = e;
    s.r0[at] = r0;
    s.r1[at] = r1;
    s.first[at] = begin;
    for (int i = begin > first ? (begin - first + ctas - 1) / ctas : 0; i < min(kSched, w.units); ++i) {
      if (first + i * ctas >= end) break;
      sm.sched[i] = make_unit(e, r0, r1, parts, m_tiles, first + i * ctas - begin);
    }
  }
  if (u == 0) {
    s.n = n;
    s.limit = limit;
  }
  return w;
}

// the i-th unit of this CTA, which is there
__device__ __forceinline__ Unit unit_at(const Smem& sm, int m_tiles, int i) {
  if (i < kSched) return sm.sched[i];
  const Groups& s = sm.groups;
  const int unit = blockIdx.x + i * gridDim.x;
  int lo = 0, hi = s.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (s.first[mid] <= unit) lo = mid;
    else hi = mid - 1;
  }
  return make_unit(s.e[lo], s.r0[lo], s.r1[lo], (s.r1[lo] - s.r0[lo] + s.limit - 1) / s.limit, m_tiles,
                   unit - s.first[lo]);
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

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// The warp's number, as a value that the compiler knows to be the warp's: what depends on it (cursors,
// turns, loops) then takes the uniform datapath, not the pipe that the codes keep busy.
__device__ __forceinline__ int warp_number() { return __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0); }

// ------------------------------------------------------------------ dequantising
__device__ __forceinline__ void dequantise(const Q4Args& a, const Q4Shape& s, const Work& w, int m_tiles,
                                           Smem& sm, uint32_t tmem) {
  const int warp = warp_number() - kEpiWarps, set = warp >> 2, lane = threadIdx.x & 31;
  const int units = w.units, scale_block = s.scale_block();
  const int pieces = scale_block / 16;   // of the scales: a lane copies one, the first lanes
  const uint32_t ring = ptx::smem_addr(&sm.code[warp][0]) + lane * 16;
  constexpr uint32_t kSlot = sizeof(CodeSlot), kScales = offsetof(CodeSlot, scales);

  // The copies run ahead of the values by kCodeSlots - 1 blocks of this warp, over the ends of units.
  // base: stages of the units before; the set takes the stages whose number is set mod kSets.
  int unit = 0, base = 0, st = set;
  const uint8_t *codes = nullptr, *scales = nullptr;
  bool there = false;   // the warp's rows of this unit are in the matrix
  auto enter = [&]() {
    const Unit u = unit_at(sm, m_tiles, unit);
    const int m = a.gated ? (warp & 3) >> 1 : 0;
    const int tile = a.gated ? u.mt * 2 + (warp & 1) : u.mt * 4 + (warp & 3);
    there = tile < s.tiles;
    const size_t block = ((size_t)u.e * s.tiles + tile) * s.blocks + w.first + st;
    codes = static_cast<const uint8_t*>(a.codes[m]) + block * kQ4CodeBytes + lane * 16;
    scales = static_cast<const uint8_t*>(a.scales[m]) + block * scale_block + lane * 16;
  };
  uint32_t to = ring;
  auto copy = [&]() {   // the next block's copies, if there is one; always one group of copies
    while (st >= w.blocks && unit < units) {
      base += w.blocks;
      ++unit;
      st = (set - base) & (kSets - 1);
      if (st < w.blocks && unit < units) enter();
    }
    if (unit < units && there) {
#pragma unroll
      for (int h = 0; h < 4; ++h) copy16(to + h * kQ4Rows * 16, codes + h * kQ4Rows * 16, 16);
      if (lane < pieces) copy16(to + kScales, scales, 16);
    }
    copies_commit();
    codes += kSets * kQ4CodeBytes;
    scales += kSets * scale_block;
    st += kSets;
    to = to == ring + (kCodeSlots - 1) * kSlot ? ring : to + kSlot;
  };
  if (st < w.blocks && units > 0) enter();
#pragma unroll 1
  for (int i = 0; i < kCodeSlots - 1; ++i) copy();

  const uint32_t at = tmem + set * 64 + ((uint32_t)(warp & 3) << 21);   // (the set's slot)
  const Q4Bits bits;
  uint32_t turn = 1;
  int from = 0;
  // this set's stages: of units * blocks, those whose number is set mod kSets
  const int64_t all = (int64_t)units * w.blocks;
  const int visits = all > set ? (int)((all - set - 1) / kSets) + 1 : 0;
#pragma unroll 1
  for (int i = 0; i < visits; ++i) {
    copy();
    copies_wait<kCodeSlots - 1>();
    __syncwarp();   // (scales are copied by other lanes)
    const CodeSlot& slot = sm.code[warp][from];
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
    if (!__all_sync(0xffffffffu, wait<20>(&sm.empty[set], turn, 1))) break;
    ptx::tc_fence_after();
#pragma unroll
    for (int h = 0; h < 4; h += 2) {
      const uint32_t pair = h == 0 ? s01 : s23;
      const Q4Scale s0 = q4_scale_pair(pair), s1 = q4_scale_pair(pair >> 16);
      const uint4 c0 = slot.codes[h][lane], c1 = slot.codes[h + 1][lane];
      const uint32_t word[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
      uint32_t v[32];
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = q4_value_pair(word[j / 4], j & 3, j < 16 ? s0 : s1, bits);
      ptx::tmem_st32(at + h * 16, v);
    }
    ptx::tmem_st_wait();
    ptx::tc_fence_before();
    __syncwarp();   // (the slot has been read, too)
    if (lane == 0) ptx::mbar_arrive(&sm.full[set]);
    turn ^= 1u;
    from = from == kCodeSlots - 1 ? 0 : from + 1;
  }
  copies_wait<0>();
}

// ------------------------------------------------------------------ loading x
__device__ __forceinline__ void load_x(const Q4Args& a, const Q4Shape& s, const Work& w, int m_tiles,
                                       Smem& sm) {
  const int warp = warp_number() - kLoadWarp, slot = warp % kSlots, lane = threadIdx.x & 31;
  // 16 bytes of a row's 128, row of eight (the slot's warps have four of them each)
  const int chunk = lane & 7, sub = (lane >> 3) + warp / kSlots * 4;
  // (row r's 16-byte piece c is at r * 128 + (c ^ r % 8) * 16)
  const uint32_t dst = ptx::smem_addr(sm.b[slot][0]) + sub * 128 + ((chunk ^ sub) << 4);
  uint32_t turn = 1;
  int st = slot;   // this warp's next stage, counted from the unit's start
  for (int unit = 0; unit < w.units; ++unit, st -= w.blocks) {
    if (st >= w.blocks) continue;
    const Unit u = unit_at(sm, m_tiles, unit);
    // this lane's rows: sub, sub + 8, ... Their addresses are found once per unit (per stage it took
    // 2048 rows times 4096 x 4096 75 us, not 72.5).
    const __nv_bfloat16* from[kUnitRows / 8];
#pragma unroll
    for (int j = 0; j < kUnitRows / 32; ++j) {
      if (32 * j >= u.n) break;
      const int src = max(source(a, sm, u.r0 + min(32 * j + lane, u.n - 1)), 0);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        from[4 * j + i] = a.x + __shfl_sync(0xffffffffu, src, 8 * i + sub) * a.ldx + chunk * 8;
    }
    for (; st < w.blocks; st += kSlots) {
      // zeros behind n_in (where there is nothing to read, any address of x)
      const int k = (w.first + st) * 128, left = s.K - k - chunk * 8;
      const uint32_t in0 = left > 0 ? 16u : 0u, in1 = left > 64 ? 16u : 0u;
      const int k0 = in0 ? k : 0, k1 = in1 ? k + 64 : 0;
      if (!__all_sync(0xffffffffu, wait<20>(&sm.empty[slot], turn, 2))) return;
      turn ^= 1u;
#pragma unroll
      for (int i = 0; i < kUnitRows / 8; ++i) {
        if (8 * i >= u.n) break;
        if (8 * i + sub < u.n) {
          copy16(dst + 8 * i * 128, from[i] + k0, in0);
          copy16(dst + 8 * i * 128 + kUnitRows * 128, from[i] + k1, in1);
        }
      }
      copies_commit();
      copies_wait<0>();
      ptx::fence_proxy_async_smem();   // (the tensor pipe reads them)
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&sm.full[slot]);
    }
  }
}

// ------------------------------------------------------------------ issuing the MMAs
// Issuing warps: with more than 64 rows the MMAs take longer than their issue, and one warp does all (two
// buffers of both warps' sums would not fit). With one for few rows too, 256 rows for 104 experts
// took 22.8 us, not 21.3, and 64 rows times 8192 x 8192 24.4, not 24.1.
__device__ __forceinline__ int mma_warps(int limit) { return limit == kSmallUnitRows ? 2 : 1; }
__device__ __forceinline__ uint32_t acc_column(int warps, int buffer, int warp) {
  return kAcc0 + buffer * 128 + (warps == 2 ? warp * 64 : 0);
}

// The whole warp goes through its stages and elects the lane that issues: with one lane in a branch of
// its own the operands were not uniform, and eight MMAs took 600 cycles to issue instead of 150. One
// warp's instructions take five cycles and more each here, and these warps' are the ring's
// pace: the slots are unrolled, so that addresses are constants.
template <int kWarps>
__device__ __forceinline__ void issue(const Work& w, int m_tiles, Smem& sm, uint32_t tmem, int warp) {
  const uint64_t ring = ptx::sdesc_k_sw128(ptx::smem_addr(sm.b[warp]));
  constexpr uint32_t kBlock16 = kUnitRows * 128 / 16;   // (a descriptor's address is in units of 16 bytes)
  const uint32_t a0 = tmem + warp * 64;
  uint64_t* const full = sm.full + warp;
  uint64_t* const empty = sm.empty + warp;
  int unit = 0, left = 0;   // this warp's stages left of the unit
  uint32_t d = 0, idesc = 0, full_turn = 0;
  bool odd = false, ok = true;   // odd: the units before this one have an odd number of stages
  Slot acc;
  uint64_t* d_full = nullptr;
  while (ok) {
#pragma unroll
    for (int i = 0; i < kSlots; i += kWarps) {
      bool first = false;
      while (left == 0) {   // (a unit of one stage may have none of this warp's)
        if (unit == w.units || !__all_sync(0xffffffffu, wait<0>(&sm.d_empty[acc.i], acc.turn ^ 1u, 3))) {
          ok = false;
          break;
        }
        idesc = ptx::idesc_bf16(128, (unit_at(sm, m_tiles, unit).n + 15) / 16 * 16);
        d = tmem + acc_column(kWarps, acc.i, warp);
        d_full = &sm.d_full[acc.i];
        left = kWarps == 1 ? w.blocks : (w.blocks + ((warp != 0) == odd ? 1 : 0)) / 2;
        odd ^= w.blocks & 1;
        first = true;
        ++unit;
        acc.next(2);
        // (for the other warp's part of the sums, or for none)
        if ((left == 0 || kWarps == 1) && ptx::elect_one()) ptx::mbar_arrive(d_full);
        __syncwarp();
      }
      if (!ok) break;
      if (!__all_sync(0xffffffffu, wait<0>(full + i, full_turn, 4))) {
        ok = false;
        break;
      }
      ptx::tc_fence_after();
      if (ptx::elect_one()) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          ptx::mma_bf16_ta(d, a0 + i * 64 + j * 8,
                           ring + (i * 2 + j / 4) * kBlock16 + (j & 3) * 2, idesc, !first || j != 0);
        ptx::mma_commit(empty + i);
        if (left == 1) ptx::mma_commit(d_full);
      }
      __syncwarp();
      --left;
    }
    full_turn ^= 1u;
  }
  // everything issued has been done before the CTA gives its memory back
  if (ptx::elect_one()) ptx::mma_commit(&sm.drain[warp]);
  wait<0>(&sm.drain[warp], 0, 6);
}

// ------------------------------------------------------------------ epilogue
__device__ __forceinline__ void store_y(uint8_t* y, bool fp32, float v) {
  if (fp32) *reinterpret_cast<float*>(y) = v;
  else *reinterpret_cast<__nv_bfloat16*>(y) = __float2bfloat16_rn(v);
}

// Waits for the pair's other CTA (once per launch).
__device__ __forceinline__ bool wait_pair(uint64_t* bar, int where) {
  uint64_t t0 = 0;
  for (uint32_t i = 1; !ptx::mbar_try_wait_cluster(bar, 0); ++i)
    if ((i & 255u) == 0u) {
      const uint64_t now = ptx::globaltimer_ns();
      if (t0 == 0) t0 = now;
      else if (now - t0 > kWaitNs) {
        record_error(&q4_fault, kErrTimeout, kAtQ4, where);
        return false;
      }
    }
  return true;
}

template <bool kGated>
__device__ __forceinline__ void epilogue(const Q4Args& a, const Q4Shape& s, const Work& w, int m_tiles,
                                         Smem& sm, uint32_t tmem) {
  const int warp = warp_number(), lane = threadIdx.x & 31, row = threadIdx.x;   // row: lane of tensor memory
  const int warps = mma_warps(sm.groups.limit);
  const int size = a.y_fp32 ? 4 : 2;
  const int64_t step = a.ldy * size;
  const bool pairs = ((reinterpret_cast<uintptr_t>(a.y) | (uint64_t)step) & (2 * size - 1)) == 0;
  Slot acc;
  bool odd = false;   // the units before have an odd number of stages
  for (int turn = 0; turn < w.units; ++turn, acc.next(2), odd ^= w.blocks & 1) {
    const Unit u = unit_at(sm, m_tiles, turn);
    uint32_t missing[kUnitRows / 32] = {};   // rows without a source: zeros
    if (a.rows != nullptr) {
#pragma unroll
      for (int j = 0; j < kUnitRows / 32; ++j) {
        const int r = 32 * j + (row & 31);
        missing[j] = __ballot_sync(0xffffffffu, r < u.n && source(a, sm, u.r0 + r) < 0);
      }
    }
    if (!ptx::epi_all(wait<100>(&sm.d_full[acc.i], acc.turn, 7))) break;
    ptx::tc_fence_after();
    // A shared unit: x's ring, whose stages have all been used, takes the other CTA's sums, [row][output].
    float* const theirs = reinterpret_cast<float*>(sm.b);
    if (w.rank == 0) {
      if (row == 0) ptx::mbar_arrive_cluster(ptx::peer_smem(&sm.pair_ready, 1));
      if (!ptx::epi_all(wait_pair(&sm.pair_full, 9))) break;
    } else if (w.rank == 1) {
      if (!ptx::epi_all(wait_pair(&sm.pair_ready, 10))) break;
    }
    const uint32_t to = w.rank == 1 ? ptx::peer_smem(theirs, 0) + row * 4 : 0u;
    const uint32_t from =
        tmem + acc_column(warps, acc.i, w.blocks == 1 && odd ? 1 : 0) + ((uint32_t)warp << 21);
    for (int c0 = 0; c0 < u.n; c0 += 16) {
      const int count = min(16, u.n - c0);   // (few rows: what is done is cut to fours of them)
      float v[16];
      ptx::tmem_ld16(from + c0, v);
      if (warps == 2 && w.blocks > 1) {
        float o[16];
        ptx::tmem_ld16(from + 64 + c0, o);
        ptx::tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] += o[j];
      } else {
        ptx::tmem_ld_wait();
      }
      if (w.rank == 1) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          if ((j & 3) == 0 && j >= count) break;
          ptx::st_cluster_f32(to + (c0 + j) * 512, v[j]);
        }
        continue;
      }
      if (w.rank == 0) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          if ((j & 3) == 0 && j >= count) break;
          v[j] += theirs[(c0 + j) * 128 + row];
        }
      }
      const uint32_t zero = (c0 < 32 ? missing[0] : c0 < 64 ? missing[1] : missing[2]) >> (c0 & 16);
      if (kGated) {
        // lanes 0 .. 63 are gates, 64 .. 127 ups; then a warp does every fourth row, a lane two outputs
        const int up = row >> 6;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          if ((j & 3) == 0 && j >= count) break;
          sm.swap[up][j][row & 63] = v[j];
        }
        ptx::named_bar_sync(1, 32 * kEpiWarps);
        float g[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float2 p = make_float2(0.f, 0.f);
          if (warp + 4 * i < count) p = *reinterpret_cast<const float2*>(&sm.swap[0][warp + 4 * i][2 * lane]);
          g[2 * i] = p.x;
          g[2 * i + 1] = p.y;
        }
        silu_all(g);
        const int first = u.mt * 64 + 2 * lane;
        uint8_t* y = static_cast<uint8_t*>(a.y) + (int64_t)(u.r0 + c0 + warp) * step + (int64_t)first * size;
#pragma unroll
        for (int i = 0; i < 4; ++i, y += 4 * step) {
          const int r = warp + 4 * i;
          if (r >= count) break;
          const float2 p = *reinterpret_cast<const float2*>(&sm.swap[1][r][2 * lane]);
          const bool none = zero >> r & 1u;
          const float o0 = none ? 0.f : g[2 * i] * p.x, o1 = none ? 0.f : g[2 * i + 1] * p.y;
          if (pairs && first + 1 < s.N) {
            if (a.y_fp32) *reinterpret_cast<float2*>(y) = make_float2(o0, o1);
            else *reinterpret_cast<__nv_bfloat162*>(y) = __floats2bfloat162_rn(o0, o1);
          } else {
            if (first < s.N) store_y(y, a.y_fp32, o0);
            if (first + 1 < s.N) store_y(y + size, a.y_fp32, o1);
          }
        }
        ptx::named_bar_sync(1, 32 * kEpiWarps);
      } else {
        uint8_t* y = static_cast<uint8_t*>(a.y) + (int64_t)(u.r0 + c0) * step + (int64_t)(u.mt * 128 + row) * size;
        const bool there = u.mt * 128 + row < s.N;
#pragma unroll
        for (int j = 0; j < 16; ++j, y += step) {
          if ((j & 3) == 0 && j >= count) break;
          if (j < count && there) store_y(y, a.y_fp32, zero >> j & 1u ? 0.f : v[j]);
        }
      }
    }
    if (w.rank == 1) ptx::mbar_arrive_cluster(ptx::peer_smem(&sm.pair_full, 0));
    ptx::tc_fence_before();
    ptx::mbar_arrive(&sm.d_empty[acc.i]);
  }
}

// One kernel for plain and gated products: a layer's launches then share their code in the SMs' instruction
// caches. (Two kernels, one after the other, took 19.2 us, not 18.2, for a decoding block's gate and up
// and down products, and a layer of one token 33.5, not 31.8.)
__global__ void __launch_bounds__(kThreads, 1)
q4_kernel(const __grid_constant__ Q4Args a, const __grid_constant__ Q4Shape s, const bool paired) {
  extern __shared__ __align__(1024) uint8_t raw[];
  Smem& sm = *reinterpret_cast<Smem*>(raw);
  const int warp = warp_number();
  if (warp == kMmaWarp) {
    ptx::tmem_alloc(&sm.tmem, 512);
    ptx::tmem_relinquish();
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < kSlots; ++i) {
      // the set's warps and the loading ones (and with dmoe_q4_set_debug_hold one that never comes)
      ptx::mbar_init(&sm.full[i], 4 + 2 + a.hold);
      ptx::mbar_init(&sm.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(&sm.d_full[i], kMmaWarps);
      ptx::mbar_init(&sm.d_empty[i], 32 * kEpiWarps);
    }
    for (int i = 0; i < kMmaWarps; ++i) ptx::mbar_init(&sm.drain[i], 1);
    ptx::mbar_init(&sm.pair_ready, 1);
    ptx::mbar_init(&sm.pair_full, 32 * kEpiWarps);
    ptx::fence_mbarrier_init();
  }
  ptx::tc_fence_before();
  pdl_wait();
  pdl_launch_dependents();
  const int m_tiles = unit_tiles(s, a.gated);
  const Work w = find_work(a, m_tiles, s.blocks, paired, sm);
  // (a pair's barriers are there before the other CTA arrives on them, and until it has)
  if (w.rank >= 0) {
    ptx::cluster_arrive();
    ptx::cluster_wait();
  } else {
    __syncthreads();
  }
  ptx::tc_fence_after();
  const uint32_t tmem = sm.tmem;
  const int issuers = mma_warps(sm.groups.limit);
  if (warp < kEpiWarps && a.gated) epilogue<true>(a, s, w, m_tiles, sm, tmem);
  else if (warp < kEpiWarps) epilogue<false>(a, s, w, m_tiles, sm, tmem);
  else if (warp < kLoadWarp) dequantise(a, s, w, m_tiles, sm, tmem);
  else if (warp < kMmaWarp) load_x(a, s, w, m_tiles, sm);
  else if (issuers == 2) issue<2>(w, m_tiles, sm, tmem, warp - kMmaWarp);
  else if (warp == kMmaWarp) issue<1>(w, m_tiles, sm, tmem, 0);
  __syncwarp();
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) ptx::tmem_dealloc(tmem, 512);
  if (w.rank >= 0) {
    ptx::cluster_arrive();
    ptx::cluster_wait();
  }
}

}  // namespace

cudaError_t launch_q4_linear(const Q4Args& a, const dmoe_q4_desc& d, cudaStream_t st) {
  const Q4Shape s = q4_shape(d);
  static std::atomic<uint32_t> ready{0};   // a bit per device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  const uint32_t bit = dev < 32 ? 1u << dev : 0u;
  if (e == cudaSuccess && (ready.load(std::memory_order_acquire) & bit) == 0u) {
    e = cudaFuncSetAttribute(q4_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(Smem));
    if (e == cudaSuccess) ready.fetch_or(bit, std::memory_order_release);
  }
  if (e != cudaSuccess) return e;
  // at most as many CTAs as units there can be, and as run at once
  const int64_t groups = a.n_groups < a.R ? a.n_groups : a.R;
  const int64_t tiles = unit_tiles(s, a.gated);
  const int64_t units = (groups + a.R / kSmallUnitRows) * tiles;
  const int sms = device_sm_count();
  if (s.blocks >= kPairStages && 2 * tiles <= sms)
    return launch_cluster(q4_kernel, dim3((unsigned)(2 * (units < sms / 2 ? units : sms / 2))),
                          dim3(kThreads), sizeof(Smem), st, 2, true, a, s, true);
  return launch_ex(q4_kernel, dim3((unsigned)(units < sms ? units : sms)), dim3(kThreads), sizeof(Smem),
                   st, true, a, s, false);
}

cudaError_t q4_fault_address(void** p) { return cudaGetSymbolAddress(p, q4_fault); }

}  // namespace dmoe

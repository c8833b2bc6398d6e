// Products of sorted rows with their experts' 4-bit matrices, plain or gate and up with SwiGLU:
// y^T = W x^T, per unit of 128 outputs (or 64 gate and 64 up outputs) and at most 128 rows of a group.
//
// A persistent CTA per SM, in roles:
//   dequantising warps (four sets of four, in turn): a lane has a row of W. Its codes come by
//       asynchronous copies into a ring of its own, become bf16 values by one exact FMA per pair
//       and go to tensor memory: the A operand of the MMAs. Through shared memory they would take
//       four times the codes' bytes twice, and 4 KB of codes have 184 cycles of an SM's share of
//       HBM's rate, in which shared memory moves 23 KB.
//   loading warps: the rows of x that the group names, a stage each in turn, by copies of 16 bytes
//       into shared memory (B). Between the copies and the tensor pipe's reads is a fence of 350
//       to 1000 cycles, so as many stages are under way as there are loading warps. (TMA gathers of
//       four rows need no fence, but took 80 cycles each: 64 rows 2500 cycles a stage.)
//   an issuing warp: tcgen05.mma, M = 128 outputs, N = the unit's rows in sixteens
//   epilogue warps: sums from tensor memory, SwiGLU, y
// Few rows: the weights' bytes are the bound, and the arithmetic on the codes is close to it (32
// pairs a row and 64 inputs, 2.75 operations each). Many rows: the tensor pipe.
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
// A stage is 128 inputs: two blocks of 64.
constexpr int kASlots = 4;                 // stages of A in tensor memory, 64 columns each
constexpr int kBRing = 128 * 1024;         // bytes of the ring of x's stages
constexpr int kBSlotsMax = 8;
constexpr int kCodeSlots = 2;              // stages of codes per set, one of them in use
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

struct Smem {
  uint8_t b[kBRing];                                       // 1024-byte aligned
  uint4 codes[kSets][kCodeSlots][4][128];                      // [set][slot][32 inputs][row]
  uint4 scales[kSets][kCodeSlots][128];                    // eight groups of a row
  float swap[2][2][64][9];                                 // ups and gates between epilogue warps
  Unit sched[kSched];                                      // the CTA's units, in its order
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

__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, int where) {
  if (ptx::mbar_wait_long(bar, parity, kWaitNs)) return true;
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

__device__ __forceinline__ int stages_of(const Q4Shape& s) { return (s.k_tiles + 1) / 2; }

// ------------------------------------------------------------------ dequantising
// The place of a row's next codes and scales: copies run ahead of the values by kCodeSlots - 1 stages
// of the set, over the ends of units.
template <bool kGated>
struct CodeCursor {
  int unit, st, base;   // unit of the CTA; base: stages of the units before this one
  int piece;            // of eight groups' scales, of the stage before
  const uint8_t* codes; // of this row, stage st
  const uint8_t* scales;
  int half;             // bytes from half block to half block
  bool row;             // this row is there
  __device__ __forceinline__ void enter(const Q4Args& a, const Q4Shape& s, const Smem& sm, int units,
                                        int m_tiles, int set, int lane_row) {
    st = (set - base) & (kSets - 1);
    piece = -1;
    if (unit >= units) return;
    const Unit u = unit_at(sm, m_tiles, unit);
    const int m = kGated ? lane_row >> 6 : 0;
    const int n = kGated ? u.mt * 64 + (lane_row & 63) : u.mt * 128 + lane_row;
    row = n < s.rows;
    if (!row) return;
    half = s.tile_rows(n) * 16;
    codes = static_cast<const uint8_t*>(a.codes[m]) + u.e * s.code_bytes() + s.code_at(n, 2 * st, 0);
    scales = static_cast<const uint8_t*>(a.scales[m]) + ((size_t)u.e * s.rows + n) * s.groups_pad * 2;
  }
};

template <bool kGated>
__device__ __forceinline__ void dequantise(const Q4Args& a, const Q4Shape& s, int m_tiles, Smem& sm,
                                           uint32_t tmem) {
  const int warp = threadIdx.x / 32 - kEpiWarps, set = warp >> 2;
  const int lane_row = threadIdx.x & 127;   // (each set: lanes 0 .. 127 of tensor memory)
  const int stages = stages_of(s), units = units_of_cta(sm.groups);
  const int per_piece = s.group == 32 ? 1 : s.group == 64 ? 2 : 3;   // log2 of stages per piece
  const uint32_t codes_at = ptx::smem_addr(&sm.codes[set][0][0][lane_row]);
  const uint32_t scales_at = ptx::smem_addr(&sm.scales[set][0][lane_row]);
  constexpr int kSlot = sizeof(sm.codes[0][0]), kHalf = sizeof(sm.codes[0][0][0]);
  CodeCursor<kGated> c;
  c.unit = 0;
  c.base = 0;
  c.enter(a, s, sm, units, m_tiles, set, lane_row);
  int copy_slot = 0, copy_piece = 0;
  auto copy = [&]() {
    while (c.unit < units && c.st >= stages) {
      c.base += stages;
      ++c.unit;
      c.enter(a, s, sm, units, m_tiles, set, lane_row);
    }
    if (c.unit < units) {
      const int piece = c.st >> per_piece;
      if (c.row) {
        const uint32_t dst = codes_at + copy_slot * kSlot;
        copy16(dst, c.codes);
        copy16(dst + kHalf, c.codes + c.half);
        if (2 * c.st + 1 < s.k_tiles) {
          copy16(dst + 2 * kHalf, c.codes + 2 * c.half);
          copy16(dst + 3 * kHalf, c.codes + 3 * c.half);
        }
        if (piece != c.piece) copy16(scales_at + copy_piece * kHalf, c.scales + piece * 16);
        c.codes += kSets * 4 * c.half;
      }
      if (piece != c.piece) copy_piece = (copy_piece + 1) % kCodeSlots;
      c.piece = piece;
      copy_slot = (copy_slot + 1) % kCodeSlots;
      c.st += kSets;
    }
    copies_commit();
  };
  for (int i = 0; i < kCodeSlots - 1; ++i) copy();
  int base = 0, slot = 0, next_piece = 0;
  bool ok = true;
  for (int unit = 0; ok && unit < units; ++unit, base += stages) {
    int piece = -1;
    uint4 sc = make_uint4(0, 0, 0, 0);
    for (int st = (set - base) & (kSets - 1); st < stages; st += kSets) {
      copy();
      copies_wait<kCodeSlots - 1>();
      if (st >> per_piece != piece) {
        piece = st >> per_piece;
        sc = sm.scales[set][next_piece][lane_row];
        next_piece = (next_piece + 1) % kCodeSlots;
      }
      // the scales of the stage's four halves of blocks, in pairs
      uint32_t p0, p1;
      if (s.group == 32) {
        p0 = st & 1 ? sc.z : sc.x;
        p1 = st & 1 ? sc.w : sc.y;
      } else {
        const int w = s.group == 64 ? st & 3 : (st & 7) >> 1;
        const uint32_t pair = w & 2 ? (w & 1 ? sc.w : sc.z) : (w & 1 ? sc.y : sc.x);
        p0 = __byte_perm(pair, 0u, s.group == 128 && (st & 1) ? 0x3232 : 0x1010);
        p1 = s.group == 64 ? __byte_perm(pair, 0u, 0x3232) : p0;
      }
      const int stage = base + st, as = stage % kASlots;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        if (b == 1 && 2 * st + 1 >= s.k_tiles) break;
        const uint4 c0 = sm.codes[set][slot][2 * b][lane_row], c1 = sm.codes[set][slot][2 * b + 1][lane_row];
        const Q4Scale s0 = q4_scale_pair(b == 0 ? p0 : p1), s1 = q4_scale_pair((b == 0 ? p0 : p1) >> 16);
        const uint32_t w[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
        uint32_t v[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = q4_value_pair(w[i / 4], i & 3, i < 16 ? s0 : s1);
        if (b == 0) {
          ok = wait(&sm.a_empty[as], ((stage / kASlots) & 1) ^ 1, 1);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          ptx::tc_fence_after();
        }
        ptx::tmem_st32(tmem + as * 64 + b * 32 + ((uint32_t)(warp & 3) << 21), v);
      }
      if (!ok) break;
      slot = (slot + 1) % kCodeSlots;
      ptx::tmem_st_wait();
      ptx::tc_fence_before();
      __syncwarp();
      if ((threadIdx.x & 31) == 0) ptx::mbar_arrive(&sm.a_full[as]);
    }
  }
  copies_wait<0>();
}

// ------------------------------------------------------------------ loading x
// The source row of sorted row r, or -1.
__device__ __forceinline__ int source(const Q4Args& a, int r) {
  if (a.rows == nullptr) return r;
  const int p = __ldg(a.rows + r), t = p >= 0 ? p / a.k : -1;
  return t < a.T_x ? t : -1;
}

__device__ __forceinline__ void load_x(const Q4Args& a, const Q4Shape& s, int m_tiles, Smem& sm,
                                       int b_slots) {
  const int warp = threadIdx.x / 32 - kLoadWarp, lane = threadIdx.x & 31;
  const int chunk = lane & 7, sub = lane >> 3;   // 16 bytes of a row's 128, row of four
  const int stages = stages_of(s), units = units_of_cta(sm.groups), block_bytes = sm.groups.widest * 128;
  const uint32_t ring = ptx::smem_addr(sm.b);
  int stage = 0;
  bool ok = true;
  for (int unit = 0; ok && unit < units; ++unit) {
    const int base = stage;
    stage += stages;
    int st = (warp - base) & (kLoadWarps - 1);   // this warp's first stage of the unit
    if (st >= stages) continue;
    const Unit u = unit_at(sm, m_tiles, unit);
    int src[kUnitRows / 32];                     // of rows lane, lane + 32, ...
#pragma unroll
    for (int j = 0; j < kUnitRows / 32; ++j)
      src[j] = 32 * j < u.n ? max(source(a, u.r0 + min(32 * j + lane, u.n - 1)), 0) : 0;
    for (; st < stages; st += kLoadWarps) {
      const int bs = (base + st) % b_slots;
      ok = __all_sync(0xffffffffu, wait(&sm.b_empty[bs], (((base + st) / b_slots) & 1) ^ 1, 2));
      if (!ok) break;
      // (row r's 16-byte piece c is at r * 128 + (c ^ r % 8) * 16)
      const uint32_t dst = ring + bs * 2 * block_bytes + sub * 128;
      const __nv_bfloat16* x = a.x + st * 128 + chunk * 8;
      const uint32_t in0 = st * 128 + chunk * 8 < s.K ? 16u : 0u;        // (zeros behind n_in)
      const uint32_t in1 = st * 128 + 64 + chunk * 8 < s.K ? 16u : 0u;
#pragma unroll
      for (int j = 0; j < kUnitRows / 32; ++j) {
        if (32 * j >= u.n) break;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int r = 32 * j + 4 * i + sub;
          const int64_t at = __shfl_sync(0xffffffffu, src[j], 4 * i + sub) * a.ldx;
          if (r < u.n) {
            const uint32_t to = dst + (32 * j + 4 * i) * 128 + ((chunk ^ ((4 * i + sub) & 7)) << 4);
            copy16(to, in0 ? x + at : a.x, in0);
            if (2 * st + 1 < s.k_tiles) copy16(to + block_bytes, in1 ? x + at + 64 : a.x, in1);
          }
        }
      }
      copies_commit();
      copies_wait<0>();
      ptx::fence_proxy_async_smem();   // (the tensor pipe reads them)
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&sm.b_full[bs]);
    }
  }
}

// ------------------------------------------------------------------ issuing the MMAs
__device__ __forceinline__ void issue(const Q4Shape& s, int m_tiles, Smem& sm, uint32_t tmem,
                                      int b_slots) {
  const int stages = stages_of(s), units = units_of_cta(sm.groups), block_bytes = sm.groups.widest * 128;
  const uint32_t ring = ptx::smem_addr(sm.b);
  int stage = 0;
  bool ok = true;
  for (int turn = 0; ok && turn < units; ++turn) {
    const Unit u = unit_at(sm, m_tiles, turn);
    const uint32_t idesc = ptx::idesc_bf16(128, (u.n + 15) / 16 * 16);
    const int buf = turn & 1;
    const uint32_t d = tmem + kAcc0 + buf * 128;
    ok = __all_sync(0xffffffffu, wait(&sm.d_empty[buf], ((turn >> 1) & 1) ^ 1, 3));
    for (int st = 0; ok && st < stages; ++st, ++stage) {
      const int as = stage % kASlots, bs = stage % b_slots;
      ok = wait(&sm.b_full[bs], (stage / b_slots) & 1, 4) && wait(&sm.a_full[as], (stage / kASlots) & 1, 5);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      ptx::tc_fence_after();
      const uint64_t b0 = ptx::sdesc_k_sw128(ring + bs * 2 * block_bytes);
      if (ptx::elect_one()) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          if (b == 1 && 2 * st + 1 >= s.k_tiles) break;
#pragma unroll
          for (int j = 0; j < 4; ++j)   // (a descriptor's address is in units of 16 bytes)
            ptx::mma_bf16_ta(d, tmem + as * 64 + b * 32 + j * 8, b0 + b * (block_bytes >> 4) + j * 2, idesc,
                             (st | b | j) != 0);
        }
        ptx::mma_commit(&sm.a_empty[as]);
        ptx::mma_commit(&sm.b_empty[bs]);
        if (st == stages - 1) ptx::mma_commit(&sm.d_full[buf]);
      }
      __syncwarp();
    }
  }
  // everything issued has been done before the CTA gives its memory back
  if (ptx::elect_one()) ptx::mma_commit(&sm.drain);
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
    if (!ptx::epi_all(wait(&sm.d_full[buf], (turn >> 1) & 1, 7))) break;
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
    for (int i = 0; i < kASlots; ++i) {
      ptx::mbar_init(&sm.a_full[i], kDeqWarps / kSets);
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
  // (a multiple of the loading warps: a slot's stages are one warp's, so that no warp waits for a
  // slot two turns ahead of another)
  static_assert(kBRing == kBSlotsMax * 64 * 256 && kBSlotsMax == 2 * kLoadWarps && kASlots == kSets, "rings");
  const int b_slots = sm.groups.widest <= 64 ? kBSlotsMax : kBSlotsMax / 2;
  if (warp < kEpiWarps) epilogue<kGated>(a, s, m_tiles, sm, tmem);
  else if (warp < kLoadWarp) dequantise<kGated>(a, s, m_tiles, sm, tmem);
  else if (warp == kMmaWarp) issue(s, m_tiles, sm, tmem, b_slots);
  else load_x(a, s, m_tiles, sm, b_slots);
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

// Tokens sorted by expert: a stable counting sort of the R = T k (token, slot) pairs over E + 1
// keys (the experts, and last the pairs without one).
//   sort_count_kernel  pairs per key of each chunk of pairs, one CTA per chunk
//   sort_place_kernel  every CTA adds up, per key, the pairs before its chunk and all of them, and
//                      goes through its chunk a tile of pairs at a time: per warp the pairs of each
//                      key by votes of the warp's lanes, a prefix over the warps, and each
//                      pair's row is its key's base, the pairs of its key in the warps before its
//                      own and those before it in its warp.
// Up to 1024 pairs take the second launch alone: 8 pairs 2.5 us, 256 2.8, 1024 4.5 (with both 5.9, 6.0
// and 6.4 us); 4096 pairs 7.0 us, 131072 10.2, 524288 of cold ids 16.2 (256 experts). Bound by the
// launches and by the chain of loads, votes, prefixes and stores: the bytes of 524288 pairs would
// take 0.9 us.
// Every count is an integer sum: the order does not depend on the order of atomics.
#include "block_reduce.cuh"
#include "dmoe_internal.cuh"

namespace dmoe {
namespace {

constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortRounds = 4;                          // pairs per thread and tile, at most
constexpr int kSortTile = kSortThreads * kSortRounds;
constexpr int kSortMaxChunks = 148;                     // every CTA of one wave takes one chunk
// A chunk of at most 60 K pairs has counts of 16 bits; larger ones have 32, and a few chunks less.
constexpr int64_t kNarrowPairs = (int64_t)kSortMaxChunks * 60 * kSortThreads;
constexpr int kWideChunks = 144;
constexpr int kMaxKeys = kMaxExperts + 1;
constexpr int kKeyBits = 9;
static_assert(kMaxExperts < 1 << kKeyBits, "the bits of a key");

__device__ __forceinline__ int sort_key(int id, int E) { return id < 0 || id >= E ? E : id; }

template <typename Count>
__global__ void __launch_bounds__(kSortThreads)
sort_count_kernel(const int32_t* __restrict__ ids, int64_t R, int E, int64_t chunk,
                  Count* __restrict__ counts) {
  __shared__ int cnt[kMaxKeys];
  const int tid = threadIdx.x;
  pdl_wait();
  pdl_launch_dependents();
  if (tid <= E) cnt[tid] = 0;
  __syncthreads();
  const int64_t begin = blockIdx.x * chunk, end = begin + chunk < R ? begin + chunk : R;
  for (int64_t i0 = begin + tid; i0 < end; i0 += kSortTile) {
    int id[kSortRounds];
#pragma unroll
    for (int j = 0; j < kSortRounds; ++j)
      id[j] = i0 + j * kSortThreads < end ? __ldcg(ids + i0 + j * kSortThreads) : 0;
#pragma unroll
    for (int j = 0; j < kSortRounds; ++j)
      if (i0 + j * kSortThreads < end) atomicAdd(&cnt[sort_key(id[j], E)], 1);
  }
  __syncthreads();
  if (tid <= E) counts[(size_t)blockIdx.x * (E + 1) + tid] = (Count)cnt[tid];
}

// A key's counts over the chunks: [0] all of them, [1] those before this CTA's. Three groups of threads
// take a third of the chunks each, 16 loads at a time.
constexpr int kSumGroups = 3;
static_assert(kSumGroups * kMaxKeys <= kSortThreads, "a thread per key and group");

// The warp's lanes with this lane's key (at most `bits` bits, or -1), by a vote per bit: they take less than
// one match over the warp, whose time goes by the number of different keys (1024 pairs, 256 experts: 4.5 us, not 5.1).
__device__ __forceinline__ uint32_t same_key(int key, int bits) {
  uint32_t same = __ballot_sync(0xffffffffu, key >= 0);
#pragma unroll
  for (int b = 0; b < kKeyBits; ++b) {
    if (b >= bits) break;
    const bool set = key >> b & 1;
    const uint32_t m = __ballot_sync(0xffffffffu, set);
    same &= set ? m : ~m;
  }
  return same;
}

// `rounds` pairs a thread and tile (the tile has rounds * blockDim.x pairs, a warp's are consecutive)
template <typename Count>
__global__ void __launch_bounds__(kSortThreads)
sort_place_kernel(const int32_t* __restrict__ ids, int64_t R, int E, int64_t chunk, int nchunks,
                  int rounds, const Count* __restrict__ counts, int32_t* __restrict__ offsets,
                  int32_t* __restrict__ rows, int32_t* __restrict__ pos, DevErrRecord* err) {
  __shared__ int cnt[kSortWarps][kMaxKeys];   // per warp and key: pairs, then the first row
  __shared__ int base[kMaxKeys];              // per key: the next tile's first row
  __shared__ int sums[2][kMaxKeys];           // per key: pairs of all chunks, and of those before
  __shared__ int iscr[32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, keys = E + 1;
  const int threads = blockDim.x, warps = threads >> 5, bits = 32 - __clz(E);
  const int64_t begin = blockIdx.x * chunk, end = begin + chunk < R ? begin + chunk : R;
  for (int i = tid; i < 2 * kMaxKeys; i += threads) (&sums[0][0])[i] = 0;
  for (int i = lane; i < keys; i += 32) cnt[warp][i] = 0;
  pdl_wait();
  pdl_launch_dependents();
  if (nchunks > 0) {
    __syncthreads();
    const int group = tid / keys, key = tid - group * keys;
    if (group < kSumGroups) {
      const int per = (nchunks + kSumGroups - 1) / kSumGroups, c1 = min(nchunks, (group + 1) * per);
      int all = 0, before = 0;
      for (int c0 = group * per; c0 < c1; c0 += 16) {
        int n[16];
#pragma unroll
        for (int j = 0; j < 16; ++j)
          n[j] = c0 + j < c1 ? __ldcg(counts + (size_t)(c0 + j) * keys + key) : 0;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          all += n[j];
          before += c0 + j < (int)blockIdx.x ? n[j] : 0;
        }
      }
      atomicAdd(&sums[0][key], all);
      atomicAdd(&sums[1][key], before);
    }
  }
  const int64_t tile = (int64_t)rounds * threads;
  for (int64_t t0 = begin; t0 == begin || t0 < end; t0 += tile) {
    int key[kSortRounds], rank[kSortRounds];
    const int64_t w0 = t0 + (int64_t)warp * (32 * rounds) + lane;
#pragma unroll
    for (int j = 0; j < kSortRounds; ++j) {
      const int64_t i = w0 + 32 * j;
      key[j] = -1;
      if (j < rounds && i < end) {
        const int id = __ldcg(ids + i);
        if (id >= E) record_error(err, kErrExpertId, kAtSort, (int)i);
        key[j] = sort_key(id, E);
      }
    }
    __syncwarp();   // (each warp has cleared its own counters)
#pragma unroll
    for (int j = 0; j < kSortRounds; ++j) {
      if (j >= rounds) break;
      const uint32_t same = same_key(key[j], bits);
      const int ahead = __popc(same & ((1u << lane) - 1u));
      if (key[j] >= 0) rank[j] = cnt[warp][key[j]] + ahead;
      __syncwarp();
      if (key[j] >= 0 && ahead == 0) cnt[warp][key[j]] += __popc(same);
      __syncwarp();
    }
    __syncthreads();
    // each key's first row in every warp: the warps' counts are summed up in place
    int mine = 0;
    if (tid < keys) {
      for (int w = 0; w < warps; w += 8) {
        int n[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) n[j] = w + j < warps ? cnt[w + j][tid] : 0;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (w + j < warps) {
            cnt[w + j][tid] = mine;
            mine += n[j];
          }
      }
    }
    if (t0 == begin) {
      int total;
      const int n = tid < keys ? (nchunks == 0 ? mine : sums[0][tid]) : 0;
      const int first = block_exclusive_scan_i(n, iscr, &total);
      if (tid < keys) {
        base[tid] = first + (nchunks == 0 ? 0 : sums[1][tid]);
        if (blockIdx.x == 0) offsets[tid] = first;
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kSortRounds; ++j) {
      if (key[j] < 0) continue;
      const int64_t i = w0 + 32 * j;
      const int r = base[key[j]] + cnt[warp][key[j]] + rank[j];
      const bool none = key[j] == E;
      pos[i] = none ? ~r : r;
      rows[r] = none ? -1 : (int)i;
    }
    if (t0 + tile >= end) break;
    __syncthreads();
    if (tid < keys) base[tid] += mine;
    for (int i = lane; i < keys; i += 32) cnt[warp][i] = 0;
    __syncthreads();
  }
}

// How R pairs are cut: up to 1024 go to one CTA, without counts (chunks 0); more are cut into chunks of
// whole tiles, a CTA each and no more than run at once, with as few pairs a thread as that
// allows (4096 pairs took 11.6 us in one CTA).
struct SortPlan {
  int chunks, rounds, threads;
  bool wide;   // counts of 32 bits
  int64_t chunk;
};
SortPlan sort_plan(int64_t R, int E) {
  SortPlan p;
  p.wide = R > kNarrowPairs;
  if (R <= kSortThreads) {
    p.chunks = 0;
    p.rounds = 1;
    p.threads = (int)((R > E + 1 ? R : E + 1) + 31) / 32 * 32;
    p.chunk = R > 0 ? R : 1;
    return p;
  }
  const int64_t pieces = (R + kSortThreads - 1) / kSortThreads;
  const int most = p.wide ? kWideChunks : kSortMaxChunks;
  const int64_t per = (pieces + most - 1) / most;   // of a thread's pairs, per chunk
  p.rounds = per < kSortRounds ? (int)per : kSortRounds;
  p.threads = kSortThreads;
  p.chunk = (per + p.rounds - 1) / p.rounds * p.rounds * kSortThreads;
  p.chunks = (int)((R + p.chunk - 1) / p.chunk);
  return p;
}

// The counts lie behind what other calls on the workspace need at zero.
constexpr size_t kSortCounts = kWsZeroEnd;
static_assert(2 * kWideChunks >= kSortMaxChunks, "the workspace does not shrink where counts widen");

template <typename Count>
cudaError_t launch(const SortPlan& p, int64_t R, int E, const int32_t* ids, int32_t* offsets,
                   int32_t* rows, int32_t* pos, void* ws, cudaStream_t s) {
  DevErrRecord* err = static_cast<DevErrRecord*>(ws);
  Count* counts = p.chunks > 0 ? reinterpret_cast<Count*>(static_cast<uint8_t*>(ws) + kSortCounts)
                               : nullptr;
  cudaError_t e = cudaSuccess;
  if (p.chunks > 0)
    e = launch_ex(sort_count_kernel<Count>, dim3(p.chunks), dim3(kSortThreads), 0, s, true, ids, R, E,
                  p.chunk, counts);
  if (e == cudaSuccess)
    e = launch_ex(sort_place_kernel<Count>, dim3(p.chunks > 0 ? p.chunks : 1), dim3(p.threads), 0, s,
                  true, ids, R, E, p.chunk, p.chunks, p.rounds, static_cast<const Count*>(counts),
                  offsets, rows, pos, err);
  if (e != cudaSuccess) return e;
  return cudaGetLastError();
}

}  // namespace

// Of as many chunks as any sort of at most R pairs has (the chunks of R itself may be fewer): a
// workspace for R pairs is large enough for fewer.
size_t sort_workspace_bytes(int64_t R, int E) {
  if (R <= kSortThreads) return kWsTickets;   // the fault record's 256 bytes
  if (R > kNarrowPairs) return kSortCounts + sizeof(int32_t) * kWideChunks * (E + 1);
  const int64_t pieces = (R + kSortThreads - 1) / kSortThreads;
  const int64_t chunks = pieces < kSortMaxChunks ? pieces : kSortMaxChunks;
  return kSortCounts + sizeof(uint16_t) * (size_t)chunks * (E + 1);
}

cudaError_t launch_sort_tokens(int64_t R, int E, const int32_t* ids, int32_t* offsets,
                               int32_t* rows, int32_t* pos, void* ws, cudaStream_t s) {
  const SortPlan p = sort_plan(R, E);
  return p.wide ? launch<int32_t>(p, R, E, ids, offsets, rows, pos, ws, s)
                : launch<uint16_t>(p, R, E, ids, offsets, rows, pos, ws, s);
}

}  // namespace dmoe

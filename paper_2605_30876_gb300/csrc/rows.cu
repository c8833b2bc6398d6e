// Token rows into the experts' order and back, and the gradients of both. All four are copies and
// short sums: they are bound by the bytes of the rows (each read once and written once), so the work
// is cut by tokens: a token's row is held in registers while its k sorted rows are written or read.
// Rows of bf16 2048 wide, 16384 tokens of eight slots, a tenth without an expert, cold: gather 92 us
// (6.6 TB/s), its gradient 88 (6.25), combine with an addend 99 (6.25), its gradient 164 (6.65);
// of the 6.8 TB/s that a copy reaches. Widths that only allow 2-byte pieces are bound by their loads'
// number: 8192 tokens of four slots, 1001 wide: gather 21.5 us (3.8 TB/s), combine's gradient 42
// (3.4).
#include <cuda_fp16.h>

#include "block_reduce.cuh"
#include "dmoe_internal.cuh"

namespace dmoe {
namespace {

constexpr int kRowThreads = 256;
constexpr int kSlotBatch = 8;   // slots whose rows are in flight together

// VB bytes of a row as loaded and stored at once
template <int VB> struct Raw;
template <> struct Raw<16> { using type = uint4; };
template <> struct Raw<4> { using type = uint32_t; };
template <> struct Raw<2> { using type = uint16_t; };

template <typename T, int VB>
struct Piece {
  static constexpr int n = VB / (int)sizeof(T);
  using raw = typename Raw<VB>::type;
  union {
    raw r;
    T e[n];
  };
  __device__ __forceinline__ Piece() {}
};

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) {
  return __float2bfloat16_rn(v);
}

template <typename T, int VB>
__device__ __forceinline__ Piece<T, VB> load_piece(const T* row, int64_t v) {
  Piece<T, VB> p;
  p.r = *(reinterpret_cast<const typename Raw<VB>::type*>(row) + v);
  return p;
}
// rows that are read once
template <typename T, int VB>
__device__ __forceinline__ Piece<T, VB> load_once(const T* row, int64_t v) {
  Piece<T, VB> p;
  p.r = __ldcs(reinterpret_cast<const typename Raw<VB>::type*>(row) + v);
  return p;
}
template <typename T, int VB>
__device__ __forceinline__ void store_piece(T* row, int64_t v, const Piece<T, VB>& p) {
  __stcs(reinterpret_cast<typename Raw<VB>::type*>(row) + v, p.r);
}

// the sorted row that a pos entry names; -1: one that is not followed
__device__ __forceinline__ int named_row(int p, int R) {
  const int r = p < 0 ? ~p : p;
  return r < R ? r : -1;
}

// Pieces of a row that a thread has in flight: narrow ones in numbers, or the bytes on their way are
// too few (one 2-byte piece a thread: 8192 x 6 rows of 1001 were combined in 82 us).
template <int VB>
constexpr int pieces_ahead() { return VB == 16 ? 1 : 4; }

// gather: a thread copies its pieces of the token's row to their k places
template <typename T, int VB>
__global__ void __launch_bounds__(kRowThreads)
gather_rows_kernel(const T* __restrict__ x, int64_t ldx, const int32_t* __restrict__ pos,
                   T* __restrict__ xs, int64_t ldxs, int64_t tokens, int k, int nv) {
  constexpr int kU = pieces_ahead<VB>();
  pdl_wait();
  pdl_launch_dependents();
  const int64_t t = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  const int v0 = blockIdx.y * blockDim.x * kU + threadIdx.x;
  if (t >= tokens || v0 >= nv) return;
  const int R = (int)(tokens * k);
  Piece<T, VB> p[kU], zero;
  zero.r = typename Raw<VB>::type{};
#pragma unroll
  for (int u = 0; u < kU; ++u)
    if (v0 + u * (int)blockDim.x < nv) p[u] = load_once<T, VB>(x + t * ldx, v0 + u * (int)blockDim.x);
  for (int j0 = 0; j0 < k; j0 += kSlotBatch) {
    int at[kSlotBatch];
#pragma unroll
    for (int j = 0; j < kSlotBatch; ++j) at[j] = j0 + j < k ? __ldg(pos + t * k + j0 + j) : R;
#pragma unroll
    for (int j = 0; j < kSlotBatch; ++j) {
      const int r = named_row(at[j], R);
      if (r < 0) continue;
      T* to = xs + r * ldxs;
#pragma unroll
      for (int u = 0; u < kU; ++u)
        if (v0 + u * (int)blockDim.x < nv)
          store_piece<T, VB>(to, v0 + u * (int)blockDim.x, at[j] < 0 ? zero : p[u]);
    }
  }
}

// combine (and, with neither gates nor an addend, the gather's gradient): a thread adds up its pieces of
// the token's k rows in fp32, in the order of the slots. The slots' positions have to be read before
// the rows; four CTAs per SM (64 registers a thread) hide it: 16384 x 8 rows of 2048 took 99 us with
// three, and 117 with CTAs that go on from token to token and read positions ahead (two per SM).
template <typename T, int VB>
__global__ void __launch_bounds__(kRowThreads, 4)
combine_rows_kernel(const T* __restrict__ ys, int64_t ldys, const int32_t* __restrict__ pos,
                    const float* __restrict__ gates, const T* add, int64_t ldadd, T* y,
                    int64_t ldy, int64_t tokens, int k, int nv) {
  constexpr int n = Piece<T, VB>::n, kU = pieces_ahead<VB>();
  pdl_wait();
  pdl_launch_dependents();
  const int64_t t = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  const int bx = blockDim.x, v0 = blockIdx.y * bx * kU + threadIdx.x;
  if (t >= tokens || v0 >= nv) return;
  const int R = (int)(tokens * k);
  float acc[kU][n];
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    Piece<T, VB> p;
    p.r = typename Raw<VB>::type{};
    if (add != nullptr && v0 + u * bx < nv) p = load_piece<T, VB>(add + t * ldadd, v0 + u * bx);
#pragma unroll
    for (int i = 0; i < n; ++i) acc[u][i] = to_f(p.e[i]);
  }
  for (int j0 = 0; j0 < k; j0 += kSlotBatch) {
    int at[kSlotBatch];
    Piece<T, VB> p[kSlotBatch][kU];
    uint32_t own = 0;
#pragma unroll
    for (int j = 0; j < kSlotBatch; ++j) at[j] = j0 + j < k ? __ldg(pos + t * k + j0 + j) : -1;
#pragma unroll
    for (int j = 0; j < kSlotBatch; ++j) {
      if (at[j] < 0 || at[j] >= R) continue;
      own |= 1u << j;
      const T* row = ys + at[j] * ldys;
#pragma unroll
      for (int u = 0; u < kU; ++u)
        if (v0 + u * bx < nv) p[j][u] = load_once<T, VB>(row, v0 + u * bx);
    }
#pragma unroll
    for (int j = 0; j < kSlotBatch; ++j)
      if (own >> j & 1u) {
        const float w = gates != nullptr ? __ldg(gates + t * k + j0 + j) : 1.f;
#pragma unroll
        for (int u = 0; u < kU; ++u)
#pragma unroll
          for (int i = 0; i < n; ++i) acc[u][i] = fmaf(w, to_f(p[j][u].e[i]), acc[u][i]);
      }
  }
#pragma unroll
  for (int u = 0; u < kU; ++u)
    if (v0 + u * bx < nv) {
      Piece<T, VB> out;
#pragma unroll
      for (int i = 0; i < n; ++i) out.e[i] = from_f<T>(acc[u][i]);
      store_piece<T, VB>(y + t * ldy, v0 + u * bx, out);
    }
}

// combine's gradient: a warp has a (token, slot). It goes over dy's row and the slot's row of ys, four
// pieces of both on their way (more where they are narrow), writes gate * dy and adds up dy * ys. The
// k warps of a token read dy's row k times, from L1 or L2 but for the first. (With dy's pieces held
// in registers for all k slots at once half as many threads fitted: 221 us, not 164, for 16384
// tokens of eight slots, 2048 wide.)
template <typename T, int VB, bool kRows, bool kGates>
__global__ void __launch_bounds__(kRowThreads)
combine_rows_backward_kernel(const T* __restrict__ dy, int64_t lddy, const T* __restrict__ ys,
                             int64_t ldys, const int32_t* __restrict__ pos,
                             const float* __restrict__ gates, T* __restrict__ dys, int64_t lddys,
                             float* __restrict__ dgates, int R, int k, int nv) {
  constexpr int n = Piece<T, VB>::n, kAhead = VB == 16 ? 4 : VB == 4 ? 8 : 16;
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const int64_t i = (int64_t)blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
  if (i >= R) return;
  const int p = __ldg(pos + i), r = named_row(p, R);
  const float g = gates != nullptr ? __ldg(gates + i) : 1.f;
  const bool own = p >= 0 && r >= 0;   // the slot has an expert
  const T* from = dy + i / k * lddy;
  const T* row = ys + (int64_t)(own ? r : 0) * ldys;
  T* to = dys + (int64_t)(r >= 0 ? r : 0) * lddys;
  float dot = 0.f;
  if (own) {
    for (int v0 = lane; v0 < nv; v0 += 32 * kAhead) {
      Piece<T, VB> d[kAhead], y[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (v0 + 32 * j < nv) {
          d[j] = load_piece<T, VB>(from, v0 + 32 * j);
          if (kGates) y[j] = load_once<T, VB>(row, v0 + 32 * j);
        }
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (v0 + 32 * j < nv) {
          if (kRows) {
            Piece<T, VB> o;
#pragma unroll
            for (int e = 0; e < n; ++e) o.e[e] = from_f<T>(g * to_f(d[j].e[e]));
            store_piece<T, VB>(to, v0 + 32 * j, o);
          }
          if (kGates) {
#pragma unroll
            for (int e = 0; e < n; ++e) dot = fmaf(to_f(d[j].e[e]), to_f(y[j].e[e]), dot);
          }
        }
    }
  } else if (kRows && r >= 0) {
    Piece<T, VB> zero;
    zero.r = typename Raw<VB>::type{};
    for (int v = lane; v < nv; v += 32) store_piece<T, VB>(to, v, zero);
  }
  if (kGates) {
    dot = warp_sum(dot);
    if (lane == 0) dgates[i] = dot;
  }
}

// pieces of a row, and the CTA's shape: `block.x` threads on a token's row, `ahead` pieces each
struct RowShape {
  int nv;
  dim3 block, grid;
};
RowShape row_shape(int64_t tokens, int d, int per_piece, int ahead) {
  RowShape s;
  s.nv = d / per_piece;
  int bx = 32;
  while (bx * ahead < s.nv && bx < kRowThreads) bx *= 2;
  s.block = dim3(bx, kRowThreads / bx);
  s.grid = dim3((unsigned)((tokens + s.block.y - 1) / s.block.y), (s.nv + bx * ahead - 1) / (bx * ahead));
  return s;
}

// the widest pieces that the rows' width, strides and bases allow
int piece_bytes(int esize, int d, std::initializer_list<const void*> ptrs,
                std::initializer_list<int64_t> lds) {
  uint64_t bits = (uint64_t)d * esize;
  for (const void* p : ptrs) bits |= reinterpret_cast<uint64_t>(p);
  for (int64_t ld : lds) bits |= (uint64_t)ld * esize;
  if (bits % 16 == 0) return 16;
  return bits % 4 == 0 ? 4 : 2;
}

// calls f(T{}, pieces' bytes as a constant) for a dtype
template <int V> struct Int { static constexpr int value = V; };
template <typename F>
cudaError_t with_type(int dtype, int vb, F f) {
  switch (dtype) {
    case DMOE_BF16:
      return vb == 16 ? f(__nv_bfloat16{}, Int<16>{})
                      : vb == 4 ? f(__nv_bfloat16{}, Int<4>{}) : f(__nv_bfloat16{}, Int<2>{});
    case DMOE_FP16:
      return vb == 16 ? f(__half{}, Int<16>{})
                      : vb == 4 ? f(__half{}, Int<4>{}) : f(__half{}, Int<2>{});
    default: return vb == 16 ? f(float{}, Int<16>{}) : f(float{}, Int<4>{});
  }
}

int dtype_bytes(int dtype) { return dtype == DMOE_FP32 ? 4 : 2; }

}  // namespace

cudaError_t launch_gather_rows(const RowsArgs& a, cudaStream_t s) {
  const int es = dtype_bytes(a.dtype);
  const int vb = piece_bytes(es, a.d, {a.tok, a.sorted_out}, {a.ldtok, a.ldsorted_out});
  return with_type(a.dtype, vb, [&](auto z, auto w) {
    using T = decltype(z);
    constexpr int VB = decltype(w)::value;
    const RowShape sh = row_shape(a.T, a.d, VB / es, pieces_ahead<VB>());
    return launch_ex(gather_rows_kernel<T, VB>, sh.grid, sh.block, 0, s, true,
                     static_cast<const T*>(a.tok), a.ldtok, a.pos, static_cast<T*>(a.sorted_out),
                     a.ldsorted_out, a.T, a.k, sh.nv);
  });
}

cudaError_t launch_combine_rows(const RowsArgs& a, cudaStream_t s) {
  const int es = dtype_bytes(a.dtype);
  const int vb = piece_bytes(es, a.d, {a.sorted, a.tok, a.tok_out},
                             {a.ldsorted, a.tok != nullptr ? a.ldtok : 0, a.ldtok_out});
  return with_type(a.dtype, vb, [&](auto z, auto w) {
    using T = decltype(z);
    constexpr int VB = decltype(w)::value;
    const RowShape sh = row_shape(a.T, a.d, VB / es, pieces_ahead<VB>());
    return launch_ex(combine_rows_kernel<T, VB>, sh.grid, sh.block, 0, s, true,
                     static_cast<const T*>(a.sorted), a.ldsorted, a.pos, a.gates,
                     static_cast<const T*>(a.tok), a.ldtok, static_cast<T*>(a.tok_out),
                     a.ldtok_out, a.T, a.k, sh.nv);
  });
}

cudaError_t launch_combine_rows_backward(const RowsArgs& a, cudaStream_t s) {
  const int es = dtype_bytes(a.dtype);
  const int vb = piece_bytes(es, a.d, {a.tok, a.sorted, a.sorted_out},
                             {a.ldtok, a.sorted != nullptr ? a.ldsorted : 0,
                              a.sorted_out != nullptr ? a.ldsorted_out : 0});
  return with_type(a.dtype, vb, [&](auto z, auto w) {
    using T = decltype(z);
    constexpr int VB = decltype(w)::value;
    const int R = (int)(a.T * a.k), warps = kRowThreads / 32;
    auto* kernel = a.dgates == nullptr ? combine_rows_backward_kernel<T, VB, true, false>
                   : a.sorted_out == nullptr ? combine_rows_backward_kernel<T, VB, false, true>
                                             : combine_rows_backward_kernel<T, VB, true, true>;
    return launch_ex(kernel, dim3((R + warps - 1) / warps), dim3(kRowThreads), 0, s, true,
                     static_cast<const T*>(a.tok), a.ldtok, static_cast<const T*>(a.sorted),
                     a.ldsorted, a.pos, a.gates, static_cast<T*>(a.sorted_out), a.ldsorted_out,
                     a.dgates, R, a.k, a.d / (VB / es));
  });
}

}  // namespace dmoe

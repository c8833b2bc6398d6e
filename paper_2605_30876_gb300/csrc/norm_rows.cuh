// What the two directions of the norms around a block share (norm_rows.cu, norm_rows_backward.cu): pieces of a
// row in a thread, rows on their way, sums over a row's group of threads, and the sizes of a launch.
#pragma once

#include <cuda_fp16.h>

#include <algorithm>
#include <type_traits>

#include "dmoe_internal.cuh"

namespace dmoe {
namespace {

template <int VB> struct Raw;
template <> struct Raw<16> { using type = uint4; };
template <> struct Raw<4> { using type = uint32_t; };
template <> struct Raw<2> { using type = uint16_t; };

__device__ __forceinline__ void from_f(float v, float* o) { *o = v; }
__device__ __forceinline__ void from_f(float v, __half* o) { *o = __float2half_rn(v); }
__device__ __forceinline__ void from_f(float v, __nv_bfloat16* o) { *o = __float2bfloat16_rn(v); }

// Two fp32 values in a register pair, for the instructions that take two at once (a row's arithmetic
// is as long as its bytes otherwise: with one value an instruction and unpacked conversions the
// forward launch of 16384 rows of 2048 took 61 us, the backward one 94, and issue slots were 70 % busy).
struct F2 {
  unsigned long long v;
  __device__ __forceinline__ F2() {}
  __device__ __forceinline__ F2(float lo, float hi) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi)); }
  __device__ __forceinline__ explicit F2(float both) : F2(both, both) {}
  __device__ __forceinline__ float lo() const {
    float a;
    asm("mov.b64 {%0, _}, %1;" : "=f"(a) : "l"(v));
    return a;
  }
  __device__ __forceinline__ float hi() const {
    float b;
    asm("mov.b64 {_, %0}, %1;" : "=f"(b) : "l"(v));
    return b;
  }
};
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return d;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
  return d;
}

// kE elements of a row that a thread holds: pieces of VB bytes, `step` pieces apart. kFull: a group's
// threads hold exactly the row (no piece has to be asked for).
template <typename T, int VB, int kE, bool kFull = false>
struct Part {
  static constexpr int n = VB / (int)sizeof(T), kP = kE / n;
  using raw = typename Raw<VB>::type;
  union {
    raw r[kP];
    T e[kE];
    uint32_t w[kE * sizeof(T) / 4];
  };
  __device__ __forceinline__ Part() {}
  __device__ __forceinline__ void load(const T* row, int v0, int step, int nv) {
#pragma unroll
    for (int j = 0; j < kP; ++j)
      if (kFull || v0 + j * step < nv)
        r[j] = __ldcs(reinterpret_cast<const raw*>(row) + v0 + j * step);
      else
        r[j] = raw{};
  }
  // a row that many tokens share
  __device__ __forceinline__ void load_shared(const T* row, int v0, int step, int nv) {
#pragma unroll
    for (int j = 0; j < kP; ++j)
      if (kFull || v0 + j * step < nv)
        r[j] = __ldg(reinterpret_cast<const raw*>(row) + v0 + j * step);
      else
        r[j] = raw{};
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int j = 0; j < kP; ++j) r[j] = raw{};
  }
  // elements 2 i and 2 i + 1
  __device__ __forceinline__ F2 get(int i) const {
    if constexpr (std::is_same_v<T, __nv_bfloat16>)
      return F2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    else if constexpr (std::is_same_v<T, __half>) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      return F2(f.x, f.y);
    } else {
      return F2(e[2 * i], e[2 * i + 1]);
    }
  }
  __device__ __forceinline__ void set(int i, F2 v) {
    if constexpr (std::is_same_v<T, __nv_bfloat16>) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v.lo(), v.hi());
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    } else if constexpr (std::is_same_v<T, __half>) {
      const __half2 b = __floats2half2_rn(v.lo(), v.hi());
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    } else {
      e[2 * i] = v.lo();
      e[2 * i + 1] = v.hi();
    }
  }
  __device__ __forceinline__ void store(T* row, int v0, int step, int nv) const {
#pragma unroll
    for (int j = 0; j < kP; ++j)
      if (kFull || v0 + j * step < nv) __stcs(reinterpret_cast<raw*>(row) + v0 + j * step, r[j]);
  }
};

// fp32 vectors of the row's width (weights, sums), the elements that a part holds
template <typename T, int VB, int kE, bool kFull>
__device__ __forceinline__ void load_vector(F2 (&o)[kE / 2], const float* w, int v0, int step, int nv,
                                            float none) {
  constexpr int n = VB / (int)sizeof(T);
  auto at = [&](int e) { return w + (v0 + e / n * step) * n + e % n; };
  auto in = [&](int e) { return w != nullptr && (kFull || v0 + e / n * step < nv); };
#pragma unroll
  for (int i = 0; i < kE; i += n % 4 == 0 ? 4 : 2) {
    if constexpr (n % 4 == 0) {
      const float4 f = in(i) ? __ldg(reinterpret_cast<const float4*>(at(i))) : make_float4(none, none, none, none);
      o[i / 2] = F2(f.x, f.y);
      o[i / 2 + 1] = F2(f.z, f.w);
    } else if constexpr (n == 2) {
      const float2 f = in(i) ? __ldg(reinterpret_cast<const float2*>(at(i))) : make_float2(none, none);
      o[i / 2] = F2(f.x, f.y);
    } else {
      const float a = in(i) ? __ldg(at(i)) : none, b = in(i + 1) ? __ldg(at(i + 1)) : none;
      o[i / 2] = F2(a, b);
    }
  }
}
template <typename T, int VB, int kE, bool kFull>
__device__ __forceinline__ void store_vector(const F2 (&v)[kE / 2], float* w, int v0, int step, int nv) {
  constexpr int n = VB / (int)sizeof(T);
  auto at = [&](int e) { return w + (v0 + e / n * step) * n + e % n; };
  auto in = [&](int e) { return kFull || v0 + e / n * step < nv; };
#pragma unroll
  for (int i = 0; i < kE; i += n % 4 == 0 ? 4 : 2) {
    if constexpr (n % 4 == 0) {
      if (in(i))
        *reinterpret_cast<float4*>(at(i)) =
            make_float4(v[i / 2].lo(), v[i / 2].hi(), v[i / 2 + 1].lo(), v[i / 2 + 1].hi());
    } else if constexpr (n == 2) {
      if (in(i)) *reinterpret_cast<float2*>(at(i)) = make_float2(v[i / 2].lo(), v[i / 2].hi());
    } else {
      if (in(i)) *at(i) = v[i / 2].lo();
      if (in(i + 1)) *at(i + 1) = v[i / 2].hi();
    }
  }
}

// Rows on their way: a thread copies its own pieces of up to kN rows into shared memory, a few tokens
// ahead (cp.async, 16 or 4 bytes each), and reads them back itself, so that nothing is synchronised
// and no registers are held. 2-byte pieces cannot be copied so, and more than 128 bytes a thread and
// token would leave no room for a token ahead: those rows are loaded when they are taken.
template <typename T, int VB, int kE, int kN, int kBlock, bool kFull>
struct Ahead {
  using P = Part<T, VB, kE, kFull>;
  static constexpr bool kAsync = VB >= 4 && kN * kE * sizeof(T) <= 128;
  // [token][row][piece][thread]
  static constexpr int kPlace = kBlock * VB, kToken = kAsync ? kN * P::kP * kPlace : 0;
  uint32_t at, put, got, end;
  __device__ __forceinline__ Ahead(void* smem, int depth)
      : at((uint32_t)__cvta_generic_to_shared(smem) + threadIdx.x * VB), put(at), got(at),
        end(at + depth * kToken) {}
  // one call a token, also for tokens that are not there (`in` is false)
  template <typename F>
  __device__ __forceinline__ void fetch(bool in, F rows_of, int v0, int step, int nv) {
    if constexpr (kAsync) {
      if (in) {
        const T* rows[kN];
        rows_of(rows);
#pragma unroll
        for (int k = 0; k < kN; ++k)
          if (kFull || rows[k] != nullptr)
#pragma unroll
            for (int j = 0; j < P::kP; ++j)
              if (kFull || v0 + j * step < nv) {
                const uint32_t to = put + (k * P::kP + j) * kPlace;
                const typename P::raw* from = reinterpret_cast<const typename P::raw*>(rows[k]) + (v0 + j * step);
                if constexpr (VB == 16)
                  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
                else
                  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
              }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      put += kToken;
      if (put == end) put = at;
    }
  }
  // the oldest token's rows (zeros where there is none)
  __device__ __forceinline__ void take(P (&o)[kN], const T* const (&rows)[kN], int v0, int step, int nv,
                                       int depth) {
    if constexpr (kAsync) {
      if (depth == 4) asm volatile("cp.async.wait_group 3;" ::: "memory");
      else if (depth == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
      else asm volatile("cp.async.wait_group 1;" ::: "memory");
#pragma unroll
      for (int k = 0; k < kN; ++k)
#pragma unroll
        for (int j = 0; j < P::kP; ++j) {
          if (!kFull) o[k].r[j] = typename P::raw{};
          if (kFull || (rows[k] != nullptr && v0 + j * step < nv)) {
            const uint32_t from = got + (k * P::kP + j) * kPlace;
            if constexpr (VB == 16) {
              uint4 v;
              asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                           : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(from) : "memory");
              o[k].r[j] = v;
            } else if constexpr (VB == 4) {
              uint32_t v;
              asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(from) : "memory");
              o[k].r[j] = v;
            }
          }
        }
      got += kToken;
      if (got == end) got = at;
    } else {
#pragma unroll
      for (int k = 0; k < kN; ++k)
        if (rows[k] != nullptr) o[k].load(rows[k], v0, step, nv); else o[k].zero();
    }
  }
};

// row t of a matrix (strides are below 2^30 elements)
template <typename T>
__device__ __forceinline__ T* row_at(T* base, int t, uint32_t ld) {
  using Byte = std::conditional_t<std::is_const_v<T>, const char, char>;
  return reinterpret_cast<T*>(reinterpret_cast<Byte*>(base) + (uint64_t)(uint32_t)t * (ld * (uint32_t)sizeof(T)));
}

// Sums of K values over the `width` threads of a row's group (a power of two up to a warp, or whole warps),
// the same in every thread. Groups of more than a warp use `scratch` (2 x 16 K floats) and a barrier of
// their own; its halves alternate from call to call, so that one barrier is enough. A group has a power of
// two of places there; those behind its warps stay zeros.
template <int K>
struct GroupSum {
  float* put;
  const float* take;
  int width, barrier, first, half;
  __device__ __forceinline__ GroupSum(float* scratch, int width_, int group)
      : width(width_), barrier(group + 1), half(0) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, per = width >> 5;
    const int places = per > 8 ? 16 : per > 4 ? 8 : per > 2 ? 4 : 2;
    first = places >> 1;
    put = scratch + (group * places + warp - group * per) * K;
    take = scratch + (group * places + (lane & (places - 1))) * K;
    if (width > 32 && places != per) {
      for (int i = threadIdx.x; i < 32 * K; i += blockDim.x) scratch[i] = 0.f;
      __syncthreads();
    }
  }
  __device__ __forceinline__ void operator()(float (&v)[K]) {
    if (width >= 32) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
      if (width == 32) return;
      if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) put[half + k] = v[k];
      asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(width) : "memory");
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = take[half + k];
      half ^= 16 * K;
      for (int o = first; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    } else {
      for (int o = width >> 1; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    }
  }
};

__device__ __forceinline__ float rstd_of(float sum, float inv_d, float eps) {
  return rsqrtf(fmaf(sum, inv_d, eps));
}

// ------------------------------------------------------------------ host side
template <int V> struct Int { static constexpr int value = V; };
template <typename F>
cudaError_t with_type(int dtype, int piece, F f) {
  auto pieces = [&](auto z) {
    if (piece == 16) return f(z, Int<16>{});
    if constexpr (sizeof(z) == 2)
      if (piece == 2) return f(z, Int<2>{});
    return f(z, Int<4>{});
  };
  switch (dtype) {
    case DMOE_BF16: return pieces(__nv_bfloat16{});
    case DMOE_FP16: return pieces(__half{});
    default: return pieces(float{});
  }
}

int esize(int dtype) { return dtype == DMOE_FP32 ? 4 : 2; }

// Bytes that every row can be read and written at a time: 16, 4 or 2. The smaller, the more instructions a
// row takes: 16384 rows in bf16 with a gate row for 32 tokens, cold, a call between two events, forward and backward, of
// 2048 (16 bytes) 52 and 82 us, of 2050 (4) 72 and 175, of 2049 (2) 158 and 479.
int piece_of_rows(const NormArgs& a) {
  const uint64_t es = esize(a.dtype);
  uint64_t bits = a.d * es;
  for (const void* p : {a.x, a.y, a.gate, a.dr, a.dn, (const void*)a.r, (const void*)a.n,
                        (const void*)a.dx, (const void*)a.dy, (const void*)a.dgate})
    bits |= reinterpret_cast<uint64_t>(p);
  const void* p[] = {a.x, a.y, a.gate, a.dr, a.dn, a.r, a.n, a.dx, a.dy, a.dgate};
  const int64_t ld[] = {a.ldx, a.ldy, a.ldgate, a.lddr, a.lddn, a.ldr, a.ldn, a.lddx, a.lddy, a.lddgate};
  for (int i = 0; i < 10; ++i)
    if (p[i] != nullptr) bits |= (uint64_t)ld[i] * es;
  return bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 2;
}

// Threads of a row's group, so that each holds at most kE elements: 8, 16 or 32, or whole warps. (Powers of two
// alone leave up to half of the threads idle: 6553 rows of 5120 in bf16 took 70 us forward and 218 backward
// so, 64 and 139 with whole warps; 26214 of 1280 61 and 122, 57 and 86.)
int group_width(int d, int n, int kE) {
  const int threads = ((d + n - 1) / n * n + kE - 1) / kE;
  return threads <= 8 ? 8 : threads <= 16 ? 16 : (threads + 31) / 32 * 32;
}

// the largest shared memory that a CTA can have, once per device and kernel
template <typename F>
cudaError_t raise_smem(F* kernel, std::atomic<uint32_t>& done) {
  int dev = 0, limit = 0;
  cudaError_t e = cudaGetDevice(&dev);
  const uint32_t bit = dev < 32 ? 1u << dev : 0u;
  if (e != cudaSuccess || (done.load(std::memory_order_relaxed) & bit) != 0u) return e;
  e = cudaDeviceGetAttribute(&limit, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, limit);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// CTAs per SM: two of 256 threads, three of 160 or fewer, or one of more
int ctas_per_sm(int most, int block) { return most > 256 ? 1 : block <= 160 ? 3 : 2; }

// Tokens that the shared memory holds rows of, with that many CTAs per SM. `fixed`: what else a CTA needs.
int tokens_ahead(int ctas, size_t fixed, int row) {
  if (row == 0) return 2;
  const size_t room = (ctas == 1 ? 227 : ctas == 2 ? 113 : 74) * 1024 - fixed;
  return (int)std::max<size_t>(2, std::min<size_t>(4, room / row));
}

// CTAs of a launch (at most `most`) and the tokens of a group's run
int runs(int64_t T, int per_cta, int64_t most, int* ctas) {
  const int64_t run = (T + most * per_cta - 1) / (most * per_cta), groups = (T + run - 1) / run;
  *ctas = (int)((groups + per_cta - 1) / per_cta);
  return (int)run;
}

}  // namespace
}  // namespace dmoe

// The norms around a block, with its gate and its residual, in one pass, and the gradients:
//   p = y * ry * w_post,  r = scale * x + gate * p,  n = r * rr * w_pre
//   ry = 1 / sqrt(mean(y^2) + eps),  rr = 1 / sqrt(mean(r^2) + eps)
// Both directions are bound by the bytes of their rows, each read once and written once. A row is held
// in registers by a group of threads (a power of two, so that a thread has a few pieces of 16 bytes);
// groups go on from row to row.
//
// Backward, with c = gate * w_post, a = dn * w_pre, yh = y * ry, rh = r * rr (r again from x and y:
// the bytes are those of reading r and y, and nothing is rounded between the two passes):
//   q  = dr + rr * (a - rh * m1),           m1 = mean(a * rh)
//   dx = scale * q,  dy = ry * (q * c - yh * m2),  m2 = mean(q * c * yh)
// m2 needs q, which needs m1; but mean(q c yh) = mean((dr + rr a) c yh) - rr m1 mean(rh c yh), so one
// reduction of three sums over the row is enough. Sums over tokens: A = sum of q * yh over the tokens
// of one gate row; dgate = w_post * A, dw_post += gate * A; dw_pre = sum of dn * rh. A group takes a
// run of tokens, so that every gate row but the first and the last of its run is complete in
// registers; those two and the weights' sums go through the workspace, and a second launch adds them
// in the order of the tokens: the same call gives the same bits.
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
// forward pass of 16384 rows of 2048 took 61 us, the backward 94, and issue slots were 70 % busy).
struct F2 {
  unsigned long long v;
  __device__ __forceinline__ F2() {}
  __device__ __forceinline__ F2(float lo, float hi) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi)); }
  __device__ __forceinline__ explicit F2(float both) : F2(both, both) {}
  __device__ __forceinline__ float lo() const {
    float a, b;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
    return a;
  }
  __device__ __forceinline__ float hi() const {
    float a, b;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
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

// Sums of K values over the `width` threads of a row's group (a power of two), the same in every
// thread. Groups of more than a warp pass `scratch` (K floats per warp of the CTA, twice) and a
// barrier of their own; `flip` changes from call to call, so that one barrier is enough.
template <int K>
__device__ __forceinline__ void group_sum(float (&v)[K], int width, int group, float* scratch, int& flip) {
  if (width >= 32) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    if (width == 32) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, nw = blockDim.x >> 5, per = width >> 5;
    float* s = scratch + flip * nw * K;
    flip ^= 1;
    if (lane == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) s[warp * K + k] = v[k];
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(width) : "memory");
    const int from = group * per + (lane & (per - 1));
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = s[from * K + k];
    for (int o = per >> 1; o > 0; o >>= 1)
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  } else {
    for (int o = width >> 1; o > 0; o >>= 1)
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  }
}

__device__ __forceinline__ float rstd_of(float sum, float inv_d, float eps) {
  return rsqrtf(fmaf(sum, inv_d, eps));
}

// A group of `width` threads takes the run of `run` rows from group * run on; the next depth - 1 are on
// their way. kFull: x, y, r and n are all there, a row is exactly what its group holds, and a group is a
// warp or more. (Asking for each of them every time was half of the instructions, and the kernel is
// bound by those: 45 us with, 33 without the questions for 16384 rows of 2048.)
template <typename T, int VB, int kE, int kBlock, bool kFull>
__global__ void __launch_bounds__(kBlock, kBlock <= 256 ? 2 : 1)
norm_kernel(const NormArgs a, int width, int depth, int run) {
  extern __shared__ float4 smem4[];
  float* scratch = reinterpret_cast<float*>(smem4);
  using P = Part<T, VB, kE, kFull>;
  constexpr int kH = kE / 2;
  constexpr bool kHold = kE <= 16;        // weights and gates stay in registers
  pdl_wait();
  pdl_launch_dependents();
  const int group = threadIdx.x / width, v0 = threadIdx.x % width, nv = a.d / P::n, G = a.gate_tokens;
  const int64_t me = (int64_t)blockIdx.x * (blockDim.x / width) + group;
  const int begin = (int)min(me * run, a.T), end = (int)min((me + 1) * run, a.T);
  int flip = 0;
  const uint32_t ldx = (uint32_t)a.ldx, ldy = (uint32_t)a.ldy, ldr = (uint32_t)a.ldr, ldn = (uint32_t)a.ldn;
  Ahead<T, VB, kE, 2, kBlock, kFull> ahead(smem4 + 8, depth);
  auto rows_of = [&](int t, const T* (&rows)[2]) {
    rows[0] = row_at(static_cast<const T*>(a.x), t, ldx);
    rows[1] = kFull || a.y != nullptr ? row_at(static_cast<const T*>(a.y), t, ldy) : nullptr;
  };
  auto fetch = [&](int t) {
    ahead.fetch(t < end, [&](const T* (&rows)[2]) { rows_of(t, rows); }, v0, width, nv);
  };
  for (int i = 0; i < depth - 1; ++i) fetch(begin + i);
  // post: gate * w_post
  F2 post[kH], pre[kHold ? kH : 1];
  if constexpr (kHold) load_vector<T, VB, kE, kFull>(pre, a.w_pre, v0, width, nv, 0.f);
  int row = G > 0 ? begin / G : 0;
  int next = begin;                       // the first token of another gate row
  const F2 scale(a.scale);
  const float inv_d = 1.f / (float)a.d;
  // (a warp's groups, where they are several, take as many turns as the longest of them)
  const int turns = !kFull && width < 32 ? run : end - begin;
  for (int turn = 0; turn < turns; ++turn) {
    const int t = begin + turn;
    const bool in = kFull || t < end;
    const int n_in = in ? nv : 0;
    fetch(t + depth - 1);
    if (!kHold || t == next) {
      load_vector<T, VB, kE, kFull>(post, a.w_post, v0, width, n_in, 1.f);
      if (a.gate != nullptr && in) {
        if (t == next && t != begin) ++row;
        P g;
        g.load_shared(static_cast<const T*>(a.gate) + (int64_t)row * a.ldgate, v0, width, nv);
#pragma unroll
        for (int e = 0; e < kH; ++e) post[e] = mul2(post[e], g.get(e));
      }
      if (t == next) next = G > 0 ? (int)min((int64_t)(row + 1) * G, a.T) : -1;
    }
    const T* rows[2];
    rows_of(t, rows);
    P v[2];
    ahead.take(v, rows, v0, width, n_in, depth);
    P &x = v[0], &y = v[1];
    F2 r[kH];
#pragma unroll
    for (int e = 0; e < kH; ++e) r[e] = y.get(e);
    float ry = 1.f;
    if (a.w_post != nullptr) {
      F2 s2(0.f);
#pragma unroll
      for (int e = 0; e < kH; ++e) s2 = fma2(r[e], r[e], s2);
      float s[1] = {s2.lo() + s2.hi()};
      group_sum(s, width, group, scratch, flip);
      ry = rstd_of(s[0], inv_d, a.eps);
      const F2 ry2(ry);
#pragma unroll
      for (int e = 0; e < kH; ++e) r[e] = mul2(r[e], ry2);
    }
    F2 s2(0.f);
#pragma unroll
    for (int e = 0; e < kH; ++e) {
      r[e] = fma2(scale, x.get(e), mul2(r[e], post[e]));
      s2 = fma2(r[e], r[e], s2);
    }
    if (kFull || a.r != nullptr) {
#pragma unroll
      for (int e = 0; e < kH; ++e) x.set(e, r[e]);
      x.store(row_at(static_cast<T*>(a.r), t, ldr), v0, width, n_in);
    }
    float rr = 1.f;
    if (kFull || a.w_pre != nullptr) {
      F2 w[kHold ? 1 : kH];
      if constexpr (!kHold) load_vector<T, VB, kE, kFull>(w, a.w_pre, v0, width, n_in, 0.f);
      float s[1] = {s2.lo() + s2.hi()};
      group_sum(s, width, group, scratch, flip);
      rr = rstd_of(s[0], inv_d, a.eps);
      const F2 rr2(rr);
#pragma unroll
      for (int e = 0; e < kH; ++e) {
        if constexpr (kHold) y.set(e, mul2(mul2(r[e], rr2), pre[e]));
        else y.set(e, mul2(mul2(r[e], rr2), w[e]));
      }
      y.store(row_at(static_cast<T*>(a.n), t, ldn), v0, width, n_in);
    }
    if (a.stats != nullptr && in && v0 == 0) {
      a.stats[t] = ry;
      a.stats[a.T + t] = rr;
    }
  }
}

// workspace: fp32 [CTAs][2][d] (dw_post, dw_pre), then [groups][2][d] (the first and the last gate
// row of a run, where they are not complete). Group i's run is the `per` tokens from i * per on.
//
// Up to 4096 elements a thread holds eight, and its sums over tokens, weights and gates stay in
// registers. Wider rows take 16 (or 32) a thread: their sums lie in shared memory, a thread's own
// places, and weights and gates come from L1 for every row. kFull: as above, with x, y, dr, dn, dx, dy
// and dw_pre there.
template <typename T, int VB, int kE, int kBlock, bool kFull>
__global__ void __launch_bounds__(kBlock, kBlock <= 256 ? 2 : 1)
norm_backward_kernel(const NormArgs a, int width, int depth, int per) {
  constexpr bool kShared = kE > 8;
  constexpr int kH = kE / 2, kR = kShared ? 1 : kH;
  extern __shared__ float4 smem4[];
  float* scratch = reinterpret_cast<float*>(smem4);
  using P = Part<T, VB, kE, kFull>;
  pdl_wait();
  pdl_launch_dependents();
  const int group = threadIdx.x / width, v0 = threadIdx.x % width, nv = a.d / P::n;
  const int per_cta = blockDim.x / width, G = a.gate_tokens, T_ = (int)a.T;
  const int64_t me = (int64_t)blockIdx.x * per_cta + group;
  const int begin = (int)min(me * per, a.T), end = (int)min((me + 1) * per, a.T);
  const float inv_d = 1.f / (float)a.d;
  float* part_w = a.workspace + (size_t)blockIdx.x * 2 * a.d;
  float* part_g = a.workspace + (size_t)gridDim.x * 2 * a.d + (size_t)me * 2 * a.d;
  int flip = 0;
  F2 A_[kR], post_[kR], pre_[kR], w_post_[kR], w_pre_[kR], gate_[kR];
  // [sum][element][thread] behind the reductions' words
  float4* sums = smem4 + 48 + threadIdx.x;
  // sum[which][pair i] = f(sum, i)
  auto update = [&](int which, auto f) {
    if constexpr (kShared) {
#pragma unroll
      for (int i = 0; i < kH; i += 2) {
        float4& at = sums[(which * (kE / 4) + i / 2) * kBlock];
        float4 v = at;
        const F2 lo = f(F2(v.x, v.y), i), hi = f(F2(v.z, v.w), i + 1);
        at = make_float4(lo.lo(), lo.hi(), hi.lo(), hi.hi());
      }
    } else {
#pragma unroll
      for (int i = 0; i < kH; ++i) {
        F2& v = which == 0 ? A_[i] : which == 1 ? post_[i] : pre_[i];
        v = f(v, i);
      }
    }
  };
#pragma unroll
  for (int which = 0; which < 3; ++which) update(which, [](F2, int) { return F2(0.f); });
  if constexpr (!kShared) {
    load_vector<T, VB, kE, kFull>(w_post_, a.w_post, v0, width, nv, 1.f);
    load_vector<T, VB, kE, kFull>(w_pre_, a.w_pre, v0, width, nv, 0.f);
#pragma unroll
    for (int i = 0; i < kH; ++i) gate_[i] = F2(1.f);
  }

  // behind the reductions' words and the sums
  Ahead<T, VB, kE, 4, kBlock, kFull> ahead(smem4 + 48 + (kShared ? 3 * kE / 4 * kBlock : 0), depth);
  const uint32_t ldx = (uint32_t)a.ldx, ldy = (uint32_t)a.ldy, lddr = (uint32_t)a.lddr, lddn = (uint32_t)a.lddn;
  auto rows_of = [&](int t, const T* (&rows)[4]) {
    rows[0] = row_at(static_cast<const T*>(a.x), t, ldx);
    rows[1] = kFull || a.y != nullptr ? row_at(static_cast<const T*>(a.y), t, ldy) : nullptr;
    rows[2] = kFull || a.dr != nullptr ? row_at(static_cast<const T*>(a.dr), t, lddr) : nullptr;
    rows[3] = kFull || a.dn != nullptr ? row_at(static_cast<const T*>(a.dn), t, lddn) : nullptr;
  };
  auto fetch = [&](int t) {
    ahead.fetch(t < end, [&](const T* (&rows)[4]) { rows_of(t, rows); }, v0, width, nv);
  };
  for (int i = 0; i < depth - 1; ++i) fetch(begin + i);
  float ry = begin < end ? __ldg(a.stats + begin) : 0.f;
  float rr = begin < end ? __ldg(a.stats + T_ + begin) : 0.f;
  int row = G > 0 ? begin / G : 0;
  int row_end = G > 0 ? (int)min((int64_t)(row + 1) * G, a.T) : T_;
  int seg = begin;                       // the first token of the run in this gate row
  auto load_gate = [&](F2 (&g)[kH]) {
    if (a.gate == nullptr) {
#pragma unroll
      for (int i = 0; i < kH; ++i) g[i] = F2(1.f);
      return;
    }
    P v;
    v.load_shared(static_cast<const T*>(a.gate) + (int64_t)row * a.ldgate, v0, width, nv);
#pragma unroll
    for (int i = 0; i < kH; ++i) g[i] = v.get(i);
  };
  if constexpr (!kShared)
    if (begin < end) load_gate(gate_);
  const bool gate_sums = a.dgate != nullptr || a.dw_post != nullptr;
  const F2 scale(a.scale);
  // a warp's groups (width < 32) take as many turns as the longest of them
  const int turns = !kFull && width < 32 ? per : end - begin;
  for (int turn = 0; turn < turns; ++turn) {
    const int t = begin + turn;
    const bool in = kFull || t < end;
    const int n_in = in ? nv : 0;
    F2 yh[kH], rh[kH], q[kH], c[kH];
    const float rr_t = rr, ry_t = ry;
    ry = t + 1 < end ? __ldg(a.stats + t + 1) : 0.f;
    rr = t + 1 < end ? __ldg(a.stats + T_ + t + 1) : 0.f;
    fetch(t + depth - 1);
    const T* rows[4];
    rows_of(t, rows);
    P in4[4];
    ahead.take(in4, rows, v0, width, n_in, depth);
    const P &x = in4[0], &y = in4[1], &dr = in4[2], &dn = in4[3];
    if constexpr (kShared) {
      load_vector<T, VB, kE, kFull>(c, a.w_post, v0, width, n_in, 1.f);
      if (a.gate != nullptr && in) {
        F2 g[kH];
        load_gate(g);
#pragma unroll
        for (int i = 0; i < kH; ++i) c[i] = mul2(c[i], g[i]);
      }
      load_vector<T, VB, kE, kFull>(q, a.w_pre, v0, width, n_in, 0.f);
    } else {
#pragma unroll
      for (int i = 0; i < kH; ++i) {
        c[i] = mul2(gate_[i], w_post_[i]);
        q[i] = w_pre_[i];
      }
    }
    F2 s0(0.f), s1(0.f), s2(0.f);
    const F2 ry2(ry_t), rr2(rr_t);
#pragma unroll
    for (int i = 0; i < kH; ++i) {
      const F2 v = mul2(dn.get(i), q[i]);
      yh[i] = mul2(y.get(i), ry2);
      const F2 p = mul2(yh[i], c[i]);
      rh[i] = mul2(fma2(scale, x.get(i), p), rr2);
      q[i] = fma2(rr2, v, dr.get(i));
      s0 = fma2(v, rh[i], s0);
      s1 = fma2(q[i], p, s1);
      s2 = fma2(rh[i], p, s2);
    }
    if (kFull || a.dw_pre != nullptr) update(2, [&](F2 v, int i) { return fma2(dn.get(i), rh[i], v); });
    float s[3] = {s0.lo() + s0.hi(), s1.lo() + s1.hi(), s2.lo() + s2.hi()};
    group_sum(s, width, group, scratch, flip);
    const float m1 = s[0] * inv_d * rr_t;
    const float m2 = a.w_post != nullptr ? fmaf(-m1, s[2], s[1]) * inv_d : 0.f;
    const F2 less1(-m1), less2(-m2);
    P o;
#pragma unroll
    for (int i = 0; i < kH; ++i) q[i] = fma2(less1, rh[i], q[i]);
    if (kFull || a.dx != nullptr) {
#pragma unroll
      for (int i = 0; i < kH; ++i) o.set(i, mul2(scale, q[i]));
      o.store(row_at(static_cast<T*>(a.dx), t, (uint32_t)a.lddx), v0, width, n_in);
    }
    if (kFull || a.dy != nullptr) {
#pragma unroll
      for (int i = 0; i < kH; ++i) o.set(i, mul2(ry2, fma2(less2, yh[i], mul2(q[i], c[i]))));
      o.store(row_at(static_cast<T*>(a.dy), t, (uint32_t)a.lddy), v0, width, n_in);
    }
    if (gate_sums) update(0, [&](F2 v, int i) { return fma2(q[i], yh[i], v); });
    if (!in || (t + 1 != row_end && t + 1 != end)) continue;
    // the end of a gate row, or of the run
    if (gate_sums) {
      F2 A[kH];
      if constexpr (kShared) load_gate(q);
      update(0, [&](F2 v, int i) {
        A[i] = v;
        return F2(0.f);
      });
      update(1, [&](F2 v, int i) {
        if constexpr (kShared) return fma2(q[i], A[i], v);
        else return fma2(gate_[i], A[i], v);
      });
      if (a.dgate != nullptr) {
        if constexpr (kShared) load_vector<T, VB, kE, kFull>(c, a.w_post, v0, width, nv, 1.f);
#pragma unroll
        for (int i = 0; i < kH; ++i) {
          if constexpr (kShared) A[i] = mul2(A[i], c[i]);
          else A[i] = mul2(A[i], w_post_[i]);
        }
        if ((int64_t)row * G == seg && t + 1 == row_end) {   // complete
#pragma unroll
          for (int i = 0; i < kH; ++i) o.set(i, A[i]);
          o.store(static_cast<T*>(a.dgate) + (int64_t)row * a.lddgate, v0, width, nv);
        } else {
          store_vector<T, VB, kE, kFull>(A, part_g + (seg == begin ? 0 : a.d), v0, width, nv);
        }
      }
    }
    if (t + 1 < end) {
      seg = t + 1;
      ++row;
      row_end = (int)min((int64_t)(row + 1) * G, a.T);
      if constexpr (!kShared) load_gate(gate_);
    }
  }
  // the CTA's sums of the weights' gradients: its groups' in turn
#pragma unroll
  for (int which = 1; which < 3; ++which) {
    if ((which == 1 ? a.dw_post : a.dw_pre) == nullptr) continue;
    F2 v[kH];
    update(which, [&](F2 f, int i) {
      v[i] = f;
      return f;
    });
    if (per_cta > 1) {
      asm volatile("cp.async.wait_all;" ::: "memory");
      __syncthreads();
      // [pair][thread], behind the reductions' words (in the place of the rows ahead, all of which
      // have been taken); only rows of up to 2048 have several groups a CTA
      float2* mine = reinterpret_cast<float2*>(smem4 + 48) + threadIdx.x;
#pragma unroll
      for (int i = 0; i < kH; ++i) mine[i * kBlock] = make_float2(v[i].lo(), v[i].hi());
      __syncthreads();
      if (group == 0)
#pragma unroll
        for (int i = 0; i < kH; ++i) {
          float2 f = mine[i * kBlock];
          for (int g = 1; g < per_cta; ++g) {
            const float2 other = mine[i * kBlock + g * width];
            f.x += other.x;
            f.y += other.y;
          }
          v[i] = F2(f.x, f.y);
        }
    }
    if (group == 0) store_vector<T, VB, kE, kFull>(v, part_w + (which - 1) * a.d, v0, width, nv);
  }
}

// Sums of what the CTAs and runs left, in 32 strips of 32 threads of kC columns each: the first two rows
// of the grid add the weights' parts, the others the gate rows that no run held alone (`share`: a block
// has one gate row of many runs, else each strip has one of its own).
template <typename T, int kC>
__global__ void __launch_bounds__(1024)
norm_finish_kernel(const NormArgs a, int ctas, int run, int share) {
  __shared__ float s[32][32 * kC];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, strip = threadIdx.x >> 5, c = (blockIdx.x * 32 + lane) * kC;
  const bool in = c < a.d;
  float v[kC];
  auto clear = [&] {
#pragma unroll
    for (int j = 0; j < kC; ++j) v[j] = 0.f;
  };
  auto add = [&](const float* from) {
    if constexpr (kC == 4) {
      const float4 f = __ldcg(reinterpret_cast<const float4*>(from));
      v[0] += f.x;
      v[1] += f.y;
      v[2] += f.z;
      v[3] += f.w;
    } else {
      v[0] += __ldcg(from);
    }
  };
  // the strips' values, strip by strip
  auto total = [&] {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kC; ++j) s[strip][j * 32 + lane] = v[j];
    __syncthreads();
    if (strip == 0)
      for (int i = 1; i < 32; ++i)
#pragma unroll
        for (int j = 0; j < kC; ++j) v[j] += s[i][j * 32 + lane];
  };
  clear();
  if (blockIdx.y < 2) {
    float* out = blockIdx.y == 0 ? a.dw_post : a.dw_pre;
    if (out == nullptr) return;
    const float* from = a.workspace + (size_t)blockIdx.y * a.d + c;
    if (in)
#pragma unroll 10
      for (int i = strip; i < ctas; i += 32) add(from + (size_t)i * 2 * a.d);
    total();
    if (strip == 0 && in)
#pragma unroll
      for (int j = 0; j < kC; ++j) out[c + j] = v[j];
    return;
  }
  // (run i is the tokens from i * run on)
  const float* parts = a.workspace + (size_t)ctas * 2 * a.d + c;
  const int T_ = (int)a.T, G = a.gate_tokens, stride = share ? 1 : 32;
  const int rows = (T_ + G - 1) / G;
  for (int g = (int)(blockIdx.y - 2) * stride + (share ? 0 : strip); g < rows;
       g += (int)(gridDim.y - 2) * stride) {
    const int lo = g * G, hi = min(lo + G, T_);
    const int first = lo / run, last = (hi - 1) / run;
    if (first == last) continue;             // (complete in its run)
    clear();
    if (in)
#pragma unroll 4
      for (int i = first + (share ? strip : 0); i <= last; i += share ? 32 : 1)
        add(parts + ((size_t)i * 2 + (i * run >= lo ? 0 : 1)) * a.d);
    if (share) total();
    if (in && (!share || strip == 0))
#pragma unroll
      for (int j = 0; j < kC; ++j) from_f(v[j], static_cast<T*>(a.dgate) + (int64_t)g * a.lddgate + c + j);
  }
}

// ------------------------------------------------------------------ host side
template <int V> struct Int { static constexpr int value = V; };
template <typename F>
cudaError_t with_type(int dtype, bool wide, F f) {
  switch (dtype) {
    case DMOE_BF16: return wide ? f(__nv_bfloat16{}, Int<16>{}) : f(__nv_bfloat16{}, Int<2>{});
    case DMOE_FP16: return wide ? f(__half{}, Int<16>{}) : f(__half{}, Int<2>{});
    default: return wide ? f(float{}, Int<16>{}) : f(float{}, Int<4>{});
  }
}

int esize(int dtype) { return dtype == DMOE_FP32 ? 4 : 2; }

// every row can be read and written 16 bytes at a time
bool wide_rows(const NormArgs& a) {
  const uint64_t es = esize(a.dtype);
  uint64_t bits = a.d * es;
  for (const void* p : {a.x, a.y, a.gate, a.dr, a.dn, (const void*)a.r, (const void*)a.n,
                        (const void*)a.dx, (const void*)a.dy, (const void*)a.dgate})
    bits |= reinterpret_cast<uint64_t>(p);
  const void* p[] = {a.x, a.y, a.gate, a.dr, a.dn, a.r, a.n, a.dx, a.dy, a.dgate};
  const int64_t ld[] = {a.ldx, a.ldy, a.ldgate, a.lddr, a.lddn, a.ldr, a.ldn, a.lddx, a.lddy, a.lddgate};
  for (int i = 0; i < 10; ++i)
    if (p[i] != nullptr) bits |= (uint64_t)ld[i] * es;
  return bits % 16 == 0;
}

// threads of a row's group: a power of two, 8 at least, so that each holds at most kE elements
int group_width(int d, int n, int kE) {
  int w = 8;
  while ((int64_t)w * kE < (d + n - 1) / n * n) w *= 2;
  return w;
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

// Tokens that the shared memory holds rows of: two CTAs of 256 threads an SM, or one of more.
// `fixed`: what else a CTA needs.
int tokens_ahead(int block, size_t fixed, int row) {
  if (row == 0) return 2;
  const size_t room = (block > 256 ? 227 * 1024 : 113 * 1024) - fixed;
  return (int)std::max<size_t>(2, std::min<size_t>(4, room / row));
}

// CTAs of a launch (at most `most`) and the tokens of a group's run
int runs(int64_t T, int per_cta, int64_t most, int* ctas) {
  const int64_t run = (T + most * per_cta - 1) / (most * per_cta), groups = (T + run - 1) / run;
  *ctas = (int)((groups + per_cta - 1) / per_cta);
  return (int)run;
}

}  // namespace

// (groups of a CTA: one of the row's width, or several that hold at most 256 threads' 32 elements)
size_t norm_workspace_bytes(int64_t T, int d, int gate_tokens) {
  const int64_t ctas = std::min<int64_t>(kNormCtas, T);
  const int64_t per_cta = std::max(d, 256 * 32);
  return (size_t)(ctas * 2 * d + (gate_tokens > 0 ? ctas * 2 * per_cta : 0)) * sizeof(float);
}

cudaError_t launch_norm_residual(const NormArgs& a, cudaStream_t s) {
  return with_type(a.dtype, wide_rows(a), [&](auto z, auto w) {
    using T = decltype(z);
    constexpr int VB = decltype(w)::value;
    auto launch = [&](auto k, auto b) {
      constexpr int kE = decltype(k)::value, kBlock = decltype(b)::value;
      const int width = group_width(a.d, VB / (int)sizeof(T), kE);
      const bool full = VB == 16 && width >= 32 && width * kE == a.d && a.y != nullptr && a.r != nullptr &&
                        a.n != nullptr;
      int block = kBlock;
      // few rows: a CTA for each, as far as there are SMs
      while (block > width && block > 32 && a.T * width / block < 152) block /= 2;
      constexpr int row = Ahead<T, VB, kE, 2, kBlock, false>::kToken;
      const int depth = tokens_ahead(kBlock, 128, row);
      int ctas = 0;
      const int run = runs(a.T, block / width, kBlock > 256 ? 152 : 304, &ctas);
      const size_t smem = 128 + (size_t)depth * row;
      static std::atomic<uint32_t> done[2];
      auto* kernel = full ? norm_kernel<T, VB, kE, kBlock, VB == 16> : norm_kernel<T, VB, kE, kBlock, false>;
      const cudaError_t e = smem > 48 * 1024 ? raise_smem(kernel, done[full ? 1 : 0]) : cudaSuccess;
      if (e != cudaSuccess) return e;
      return launch_ex(kernel, dim3(ctas), dim3(block), smem, s, true, a, width, depth, run);
    };
    if (a.d <= 4096) return launch(Int<16>{}, Int<256>{});
    return a.d <= 8192 ? launch(Int<16>{}, Int<512>{}) : launch(Int<32>{}, Int<512>{});
  });
}

cudaError_t launch_norm_residual_backward(const NormArgs& a, cudaStream_t s) {
  return with_type(a.dtype, wide_rows(a), [&](auto z, auto w) {
    using T = decltype(z);
    constexpr int VB = decltype(w)::value;
    auto launch = [&](auto k, auto b) {
      constexpr int kE = decltype(k)::value, kBlock = decltype(b)::value;
      const int width = group_width(a.d, VB / (int)sizeof(T), kE), per_cta = kBlock / width;
      const bool full = VB == 16 && width >= 32 && width * kE == a.d && a.y != nullptr && a.dr != nullptr &&
                        a.dn != nullptr && a.dx != nullptr && a.dy != nullptr && a.dw_pre != nullptr;
      int ctas = 0;
      const int run = runs(a.T, per_cta, kBlock > 256 ? kNormCtas / 2 : kNormCtas, &ctas);
      // the reductions' words (three sums a warp, twice), the sums of wide rows, the rows ahead (and
      // in their place the groups' sums together)
      constexpr int row = Ahead<T, VB, kE, 4, kBlock, false>::kToken;
      constexpr size_t fixed = 192 * sizeof(float) + (kE > 8 ? 3 * kE * kBlock * sizeof(float) : 0);
      const int depth = tokens_ahead(kBlock, fixed, row);
      const size_t smem =
          fixed + std::max<size_t>((size_t)depth * row, per_cta > 1 ? kE * kBlock * sizeof(float) : 0);
      auto* kernel = full ? norm_backward_kernel<T, VB, kE, kBlock, VB == 16>
                          : norm_backward_kernel<T, VB, kE, kBlock, false>;
      cudaError_t e = cudaSuccess;
      if (smem > 48 * 1024) {
        static std::atomic<uint32_t> done[2];
        e = raise_smem(kernel, done[full ? 1 : 0]);
      }
      if (e == cudaSuccess)
        e = launch_ex(kernel, dim3(ctas), dim3(kBlock), smem, s, true, a, width, depth, run);
      const bool gates = a.dgate != nullptr && a.gate_tokens > 1;
      if (e != cudaSuccess || (a.dw_post == nullptr && a.dw_pre == nullptr && !gates)) return e;
      const int64_t rows = gates ? (a.T + a.gate_tokens - 1) / a.gate_tokens : 0;
      const bool share = gates && a.gate_tokens / run >= 16;
      const int extra = (int)std::min<int64_t>(share ? rows : (rows + 31) / 32, 64);
      return a.d % 4 == 0 ? launch_ex(norm_finish_kernel<T, 4>, dim3((a.d + 127) / 128, 2 + extra), dim3(1024),
                                      0, s, true, a, ctas, run, share ? 1 : 0)
                          : launch_ex(norm_finish_kernel<T, 1>, dim3((a.d + 31) / 32, 2 + extra), dim3(1024),
                                      0, s, true, a, ctas, run, share ? 1 : 0);
    };
    if (a.d <= 2048) return launch(Int<8>{}, Int<256>{});
    if (a.d <= 4096) return launch(Int<8>{}, Int<512>{});
    if (a.d <= 8192) return launch(Int<16>{}, Int<512>{});
    return launch(Int<32>{}, Int<512>{});
  });
}

}  // namespace dmoe

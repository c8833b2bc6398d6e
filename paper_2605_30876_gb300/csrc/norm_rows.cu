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

#include "dmoe_internal.cuh"

namespace dmoe {
namespace {

template <int VB> struct Raw;
template <> struct Raw<16> { using type = uint4; };
template <> struct Raw<4> { using type = uint32_t; };
template <> struct Raw<2> { using type = uint16_t; };

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_f(float v, float* o) { *o = v; }
__device__ __forceinline__ void from_f(float v, __half* o) { *o = __float2half_rn(v); }
__device__ __forceinline__ void from_f(float v, __nv_bfloat16* o) { *o = __float2bfloat16_rn(v); }

// kE elements of a row that a thread holds: pieces of VB bytes, `step` pieces apart
template <typename T, int VB, int kE>
struct Part {
  static constexpr int n = VB / (int)sizeof(T), kP = kE / n;
  using raw = typename Raw<VB>::type;
  union {
    raw r[kP];
    T e[kE];
  };
  __device__ __forceinline__ Part() {}
  __device__ __forceinline__ void load(const T* row, int v0, int step, int nv) {
#pragma unroll
    for (int j = 0; j < kP; ++j)
      if (v0 + j * step < nv)
        r[j] = __ldcs(reinterpret_cast<const raw*>(row) + v0 + j * step);
      else
        r[j] = raw{};
  }
  // a row that many tokens share
  __device__ __forceinline__ void load_shared(const T* row, int v0, int step, int nv) {
#pragma unroll
    for (int j = 0; j < kP; ++j)
      if (v0 + j * step < nv)
        r[j] = __ldg(reinterpret_cast<const raw*>(row) + v0 + j * step);
      else
        r[j] = raw{};
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int j = 0; j < kP; ++j) r[j] = raw{};
  }
  __device__ __forceinline__ float get(int i) const { return to_f(e[i]); }
  __device__ __forceinline__ void set(int i, float v) { from_f(v, &e[i]); }
  __device__ __forceinline__ void store(T* row, int v0, int step, int nv) const {
#pragma unroll
    for (int j = 0; j < kP; ++j)
      if (v0 + j * step < nv) __stcs(reinterpret_cast<raw*>(row) + v0 + j * step, r[j]);
  }
};

// column of element i of a thread's part
template <typename T, int VB>
__device__ __forceinline__ int column(int i, int v0, int step) {
  constexpr int n = VB / (int)sizeof(T);
  return (v0 + i / n * step) * n + i % n;
}
// fp32 vectors of the row's width (weights, sums), the elements that a part holds
template <typename T, int VB, int kE>
__device__ __forceinline__ void load_vector(float (&o)[kE], const float* w, int v0, int step, int nv,
                                            float none) {
  constexpr int n = VB / (int)sizeof(T);
#pragma unroll
  for (int i = 0; i < kE; i += n) {
    const bool in = w != nullptr && v0 + i / n * step < nv;
    const float* from = w + column<T, VB>(i, v0, step);
    if constexpr (n % 4 == 0) {
#pragma unroll
      for (int j = 0; j < n; j += 4) {
        const float4 f = in ? __ldg(reinterpret_cast<const float4*>(from + j))
                            : make_float4(none, none, none, none);
        o[i + j] = f.x;
        o[i + j + 1] = f.y;
        o[i + j + 2] = f.z;
        o[i + j + 3] = f.w;
      }
    } else {
#pragma unroll
      for (int j = 0; j < n; ++j) o[i + j] = in ? __ldg(from + j) : none;
    }
  }
}
template <typename T, int VB, int kE>
__device__ __forceinline__ void store_vector(const float (&v)[kE], float* w, int v0, int step, int nv) {
  constexpr int n = VB / (int)sizeof(T);
#pragma unroll
  for (int i = 0; i < kE; i += n)
    if (v0 + i / n * step < nv) {
      float* to = w + column<T, VB>(i, v0, step);
      if constexpr (n % 4 == 0) {
#pragma unroll
        for (int j = 0; j < n; j += 4)
          *reinterpret_cast<float4*>(to + j) = make_float4(v[i + j], v[i + j + 1], v[i + j + 2], v[i + j + 3]);
      } else {
#pragma unroll
        for (int j = 0; j < n; ++j) to[j] = v[i + j];
      }
    }
}

// Sums of K values over the kG... threads of a row's group (`width`, a power of two), the same in
// every thread. Groups of more than a warp pass `scratch` (K floats per warp of the CTA, twice) and a
// barrier of their own; `flip` changes from call to call, so that one barrier is enough.
template <int K>
__device__ __forceinline__ void group_sum(float (&v)[K], int width, int group, float* scratch, int& flip) {
  for (int o = min(width, 32) >> 1; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  if (width <= 32) return;
  const int warp = threadIdx.x >> 5, nw = blockDim.x >> 5, per = width >> 5;
  float* s = scratch + flip * nw * K;
  flip ^= 1;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) s[warp * K + k] = v[k];
  asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(width) : "memory");
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = 0.f;
  for (int w = group * per; w < (group + 1) * per; ++w)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += s[w * K + k];
}

__device__ __forceinline__ float rstd_of(float sum, int d, float eps) {
  return 1.f / sqrtf(sum / (float)d + eps);
}

// A group of `width` threads takes every groups-th row.
template <typename T, int VB, int kE>
__global__ void __launch_bounds__(512)
norm_kernel(const NormArgs a, int width) {
  extern __shared__ float scratch[];
  using P = Part<T, VB, kE>;
  pdl_wait();
  pdl_launch_dependents();
  const int group = threadIdx.x / width, v0 = threadIdx.x % width, nv = a.d / P::n;
  const int per_cta = blockDim.x / width;
  const int64_t step = (int64_t)gridDim.x * per_cta;
  int flip = 0;
  // (all threads of a warp stay to the end: its groups' sums are taken together)
  const int64_t first = (int64_t)blockIdx.x * per_cta, rounds = (a.T - first + step - 1) / step;
  for (int64_t i = 0; i < rounds; ++i) {
    const int64_t t = first + group + i * step;
    const bool in = t < a.T;
    const int n_in = in ? nv : 0;
    P x, y;
    if (a.x != nullptr) x.load(static_cast<const T*>(a.x) + t * a.ldx, v0, width, n_in); else x.zero();
    if (a.y != nullptr) y.load(static_cast<const T*>(a.y) + t * a.ldy, v0, width, n_in); else y.zero();
    float r[kE];
    float ry = 1.f;
    if (a.w_post != nullptr) {
      float s[1] = {0.f};
#pragma unroll
      for (int e = 0; e < kE; ++e) s[0] = fmaf(y.get(e), y.get(e), s[0]);
      group_sum(s, width, group, scratch, flip);
      ry = rstd_of(s[0], a.d, a.eps);
      float w[kE];
      load_vector<T, VB>(w, a.w_post, v0, width, n_in, 0.f);
#pragma unroll
      for (int e = 0; e < kE; ++e) r[e] = y.get(e) * ry * w[e];
    } else {
#pragma unroll
      for (int e = 0; e < kE; ++e) r[e] = y.get(e);
    }
    if (a.gate != nullptr) {
      P g;
      const int64_t row = in ? (int64_t)((uint32_t)t / (uint32_t)a.gate_tokens) : 0;
      g.load_shared(static_cast<const T*>(a.gate) + row * a.ldgate, v0, width, n_in);
#pragma unroll
      for (int e = 0; e < kE; ++e) r[e] *= g.get(e);
    }
    float s[1] = {0.f};
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      r[e] = fmaf(a.scale, x.get(e), r[e]);
      s[0] = fmaf(r[e], r[e], s[0]);
    }
    if (a.r != nullptr) {
#pragma unroll
      for (int e = 0; e < kE; ++e) x.set(e, r[e]);
      x.store(static_cast<T*>(a.r) + t * a.ldr, v0, width, n_in);
    }
    float rr = 1.f;
    if (a.w_pre != nullptr) {
      group_sum(s, width, group, scratch, flip);
      rr = rstd_of(s[0], a.d, a.eps);
      float w[kE];
      load_vector<T, VB>(w, a.w_pre, v0, width, n_in, 0.f);
#pragma unroll
      for (int e = 0; e < kE; ++e) y.set(e, r[e] * rr * w[e]);
      y.store(static_cast<T*>(a.n) + t * a.ldn, v0, width, n_in);
    }
    if (a.stats != nullptr && in && v0 == 0) {
      a.stats[t] = ry;
      a.stats[a.T + t] = rr;
    }
  }
}

// The run of tokens that group i of n takes.
__device__ __forceinline__ int run_begin(int64_t T, int64_t i, int64_t n) { return (int)(i * T / n); }

// workspace: fp32 [CTAs][2][d] (dw_post, dw_pre), then [groups][2][d] (the first and the last gate
// row of a run, where they are not complete)
//
// Up to 2048 elements a thread holds eight, and its sums over tokens, weights and gates stay in
// registers. Wider rows take 16 (or 32) a thread: their sums lie in shared memory, a thread's own
// places, and weights and gates come from L1 for every row.
template <typename T, int VB, int kE>
__global__ void __launch_bounds__(kE <= 8 ? 256 : 512, kE <= 8 ? 2 : 1)
norm_backward_kernel(const NormArgs a, int width) {
  constexpr bool kShared = kE > 8;
  extern __shared__ float4 smem4[];
  float* scratch = reinterpret_cast<float*>(smem4);
  using P = Part<T, VB, kE>;
  pdl_wait();
  pdl_launch_dependents();
  const int group = threadIdx.x / width, v0 = threadIdx.x % width, nv = a.d / P::n;
  const int per_cta = blockDim.x / width, G = a.gate_tokens;
  const int64_t groups = (int64_t)gridDim.x * per_cta, me = (int64_t)blockIdx.x * per_cta + group;
  const int begin = run_begin(a.T, me, groups), end = run_begin(a.T, me + 1, groups);
  const float inv_d = 1.f / (float)a.d;
  float* part_w = a.workspace + (size_t)blockIdx.x * 2 * a.d;
  float* part_g = a.workspace + (size_t)gridDim.x * 2 * a.d + (size_t)me * 2 * a.d;
  int flip = 0;
  constexpr int kReg = kShared ? 1 : kE;
  float A_[kReg], post_[kReg], pre_[kReg], w_post_[kReg], w_pre_[kReg], gate_[kReg];
  // [sum][element][thread] behind the reductions' words
  float4* sums = smem4 + 48 + threadIdx.x;
  auto at = [&](int which, int e) -> float4& { return sums[(which * (kE / 4) + e / 4) * blockDim.x]; };
  // sum[which][e .. e + 3] = f(sum, element) for four elements at a time
  auto update = [&](int which, auto f) {
    if constexpr (kShared) {
#pragma unroll
      for (int e = 0; e < kE; e += 4) {
        float4 v = at(which, e);
        v.x = f(v.x, e);
        v.y = f(v.y, e + 1);
        v.z = f(v.z, e + 2);
        v.w = f(v.w, e + 3);
        at(which, e) = v;
      }
    } else {
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        float& v = which == 0 ? A_[e] : which == 1 ? post_[e] : pre_[e];
        v = f(v, e);
      }
    }
  };
  for (int which = 0; which < 3; ++which) update(which, [](float, int) { return 0.f; });
  if constexpr (!kShared) {
    load_vector<T, VB>(w_post_, a.w_post, v0, width, nv, 1.f);
    load_vector<T, VB>(w_pre_, a.w_pre, v0, width, nv, 0.f);
#pragma unroll
    for (int e = 0; e < kE; ++e) gate_[e] = 1.f;
  }

  P x, y, dr, dn;
  float ry = 0.f, rr = 0.f;
  auto load = [&](int64_t t, bool in) {
    const int n_in = in ? nv : 0;
    x.load(static_cast<const T*>(a.x) + t * a.ldx, v0, width, n_in);
    if (a.y != nullptr) y.load(static_cast<const T*>(a.y) + t * a.ldy, v0, width, n_in); else y.zero();
    if (a.dr != nullptr) dr.load(static_cast<const T*>(a.dr) + t * a.lddr, v0, width, n_in); else dr.zero();
    if (a.dn != nullptr) dn.load(static_cast<const T*>(a.dn) + t * a.lddn, v0, width, n_in); else dn.zero();
    ry = in ? __ldg(a.stats + t) : 0.f;
    rr = in ? __ldg(a.stats + a.T + t) : 0.f;
  };
  load(begin, begin < end);
  int row = G > 0 ? begin / G : 0;
  int row_end = (int)(G > 0 ? min((int64_t)(row + 1) * G, a.T) : a.T);
  int seg = begin;                       // the first token of the run in this gate row
  auto load_gate = [&](float (&g)[kE]) {
    if (a.gate == nullptr) {
#pragma unroll
      for (int e = 0; e < kE; ++e) g[e] = 1.f;
      return;
    }
    P v;
    v.load_shared(static_cast<const T*>(a.gate) + (int64_t)row * a.ldgate, v0, width, nv);
#pragma unroll
    for (int e = 0; e < kE; ++e) g[e] = v.get(e);
  };
  if constexpr (!kShared)
    if (begin < end) load_gate(gate_);
  // a warp's groups (width < 32) take as many turns as the longest of them
  const int turns = width < 32 ? (int)((a.T + groups - 1) / groups) : end - begin;
  for (int i = 0; i < turns; ++i) {
    const int t = begin + i;
    const bool in = t < end;
    const int n_in = in ? nv : 0;
    float yh[kE], rh[kE], q[kE], c[kE];
    float s[3] = {0.f, 0.f, 0.f};
    const float rr_t = rr, ry_t = ry;
    if constexpr (kShared) {
      load_vector<T, VB>(c, a.w_post, v0, width, n_in, 1.f);
      if (a.gate != nullptr && in) {
        float g[kE];
        load_gate(g);
#pragma unroll
        for (int e = 0; e < kE; ++e) c[e] *= g[e];
      }
      load_vector<T, VB>(q, a.w_pre, v0, width, n_in, 0.f);
    } else {
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        c[e] = gate_[e] * w_post_[e];
        q[e] = w_pre_[e];
      }
    }
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const float v = dn.get(e) * q[e];
      yh[e] = y.get(e) * ry_t;
      rh[e] = fmaf(a.scale, x.get(e), yh[e] * c[e]) * rr_t;
      q[e] = fmaf(rr_t, v, dr.get(e));
      s[0] = fmaf(v, rh[e], s[0]);
      s[1] = fmaf(q[e], c[e] * yh[e], s[1]);
      s[2] = fmaf(rh[e], c[e] * yh[e], s[2]);
    }
    if (a.dw_pre != nullptr) update(2, [&](float v, int e) { return fmaf(dn.get(e), rh[e], v); });
    load(t + 1, t + 1 < end);            // the next token's rows are on their way during the sums
    group_sum(s, width, group, scratch, flip);
    const float m1 = s[0] * inv_d * rr_t;
    const float m2 = a.w_post != nullptr ? fmaf(-m1, s[2], s[1]) * inv_d : 0.f;
    P o;
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      q[e] = fmaf(-m1, rh[e], q[e]);
      o.set(e, a.scale * q[e]);
    }
    if (a.dx != nullptr) o.store(static_cast<T*>(a.dx) + (int64_t)t * a.lddx, v0, width, n_in);
    if (a.dy != nullptr) {
#pragma unroll
      for (int e = 0; e < kE; ++e) o.set(e, ry_t * fmaf(-m2, yh[e], q[e] * c[e]));
      o.store(static_cast<T*>(a.dy) + (int64_t)t * a.lddy, v0, width, n_in);
    }
    const bool gate_sums = a.dgate != nullptr || a.dw_post != nullptr;
    if (gate_sums) update(0, [&](float v, int e) { return fmaf(q[e], yh[e], v); });
    if (!in || (t + 1 != row_end && t + 1 != end)) continue;
    // the end of a gate row, or of the run
    if (gate_sums) {
      float A[kE];
      if constexpr (kShared) load_gate(q);
#pragma unroll
      for (int e = 0; e < kE; ++e) A[e] = 0.f;
      update(0, [&](float v, int e) { A[e] = v; return 0.f; });
      update(1, [&](float v, int e) {
        if constexpr (kShared) return fmaf(q[e], A[e], v);
        else return fmaf(gate_[e], A[e], v);
      });
      if (a.dgate != nullptr) {
        if constexpr (kShared) load_vector<T, VB>(c, a.w_post, v0, width, nv, 1.f);
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          if constexpr (kShared) A[e] *= c[e];
          else A[e] *= w_post_[e];
        }
        if ((int64_t)row * G == seg && t + 1 == row_end) {   // complete
#pragma unroll
          for (int e = 0; e < kE; ++e) o.set(e, A[e]);
          o.store(static_cast<T*>(a.dgate) + (int64_t)row * a.lddgate, v0, width, nv);
        } else {
          store_vector<T, VB>(A, part_g + (seg == begin ? 0 : a.d), v0, width, nv);
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
  for (int which = 1; which < 3; ++which) {
    if ((which == 1 ? a.dw_post : a.dw_pre) == nullptr) continue;
    float v[kE];
    update(which, [&](float f, int e) { v[e] = f; return f; });
    if (per_cta > 1) {
      __syncthreads();
      // [element][thread], behind the reductions' words (and the sums)
      float* mine = scratch + 192 + (kShared ? 3 * kE * blockDim.x : 0) + threadIdx.x;
#pragma unroll
      for (int e = 0; e < kE; ++e) mine[e * blockDim.x] = v[e];
      __syncthreads();
      if (group == 0)
#pragma unroll
        for (int e = 0; e < kE; ++e)
          for (int g = 1; g < per_cta; ++g) v[e] += mine[e * blockDim.x + g * width];
    }
    if (group == 0) store_vector<T, VB>(v, part_w + (which - 1) * a.d, v0, width, nv);
  }
}

// Sums of what the CTAs and runs left, 32 columns a block in 32 strips: the first two rows of the grid
// add the weights' parts, the others the gate rows that no run held alone (`share`: a block has one gate
// row of many runs, else each strip has one of its own).
template <typename T>
__global__ void __launch_bounds__(1024)
norm_finish_kernel(const NormArgs a, int ctas, int64_t groups, int share) {
  __shared__ float s[32][33];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, strip = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  const bool in = c < a.d;
  // the strips' values, strip by strip
  auto total = [&](float v) {
    __syncthreads();
    s[strip][lane] = v;
    __syncthreads();
    if (strip == 0)
      for (int i = 1; i < 32; ++i) v += s[i][lane];
    return v;
  };
  if (blockIdx.y < 2) {
    float* out = blockIdx.y == 0 ? a.dw_post : a.dw_pre;
    if (out == nullptr) return;
    const float* from = a.workspace + (size_t)blockIdx.y * a.d + c;
    float v = 0.f;
    if (in)
#pragma unroll 10
      for (int i = strip; i < ctas; i += 32) v += __ldcg(from + (size_t)i * 2 * a.d);
    v = total(v);
    if (strip == 0 && in) out[c] = v;
    return;
  }
  const float* parts = a.workspace + (size_t)ctas * 2 * a.d + c;
  const int G = a.gate_tokens, per = share ? 1 : 32;
  const int64_t rows = (a.T + G - 1) / G;
  for (int64_t g = (int64_t)(blockIdx.y - 2) * per + (share ? 0 : strip); g < rows;
       g += (int64_t)(gridDim.y - 2) * per) {
    const int64_t lo = g * G, hi = min(lo + G, a.T);
    // the runs that hold tokens lo and hi - 1 (run i is [i T / n, (i + 1) T / n))
    const int64_t first = ((lo + 1) * groups - 1) / a.T, last = (hi * groups - 1) / a.T;
    if (first == last) continue;             // (complete in its run)
    float v = 0.f;
    if (in)
#pragma unroll 4
      for (int64_t i = first + (share ? strip : 0); i <= last; i += share ? 32 : 1) {
        const int begin = run_begin(a.T, i, groups);
        if (begin < run_begin(a.T, i + 1, groups))   // (a run may have no tokens)
          v += __ldcg(parts + ((size_t)i * 2 + (begin >= lo ? 0 : 1)) * a.d);
      }
    if (share) v = total(v);
    if (in && (!share || strip == 0)) from_f(v, static_cast<T*>(a.dgate) + g * a.lddgate + c);
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

int64_t run_groups(int64_t T, int width, int block, int* ctas) {
  const int per = block / width;
  *ctas = (int)std::min<int64_t>(kNormCtas, (T + per - 1) / per);
  return (int64_t)*ctas * per;
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
    constexpr int VB = decltype(w)::value, kE = 32;
    const int width = group_width(a.d, VB / (int)sizeof(T), kE);
    int block = std::max(width, 256);
    // few rows: a CTA for each, as far as there are SMs
    while (block > width && block > 32 && a.T * width / block < 152) block /= 2;
    const int per = block / width;
    const int64_t need = (a.T + per - 1) / per;
    const int grid = (int)std::min<int64_t>(need, 152 * 8);
    return launch_ex(norm_kernel<T, VB, kE>, dim3(grid), dim3(block), 2 * block / 32 * sizeof(float), s,
                     true, a, width);
  });
}

cudaError_t launch_norm_residual_backward(const NormArgs& a, cudaStream_t s) {
  return with_type(a.dtype, wide_rows(a), [&](auto z, auto w) {
    using T = decltype(z);
    constexpr int VB = decltype(w)::value;
    auto run = [&](auto k) {
      constexpr int kE = decltype(k)::value;
      const int width = group_width(a.d, VB / (int)sizeof(T), kE);
      const int block = std::max(width, 256);
      int ctas = 0;
      const int64_t groups = run_groups(a.T, width, block, &ctas);
      // the reductions' words (three sums a warp, twice), the sums of wide rows, the groups' together
      const size_t smem = 192 * sizeof(float) + (kE > 8 ? 3 * kE * block * sizeof(float) : 0) +
                          (block > width ? kE * block * sizeof(float) : 0);
      cudaError_t e = cudaSuccess;
      if (smem > 48 * 1024) {
        static std::atomic<uint32_t> done;
        e = raise_smem(norm_backward_kernel<T, VB, kE>, done);
      }
      if (e == cudaSuccess)
        e = launch_ex(norm_backward_kernel<T, VB, kE>, dim3(ctas), dim3(block), smem, s, true, a, width);
      const bool gates = a.dgate != nullptr && a.gate_tokens > 1;
      if (e != cudaSuccess || (a.dw_post == nullptr && a.dw_pre == nullptr && !gates)) return e;
      const int64_t rows = gates ? (a.T + a.gate_tokens - 1) / a.gate_tokens : 0;
      const bool share = gates && groups / rows >= 16;
      const int extra = (int)std::min<int64_t>(share ? rows : (rows + 31) / 32, 64);
      return launch_ex(norm_finish_kernel<T>, dim3((a.d + 31) / 32, 2 + extra), dim3(1024), 0, s, true, a,
                       ctas, groups, share ? 1 : 0);
    };
    if (a.d <= 2048) return run(Int<8>{});
    if (a.d <= 8192) return run(Int<16>{});
    return run(Int<32>{});
  });
}

}  // namespace dmoe

// The norms around a block, with its gate and its residual, in one pass:
//   p = y * ry * w_post,  r = scale * x + gate * p,  n = r * rr * w_pre
//   ry = 1 / sqrt(mean(y^2) + eps),  rr = 1 / sqrt(mean(r^2) + eps)
// Both directions are bound by the bytes of their rows, each read once and written once. A row is held
// in registers by a group of threads, a few pieces of 16 bytes each;
// groups go on from row to row. The gradients: norm_rows_backward.cu.
#include "norm_rows.cuh"

namespace dmoe {
namespace {

// A group of `width` threads takes the run of `run` rows from group * run on; the next depth - 1 are on
// their way. kFull: x, y, r and n are all there, a row is exactly what its group holds, and a group is a
// warp or more. (Asking for each of them every time is a fifth of the instructions: 16384 rows of 2048 in bf16 without
// a gate, cold, a launch's own time: 45.2 us without this form and 43.6 with it, 6.1 TB/s; the backward pass's first launch
// 77.8 and 68, 5.9 TB/s.)
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
  GroupSum<1> group_sum(scratch, width, group);
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
  // the next gate row, on its way while a run of tokens has this one (a gate for each token, 14511 rows of 1632: 57 us
  // asked for in turn, 47 so)
  Part<T, VB, kHold ? kE : P::n, kFull> gate_next;
  auto ask_gate = [&](int g) {
    if (a.gate != nullptr && (int64_t)g * G < end)
      gate_next.load_shared(static_cast<const T*>(a.gate) + (int64_t)g * a.ldgate, v0, width, nv);
  };
  if constexpr (kHold)
    if (begin < end) ask_gate(row);
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
        if constexpr (kHold) g = gate_next;
        else g.load_shared(static_cast<const T*>(a.gate) + (int64_t)row * a.ldgate, v0, width, nv);
#pragma unroll
        for (int e = 0; e < kH; ++e) post[e] = mul2(post[e], g.get(e));
        if constexpr (kHold) ask_gate(row + 1);
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
      group_sum(s);
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
      group_sum(s);
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

}  // namespace

cudaError_t launch_norm_residual(const NormArgs& a, cudaStream_t s) {
  return with_type(a.dtype, piece_of_rows(a), [&](auto z, auto w) {
    using T = decltype(z);
    constexpr int VB = decltype(w)::value;
    auto launch = [&](auto k, auto b) {
      constexpr int kE = decltype(k)::value, kBlock = decltype(b)::value;
      const int width = group_width(a.d, VB / (int)sizeof(T), kE);
      const bool full = VB == 16 && width >= 32 && width * kE == a.d && a.y != nullptr && a.r != nullptr &&
                        a.n != nullptr;
      int per_cta = std::max(1, kBlock / width);
      const int per_sm = ctas_per_sm(kBlock, per_cta * width);
      // few rows: a CTA for each, as far as there are SMs
      while (per_cta > 1 && per_cta * width > 32 && a.T / per_cta < 152) per_cta = (per_cta + 1) / 2;
      const int block = per_cta * width;
      constexpr int row = Ahead<T, VB, kE, 2, kBlock, false>::kToken;
      const int depth = tokens_ahead(per_sm, 128, row);
      int ctas = 0;
      const int run = runs(a.T, per_cta, 152 * per_sm, &ctas);
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

}  // namespace dmoe

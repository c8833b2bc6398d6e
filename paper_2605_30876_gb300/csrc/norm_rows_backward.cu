// The gradients of the norms around a block (norm_rows.cu).
//   p = y * ry * w_post,  r = scale * x + gate * p,  n = r * rr * w_pre
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
#include "norm_rows.cuh"

namespace dmoe {
namespace {

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
  GroupSum<3> group_sum(scratch, width, group);
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
    // (r hat, for which x is read, counts through dn alone)
    rows[0] = kFull || a.dn != nullptr ? row_at(static_cast<const T*>(a.x), t, ldx) : nullptr;
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
    group_sum(s);
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

}  // namespace

// (groups of a CTA: one of the row's width, or several that hold at most 256 threads' 32 elements)
size_t norm_workspace_bytes(int64_t T, int d, int gate_tokens) {
  const int64_t ctas = std::min<int64_t>(kNormCtas, T);
  const int64_t per_cta = std::max(d, 256 * 32);
  return (size_t)(ctas * 2 * d + (gate_tokens > 0 ? ctas * 2 * per_cta : 0)) * sizeof(float);
}

cudaError_t launch_norm_residual_backward(const NormArgs& a, cudaStream_t s) {
  return with_type(a.dtype, piece_of_rows(a), [&](auto z, auto w) {
    using T = decltype(z);
    constexpr int VB = decltype(w)::value;
    auto launch = [&](auto k, auto b) {
      constexpr int kE = decltype(k)::value, kBlock = decltype(b)::value;
      const int width = group_width(a.d, VB / (int)sizeof(T), kE), per_cta = std::max(1, kBlock / width);
      const int block = per_cta * width, per_sm = ctas_per_sm(kBlock, block);
      const bool full = VB == 16 && width >= 32 && width * kE == a.d && a.y != nullptr && a.dr != nullptr &&
                        a.dn != nullptr && a.dx != nullptr && a.dy != nullptr && a.dw_pre != nullptr;
      int ctas = 0;
      const int run = runs(a.T, per_cta, 152 * per_sm, &ctas);
      // the reductions' words (three sums a warp, twice), the sums of wide rows, the rows ahead (and
      // in their place the groups' sums together)
      constexpr int row = Ahead<T, VB, kE, 4, kBlock, false>::kToken;
      constexpr size_t fixed = 192 * sizeof(float) + (kE > 8 ? 3 * kE * kBlock * sizeof(float) : 0);
      const int depth = tokens_ahead(per_sm, fixed, row);
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
        e = launch_ex(kernel, dim3(ctas), dim3(block), smem, s, true, a, width, depth, run);
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

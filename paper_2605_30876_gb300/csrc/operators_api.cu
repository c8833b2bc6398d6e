// C-ABI entry points of the calls that do a layer by its parts: argument checks and launches.
// Nothing here allocates device memory or synchronises.
#include <algorithm>

#include "dmoe_internal.cuh"
#include "q4.cuh"

using namespace dmoe;

namespace {

constexpr int64_t kMaxPairs = 1 << 30;
constexpr int kMaxRowWidth = 1 << 20;

std::atomic<int32_t> g_q4_hold{0};       // dmoe_q4_set_debug_hold
std::atomic<int32_t> g_expert_hold{0};   // dmoe_expert_set_debug_hold

dmoe_status status_of(cudaError_t e) {
  if (e == cudaSuccess) return DMOE_OK;
  set_last_error(e);
  return DMOE_ERR_CUDA;
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool given16(const void* p) { return p != nullptr && aligned(p, 16); }
bool null_or16(const void* p) { return aligned(p, 16); }

dmoe_status check_pairs(int64_t T, int32_t k) {
  if (T < 0 || k <= 0) return DMOE_ERR_INVALID_ARG;
  if (k > kMaxTopK || T > kMaxPairs / k) return DMOE_ERR_UNSUPPORTED;
  return DMOE_OK;
}

dmoe_status check_sort(int64_t T, int32_t k, int32_t E) {
  const dmoe_status st = check_pairs(T, k);
  if (st != DMOE_OK) return st;
  if (E <= 0) return DMOE_ERR_INVALID_ARG;
  return E > kMaxExperts ? DMOE_ERR_UNSUPPORTED : DMOE_OK;
}

dmoe_status check_rows(int32_t dtype, int64_t T, int32_t k, int32_t d) {
  if (dtype < DMOE_BF16 || dtype > DMOE_FP32 || d <= 0) return DMOE_ERR_INVALID_ARG;
  if (d > kMaxRowWidth) return DMOE_ERR_UNSUPPORTED;
  return check_pairs(T, k);
}

// a matrix of rows: there, on an element boundary, its stride at least its width
bool matrix(const void* p, int64_t ld, int32_t dtype, int32_t d) {
  return p != nullptr && aligned(p, dtype == DMOE_FP32 ? 4 : 2) && ld >= d;
}

dmoe_status check_q4(const dmoe_q4_desc* d) {
  if (d == nullptr) return DMOE_ERR_INVALID_ARG;
  if (d->n_experts <= 0 || d->n_out <= 0 || d->n_in <= 0 || d->group <= 0)
    return DMOE_ERR_INVALID_ARG;
  if (d->group != 32 && d->group != 64 && d->group != 128) return DMOE_ERR_UNSUPPORTED;
  if (d->n_experts > kMaxQ4Experts || d->n_out > 65536 || d->n_in > kMaxDModel ||
      d->n_in % d->group != 0)
    return DMOE_ERR_UNSUPPORTED;
  return DMOE_OK;
}

dmoe_status run_q4(const dmoe_q4_desc* desc, int64_t R, int32_t n_groups, const void* x,
                   int64_t ldx, int64_t T_x, const int32_t* rows, int32_t k,
                   const int32_t* offsets, const int32_t* expert_ids,
                   std::initializer_list<const void*> weights, void* y, int64_t ldy,
                   int32_t y_dtype, void* stream) {
  const dmoe_status st = check_q4(desc);
  if (st != DMOE_OK) return st;
  if (R < 0 || T_x < 0 || n_groups <= 0 || k <= 0 || ldx < desc->n_in || ldy < desc->n_out ||
      (y_dtype != DMOE_BF16 && y_dtype != DMOE_FP32))
    return DMOE_ERR_INVALID_ARG;
  if (R > kMaxPairs || n_groups > kMaxQ4Experts || k > kMaxTopK) return DMOE_ERR_UNSUPPORTED;
  // the kernel counts its units (64 rows x 64 outputs of a group) in 32 bits, whatever the offsets hold
  if ((R / 64 + 1) * ((desc->n_out + 63) / 64) * n_groups > INT32_MAX) return DMOE_ERR_UNSUPPORTED;
  if ((offsets == nullptr && n_groups != 1) ||
      (expert_ids == nullptr && n_groups > desc->n_experts) || (rows == nullptr && T_x < R))
    return DMOE_ERR_INVALID_ARG;
  if (R == 0) return DMOE_OK;
  for (const void* w : weights)
    if (!given16(w)) return DMOE_ERR_INVALID_ARG;
  if (!null_or16(rows) || !null_or16(offsets) || !null_or16(expert_ids) || T_x == 0 ||
      x == nullptr || y == x || !matrix(y, ldy, y_dtype, desc->n_out))
    return DMOE_ERR_INVALID_ARG;
  // rows of x are read 16 bytes at a time, their indices held in 32 bits
  if (!aligned(x, 16) || ldx % 8 != 0) return DMOE_ERR_INVALID_ARG;
  if (T_x > (int64_t)INT32_MAX || ldx >= (int64_t)1 << 39) return DMOE_ERR_UNSUPPORTED;
  Q4Args a{};
  a.x = static_cast<const __nv_bfloat16*>(x);
  a.ldx = ldx;
  a.T_x = T_x;
  a.rows = rows;
  a.k = k;
  a.offsets = offsets;
  a.expert_ids = expert_ids;
  int m = 0;
  for (const void* w : weights) {
    (m % 2 == 0 ? a.codes : a.scales)[m / 2] = w;
    ++m;
  }
  a.y = y;
  a.ldy = ldy;
  a.y_fp32 = y_dtype == DMOE_FP32;
  a.gated = weights.size() == 4;
  a.R = R;
  a.n_groups = n_groups;
  a.n_experts = desc->n_experts;
  a.hold = g_q4_hold.load(std::memory_order_relaxed) != 0 ? 1 : 0;
  return status_of(launch_q4_linear(a, *desc, static_cast<cudaStream_t>(stream)));
}

dmoe_status check_expert(const dmoe_expert_desc* d, int64_t R, int64_t n_groups) {
  if (d == nullptr || R < 0 || n_groups <= 0 || d->n_experts <= 0 || d->d_model <= 0 ||
      d->d_ff <= 0 || (d->dtype != DMOE_BF16 && d->dtype != DMOE_FP16))
    return DMOE_ERR_INVALID_ARG;
  // rows and matrices are read in boxes of 16 bytes; a unit's place is packed in 8 bits each
  if (d->d_model % 8 != 0 || d->d_ff % 8 != 0 || d->d_model > kMaxDModel || d->d_ff > kMaxDModel ||
      d->n_experts > kMaxFfnExperts || n_groups > kMaxFfnExperts || R > kMaxPairs)
    return DMOE_ERR_UNSUPPORTED;
  // units (up to 256 rows x 128 features of a group) are counted in 32 bits, whatever offsets hold
  const int64_t tiles = (std::max(d->d_model, d->d_ff) + 127) / 128;
  if ((R / 32 < 8 ? 2 : R / 256 + 1) * tiles * n_groups > INT32_MAX) return DMOE_ERR_UNSUPPORTED;
  return DMOE_OK;
}

// a matrix whose rows are read or written 16 bytes at a time
bool matrix16(const void* p, int64_t ld, int32_t d) {
  return given16(p) && ld >= d && ld % 8 == 0 && ld < (int64_t)1 << 38;
}

// no output is an input that is read, or another output (NULL: there is none)
bool apart(std::initializer_list<const void*> outs, std::initializer_list<const void*> ins) {
  for (const void* const* o = outs.begin(); o != outs.end(); ++o) {
    if (*o == nullptr) continue;
    if (std::find(ins.begin(), ins.end(), *o) != ins.end() || std::find(o + 1, outs.end(), *o) != outs.end())
      return false;
  }
  return true;
}

FfnArgs expert_args(const dmoe_expert_desc* d, int64_t R, int32_t n_groups, const int32_t* offsets,
                    const void* w_gate, const void* w_up, const void* w_down) {
  FfnArgs a{};
  a.dtype = d->dtype;
  a.n_experts = d->n_experts;
  a.d = d->d_model;
  a.I = d->d_ff;
  a.R = R;
  a.n_groups = n_groups;
  a.offsets = offsets;
  a.w_gate = w_gate;
  a.w_up = w_up;
  a.w_down = w_down;
  a.hold = g_expert_hold.load(std::memory_order_relaxed) != 0 ? 1 : 0;
  return a;
}

dmoe_status check_norm(const dmoe_norm_desc* d) {
  if (d == nullptr || d->dtype < DMOE_BF16 || d->dtype > DMOE_FP32 || d->d <= 0 || d->T < 0 ||
      d->gate_tokens < 0 || !(d->eps >= 0.f))
    return DMOE_ERR_INVALID_ARG;
  return d->d > kMaxDModel || d->T > kMaxPairs ? DMOE_ERR_UNSUPPORTED : DMOE_OK;
}

// a row's place is computed from 32-bit numbers of tokens and bytes
bool strides_fit(std::initializer_list<int64_t> lds) {
  for (int64_t ld : lds)
    if (ld >= (int64_t)1 << 30) return false;
  return true;
}

// what both directions read: x; y, its weight and its gate, or none of the three
bool norm_inputs(const dmoe_norm_desc* d, const void* x, int64_t ldx, const void* y, int64_t ldy,
                 const float* w_post, const void* gate, int64_t ldgate, const float* w_pre,
                 NormArgs* a) {
  if (!matrix(x, ldx, d->dtype, d->d) || (y != nullptr && !matrix(y, ldy, d->dtype, d->d)) ||
      (y == nullptr && (w_post != nullptr || gate != nullptr)) || !null_or16(w_post) ||
      !null_or16(w_pre) ||
      (gate != nullptr && (!matrix(gate, ldgate, d->dtype, d->d) || d->gate_tokens == 0)))
    return false;
  *a = NormArgs{};
  a->dtype = d->dtype;
  a->T = d->T;
  a->d = d->d;
  a->gate_tokens = gate != nullptr ? (int)std::min<int64_t>(d->gate_tokens, d->T) : 0;
  a->scale = d->scale;
  a->eps = d->eps;
  a->x = x;
  a->ldx = ldx;
  a->y = y;
  a->ldy = ldy;
  a->gate = gate;
  a->ldgate = ldgate;
  a->w_post = w_post;
  a->w_pre = w_pre;
  return true;
}

}  // namespace

extern "C" {

dmoe_status dmoe_sort_workspace_size(int64_t T, int32_t k, int32_t E, size_t* bytes) {
  if (bytes == nullptr) return DMOE_ERR_INVALID_ARG;
  const dmoe_status st = check_sort(T, k, E);
  if (st != DMOE_OK) return st;
  *bytes = sort_workspace_bytes(T * k, E);
  return DMOE_OK;
}

dmoe_status dmoe_sort_tokens(int64_t T, int32_t k, int32_t E, const int32_t* topk_idx,
                             int32_t* offsets, int32_t* rows, int32_t* pos, void* workspace,
                             size_t workspace_bytes, void* stream) {
  const dmoe_status st = check_sort(T, k, E);
  if (st != DMOE_OK) return st;
  if (!given16(offsets) || (T > 0 && !(given16(topk_idx) && given16(rows) && given16(pos))))
    return DMOE_ERR_INVALID_ARG;
  if (workspace == nullptr || !aligned(workspace, 256)) return DMOE_ERR_INVALID_ARG;
  const size_t need = sort_workspace_bytes(T * k, E);
  if (workspace_bytes < need) return DMOE_ERR_WORKSPACE;
  drop_parts_below(workspace, need);
  return status_of(launch_sort_tokens(T * k, E, topk_idx, offsets, rows, pos, workspace,
                                      static_cast<cudaStream_t>(stream)));
}

dmoe_status dmoe_gather_rows(int32_t dtype, int64_t T, int32_t k, int32_t d, const void* x,
                             int64_t ldx, const int32_t* pos, void* xs, int64_t ldxs,
                             void* stream) {
  const dmoe_status st = check_rows(dtype, T, k, d);
  if (st != DMOE_OK || T == 0) return st;
  if (!matrix(x, ldx, dtype, d) || !matrix(xs, ldxs, dtype, d) || !given16(pos) || x == xs)
    return DMOE_ERR_INVALID_ARG;
  RowsArgs a{};
  a.dtype = dtype;
  a.T = T;
  a.k = k;
  a.d = d;
  a.pos = pos;
  a.tok = x;
  a.ldtok = ldx;
  a.sorted_out = xs;
  a.ldsorted_out = ldxs;
  return status_of(launch_gather_rows(a, static_cast<cudaStream_t>(stream)));
}

dmoe_status dmoe_combine_rows(int32_t dtype, int64_t T, int32_t k, int32_t d, const void* ys,
                              int64_t ldys, const int32_t* pos, const float* gates,
                              const void* add, int64_t ldadd, void* y, int64_t ldy,
                              void* stream) {
  const dmoe_status st = check_rows(dtype, T, k, d);
  if (st != DMOE_OK || T == 0) return st;
  if (!matrix(ys, ldys, dtype, d) || !matrix(y, ldy, dtype, d) || !given16(pos) ||
      !null_or16(gates) || y == ys || (add != nullptr && !matrix(add, ldadd, dtype, d)) ||
      (add == y && ldadd != ldy))
    return DMOE_ERR_INVALID_ARG;
  RowsArgs a{};
  a.dtype = dtype;
  a.T = T;
  a.k = k;
  a.d = d;
  a.pos = pos;
  a.gates = gates;
  a.tok = add;
  a.ldtok = ldadd;
  a.sorted = ys;
  a.ldsorted = ldys;
  a.tok_out = y;
  a.ldtok_out = ldy;
  return status_of(launch_combine_rows(a, static_cast<cudaStream_t>(stream)));
}

dmoe_status dmoe_gather_rows_backward(int32_t dtype, int64_t T, int32_t k, int32_t d,
                                      const void* dxs, int64_t lddxs, const int32_t* pos,
                                      void* dx, int64_t lddx, void* stream) {
  return dmoe_combine_rows(dtype, T, k, d, dxs, lddxs, pos, nullptr, nullptr, 0, dx, lddx, stream);
}

dmoe_status dmoe_combine_rows_backward(int32_t dtype, int64_t T, int32_t k, int32_t d,
                                       const void* dy, int64_t lddy, const void* ys,
                                       int64_t ldys, const int32_t* pos, const float* gates,
                                       void* dys, int64_t lddys, float* dgates, void* stream) {
  const dmoe_status st = check_rows(dtype, T, k, d);
  if (st != DMOE_OK || T == 0) return st;
  if (!matrix(dy, lddy, dtype, d) || !given16(pos) || !null_or16(gates) || !null_or16(dgates) ||
      (dys == nullptr && dgates == nullptr) ||
      (dys != nullptr && !matrix(dys, lddys, dtype, d)) ||
      (dgates != nullptr && !matrix(ys, ldys, dtype, d)) ||
      (dys != nullptr && (dys == dy || dys == ys)) || (gates != nullptr && gates == dgates))
    return DMOE_ERR_INVALID_ARG;
  RowsArgs a{};
  a.dtype = dtype;
  a.T = T;
  a.k = k;
  a.d = d;
  a.pos = pos;
  a.gates = gates;
  a.tok = dy;
  a.ldtok = lddy;
  a.sorted = dgates != nullptr ? ys : nullptr;
  a.ldsorted = ldys;
  a.sorted_out = dys;
  a.ldsorted_out = lddys;
  a.dgates = dgates;
  return status_of(launch_combine_rows_backward(a, static_cast<cudaStream_t>(stream)));
}

dmoe_status dmoe_q4_size(const dmoe_q4_desc* desc, size_t* codes_bytes, size_t* scales_bytes) {
  if (codes_bytes == nullptr || scales_bytes == nullptr) return DMOE_ERR_INVALID_ARG;
  const dmoe_status st = check_q4(desc);
  if (st != DMOE_OK) return st;
  const Q4Shape s = q4_shape(*desc);
  *codes_bytes = s.code_bytes() * desc->n_experts;
  *scales_bytes = s.scale_bytes() * desc->n_experts;
  return DMOE_OK;
}

dmoe_status dmoe_q4_quantize(const dmoe_q4_desc* desc, const void* w, void* codes, void* scales,
                             void* stream) {
  const dmoe_status st = check_q4(desc);
  if (st != DMOE_OK) return st;
  if (!given16(w) || !given16(codes) || !given16(scales)) return DMOE_ERR_INVALID_ARG;
  return status_of(launch_q4_quantize(*desc, w, codes, scales, static_cast<cudaStream_t>(stream)));
}

dmoe_status dmoe_q4_dequantize(const dmoe_q4_desc* desc, const void* codes, const void* scales,
                               void* w, void* stream) {
  const dmoe_status st = check_q4(desc);
  if (st != DMOE_OK) return st;
  if (!given16(w) || !given16(codes) || !given16(scales)) return DMOE_ERR_INVALID_ARG;
  return status_of(launch_q4_dequantize(*desc, codes, scales, w,
                                        static_cast<cudaStream_t>(stream)));
}

dmoe_status dmoe_q4_linear(const dmoe_q4_desc* desc, int64_t R, int32_t n_groups, const void* x,
                           int64_t ldx, int64_t T_x, const int32_t* rows, int32_t k,
                           const int32_t* offsets, const int32_t* expert_ids,
                           const void* codes, const void* scales, void* y, int64_t ldy,
                           int32_t y_dtype, void* stream) {
  return run_q4(desc, R, n_groups, x, ldx, T_x, rows, k, offsets, expert_ids, {codes, scales}, y,
                ldy, y_dtype, stream);
}

dmoe_status dmoe_q4_swiglu(const dmoe_q4_desc* desc, int64_t R, int32_t n_groups, const void* x,
                           int64_t ldx, int64_t T_x, const int32_t* rows, int32_t k,
                           const int32_t* offsets, const int32_t* expert_ids,
                           const void* gate_codes, const void* gate_scales,
                           const void* up_codes, const void* up_scales, void* y, int64_t ldy,
                           int32_t y_dtype, void* stream) {
  return run_q4(desc, R, n_groups, x, ldx, T_x, rows, k, offsets, expert_ids,
                {gate_codes, gate_scales, up_codes, up_scales}, y, ldy, y_dtype, stream);
}

dmoe_status dmoe_q4_set_debug_hold(int32_t hold) {
  if (hold < 0) return DMOE_ERR_INVALID_ARG;
  g_q4_hold.store(hold);
  return DMOE_OK;
}

dmoe_status dmoe_q4_device_error(void* stream, int32_t* info) {
  void* record = nullptr;
  const cudaError_t e = q4_fault_address(&record);
  if (e != cudaSuccess) return status_of(e);
  const dmoe_status st = dmoe_get_device_error(record, stream, info);
  if (st == DMOE_ERR_TIMEOUT) g_q4_hold.store(0);
  return st;
}

dmoe_status dmoe_expert_ffn(const dmoe_expert_desc* desc, int64_t R, int32_t n_groups,
                            const void* x, int64_t ldx, const int32_t* offsets,
                            const int32_t* expert_ids, const void* w_gate, const void* w_up,
                            const void* w_down, void* pre, void* h, void* y, int64_t ldy,
                            int32_t zero_rest, void* stream) {
  const dmoe_status st = check_expert(desc, R, n_groups);
  if (st != DMOE_OK) return st;
  if ((offsets == nullptr && n_groups != 1) ||
      (expert_ids == nullptr && n_groups > desc->n_experts))
    return DMOE_ERR_INVALID_ARG;
  if (R == 0) return DMOE_OK;
  if (!matrix16(x, ldx, desc->d_model) || !matrix16(y, ldy, desc->d_model) || !given16(h) ||
      !null_or16(pre) || !given16(w_gate) || !given16(w_up) || !given16(w_down) ||
      !null_or16(offsets) || !null_or16(expert_ids) ||
      !apart({pre, h, y}, {x, offsets, expert_ids, w_gate, w_up, w_down}))
    return DMOE_ERR_INVALID_ARG;
  FfnArgs a = expert_args(desc, R, n_groups, offsets, w_gate, w_up, w_down);
  a.expert_ids = expert_ids;
  a.x = x;
  a.ldx = ldx;
  a.pre = pre;
  a.h = h;
  a.y = y;
  a.ldy = ldy;
  a.zero_rest = zero_rest != 0;
  return status_of(launch_expert_ffn(a, static_cast<cudaStream_t>(stream)));
}

dmoe_status dmoe_expert_ffn_backward(const dmoe_expert_desc* desc, int64_t R, const void* dy,
                                     int64_t lddy, const void* x, int64_t ldx,
                                     const int32_t* offsets, const void* w_gate, const void* w_up,
                                     const void* w_down, const void* pre, const void* h, void* dpre,
                                     void* dx, int64_t lddx, void* dw_gate, void* dw_up,
                                     void* dw_down, int32_t zero_rest, void* stream) {
  const int32_t n_groups = desc != nullptr ? desc->n_experts : 0;
  const dmoe_status st = check_expert(desc, R, n_groups);
  if (st != DMOE_OK) return st;
  const bool inner = dx != nullptr || dw_gate != nullptr;
  if ((offsets == nullptr && n_groups != 1) || (!inner && dw_down == nullptr) ||
      (dw_gate == nullptr) != (dw_up == nullptr) || !null_or16(dw_gate) || !null_or16(dw_up) ||
      !null_or16(dw_down) || !apart({dw_gate, dw_up, dw_down}, {}))
    return DMOE_ERR_INVALID_ARG;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (R == 0) {   // no rows: the weights' gradients are zeros
    const size_t bytes = (size_t)2 * desc->n_experts * desc->d_model * desc->d_ff;
    for (void* dw : {dw_gate, dw_up, dw_down})
      if (dw != nullptr) {
        const cudaError_t e = cudaMemsetAsync(dw, 0, bytes, s);
        if (e != cudaSuccess) return status_of(e);
      }
    return DMOE_OK;
  }
  if (!matrix16(dy, lddy, desc->d_model) || !null_or16(offsets) ||
      (inner && (!given16(w_down) || !given16(pre) || !given16(dpre) || dpre == h || dpre == x)) ||
      (dx != nullptr && (!matrix16(dx, lddx, desc->d_model) || !given16(w_gate) || !given16(w_up) || dx == x)) ||
      (dw_gate != nullptr && !matrix16(x, ldx, desc->d_model)) ||
      (dw_down != nullptr && !given16(h)))
    return DMOE_ERR_INVALID_ARG;
  // (what this call does not read may well be an output's place: h where dw_down is not wanted)
  auto where = [](bool read, const void* p) { return read ? p : nullptr; };
  if (!apart({inner ? dpre : nullptr, dx, dw_gate, dw_up, dw_down},
             {dy, offsets, where(dw_gate != nullptr, x), where(inner, w_down), where(inner, pre),
              where(dx != nullptr, w_gate), where(dx != nullptr, w_up), where(dw_down != nullptr, h)}))
    return DMOE_ERR_INVALID_ARG;
  FfnArgs a = expert_args(desc, R, n_groups, offsets, w_gate, w_up, w_down);
  a.dy = dy;
  a.lddy = lddy;
  a.x = x;
  a.ldx = ldx;
  a.pre = const_cast<void*>(pre);
  a.h = const_cast<void*>(h);
  a.dpre = dpre;
  a.dx = dx;
  a.lddx = lddx;
  a.dw_gate = dw_gate;
  a.dw_up = dw_up;
  a.dw_down = dw_down;
  a.zero_rest = zero_rest != 0;
  return status_of(launch_expert_ffn_backward(a, s));
}

dmoe_status dmoe_expert_device_error(void* stream, int32_t* info) {
  void* record = nullptr;
  const cudaError_t e = ffn_fault_address(&record);
  if (e != cudaSuccess) return status_of(e);
  const dmoe_status st = dmoe_get_device_error(record, stream, info);
  if (st == DMOE_ERR_TIMEOUT) g_expert_hold.store(0);
  return st;
}

dmoe_status dmoe_expert_set_debug_hold(int32_t hold) {
  if (hold < 0) return DMOE_ERR_INVALID_ARG;
  g_expert_hold.store(hold);
  return DMOE_OK;
}

dmoe_status dmoe_norm_residual(const dmoe_norm_desc* desc, const void* x, int64_t ldx, const void* y,
                               int64_t ldy, const float* w_post, const void* gate, int64_t ldgate,
                               const float* w_pre, void* r, int64_t ldr, void* n, int64_t ldn,
                               float* stats, void* stream) {
  const dmoe_status st = check_norm(desc);
  if (st != DMOE_OK || desc->T == 0) return st;
  const int dt = desc->dtype, d = desc->d;
  NormArgs a;
  if (!norm_inputs(desc, x, ldx, y, ldy, w_post, gate, ldgate, w_pre, &a) ||
      (w_pre == nullptr) != (n == nullptr) || (r == nullptr && n == nullptr) ||
      (r != nullptr && !matrix(r, ldr, dt, d)) || (n != nullptr && !matrix(n, ldn, dt, d)) ||
      !null_or16(stats) || !apart({r, n, stats}, {w_post, gate, w_pre}) || !apart({r, stats}, {y}) ||
      !apart({n, stats}, {x}) || (r == x && ldr != ldx) || (n != nullptr && n == y && ldn != ldy))
    return DMOE_ERR_INVALID_ARG;
  if (!strides_fit({ldx, y != nullptr ? ldy : 0, r != nullptr ? ldr : 0, n != nullptr ? ldn : 0}))
    return DMOE_ERR_UNSUPPORTED;
  a.r = r;
  a.ldr = ldr;
  a.n = n;
  a.ldn = ldn;
  a.stats = stats;
  return status_of(launch_norm_residual(a, static_cast<cudaStream_t>(stream)));
}

dmoe_status dmoe_norm_workspace_size(const dmoe_norm_desc* desc, size_t* bytes) {
  if (bytes == nullptr) return DMOE_ERR_INVALID_ARG;
  const dmoe_status st = check_norm(desc);
  if (st != DMOE_OK) return st;
  *bytes = norm_workspace_bytes(desc->T, desc->d, desc->gate_tokens > 0 ? 1 : 0);
  return DMOE_OK;
}

dmoe_status dmoe_norm_residual_backward(
    const dmoe_norm_desc* desc, const void* x, int64_t ldx, const void* y, int64_t ldy,
    const float* w_post, const void* gate, int64_t ldgate, const float* w_pre, const float* stats,
    const void* dr, int64_t lddr, const void* dn, int64_t lddn, void* dx, int64_t lddx, void* dy,
    int64_t lddy, void* dgate, int64_t lddgate, float* dw_post, float* dw_pre, void* workspace,
    size_t workspace_bytes, void* stream) {
  const dmoe_status st = check_norm(desc);
  if (st != DMOE_OK) return st;
  const int dt = desc->dtype, d = desc->d;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if ((dx == nullptr && dy == nullptr && dgate == nullptr && dw_post == nullptr && dw_pre == nullptr) ||
      !null_or16(dw_post) || !null_or16(dw_pre) || (dw_post != nullptr && dw_post == dw_pre))
    return DMOE_ERR_INVALID_ARG;
  if (desc->T == 0) {   // no tokens: the weights' gradients are zeros
    for (float* dw : {dw_post, dw_pre})
      if (dw != nullptr) {
        const cudaError_t e = cudaMemsetAsync(dw, 0, sizeof(float) * d, s);
        if (e != cudaSuccess) return status_of(e);
      }
    return DMOE_OK;
  }
  NormArgs a;
  if (!norm_inputs(desc, x, ldx, y, ldy, w_post, gate, ldgate, w_pre, &a) || !given16(stats) ||
      (dr == nullptr && dn == nullptr) || (dr != nullptr && !matrix(dr, lddr, dt, d)) ||
      (dn != nullptr && (!matrix(dn, lddn, dt, d) || w_pre == nullptr)) ||
      (dx != nullptr && !matrix(dx, lddx, dt, d)) ||
      (dy != nullptr && (!matrix(dy, lddy, dt, d) || y == nullptr)) ||
      (dgate != nullptr && (!matrix(dgate, lddgate, dt, d) || gate == nullptr)) ||
      (dw_post != nullptr && w_post == nullptr) || (dw_pre != nullptr && w_pre == nullptr))
    return DMOE_ERR_INVALID_ARG;
  if (!apart({dx, dy, dgate, dw_post, dw_pre}, {x, y, w_post, gate, w_pre, stats, dr, dn, workspace}))
    return DMOE_ERR_INVALID_ARG;
  // (a gate row of one token is complete where its token is)
  const bool gate_parts = dgate != nullptr && a.gate_tokens > 1;
  if (dw_post != nullptr || dw_pre != nullptr || gate_parts) {
    if (workspace == nullptr || !aligned(workspace, 16)) return DMOE_ERR_INVALID_ARG;
    if (workspace_bytes < norm_workspace_bytes(desc->T, d, gate_parts ? 1 : 0)) return DMOE_ERR_WORKSPACE;
  }
  if (!strides_fit({ldx, y != nullptr ? ldy : 0, dr != nullptr ? lddr : 0, dn != nullptr ? lddn : 0,
                    dx != nullptr ? lddx : 0, dy != nullptr ? lddy : 0}))
    return DMOE_ERR_UNSUPPORTED;
  a.stats = const_cast<float*>(stats);
  a.dr = dr;
  a.lddr = lddr;
  a.dn = dn;
  a.lddn = lddn;
  a.dx = dx;
  a.lddx = lddx;
  a.dy = dy;
  a.lddy = lddy;
  a.dgate = dgate;
  a.lddgate = lddgate;
  a.dw_post = dw_post;
  a.dw_pre = dw_pre;
  a.workspace = static_cast<float*>(workspace);
  return status_of(launch_norm_residual_backward(a, s));
}

}  // extern "C"

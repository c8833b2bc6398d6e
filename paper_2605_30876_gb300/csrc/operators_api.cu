// C-ABI entry points of the calls that do a layer by its parts: argument checks and launches.
// Nothing here allocates device memory or synchronises.
#include "dmoe_internal.cuh"
#include "q4.cuh"

using namespace dmoe;

namespace {

constexpr int64_t kMaxPairs = 1 << 30;
constexpr int kMaxRowWidth = 1 << 20;

std::atomic<int32_t> g_q4_hold{0};   // dmoe_q4_set_debug_hold

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

}  // extern "C"

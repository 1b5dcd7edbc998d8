// C-ABI entry points of the operators that a layer is adapted with (include/cascade_attn.h): layer norm, low-rank adapters, the optimizer's
// step.  Argument checks and launches; every failing call returns before touching the GPU.
#include <cmath>
#include <cstdint>

#include "ca_internal.hpp"

namespace {

bool aligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
bool eps_ok(float eps) { return eps >= 0.f && std::isfinite(eps); }
bool dtype_ok(int32_t t) { return t == CA_F32 || t == CA_BF16; }
uintptr_t size_of(int32_t dtype) { return dtype == CA_F32 ? 4 : 2; }

constexpr int64_t kMaxRows = int64_t(1) << 30, kMaxGroups = int64_t(1) << 20;

int32_t check_row_norm(const ca::RowNorm& n) {
  if (n.rows < 0 || n.groups < 1 || n.rows % n.groups != 0 || !eps_ok(n.eps) || !dtype_ok(n.dtype) || !dtype_ok(n.w_dtype)) return CA_EINVAL;
  if (n.dtype == CA_F32 && n.w_dtype != CA_F32) return CA_EINVAL;
  if (n.rows > kMaxRows || n.groups > kMaxGroups || n.width < 1 || n.width > CA_LAYER_NORM_MAX_WIDTH) return CA_EUNSUPPORTED;
  if (n.rows > 0 && (!n.x || !aligned(n.x, size_of(n.dtype)) || (n.rows > 1 && (n.ldx < n.width || n.ldy < n.width)))) return CA_EINVAL;
  if (!aligned(n.w, size_of(n.w_dtype)) || !aligned(n.b, size_of(n.w_dtype))) return CA_EINVAL;
  return (n.w || n.b) && n.groups > 1 && n.ldw < n.width ? CA_EINVAL : CA_OK;
}

constexpr int64_t kMaxAdaptedRows = int64_t(1) << 27, kMaxLd = int64_t(1) << 22;
constexpr int32_t kMaxColumns = 1 << 20;

int32_t check_ld(int64_t ld, int64_t cols) {
  if (ld < cols || ld % 8 != 0) return CA_EINVAL;
  return ld >= kMaxLd ? CA_EUNSUPPORTED : CA_OK;
}

int32_t check_adapted(int64_t m_rows, int32_t n_out, int32_t k_in, int32_t adapters, int32_t rank) {
  if (m_rows < 0 || adapters < 1) return CA_EINVAL;
  if (m_rows > kMaxAdaptedRows || n_out < 8 || n_out % 8 != 0 || n_out > kMaxColumns || k_in < 128 || k_in % 128 != 0 || k_in > kMaxColumns ||
      adapters > CA_MAX_ADAPTERS || (rank != 32 && rank != 64 && rank != 128))
    return CA_EUNSUPPORTED;
  return CA_OK;
}

// the products of the backward pass sum over the columns of Y too
int32_t check_adapted_backward(int64_t m_rows, int32_t n_out, int32_t k_in, int32_t adapters, int32_t rank) {
  if (int32_t rc = check_adapted(m_rows, n_out, k_in, adapters, rank)) return rc;
  const int64_t largest = int64_t(adapters) * rank * (n_out > k_in ? n_out : k_in);           // a launch may have 2^32 threads
  return n_out % 128 != 0 || largest > (int64_t(1) << 30) ? CA_EUNSUPPORTED : CA_OK;
}

// of the state's two buffers: codes and fp32 values are moved in pieces of up to 16 bytes
int32_t check_adamw(const ca_adamw_tensor& t, int32_t state_bits) {
  if (t.n < 0 || !dtype_ok(t.param_dtype) || !dtype_ok(t.grad_dtype)) return CA_EINVAL;
  if (t.n > CA_ADAMW_MAX_VALUES) return CA_EUNSUPPORTED;
  if (t.n == 0 || !t.grad) return CA_OK;
  if (!t.param || !t.m || !t.v || !t.step) return CA_EINVAL;
  if (!aligned(t.param, size_of(t.param_dtype)) || !aligned(t.grad, size_of(t.grad_dtype)) || !aligned(t.copy, 2) || !aligned(t.m, 16) || !aligned(t.v, 16) ||
      !aligned(t.step, 16))
    return CA_EINVAL;
  if (t.copy && t.param_dtype != CA_F32) return CA_EINVAL;
  return state_bits == 8 && (!t.m_scale || !t.v_scale || !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4)) ? CA_EINVAL : CA_OK;
}

}  // namespace

extern "C" {

int32_t layer_norm(const void* x_dev, int32_t dtype, const void* weight_dev, const void* bias_dev, int32_t weight_dtype, float eps, void* y_dev,
                   int64_t rows, int32_t width, int64_t groups, int64_t ldx, int64_t ldw, int64_t ldy, void* hip_stream) {
  const ca::RowNorm n{x_dev, weight_dev, bias_dev, rows, groups, ldx, ldy, ldw, width, dtype, weight_dtype, eps};
  if (int32_t rc = check_row_norm(n)) return rc;
  if (rows == 0) return CA_OK;
  if (!y_dev || !aligned(y_dev, size_of(dtype))) return CA_EINVAL;
  return ca::launch_layer_norm(n, y_dev, hip_stream);
}

size_t layer_norm_backward_workspace(int64_t rows, int32_t width, int64_t groups) {
  if (rows < 0 || groups < 1 || rows % groups != 0 || rows > kMaxRows || groups > kMaxGroups || width < 1 || width > CA_LAYER_NORM_MAX_WIDTH) return 0;
  return ca::layer_norm_backward_bytes(rows, width, groups);
}

int32_t layer_norm_backward(const void* dy_dev, const void* x_dev, int32_t dtype, const void* weight_dev, int32_t weight_dtype, float eps, void* dx_dev,
                            float* dweight_dev, float* dbias_dev, int64_t rows, int32_t width, int64_t groups, int64_t lddy, int64_t ldx, int64_t ldw,
                            int64_t lddx, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  const ca::RowNorm n{x_dev, weight_dev, nullptr, rows, groups, ldx, lddx, ldw, width, dtype, weight_dtype, eps};
  if (int32_t rc = check_row_norm(n)) return rc;
  if (!aligned(dweight_dev, 4) || !aligned(dbias_dev, 4)) return CA_EINVAL;
  if (rows > 0 && (!dy_dev || !dx_dev || !aligned(dy_dev, size_of(dtype)) || !aligned(dx_dev, size_of(dtype)) || (rows > 1 && lddy < width))) return CA_EINVAL;
  if (dweight_dev || dbias_dev) {
    const size_t need = ca::layer_norm_backward_bytes(rows, width, groups);
    if (need > 0 && (!workspace_dev || !aligned(workspace_dev, 16) || workspace_bytes < need)) return CA_EINVAL;
  }
  return ca::launch_layer_norm_backward(n, dy_dev, lddy, dx_dev, dweight_dev, dbias_dev, workspace_dev, hip_stream);
}

size_t layer_linear_adapted_workspace(int64_t m_rows, int32_t rank) {
  return m_rows < 0 || m_rows > kMaxAdaptedRows || (rank != 32 && rank != 64 && rank != 128) ? 0 : ca::adapted_bytes(m_rows, rank);
}

int32_t layer_linear_adapted_bf16(const void* x_dev, const void* w_dev, const void* down_dev, const void* up_dev, const float* scales_dev,
                                  const int32_t* index_dev, void* low_dev, void* y_dev, int64_t m_rows, int32_t n_out, int32_t k_in, int32_t adapters,
                                  int32_t rank, int64_t ldx, int64_t ldw, int64_t ldy, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  if (int32_t rc = check_adapted(m_rows, n_out, k_in, adapters, rank)) return rc;
  for (int64_t ld : {ldx, ldw})
    if (int32_t rc = check_ld(ld, k_in)) return rc;
  if (ldy < n_out || ldy % 8 != 0) return CA_EINVAL;
  if (m_rows == 0) return CA_OK;
  for (const void* p : {x_dev, w_dev, down_dev, up_dev, static_cast<const void*>(low_dev), static_cast<const void*>(y_dev)})
    if (!p || !aligned(p, 16)) return CA_EINVAL;
  if (!scales_dev || !index_dev || !aligned(scales_dev, 4) || !aligned(index_dev, 4)) return CA_EINVAL;
  const size_t need = ca::adapted_bytes(m_rows, rank);
  if (need > 0 && (!workspace_dev || !aligned(workspace_dev, 16) || workspace_bytes < need)) return CA_EINVAL;
  const ca::AdaptedLinear p{x_dev, w_dev, down_dev, up_dev, scales_dev, index_dev, m_rows, ldx, ldw, ldy, n_out, k_in, adapters, rank};
  return ca::launch_gemm_adapted(p, y_dev, low_dev, workspace_dev, hip_stream);
}

size_t layer_linear_adapted_backward_workspace(int64_t m_rows, int32_t n_out, int32_t k_in, int32_t adapters, int32_t rank) {
  return check_adapted_backward(m_rows, n_out, k_in, adapters, rank) ? 0 : ca::adapted_backward_bytes(m_rows, n_out, k_in, adapters, rank);
}

int32_t layer_linear_adapted_backward_bf16(const void* dy_dev, const void* x_dev, const void* w_t_dev, const void* down_dev, const void* up_dev,
                                           const float* scales_dev, const int32_t* index_dev, const void* low_dev, void* dx_dev, void* d_down_dev,
                                           void* d_up_dev, int64_t m_rows, int32_t n_out, int32_t k_in, int32_t adapters, int32_t rank, int32_t rank_used,
                                           int64_t lddy, int64_t ldx, int64_t ldw_t, int64_t lddx, void* workspace_dev, size_t workspace_bytes,
                                           void* hip_stream) {
  if (int32_t rc = check_adapted_backward(m_rows, n_out, k_in, adapters, rank)) return rc;
  if (rank_used < 1 || rank_used > rank || (!dx_dev && !d_down_dev && !d_up_dev)) return CA_EINVAL;
  if (int32_t rc = check_ld(lddy, n_out)) return rc;
  if (d_down_dev)
    if (int32_t rc = check_ld(ldx, k_in)) return rc;
  if (dx_dev) {
    if (int32_t rc = check_ld(ldw_t, n_out)) return rc;
    if (lddx < k_in || lddx % 8 != 0) return CA_EINVAL;
  }
  if (!workspace_dev || !aligned(workspace_dev, 16) || workspace_bytes < ca::adapted_backward_bytes(m_rows, n_out, k_in, adapters, rank)) return CA_EINVAL;
  if (!aligned(d_down_dev, 2) || !aligned(d_up_dev, 2) || !aligned(dx_dev, 16)) return CA_EINVAL;
  if (m_rows > 0) {
    for (const void* p : {dy_dev, up_dev, dx_dev ? w_t_dev : dy_dev, dx_dev ? down_dev : dy_dev, d_down_dev ? x_dev : dy_dev, d_up_dev ? low_dev : dy_dev})
      if (!p || !aligned(p, 16)) return CA_EINVAL;
    if (!scales_dev || !index_dev || !aligned(scales_dev, 4) || !aligned(index_dev, 4)) return CA_EINVAL;
  }
  const ca::AdaptedLinear p{x_dev, w_t_dev, down_dev, up_dev, scales_dev, index_dev, m_rows, ldx, ldw_t, lddx, n_out, k_in, adapters, rank};
  return ca::launch_adapted_backward(p, dy_dev, lddy, low_dev, rank_used, m_rows > 0 ? dx_dev : nullptr, d_down_dev, d_up_dev, workspace_dev, hip_stream);
}

int32_t layer_adamw(const ca_adamw_tensor* tensors, const ca_adamw_tensor* tensors_dev, int32_t n_tensors, int32_t state_bits, double lr, double beta1,
                    double beta2, double eps, double weight_decay, double grad_scale, void* hip_stream) {
  if (n_tensors < 0 || (n_tensors > 0 && (!tensors || !tensors_dev)) || !aligned(tensors_dev, 16) || (state_bits != 8 && state_bits != 32)) return CA_EINVAL;
  if (!(lr >= 0.) || !(weight_decay >= 0.) || !(beta1 >= 0. && beta1 < 1.) || !(beta2 >= 0. && beta2 < 1.) || !(float(eps) >= 0x1p-126f)) return CA_EINVAL;
  if (!std::isfinite(float(lr)) || !std::isfinite(lr * weight_decay) || !std::isfinite(float(eps)) || !std::isfinite(float(grad_scale))) return CA_EINVAL;
  for (int32_t i = 0; i < n_tensors; ++i)
    if (int32_t rc = check_adamw(tensors[i], state_bits)) return rc;
  return ca::launch_adamw(tensors, tensors_dev, n_tensors, state_bits, lr, beta1, beta2, eps, weight_decay, grad_scale, hip_stream);
}

int32_t layer_adamw_values(const void* m_codes_dev, const void* v_codes_dev, const float* m_scales_dev, const float* v_scales_dev, float* m_dev,
                           float* v_dev, int64_t n, void* hip_stream) {
  if (n < 0 || n % 256 != 0) return CA_EINVAL;
  if (n == 0) return CA_OK;
  for (const void* p : {m_codes_dev, v_codes_dev, static_cast<const void*>(m_dev), static_cast<const void*>(v_dev)})
    if (!p || !aligned(p, 16)) return CA_EINVAL;
  if (!m_scales_dev || !v_scales_dev || !aligned(m_scales_dev, 4) || !aligned(v_scales_dev, 4)) return CA_EINVAL;
  return ca::launch_adamw_values(m_codes_dev, v_codes_dev, m_scales_dev, v_scales_dev, m_dev, v_dev, n, hip_stream);
}

}  // extern "C"

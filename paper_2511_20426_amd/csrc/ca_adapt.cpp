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

}  // extern "C"

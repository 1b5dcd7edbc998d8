// C-ABI entry points of the operators around the attention of a layer (include/cascade_attn.h): argument checks and launches.
// Every failing call returns before touching metadata or the GPU.
#include <cmath>
#include <cstdint>

#include "ca_internal.hpp"

namespace {

using ca::rope_geom;
using ca::strides_ok;

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// frames are 32-bit numbers in the kernels
bool frames_fit(int64_t first_frame, int64_t n_tokens) { return first_frame <= INT32_MAX && n_tokens <= INT32_MAX - first_frame; }

bool eps_ok(float eps) { return eps >= 0.f && std::isfinite(eps); }

// queries or keys of a norm call: both of x and y or neither, the weight with them
int32_t norm_tensors(const ca_config& c, const ca_heads* x, const void* weight, const ca_heads* y, const ca_heads* dz, bool backward,
                     ca::NormTensors* out) {
  *out = ca::NormTensors{};
  if (!x) return y || dz ? CA_EINVAL : CA_OK;
  if (!y || !weight || (backward && !dz)) return CA_EINVAL;
  for (const ca_heads* t : {x, y, dz})
    if (t && (!t->dev || !strides_ok(c, t->dev, t->tok_stride, t->head_stride))) return CA_EINVAL;
  if (!aligned16(weight)) return CA_EINVAL;
  out->x = x->dev; out->x_tok = x->tok_stride; out->x_head = x->head_stride;
  out->y = y->dev; out->y_tok = y->tok_stride; out->y_head = y->head_stride;
  out->w = weight;
  if (dz) out->dz = dz->dev, out->dz_tok = dz->tok_stride, out->dz_head = dz->head_stride;
  return CA_OK;
}

constexpr int64_t kMaxRows = int64_t(1) << 30, kMaxLd = int64_t(1) << 22;

// a row stride of bf16 elements
int32_t check_ld(int64_t ld, int64_t cols) {
  if (ld < cols || ld % 8 != 0) return CA_EINVAL;
  return ld >= kMaxLd ? CA_EUNSUPPORTED : CA_OK;
}

int32_t check_gated(int32_t activation, int64_t m_rows, int32_t n_hidden, int32_t k_in) {
  if ((activation != CA_SILU && activation != CA_GELU) || m_rows < 0) return CA_EINVAL;
  if (m_rows > kMaxRows || n_hidden < 8 || n_hidden % 8 != 0 || k_in < 128 || k_in % 128 != 0) return CA_EUNSUPPORTED;
  return CA_OK;
}

// rows and twice the columns, in whole steps, are row strides of the backward pass's products
int32_t check_gated_backward(int64_t m_rows, int32_t n_hidden, int32_t k_in) {
  if (int32_t rc = check_gated(CA_SILU, m_rows, n_hidden, k_in)) return rc;
  return m_rows > kMaxLd - 256 || n_hidden > kMaxLd / 2 - 64 || k_in >= kMaxLd ? CA_EUNSUPPORTED : CA_OK;
}

}  // namespace

extern "C" {

int32_t layer_qk_norm_rope(const ca_ctx* ctx, const ca_heads* q, const ca_heads* k, const void* q_weight_dev, const void* k_weight_dev,
                           float eps, const ca_heads* q_out, const ca_heads* k_out, int64_t n_tokens, int64_t first_frame, void* hip_stream) {
  if (!ctx || n_tokens < 0 || first_frame < 0 || !eps_ok(eps) || (!q && !k)) return CA_EINVAL;
  if (!ctx->pool) return CA_ENOPOOL;
  if (!frames_fit(first_frame, n_tokens)) return CA_EUNSUPPORTED;
  if (n_tokens == 0) return CA_OK;
  const ca::CacheMeta& m = ctx->meta;
  ca::NormTensors tq, tk;
  if (int32_t rc = norm_tensors(m.cfg(), q, q_weight_dev, q_out, nullptr, false, &tq)) return rc;
  if (int32_t rc = norm_tensors(m.cfg(), k, k_weight_dev, k_out, nullptr, false, &tk)) return rc;
  return ca::launch_norm_rope(rope_geom(m), m.cfg().dtype, tq, tk, eps, n_tokens, first_frame, hip_stream);
}

size_t layer_qk_norm_rope_workspace(const ca_ctx* ctx) { return ctx ? ca::norm_rope_backward_bytes(ctx->meta.cfg().head_dim) : 0; }

int32_t layer_qk_norm_rope_backward(const ca_ctx* ctx, const ca_heads* dq_out, const ca_heads* dk_out, const ca_heads* q, const ca_heads* k,
                                    const void* q_weight_dev, const void* k_weight_dev, float eps, const ca_heads* dq, const ca_heads* dk,
                                    float* dq_weight_dev, float* dk_weight_dev, int64_t n_tokens, int64_t first_frame, void* workspace_dev,
                                    size_t workspace_bytes, void* hip_stream) {
  if (!ctx || n_tokens < 0 || first_frame < 0 || !eps_ok(eps) || (!q && !k)) return CA_EINVAL;
  if ((q && !dq_weight_dev) || (k && !dk_weight_dev) || !workspace_dev || !aligned16(workspace_dev)) return CA_EINVAL;
  if (!ctx->pool) return CA_ENOPOOL;
  if (!frames_fit(first_frame, n_tokens)) return CA_EUNSUPPORTED;
  const ca::CacheMeta& m = ctx->meta;
  if (workspace_bytes < ca::norm_rope_backward_bytes(m.cfg().head_dim)) return CA_EINVAL;
  ca::NormTensors tq{}, tk{};
  if (n_tokens > 0) {
    if (int32_t rc = norm_tensors(m.cfg(), q, q_weight_dev, dq, dq_out, true, &tq)) return rc;
    if (int32_t rc = norm_tensors(m.cfg(), k, k_weight_dev, dk, dk_out, true, &tk)) return rc;
  } else {                                        // of no tokens the weights' gradients are zero
    if (q) tq.x = dq_weight_dev;
    if (k) tk.x = dk_weight_dev;
  }
  return ca::launch_norm_rope_backward(rope_geom(m), m.cfg().dtype, tq, tk, eps, n_tokens, first_frame, dq_weight_dev, dk_weight_dev,
                                       workspace_dev, hip_stream);
}

int32_t kv_cache_append_batch_norm(ca_ctx* ctx, int32_t n_blocks, const int64_t* block_ids, const int32_t* timesteps, int32_t prompt_epoch,
                                   const void* const* k_dev, const void* const* v_dev, int64_t tok_stride, int64_t head_stride,
                                   const void* k_weight_dev, float eps, void* hip_stream, int32_t* slots_out) {
  if (!ctx || !block_ids || !timesteps || n_blocks < 1 || n_blocks > ca::kMaxInflight || !eps_ok(eps)) return CA_EINVAL;
  if (!ctx->pool) return CA_ENOPOOL;
  if (!k_dev || !v_dev || !k_weight_dev || !aligned16(k_weight_dev)) return CA_EINVAL;
  // as kv_cache_append_batch: the entries take effect in order on a copy, all or none
  ca::CacheMeta next = ctx->meta;
  const ca_config& c = next.cfg();
  int32_t slots[ca::kMaxInflight];
  int64_t first_frame[ca::kMaxInflight];
  for (int i = 0; i < n_blocks; ++i) {
    if (int32_t rc = next.check_append(block_ids[i], &slots[i])) return rc;
    for (int j = 0; j < i; ++j)
      if (block_ids[j] == block_ids[i]) return CA_EINVAL;
    if (block_ids[i] > INT32_MAX / c.frames_per_block - 1) return CA_EUNSUPPORTED;
    next.commit_append(slots[i], block_ids[i], timesteps[i], prompt_epoch);
    first_frame[i] = int64_t(c.frames_per_block) * block_ids[i];
    if (!k_dev[i] || !v_dev[i] || !strides_ok(c, k_dev[i], tok_stride, head_stride) || !strides_ok(c, v_dev[i], tok_stride, head_stride))
      return CA_EINVAL;
  }
  const int32_t rc = ca::launch_cache_write_norm(rope_geom(next), c.dtype, n_blocks, k_dev, v_dev, tok_stride, head_stride, first_frame,
                                                 next.block_tokens(), c.page_tokens, next.pages_per_block(), slots, k_weight_dev, eps,
                                                 ctx->pool, hip_stream);
  if (rc != CA_OK) return rc;
  ctx->meta = next;
  if (slots_out)
    for (int i = 0; i < n_blocks; ++i) slots_out[i] = slots[i];
  return CA_OK;
}

int32_t layer_quantize_rows_i8(const void* x_dev, int32_t dtype, int8_t* codes_dev, float* scales_dev, int64_t rows, int32_t k_in, int64_t ldx,
                               int64_t ld_codes, void* hip_stream) {
  if (rows < 0 || (dtype != CA_F32 && dtype != CA_BF16)) return CA_EINVAL;
  if (rows > kMaxRows || k_in < 1 || k_in > CA_I8_MAX_K) return CA_EUNSUPPORTED;
  if (ldx < k_in || ld_codes < (k_in + 255) / 256 * 256 || ld_codes % 16 != 0) return CA_EINVAL;
  if (rows == 0) return CA_OK;
  if (!x_dev || !codes_dev || !scales_dev || !aligned16(codes_dev) || reinterpret_cast<uintptr_t>(scales_dev) % 4 != 0 ||
      reinterpret_cast<uintptr_t>(x_dev) % (dtype == CA_BF16 ? 2 : 4) != 0)
    return CA_EINVAL;
  return ca::launch_quantize_rows(dtype, x_dev, codes_dev, scales_dev, rows, k_in, ldx, ld_codes, hip_stream);
}

int32_t layer_linear_i8(const int8_t* x_codes_dev, const float* x_scales_dev, const int8_t* w_codes_dev, const float* w_scales_dev, void* y_dev,
                        int64_t m_rows, int32_t n_out, int32_t k_in, int64_t ldx, int64_t ldw, int64_t ldy, void* hip_stream) {
  if (m_rows < 0) return CA_EINVAL;
  if (m_rows > kMaxRows || n_out < 8 || n_out % 8 != 0 || k_in < 1 || k_in > CA_I8_MAX_K) return CA_EUNSUPPORTED;
  const int64_t k = (k_in + 255) / 256 * 256;
  if (ldx < k || ldw < k || ldy < n_out || ldx % 16 != 0 || ldw % 16 != 0 || ldy % 8 != 0) return CA_EINVAL;
  if (ldx >= 2 * kMaxLd || ldw >= 2 * kMaxLd) return CA_EUNSUPPORTED;
  if (m_rows == 0) return CA_OK;
  if (!x_codes_dev || !x_scales_dev || !w_codes_dev || !w_scales_dev || !y_dev) return CA_EINVAL;
  if (!aligned16(x_codes_dev) || !aligned16(w_codes_dev) || !aligned16(y_dev) || !aligned16(w_scales_dev) ||
      reinterpret_cast<uintptr_t>(x_scales_dev) % 4 != 0)
    return CA_EINVAL;
  return ca::launch_gemm_i8(x_codes_dev, x_scales_dev, w_codes_dev, w_scales_dev, y_dev, m_rows, n_out, k_in, ldx, ldw, ldy, hip_stream);
}

size_t layer_linear_i8_workspace(int64_t m_rows, int32_t k_in) {
  if (m_rows < 0 || m_rows > kMaxRows || k_in < 1 || k_in > CA_I8_MAX_K) return 0;
  return size_t(m_rows) * ((size_t(k_in) + 255) / 256 * 256 + 4) + 16;
}

int32_t layer_linear_i8_values(const void* x_dev, int32_t dtype, const int8_t* w_codes_dev, const float* w_scales_dev, void* y_dev, int64_t m_rows,
                               int32_t n_out, int32_t k_in, int64_t ldx, int64_t ldw, int64_t ldy, void* workspace_dev, size_t workspace_bytes,
                               void* hip_stream) {
  if (m_rows < 0 || (dtype != CA_F32 && dtype != CA_BF16)) return CA_EINVAL;
  if (m_rows > kMaxRows || n_out < 8 || n_out % 8 != 0 || k_in < 1 || k_in > CA_I8_MAX_K) return CA_EUNSUPPORTED;
  if (ldx < k_in || ldw < (k_in + 255) / 256 * 256 || ldy < n_out || ldw % 16 != 0 || ldy % 8 != 0) return CA_EINVAL;
  if (ldx >= kMaxLd || ldw >= 2 * kMaxLd) return CA_EUNSUPPORTED;
  if (!workspace_dev || !aligned16(workspace_dev) || workspace_bytes < layer_linear_i8_workspace(m_rows, k_in)) return CA_EINVAL;
  if (m_rows == 0) return CA_OK;
  if (!x_dev || !w_codes_dev || !w_scales_dev || !y_dev) return CA_EINVAL;
  if (!aligned16(w_codes_dev) || !aligned16(y_dev) || !aligned16(w_scales_dev) || reinterpret_cast<uintptr_t>(x_dev) % (dtype == CA_BF16 ? 2 : 4) != 0)
    return CA_EINVAL;
  return ca::launch_gemm_i8_values(dtype, x_dev, ldx, w_codes_dev, w_scales_dev, y_dev, m_rows, n_out, k_in, ldw, ldy, workspace_dev, hip_stream);
}

int32_t layer_gated_bf16(const void* x_dev, const void* w_gate_dev, const void* w_up_dev, void* h_dev, float* saved_dev,
                         int32_t activation, int64_t m_rows, int32_t n_hidden, int32_t k_in, int64_t ldx, int64_t ldw_gate, int64_t ldw_up,
                         int64_t ldh, void* hip_stream) {
  if (int32_t rc = check_gated(activation, m_rows, n_hidden, k_in)) return rc;
  for (int64_t ld : {ldx, ldw_gate, ldw_up})
    if (int32_t rc = check_ld(ld, k_in)) return rc;
  if (ldh < n_hidden || ldh % 8 != 0) return CA_EINVAL;
  if (m_rows == 0) return CA_OK;
  for (const void* p : {x_dev, w_gate_dev, w_up_dev, static_cast<const void*>(h_dev)})
    if (!p || !aligned16(p)) return CA_EINVAL;
  if (!aligned16(saved_dev)) return CA_EINVAL;
  return ca::launch_gemm_gated(x_dev, w_gate_dev, w_up_dev, h_dev, saved_dev, activation, m_rows, n_hidden, k_in, ldx, ldw_gate, ldw_up,
                               ldh, hip_stream);
}

size_t layer_gated_saved_bytes(int64_t m_rows, int32_t n_hidden) {
  return check_gated(CA_SILU, m_rows, n_hidden, 128) ? 0 : size_t(ca::gated_saved_values(m_rows, n_hidden)) * sizeof(float);
}

size_t layer_gated_backward_workspace(int64_t m_rows, int32_t n_hidden, int32_t k_in) {
  return check_gated_backward(m_rows, n_hidden, k_in) ? 0 : ca::gated_workspace(m_rows, n_hidden, k_in).bytes;
}

int32_t layer_gated_backward_bf16(const void* dh_dev, const void* x_dev, const void* w_gate_dev, const void* w_up_dev, const float* saved_dev,
                                  int32_t activation, void* dx_dev, void* dw_gate_dev, void* dw_up_dev, int64_t m_rows,
                                  int32_t n_hidden, int32_t k_in, int64_t lddh, int64_t ldx, int64_t ldw_gate, int64_t ldw_up,
                                  int64_t lddx, int64_t lddw, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  if (int32_t rc = check_gated(activation, m_rows, n_hidden, k_in)) return rc;
  for (int64_t ld : {ldx, ldw_gate, ldw_up, lddx, lddw})
    if (int32_t rc = check_ld(ld, k_in)) return rc;
  if (int32_t rc = check_ld(lddh, n_hidden)) return rc;
  if (int32_t rc = check_gated_backward(m_rows, n_hidden, k_in)) return rc;
  if (!workspace_dev || !aligned16(workspace_dev) || workspace_bytes < ca::gated_workspace(m_rows, n_hidden, k_in).bytes) return CA_EINVAL;
  if (m_rows > 0)
    for (const void* p : {dh_dev, x_dev, static_cast<const void*>(saved_dev)})
      if (!p) return CA_EINVAL;
  if (!w_gate_dev || !w_up_dev || (!dx_dev && !dw_gate_dev && !dw_up_dev)) return CA_EINVAL;
  for (const void* p : {dh_dev, x_dev, w_gate_dev, w_up_dev, static_cast<const void*>(saved_dev), static_cast<const void*>(dx_dev), static_cast<const void*>(dw_gate_dev),
                        static_cast<const void*>(dw_up_dev)})
    if (!aligned16(p)) return CA_EINVAL;
  return ca::launch_gated_backward(dh_dev, x_dev, w_gate_dev, w_up_dev, saved_dev, activation, m_rows > 0 ? dx_dev : nullptr, dw_gate_dev,
                                   dw_up_dev, m_rows, n_hidden, k_in, lddh, ldx, ldw_gate, ldw_up, lddx, lddw, workspace_dev, hip_stream);
}

}  // extern "C"

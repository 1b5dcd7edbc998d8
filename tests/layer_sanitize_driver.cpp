// Drives the argument checks of the operators around the attention (ca_layer.cpp) under AddressSanitizer and UBSan; the kernel
// launchers are replaced by the stubs below, which only check what they are handed.
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include <limits>
#include <vector>

#include "ca_internal.hpp"

static int launches = 0;
#define REQUIRE(x)                                                        \
  do {                                                                    \
    if (!(x)) {                                                           \
      std::fprintf(stderr, "%s:%d: %s\n", __FILE__, __LINE__, #x);        \
      std::exit(1);                                                       \
    }                                                                     \
  } while (0)

namespace ca {
int32_t launch_norm_rope(const RopeGeom& g, int, const NormTensors& q, const NormTensors& k, float, int64_t n, int64_t first, void*) {
  REQUIRE(g.heads == 2 && n > 0 && first >= 0 && (q.x || k.x));
  for (const NormTensors* t : {&q, &k}) REQUIRE((t->x == nullptr) == (t->y == nullptr) && (t->x == nullptr) == (t->w == nullptr));
  ++launches;
  return CA_OK;
}
size_t norm_rope_backward_bytes(int32_t head_dim) { return size_t(head_dim) * 8; }
int32_t launch_norm_rope_backward(const RopeGeom&, int, const NormTensors& q, const NormTensors& k, float, int64_t n, int64_t, float* dqw, float* dkw,
                                  void* workspace, void*) {
  REQUIRE(workspace && (q.x || k.x) && (!q.x || dqw) && (!k.x || dkw) && (n == 0 || !q.x || (q.dz && q.y)));
  ++launches;
  return CA_OK;
}
int32_t launch_cache_write_norm(const RopeGeom&, int, int32_t n_blocks, const void* const* k, const void* const* v, int64_t, int64_t, const int64_t* first,
                                int32_t, int32_t, int32_t, const int32_t* slot, const void* w, float, void* pool, void*) {
  for (int i = 0; i < n_blocks; ++i) REQUIRE(k[i] && v[i] && first[i] >= 0 && slot[i] >= 0);
  REQUIRE(w && pool);
  ++launches;
  return CA_OK;
}
int32_t launch_quantize_rows(int, const void* x, void* codes, float* scales, int64_t rows, int32_t k, int64_t ldx, int64_t ld_codes, void*) {
  REQUIRE(x && codes && scales && rows > 0 && k > 0 && ldx >= k && ld_codes >= (k + 255) / 256 * 256);
  ++launches;
  return CA_OK;
}
int32_t launch_gemm_i8(const void* x, const float* xs, const void* w, const float* ws, void* y, int64_t M, int32_t, int32_t K, int64_t ldx, int64_t ldw,
                       int64_t, void*) {
  REQUIRE(x && xs && w && ws && y && M > 0 && ldx >= K && ldw >= K);
  ++launches;
  return CA_OK;
}
int32_t launch_gemm_i8_values(int, const void* x, int64_t, const void* w, const float* ws, void* y, int64_t M, int32_t, int32_t, int64_t, int64_t,
                              void* workspace, void*) {
  REQUIRE(x && w && ws && y && workspace && M > 0);
  ++launches;
  return CA_OK;
}
int32_t launch_gemm_gated(const void* x, const void* wg, const void* wu, void* h, float*, int, int64_t M, int32_t, int32_t, int64_t, int64_t, int64_t,
                          int64_t, void*) {
  REQUIRE(x && wg && wu && h && M > 0);
  ++launches;
  return CA_OK;
}
GatedWorkspace gated_workspace(int64_t M, int32_t F, int32_t K) {
  GatedWorkspace w{};
  w.Mp = (M + 127) / 128 * 128;
  w.Fp = (int64_t(F) + 63) / 64 * 64;
  w.bytes = size_t(w.Mp) * size_t(w.Fp) + size_t(K);
  return w;
}
int32_t launch_gated_backward(const void* dh, const void* x, const void*, const void*, const float* saved, int, void* dx, void* dwg, void* dwu, int64_t M,
                              int32_t, int32_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, void* workspace, void*) {
  REQUIRE(workspace && (M == 0 || (dh && x && saved)) && (dx || dwg || dwu));
  ++launches;
  return CA_OK;
}
int32_t launch_rope_apply(const RopeGeom&, int, const void*, void*, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, void*) { return CA_OK; }
int32_t launch_cache_write(const RopeGeom&, int, int32_t, const void* const*, const void* const*, int64_t, int64_t, const int64_t*, int32_t, int32_t,
                           int32_t, const int32_t*, void*, void*) { return CA_OK; }
int32_t launch_attn_f32(const AttnPlan&, const void*, void*, const void*, void*) { return CA_OK; }
int32_t launch_attn_bf16(const AttnPlan&, int, const void*, void*, const void*, void*, int, void*) { return CA_OK; }
int32_t launch_attn_bf16_rope(const AttnPlan&, const QRopePlan&, int, const void*, void*, const void*, void*, int, void*) { return CA_OK; }
int32_t launch_attn_bf16_static(const AttnPlan&, int, const void*, void*, const void*, void*) { return CA_OK; }
int32_t attn_bf16_variant_ok(int) { return CA_OK; }
void attn_static_scratch_prepare() {}
int32_t run_mfma_microbench(int, int, void*, size_t, void*, double*, double*) { return CA_OK; }
int32_t launch_gemm_bf16(const void*, const void*, void*, int64_t, int32_t, int32_t, int64_t, int64_t, int64_t, void*) { return CA_OK; }
int32_t launch_gemm_qkv_publish(const RopeGeom&, int32_t, int32_t, int32_t, const int32_t*, const int64_t*, const void*, int64_t, const void*, int64_t,
                                int32_t, void*, void*, void*) { return CA_OK; }
const char* last_device_error() { return ""; }
}  // namespace ca

int main() {
  ca_config c{2, 128, 3, 4, 5, 44, 42, 42, 10000.0, 0, 2, 2, 128, CA_BF16};
  ca_ctx* ctx = nullptr;
  void* const pool = reinterpret_cast<void*>(uintptr_t(1) << 40);          // never dereferenced by the stubs
  REQUIRE(ca_create(&c, pool, ca_pool_bytes(&c), &ctx) == CA_OK);
  void* const p = reinterpret_cast<void*>(uintptr_t(4096));
  float* const f = static_cast<float*>(p);
  int8_t* const i8 = static_cast<int8_t*>(p);
  const int64_t odd[] = {std::numeric_limits<int64_t>::min(), -1, 0, 1, 7, 8, 128, 255, 256, 1 << 22, int64_t(1) << 31, int64_t(1) << 40,
                         std::numeric_limits<int64_t>::max()};
  const int32_t odd32[] = {std::numeric_limits<int32_t>::min(), -1, 0, 1, 8, 100, 128, 256, 1 << 17, (1 << 17) + 1, std::numeric_limits<int32_t>::max()};
  const ca_heads t{p, 256, 128};
  const size_t work = layer_qk_norm_rope_workspace(ctx);
  REQUIRE(layer_qk_norm_rope_workspace(nullptr) == 0);
  REQUIRE(layer_qk_norm_rope(nullptr, &t, &t, p, p, 1e-6f, &t, &t, 4, 0, nullptr) == CA_EINVAL);
  for (int64_t a : odd)
    for (int64_t b : odd) {
      const ca_heads s{p, a, b};
      layer_qk_norm_rope(ctx, &s, &t, p, p, 1e-6f, &t, &s, 4, 0, nullptr);
      layer_qk_norm_rope(ctx, &t, nullptr, p, nullptr, 1e-6f, &t, nullptr, a, b, nullptr);
      layer_qk_norm_rope_backward(ctx, &t, &s, &t, &t, p, p, 1e-6f, &t, &t, f, f, a, b, p, work, nullptr);
      const int64_t id = a;
      const int32_t step = 0;
      const void* const k = p;
      kv_cache_append_batch_norm(ctx, 1, &id, &step, 0, &k, &k, a, b, p, 1e-6f, nullptr, nullptr);
      for (int32_t n : odd32)
        for (int32_t m : odd32) {
          layer_quantize_rows_i8(p, CA_BF16, i8, f, a, n, b, b, nullptr);
          layer_linear_i8(i8, f, i8, f, p, a, n, m, b, b, b, nullptr);
          layer_linear_i8_values(p, CA_F32, i8, f, p, a, n, m, b, b, b, p, layer_linear_i8_workspace(a, m), nullptr);
          layer_gated_bf16(p, p, p, p, f, CA_GELU, a, n, m, b, b, b, b, nullptr);
          layer_gated_saved_bytes(a, n);
          layer_gated_backward_bf16(p, p, p, p, f, CA_SILU, p, p, p, a, n, m, b, b, b, b, b, b, p, layer_gated_backward_workspace(a, n, m), nullptr);
        }
    }
  REQUIRE(layer_quantize_rows_i8(p, CA_BF16, i8, f, 3, 300, 300, 512, nullptr) == CA_OK);
  REQUIRE(layer_linear_i8(i8, f, i8, f, p, 3, 16, 300, 512, 512, 16, nullptr) == CA_OK);
  REQUIRE(layer_gated_bf16(p, p, p, p, nullptr, CA_SILU, 3, 16, 128, 128, 128, 128, 16, nullptr) == CA_OK);
  REQUIRE(launches > 3);
  ca_destroy(ctx);
  std::printf("layer sanitizer driver: ok\n");
  return 0;
}

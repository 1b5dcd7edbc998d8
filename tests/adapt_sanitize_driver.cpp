// Drives the argument checks of the operators that a layer is adapted with (ca_adapt.cpp) under AddressSanitizer and UBSan; the kernel launchers are
// replaced by the stubs below, which only check what they are handed.
#include <cstdio>
#include <cstdlib>
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
int32_t launch_layer_norm(const RowNorm& n, const void* y, void*) {
  REQUIRE(n.x && y && n.rows > 0 && n.groups > 0 && n.rows % n.groups == 0 && n.width > 0 && n.width <= CA_LAYER_NORM_MAX_WIDTH);
  REQUIRE(n.rows == 1 || (n.ldx >= n.width && n.ldy >= n.width));
  REQUIRE(n.groups == 1 || (!n.w && !n.b) || n.ldw >= n.width);
  ++launches;
  return CA_OK;
}
size_t layer_norm_backward_bytes(int64_t rows, int32_t width, int64_t groups) { return rows / groups > 64 ? size_t(groups) * 16 * size_t(width) : 0; }
int32_t launch_layer_norm_backward(const RowNorm& n, const void* dy, int64_t lddy, void* dx, float* dw, float* db, void* workspace, void*) {
  REQUIRE(n.rows == 0 || (n.x && dy && dx && (n.rows == 1 || lddy >= n.width)));
  REQUIRE((!dw && !db) || layer_norm_backward_bytes(n.rows, n.width, n.groups) == 0 || workspace);
  ++launches;
  return CA_OK;
}
size_t adapted_bytes(int64_t M, int32_t rank) { return M <= 32 ? size_t(M) * size_t(rank) : 0; }
int32_t launch_gemm_adapted(const AdaptedLinear& p, void* y, void* low, void* workspace, void*) {
  REQUIRE(p.x && p.w && p.down && p.up && p.scales && p.index && y && low && p.M > 0 && p.N % 8 == 0 && p.K % 128 == 0 && p.ldx >= p.K && p.ldw >= p.K && p.ldy >= p.N);
  REQUIRE((p.rank == 32 || p.rank == 64 || p.rank == 128) && p.adapters > 0 && p.adapters <= CA_MAX_ADAPTERS && (p.M > 32 || workspace));
  ++launches;
  return CA_OK;
}
size_t adapted_backward_bytes(int64_t M, int32_t N, int32_t K, int32_t adapters, int32_t rank) {
  return size_t(M) * size_t(rank) + (size_t(N) + size_t(K)) * size_t(adapters) * size_t(rank);
}
int32_t launch_adapted_backward(const AdaptedLinear& p, const void* dy, int64_t lddy, const void* low, int32_t used, void* dx, void* d_down, void* d_up,
                                void* workspace, void*) {
  REQUIRE(workspace && used > 0 && used <= p.rank && (p.M == 0 || (dy && lddy >= p.N && p.index && p.scales && p.up)));
  REQUIRE(p.M == 0 || ((!dx || (p.w && p.down && p.ldy >= p.K)) && (!d_down || p.x) && (!d_up || low)));
  ++launches;
  return CA_OK;
}
int32_t launch_adamw(const ca_adamw_tensor* tensors, const ca_adamw_tensor* table, int32_t n, int32_t bits, double lr, double b1, double b2, double eps, double wd,
                     double, void*) {
  REQUIRE(n == 0 || (tensors && table));
  REQUIRE((bits == 8 || bits == 32) && lr >= 0 && wd >= 0 && b1 >= 0 && b1 < 1 && b2 >= 0 && b2 < 1 && eps > 0);
  for (int32_t i = 0; i < n; ++i)
    REQUIRE(tensors[i].n >= 0 && (tensors[i].n == 0 || !tensors[i].grad || (tensors[i].param && tensors[i].m && tensors[i].v && tensors[i].step)));
  ++launches;
  return CA_OK;
}
int32_t launch_adamw_values(const void* m, const void* v, const float* ms, const float* vs, float* mo, float* vo, int64_t n, void*) {
  REQUIRE(m && v && ms && vs && mo && vo && n > 0 && n % 256 == 0);
  ++launches;
  return CA_OK;
}
}  // namespace ca

int main() {
  void* const p = reinterpret_cast<void*>(uintptr_t(4096));                // never dereferenced by the stubs
  float* const f = static_cast<float*>(p);
  int32_t* const i32 = static_cast<int32_t*>(p);
  const int64_t odd[] = {std::numeric_limits<int64_t>::min(), -1, 0, 1, 7, 8, 128, 256, 1 << 22, int64_t(1) << 31, int64_t(1) << 40,
                         std::numeric_limits<int64_t>::max()};
  const int32_t odd32[] = {std::numeric_limits<int32_t>::min(), -1, 0, 1, 8, 32, 128, 256, 4096, 1 << 20, std::numeric_limits<int32_t>::max()};
  for (int64_t a : odd)
    for (int64_t b : odd) {
      layer_adamw_values(p, p, f, f, f, f, a, nullptr);
      for (int32_t n : odd32) {
        layer_norm(p, n & 1, p, p, CA_F32, 1e-6f, p, a, n, b, a, b, a, nullptr);
        layer_norm(p, CA_BF16, p, p, CA_BF16, 1e-6f, p, a, n, 1, b, b, b, nullptr);
        layer_norm_backward(p, p, CA_BF16, p, CA_F32, 1e-6f, p, f, f, a, n, b, a, b, a, b, p, layer_norm_backward_workspace(a, n, b), nullptr);
        ca_adamw_tensor t{p, p, nullptr, p, p, f, f, i32, a, n & 1, CA_F32};
        layer_adamw(&t, &t, n > 1 ? 1 : n, n & 8 ? 8 : 32, double(b), 0.9, 0.99, 1e-8, double(a), 1.0, nullptr);
        for (int32_t m : odd32) {
          layer_linear_adapted_bf16(p, p, p, p, f, i32, p, p, a, n, m, 3, 32, b, b, b, p, layer_linear_adapted_workspace(a, 32), nullptr);
          layer_linear_adapted_bf16(p, p, p, p, f, i32, p, p, 40, 256, 128, n, m, b, a, b, nullptr, 0, nullptr);
          layer_linear_adapted_backward_bf16(p, p, p, p, p, f, i32, p, p, p, p, a, n, m, 3, 64, 5, b, b, b, b, p,
                                             layer_linear_adapted_backward_workspace(a, n, m, 3, 64), nullptr);
          layer_linear_adapted_backward_bf16(p, p, p, p, p, f, i32, p, p, p, p, 40, 256, 128, n, 64, m, 256, b, 256, b, p,
                                             layer_linear_adapted_backward_workspace(40, 256, 128, n, 64), nullptr);
        }
      }
    }
  REQUIRE(layer_norm(p, CA_BF16, p, nullptr, CA_F32, 1e-6f, p, 6, 64, 3, 64, 64, 64, nullptr) == CA_OK);
  REQUIRE(layer_linear_adapted_bf16(p, p, p, p, f, i32, p, p, 40, 256, 128, 3, 32, 128, 128, 256, nullptr, 0, nullptr) == CA_OK);
  std::vector<ca_adamw_tensor> many(700, ca_adamw_tensor{p, p, nullptr, p, p, f, f, i32, 300, CA_F32, CA_BF16});
  REQUIRE(layer_adamw(many.data(), static_cast<ca_adamw_tensor*>(p), 700, 8, 1e-3, 0.9, 0.99, 1e-8, 0.1, 1.0, nullptr) == CA_OK);
  REQUIRE(launches > 3);
  std::printf("adapt sanitizer driver: ok\n");
  return 0;
}

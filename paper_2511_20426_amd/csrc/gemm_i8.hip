// Y[M,N] = (X[M,K] . W[N,K]') * scale of X's row * scale of W's row, X and W in 8 bits, whole sums in 32 bits, Y in bf16.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "ca_internal.hpp"

namespace ca {
namespace {

#include "rope_device.hpp"
#include "gemm_tiles.hpp"
#include "gemm_tile_kernel.hpp"
#include "gemm_ops.hpp"
#include "gemm_op_tiles.hpp"
#include "gemm_few.hpp"

constexpr int kFewTokens = 32;

}  // namespace

int32_t launch_gemm_i8(const void* x, const float* x_scales, const void* w, const float* w_scales, void* y, int64_t M, int32_t N, int32_t K,
                       int64_t ldx, int64_t ldw, int64_t ldy, void* stream) {
  if (M == 0) return CA_OK;
  OpArgs a{};
  a.x = x; a.w = w; a.y = y; a.w2 = w_scales; a.xs = x_scales;
  a.ldy = ldy;
  a.M = int32_t(M); a.N = N; a.K = (K + 255) / 256 * 256;
  a.ldx = int32_t(ldx); a.ldw = int32_t(ldw);
  const KernelLds kernels[] = {{reinterpret_cast<const void*>(gemm_op_kernel<Tile128, I8>), Tile128::kLds},
                               {reinterpret_cast<const void*>(gemm_op_kernel<Tile64, I8>), Tile64::kLds}};
  if (const int32_t rc = ensure_dynamic_lds(kernels, 2, kLdsI8); rc != CA_OK) return rc;
  if (M <= kFewTokens) return enqueue_few<I8>(a, "gemm_i8.hip", stream);
  const int64_t tiles = ((M + 127) / 128) * ((N + 127) / 128);
  return tiles >= 128 ? enqueue_op_tile<Tile128, I8>(a, "gemm_i8.hip", stream) : enqueue_op_tile<Tile64, I8>(a, "gemm_i8.hip", stream);
}

}  // namespace ca

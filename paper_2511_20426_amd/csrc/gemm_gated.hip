// H[M,F] = act(X Wg') * (X Wu') in bf16 with fp32 accumulation: both projections of a gated feed-forward block, the activation and
// the product in one kernel.
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

int32_t launch_gemm_gated(const void* x, const void* w_gate, const void* w_up, void* h, void* g, void* u, int activation, int64_t M, int32_t F,
                          int32_t K, int64_t ldx, int64_t ldwg, int64_t ldwu, int64_t ldh, int64_t ld_saved, void* stream) {
  if (M == 0) return CA_OK;
  OpArgs a{};
  a.x = x; a.w = w_gate; a.w2 = w_up; a.y = h;
  a.g = static_cast<uint16_t*>(g); a.u = static_cast<uint16_t*>(u);
  a.ldy = ldh; a.ld_saved = ld_saved;
  a.M = int32_t(M); a.N = F; a.K = 2 * K;
  a.ldx = int32_t(2 * ldx); a.ldw = int32_t(2 * ldwg); a.ldw2 = int32_t(2 * ldwu);
  activation_factors(activation, &a.act0, &a.act1);
  const KernelLds kernels[] = {{reinterpret_cast<const void*>(gemm_op_kernel<Tile128, Gated>), Tile128::kLds},
                               {reinterpret_cast<const void*>(gemm_op_kernel<Tile64, Gated>), Tile64::kLds}};
  if (const int32_t rc = ensure_dynamic_lds(kernels, 2, kLdsGated); rc != CA_OK) return rc;
  if (M <= kFewTokens) return enqueue_few<Gated>(a, "gemm_gated.hip", stream);
  const int64_t tiles = ((M + 127) / 128) * ((F + 63) / 64);
  return tiles >= 128 ? enqueue_op_tile<Tile128, Gated>(a, "gemm_gated.hip", stream) : enqueue_op_tile<Tile64, Gated>(a, "gemm_gated.hip", stream);
}

}  // namespace ca

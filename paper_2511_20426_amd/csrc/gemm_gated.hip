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
#include "quantize_device.hpp"
#include "gemm_ops.hpp"
#include "gemm_op_rows.hpp"
#include "gemm_op_tiles.hpp"
#include "gemm_few.hpp"

constexpr int kFewTokens = 32;

using Tile64Tall = TileShape<64, 64, 4, 2, 6>;     // (a wave has two sub-tiles over the columns: gate and up)

constexpr OpModel kModel[] = {{256, 256, 1, 1580, 985, 1240, 6120}, {192, 256, 1, 2530, 765, 975, 4240}, {128, 256, 1, 2720, 610, 755, 2770},
                              {256, 128, 1, 0, 745, 835, 5100},     {128, 128, 1, 0, 450, 485, 2900},   {64, 64, 2, 0, 230, 360, 1725},
                              {64, 64, 1, 0, 165, 165, 3000}};

}  // namespace

int32_t launch_gemm_gated(const void* x, const void* w_gate, const void* w_up, void* h, float* saved, int activation, int64_t M, int32_t F,
                          int32_t K, int64_t ldx, int64_t ldwg, int64_t ldwu, int64_t ldh, void* stream) {
  if (M == 0) return CA_OK;
  OpArgs a{};
  a.x = x; a.w = w_gate; a.w2 = w_up; a.y = h;
  a.g = saved; a.u = saved ? saved + gated_saved_values(M, F) / 2 : nullptr;
  a.ldy = ldh;
  a.M = int32_t(M); a.N = F; a.K = 2 * K;
  a.ldx = int32_t(2 * ldx); a.ldw = int32_t(2 * ldwg); a.ldw2 = int32_t(2 * ldwu);
  activation_factors(activation, &a.act0, &a.act1);
  const KernelLds kernels[] = {{reinterpret_cast<const void*>(gemm_op_rows_kernel<8, Gated>), kOpRowsLds},
                               {reinterpret_cast<const void*>(gemm_op_rows_kernel<6, Gated>), kOpRowsLds},
                               {reinterpret_cast<const void*>(gemm_op_rows_kernel<4, Gated>), kOpRowsLds},
                               {reinterpret_cast<const void*>(gemm_op_kernel<Tile256x128, Gated>), Tile256x128::kLds},
                               {reinterpret_cast<const void*>(gemm_op_kernel<Tile128, Gated>), Tile128::kLds},
                               {reinterpret_cast<const void*>(gemm_op_kernel<Tile64, Gated>), Tile64::kLds},
                               {reinterpret_cast<const void*>(gemm_op_kernel<Tile64Tall, Gated>), Tile64Tall::kLds}};
  if (const int32_t rc = ensure_dynamic_lds(kernels, 7, kLdsGated); rc != CA_OK) return rc;
  int n_cu = 0;
  if (const int32_t rc = device_cu_count(&n_cu); rc != CA_OK) return rc;
  constexpr const char* kWhat = "gemm_gated.hip";
  if (M <= kFewTokens) return enqueue_few<Gated>(a, kWhat, stream);
  switch (pick_op(kModel, M, 2 * int64_t(F), a.K / 128, n_cu)) {
    case kOpRows256: return enqueue_op_rows<8, Gated>(a, kWhat, stream);
    case kOpRows192: return enqueue_op_rows<6, Gated>(a, kWhat, stream);
    case kOpRows128: return enqueue_op_rows<4, Gated>(a, kWhat, stream);
    case kOpTile256x128: return enqueue_op_tile<Tile256x128, Gated>(a, kWhat, stream);
    case kOpTile128: return enqueue_op_tile<Tile128, Gated>(a, kWhat, stream);
    case kOpTile64: return enqueue_op_tile<Tile64, Gated>(a, kWhat, stream);
    default: return enqueue_op_tile<Tile64Tall, Gated>(a, kWhat, stream);
  }
}

}  // namespace ca

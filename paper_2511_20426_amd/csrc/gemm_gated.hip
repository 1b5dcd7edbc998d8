// H[M,F] = act(X Wg') * (X Wu') in bf16 with fp32 accumulation: both projections of a gated feed-forward block, the activation and
// the product in one kernel.  Bound by the matrix pipe as the linear maps are: 23400 x 13824 x 5120 4287 us = 1546 TFLOP/s, the activation's
// part of a tile of 256 x 128 is about 1 us of 102.
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

// Up to two tiles of 16 tokens the weights' way from memory is what counts (gemm_few.hpp).  Us, few tokens' kernel / the fastest tile, weights
// in the caches: 23 x 2384 x 2560 9.9 / 10.8, 1 x 152 x 5120 11.9 / 17.5, 31 x 1608 x 2560 10.7 / 10.8; from memory 1 x 13824 x 5120
// 52.5 / 54.3, 8 x 8816 x 3840 31.9 / 35.5.
constexpr int kFewTokens = 32;

using Tile64Tall = TileShape<64, 64, 4, 2, 6>;     // (a wave has two sub-tiles over the columns: gate and up)

// Fitted to 85 products of up to 23400 rows, 13824 columns and k 5120 (64 x 64: two a CU, then one of eight waves); the pick is 0.6 % slower than
// the fastest of the seven in the geometric mean, 12 % at the worst.  By tile in this order, us: 23400 x 13824 x 5120 4287 / 4728 / 5793 /
// 6276 / 8090 / 11548 / -, 4680 x 4096 x 1536 99 / 103 / 103 / 123 / 139 / 181 / -, 300 x 4096 x 1536 31.8 / 25.5 / 20.7 / 23.9 / 14.6 /
// 16.7 / -, 3974 x 728 x 128 10.6 / 8.9 / 7.6 / 8.5 / 9.6 / 9.7 / 14.7.
constexpr OpModel kModel[] = {{256, 256, 1, 2780, 945, 1200, 5330}, {192, 256, 1, 3110, 755, 1000, 3750}, {128, 256, 1, 3010, 580, 735, 2715},
                              {256, 128, 1, 0, 730, 835, 5310},     {128, 128, 1, 0, 430, 480, 2925},     {64, 64, 2, 0, 225, 355, 1680},
                              {64, 64, 1, 0, 225, 195, 1795}};

}  // namespace

int32_t launch_gemm_gated(const void* x, const void* w_gate, const void* w_up, void* h, float* saved, int activation, int64_t M, int32_t F,
                          int32_t K, int64_t ldx, int64_t ldwg, int64_t ldwu, int64_t ldh, void* stream) {
  if (M == 0) return CA_OK;
  if (M <= kFewTokens && F > kFewColumns) return CA_EUNSUPPORTED;
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

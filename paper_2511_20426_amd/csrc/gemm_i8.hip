// Y[M,N] = (X[M,K] . W[N,K]') * scale of X's row * scale of W's row, X and W in 8 bits, whole sums in 32 bits, Y in bf16.
// Large products are bound by the matrix pipe at the clock that the chip's power leaves it: 23400 x 15360 x 5120 1276 us = 2890 TOP/s where the
// same tiles reach 1500 TFLOP/s in bf16 (stages of 128 bytes take as long, and hold twice as many k).
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
// in the caches: 23 x 2552 x 2560 6.3 / 7.1, 2 x 232 x 3840 6.3 / 8.4, 24 x 4160 x 2048 6.7 / 6.3; from memory one token 15360 x 5120
// 16.2 / 16.9, 5120 x 5120 9.3 / 12.4.
constexpr int kFewTokens = 32;

// Fitted to 86 products of up to 23400 rows, 15360 columns and k 5120 (64 x 64: two a CU, then one of eight waves); the pick is 0.5 % slower than
// the fastest of the seven in the geometric mean, 7 % at the worst.  By tile in this order, us: 23400 x 15360 x 5120 1276 / 1280 / 1528 / 1730
// / 1939 / 2868 / -, 4680 x 4608 x 1536 40.5 / 34.5 / 38.0 / 45.3 / 51.2 / 68.1 / -, 1560 x 1536 x 1536 20.9 / 16.9 / 13.1 / 14.2 / 9.5 /
// 11.6 / -, 13427 x 304 x 256 9.6 / 8.2 / 7.1 / 8.1 / 9.2 / 9.3 / -, 64 x 1448 x 640 12.9 / 10.5 / 8.9 / 9.4 / 6.8 / 6.4 / 6.8.
constexpr OpModel kModel[] = {{256, 256, 1, 1980, 960, 1270, 5400}, {192, 256, 1, 2140, 770, 1010, 4460}, {128, 256, 1, 2340, 580, 745, 3350},
                              {256, 128, 1, 0, 705, 840, 5650},     {128, 128, 1, 0, 455, 470, 3680},     {64, 64, 2, 0, 290, 370, 1990},
                              {64, 64, 1, 0, 255, 190, 2000}};

// Whether the codes of few tokens are made in the product's launch: they are unless making them in every workgroup costs more than the launch
// that it saves.  Us, ahead / in the launch, weights from memory: one token 512 x 230 5.7 / 3.1, 4608 x 1536 7.5 / 5.3, 5120 x 5120 13.0 /
// 8.0, 15360 x 5120 20.2 / 16.1; two 5120 x 5120 13.4 / 8.9, 15360 x 5120 20.1 / 21.1; four 4608 x 1536 8.0 / 5.7, 1536 x 5120 9.2 / 8.7; twelve
// 512 x 230 6.2 / 4.9, 4608 x 1536 8.5 / 7.7, 15360 x 512 8.0 / 8.7.
bool codes_in_launch(int64_t M, int32_t N, int32_t K) {
  if (K <= CodesTwelve::kMost) return M <= (N <= 8192 ? CodesTwelve::kTokens : 8);
  if (K > CodesOne::kMost) return false;
  return M == 1 || (M == 2 && N <= 12288) || (M <= CodesFour::kTokens && M * ((N + 15) / 16) * K <= 6000000);
}

// one call of any size readies all kernels for stream capture
int32_t i8_ready() {
  const KernelLds kernels[] = {{reinterpret_cast<const void*>(gemm_op_rows_kernel<8, I8>), kOpRowsLds},
                               {reinterpret_cast<const void*>(gemm_op_rows_kernel<6, I8>), kOpRowsLds},
                               {reinterpret_cast<const void*>(gemm_op_rows_kernel<4, I8>), kOpRowsLds},
                               {reinterpret_cast<const void*>(gemm_op_kernel<Tile256x128, I8>), Tile256x128::kLds},
                               {reinterpret_cast<const void*>(gemm_op_kernel<Tile128, I8>), Tile128::kLds},
                               {reinterpret_cast<const void*>(gemm_op_kernel<Tile64, I8>), Tile64::kLds},
                               {reinterpret_cast<const void*>(gemm_op_kernel<Tile64Wide, I8>), Tile64Wide::kLds}};
  return ensure_dynamic_lds(kernels, 7, kLdsI8);
}

}  // namespace

int32_t launch_gemm_i8(const void* x, const float* x_scales, const void* w, const float* w_scales, void* y, int64_t M, int32_t N, int32_t K,
                       int64_t ldx, int64_t ldw, int64_t ldy, void* stream) {
  if (M == 0) return CA_OK;
  if (M <= kFewTokens && N > kFewColumns) return CA_EUNSUPPORTED;
  OpArgs a{};
  a.x = x; a.w = w; a.y = y; a.w2 = w_scales; a.xs = x_scales;
  a.ldy = ldy;
  a.M = int32_t(M); a.N = N; a.K = (K + 255) / 256 * 256;
  a.ldx = int32_t(ldx); a.ldw = int32_t(ldw);
  if (const int32_t rc = i8_ready(); rc != CA_OK) return rc;
  int n_cu = 0;
  if (const int32_t rc = device_cu_count(&n_cu); rc != CA_OK) return rc;
  constexpr const char* kWhat = "gemm_i8.hip";
  if (M <= kFewTokens) return enqueue_few<I8>(a, kWhat, stream);
  switch (pick_op(kModel, M, N, a.K / 128, n_cu)) {
    case kOpRows256: return enqueue_op_rows<8, I8>(a, kWhat, stream);
    case kOpRows192: return enqueue_op_rows<6, I8>(a, kWhat, stream);
    case kOpRows128: return enqueue_op_rows<4, I8>(a, kWhat, stream);
    case kOpTile256x128: return enqueue_op_tile<Tile256x128, I8>(a, kWhat, stream);
    case kOpTile128: return enqueue_op_tile<Tile128, I8>(a, kWhat, stream);
    case kOpTile64: return enqueue_op_tile<Tile64, I8>(a, kWhat, stream);
    default: return enqueue_op_tile<Tile64Wide, I8>(a, kWhat, stream);
  }
}

int32_t launch_gemm_i8_values(int dtype, const void* x, int64_t ldx, const void* w, const float* w_scales, void* y, int64_t M, int32_t N, int32_t K,
                              int64_t ldw, int64_t ldy, void* workspace, void* stream) {
  if (M == 0) return CA_OK;
  if (M <= kFewTokens && N > kFewColumns) return CA_EUNSUPPORTED;
  if (const int32_t rc = i8_ready(); rc != CA_OK) return rc;
  const auto kernel = M == 1                         ? gemm_few_kernel<I8, 1, CodesOne>
                      : K > CodesTwelve::kMost       ? M == 2 ? gemm_few_kernel<I8, 1, CodesTwo> : gemm_few_kernel<I8, 1, CodesFour>
                      : M <= CodesFourShort::kTokens ? gemm_few_kernel<I8, 1, CodesFourShort>
                                                     : gemm_few_kernel<I8, 1, CodesTwelve>;
  if (dtype == CA_BF16 && K >= 8 && codes_in_launch(M, N, K)) {
    OpArgs a{};
    a.x = x; a.w = w; a.y = y; a.w2 = w_scales;
    a.ldy = ldy;
    a.M = int32_t(M); a.N = N; a.K = (K + 255) / 256 * 256; a.k_values = K;
    a.ldx = int32_t(2 * ldx); a.ldw = int32_t(ldw);
    hipLaunchKernelGGL(kernel, dim3(unsigned((N + 15) / 16)), dim3(64 * kFewWaves), 0, static_cast<hipStream_t>(stream), a);
    return finish_launch("gemm_i8.hip");
  }
  const int64_t ld = (K + 255) / 256 * 256;
  float* const scales = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + M * ld);
  if (const int32_t rc = launch_quantize_rows(dtype, x, workspace, scales, M, K, ldx, ld, stream); rc != CA_OK) return rc;
  return launch_gemm_i8(workspace, scales, w, w_scales, y, M, N, K, ld, ldw, ldy, stream);
}

}  // namespace ca

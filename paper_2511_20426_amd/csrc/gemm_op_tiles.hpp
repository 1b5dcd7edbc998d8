// The 8-bit linear map and the gated projections in the compiled tiles of gemm_tile_kernel.hpp, a workgroup a tile.  8 bits put 128 k
// into a stage where bf16 has 64, and an MFMA of the same 16 bytes a lane and the same time multiplies twice as many.
//
// Gated: of a tile's W rows one half are the gate's and one the up projection's, dealt so that a wave has both for the same
// columns: of its kTn sub-tiles of 16 rows the first half are gate rows, the second the up rows of the same columns, and a lane
// ends up with g and u of the same elements.  The products meet in registers; neither is written unless training asks for them.
// (Included behind gemm_ops.hpp.)
#pragma once

template <typename T, typename Op>
__global__ __launch_bounds__(T::kThreads) void gemm_op_kernel(OpArgs a) {
  using Products = typename Op::Products;
  constexpr int BM = T::kBm, BN = T::kBn, kWavesM = T::kWavesAlongM, kStages = T::kRing;
  constexpr int kCols = Op::kGated ? BN / 2 : BN;                   // of the result
  static_assert(!Op::kGated || (T::kTn % 2 == 0 && T::kLoadsW * 8 <= 16), "a wave has gate and up rows of the same columns, and loads rows of one of them");
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l15 = lane & 15, grp = lane >> 4;
  const int wm = wave % kWavesM, wn = wave / kWavesM;
  const int nth = int(blockIdx.x & 7) * a.more + int(blockIdx.x >> 3);          // XCD x takes a contiguous range of the tiles
  if (nth >= a.tiles_m * a.tiles_n) return;
  int tm, tn;
  tile_at(a.tiles_m, a.tiles_n, nth, &tm, &tn);
  const int m0 = tm * BM, n0 = tn * kCols;

  // load i of a wave brings 8 rows of 128 bytes, chunks swizzled by the row; rows past the end re-read the last one
  uint32_t offw[T::kLoadsW], offx[T::kLoadsX];
  const uint8_t* wbase = static_cast<const uint8_t*>(a.w);
  int ldw = a.ldw, first = 0;                                       // first: of the tile's columns, that of the wave's row 0
  if constexpr (Op::kGated) {
    const int sub = wave * T::kLoadsW / 2, in_wave = sub % T::kTn, up = in_wave >= T::kTn / 2;
    wbase = static_cast<const uint8_t*>(up ? a.w2 : a.w);
    ldw = up ? a.ldw2 : a.ldw;
    first = (sub / T::kTn * (T::kTn / 2) + in_wave - up * (T::kTn / 2) - sub) * 16;
  }
#pragma unroll
  for (int i = 0; i < T::kLoadsW; ++i) {
    const int row = (wave * T::kLoadsW + i) * 8 + (lane >> 3), c = (lane & 7) ^ ((row >> 1) & 7);
    offw[i] = uint32_t(min(n0 + row + first, a.N - 1) - n0) * uint32_t(ldw) + c * 16;
  }
#pragma unroll
  for (int i = 0; i < T::kLoadsX; ++i) {
    const int row = (wave * T::kLoadsX + i) * 8 + (lane >> 3), c = (lane & 7) ^ ((row >> 1) & 7);
    offx[i] = uint32_t(min(m0 + row, a.M - 1) - m0) * uint32_t(a.ldx) + c * 16;
  }
  uint64_t base_w = reinterpret_cast<uint64_t>(wbase + int64_t(n0) * ldw);
  uint64_t base_x = reinterpret_cast<uint64_t>(static_cast<const uint8_t*>(a.x) + int64_t(m0) * a.ldx);
  int n_stages = a.K / 128;
  if constexpr (Op::kPart) {                                        // grid.y: the part
    const int begin = int(blockIdx.y) * a.k_values;
    base_w += uint64_t(begin) * 128;
    base_x += uint64_t(begin) * 128;
    n_stages = min(a.k_values, n_stages - begin);
  }
#include "gemm_tile_loop.hpp"

  if constexpr (Op::kPart) {                                        // straight from registers, 16 bytes to a lane
#pragma unroll
    for (int i = 0; i < T::kTn; ++i)
#pragma unroll
      for (int j = 0; j < T::kTm; ++j) {
        const int row = m0 + (wm * T::kTm + j) * 16 + l15, col = n0 + (wn * T::kTn + i) * 16 + 4 * grp;
        if (row < a.M && col < a.N) *reinterpret_cast<f32x4*>(a.g + (int64_t(blockIdx.y) * a.M + row) * a.N + col) = acc[i][j];
      }
    return;
  }
  // ---- the results go through LDS to leave row by row.  A lane has columns 4 grp .. +3 of row l15 of a sub-tile.
  constexpr int kPitch = kCols * 2 + 16;
  if constexpr (Op::kGated) {
    constexpr int kHalf = T::kTn / 2;
#pragma unroll
    for (int i = 0; i < kHalf; ++i)
#pragma unroll
      for (int j = 0; j < T::kTm; ++j) {
        const f32x4 &g = acc[i][j], &u = acc[i + kHalf][j];
        const int row = (wm * T::kTm + j) * 16 + l15, col = (wn * kHalf + i) * 16 + 4 * grp;
        float h[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = gated_value(g[e], u[e], a.act0, a.act1);
        uint32_t* to = reinterpret_cast<uint32_t*>(lds + row * kPitch + col * 2);
        to[0] = pack_bf16(h[0], h[1]);
        to[1] = pack_bf16(h[2], h[3]);
        if (a.g && m0 + row < a.M && n0 + col < a.N) {
          const int64_t at = saved_at(m0 + row, n0 + col, a.N);
          *reinterpret_cast<f32x4*>(a.g + at) = g;
          *reinterpret_cast<f32x4*>(a.u + at) = u;
        }
      }
  } else {
    float xs[T::kTm];
#pragma unroll
    for (int j = 0; j < T::kTm; ++j) xs[j] = a.xs[min(m0 + (wm * T::kTm + j) * 16 + l15, a.M - 1)];
#pragma unroll
    for (int i = 0; i < T::kTn; ++i) {
      const int col = (wn * T::kTn + i) * 16 + 4 * grp;
      float ws[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) ws[e] = static_cast<const float*>(a.w2)[min(n0 + col + e, a.N - 1)];
#pragma unroll
      for (int j = 0; j < T::kTm; ++j) {
        uint32_t* to = reinterpret_cast<uint32_t*>(lds + ((wm * T::kTm + j) * 16 + l15) * kPitch + col * 2);
        to[0] = pack_bf16(scaled(acc[i][j][0], xs[j], ws[0]), scaled(acc[i][j][1], xs[j], ws[1]));
        to[1] = pack_bf16(scaled(acc[i][j][2], xs[j], ws[2]), scaled(acc[i][j][3], xs[j], ws[3]));
      }
    }
  }
  __syncthreads();
  constexpr int kChunks = kCols / 8, kRows = T::kThreads / kChunks;
  const int c = tid % kChunks;
#pragma unroll 4
  for (int row = tid / kChunks; row < BM; row += kRows) {
    const u32x4 v = *reinterpret_cast<const u32x4*>(lds + row * kPitch + c * 16);
    if (m0 + row < a.M && n0 + c * 8 < a.N)
      __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.y) + int64_t(m0 + row) * a.ldy + n0 + c * 8));
  }
}

template <typename T, typename Op>
int32_t enqueue_op_tile(OpArgs& a, const char* what, void* stream, unsigned parts = 1) {
  constexpr int kCols = Op::kGated ? T::kBn / 2 : T::kBn;
  a.tiles_m = (a.M + T::kBm - 1) / T::kBm;
  a.tiles_n = (a.N + kCols - 1) / kCols;
  const int64_t tiles = int64_t(a.tiles_m) * a.tiles_n;
  if ((tiles + 7) * T::kThreads * parts >= (int64_t(1) << 32)) return CA_EUNSUPPORTED;      // a launch may have 2^32 threads
  a.more = int32_t((tiles + 7) / 8);
  hipLaunchKernelGGL((gemm_op_kernel<T, Op>), dim3(unsigned(a.more) * 8, parts), dim3(T::kThreads), T::kLds, static_cast<hipStream_t>(stream), a);
  return finish_launch(what);
}

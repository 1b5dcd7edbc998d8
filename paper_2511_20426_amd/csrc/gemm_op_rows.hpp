// The 8-bit linear map and the gated projections in tiles of 256 rows of W: the kernels around the assembly that gen_gemm_rows.py emits
// for them, which documents the pipeline, the register map and how the results leave.  The dealing of tiles and the lanes' parts
// in loads and reads are those of gemm_rows.hip.
// (Included behind gemm_ops.hpp.)
#pragma once

#include "gemm_rows_gated_clobbers.inc"
#include "gemm_rows_i8_clobbers.inc"

constexpr int kOpRowsLds = 160 * 1024;            // 3 stages of W, 2 of X
constexpr int kOpFormThrough = 1, kOpFormPast = 2;   // results written through L2, past the caches; 0: left in L2
constexpr int kOpList = 64;                       // tiles of a workgroup: one to a lane

// kMt: 16-row sub-tiles of X to a wave; a tile of Y has 32 kMt rows and 256 columns, gated 128.
template <int kMt, typename Op>
__global__ __launch_bounds__(256, 1) void gemm_op_rows_kernel(OpArgs a) {
  constexpr int kTileRows = 32 * kMt, kWaveRows = 16 * kMt, kWaveCols = Op::kGated ? 64 : 128;
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  const int tid = threadIdx.x, lane = tid & 63, l15 = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave & 1, wn = wave >> 1;
  // ---- this workgroup's tiles, one to a lane
  const int xcd = int(blockIdx.x & 7), j = int(blockIdx.x >> 3) & 31, first = int(blockIdx.x >> 8) * kOpList;
  const int total = a.tiles_m * a.tiles_n, full = total >> 8, left = total & 255, share = last_round_share(left);
  const int mine = full + (j < share && xcd * share + j < left ? 1 : 0);
  const int tiles = min(mine - first, kOpList);
  if (tiles <= 0) return;
  const int r = min(first + lane, mine - 1);
  int list_m, list_n;
  tile_at(a.tiles_m, a.tiles_n, r < full ? r * 256 + xcd * 32 + j : full * 256 + xcd * share + j, &list_m, &list_n);

  // ---- the lane's part in loads: load i of a wave brings LDS rows (8 wave + i) 8 .. +7 of W (gated: waves 0 and 2 the gate's, 1 and 3 the
  // up projection's of the same columns), (kMt wave + i) 8 .. of X
  const int roww = (Op::kGated ? wave >> 1 : wave) * 64 + (lane >> 3), rowx = wave * 8 * kMt + (lane >> 3);
  const int chunkw = ((lane & 7) ^ ((lane >> 4) & 1)) * 16, chunkx = ((lane & 7) ^ (lane >> 4)) * 16;
  // ... in operand reads (lane = row l15 of a sub-tile, 16 bytes of group grp) ...
  const int aw0 = (wn * 128 + 8 * (l15 >> 2) + (l15 & 3)) * 128 + ((grp ^ (l15 >> 1)) << 4);
  const int ax0 = (wm * kWaveRows + l15) * 128 + ((grp ^ (l15 >> 1)) << 4);
  // ... and of the results: of the first eight rows of sub-tile 0 row l15 % 8, columns 32 (l15 / 8) + 8 grp ..
  const int row = wm * kWaveRows + (l15 & 7), col = wn * kWaveCols + 32 * (l15 >> 3) + 8 * grp;
  const uint64_t ylane = uint64_t(row) * uint64_t(a.ldy) * 2 + uint64_t(col) * 2;
  const bool up = Op::kGated && (wave & 1);
  const uint64_t x = reinterpret_cast<uint64_t>(a.x), w = reinterpret_cast<uint64_t>(up ? a.w2 : a.w), y = reinterpret_cast<uint64_t>(a.y);
  const uint64_t tile_y = uint64_t(a.ldy) * 2 * kTileRows, row8 = uint64_t(a.ldy) * 2 * 8;
  const uint32_t ldw2 = uint32_t(up ? a.ldw2 : a.ldw), ldx2 = uint32_t(a.ldx);       // bytes
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds));
#define CA_GEMM_OP_ROWS_OPERANDS                                                                                       \
  [x_lo] "s"(uint32_t(x)), [x_hi] "s"(uint32_t(x >> 32)), [w_lo] "s"(uint32_t(w)), [w_hi] "s"(uint32_t(w >> 32)),      \
      [y_lo] "s"(uint32_t(y)), [y_hi] "s"(uint32_t(y >> 32)), [tile_x] "s"(ldx2 * kTileRows),                          \
      [tile_w] "s"(ldw2 * (2 * kWaveCols)), [tile_y_lo] "s"(uint32_t(tile_y)), [tile_y_hi] "s"(uint32_t(tile_y >> 32)),\
      [row8_lo] "s"(uint32_t(row8)), [row8_hi] "s"(uint32_t(row8 >> 32)), [ldw2] "s"(ldw2), [ldx2] "s"(ldx2),          \
      [M] "s"(a.M), [N] "s"(a.N), [n_stages] "s"(a.K / 128), [tiles] "s"(tiles), [form] "s"(a.more), [wave] "s"(wave), \
      [lds0] "s"(lds0), [list_m] "v"(list_m), [list_n] "v"(list_n), [roww] "v"(roww), [rowx] "v"(rowx),                \
      [chunkw] "v"(chunkw), [chunkx] "v"(chunkx), [aw0] "v"(aw0), [ax0] "v"(ax0), [row] "v"(row), [col] "v"(col),      \
      [ylane_lo] "v"(uint32_t(ylane)), [ylane_hi] "v"(uint32_t(ylane >> 32))
  if constexpr (Op::kGated) {
    const uint64_t g = reinterpret_cast<uint64_t>(a.g), u = reinterpret_cast<uint64_t>(a.u);
#define CA_GEMM_GATED_OPERANDS                                                                                         \
  CA_GEMM_OP_ROWS_OPERANDS, [g] "s"(g), [g_lo] "s"(uint32_t(g)), [g_hi] "s"(uint32_t(g >> 32)), [u_lo] "s"(uint32_t(u)), \
      [u_hi] "s"(uint32_t(u >> 32)), [blocks_n] "s"((a.N + 31) / 32), [act0] "s"(a.act0), [act1] "s"(a.act1)
    if constexpr (kMt == 8) {
      asm volatile(
#include "gemm_rows_gated_256_gfx950.inc"
          :: CA_GEMM_GATED_OPERANDS : "memory", "vcc", "scc", "m0", CA_GEMM_ROWS_GATED_CLOBBERS256);
    } else if constexpr (kMt == 6) {
      asm volatile(
#include "gemm_rows_gated_192_gfx950.inc"
          :: CA_GEMM_GATED_OPERANDS : "memory", "vcc", "scc", "m0", CA_GEMM_ROWS_GATED_CLOBBERS192);
    } else {
      asm volatile(
#include "gemm_rows_gated_128_gfx950.inc"
          :: CA_GEMM_GATED_OPERANDS : "memory", "vcc", "scc", "m0", CA_GEMM_ROWS_GATED_CLOBBERS128);
    }
  } else {
    const uint64_t xs = reinterpret_cast<uint64_t>(a.xs), ws = reinterpret_cast<uint64_t>(a.w2);
#define CA_GEMM_I8_OPERANDS                                                                                            \
  CA_GEMM_OP_ROWS_OPERANDS, [xs_lo] "s"(uint32_t(xs)), [xs_hi] "s"(uint32_t(xs >> 32)), [ws_lo] "s"(uint32_t(ws)),     \
      [ws_hi] "s"(uint32_t(ws >> 32))
    if constexpr (kMt == 8) {
      asm volatile(
#include "gemm_rows_i8_256_gfx950.inc"
          :: CA_GEMM_I8_OPERANDS : "memory", "vcc", "scc", "m0", CA_GEMM_ROWS_I8_CLOBBERS256);
    } else if constexpr (kMt == 6) {
      asm volatile(
#include "gemm_rows_i8_192_gfx950.inc"
          :: CA_GEMM_I8_OPERANDS : "memory", "vcc", "scc", "m0", CA_GEMM_ROWS_I8_CLOBBERS192);
    } else {
      asm volatile(
#include "gemm_rows_i8_128_gfx950.inc"
          :: CA_GEMM_I8_OPERANDS : "memory", "vcc", "scc", "m0", CA_GEMM_ROWS_I8_CLOBBERS128);
    }
  }
}

template <int kMt, typename Op>
int32_t enqueue_op_rows(OpArgs& a, const char* what, void* stream) {
  constexpr int kCols = Op::kGated ? 128 : 256;
  a.tiles_m = (a.M + 32 * kMt - 1) / (32 * kMt);
  a.tiles_n = (a.N + kCols - 1) / kCols;
  const int64_t total = int64_t(a.tiles_m) * a.tiles_n, rounds = (total + 255) / 256;
  if (total >= (int64_t(1) << 30)) return CA_EUNSUPPORTED;
  const unsigned workgroups = total < 256 ? 8 * unsigned(last_round_share(int(total))) : 256 * unsigned((rounds + kOpList - 1) / kOpList);
  // how results leave: as enqueue_gemm_rows says
  const bool whole_lines = a.ldy % 64 == 0 && reinterpret_cast<uintptr_t>(a.y) % 128 == 0;
  a.more = whole_lines ? kOpFormPast | kOpFormThrough << 2 : (rounds <= 1 ? kOpFormThrough << 2 : 0);
  const auto kernel = gemm_op_rows_kernel<kMt, Op>;
  hipLaunchKernelGGL(kernel, dim3(workgroups), dim3(256), kOpRowsLds, static_cast<hipStream_t>(stream), a);
  return finish_launch(what);
}

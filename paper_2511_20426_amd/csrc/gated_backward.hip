// The gradients of the gated projections H = act(G) * U, G = X Wg', U = X Wu' (F columns, rows of K):
//
//   dG = dH U act'(G),  dU = dH act(G);  dX = dG Wg + dU Wu,  dWg = dG' X,  dWu = dU' X
//
// The products are the framework's own linear map, which multiplies rows by rows: one launch forms dG and dU from dH and the saved
// projections, in rows (side by side, [M][2 Fp], for dX) and transposed ([2 F][Mp], for dW), and lays out X' [K][Mp] and [Wg; Wu]' [K][2 Fp]
// in the workspace.  Fp and Mp are F and M filled up with zeros to whole steps of the products (2 Fp and Mp are multiples of 128).  There dG
// and dU are rounded to bf16, the type that the matrix products take: with the result's own rounding gradients are 2.35e-3 of their norm
// off, 1.66e-3 of which is that of the result.  (With G and U saved in bf16 as well it was 3.1e-3: they are saved in fp32.)  In two bf16 values
// each, as below, the products are twice as long: 4680 x 4096 x 1536 dX 92 and dW 90 us, 177 and 169 so.  dX is one product over both, so that
// their sum is not rounded in between.
//
// Of up to 32 rows all of it is one pass over the weights, read once, and their gradients, written once, with nothing laid out
// (gated_few_grad_kernel, gated_some_grad_kernel), bound by memory: dG and dU go into the products in fp32 (up to four rows) or as two bf16 values
// each, which stand for 16 bits and more, and gradients are 1.66e-3 of their norm off, the rounding of the result.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "ca_internal.hpp"

namespace ca {
namespace {

#include "rope_device.hpp"
#include "gemm_tiles.hpp"
#include "gemm_tile_kernel.hpp"
#include "gemm_ops.hpp"
#include "gemm_op_tiles.hpp"

constexpr int kSide = 64;                         // of a tile that is transposed
constexpr int kRow = kSide / 2 + 1;               // dwords of its rows in LDS: columns are read without conflicts

// Tile (rows of 64 values as 8 chunks of 16 bytes) to LDS, and from there 8 consecutive rows' values of a column.
__device__ __forceinline__ void put_chunk(uint32_t* tile, int row, int chunk, const U4& v) {
  uint32_t* to = tile + row * kRow + chunk * 4;
  to[0] = v.x; to[1] = v.y; to[2] = v.z; to[3] = v.w;
}
__device__ __forceinline__ U4 column_chunk(const uint32_t* tile, int col, int chunk) {
  uint32_t e[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t w = tile[(chunk * 8 + j) * kRow + (col >> 1)];
    e[j] = col & 1 ? w >> 16 : w & 0xffffu;
  }
  return U4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16};
}

// A matrix to transpose: tiles_c tiles of 64 columns, as many rows of tiles as its part of the grid has.
struct TransposeArgs {
  const uint16_t* x;                              // [rows][ldx]
  uint16_t* y;                                    // [cols][ldy], columns from rows up to whole tiles are zero
  int64_t ldx, ldy;
  int32_t rows, cols;
};

__device__ __forceinline__ void transpose_tile(const TransposeArgs& a, uint32_t* tile, int nth) {
  const int t = threadIdx.x, chunk = t & 7, tiles_c = (a.cols + kSide - 1) / kSide;
  const int c0 = nth % tiles_c * kSide, r0 = nth / tiles_c * kSide;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = (t >> 3) + 32 * i;
    U4 v = {0, 0, 0, 0};
    if (r0 + row < a.rows && c0 + chunk * 8 < a.cols) v = load_once(a.x + int64_t(r0 + row) * a.ldx + c0 + chunk * 8);
    put_chunk(tile, row, chunk, v);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int col = (t >> 3) + 32 * i;
    if (c0 + col < a.cols) *reinterpret_cast<U4*>(a.y + int64_t(c0 + col) * a.ldy + r0 + chunk * 8) = column_chunk(tile, col, chunk);
  }
}

struct GatedGradArgs {
  const uint16_t* dh;
  const float *g, *u;
  uint16_t *rows, *cols;                          // [M][2 Fp] and [2 F][Mp]
  int64_t lddh;
  int32_t M, F, Mp, Fp;
  float act0, act1;
};

// act and act' of a gate: act' = s + g s (1 - s) p'(g), p = g (act0 + act1 g^2).  (The bound on g for p would make a number of a NaN.)
__device__ __forceinline__ void activation(float g, float act0, float act1, float* act, float* slope) {
  float p;
  const float s = act_sigmoid(g, act0, act1, &p), c = __builtin_amdgcn_fmed3f(g, -1e4f, 1e4f);
  *act = g * s;
  *slope = g == g ? fmaf(c * s * (1.f - s), fmaf(c * c, 3.f * act1, act0), s) : g;
}

__device__ __forceinline__ void gated_grad_tile(const GatedGradArgs& a, uint32_t (*tile)[kSide * kRow], int nth) {
  const int t = threadIdx.x, chunk = t & 7, tiles_f = a.Fp / kSide;
  const int f0 = nth % tiles_f * kSide, m0 = nth / tiles_f * kSide;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = (t >> 3) + 32 * i, m = m0 + row, f = f0 + chunk * 8;
    U4 dg = {0, 0, 0, 0}, du = {0, 0, 0, 0};
    if (m < a.M && f < a.F) {
      Vec8<uint16_t> dh;
      dh.load(a.dh + int64_t(m) * a.lddh + f);
      float g[8], u[8], v[8], w[8];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int64_t at = saved_at(m, f + 4 * half, a.F);
        *reinterpret_cast<f32x4*>(g + 4 * half) = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(a.g + at));
        *reinterpret_cast<f32x4*>(u + 4 * half) = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(a.u + at));
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float act, slope;
        activation(g[j], a.act0, a.act1, &act, &slope);
        v[j] = dh.v[j] * u[j] * slope;
        w[j] = dh.v[j] * act;
      }
      dg = U4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
      du = U4{pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3]), pack_bf16(w[4], w[5]), pack_bf16(w[6], w[7])};
    }
    if (m < a.M) {
      uint16_t* to = a.rows + int64_t(m) * 2 * a.Fp + f;
      *reinterpret_cast<U4*>(to) = dg;
      *reinterpret_cast<U4*>(to + a.Fp) = du;
    }
    put_chunk(tile[0], row, chunk, dg);
    put_chunk(tile[1], row, chunk, du);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int col = (t >> 3) + 32 * i, m = m0 + chunk * 8;
    if (f0 + col >= a.F) continue;
    uint16_t* to = a.cols + int64_t(f0 + col) * a.Mp + m;
    *reinterpret_cast<U4*>(to) = column_chunk(tile[0], col, chunk);
    *reinterpret_cast<U4*>(to + int64_t(a.F) * a.Mp) = column_chunk(tile[1], col, chunk);
  }
}

// What the products take, in one launch: memory bound, 4680 x 4096 x 1536 70 us (81 in a launch for the gradients and two for the
// transpositions).  The first grad_tiles workgroups form dG and dU, then come the tiles of each matrix that is transposed.
struct GatedLayoutArgs {
  GatedGradArgs grad;
  TransposeArgs t[3];
  int32_t grad_tiles, ends[3];                    // ends: of the matrices' workgroups
};

__global__ __launch_bounds__(256) void gated_layout_kernel(GatedLayoutArgs a) {
  __shared__ uint32_t tile[2][kSide * kRow];
  const int b = int(blockIdx.x);
  if (b < a.grad_tiles)
    gated_grad_tile(a.grad, tile, b);
  else if (b < a.ends[0])
    transpose_tile(a.t[0], tile[0], b - a.grad_tiles);
  else if (b < a.ends[1])
    transpose_tile(a.t[1], tile[0], b - a.ends[0]);
  else
    transpose_tile(a.t[2], tile[0], b - a.ends[1]);
}

// Up to four rows: both weights read and their gradients written once are what counts (one row of 13824 x 5120 133 us, 566 MB; four 136; of 4096 x
// 1536 18.0 and 18.5).  A workgroup takes 128 columns of K and `each` columns f of the projections: sixteen threads eight columns of K
// each, and sixteen such rows of threads every sixteenth f.  dG and dU of the f are formed in LDS, in fp32; of each f a thread reads its
// part of Wg and Wu, adds to its sums of dX, and forms and writes its part of dWg and dWu from X's rows, which it keeps.  The sums of
// dX of a workgroup's f go to the workspace; a second launch adds them up in order.
struct GatedFewArgs {
  const uint16_t *dh, *x, *wg, *wu;
  const float *g, *u;
  uint16_t *dwg, *dwu;                            // null: not asked for
  float* partials;                                // [parts of f][M][K], or null: dX is not asked for
  int64_t lddh, ldx, ldwg, ldwu, lddw;
  int32_t M, F, K, each;
  float act0, act1;
};

constexpr int kFewGradRows = 4, kSomeGradRows = 32;       // rows of the two kernels for few

__global__ __launch_bounds__(256) void gated_few_grad_kernel(GatedFewArgs a) {
  constexpr int kRows = kFewGradRows;
  extern __shared__ __attribute__((aligned(16))) float grads[];        // [f of the workgroup][dG | dU][kRows]; then the sums of dX
  const int t = threadIdx.x, k = (blockIdx.x * 16 + (t & 15)) * 8, lane_f = t >> 4;
  const int f0 = blockIdx.y * a.each, count = min(a.each, a.F - f0);
  for (int i = t; i < count * kRows; i += 256) {
    const int f = i / kRows, m = i - f * kRows;
    float dg = 0.f, du = 0.f;
    if (m < a.M) {
      const int64_t at = saved_at(m, (f0 + f) & ~3, a.F) + ((f0 + f) & 3);
      const float dh = __uint_as_float(uint32_t(a.dh[int64_t(m) * a.lddh + f0 + f]) << 16);
      float act, slope;
      activation(a.g[at], a.act0, a.act1, &act, &slope);
      dg = dh * a.u[at] * slope;
      du = dh * act;
    }
    grads[f * 2 * kRows + m] = dg;
    grads[f * 2 * kRows + kRows + m] = du;
  }
  U4 x[kRows];
#pragma unroll
  for (int m = 0; m < kRows; ++m) x[m] = m < a.M ? *reinterpret_cast<const U4*>(a.x + int64_t(m) * a.ldx + k) : U4{0, 0, 0, 0};
  __syncthreads();
  float dx[kRows][8];
#pragma unroll
  for (int m = 0; m < kRows; ++m)
#pragma unroll
    for (int j = 0; j < 8; ++j) dx[m][j] = 0.f;
  for (int f = lane_f; f < count; f += 16) {
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      float d[kRows];
#pragma unroll
      for (int m = 0; m < kRows; m += 4) *reinterpret_cast<f32x4*>(d + m) = *reinterpret_cast<const f32x4*>(grads + (f * 2 + side) * kRows + m);
      if (a.partials) {
        Vec8<uint16_t> w;
        w.load((side ? a.wu + (f0 + f) * a.ldwu : a.wg + (f0 + f) * a.ldwg) + k);
#pragma unroll
        for (int m = 0; m < kRows; ++m)
#pragma unroll
          for (int j = 0; j < 8; ++j) dx[m][j] = fmaf(d[m], w.v[j], dx[m][j]);
      }
      uint16_t* const dw = side ? a.dwu : a.dwg;
      if (dw) {
        Vec8<uint16_t> s;
#pragma unroll
        for (int j = 0; j < 8; ++j) s.v[j] = 0.f;
#pragma unroll
        for (int m = 0; m < kRows; ++m) {
          const uint32_t w[4] = {x[m].x, x[m].y, x[m].z, x[m].w};
#pragma unroll
          for (int j = 0; j < 8; ++j) s.v[j] = fmaf(d[m], j & 1 ? bf16_hi(w[j / 2]) : bf16_lo(w[j / 2]), s.v[j]);
        }
        s.store(dw + (f0 + f) * a.lddw + k);
      }
    }
  }
  if (!a.partials) return;
  __syncthreads();
#pragma unroll
  for (int m = 0; m < kRows; ++m)                  // over the four rows of threads of a wave ...
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      dx[m][j] += __shfl_xor(dx[m][j], 16, 64);
      dx[m][j] += __shfl_xor(dx[m][j], 32, 64);
    }
  if ((t & 63) < 16) {
#pragma unroll
    for (int m = 0; m < kRows; ++m)
#pragma unroll
      for (int j = 0; j < 8; ++j) grads[((t >> 6) * kRows + m) * 128 + (t & 15) * 8 + j] = dx[m][j];
  }
  __syncthreads();
  for (int i = t; i < a.M * 128; i += 256) {       // ... and over the waves
    float v = grads[i];
#pragma unroll
    for (int w = 1; w < 4; ++w) v += grads[w * kRows * 128 + i];
    a.partials[(int64_t(blockIdx.y) * a.M + i / 128) * a.K + blockIdx.x * 128 + i % 128] = v;
  }
}

// Eight rows of eight values (16 bytes each) become eight fragments of the matrix instruction: of each column its eight rows' values.
__device__ __forceinline__ void columns_of(const U4 (&rows)[8], Bf16Products::Frag (&cols)[8]) {
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    uint32_t w[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const U4 &lo = rows[2 * p], &hi = rows[2 * p + 1];
      const uint32_t a = c < 2 ? lo.x : c < 4 ? lo.y : c < 6 ? lo.z : lo.w, b = c < 2 ? hi.x : c < 4 ? hi.y : c < 6 ? hi.z : hi.w;
      w[p] = __builtin_amdgcn_perm(b, a, c & 1 ? 0x07060302 : 0x05040100);
    }
    cols[c] = __builtin_bit_cast(Bf16Products::Frag, U4{w[0], w[1], w[2], w[3]});
  }
}

// The larger part of a value that is cut to bf16, and what that leaves over: as two operands of the matrix pipe they stand for 16 bits of the
// value and more (the rest is rounded to bf16, half a step of 2^-7 of it).  Of a value that bf16 holds the rest is 2^-24 of it instead of zero, and
// of an infinity an infinity, so that an infinite weight or activation meets two factors of one sign and not a zero.
__device__ __forceinline__ float rest_of(float v) {
  return copysignf(fmaxf(fabsf(v - __uint_as_float(__float_as_uint(v) & 0xffff0000u)), fabsf(v) * 0x1p-24f), v);
}
__device__ __forceinline__ uint2 cut_bf16(const float (&v)[4]) {
  auto upper = [](float lo, float hi) { return uint32_t(__builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302)); };
  return uint2{upper(v[0], v[1]), upper(v[2], v[3])};
}

// Up to 32 rows, on the matrix pipe, still one pass over the weights and their gradients with nothing laid out.  A workgroup takes 128 columns
// of K and `each` columns f in chunks of 128, whose dG and dU it forms in LDS, in two parts of bf16, by rows and by columns; each wave takes 32 of a chunk.  A
// lane brings 16 bytes of eight rows of W, whose columns in registers are what dX's product multiplies, and keeps the columns of X that the
// weights' gradients multiply.  Of 16 x 16 products c = 0 .. 7 row i stands for column 8 i + c of the 128, so that a lane's results are 32
// neighbours.  The waves' sums of dX meet in LDS, the workgroups' in the workspace.  Bound by memory as the kernel above: 16 rows of 13824 x 5120
// 160 us (240 by the products of more rows, with their layout), of 1920 x 3840 26.8 (35.6), 32 rows 170 (246) and 27.6 (39.2); eight rows by
// the kernel above took 163 and 33, here 160 and 25.9.  The parts' products and LDS are 1 us of the small ones and 5 of the large (rounded to bf16
// instead 156, 25.8, 165, 27.2, 155, 24.9).
template <int kTiles>
constexpr int kSomeGradLds = 8 * (16 * kTiles * 136 + 128 * 40);       // 57 and 74 KB: two workgroups to a CU

// kEarly: a chunk's weights are asked for ahead of the products of the chunk before, else behind those of dX, where their registers are free.  With
// two tiles of rows some registers are spilled for it, which pays in long walks only; us, 17 rows early / late: 456 x 1024 (one chunk) 12.7 /
// 11.7, 8192 x 1536 (two) 39.8 / 39.0, 13824 x 2048 (four) 67.2 / 64.3, 6912 x 5120 (five) 91.7 / 93.8, 13824 x 5120 (nine) 167 / 170.  With one
// nothing is spilled: 8 rows of 13824 x 2048 65.2 / 63.4, of 6912 x 5120 88 / 91, of 13824 x 5120 160 / 169.
constexpr int kEarlyFrom = 5 * 128;               // columns f of a workgroup

template <int kTiles, bool kEarly>
__global__ __launch_bounds__(256, 2) void gated_some_grad_kernel(GatedFewArgs a) {
  using Frag = Bf16Products::Frag;
  constexpr int kChunk = 128, kRows = 16 * kTiles, kPitch = kChunk + 8, kColPitch = 32 + 8, kSumPitch = 128 + 4;
  static_assert(kSomeGradLds<kTiles> == 2 * 2 * 2 * (kRows * kPitch + kChunk * kColPitch) && kSomeGradLds<kTiles> >= 4 * 16 * kSumPitch * 4,
                "the sums take the gradients' place");
  extern __shared__ __attribute__((aligned(16))) uint8_t some_lds[];
  uint16_t* const by_row = reinterpret_cast<uint16_t*>(some_lds);            // [dG | dU][cut | rest][row][f]
  uint16_t* const by_col = by_row + 2 * 2 * kRows * kPitch;             // [dG | dU][cut | rest][f][row]
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), l15 = lane & 15, grp = lane >> 4;
  const int k0 = blockIdx.x * 128, f0 = blockIdx.y * a.each, count = min(a.each, a.F - f0);
  Frag xt[8];
  U4 w[2][8];
  auto request = [&](int side, int chunk) {       // rows past the end re-read the last one; they become zeros (it may hold an infinity)
    const int64_t ld = side ? a.ldwu : a.ldwg;
    const uint8_t* const from = reinterpret_cast<const uint8_t*>((side ? a.wu : a.wg) + (f0 + chunk) * ld + k0);
    const uint32_t at = uint32_t(min(32 * wave + 8 * grp, a.F - 8 - f0 - chunk)) * uint32_t(2 * ld) + 16u * l15;      // (128 rows of 2^22 values are 2^30 bytes)
#pragma unroll
    for (int e = 0; e < 8; ++e) w[side][e] = *reinterpret_cast<const U4*>(from + 2 * e * ld + at);
  };
  {
    U4 x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 8 * grp + e < a.M ? *reinterpret_cast<const U4*>(a.x + int64_t(8 * grp + e) * a.ldx + k0 + 8 * l15) : U4{0, 0, 0, 0};
    if (a.partials) {
      request(0, 0);
      request(1, 0);
    }
    columns_of(x, xt);
  }
  f32x4 dx[8][kTiles];
#pragma unroll
  for (int c = 0; c < 8; ++c)
#pragma unroll
    for (int i = 0; i < kTiles; ++i) dx[c][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](int side, int chunk) {
    if (a.partials) {
      if (chunk + kChunk > count && 32 * wave + 8 * grp >= count - chunk) {       // (F and `each` are whole eights: a lane's rows exist or do not)
#pragma unroll
        for (int e = 0; e < 8; ++e) w[side][e] = U4{0, 0, 0, 0};
      }
      Frag wt[8];
      columns_of(w[side], wt);
      if (kEarly && chunk + kChunk < count) request(side, chunk + kChunk);
#pragma unroll
      for (int i = 0; i < 2 * kTiles; ++i) {
        const Frag d = *reinterpret_cast<const Frag*>(by_row + ((2 * side + i % 2) * kRows + 16 * (i / 2) + l15) * kPitch + 32 * wave + 8 * grp);
#pragma unroll
        for (int c = 0; c < 8; ++c) dx[c][i / 2] = Bf16Products::multiply(wt[c], d, dx[c][i / 2]);
      }
      if (!kEarly && chunk + kChunk < count) request(side, chunk + kChunk);
    }
    uint16_t* const dw = side ? a.dwu : a.dwg;
    if (!dw) return;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int in = 32 * wave + 16 * half + l15;
      __builtin_amdgcn_sched_barrier(0);          // (parts that run into each other need more registers than there are)
      const uint16_t* const from = by_col + (2 * side * kChunk + in) * kColPitch + 8 * grp;
      const Frag cut = *reinterpret_cast<const Frag*>(from), rest = *reinterpret_cast<const Frag*>(from + kChunk * kColPitch);
      f32x4 o[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) o[c] = Bf16Products::multiply(xt[c], cut, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
      for (int c = 0; c < 8; ++c) o[c] = Bf16Products::multiply(xt[c], rest, o[c]);
      if (chunk + in < count) {
        uint16_t* const to = dw + int64_t(f0 + chunk + in) * a.lddw + k0 + 32 * grp;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *reinterpret_cast<U4*>(to + 8 * r) = U4{pack_bf16(o[0][r], o[1][r]), pack_bf16(o[2][r], o[3][r]), pack_bf16(o[4][r], o[5][r]), pack_bf16(o[6][r], o[7][r])};
      }
    }
  };
  for (int chunk = 0; chunk < count; chunk += kChunk) {
    if (chunk > 0) __syncthreads();
    for (int i = t; i < 32 * (kChunk / 4); i += 256) {
      const int m = i % 32, f = i / 32 * 4, n = f0 + chunk + f;
      float dg[4] = {}, du[4] = {};
      if (m < a.M && chunk + f < count) {
        const int64_t at = saved_at(m, n, a.F);
        const f32x4 g = *reinterpret_cast<const f32x4*>(a.g + at), u = *reinterpret_cast<const f32x4*>(a.u + at);
        const uint2 dh2 = *reinterpret_cast<const uint2*>(a.dh + int64_t(m) * a.lddh + n);
        const float dh[4] = {bf16_lo(dh2.x), bf16_hi(dh2.x), bf16_lo(dh2.y), bf16_hi(dh2.y)};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float act, slope;
          activation(g[j], a.act0, a.act1, &act, &slope);
          dg[j] = dh[j] * u[j] * slope;
          du[j] = dh[j] * act;
        }
      }
#pragma unroll
      for (int side = 0; side < 2; ++side) {
        const float(&d)[4] = side ? du : dg;
        const uint2 part[2] = {cut_bf16(d), uint2{pack_bf16(rest_of(d[0]), rest_of(d[1])), pack_bf16(rest_of(d[2]), rest_of(d[3]))}};
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          if (m < kRows) *reinterpret_cast<uint2*>(by_row + ((2 * side + p) * kRows + m) * kPitch + f) = part[p];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            by_col[((2 * side + p) * kChunk + f + j) * kColPitch + m] = uint16_t((j & 2 ? part[p].y : part[p].x) >> (j & 1 ? 16 : 0));
        }
      }
    }
    __syncthreads();
    multiply(0, chunk);
    __builtin_amdgcn_sched_barrier(0);
    multiply(1, chunk);
  }
  if (!a.partials) return;
  float* const sums = reinterpret_cast<float*>(some_lds);               // [wave][row of 16][128]
#pragma unroll
  for (int i = 0; i < kTiles; ++i) {
    if (16 * i >= a.M) break;
    __syncthreads();
    float* const to = sums + (wave * 16 + l15) * kSumPitch + 32 * grp;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      *reinterpret_cast<f32x4*>(to + 8 * r) = f32x4{dx[0][i][r], dx[1][i][r], dx[2][i][r], dx[3][i][r]};
      *reinterpret_cast<f32x4*>(to + 8 * r + 4) = f32x4{dx[4][i][r], dx[5][i][r], dx[6][i][r], dx[7][i][r]};
    }
    __syncthreads();
    for (int j = t; j < 16 * 32; j += 256) {
      const int m = j / 32, k = j % 32 * 4;
      f32x4 v = *reinterpret_cast<const f32x4*>(sums + m * kSumPitch + k);
#pragma unroll
      for (int of = 1; of < 4; ++of) v += *reinterpret_cast<const f32x4*>(sums + (of * 16 + m) * kSumPitch + k);
      if (16 * i + m < a.M) *reinterpret_cast<f32x4*>(a.partials + (int64_t(blockIdx.y) * a.M + 16 * i + m) * a.K + k0 + k) = v;
    }
  }
}

// A product from the sums of its parts (N is a multiple of 128): four columns to a thread, each of a workgroup's waves has every fourth part.
__global__ __launch_bounds__(256) void gated_sum_kernel(const float* partials, int parts, int M, int N, uint16_t* y, int64_t ldy) {
  __shared__ f32x4 sums[3][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = (blockIdx.x * 64 + lane) * 4;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (i < M * N) {
#pragma unroll 8
    for (int p = wave; p < parts; p += 4) v += *reinterpret_cast<const f32x4*>(partials + int64_t(p) * M * N + i);
  }
  if (wave > 0) sums[wave - 1][lane] = v;
  __syncthreads();
  if (wave > 0 || i >= M * N) return;
#pragma unroll
  for (int s = 0; s < 3; ++s) v += sums[s][lane];
  *reinterpret_cast<uint2*>(y + int64_t(i / N) * ldy + i % N) = uint2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
}

constexpr int kFewGradMost = 512;                 // columns f of a workgroup of gated_few_grad_kernel

// columns f to a workgroup: enough workgroups to fill the chip, 64 to 512 columns; of more than kFewGradRows rows chunks of 128, two
// workgroups to a CU at most.  (Of an MI355X's 256 CUs, here and in walk_of: the workspace's size goes by it, which is asked for without a device.)
int few_grad_each(int64_t M, int32_t F, int32_t K) {
  if (M <= kFewGradRows) return int(std::clamp<int64_t>(int64_t(F) * (K / 128) / 1024 / 16 * 16, 64, kFewGradMost));
  const int64_t parts = std::max(512 / (K / 128), 1);
  return int((F + 128 * parts - 1) / (128 * parts) * 128);
}

int32_t sum_parts(const float* partials, int parts, int64_t M, int32_t N, void* y, int64_t ldy, void* stream) {
  hipLaunchKernelGGL(gated_sum_kernel, dim3(unsigned((M * N / 4 + 63) / 64)), dim3(256), 0, static_cast<hipStream_t>(stream), partials, parts, int(M), N,
                     static_cast<uint16_t*>(y), ldy);
  return finish_launch("gated_backward.hip");
}

int32_t launch_few_grad(GatedFewArgs a, void* dx, int64_t lddx, void* stream) {
  a.each = few_grad_each(a.M, a.F, a.K);
  const unsigned parts = unsigned((a.F + a.each - 1) / a.each);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 grid(unsigned(a.K / 128), parts);
  if (a.M > 16 && a.each >= kEarlyFrom)
    hipLaunchKernelGGL((gated_some_grad_kernel<2, true>), grid, dim3(256), kSomeGradLds<2>, s, a);
  else if (a.M > 16)
    hipLaunchKernelGGL((gated_some_grad_kernel<2, false>), grid, dim3(256), kSomeGradLds<2>, s, a);
  else if (a.M > kFewGradRows)
    hipLaunchKernelGGL((gated_some_grad_kernel<1, true>), grid, dim3(256), kSomeGradLds<1>, s, a);
  else
    hipLaunchKernelGGL(gated_few_grad_kernel, grid, dim3(256), unsigned(std::max(a.each * 2, 4 * 128) * kFewGradRows * 4), s, a);      // up to 16 KB of LDS
  if (const int32_t rc = finish_launch("gated_backward.hip"); rc != CA_OK || !dx) return rc;
  return sum_parts(a.partials, int(parts), a.M, a.K, dx, lddx, stream);
}

// How a product of M x N over `stages` of 64 is taken: whole by the linear map (parts 1), or in tiles of 64 x 64 with its walk in parts
struct Walk {
  int parts, stages;                              // of a part
};

// Of few tiles and a long walk the chip is filled by parts of it, whose sums a second launch adds up: the cheapest by the linear map's
// model and, for parts, by rounds of workgroups over the CUs, the second launch and the sums' way through the caches, in nanoseconds fitted
// to 36 products in up to 32 parts (the pick is 0.5 % behind the fastest in the geometric mean, 6 % at the worst).  Us of the backward pass of
// dX alone, whole / in parts: 17 x 7664 x 640 59.1 / 23.7, 300 x 4096 x 1536 44.5 / 36.3, 64 x 13824 x 5120 260 / 178, 500 x 1000 x 2048 20.9 / 25.7
// (whole); of the weights' 7776 x 128 x 640 35.8 / 24.0, 3325 x 168 x 2048 25.7 / 29.3 (whole).
Walk walk_of(int64_t M, int32_t N, int64_t stages) {
  constexpr int kCu = 256, kStage = 110, kTileEnd = 2900, kSecond = 7000, kValues = 156;       // kValues: of a part a nanosecond
  Walk best{1, int(stages)};
  if (M == 0 || M * N > (int64_t(1) << 26)) return best;
  int64_t least = gemm_bf16_cost(M, N, int32_t(64 * stages), kCu);
  const int64_t tiles = ((M + 63) / 64) * (N / 64);
  for (int64_t cut = 2; cut <= 32 && cut * 4 <= stages; ++cut) {
    const int64_t each = (stages + cut - 1) / cut, parts = (stages + each - 1) / each, rounds = (tiles * parts + kCu - 1) / kCu;
    const int64_t cost = rounds * (each * kStage + kTileEnd) + kSecond + parts * M * N / kValues;
    if (cost < least) {
      least = cost;
      best = Walk{int(parts), int(each)};
    }
  }
  return best;
}

size_t walk_bytes(int64_t M, int32_t N, int64_t stages) {
  const Walk w = walk_of(M, N, stages);
  return w.parts > 1 ? size_t(w.parts) * M * N * 4 : 0;
}

// y[M][N] = x w', rows of k = 64 stages
int32_t product(const uint16_t* x, const uint16_t* w, void* y, int64_t M, int32_t N, int64_t k, int64_t ldy, float* partials, void* stream) {
  const Walk walk = walk_of(M, N, k / 64);
  if (walk.parts == 1) return launch_gemm_bf16(x, w, y, M, N, int32_t(k), k, k, ldy, stream);
  OpArgs a{};
  a.x = x; a.w = w; a.g = partials;
  a.M = int32_t(M); a.N = N; a.K = int32_t(2 * k);
  a.ldx = a.ldw = a.K;
  a.k_values = walk.stages;
  const int32_t rc = enqueue_op_tile<Tile64Wide, PlainPart>(a, "gated_backward.hip", stream, unsigned(walk.parts));
  return rc != CA_OK ? rc : sum_parts(partials, walk.parts, M, N, y, ldy, stream);
}

}  // namespace

GatedWorkspace gated_workspace(int64_t M, int32_t F, int32_t K) {
  GatedWorkspace w{};
  w.Mp = M > 0 ? (M + 127) / 128 * 128 : 128;      // (of no rows the weights' gradients are zero)
  w.Fp = (int64_t(F) + 63) / 64 * 64;
  auto whole = [](int64_t elements) { return (size_t(elements) * 2 + 255) / 256 * 256; };
  if (M > 0 && M <= kSomeGradRows) {
    const int64_t each = few_grad_each(M, F, K);
    w.bytes = whole(2 * ((F + each - 1) / each) * M * K);
    return w;
  }
  w.rows = 0;
  w.cols = w.rows + whole(M * 2 * w.Fp);
  w.xt = w.cols + whole(2 * int64_t(F) * w.Mp);
  w.wt = w.xt + whole(K * w.Mp);
  w.parts = w.wt + whole(K * 2 * w.Fp);
  size_t parts = walk_bytes(M, K, 2 * w.Fp / 64);
  for (int64_t rows : {int64_t(F), 2 * int64_t(F)}) parts = std::max(parts, walk_bytes(rows, K, w.Mp / 64));      // dWg, dWu on their own or as one
  w.bytes = w.parts + parts;
  return w;
}

int32_t launch_gated_backward(const void* dh, const void* x, const void* w_gate, const void* w_up, const float* saved, int activation, void* dx,
                              void* dw_gate, void* dw_up, int64_t M, int32_t F, int32_t K, int64_t lddh, int64_t ldx, int64_t ldwg, int64_t ldwu,
                              int64_t lddx, int64_t lddw, void* workspace, void* stream) {
  const GatedWorkspace at = gated_workspace(M, F, K);
  const float* const saved_up = saved + gated_saved_values(M, F) / 2;
  float act0, act1;
  activation_factors(activation, &act0, &act1);
  // (one call of any size readies all of them for stream capture)
  const KernelLds kernels[] = {{reinterpret_cast<const void*>(gemm_op_kernel<Tile64Wide, PlainPart>), Tile64Wide::kLds},
                               {reinterpret_cast<const void*>(gated_some_grad_kernel<1, true>), kSomeGradLds<1>},
                               {reinterpret_cast<const void*>(gated_some_grad_kernel<2, false>), kSomeGradLds<2>},
                               {reinterpret_cast<const void*>(gated_some_grad_kernel<2, true>), kSomeGradLds<2>}};
  if (const int32_t rc = ensure_dynamic_lds(kernels, 4, kLdsGatedBackward); rc != CA_OK) return rc;
  if (const int32_t rc = gemm_tiles_ready(); rc != CA_OK) return rc;
  if (const int32_t rc = gemm_rows_ready(); rc != CA_OK) return rc;
  if (M > 0 && M <= kSomeGradRows) {
    const GatedFewArgs a{static_cast<const uint16_t*>(dh), static_cast<const uint16_t*>(x), static_cast<const uint16_t*>(w_gate),
                         static_cast<const uint16_t*>(w_up), saved, saved_up, static_cast<uint16_t*>(dw_gate), static_cast<uint16_t*>(dw_up),
                         dx ? static_cast<float*>(workspace) : nullptr, lddh, ldx, ldwg, ldwu, lddw, int32_t(M), F, K, 0, act0, act1};
    return launch_few_grad(a, dx, lddx, stream);
  }
  uint8_t* const ws = static_cast<uint8_t*>(workspace);
  uint16_t *const rows = reinterpret_cast<uint16_t*>(ws + at.rows), *const cols = reinterpret_cast<uint16_t*>(ws + at.cols);
  uint16_t *const xt = reinterpret_cast<uint16_t*>(ws + at.xt), *const wt = reinterpret_cast<uint16_t*>(ws + at.wt);
  const int32_t Mp = int32_t(at.Mp), Fp = int32_t(at.Fp);
  GatedLayoutArgs a{};
  a.grad = GatedGradArgs{static_cast<const uint16_t*>(dh), saved, saved_up, rows, cols, lddh, int32_t(M), F, Mp, Fp, act0, act1};
  // matrices of which nothing is asked have no workgroups
  a.t[0] = TransposeArgs{static_cast<const uint16_t*>(w_gate), wt, ldwg, 2 * at.Fp, F, K};
  a.t[1] = TransposeArgs{static_cast<const uint16_t*>(w_up), wt + at.Fp, ldwu, 2 * at.Fp, F, K};
  a.t[2] = TransposeArgs{static_cast<const uint16_t*>(x), xt, ldx, at.Mp, int32_t(M), K};
  const int64_t grad = int64_t(Fp / kSide) * (Mp / kSide), of_w = dx ? int64_t(K / kSide) * (Fp / kSide) : 0;
  const int64_t of_x = dw_gate || dw_up ? int64_t(K / kSide) * (Mp / kSide) : 0;
  if (grad + 2 * of_w + of_x >= (1 << 24)) return CA_EUNSUPPORTED;      // (a launch has fewer than 2^32 threads)
  a.grad_tiles = int32_t(grad);
  a.ends[0] = int32_t(grad + of_w);
  a.ends[1] = int32_t(grad + 2 * of_w);
  a.ends[2] = int32_t(grad + 2 * of_w + of_x);
  hipLaunchKernelGGL(gated_layout_kernel, dim3(unsigned(a.ends[2])), dim3(256), 0, static_cast<hipStream_t>(stream), a);
  if (const int32_t rc = finish_launch("gated_backward.hip"); rc != CA_OK) return rc;
  float* const partials = reinterpret_cast<float*>(ws + at.parts);
  if (dx)
    if (const int32_t rc = product(rows, wt, dx, M, K, 2 * at.Fp, lddx, partials, stream); rc != CA_OK) return rc;
  // the weights' gradients in one product where they follow one another
  const bool one = dw_gate && dw_up && static_cast<uint8_t*>(dw_up) == static_cast<uint8_t*>(dw_gate) + int64_t(F) * lddw * 2;
  for (int side = 0; side < (one ? 1 : 2); ++side) {
    void* const dw = side ? dw_up : dw_gate;
    if (!dw) continue;
    if (const int32_t rc = product(cols + side * int64_t(F) * at.Mp, xt, dw, int64_t(one ? 2 : 1) * F, K, at.Mp, lddw, partials, stream); rc != CA_OK) return rc;
  }
  return CA_OK;
}

}  // namespace ca

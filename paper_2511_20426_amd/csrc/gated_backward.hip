// The gradients of the gated projections H = act(G) * U, G = X Wg', U = X Wu' (F columns, rows of K):
//
//   dG = dH U act'(G),  dU = dH act(G);  dX = dG Wg + dU Wu,  dWg = dG' X,  dWu = dU' X
//
// The products are the framework's own linear map, which multiplies rows by rows: one launch forms dG and dU from dH and the saved
// projections, in rows (side by side, [M][2 Fp], for dX) and transposed ([2 F][Mp], for dW), and lays out X' [K][Mp] and [Wg; Wu]' [K][2 Fp]
// in the workspace.  Fp and Mp are F and M filled up with zeros to whole steps of the products (2 Fp and Mp are multiples of 128).  dG
// and dU are rounded to bf16, the type that the matrix products take: with the result's own rounding gradients are 2.3e-3 of their norm
// off, 1.7e-3 of which is that of the result.  (With G and U saved in bf16 as well it was 3.1e-3: they are saved in fp32.)  dX is one
// product over both, so that their sum is not rounded in between.
//
// Of up to 8 rows all of it is one pass over the weights, read once, and their gradients, written once, with nothing laid out
// (gated_few_grad_kernel).
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

// Few rows: both weights read and their gradients written once are what counts (one row of 13824 x 5120 130 us, 566 MB; of 4096 x 1536 18.6 us,
// eight 24.2; by the products of more rows nine take 32.9, and sixteen taken here, with 256 registers, took 57.6).  A workgroup takes 128 columns of K and `each` columns f of the projections: sixteen threads eight columns of K each, and
// sixteen such rows of threads every sixteenth f.  dG and dU of the f are formed in LDS, in fp32; of each f a thread reads its part of Wg and
// Wu, adds to its sums of dX, and forms and writes its part of dWg and dWu from X's rows, which it keeps.  The sums of dX of a
// workgroup's f go to the workspace; a second launch adds them up in order.
struct GatedFewArgs {
  const uint16_t *dh, *x, *wg, *wu;
  const float *g, *u;
  uint16_t *dwg, *dwu;                            // null: not asked for
  float* partials;                                // [parts of f][M][K], or null: dX is not asked for
  int64_t lddh, ldx, ldwg, ldwu, lddw;
  int32_t M, F, K, each;
  float act0, act1;
};

template <int kRows>
__global__ __launch_bounds__(256) void gated_few_grad_kernel(GatedFewArgs a) {
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

// A product from the sums of its parts, four columns to a thread (N is a multiple of 128)
__global__ __launch_bounds__(256) void gated_sum_kernel(const float* partials, int parts, int M, int N, uint16_t* y, int64_t ldy) {
  const int i = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= M * N) return;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int p = 0; p < parts; ++p) v += *reinterpret_cast<const f32x4*>(partials + int64_t(p) * M * N + i);
  *reinterpret_cast<uint2*>(y + int64_t(i / N) * ldy + i % N) = uint2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
}

constexpr int kFewGradRows = 8, kFewGradMost = 512;       // rows; columns f of a workgroup

// columns f to a workgroup: enough workgroups to fill the chip, 64 to 512 columns
int few_grad_each(int32_t F, int32_t K) {
  const int64_t each = int64_t(F) * (K / 128) / 1024 / 16 * 16;
  return int(each < 64 ? 64 : (each > kFewGradMost ? kFewGradMost : each));
}

int32_t sum_parts(const float* partials, int parts, int64_t M, int32_t N, void* y, int64_t ldy, void* stream) {
  hipLaunchKernelGGL(gated_sum_kernel, dim3(unsigned((M * N / 4 + 255) / 256)), dim3(256), 0, static_cast<hipStream_t>(stream), partials, parts, int(M), N,
                     static_cast<uint16_t*>(y), ldy);
  return finish_launch("gated_backward.hip");
}

int32_t launch_few_grad(GatedFewArgs a, void* dx, int64_t lddx, void* stream) {
  a.each = few_grad_each(a.F, a.K);
  const unsigned parts = unsigned((a.F + a.each - 1) / a.each);
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto bytes = [&](int rows) { return unsigned(std::max(a.each * 2, 4 * 128) * rows * 4); };        // up to 32 KB
  const dim3 grid(unsigned(a.K / 128), parts);
  if (a.M <= 4)
    hipLaunchKernelGGL(gated_few_grad_kernel<4>, grid, dim3(256), bytes(4), s, a);
  else
    hipLaunchKernelGGL(gated_few_grad_kernel<8>, grid, dim3(256), bytes(8), s, a);
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
  if (M > 0 && M <= kFewGradRows) {
    const int64_t each = few_grad_each(F, K);
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
  const KernelLds kernel[] = {{reinterpret_cast<const void*>(gemm_op_kernel<Tile64Wide, PlainPart>), Tile64Wide::kLds}};
  if (const int32_t rc = ensure_dynamic_lds(kernel, 1, kLdsGatedBackward); rc != CA_OK) return rc;
  if (const int32_t rc = gemm_tiles_ready(); rc != CA_OK) return rc;
  if (const int32_t rc = gemm_rows_ready(); rc != CA_OK) return rc;
  if (M > 0 && M <= kFewGradRows) {
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

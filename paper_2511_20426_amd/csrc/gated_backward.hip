// The gradients of the gated projections H = act(G) * U, G = X Wg', U = X Wu' (F columns, rows of K):
//
//   dG = dH U act'(G),  dU = dH act(G);  dX = dG Wg + dU Wu,  dWg = dG' X,  dWu = dU' X
//
// The products are the framework's own linear map, which multiplies rows by rows: one launch forms dG and dU from dH and the saved
// projections and writes them in rows (side by side, [M][2 Fp], for dX) and transposed ([2 F][Mp], for dW), others lay out X' [K][Mp]
// and [Wg; Wu]' [K][2 Fp] in the workspace.  Fp and Mp are F and M filled up with zeros to whole steps of the products (2 Fp and Mp
// are multiples of 128).  dG and dU are rounded to bf16, the type that the matrix products take: with the result's own rounding
// gradients are 2.3e-3 of their norm off, 1.7e-3 of which is that of the result.  (With G and U saved in bf16 as well it was 3.1e-3:
// they are saved in fp32.)  dX is one product over both, so that their sum is not rounded in between.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "ca_internal.hpp"

namespace ca {
namespace {

#include "rope_device.hpp"
#include "gemm_tiles.hpp"
#include "gemm_tile_kernel.hpp"
#include "gemm_ops.hpp"

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

struct TransposeArgs {
  const uint16_t* x[2];                           // grid.z picks one: [rows][ldx]
  uint16_t* y[2];                                 // [cols][ldy], columns rows .. rows_padded are zero
  int64_t ldx[2], ldy;
  int32_t rows, cols, rows_padded;
};

__global__ __launch_bounds__(256) void transpose_kernel(TransposeArgs a) {
  __shared__ uint32_t tile[kSide * kRow];
  const int t = threadIdx.x, chunk = t & 7;
  const int c0 = blockIdx.x * kSide, r0 = blockIdx.y * kSide;
  const uint16_t* x = a.x[blockIdx.z];
  const int64_t ldx = a.ldx[blockIdx.z];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = (t >> 3) + 32 * i;
    U4 v = {0, 0, 0, 0};
    if (r0 + row < a.rows && c0 + chunk * 8 < a.cols) v = load_once(x + int64_t(r0 + row) * ldx + c0 + chunk * 8);
    put_chunk(tile, row, chunk, v);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int col = (t >> 3) + 32 * i;
    if (c0 + col < a.cols && r0 + chunk * 8 < a.rows_padded)
      *reinterpret_cast<U4*>(a.y[blockIdx.z] + int64_t(c0 + col) * a.ldy + r0 + chunk * 8) = column_chunk(tile, col, chunk);
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

__global__ __launch_bounds__(256) void gated_grad_kernel(GatedGradArgs a) {
  __shared__ uint32_t tile[2][kSide * kRow];
  const int t = threadIdx.x, chunk = t & 7;
  const int f0 = blockIdx.x * kSide, m0 = blockIdx.y * kSide;
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
        // act' = s + g s (1 - s) p'(g), p = g (act0 + act1 g^2)
        float p;
        const float s = act_sigmoid(g[j], a.act0, a.act1, &p);
        const float c = __builtin_amdgcn_fmed3f(g[j], -1e4f, 1e4f);
        const float slope = fmaf(c * c, 3.f * a.act1, a.act0);
        v[j] = dh.v[j] * u[j] * fmaf(c * s * (1.f - s), slope, s);
        w[j] = dh.v[j] * (g[j] * s);
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
    if (f0 + col >= a.F || m >= a.Mp) continue;
    uint16_t* to = a.cols + int64_t(f0 + col) * a.Mp + m;
    *reinterpret_cast<U4*>(to) = column_chunk(tile[0], col, chunk);
    *reinterpret_cast<U4*>(to + int64_t(a.F) * a.Mp) = column_chunk(tile[1], col, chunk);
  }
}

int32_t transpose(const TransposeArgs& a, int n, void* stream) {
  const dim3 grid(unsigned((a.cols + kSide - 1) / kSide), unsigned(a.rows_padded / kSide), unsigned(n));
  if (grid.y > 65535) return CA_EUNSUPPORTED;
  hipLaunchKernelGGL(transpose_kernel, grid, dim3(256), 0, static_cast<hipStream_t>(stream), a);
  return finish_launch("gated_backward.hip");
}

}  // namespace

GatedWorkspace gated_workspace(int64_t M, int32_t F, int32_t K) {
  GatedWorkspace w;
  w.Mp = M > 0 ? (M + 127) / 128 * 128 : 128;      // (of no rows the weights' gradients are zero)
  w.Fp = (int64_t(F) + 63) / 64 * 64;
  auto whole = [](int64_t elements) { return (size_t(elements) * 2 + 255) / 256 * 256; };
  w.rows = 0;
  w.cols = w.rows + whole(M * 2 * w.Fp);
  w.xt = w.cols + whole(2 * int64_t(F) * w.Mp);
  w.wt = w.xt + whole(K * w.Mp);
  w.bytes = w.wt + whole(K * 2 * w.Fp);
  return w;
}

int32_t launch_gated_backward(const void* dh, const void* x, const void* w_gate, const void* w_up, const float* saved, int activation,
                              void* dx, void* dw_gate, void* dw_up, int64_t M, int32_t F, int32_t K, int64_t lddh, int64_t ldx, int64_t ldwg,
                              int64_t ldwu, int64_t lddx, int64_t lddw, void* workspace, void* stream) {
  const GatedWorkspace at = gated_workspace(M, F, K);
  uint8_t* const ws = static_cast<uint8_t*>(workspace);
  uint16_t *const rows = reinterpret_cast<uint16_t*>(ws + at.rows), *const cols = reinterpret_cast<uint16_t*>(ws + at.cols);
  uint16_t *const xt = reinterpret_cast<uint16_t*>(ws + at.xt), *const wt = reinterpret_cast<uint16_t*>(ws + at.wt);
  GatedGradArgs a{static_cast<const uint16_t*>(dh), saved, saved + gated_saved_values(M, F) / 2, rows, cols, lddh, int32_t(M), F, int32_t(at.Mp), int32_t(at.Fp), 0.f, 0.f};
  activation_factors(activation, &a.act0, &a.act1);
  const dim3 grid(unsigned(at.Fp / kSide), unsigned(at.Mp / kSide));
  hipLaunchKernelGGL(gated_grad_kernel, grid, dim3(256), 0, static_cast<hipStream_t>(stream), a);
  if (const int32_t rc = finish_launch("gated_backward.hip"); rc != CA_OK) return rc;
  if (dx) {
    const TransposeArgs t{{static_cast<const uint16_t*>(w_gate), static_cast<const uint16_t*>(w_up)}, {wt, wt + at.Fp}, {ldwg, ldwu}, 2 * at.Fp,
                          F, K, int32_t(at.Fp)};
    if (const int32_t rc = transpose(t, 2, stream); rc != CA_OK) return rc;
    if (const int32_t rc = launch_gemm_bf16(rows, wt, dx, M, K, int32_t(2 * at.Fp), 2 * at.Fp, 2 * at.Fp, lddx, stream); rc != CA_OK) return rc;
  }
  if (!dw_gate && !dw_up) return CA_OK;
  const TransposeArgs t{{static_cast<const uint16_t*>(x), nullptr}, {xt, nullptr}, {ldx, 0}, at.Mp, int32_t(M), K, int32_t(at.Mp)};
  if (const int32_t rc = transpose(t, 1, stream); rc != CA_OK) return rc;
  // both in one product where they follow one another
  const int32_t both = dw_gate && dw_up && static_cast<uint8_t*>(dw_up) == static_cast<uint8_t*>(dw_gate) + int64_t(F) * lddw * 2 ? 2 : 1;
  for (int side = 0; side < 2; side += both) {
    void* const dw = side ? dw_up : dw_gate;
    if (!dw) continue;
    if (const int32_t rc = launch_gemm_bf16(cols + side * int64_t(F) * at.Mp, xt, dw, int64_t(both) * F, K, int32_t(at.Mp), at.Mp, at.Mp, lddw, stream);
        rc != CA_OK)
      return rc;
  }
  return CA_OK;
}

}  // namespace ca

// The 8-bit linear map and the gated projections for few tokens (single tokens when serving): the weights' way from memory is all
// there is.  A workgroup of eight waves takes 16 columns of the result, and its waves share k: each brings 128 bytes of 16 rows of W
// at a time straight from memory into the registers that the MFMA multiplies from (no LDS: nothing is used twice), several such
// pieces ahead, with X's rows from L2.  The waves' sums meet in LDS, in order.
// (Included behind gemm_ops.hpp.)
#pragma once

constexpr int kFewWaves = 8;

// kTiles: tiles of 16 tokens
template <typename Op, int kTiles>
__global__ __launch_bounds__(64 * kFewWaves) void gemm_few_kernel(OpArgs a) {
  constexpr int kSides = Op::kGated ? 2 : 1, kAhead = kTiles == 1 ? 4 : 2;
  using Products = typename Op::Products;
  using Frag = typename Products::Frag;
  using Sums = typename Products::Sums;
  __shared__ Sums part[kFewWaves][kSides][kTiles][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l15 = lane & 15, grp = lane >> 4;
  const int n0 = blockIdx.x * 16, row = min(n0 + l15, a.N - 1);          // rows past the end re-read the last one
  const uint8_t* w[kSides];
  w[0] = static_cast<const uint8_t*>(a.w) + int64_t(row) * a.ldw + grp * 16;
  if constexpr (Op::kGated) w[1] = static_cast<const uint8_t*>(a.w2) + int64_t(row) * a.ldw2 + grp * 16;
  const uint8_t* x[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) x[t] = static_cast<const uint8_t*>(a.x) + int64_t(min(16 * t + l15, a.M - 1)) * a.ldx + grp * 16;
  Sums acc[kSides][kTiles];
#pragma unroll
  for (int s = 0; s < kSides; ++s)
#pragma unroll
    for (int t = 0; t < kTiles; ++t) acc[s][t] = Sums{0, 0, 0, 0};
  auto pieces = [&](auto count, int first) {
    constexpr int n = decltype(count)::value;
    Frag fw[n][kSides][2], fx[n][kTiles][2];
#pragma unroll
    for (int i = 0; i < n; ++i)
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        const int64_t at = int64_t(first + i * kFewWaves) * 128 + kk * 64;
#pragma unroll
        for (int s = 0; s < kSides; ++s) fw[i][s][kk] = __builtin_nontemporal_load(reinterpret_cast<const Frag*>(w[s] + at));
#pragma unroll
        for (int t = 0; t < kTiles; ++t) fx[i][t][kk] = *reinterpret_cast<const Frag*>(x[t] + at);
      }
#pragma unroll
    for (int i = 0; i < n; ++i)
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int s = 0; s < kSides; ++s)
#pragma unroll
          for (int t = 0; t < kTiles; ++t) acc[s][t] = Products::multiply(fw[i][s][kk], fx[i][t][kk], acc[s][t]);
  };
  const int units = a.K / 128;
  int u = wave;
  for (; u + (kAhead - 1) * kFewWaves < units; u += kAhead * kFewWaves) pieces(std::integral_constant<int, kAhead>{}, u);
  for (; u < units; u += kFewWaves) pieces(std::integral_constant<int, 1>{}, u);
#pragma unroll
  for (int s = 0; s < kSides; ++s)
#pragma unroll
    for (int t = 0; t < kTiles; ++t) part[wave][s][t][lane] = acc[s][t];
  __syncthreads();
  if (wave >= kTiles) return;
  Sums sum[kSides];
#pragma unroll
  for (int s = 0; s < kSides; ++s) {
    sum[s] = part[0][s][wave][lane];
#pragma unroll
    for (int i = 1; i < kFewWaves; ++i) sum[s] += part[i][s][wave][lane];
  }
  // a lane has columns 4 grp .. +3 of token l15
  const int m = 16 * wave + l15, n = n0 + 4 * grp;
  if (m >= a.M || n >= a.N) return;
  auto leave = [&](void* y, int64_t ld, float v0, float v1, float v2, float v3) {
    uint2 out = {pack_bf16(v0, v1), pack_bf16(v2, v3)};
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(y) + int64_t(m) * ld + n) = out;
  };
  if constexpr (Op::kGated) {
    const Sums &g = sum[0], &v = sum[1];
    leave(a.y, a.ldy, gated_value(g[0], v[0], a.act0, a.act1), gated_value(g[1], v[1], a.act0, a.act1),
          gated_value(g[2], v[2], a.act0, a.act1), gated_value(g[3], v[3], a.act0, a.act1));
    if (a.g) {
      leave(a.g, a.ld_saved, g[0], g[1], g[2], g[3]);
      leave(a.u, a.ld_saved, v[0], v[1], v[2], v[3]);
    }
  } else {
    const float xs = a.xs[m], *ws = static_cast<const float*>(a.w2) + n;
    leave(a.y, a.ldy, scaled(sum[0][0], xs, ws[0]), scaled(sum[0][1], xs, ws[1]), scaled(sum[0][2], xs, ws[2]), scaled(sum[0][3], xs, ws[3]));
  }
}

template <typename Op>
int32_t enqueue_few(const OpArgs& a, const char* what, void* stream) {
  const dim3 grid(unsigned((a.N + 15) / 16)), block(64 * kFewWaves);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (a.M <= 16)
    hipLaunchKernelGGL((gemm_few_kernel<Op, 1>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((gemm_few_kernel<Op, 2>), grid, block, 0, s, a);
  return finish_launch(what);
}

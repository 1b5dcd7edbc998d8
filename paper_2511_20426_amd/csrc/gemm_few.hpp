// The 8-bit linear map and the gated projections for few tokens (single tokens when serving): the weights' way from memory is all
// there is.  A workgroup takes 16 columns of the result, and its waves share k: each brings 128 bytes of 16 rows of W at a time
// straight from memory into the registers that the MFMA multiplies from (no LDS: nothing is used twice), kAhead such pieces on their
// way while one is multiplied, with X's rows from L2 (lanes of rows that do not exist ask for nothing: a row asked for by all sixteen
// costs as much of the way from L2 as W does).  The waves' sums meet in LDS, in order.
//
// Of up to four tokens in bf16 the 8-bit codes are made here (kCodes): every workgroup makes them for itself, while its first pieces
// of W are on their way, instead of a launch of its own ahead of this one.
// (Included behind quantize_device.hpp and gemm_ops.hpp.)
#pragma once

constexpr int kFewWaves = 4, kFewAhead = 4;
constexpr int kCodeRows = 4, kCodeHeld = 3, kCodeK = 8 * 64 * kFewWaves * kCodeHeld;       // tokens and k that fit; vectors of a thread

// kTiles: tiles of 16 tokens.  kCodes: a.x is bf16 [M][ldx bytes], M up to kCodeRows, K values up to kCodeK, 16-byte aligned rows.
template <typename Op, int kTiles, bool kCodes>
__global__ __launch_bounds__(64 * kFewWaves) void gemm_few_kernel(OpArgs a) {
  constexpr int kSides = Op::kGated ? 2 : 1, kAhead = kFewAhead, kWaves = kFewWaves;
  using Products = typename Op::Products;
  using Frag = typename Products::Frag;
  using Sums = typename Products::Sums;
  __shared__ Sums part[kWaves][kSides][kTiles][64];
  __shared__ __attribute__((aligned(16))) uint8_t codes[kCodes ? kCodeRows : 1][kCodes ? kCodeK + 16 : 16];
  __shared__ uint32_t most_of[kCodeRows][kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l15 = lane & 15, grp = lane >> 4;
  const int n0 = blockIdx.x * 16, row = min(n0 + l15, a.N - 1);          // rows past the end re-read the last one
  const uint8_t* w[kSides];
  w[0] = static_cast<const uint8_t*>(a.w) + int64_t(row) * a.ldw + grp * 16;
  if constexpr (Op::kGated) w[1] = static_cast<const uint8_t*>(a.w2) + int64_t(row) * a.ldw2 + grp * 16;
  U4 held[kCodes ? kCodeRows : 1][kCodeHeld];
  const int vectors = a.k_values / 8;                                   // of a row
  if constexpr (kCodes) {
#pragma unroll
    for (int r = 0; r < kCodeRows; ++r)
#pragma unroll
      for (int v = 0; v < kCodeHeld; ++v) {
        const int at = int(threadIdx.x) + v * 64 * kWaves;
        held[r][v] = U4{0, 0, 0, 0};
        if (r < a.M && at < vectors) held[r][v] = *reinterpret_cast<const U4*>(static_cast<const uint8_t*>(a.x) + int64_t(r) * a.ldx + at * 16);
      }
  }
  const uint8_t* x[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) x[t] = static_cast<const uint8_t*>(a.x) + int64_t(min(16 * t + l15, a.M - 1)) * a.ldx + grp * 16;
  Sums acc[kSides][kTiles];
#pragma unroll
  for (int s = 0; s < kSides; ++s)
#pragma unroll
    for (int t = 0; t < kTiles; ++t) acc[s][t] = Sums{0, 0, 0, 0};
  // piece i of the wave is number wave + i kWaves of the row's
  const int pieces = (a.K / 128 - wave + kWaves - 1) / kWaves;
  Frag fw[kAhead][kSides][2], fx[kAhead][kTiles][2] = {};
  auto request = [&](int slot, int i) {
    const int64_t at = int64_t(wave + i * kWaves) * 128;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
      for (int s = 0; s < kSides; ++s) fw[slot][s][kk] = *reinterpret_cast<const Frag*>(w[s] + at + kk * 64);
    }
    if constexpr (kCodes) return;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
      if (16 * t + l15 < a.M) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) fx[slot][t][kk] = *reinterpret_cast<const Frag*>(x[t] + at + kk * 64);
      }
  };
  auto multiply = [&](int slot, int i) {
    if constexpr (kCodes) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
        fx[slot][0][kk] = *reinterpret_cast<const Frag*>(codes[min(l15, a.M - 1)] + (wave + i * kWaves) * 128 + kk * 64 + grp * 16);
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int s = 0; s < kSides; ++s)
#pragma unroll
        for (int t = 0; t < kTiles; ++t) acc[s][t] = Products::multiply(fw[slot][s][kk], fx[slot][t][kk], acc[s][t]);
  };
  const bool deep = pieces >= kAhead;
  if (deep) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) request(j, j);
  }
  if constexpr (kCodes) {
    uint32_t most[kCodeRows] = {};
#pragma unroll
    for (int r = 0; r < kCodeRows; ++r) {
      if (r >= a.M) break;
      most[r] = 0;
#pragma unroll
      for (int v = 0; v < kCodeHeld; ++v)
#pragma unroll
        for (uint32_t two : {held[r][v].x, held[r][v].y, held[r][v].z, held[r][v].w})
          most[r] = max(most[r], max(two << 16 & 0x7fff0000u, two & 0x7fff0000u));
#pragma unroll
      for (int d = 1; d < 64; d *= 2) most[r] = max(most[r], uint32_t(__shfl_xor(int(most[r]), d, 64)));
      if (lane == 0) most_of[r][wave] = most[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kCodeRows; ++r) {
      if (r >= a.M) break;
      const RowScale of(max(max(most_of[r][0], most_of[r][1]), max(most_of[r][2], most_of[r][3])));
#pragma unroll
      for (int v = 0; v < kCodeHeld; ++v) {
        const int at = int(threadIdx.x) + v * 64 * kWaves;
        if (at < a.K / 8) *reinterpret_cast<uint2*>(codes[r] + at * 8) = row_codes(of, held[r][v]);
      }
    }
    __syncthreads();
  }
  int i = 0;
  if (deep) {
    for (; i + 2 * kAhead <= pieces; i += kAhead)
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        multiply(j, i + j);
        request(j, i + j + kAhead);
      }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) multiply(j, i + j);
    i += kAhead;
  }
#pragma unroll
  for (int j = 0; j < kAhead - 1; ++j)
    if (i + j < pieces) request(j, i + j);
#pragma unroll
  for (int j = 0; j < kAhead - 1; ++j)
    if (i + j < pieces) multiply(j, i + j);
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
    for (int i = 1; i < kWaves; ++i) sum[s] += part[i][s][wave][lane];
  }
  // a lane has columns 4 grp .. +3 of token l15
  const int m = 16 * wave + l15, n = n0 + 4 * grp;
  if (m >= a.M || n >= a.N) return;
  auto leave = [&](float v0, float v1, float v2, float v3) {
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.y) + int64_t(m) * a.ldy + n) = uint2{pack_bf16(v0, v1), pack_bf16(v2, v3)};
  };
  if constexpr (Op::kGated) {
    const Sums &g = sum[0], &v = sum[1];
    leave(gated_value(g[0], v[0], a.act0, a.act1), gated_value(g[1], v[1], a.act0, a.act1),
          gated_value(g[2], v[2], a.act0, a.act1), gated_value(g[3], v[3], a.act0, a.act1));
    if (a.g) {
      const int64_t at = saved_at(m, n, a.N);
      *reinterpret_cast<Sums*>(a.g + at) = g;
      *reinterpret_cast<Sums*>(a.u + at) = v;
    }
  } else {
    float xs;
    if constexpr (kCodes)
      xs = row_scale(max(max(most_of[m][0], most_of[m][1]), max(most_of[m][2], most_of[m][3])));
    else
      xs = a.xs[m];
    const float* ws = static_cast<const float*>(a.w2) + n;
    leave(scaled(sum[0][0], xs, ws[0]), scaled(sum[0][1], xs, ws[1]), scaled(sum[0][2], xs, ws[2]), scaled(sum[0][3], xs, ws[3]));
  }
}

template <typename Op>
int32_t enqueue_few(const OpArgs& a, const char* what, void* stream) {
  const unsigned groups = unsigned((a.N + 15) / 16);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (a.M <= 16)
    hipLaunchKernelGGL((gemm_few_kernel<Op, 1, false>), dim3(groups), dim3(64 * kFewWaves), 0, s, a);
  else
    hipLaunchKernelGGL((gemm_few_kernel<Op, 2, false>), dim3(groups), dim3(64 * kFewWaves), 0, s, a);
  return finish_launch(what);
}

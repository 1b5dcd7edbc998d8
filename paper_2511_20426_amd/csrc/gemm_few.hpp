// The 8-bit linear map and the gated projections for few tokens (single tokens when serving): the weights' way from memory is all
// there is.  A workgroup takes 16 columns of the result, and its waves share k: each brings 128 bytes of 16 rows of W at a time
// straight from memory into the registers that the MFMA multiplies from (no LDS: nothing is used twice), kAhead such pieces on their
// way while one is multiplied, with X's rows from L2 (lanes of rows that do not exist ask for nothing: a row asked for by all sixteen
// costs as much of the way from L2 as W does).  The waves' sums meet in LDS, in order.
//
// The 8-bit codes of tokens in bf16 can be made here (Codes): every workgroup makes them for itself, while its first pieces of W are on
// their way, instead of a launch of its own ahead of this one.  All threads take a token's values together, or each wave a token.
// (Included behind quantize_device.hpp and gemm_ops.hpp.)
#pragma once

constexpr int kFewWaves = 4, kFewAhead = 4;

// The codes that a launch makes: of kThread tokens at a time a thread has kHeld vectors of eight values each; kWaves waves share a token.
template <int kThread, int kHeldOf, int kWavesOf>
struct Codes {
  static constexpr int kRows = kThread, kHeld = kHeldOf, kWaves = kWavesOf;
  static constexpr int kTokens = kRows * kFewWaves / kWaves, kMost = 8 * 64 * kHeld * kWaves;      // tokens, and values of each
};
using NoCodes = Codes<0, 0, 1>;
using CodesOne = Codes<1, 3, kFewWaves>;          // one token of up to 6144, by all waves
using CodesTwo = Codes<2, 3, kFewWaves>;          // two
using CodesFour = Codes<4, 3, kFewWaves>;         // four
using CodesFourShort = Codes<1, 3, 1>;            // four of up to 1536, each by a wave
using CodesTwelve = Codes<3, 3, 1>;               // twelve (rows that are not there are read as the last one)

// Values 8 v .. +7 of a row of k >= 8 in bf16, of any alignment: the load of eight that lie in the row, and of them, once they are
// there, the ones meant, zeros behind the row's end.  (A branch for the row's end would wait for its loads.)
__device__ __forceinline__ U4 load_eight(const uint16_t* row, int v, int k) {
  struct __attribute__((packed, aligned(2))) Eight { uint32_t w[4]; };
  const Eight e = *reinterpret_cast<const Eight*>(row + min(8 * v, k - 8));
  return U4{e.w[0], e.w[1], e.w[2], e.w[3]};
}
__device__ __forceinline__ U4 eight_of(const U4& e, int v, int k) {
  const int past = max(8 * v - (k - 8), 0);
  uint64_t lo = e.x | uint64_t(e.y) << 32, hi = e.z | uint64_t(e.w) << 32;
  if (k % 8 != 0) {
    const int bits = 16 * (past & 3);
    lo = past & 4 ? hi : lo;
    hi = past & 4 ? 0 : hi;
    lo = lo >> bits | (hi << 1) << (63 - bits);
    hi >>= bits;
  }
  if (past >= 8) lo = hi = 0;
  return U4{uint32_t(lo), uint32_t(lo >> 32), uint32_t(hi), uint32_t(hi >> 32)};
}

// kTiles: tiles of 16 tokens.  With codes a.x is bf16 [M][ldx bytes], a.k_values (8 or more) to a row, no more of both than Code has.
template <typename Op, int kTiles, typename Code>
__global__ __launch_bounds__(64 * kFewWaves) void gemm_few_kernel(OpArgs a) {
  constexpr int kSides = Op::kGated ? 2 : 1, kAhead = kFewAhead, kWaves = kFewWaves;
  using Products = typename Op::Products;
  using Frag = typename Products::Frag;
  using Sums = typename Products::Sums;
  __shared__ Sums part[kWaves][kSides][kTiles][64];
  constexpr bool kCodes = Code::kRows > 0;
  __shared__ __attribute__((aligned(16))) uint8_t codes[kCodes ? Code::kTokens : 1][Code::kMost + 16];
  __shared__ uint32_t most_of[kCodes ? Code::kTokens : 1][Code::kWaves];
  // (a scalar, so that what goes by it is branched around: an MFMA runs whatever the mask of lanes is)
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l15 = lane & 15, grp = lane >> 4;
  const int n0 = blockIdx.x * 16, row = min(n0 + l15, a.N - 1);          // rows past the end re-read the last one
  const uint8_t* w[kSides];
  w[0] = static_cast<const uint8_t*>(a.w) + int64_t(row) * a.ldw + grp * 16;
  if constexpr (Op::kGated) w[1] = static_cast<const uint8_t*>(a.w2) + int64_t(row) * a.ldw2 + grp * 16;
  U4 held[kCodes ? Code::kRows : 1][kCodes ? Code::kHeld : 1];
  constexpr int kEach = kWaves / Code::kWaves;                          // tokens that the workgroup takes at a time
  auto code_row = [&](int r) { return wave / Code::kWaves + r * kEach; };
  auto code_vector = [&](int v) { return wave % Code::kWaves * 64 + lane + v * 64 * Code::kWaves; };
  if constexpr (kCodes) {
#pragma unroll
    for (int r = 0; r < Code::kRows; ++r)
#pragma unroll
      for (int v = 0; v < Code::kHeld; ++v)
        held[r][v] = load_eight(reinterpret_cast<const uint16_t*>(static_cast<const uint8_t*>(a.x) + int64_t(min(code_row(r), a.M - 1)) * a.ldx), code_vector(v),
                                a.k_values);
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
  const int all = a.K / 128, pieces = (all - wave + kWaves - 1) / kWaves;
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
  auto make_codes = [&]() {
    if constexpr (!kCodes) return;
    uint32_t most[kCodes ? Code::kRows : 1] = {};
#pragma unroll
    for (int r = 0; r < Code::kRows; ++r) {
      if (code_row(r) >= a.M) break;
#pragma unroll
      for (int v = 0; v < Code::kHeld; ++v) {
        held[r][v] = eight_of(held[r][v], code_vector(v), a.k_values);
#pragma unroll
        for (uint32_t two : {held[r][v].x, held[r][v].y, held[r][v].z, held[r][v].w})
          most[r] = max(most[r], max(two << 16 & 0x7fff0000u, two & 0x7fff0000u));
      }
#pragma unroll
      for (int d = 1; d < 64; d *= 2) most[r] = max(most[r], uint32_t(__shfl_xor(int(most[r]), d, 64)));
      if (lane == 0) most_of[code_row(r)][wave % Code::kWaves] = most[r];
    }
    if constexpr (Code::kWaves > 1) __syncthreads();
#pragma unroll
    for (int r = 0; r < Code::kRows; ++r) {
      const int row = code_row(r);
      if (row >= a.M) break;
#pragma unroll
      for (int w = 0; w < Code::kWaves && Code::kWaves > 1; ++w) most[r] = max(most[r], most_of[row][w]);
      const RowScale of(most[r]);
#pragma unroll
      for (int v = 0; v < Code::kHeld; ++v)
        if (code_vector(v) < a.K / 8) *reinterpret_cast<uint2*>(codes[row] + code_vector(v) * 8) = row_codes(of, held[r][v]);
    }
    __syncthreads();
  };
  // (A wait behind a branch that some loads are in is for all of them: each way has its own code.)
  if (all / kWaves >= kAhead) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) request(j, j);
    make_codes();
    int i = 0;
    for (; i + 2 * kAhead <= pieces; i += kAhead)
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        multiply(j, i + j);
        request(j, i + j + kAhead);
      }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      multiply(j, i + j);
      if (i + j + kAhead < pieces) request(j, i + j + kAhead);
    }
#pragma unroll
    for (int j = 0; j < kAhead - 1; ++j)
      if (i + j + kAhead < pieces) multiply(j, i + j + kAhead);
  } else {
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (j < pieces) request(j, j);
    make_codes();
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (j < pieces) multiply(j, j);
  }
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
    if constexpr (kCodes) {
      uint32_t most = most_of[m][0];
#pragma unroll
      for (int w = 1; w < Code::kWaves; ++w) most = max(most, most_of[m][w]);
      xs = row_scale(most);
    } else {
      xs = a.xs[m];
    }
    const float* ws = static_cast<const float*>(a.w2) + n;
    leave(scaled(sum[0][0], xs, ws[0]), scaled(sum[0][1], xs, ws[1]), scaled(sum[0][2], xs, ws[2]), scaled(sum[0][3], xs, ws[3]));
  }
}

constexpr int kFewColumns = (1 << 28) - 16;       // of a result: 16 to a workgroup of 256, and a launch has fewer than 2^32 threads

template <typename Op>
int32_t enqueue_few(const OpArgs& a, const char* what, void* stream) {
  const unsigned groups = unsigned((a.N + 15) / 16);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (a.M <= 16)
    hipLaunchKernelGGL((gemm_few_kernel<Op, 1, NoCodes>), dim3(groups), dim3(64 * kFewWaves), 0, s, a);
  else
    hipLaunchKernelGGL((gemm_few_kernel<Op, 2, NoCodes>), dim3(groups), dim3(64 * kFewWaves), 0, s, a);
  return finish_launch(what);
}

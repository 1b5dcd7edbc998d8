// Per-head RMS norm of queries and keys with the 3-axis rotation in the same pass, and its gradients (gfx950).
//
//   y = w x r,  r = 1 / sqrt(mean(x^2) + eps),  z = R y           (R turns pair j by position * theta^(-2j/Da))
//   dy = R' dz,  dw = sum over tokens and heads of dy x r,  dn = dy w,  dx = r (dn - x r mean(dn x r))
//
// Memory bound: forward reads x and writes z once, backward reads x and dz and writes dx; statistics and products are fp32, with
// one rounding of each result to the storage type.  The gradients of the weights are summed in fp32 by each lane over the tokens
// and heads that it meets, over a workgroup's lanes in LDS and over the workgroups by a second small launch in fp64, in an order
// that depends on the sizes alone: no atomics, the same bits every time.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ca_internal.hpp"

namespace ca {
namespace {

#include "rope_device.hpp"
#include "norm_device.hpp"

constexpr int kMaxWorkgroups = 2048;              // of a backward launch: each leaves a partial sum of the weights' gradients

struct NormSide {                                 // queries or keys
  const void* x;
  const void* w;
  const void* dz;                                 // backward only
  void* y;                                        // forward: z, backward: dx
  int64_t x_tok, x_head, dz_tok, dz_head, y_tok, y_head;
};

struct NormArgs {
  NormSide side[2];
  int64_t n_tokens, first_frame;
  float* partials;                                // backward: [workgroup][side][head_dim]
  float eps;
  int32_t rows, rows_per_group;                   // heads of all sides, and of them a workgroup's
};

// cos / sin of the lane's four pairs at token n: a lane evaluates one pair of the token's and takes its four from the others
template <bool kFp64>
__device__ __forceinline__ void token_angles(const RopeGeom& g, int64_t n, int64_t first_frame, int lane, int c8, float* cs, float* sn) {
  const TokenPos p = token_pos_any(n, first_frame, g.grid_h, g.grid_w);
  float c1, s1;
  pair_cs<kFp64>(g, p, lane % (g.head_dim / 2), &c1, &s1);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    cs[j] = __shfl(c1, c8 * 4 + j, 64);
    sn[j] = __shfl(s1, c8 * 4 + j, 64);
  }
}

// A wave takes a token: its lanes cover 64 / chunks heads at a time (1 KB of bf16), rows_per_group heads in all, kAhead loads
// requested together, no more than there are (four for one head of each: 23400 tokens of 1 + 1 heads 20.1 us for 18.9, backward 48 for 25).
// Queries first, then keys: a loop over both picked the side for each load and weight (23400 tokens of 40 + 40 heads 192 us, now 178, the
// rate of a copy; 4680 of 12 + 12 18.5, now 13.4).
template <typename T, int kAhead>
__global__ __launch_bounds__(256) void norm_rope_kernel(RopeGeom g, NormArgs a) {
  const int chunks = g.head_dim / 8, head_slots = 64 / chunks;
  const int64_t n = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (n >= a.n_tokens) return;
  const int lane = threadIdx.x & 63, c8 = lane % chunks, hs = lane / chunks;
  const int r0 = blockIdx.y * a.rows_per_group, r1 = min(r0 + a.rows_per_group, a.rows);
  float cs[4], sn[4];
  bool angles = false;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int first = max(r0 - s * g.heads, 0), end = min(r1 - s * g.heads, g.heads);        // the group's heads of this side
    if (first >= end) continue;
    const NormSide& side = a.side[s];
    const T* const x = static_cast<const T*>(side.x) + n * side.x_tok + c8 * 8;
    T* const y = static_cast<T*>(side.y) + n * side.y_tok + c8 * 8;
    Vec8<T> w;
    w.load(static_cast<const T*>(side.w) + c8 * 8);
    for (int h = first + hs; h - hs < end; h += kAhead * head_slots) {
      Vec8<T> e[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) e[i].load(x + int64_t(min(h + i * head_slots, end - 1)) * side.x_head);      // past the last: that again
      if (!angles) token_angles<sizeof(T) == 4>(g, n, a.first_frame, lane, c8, cs, sn);
      angles = true;
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        norm8(e[i], w.v, chunks, a.eps);
        rotate8(e[i], cs, sn);
        if (h + i * head_slots < end) e[i].store(y + int64_t(h + i * head_slots) * side.y_head);
      }
    }
  }
}

// (Of one load's heads in bf16 129 registers would do; held to 128 there are four waves to a SIMD: 23400 tokens of 1 + 1 heads 25.5 us, 33.5 of three.)
// A wave takes the tokens that lie a launch's waves apart, of each all heads or a group's, and keeps the sums of dy x r of its lanes.  With the
// second launch 23400 tokens of 40 + 40 heads 262 us (5.5 TB/s), 4680 of 12 + 12 24.4.
template <typename T, int kAhead>
__global__ __launch_bounds__(256, kAhead == 1 && sizeof(T) == 2 ? 4 : 1) void norm_rope_backward_kernel(RopeGeom g, NormArgs a) {
  __shared__ float sums[4][2][2 * kMaxPairs];
  const int chunks = g.head_dim / 8, head_slots = 64 / chunks;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c8 = lane % chunks, hs = lane / chunks;
  const int r0 = blockIdx.y * a.rows_per_group, r1 = min(r0 + a.rows_per_group, a.rows);
  Vec8<T> w[2];
  float dw[2][8];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    if (s == 0 || a.rows > g.heads) w[s].load(static_cast<const T*>(a.side[s].w) + c8 * 8);
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[s][j] = 0.f;
  }
  for (int64_t n = int64_t(blockIdx.x) * 4 + wave; n < a.n_tokens; n += int64_t(gridDim.x) * 4) {
    float cs[4], sn[4];
    bool angles = false;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int first = max(r0 - s * g.heads, 0), end = min(r1 - s * g.heads, g.heads);      // the group's heads of this side
      if (first >= end) continue;
      const NormSide& side = a.side[s];
      const T* const x0 = static_cast<const T*>(side.x) + n * side.x_tok + c8 * 8;
      const T* const dz0 = static_cast<const T*>(side.dz) + n * side.dz_tok + c8 * 8;
      T* const y0 = static_cast<T*>(side.y) + n * side.y_tok + c8 * 8;
      for (int h = first + hs; h - hs < end; h += kAhead * head_slots) {
        Vec8<T> x[kAhead], d[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {         // past the last head: that one again
          const int64_t at = min(h + i * head_slots, end - 1);
          x[i].load(x0 + at * side.x_head);
          d[i].load(dz0 + at * side.dz_head);
        }
        if (!angles) {
          token_angles<sizeof(T) == 4>(g, n, a.first_frame, lane, c8, cs, sn);
#pragma unroll
          for (int j = 0; j < 4; ++j) sn[j] = -sn[j];        // R' turns back
          angles = true;
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const bool mine = h + i * head_slots < end;
          rotate8(d[i], cs, sn);
          float by, dot = 0.f;
          const float rstd = head_rstd(x[i], chunks, a.eps, &by), out = rstd * by;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            x[i].v[j] *= rstd;
            dw[s][j] += mine ? d[i].v[j] * x[i].v[j] : 0.f;
            d[i].v[j] *= w[s].v[j];
            dot = fmaf(d[i].v[j], x[i].v[j], dot);
          }
          const float mean = head_sum(dot, chunks) * (1.f / float(8 * chunks));
#pragma unroll
          for (int j = 0; j < 8; ++j) d[i].v[j] = out * fmaf(-x[i].v[j], mean, d[i].v[j]);
          if (mine) d[i].store(y0 + int64_t(h + i * head_slots) * side.y_head);
        }
      }
    }
  }
  for (int d = chunks; d < 64; d *= 2)             // over the heads that a wave's load covers
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) dw[s][j] += __shfl_xor(dw[s][j], d, 64);
  if (lane < chunks) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) sums[wave][s][lane * 8 + j] = dw[s][j];
  }
  __syncthreads();
  float* out = a.partials + (int64_t(blockIdx.y) * gridDim.x + blockIdx.x) * 2 * g.head_dim;
  for (int i = threadIdx.x; i < 2 * g.head_dim; i += 256) {
    const int s = i / g.head_dim, d = i - s * g.head_dim;
    out[i] = (sums[0][s][d] + sums[1][s][d]) + (sums[2][s][d] + sums[3][s][d]);
  }
}

// dw[side][d] from the workgroups' sums: 16 columns to a workgroup, its 64 rows of threads share the partials
constexpr int kGradCols = 16;
__global__ __launch_bounds__(1024) void norm_weight_grad_kernel(const float* partials, int n_partials, int head_dim, float* dw0, float* dw1) {
  __shared__ double sums[1024 / kGradCols][kGradCols + 1];
  const int x = threadIdx.x % kGradCols, y = threadIdx.x / kGradCols, col = blockIdx.x * kGradCols + x;
  double v = 0.;
#pragma unroll 8
  for (int i = y; i < n_partials; i += 1024 / kGradCols) v += double(partials[int64_t(i) * 2 * head_dim + col]);
  sums[y][x] = v;
  __syncthreads();
  for (int half = 1024 / kGradCols / 2; half > 0; half /= 2) {
    if (y < half) sums[y][x] += sums[y + half][x];
    __syncthreads();
  }
  if (y != 0) return;
  float* dw = col < head_dim ? dw0 : dw1;
  if (dw) dw[col < head_dim ? col : col - head_dim] = float(sums[0][x]);
}

// workgroups of four waves along the tokens, and groups of rows where there are few tokens
struct NormGrid {
  unsigned x, y;
  int32_t rows_per_group;
};

NormGrid norm_grid(int64_t workgroups, int rows, int head_dim, int fill) {
  const int slots = 512 / head_dim;               // heads of a wave's load
  int groups = 1;
  while (workgroups * groups < fill && groups * slots < rows) groups *= 2;
  NormGrid out;
  out.rows_per_group = (rows + groups - 1) / groups;
  out.x = unsigned(workgroups);
  out.y = unsigned((rows + out.rows_per_group - 1) / out.rows_per_group);
  return out;
}

// Loads of a side's heads that a wave requests together: as many as one of its row groups has, up to `most`
int norm_ahead(const RopeGeom& g, const NormGrid& grid, int most) {
  const int slots = 512 / g.head_dim, heads = grid.rows_per_group < g.heads ? grid.rows_per_group : g.heads;
  return std::min((heads + slots - 1) / slots, most);
}

int norm_sides(const RopeGeom& g, const NormTensors& q, const NormTensors& k, int64_t n_tokens, int64_t first_frame, float eps, NormArgs* a) {
  int n = 0;
  for (const NormTensors* t : {&q, &k}) {
    if (!t->x) continue;
    a->side[n++] = NormSide{t->x, t->w, t->dz, t->y, t->x_tok, t->x_head, t->dz_tok, t->dz_head, t->y_tok, t->y_head};
  }
  a->n_tokens = n_tokens;
  a->first_frame = first_frame;
  a->eps = eps;
  a->rows = n * g.heads;
  return n;
}

// Each workgroup of a backward launch leaves partial sums that the second launch reads: 512 of them, more where there is much to read or
// there are many tokens (each with its angles).  Us with up to 512 / 1024 / 2048, both launches: 4680 tokens of 12 + 12 heads 23.6 / 25.5 / 24.9,
// 12000 of 16 + 16 70.5 / 67.3 / 66.2, 23400 of 40 + 40 273 / 280 / 262, of 1 + 1 28.8 / 25.3 / 30.0; heads are dealt to groups up to
// 256 workgroups (1000 tokens of 5 + 5 heads 10.8, up to 512 13.1).
NormGrid backward_grid(const RopeGeom& g, int64_t n_tokens, int rows, int bytes_of_value) {
  const int64_t all = (n_tokens + 3) / 4, read = 2 * n_tokens * rows * g.head_dim * bytes_of_value;
  const int64_t most = read > (int64_t(128) << 20) ? kMaxWorkgroups : n_tokens > 16384 ? kMaxWorkgroups / 2 : kMaxWorkgroups / 4;
  return norm_grid(std::min(all, most), rows, g.head_dim, 256);
}

}  // namespace

int32_t launch_norm_rope(const RopeGeom& g, int dtype, const NormTensors& q, const NormTensors& k, float eps, int64_t n_tokens,
                         int64_t first_frame, void* stream) {
  if (n_tokens == 0) return CA_OK;
  NormArgs a{};
  if (norm_sides(g, q, k, n_tokens, first_frame, eps, &a) == 0) return CA_EINVAL;
  const int64_t gx = (n_tokens + 3) / 4;
  if (gx >= (1 << 24)) return CA_EUNSUPPORTED;     // (a launch has fewer than 2^32 threads)
  const NormGrid grid = norm_grid(gx, a.rows, g.head_dim, 2048);
  a.rows_per_group = grid.rows_per_group;
  using Kernel = void (*)(RopeGeom, NormArgs);
  static constexpr Kernel kKernels[2][4] = {{norm_rope_kernel<float, 1>, norm_rope_kernel<float, 2>, norm_rope_kernel<float, 3>, norm_rope_kernel<float, 4>},
                                            {norm_rope_kernel<uint16_t, 1>, norm_rope_kernel<uint16_t, 2>, norm_rope_kernel<uint16_t, 3>,
                                             norm_rope_kernel<uint16_t, 4>}};
  const Kernel kernel = kKernels[dtype == CA_BF16][norm_ahead(g, grid, 4) - 1];
  hipLaunchKernelGGL(kernel, dim3(grid.x, grid.y), dim3(256), 0, static_cast<hipStream_t>(stream), g, a);
  return finish_launch("norm_rope.hip");
}

size_t norm_rope_backward_bytes(int32_t head_dim) { return size_t(kMaxWorkgroups) * 2 * head_dim * sizeof(float); }

int32_t launch_norm_rope_backward(const RopeGeom& g, int dtype, const NormTensors& q, const NormTensors& k, float eps, int64_t n_tokens,
                                  int64_t first_frame, float* dq_weight, float* dk_weight, void* workspace, void* stream) {
  NormArgs a{};
  const int sides = norm_sides(g, q, k, n_tokens, first_frame, eps, &a);
  if (sides == 0) return CA_EINVAL;
  a.partials = static_cast<float*>(workspace);
  hipStream_t s = static_cast<hipStream_t>(stream);
  int n_partials = 0;
  if (n_tokens > 0) {
    const NormGrid grid = backward_grid(g, n_tokens, a.rows, dtype == CA_BF16 ? 2 : 4);
    a.rows_per_group = grid.rows_per_group;
    n_partials = int(grid.x * grid.y);
    using Kernel = void (*)(RopeGeom, NormArgs);
    static constexpr Kernel kKernels[2][3] = {
        {norm_rope_backward_kernel<float, 1>, norm_rope_backward_kernel<float, 2>, norm_rope_backward_kernel<float, 3>},
        {norm_rope_backward_kernel<uint16_t, 1>, norm_rope_backward_kernel<uint16_t, 2>, norm_rope_backward_kernel<uint16_t, 3>}};
    const Kernel kernel = kKernels[dtype == CA_BF16][norm_ahead(g, grid, 3) - 1];
    hipLaunchKernelGGL(kernel, dim3(grid.x, grid.y), dim3(256), 0, s, g, a);
    if (const int32_t rc = finish_launch("norm_rope.hip"); rc != CA_OK) return rc;
  }
  float* const dw[2] = {q.x ? dq_weight : dk_weight, sides == 2 ? dk_weight : nullptr};
  hipLaunchKernelGGL(norm_weight_grad_kernel, dim3(unsigned(2 * g.head_dim / kGradCols)), dim3(1024), 0, s, a.partials, n_partials, g.head_dim, dw[0], dw[1]);
  return finish_launch("norm_rope.hip");
}

}  // namespace ca

// The AdamW step of many tensors in one launch, with states in 32 bits or in 8 (gfx950).
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  p = (1 - lr wd) p - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)
//
// Memory bound: each value is read and written once where it lies.  States in 8 bits are codes with a scale a (fp32) for every 256 values of a
// tensor: m = sign(c) a (c / 127)^2, v = a (c / 255)^4.  The square and the fourth power give small magnitudes finer steps: a code is off by at most half
// of one, 1 / c of m and 2 / c of v, where equal steps would leave nothing of what is 250 times smaller than the block's largest; and a v above zero
// keeps a code above zero, so that no step divides by eps alone.  With states in 8 bits m and v are computed in 64 bits, at the rate of fp32 here, so
// that the codes are those of exact arithmetic: an estimate in fp32 says between which two codes a value lies, a comparison with the border in 64 bits
// says which of them it is.
//
// A wave takes 512 values at a time, 8 to a lane, 32 lanes to a block.  What tensors there are comes with the launch (40 to one), so that nothing
// has to be copied ahead of it.  How many steps a tensor has behind it is counted on the device, by a small launch ahead that leaves what the step needs of
// it, so that a captured step goes on counting in every replay.  (Counted by the workgroup of a tensor that ends last, by a ticket, it was one
// launch, but each ticket took 40 ns: 3 x 4096 x 1536 values, 4608 workgroups, 289 us.)
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ca_internal.hpp"

namespace ca {
namespace {

#include "rope_device.hpp"

constexpr int kMostTensors = 40 /* at most a wave */, kUnit = 512, kWaves = 4;

struct AdamTensor {
  void* p;
  const void* g;
  uint16_t* copy;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  int32_t* step;                                  // [0] steps done; [1], [2] lr / (1 - b1^t) and 1 / sqrt(1 - b2^t) in fp32
  int64_t n;
  int32_t first, types;                           // workgroup of the launch; bit 0: parameters in bf16, bit 1: gradients
};

struct AdamArgs {
  double beta1, beta2, grad_scale;
  float lr, keep, eps;                            // keep: 1 - lr wd
  int32_t tensors, units;                         // units of a workgroup
  AdamTensor of[kMostTensors];
};
static_assert(sizeof(AdamArgs) <= 4096, "a launch's arguments");

// Eight values of any alignment that their type allows
struct __attribute__((packed, aligned(4))) Packed4 { uint32_t w[4]; };
struct __attribute__((packed, aligned(2))) Packed2 { uint32_t w[4]; };

__device__ __forceinline__ void load8(const void* from, int64_t at, int left, bool half, float (&to)[8]) {
  if (half) {
    const uint16_t* const p = static_cast<const uint16_t*>(from) + at;
    if (left >= 8) {
      const Packed2 a = *reinterpret_cast<const Packed2*>(p);
#pragma unroll
      for (int j = 0; j < 4; ++j) to[2 * j] = bf16_lo(a.w[j]), to[2 * j + 1] = bf16_hi(a.w[j]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) to[j] = j < left ? __uint_as_float(uint32_t(p[j]) << 16) : 0.f;
    }
  } else {
    const float* const p = static_cast<const float*>(from) + at;
    if (left >= 8) {
      const Packed4 a = *reinterpret_cast<const Packed4*>(p), b = *reinterpret_cast<const Packed4*>(p + 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) to[j] = __uint_as_float(a.w[j]), to[4 + j] = __uint_as_float(b.w[j]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) to[j] = j < left ? p[j] : 0.f;
    }
  }
}

__device__ __forceinline__ void store8_half(uint16_t* p, int left, const float (&v)[8]) {
  if (left >= 8) {
    *reinterpret_cast<Packed2*>(p) = Packed2{{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])}};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) p[j] = uint16_t(pack_bf16(v[j], v[j]));
  }
}
__device__ __forceinline__ void store8(float* p, int left, const float (&v)[8]) {
  if (left >= 8) {
    *reinterpret_cast<Packed4*>(p) = Packed4{{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])}};
    *reinterpret_cast<Packed4*>(p + 4) = Packed4{{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])}};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) p[j] = v[j];
  }
}

template <int kCtrl>
__device__ __forceinline__ uint32_t dpp_max(uint32_t x) {
  return max(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), kCtrl, 0xf, 0xf, true)));
}
// the largest of 32 lanes, in all of them
__device__ __forceinline__ uint32_t block_max(uint32_t x) {
  x = dpp_max<0xb1>(x);                          // quad_perm [1, 0, 3, 2]
  x = dpp_max<0x4e>(x);                          // quad_perm [2, 3, 0, 1]
  x = dpp_max<0x141>(x);                         // row_half_mirror
  x = dpp_max<0x140>(x);                         // row_mirror
  return max(x, uint32_t(__shfl_xor(int(x), 16, 64)));
}

__device__ __forceinline__ double m_of(int c, double a) { return a * (double(c * abs(c)) * (1. / (127. * 127.))); }
__device__ __forceinline__ double v_of(int c, double a) {
  const double square = double(c * c);
  return a * (square * square * (1. / (255. * 255. * 255. * 255.)));
}

// The code of a magnitude x beside the scale a > 0: round(127 sqrt(x / a)); x / a is in `part`
__device__ __forceinline__ int m_code(double x, double a, float part) {
  const int c = min(int(127.f * __builtin_amdgcn_sqrtf(part)), 127);                 // one too few at most, next to a whole number
  const double b = double((2 * c + 1) * (2 * c + 1));
  return min(c + int(x * (4. * 127. * 127.) >= a * b), 127);
}
// round(255 (x / a)^(1/4)), at least 1 for x > 0
__device__ __forceinline__ int v_code(double x, double a, float part) {
  const int c = min(int(255.f * __builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(part))), 255);
  const double b = double((2 * c + 1) * (2 * c + 1));
  return x > 0. ? max(1, min(c + int(x * (510. * 510. * 510. * 510.) >= a * (b * b)), 255)) : 0;
}

__device__ __forceinline__ double power(double x, int n) {
  double r = 1.;
  for (; n > 0; n >>= 1) {
    if (n & 1) r *= x;
    x *= x;
  }
  return r;
}

__global__ __launch_bounds__(64) void adamw_count_kernel(AdamArgs a) {
  if (int(threadIdx.x) >= a.tensors) return;
  int32_t* const step = a.of[threadIdx.x].step;
  const int now = step[0] + 1;
  step[0] = now;
  step[1] = __float_as_int(float(double(a.lr) / (1. - power(a.beta1, now))));
  step[2] = __float_as_int(float(1. / sqrt(1. - power(a.beta2, now))));
}

template <int kBits>
__global__ __launch_bounds__(64 * kWaves) void adamw_kernel(AdamArgs a) {
  int i = 0;
  while (i + 1 < a.tensors && int(blockIdx.x) >= a.of[i + 1].first) ++i;
  const AdamTensor t = a.of[i];
  const int64_t units = (t.n + kUnit - 1) / kUnit, begin = int64_t(int(blockIdx.x) - t.first) * a.units;
  const int64_t end = begin + a.units < units ? begin + a.units : units;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const float rate = __int_as_float(t.step[1]), by = __int_as_float(t.step[2]);
  const bool half_p = t.types & 1, half_g = t.types & 2;
  for (int64_t u = begin + wave; u < end; u += kWaves) {
    const int64_t at = u * kUnit + lane * 8;
    const int left = int(t.n - at < 8 ? t.n - at : 8);                              // (zero and less behind the end)
    float p[8], g[8], m[8], v[8];
    load8(t.g, at, left, half_g, g);
    if constexpr (kBits == 32) {
      load8(t.m, at, left, false, m);
      load8(t.v, at, left, false, v);
      load8(t.p, at, left, half_p, p);
      const float scale = float(a.grad_scale), b1 = float(a.beta1), b2 = float(a.beta2), c1 = float(1. - a.beta1), c2 = float(1. - a.beta2);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        g[j] *= scale;
        m[j] = fmaf(b1, m[j], c1 * g[j]);
        v[j] = fmaf(b2, v[j], c2 * (g[j] * g[j]));
      }
      store8(static_cast<float*>(t.m) + at, left, m);
      store8(static_cast<float*>(t.v) + at, left, v);
    } else {
      // codes and scales are there up to the block's end, of the last unit's second block only if it has values
      const int64_t block = at >> 8;
      const bool there = block * 256 < t.n;
      const uint2 cm = there ? *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.m) + at) : make_uint2(0, 0);
      const uint2 cv = there ? *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.v) + at) : make_uint2(0, 0);
      const double am = there ? double(t.m_scale[block]) : 0., av = there ? double(t.v_scale[block]) : 0.;
      load8(t.p, at, left, half_p, p);
      double dm[8], dv[8];
      uint32_t most_m = 0, most_v = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int old_m = int(int8_t((j < 4 ? cm.x : cm.y) >> (8 * (j % 4)))), old_v = int((j < 4 ? cv.x : cv.y) >> (8 * (j % 4)) & 255);
        const double scaled = double(g[j]) * a.grad_scale;
        dm[j] = fma(a.beta1, m_of(old_m, am), (1. - a.beta1) * scaled);
        dv[j] = fma(a.beta2, v_of(old_v, av), (1. - a.beta2) * (scaled * scaled));
        if (j >= left) dm[j] = dv[j] = 0.;
        m[j] = float(dm[j]);
        v[j] = float(dv[j]);
        most_m = max(most_m, __float_as_uint(m[j]) & 0x7fffffffu);                   // (a NaN is more than any number so)
        most_v = max(most_v, __float_as_uint(v[j]) & 0x7fffffffu);
      }
      most_m = block_max(most_m);
      most_v = block_max(most_v);
      const double new_m = double(__uint_as_float(most_m)), new_v = double(__uint_as_float(most_v));
      const double per_m = 1. / new_m, per_v = 1. / new_v;
      uint32_t codes_m[2] = {0, 0}, codes_v[2] = {0, 0};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const double size = fabs(dm[j]);
        int c = m_code(size, new_m, float(size * per_m)), d = v_code(dv[j], new_v, float(dv[j] * per_v));
        // of a block of zeros all are zeros; one that holds an infinity or NaN is not a number: its largest code times such a scale
        c = most_m == 0 ? 0 : most_m >= 0x7f800000u ? 127 : c;
        d = most_v == 0 ? 0 : most_v >= 0x7f800000u ? 255 : d;
        c = dm[j] < 0. ? -c : c;
        codes_m[j / 4] |= uint32_t(c & 255) << (8 * (j % 4));
        codes_v[j / 4] |= uint32_t(d) << (8 * (j % 4));
      }
      if (there) {
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(t.m) + at) = make_uint2(codes_m[0], codes_m[1]);
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(t.v) + at) = make_uint2(codes_v[0], codes_v[1]);
        if ((lane & 31) == 0) {
          t.m_scale[block] = __uint_as_float(most_m);
          t.v_scale[block] = __uint_as_float(most_v);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = fmaf(a.keep, p[j], -rate * (m[j] / fmaf(sqrtf(v[j]), by, a.eps)));
    if (half_p) store8_half(static_cast<uint16_t*>(t.p) + at, left, p); else store8(static_cast<float*>(t.p) + at, left, p);
    if (t.copy) store8_half(t.copy + at, left, p);
  }
}

// What states in 8 bits stand for
__global__ __launch_bounds__(256) void adamw_values_kernel(const int8_t* m, const uint8_t* v, const float* m_scale, const float* v_scale, float* m_out,
                                                           float* v_out, int64_t n) {
  for (int64_t at = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 8; at < n; at += int64_t(gridDim.x) * 2048) {
    const uint2 cm = *reinterpret_cast<const uint2*>(m + at), cv = *reinterpret_cast<const uint2*>(v + at);
    const double am = double(m_scale[at >> 8]), av = double(v_scale[at >> 8]);
    uint32_t to[2][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      to[0][j] = __float_as_uint(float(m_of(int(int8_t((j < 4 ? cm.x : cm.y) >> (8 * (j % 4)))), am)));
      to[1][j] = __float_as_uint(float(v_of(int((j < 4 ? cv.x : cv.y) >> (8 * (j % 4)) & 255), av)));
    }
    store_once(m_out + at, U4{to[0][0], to[0][1], to[0][2], to[0][3]});
    store_once(m_out + at + 4, U4{to[0][4], to[0][5], to[0][6], to[0][7]});
    store_once(v_out + at, U4{to[1][0], to[1][1], to[1][2], to[1][3]});
    store_once(v_out + at + 4, U4{to[1][4], to[1][5], to[1][6], to[1][7]});
  }
}

// Units of a workgroup: one to a wave until the launch has several thousand workgroups
constexpr int64_t kWorkgroups = 4096;

}  // namespace

int32_t launch_adamw(const ca_adamw_tensor* tensors, int32_t n_tensors, int32_t state_bits, double lr, double beta1, double beta2, double eps,
                     double weight_decay, double grad_scale, void* stream) {
  AdamArgs a{};
  a.beta1 = beta1; a.beta2 = beta2; a.grad_scale = grad_scale;
  a.lr = float(lr); a.keep = float(1. - lr * weight_decay); a.eps = float(eps);
  for (int32_t from = 0; from < n_tensors;) {
    int64_t units = 0;
    int32_t to = from;
    a.tensors = 0;
    for (; to < n_tensors && a.tensors < kMostTensors; ++to) {
      const ca_adamw_tensor& t = tensors[to];
      if (t.n == 0 || !t.grad) continue;
      a.of[a.tensors++] = AdamTensor{t.param, t.grad, static_cast<uint16_t*>(t.copy), t.m, t.v, t.m_scale, t.v_scale, t.step, t.n, 0,
                                     (t.param_dtype == CA_BF16 ? 1 : 0) | (t.grad_dtype == CA_BF16 ? 2 : 0)};
      units += (t.n + kUnit - 1) / kUnit;
    }
    from = to;
    if (a.tensors == 0) continue;
    a.units = int32_t(std::max<int64_t>(1, units / (kWaves * kWorkgroups))) * kWaves;
    int32_t workgroups = 0;
    for (int i = 0; i < a.tensors; ++i) {
      a.of[i].first = workgroups;
      workgroups += int32_t(((a.of[i].n + kUnit - 1) / kUnit + a.units - 1) / a.units);
    }
    hipLaunchKernelGGL(adamw_count_kernel, dim3(1), dim3(64), 0, static_cast<hipStream_t>(stream), a);
    if (const int32_t rc = finish_launch("adamw.hip"); rc != CA_OK) return rc;
    hipLaunchKernelGGL(state_bits == 8 ? adamw_kernel<8> : adamw_kernel<32>, dim3(unsigned(workgroups)), dim3(64 * kWaves), 0, static_cast<hipStream_t>(stream), a);
    if (const int32_t rc = finish_launch("adamw.hip"); rc != CA_OK) return rc;
  }
  return CA_OK;
}

int32_t launch_adamw_values(const void* m, const void* v, const float* m_scale, const float* v_scale, float* m_out, float* v_out, int64_t n, void* stream) {
  if (n == 0) return CA_OK;
  const int64_t all = (n + 2047) / 2048;
  hipLaunchKernelGGL(adamw_values_kernel, dim3(unsigned(std::min<int64_t>(all, 16384))), dim3(256), 0, static_cast<hipStream_t>(stream),
                     static_cast<const int8_t*>(m), static_cast<const uint8_t*>(v), m_scale, v_scale, m_out, v_out, n);
  return finish_launch("adamw.hip");
}

}  // namespace ca

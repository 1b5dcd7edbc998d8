// The AdamW step of many tensors in one launch, with states in 32 bits or in 8 (gfx950).
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  p = (1 - lr wd) p - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)
//
// Memory bound: each value is read and written once where it lies (3 x 13824 x 5120 values in bf16: states in 32 bits 900 us, 5.2 TB/s, the rate of a
// copy; in 8 bits 550, 3.9 TB/s, where some 70 instructions a value share the time with the memory).  States in 8 bits are codes with a scale a (fp32) for every 256 values of a
// tensor: m = sign(c) a (c / 127)^2, v = a (c / 255)^4.  The square and the fourth power give small magnitudes finer steps: a code is off by at most half
// of one, 1 / c of m and 2 / c of v, where equal steps would leave nothing of what is 250 times smaller than the block's largest; and a v above zero
// keeps a code above zero, so that no step divides by eps alone.  With states in 8 bits m and v are computed in 64 bits, at the rate of fp32 here, so
// that the codes are those of exact arithmetic: an estimate in fp32 says between which two codes a value lies, a comparison with the border in 64 bits
// says which of them it is.
//
// A wave takes 512 values at a time, 8 to a lane, 32 lanes to a block.  Where the parameters and their states are lies in a table on the device, which the
// caller keeps; the gradients' addresses come with the launch, 300 to one (with all addresses in the launch it were 40: 120 tensors of 49152 values in
// fp32 three launches of 17 us and three more that count).  How many steps a tensor has behind it is counted on the device, by a small launch ahead that leaves what the step needs of
// it, so that a captured step goes on counting in every replay.  (Counted by the workgroup of a tensor that ends last, by a ticket, it was one
// launch, but each ticket took 40 ns: 3 x 4096 x 1536 values, 4608 workgroups, 289 us.)
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ca_internal.hpp"

namespace ca {
namespace {

#include "rope_device.hpp"

constexpr int kMostTensors = 300, kUnit = 512, kWaves = 4;

// a tensor as a workgroup sees it: of the table, whose values all lanes share, so that they come by scalar loads
typedef const __attribute__((address_space(4))) ca_adamw_tensor* AdamTable;

struct AdamArgs {
  const ca_adamw_tensor* table;                   // step: [0] steps done; [1], [2] lr / (1 - b1^t) and 1 / sqrt(1 - b2^t) in fp32
  double beta1, beta2, grad_scale;
  float lr, keep, eps;                            // keep: 1 - lr wd
  int32_t tensors, units;                         // units of a workgroup
  uint64_t grads[kMostTensors];                   // and 1 where they are bf16; 0: the tensor is left out
  int32_t first[kMostTensors];                    // workgroup of the launch; of a tensor that is left out that of the next one
};
static_assert(sizeof(AdamArgs) <= 4096, "a launch's arguments");

typedef __attribute__((ext_vector_type(8))) float F8;

// Eight values of any alignment that their type allows; zeros from `left` on
struct __attribute__((packed, aligned(4))) Packed4 { uint32_t w[4]; };
struct __attribute__((packed, aligned(2))) Packed2 { uint32_t w[4]; };

template <bool kHalf>
__device__ __forceinline__ void load8(const void* from, int64_t at, int left, F8& to) {
  if constexpr (kHalf) {
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

__device__ __forceinline__ void store8_half(uint16_t* p, int left, const F8& v) {
  if (left >= 8) {
    *reinterpret_cast<Packed2*>(p) = Packed2{{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])}};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) p[j] = uint16_t(pack_bf16(v[j], v[j]));
  }
}
__device__ __forceinline__ void store8(float* p, int left, const F8& v) {
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

// What codes stand for beside a scale, without what belongs to all codes: m = m_size / 127^2 a, v = v_size / 255^4 a
constexpr double kPerM = 1. / (127. * 127.), kPerV = 1. / (255. * 255. * 255. * 255.);
__device__ __forceinline__ double m_size(int c) { return double(c * abs(c)); }
__device__ __forceinline__ double v_size(int c) {
  const double square = double(c * c);
  return square * square;
}

// Codes of eight magnitudes x (xf: in fp32) beside the scale a: round(kMost (|x| / a)^(1/2)), of the second moment the (1/4).  An estimate in fp32 is off
// by less than 1e-4 (kMost times five roundings); where one of the eight lies as near to a border between two codes as that (a wave in five), or the
// scale is no ordinary number, the border is compared with in 64 bits.
template <bool kSecond>
__device__ __forceinline__ void codes8(const double (&x)[8], const F8& xf, float a, int (&code)[8]) {
  constexpr float kMost = kSecond ? 255.f : 127.f;
  const float part = __builtin_amdgcn_rcpf(a);
  bool near = !(a >= 0x1p-100f && a <= 0x1p100f);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float t = __builtin_amdgcn_sqrtf(fabsf(xf[j]) * part);
    if (kSecond) t = __builtin_amdgcn_sqrtf(t);
    t *= kMost;
    const float whole = rintf(t);
    near |= fabsf(t - whole) > 0.4999f;
    code[j] = int(whole);
    if (kSecond) code[j] = max(code[j], min(__double2hiint(x[j]), 1));                // (a double above zero has bits in its upper half, from 2^-1042 on)
  }
  if (__any(near)) {
    const double scale = double(a), per = 1. / scale;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float t = __builtin_amdgcn_sqrtf(float(fabs(x[j]) * per));
      if (kSecond) t = __builtin_amdgcn_sqrtf(t);
      int c = min(int(t * kMost), int(kMost));                     // the code or one below
      double b = double((2 * c + 1) * (2 * c + 1)), of = fabs(x[j]) * (4. * kMost * kMost);
      if (kSecond) b *= b, of *= 4. * kMost * kMost;
      c = min(c + int(of >= scale * b), int(kMost));
      if (kSecond) c = x[j] > 0. ? max(c, 1) : 0;
      // of a block of zeros all are zeros; one that holds an infinity or NaN is not a number: its largest code times such a scale
      code[j] = a == 0.f ? 0 : a <= 0x1.fffffep127f ? c : int(kMost);
    }
  }
}

// The root of a number of fp32 to a rounding or so; those below the normal ones, which the instruction takes for zeros, only where they matter: beside an
// eps of 2^-30 and more a root of 2^-63 does not
template <bool kSmall>
__device__ __forceinline__ float root(float x) {
  const bool small = kSmall && x < 0x1p-96f;
  return __builtin_amdgcn_sqrtf(small ? x * 0x1p64f : x) * (small ? 0x1p-32f : 1.f);
}

template <bool kSmall>
__device__ __forceinline__ void move8(F8& p, const F8& m, const F8& v, float keep, float rate, float by, float eps) {
#pragma unroll
  for (int j = 0; j < 8; ++j) p[j] = fmaf(keep, p[j], -rate * (m[j] * __builtin_amdgcn_rcpf(fmaf(root<kSmall>(v[j]), by, eps))));
}

__device__ __forceinline__ double power(double x, int n) {
  double r = 1.;
  for (; n > 0; n >>= 1) {
    if (n & 1) r *= x;
    x *= x;
  }
  return r;
}

__global__ __launch_bounds__(kMostTensors) void adamw_count_kernel(AdamArgs a) {
  const int i = threadIdx.x;
  if (i >= a.tensors || a.grads[i] == 0) return;
  int32_t* const step = a.table[i].step;
  const int now = step[0] + 1;
  step[0] = now;
  step[1] = __float_as_int(float(double(a.lr) / (1. - power(a.beta1, now))));
  step[2] = __float_as_int(float(1. / sqrt(1. - power(a.beta2, now))));
}

struct AdamTensor {
  void* p;
  const void* g;
  uint16_t* copy;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  const int32_t* step;
  int64_t n;
};

// units begin + wave, + kWaves .. below end
template <int kBits, bool kHalfP, bool kHalfG>
__device__ __forceinline__ void step_units(const AdamArgs& a, const AdamTensor t, int64_t begin, int64_t end) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const float rate = __int_as_float(t.step[1]), by = __int_as_float(t.step[2]);
  for (int64_t u = begin + wave; u < end; u += kWaves) {
    const int64_t at = u * kUnit + lane * 8;
    const int left = int(t.n - at < 8 ? t.n - at : 8);                              // (zero and less behind the end)
    F8 p, g, m, v;
    load8<kHalfG>(t.g, at, left, g);
    if constexpr (kBits == 32) {
      load8<false>(t.m, at, left, m);
      load8<false>(t.v, at, left, v);
      load8<kHalfP>(t.p, at, left, p);
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
      const float am = there ? t.m_scale[block] : 0.f, av = there ? t.v_scale[block] : 0.f;
      load8<kHalfP>(t.p, at, left, p);
      uint32_t most_m = 0, most_v = 0;
      const double keep_m = a.beta1 * kPerM * double(am), keep_v = a.beta2 * kPerV * double(av);
      const double add_m = (1. - a.beta1) * a.grad_scale, add_v = (1. - a.beta2) * a.grad_scale * a.grad_scale;
      double dm[8], dv[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int old_m = int(int8_t((j < 4 ? cm.x : cm.y) >> (8 * (j % 4)))), old_v = int((j < 4 ? cv.x : cv.y) >> (8 * (j % 4)) & 255);
        const double grad = double(g[j]);                           // (behind the end gradients and codes are zeros)
        dm[j] = fma(keep_m, m_size(old_m), add_m * grad);
        dv[j] = fma(keep_v, v_size(old_v), add_v * (grad * grad));
        m[j] = float(dm[j]);
        v[j] = float(dv[j]);
        most_m = max(most_m, __float_as_uint(m[j]) & 0x7fffffffu);                   // (a NaN is more than any number so)
        most_v = max(most_v, __float_as_uint(v[j]) & 0x7fffffffu);
      }
      most_m = block_max(most_m);
      most_v = block_max(most_v);
      int new_m[8], new_v[8];
      codes8<false>(dm, m, __uint_as_float(most_m), new_m);
      codes8<true>(dv, v, __uint_as_float(most_v), new_v);
      uint32_t codes_m[2] = {0, 0}, codes_v[2] = {0, 0};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        codes_m[j / 4] |= uint32_t((__double2hiint(dm[j]) < 0 ? -new_m[j] : new_m[j]) & 255) << (8 * (j % 4));
        codes_v[j / 4] |= uint32_t(new_v[j]) << (8 * (j % 4));
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
    if (a.eps >= 0x1p-30f) move8<false>(p, m, v, a.keep, rate, by, a.eps); else move8<true>(p, m, v, a.keep, rate, by, a.eps);
    if constexpr (kHalfP) store8_half(static_cast<uint16_t*>(t.p) + at, left, p); else store8(static_cast<float*>(t.p) + at, left, p);
    if (t.copy) store8_half(t.copy + at, left, p);
  }
}

template <int kBits>
__global__ __launch_bounds__(64 * kWaves) void adamw_kernel(AdamArgs a) {
  int i = 0, behind = a.tensors;                  // the last tensor that begins at this workgroup or before
  while (behind - i > 1) {
    const int mid = (i + behind) >> 1;
    if (a.first[mid] <= int(blockIdx.x)) i = mid; else behind = mid;
  }
  const AdamTable of = reinterpret_cast<AdamTable>(reinterpret_cast<uintptr_t>(a.table)) + i;
  const uint64_t grad = a.grads[i];
  const AdamTensor t{of->param, reinterpret_cast<const void*>(grad & ~uint64_t(1)), static_cast<uint16_t*>(of->copy), of->m, of->v, of->m_scale, of->v_scale,
                     of->step, of->n};
  const int64_t units = (t.n + kUnit - 1) / kUnit, begin = int64_t(int(blockIdx.x) - a.first[i]) * a.units;
  const int64_t end = begin + a.units < units ? begin + a.units : units;
  switch ((of->param_dtype == CA_BF16 ? 1 : 0) | (grad & 1 ? 2 : 0)) {
    case 0: return step_units<kBits, false, false>(a, t, begin, end);
    case 1: return step_units<kBits, true, false>(a, t, begin, end);
    case 2: return step_units<kBits, false, true>(a, t, begin, end);
    default: return step_units<kBits, true, true>(a, t, begin, end);
  }
}

// What states in 8 bits stand for.  Four values to a lane, whole lines to a store: eight to a lane, stores of every other 16 bytes, took 530 us for
// 3 x 13824 x 5120 values.
__global__ __launch_bounds__(256) void adamw_values_kernel(const int8_t* m, const uint8_t* v, const float* m_scale, const float* v_scale, float* m_out,
                                                           float* v_out, int64_t n) {
  for (int64_t at = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 4; at < n; at += int64_t(gridDim.x) * 1024) {
    const uint32_t cm = *reinterpret_cast<const uint32_t*>(m + at), cv = *reinterpret_cast<const uint32_t*>(v + at);
    const double am = double(m_scale[at >> 8]) * kPerM, av = double(v_scale[at >> 8]) * kPerV;
    uint32_t to[2][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      to[0][j] = __float_as_uint(float(m_size(int(int8_t(cm >> (8 * j)))) * am));
      to[1][j] = __float_as_uint(float(v_size(int(cv >> (8 * j) & 255)) * av));
    }
    store_once(m_out + at, U4{to[0][0], to[0][1], to[0][2], to[0][3]});
    store_once(v_out + at, U4{to[1][0], to[1][1], to[1][2], to[1][3]});
  }
}

// Workgroups of a launch, from which on each of their waves takes several units.  Us for 3 x 13824 x 5120 values with 4096 / 16384 / 65536 of them (where
// the last round of them is a small part): 32 bits 1003 / 955 / 900, 8 bits 562 / 547 / 571.
constexpr int64_t kWorkgroups32 = 65536, kWorkgroups8 = 16384;

}  // namespace

int32_t launch_adamw(const ca_adamw_tensor* tensors, const ca_adamw_tensor* tensors_dev, int32_t n_tensors, int32_t state_bits, double lr, double beta1,
                     double beta2, double eps, double weight_decay, double grad_scale, void* stream) {
  AdamArgs a;
  a.beta1 = beta1; a.beta2 = beta2; a.grad_scale = grad_scale;
  a.lr = float(lr); a.keep = float(1. - lr * weight_decay); a.eps = float(eps);
  const int64_t most = kWaves * (state_bits == 8 ? kWorkgroups8 : kWorkgroups32);
  for (int32_t from = 0; from < n_tensors; from += kMostTensors) {
    a.table = tensors_dev + from;
    a.tensors = std::min(n_tensors - from, kMostTensors);
    int64_t units = 0, workgroups = 0;
    for (int i = 0; i < a.tensors; ++i)
      if (const ca_adamw_tensor& t = tensors[from + i]; t.grad) units += (t.n + kUnit - 1) / kUnit;
    a.units = int32_t(std::max<int64_t>(1, units / most)) * kWaves;
    for (int i = 0; i < a.tensors; ++i) {
      const ca_adamw_tensor& t = tensors[from + i];
      const bool there = t.grad && t.n > 0;
      a.grads[i] = there ? uint64_t(reinterpret_cast<uintptr_t>(t.grad)) | (t.grad_dtype == CA_BF16 ? 1 : 0) : 0;
      a.first[i] = int32_t(workgroups);
      if (there) workgroups += ((t.n + kUnit - 1) / kUnit + a.units - 1) / a.units;
    }
    if (workgroups == 0) continue;
    hipLaunchKernelGGL(adamw_count_kernel, dim3(1), dim3(kMostTensors), 0, static_cast<hipStream_t>(stream), a);
    if (const int32_t rc = finish_launch("adamw.hip"); rc != CA_OK) return rc;
    hipLaunchKernelGGL(state_bits == 8 ? adamw_kernel<8> : adamw_kernel<32>, dim3(unsigned(workgroups)), dim3(64 * kWaves), 0, static_cast<hipStream_t>(stream), a);
    if (const int32_t rc = finish_launch("adamw.hip"); rc != CA_OK) return rc;
  }
  return CA_OK;
}

int32_t launch_adamw_values(const void* m, const void* v, const float* m_scale, const float* v_scale, float* m_out, float* v_out, int64_t n, void* stream) {
  if (n == 0) return CA_OK;
  const int64_t all = (n + 1023) / 1024;
  hipLaunchKernelGGL(adamw_values_kernel, dim3(unsigned(std::min<int64_t>(all, 16384))), dim3(256), 0, static_cast<hipStream_t>(stream),
                     static_cast<const int8_t*>(m), static_cast<const uint8_t*>(v), m_scale, v_scale, m_out, v_out, n);
  return finish_launch("adamw.hip");
}

}  // namespace ca

// Rows of activations or weights brought to 8 bits with a scale each: scale = largest magnitude / 127, codes = round-half-even(127 x /
// largest).  Memory bound: x is read once (rows of up to kHeld vectors a lane stay in registers between the two passes over them)
// and the codes written once, padded with zeros to the products' step of 256.
#include <hip/hip_runtime.h>

#include "ca_internal.hpp"

namespace ca {
namespace {

#include "rope_device.hpp"
#include "quantize_device.hpp"

constexpr int kHeld = 4;                          // vectors of eight values that a lane keeps

template <typename T>
struct RowLoad;
template <>
struct RowLoad<uint16_t> {
  static __device__ __forceinline__ float at(const uint16_t* p) { return __uint_as_float(uint32_t(*p) << 16); }
};
template <>
struct RowLoad<float> {
  static __device__ __forceinline__ float at(const float* p) { return *p; }
};

// values 8 v .. +7 of a row of k; those behind its end are zero.  kVec: rows are 16-byte aligned
template <typename T, bool kVec>
__device__ __forceinline__ void load_values(const T* row, int v, int k, float* x) {
  if (kVec && 8 * v + 8 <= k) {
    Vec8<T> e;
    e.load(row + 8 * v);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = e.v[j];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = 8 * v + j < k ? RowLoad<T>::at(row + 8 * v + j) : 0.f;
  }
}

struct QuantizeArgs {
  const void* x;
  int8_t* codes;
  float* scales;
  int64_t rows, ldx, ld_codes;
  int32_t k, k_padded;
};

template <typename T, bool kVec, int kThreads>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantizeArgs a) {
  constexpr int kRows = 256 / kThreads;           // of a workgroup
  __shared__ uint32_t most_of[4];
  const int t = threadIdx.x % kThreads;
  const int64_t row = int64_t(blockIdx.x) * kRows + threadIdx.x / kThreads;
  if (kThreads == 64 && row >= a.rows) return;    // (a wave's row; with more threads to a row each workgroup has one)
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  const int vectors = (a.k + 7) / 8;
  float held[kHeld][8];
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) load_values<T, kVec>(x, t + i * kThreads, a.k, held[i]);
#pragma unroll
  for (int i = 0; i < kHeld; ++i) most = max(most, magnitude(held[i]));
  for (int v = t + kHeld * kThreads; v < vectors; v += kThreads) {
    float e[8];
    load_values<T, kVec>(x, v, a.k, e);
    most = max(most, magnitude(e));
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) most = max(most, uint32_t(__shfl_xor(int(most), d, 64)));
  if (kThreads > 64) {
    if ((threadIdx.x & 63) == 0) most_of[threadIdx.x >> 6] = most;
    __syncthreads();
    most = max(max(most_of[0], most_of[1]), max(most_of[2], most_of[3]));
  }
  const RowScale s(most);
  int8_t* codes = a.codes + row * a.ld_codes;
  auto leave = [&](int v, const float* e) {
    uint32_t out[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (s.finite) out[j >> 2] |= uint32_t(uint8_t(s.code<T>(e[j]))) << (8 * (j & 3));
    *reinterpret_cast<uint2*>(codes + 8 * v) = uint2{out[0], out[1]};
  };
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (t + i * kThreads < a.k_padded / 8) leave(t + i * kThreads, held[i]);
  for (int v = t + kHeld * kThreads; v < a.k_padded / 8; v += kThreads) {
    float e[8];
    load_values<T, kVec>(x, v, a.k, e);
    leave(v, e);
  }
  if (t == 0) a.scales[row] = row_scale(most);
}

template <typename T, bool kVec>
int32_t enqueue_quantize(const QuantizeArgs& a, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (a.rows >= 1024) {
    const int64_t groups = (a.rows + 3) / 4;
    if (groups > (1 << 24)) return CA_EUNSUPPORTED;
    hipLaunchKernelGGL((quantize_rows_kernel<T, kVec, 64>), dim3(unsigned(groups)), dim3(256), 0, s, a);
  } else {
    hipLaunchKernelGGL((quantize_rows_kernel<T, kVec, 256>), dim3(unsigned(a.rows)), dim3(256), 0, s, a);
  }
  return finish_launch("quantize.hip");
}

}  // namespace

int32_t launch_quantize_rows(int dtype, const void* x, void* codes, float* scales, int64_t rows, int32_t k, int64_t ldx, int64_t ld_codes,
                             void* stream) {
  if (rows == 0) return CA_OK;
  const QuantizeArgs a{x, static_cast<int8_t*>(codes), scales, rows, ldx, ld_codes, k, (k + 255) / 256 * 256};
  const bool vec = (reinterpret_cast<uintptr_t>(x) | uint64_t(ldx) * (dtype == CA_BF16 ? 2 : 4)) % 16 == 0;
  if (dtype == CA_BF16) return vec ? enqueue_quantize<uint16_t, true>(a, stream) : enqueue_quantize<uint16_t, false>(a, stream);
  return vec ? enqueue_quantize<float, true>(a, stream) : enqueue_quantize<float, false>(a, stream);
}

}  // namespace ca

// Rows of activations or weights brought to 8 bits with a scale each: scale = largest magnitude / 127, codes = round-half-even(127 x /
// largest).  Memory bound: x is read once (rows of up to kHeld vectors a lane stay in registers between the two passes over them)
// and the codes written once, padded with zeros to the products' step of 256.
#include <hip/hip_runtime.h>

#include "ca_internal.hpp"

namespace ca {
namespace {

#include "rope_device.hpp"
#include "quantize_device.hpp"

// values 8 v .. +7 of a row of k, aligned as its values are (memory is read 16 bytes at a time all the same); those behind its end are zero
template <typename T>
__device__ __forceinline__ void load_values(const T* row, int v, int k, float* x) {
  struct __attribute__((packed, aligned(sizeof(T)))) Eight { uint32_t w[2 * sizeof(T)]; };
  if (8 * v + 8 <= k) {
    const Eight e = *reinterpret_cast<const Eight*>(row + 8 * v);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      x[j] = sizeof(T) == 4 ? __uint_as_float(e.w[j % (2 * sizeof(T))]) : j & 1 ? bf16_hi(e.w[j / 2]) : bf16_lo(e.w[j / 2]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool there = 8 * v + j < k;
      if constexpr (sizeof(T) == 4)
        x[j] = there ? row[8 * v + j] : 0.f;
      else
        x[j] = there ? __uint_as_float(uint32_t(row[8 * v + j]) << 16) : 0.f;
    }
  }
}

struct QuantizeArgs {
  const void* x;
  int8_t* codes;
  float* scales;
  int64_t rows, ldx, ld_codes;
  int32_t k, k_padded;
};

// kThreads: of a row; kHeld: vectors of eight values that each of them keeps between the two passes
template <typename T, int kThreads, int kHeld>
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
  for (int i = 0; i < kHeld; ++i) load_values<T>(x, t + i * kThreads, a.k, held[i]);
#pragma unroll
  for (int i = 0; i < kHeld; ++i) most = max(most, magnitude(held[i]));
  for (int v = t + kHeld * kThreads; v < vectors; v += kThreads) {
    float e[8];
    load_values<T>(x, v, a.k, e);
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
  auto leave = [&](int v, const float* e) { *reinterpret_cast<uint2*>(codes + 8 * v) = s.codes<T>(e); };
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (t + i * kThreads < a.k_padded / 8) leave(t + i * kThreads, held[i]);
  for (int v = t + kHeld * kThreads; v < a.k_padded / 8; v += kThreads) {
    float e[8];
    load_values<T>(x, v, a.k, e);
    leave(v, e);
  }
  if (t == 0) a.scales[row] = row_scale(most);
}

template <typename T>
int32_t enqueue_quantize(const QuantizeArgs& a, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  // A wave takes a row that its registers hold, if there are rows enough to fill the chip, else a workgroup.  23400 rows of 5120 in bf16 65 us
  // (5.5 TB/s), 95 by waves that read most of a row twice.
  if (a.rows >= 1024 && a.k <= 8 * 64 * 4) {
    const int64_t groups = (a.rows + 3) / 4;
    if (groups >= (1 << 24)) return CA_EUNSUPPORTED;
    hipLaunchKernelGGL((quantize_rows_kernel<T, 64, 4>), dim3(unsigned(groups)), dim3(256), 0, s, a);
  } else {
    if (a.rows >= (1 << 24)) return CA_EUNSUPPORTED;      // (a launch has fewer than 2^32 threads)
    if (a.k <= 8 * 256 * 4)
      hipLaunchKernelGGL((quantize_rows_kernel<T, 256, 4>), dim3(unsigned(a.rows)), dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((quantize_rows_kernel<T, 256, 8>), dim3(unsigned(a.rows)), dim3(256), 0, s, a);
  }
  return finish_launch("quantize.hip");
}

}  // namespace

int32_t launch_quantize_rows(int dtype, const void* x, void* codes, float* scales, int64_t rows, int32_t k, int64_t ldx, int64_t ld_codes,
                             void* stream) {
  if (rows == 0) return CA_OK;
  const QuantizeArgs a{x, static_cast<int8_t*>(codes), scales, rows, ldx, ld_codes, k, (k + 255) / 256 * 256};
  return dtype == CA_BF16 ? enqueue_quantize<uint16_t>(a, stream) : enqueue_quantize<float>(a, stream);
}

}  // namespace ca

// Device-side pieces of the per-head RMS norm that stands ahead of the rotation, shared by the kernels that norm queries and keys:
// they produce the same bits.  A head's D values lie in D / 8 neighbouring lanes (4, 8 or 16), eight to a lane.
// (Included inside namespace ca { namespace { ... } }, behind rope_device.hpp.)
#pragma once

template <int kCtrl>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), kCtrl, 0xf, 0xf, true));
}

// The sum over the `chunks` (4, 8 or 16) neighbouring lanes that hold a head, in all of them: by exchange inside quads, then with
// the mirrored half row and row, which hold the other quads' sums.  Every lane adds the same pairs in the same order.
__device__ __forceinline__ float head_sum(float x, int chunks) {
  x = dpp_add<0xb1>(x);                          // quad_perm [1, 0, 3, 2]
  x = dpp_add<0x4e>(x);                          // quad_perm [2, 3, 0, 1]
  const float eight = dpp_add<0x141>(x);         // row_half_mirror
  const float sixteen = dpp_add<0x140>(eight);   // row_mirror
  return chunks == 16 ? sixteen : (chunks == 8 ? eight : x);
}

// mean(x^2) + eps of the head that the lane's eight values are part of
template <typename T>
__device__ __forceinline__ float head_mean(const Vec8<T>& x, int chunks, float eps) {
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) s = fmaf(x.v[j], x.v[j], s);
  return fmaf(head_sum(s, chunks), 1.f / float(8 * chunks), eps);
}

// 1 / sqrt(mean(x^2) + eps) of x times `by`: 1, or of a head whose squares leave fp32's range (values of 1e19, or of 1e-19 beside a small eps) a power
// of two that brings x back into it first.  (All lanes of a head take the same way, and the sums read no others'.)
template <typename T>
__device__ __forceinline__ float head_rstd(Vec8<T>& x, int chunks, float eps, float* by) {
  float mean = head_mean(x, chunks, eps);
  *by = 1.f;
  if (__builtin_expect(!(mean >= 0x1p-90f && mean <= 0x1p100f), 0)) {
    *by = mean > 1.f ? 0x1p-72f : 0x1p90f;
#pragma unroll
    for (int j = 0; j < 8; ++j) x.v[j] *= *by;
    mean = head_mean(x, chunks, eps * *by * *by);
  }
  return 1.f / sqrtf(mean);
}

// x <- w x / sqrt(mean(x^2) + eps), in fp32
template <typename T>
__device__ __forceinline__ void norm8(Vec8<T>& x, const float* w, int chunks, float eps) {
  float by;
  const float r = head_rstd(x, chunks, eps, &by);
#pragma unroll
  for (int j = 0; j < 8; ++j) x.v[j] = x.v[j] * r * w[j];
}

// Device-side pieces of the 8-bit codes of a row: scale = largest magnitude / 127, code = round-half-even(127 x / largest).
//
// Codes are those of exact arithmetic.  Of bf16 values 127 x is exact in fp32, and a quotient that is not a tie lies at least 2^-16
// (relative) off one: the quotient by the reciprocal with one correction is off by less than 2^-23, and it is exact where the
// quotient is representable, as ties are.  For fp32 values next to a tie the quotient is formed again in fp64.
// (Included inside namespace ca { namespace { ... } }, behind rope_device.hpp.)
#pragma once

__device__ __forceinline__ uint32_t magnitude(const float* x) {      // as bits: NaN above infinity above all others
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(x[j]) & 0x7fffffffu);
  return m;
}

// A row's quotients: values and largest magnitude are brought near 1 by a power of two first where 127 x or the reciprocal would
// leave the range of fp32.
struct RowScale {
  float by127, most, inv;                         // most: the largest magnitude after that
  bool finite;
  __device__ __forceinline__ explicit RowScale(uint32_t bits) {
    const float m = __uint_as_float(bits), by = m > 0x1p100f ? 0x1p-64f : (m < 0x1p-64f ? 0x1p80f : 1.f);
    finite = bits < 0x7f800000u;
    by127 = 127.f * by;
    most = m * by;
    inv = finite && bits != 0 ? 1.f / most : 0.f;
  }
  // the code of x in the low eight bits: 1.5 2^23 is added, whose last place is 1, so that the sum's rounding is the code's
  template <typename T>
  __device__ __forceinline__ uint32_t code(float x) const {
    const float t = x * by127;
    float q = t * inv;
    q = fmaf(fmaf(-q, most, t), inv, q);
    if (sizeof(T) == 4 && fabsf(fabsf(q - truncf(q)) - 0.5f) < 1e-4f) q = float(rint(double(x) * double(by127) / double(most)));
    return __float_as_uint(q + 12582912.f);
  }
  template <typename T>
  __device__ __forceinline__ uint2 codes(const float* x) const {
    uint32_t out[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t lo = __builtin_amdgcn_perm(code<T>(x[4 * i + 1]), code<T>(x[4 * i]), 0x0c0c0400);
      const uint32_t hi = __builtin_amdgcn_perm(code<T>(x[4 * i + 3]), code<T>(x[4 * i + 2]), 0x04000c0c);
      out[i] = finite ? lo | hi : 0;
    }
    return uint2{out[0], out[1]};
  }
};

__device__ __forceinline__ float row_scale(uint32_t most) {
  return most < 0x7f800000u ? __uint_as_float(most) / 127.f : __uint_as_float(0x7fc00000u);
}

// the codes of eight bf16 values
__device__ __forceinline__ uint2 row_codes(const RowScale& s, const U4& v) {
  const float x[8] = {bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y), bf16_lo(v.z), bf16_hi(v.z), bf16_lo(v.w), bf16_hi(v.w)};
  return s.codes<uint16_t>(x);
}

// What the kernels of the 8-bit linear map and of the gated projections share: arguments, products, epilogues.
// (Included inside namespace ca { namespace { ... } }, behind rope_device.hpp, gemm_tiles.hpp and gemm_tile_kernel.hpp.)
#pragma once

typedef __attribute__((ext_vector_type(4))) int32_t i32x4;

struct OpArgs {
  const void* x;                                  // [M][ldx bytes]
  const void* w;                                  // [N][ldw bytes]; gated: the gate's
  void* y;                                        // bf16 [M][ldy]
  const void* w2;                                 // gated: the up projection's weights [N][ldw2 bytes]; 8 bits: scales of w's rows
  const float* xs;                                // 8 bits: scales of x's rows
  uint16_t* g;                                    // gated, training: both projections, or null
  uint16_t* u;
  int64_t ldy, ld_saved;                          // in elements
  int32_t M, N, K, ldx, ldw, ldw2;                // K in bytes of a row: a multiple of 256
  int32_t tiles_m, tiles_n, more;                 // as in LinearArgs
  float act0, act1;                               // gated: act(g) = g sigmoid(g (act0 + act1 g^2))
};

// silu and gelu (its tanh form) are both g sigmoid(p), p = g (act0 + act1 g^2): tanh(z) = 2 sigmoid(2z) - 1.  g is held within 1e4
// for p, where the sigmoid is 0 or 1 long before, so that the cube of a large g does not overflow against a factor of zero.
__device__ __forceinline__ float act_sigmoid(float g, float act0, float act1, float* p_over_g) {
  const float c = __builtin_amdgcn_fmed3f(g, -1e4f, 1e4f);
  *p_over_g = fmaf(c * c, act1, act0);
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(c * *p_over_g * -1.44269504088896341f));
}
__device__ __forceinline__ float gated_value(float g, float u, float act0, float act1) {
  float p;
  return g * act_sigmoid(g, act0, act1, &p) * u;
}

struct I8 {
  struct Products {                               // of codes: the sums are whole numbers, exact up to 2^17 of k
    using Frag = i32x4;
    using Sums = i32x4;
    static __device__ __forceinline__ Sums multiply(const Frag& w, const Frag& x, const Sums& c) {
      return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, c, 0, 0, 0);
    }
  };
  static constexpr bool kGated = false;
};
struct Gated {
  using Products = Bf16Products;
  static constexpr bool kGated = true;
};

// y = sum * scale of the token * scale of the channel, in fp32; rounded to bf16 once by the caller
__device__ __forceinline__ float scaled(int32_t sum, float xs, float ws) { return float(sum) * xs * ws; }

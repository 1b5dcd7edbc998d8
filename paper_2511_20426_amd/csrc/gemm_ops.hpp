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
  float* g;                                       // gated, training: both projections in blocks (saved_at), or null
  float* u;
  int64_t ldy;                                    // in elements
  int32_t M, N, K, ldx, ldw, ldw2;                // K in bytes of a row: a multiple of 256
  int32_t tiles_m, tiles_n, more;                 // as in LinearArgs
  int32_t k_values;                               // 8 bits of values that are made codes on the way: values of a row; in parts: stages of one
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
  static constexpr bool kGated = false, kPart = false;
};
struct Gated {
  using Products = Bf16Products;
  static constexpr bool kGated = true, kPart = false;
};
struct PlainPart {                                // sums of a part of k, in fp32, to g [part][M][N]
  using Products = Bf16Products;
  static constexpr bool kGated = false, kPart = true;
};

// Where four values of a projection from column n (a multiple of four) of row m on lie among the saved ones of N columns: in blocks of 16
// rows and 32 columns, of each first the four columns from 0, 8, 16, 24 of every row, then those from 4, 12, 20, 28.  So the accumulators of a
// matrix instruction leave in one piece (gen_gemm_rows.py).  In rows, 16 bytes a lane 32 apart, a training step of
// 4680 x 4096 x 1536 took 445 us, 397 in blocks and past the caches (400 left in them).
__device__ __forceinline__ int64_t saved_at(int m, int n, int N) {
  return (int64_t(m >> 4) * ((N + 31) >> 5) + (n >> 5)) * 512 + (n >> 2 & 1) * 256 + ((n >> 3 & 3) * 16 + (m & 15)) * 4;
}

// y = sum * scale of the token * scale of the channel, in fp32; rounded to bf16 once by the caller
__device__ __forceinline__ float scaled(int32_t sum, float xs, float ws) { return float(sum) * xs * ws; }

// What one of these products may be taken by, cheapest first by a model of what was measured, in nanoseconds (`rows` rows of X and `cols`
// of W to a tile): start + whole rounds of tiles over the CUs x (stages x full + tile) + a last round (stages x stage + tile), the stage
// of a last round between `stage` and `full` from half of the slots on in proportion.
struct OpModel {
  int rows, cols, per_cu, start, stage, full, tile;
};

template <int kN>
int pick_op(const OpModel (&models)[kN], int64_t M, int64_t w_rows, int64_t stages, int n_cu) {
  int64_t best = INT64_MAX;
  int at = 0;
  for (int i = 0; i < kN; ++i) {
    const OpModel& m = models[i];
    const int64_t tiles = ((M + m.rows - 1) / m.rows) * ((w_rows + m.cols - 1) / m.cols), slots = int64_t(n_cu) * m.per_cu, left = tiles % slots;
    const int64_t stage = m.stage + (2 * left > slots ? (m.full - m.stage) * (2 * left - slots) / slots : 0);
    const int64_t cost = m.start + tiles / slots * (stages * m.full + m.tile) + (left > 0 ? stages * stage + m.tile : 0);
    if (cost < best) {
      best = cost;
      at = i;
    }
  }
  return at;
}

enum { kOpRows256, kOpRows192, kOpRows128, kOpTile256x128, kOpTile128, kOpTile64, kOpTile64Wide };

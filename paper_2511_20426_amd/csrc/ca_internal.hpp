// Internal declarations shared by the host metadata, the C-ABI layer and the kernel launchers.
// Not part of the public boundary (that is include/cascade_attn.h).
#pragma once

#include <cstddef>
#include <cstdint>
#include <vector>

#include "cascade_attn.h"

namespace ca {

constexpr int kMaxPairs = 64;      // head_dim <= 128
constexpr int kMaxKvBlocks = 32;   // sink + window + max_inflight
constexpr int kMaxInflight = 8;
// Scratch behind the bf16 pool pages: partial results of the attention kernel's split work items
// (at most kMaxPartials of them, one 256-row tile of fp32 accumulators + reference + row sum each).
constexpr int kMaxPartials = 256;
constexpr size_t kAttnScratchBytes = size_t(kMaxPartials) * 256 * 132 * 4;

// ----------------------------------------------------------------------------- host metadata
// Slot map, tags and the visibility rule; plain C++, no HIP (Sec. 3.3: shared KV pool with a
// rolling window and a sink block; Alg. 1: blocks move NOISY -> CLEAN when they complete tc).
class CacheMeta {
 public:
  static int32_t validate(const ca_config& c);
  explicit CacheMeta(const ca_config& c);

  const ca_config& cfg() const { return cfg_; }
  int block_tokens() const { return L_; }
  int pages_per_block() const { return P_; }
  int n_slots() const { return n_slots_; }
  size_t elem_bytes() const { return cfg_.dtype == CA_BF16 ? 2 : 4; }
  size_t page_elems() const { return size_t(cfg_.page_tokens) * cfg_.head_dim; }
  size_t pair_bytes() const { return 2 * page_elems() * elem_bytes(); }
  size_t page_bytes_total() const { return size_t(n_slots_) * P_ * cfg_.heads * pair_bytes(); }
  size_t pool_bytes() const { return page_bytes_total() + (cfg_.dtype == CA_BF16 ? kAttnScratchBytes : 0); }

  int32_t slot_of(int64_t g, int32_t* slot) const;       // the fixed rule, resident or not
  int32_t find(int64_t g, int32_t* slot) const;          // CA_ENOENT unless resident
  int32_t check_append(int64_t g, int32_t* slot) const;  // what append would do, no change
  void commit_append(int32_t slot, int64_t g, int32_t timestep, int32_t epoch);
  int32_t promote(int64_t g);
  int32_t evict(int64_t g);
  void retag(int32_t epoch);
  int32_t snapshot(ca_slot_info* out, int32_t cap, int32_t* n_out) const;

  // KV sequence of one forward and the block-pair mask.  kv_ids/kv_slots get n_kv entries,
  // n_vis[i] = number of leading KV entries query block i sees (the sequence is ordered so
  // that the visible set of every query block is a prefix).
  int32_t plan_forward(const int64_t* inflight, int32_t n_inflight, int32_t mode,
                       std::vector<int64_t>* kv_ids, std::vector<int32_t>* kv_slots,
                       std::vector<int32_t>* n_vis) const;

  const double* rope_freq() const { return freq_; }      // per pair, kMaxPairs entries

 private:
  ca_config cfg_;
  int L_, P_, n_slots_;
  std::vector<int64_t> block_;
  std::vector<int32_t> state_, timestep_, epoch_;
  double freq_[kMaxPairs];
};

// ----------------------------------------------------------------------------- kernel launchers
struct RopeGeom {
  double freq[kMaxPairs];   // angle per unit position for pair j
  int32_t pairs_t, pairs_h; // pairs [0,pairs_t) use the frame, [pairs_t,pairs_t+pairs_h) the row, rest the col
  int32_t grid_h, grid_w;
  int32_t heads, head_dim;
};

// y = rope(x) on [n_tokens, heads, head_dim]; token n sits at frame first_frame + n/(gh*gw).
int32_t launch_rope_apply(const RopeGeom& g, int dtype, const void* x, void* y, int64_t n_tokens,
                          int64_t first_frame, int64_t tok_stride, int64_t head_stride,
                          int64_t y_tok_stride, int64_t y_head_stride, void* stream);

// Fused K-rotation + K/V page store of n_blocks (1..kMaxInflight) blocks into their slots, one
// launch for all of them (bf16).
int32_t launch_cache_write(const RopeGeom& g, int dtype, int32_t n_blocks, const void* const* k,
                           const void* const* v, int64_t tok_stride, int64_t head_stride,
                           const int64_t* first_frame, int32_t block_tokens, int32_t page_tokens,
                           int32_t pages_per_block, const int32_t* slot, void* pool, void* stream);

// The same with each head of K normed ahead of its rotation (norm_weight: head_dim values of the storage type).
int32_t launch_cache_write_norm(const RopeGeom& g, int dtype, int32_t n_blocks, const void* const* k,
                                const void* const* v, int64_t tok_stride, int64_t head_stride,
                                const int64_t* first_frame, int32_t block_tokens, int32_t page_tokens,
                                int32_t pages_per_block, const int32_t* slot, const void* norm_weight, float norm_eps, void* pool,
                                void* stream);

// Per-head RMS norm and rotation of queries, keys or both (x null: not these) in one pass, and its gradients.
struct NormTensors {
  const void* x;
  const void* w;                                  // head_dim values of the storage type
  const void* dz;                                 // backward: gradient of the result
  void* y;                                        // the result; backward: gradient of x
  int64_t x_tok, x_head, dz_tok, dz_head, y_tok, y_head;
};
int32_t launch_norm_rope(const RopeGeom& g, int dtype, const NormTensors& q, const NormTensors& k, float eps, int64_t n_tokens,
                         int64_t first_frame, void* stream);
size_t norm_rope_backward_bytes(int32_t head_dim);
int32_t launch_norm_rope_backward(const RopeGeom& g, int dtype, const NormTensors& q, const NormTensors& k, float eps, int64_t n_tokens,
                                  int64_t first_frame, float* dq_weight, float* dk_weight, void* workspace, void* stream);

struct AttnPlan {
  int32_t heads, head_dim, page_tokens, pages_per_block, block_tokens;
  int32_t n_q_blocks;                 // query blocks of this launch; query rows are n_q_blocks * block_tokens
  int32_t n_kv;                       // length of the KV sequence
  int32_t kv_slot[kMaxKvBlocks];
  int32_t n_vis[kMaxInflight];        // visible prefix length per query block
  int32_t uniform;                    // every query block sees the same prefix, n_vis[0]
};

int32_t launch_attn_f32(const AttnPlan& p, const void* q, void* out, const void* pool, void* stream);
// scratch: room for max_partials partial results (kAttnScratchBytes / kMaxPartials bytes each) of
// split work items, or nullptr / 0: then no KV walk is split.
int32_t launch_attn_bf16(const AttnPlan& p, int variant, const void* q, void* out, const void* pool,
                         void* scratch, int max_partials, void* stream);
int32_t attn_bf16_variant_ok(int variant);
// The same launch on queries that are not rotated yet: the kernel rotates them as it loads them.
// q is [rows, heads, head_dim] with the given strides; first_frame[i] is the first latent frame of
// query block i of the launch.
struct QRopePlan {
  RopeGeom geom;
  int64_t first_frame[kMaxInflight];
  int64_t tok_stride, head_stride;
};
int32_t launch_attn_bf16_rope(const AttnPlan& p, const QRopePlan& rp, int variant, const void* q, void* out,
                              const void* pool, void* scratch, int max_partials, void* stream);
// The same launch with the partial results in the library's own static device array (one copy per
// GPU, kept for the life of the process) instead of caller memory; CA_ETOOBIG if the split the
// device asks for needs more partial tiles than that array holds.  attn_static_scratch_prepare
// looks the array's address up for the current device ahead of the first launch (errors ignored:
// the launch looks again).
int32_t launch_attn_bf16_static(const AttnPlan& p, int variant, const void* q, void* out, const void* pool,
                                void* stream);
void attn_static_scratch_prepare();

int32_t run_mfma_microbench(int data_kind, int trips, void* scratch, size_t scratch_bytes, void* stream,
                            double* tflops, double* clock_ghz);
int32_t launch_gemm_bf16(const void* x, const void* w, void* y, int64_t M, int32_t N, int32_t K,
                         int64_t ldx, int64_t ldw, int64_t ldy, void* stream);
// What it costs by the model that picks its tile, in nanoseconds
int64_t gemm_bf16_cost(int64_t M, int32_t N, int32_t K, int n_cu);
// The same in tiles of tile_rows (256, 192 or 128) x 256, a workgroup taking several one after the other; gemm_rows_ready
// readies its kernels for stream capture.
int32_t launch_gemm_rows(int tile_rows, const void* x, const void* w, void* y, int32_t M, int32_t N, int32_t K,
                         int64_t ldx, int64_t ldw, int64_t ldy, void* stream);
int32_t gemm_rows_ready();
// ... in a compiled tile (a GemmTile of up to 128 columns), each workgroup one
int32_t launch_gemm_tile(int tile, const void* x, const void* w, void* y, int32_t M, int32_t N, int32_t K,
                         int64_t ldx, int64_t ldw, int64_t ldy, void* stream);
int32_t gemm_tiles_ready();
// The QKV projection of n_blocks blocks (x rows: block b at b * block_tokens; w rows: q|k|v, head,
// dim) with the publication of K/V to the blocks' slots fused into its epilogue; q_out gets the
// packed, unrotated queries [n_blocks * block_tokens][heads * 128].
int32_t launch_gemm_qkv_publish(const RopeGeom& g, int32_t n_blocks, int32_t block_tokens, int32_t pages_per_block,
                                const int32_t* slot, const int64_t* first_frame, const void* x, int64_t ldx,
                                const void* w, int64_t ldw, int32_t K, void* q_out, void* pool, void* stream);
// Rows of x (CA_BF16 or CA_F32) brought to 8 bits: codes [rows][ld_codes], zeros from k to the next multiple of 256.
int32_t launch_quantize_rows(int dtype, const void* x, void* codes, float* scales, int64_t rows, int32_t k, int64_t ldx, int64_t ld_codes,
                             void* stream);
// Y = (X . W') * x_scales * w_scales; rows of X and W hold codes up to the next multiple of 256 of K.
int32_t launch_gemm_i8(const void* x, const float* x_scales, const void* w, const float* w_scales, void* y, int64_t M, int32_t N, int32_t K,
                       int64_t ldx, int64_t ldw, int64_t ldy, void* stream);
// The same of values of X (CA_BF16 or CA_F32), with room in the workspace for their codes [M][K up to 256s] and scales.
int32_t launch_gemm_i8_values(int dtype, const void* x, int64_t ldx, const void* w, const float* w_scales, void* y, int64_t M, int32_t N, int32_t K,
                              int64_t ldw, int64_t ldy, void* workspace, void* stream);
// H = act(X Wg') * (X Wu'); with saved the projections themselves in fp32 as well, the gate's and the up projection's in one half each
inline int64_t gated_saved_values(int64_t M, int32_t F) { return 2 * ((M + 15) / 16 * 16) * ((int64_t(F) + 31) / 32 * 32); }
int32_t launch_gemm_gated(const void* x, const void* w_gate, const void* w_up, void* h, float* saved, int activation, int64_t M, int32_t F,
                          int32_t K, int64_t ldx, int64_t ldwg, int64_t ldwu, int64_t ldh, void* stream);
// act(g) = g sigmoid(g (act0 + act1 g^2))
inline void activation_factors(int activation, float* act0, float* act1) {
  *act0 = activation == CA_GELU ? 1.5957691216057308f : 1.f;                       // 2 sqrt(2 / pi)
  *act1 = activation == CA_GELU ? 1.5957691216057308f * 0.044715f : 0.f;
}
// Where the backward pass of the gated projections keeps what it multiplies: offsets in bytes.
struct GatedWorkspace {
  int64_t Mp, Fp;
  size_t rows, cols, xt, wt, parts, bytes;
};
GatedWorkspace gated_workspace(int64_t M, int32_t F, int32_t K);
int32_t launch_gated_backward(const void* dh, const void* x, const void* w_gate, const void* w_up, const float* saved, int activation,
                              void* dx, void* dw_gate, void* dw_up, int64_t M, int32_t F, int32_t K, int64_t lddh, int64_t ldx, int64_t ldwg,
                              int64_t ldwu, int64_t lddx, int64_t lddw, void* workspace, void* stream);
// Layer norm of rows and its gradients; groups of equally many consecutive rows have weights and biases of their own (null: none).
struct RowNorm {
  const void* x;
  const void* w;
  const void* b;
  int64_t rows, groups, ldx, ldy, ldw;
  int32_t width, dtype, w_dtype;
  float eps;
};
int32_t launch_layer_norm(const RowNorm& n, const void* y, void* stream);
size_t layer_norm_backward_bytes(int64_t rows, int32_t width, int64_t groups);
int32_t launch_layer_norm_backward(const RowNorm& n, const void* dy, int64_t lddy, void* dx, float* dw, float* db, void* workspace, void* stream);
// The AdamW step (tensors without a gradient or values are left out), and what states in 8 bits stand for: n values, a multiple of 256
int32_t launch_adamw(const ca_adamw_tensor* tensors, const ca_adamw_tensor* tensors_dev, int32_t n_tensors, int32_t state_bits, double lr, double beta1,
                     double beta2, double eps, double weight_decay, double grad_scale, void* stream);
int32_t launch_adamw_values(const void* m, const void* v, const float* m_scale, const float* v_scale, float* m_out, float* v_out, int64_t n, void* stream);
// Y = X W' + (s_g X A_g') B_g' with g = index of the row (down: A [adapters][rank][K], up: B [adapters][N][rank]; rank 32, 64 or 128), low [2][M][rank] gets
// s_g X A_g' and what its rounding left.  Backward (w: the weights transposed [K][N], ldy: the row stride of dX): the gradients of X and of the adapters' first rank_used; those
// that are null are left out.
struct AdaptedLinear {
  const void* x;
  const void* w;
  const void* down;
  const void* up;
  const float* scales;
  const int32_t* index;
  int64_t M, ldx, ldw, ldy;
  int32_t N, K, adapters, rank;
};
size_t adapted_bytes(int64_t M, int32_t rank);
int32_t launch_gemm_adapted(const AdaptedLinear& p, void* y, void* low, void* workspace, void* stream);
size_t adapted_backward_bytes(int64_t M, int32_t N, int32_t K, int32_t adapters, int32_t rank);
int32_t launch_adapted_backward(const AdaptedLinear& p, const void* dy, int64_t lddy, const void* low, int32_t rank_used, void* dx, void* d_down, void* d_up,
                                void* workspace, void* stream);
// Per-device facts and one-time kernel attributes, cached for up to kMaxDevices devices (thread
// safe: the cached values are idempotent and written with relaxed atomics).
constexpr int kMaxDevices = 64;
int32_t device_cu_count(int* n_cu);                                   // of the current device
// A call may take one of several kernels by its size.  All of them get their LDS attribute with the first call of
// any size, so that one eager call readies every later one for stream capture.
struct KernelLds {
  const void* kernel;
  int bytes;
};
enum LdsSlot { kLdsAttn, kLdsAttnRope, kLdsGemm, kLdsGemmRows, kLdsGemmPublish, kLdsI8, kLdsGated, kLdsGatedBackward, kLdsAdapted, kLdsSlots };
int32_t ensure_dynamic_lds(const KernelLds* kernels, int n, LdsSlot slot);   // slot: which set of kernels
int32_t finish_launch(const char* what);   // launchers end with this: CA_OK, or CA_EDEVICE after recording HIP's last error
int32_t device_failure(const char* what, int hip_error);   // records the text, clears HIP's last error, returns CA_EDEVICE
const char* last_device_error();

}  // namespace ca

namespace ca {

inline RopeGeom rope_geom(const CacheMeta& m) {
  RopeGeom g{};
  const ca_config& c = m.cfg();
  for (int i = 0; i < kMaxPairs; ++i) g.freq[i] = m.rope_freq()[i];
  g.pairs_t = c.rope_dim_t / 2;
  g.pairs_h = c.rope_dim_h / 2;
  g.grid_h = c.grid_h;
  g.grid_w = c.grid_w;
  g.heads = c.heads;
  g.head_dim = c.head_dim;
  return g;
}

// A [token, head, dim] view must address whole 8-element groups on 16-byte (bf16) or
// 32-byte (fp32) boundaries: the kernels move 8 elements at a time.
inline bool strides_ok(const ca_config& c, const void* p, int64_t tok_stride, int64_t head_stride) {
  if (tok_stride < 0 || head_stride < 0) return false;
  if (head_stride < c.head_dim && c.heads > 1) return false;
  if (tok_stride < c.head_dim) return false;
  if ((tok_stride % 8) || (head_stride % 8)) return false;
  if (reinterpret_cast<uintptr_t>(p) % 16) return false;
  return true;
}

}  // namespace ca

struct ca_ctx {
  ca::CacheMeta meta;
  void* pool;
  size_t pool_bytes;
  int32_t variant;
  explicit ca_ctx(const ca_config& c) : meta(c), pool(nullptr), pool_bytes(0), variant(0) {}
};

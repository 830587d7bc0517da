// Host-side launchers of the token operators' kernels (include/dycl_tokens.h).
// They do not check arguments: the C entry points validate every one before any
// launch, and each launcher is called with at least one row.  Each launch is
// checked before the next one that reads what it writes.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace dycl {
namespace k {

// throws HipError if the launch just made was refused
void launched(const char* what);

struct NormArgs {
  const void *x, *y, *gate;      // [n][d]; y, gate may be null
  int x_f32, y_f32;
  int64_t ldx, ldy, ldg;
  int gate_act;                  // 0 none, 1 sigmoid, 2 SiLU
  const float* row_gate;         // [n] or null
  const float* channel_scale;    // [d] or null
  float residual_scale;
  int post, pre;                 // dycl_norm_kind
  const float *post_w, *post_b, *pre_w, *pre_b;
  float eps;
  int64_t n;
  int d;
  void *h, *u;                   // null: not written
  int u_f32;
  int64_t ldh, ldu;
};
constexpr int kNormMaxD = 32768;
void token_norm(const NormArgs& a, hipStream_t stream);

struct RouteArgs {
  const void* logits;
  int logits_f32;
  int64_t ldl;
  const float* bias;
  const uint8_t* mask;
  int64_t n;
  int experts, groups, top_groups, k, sigmoid, renormalise;
  float scale;
  int32_t* ids;
  float* weights;
  int32_t *offsets, *order, *slots;   // null: no partition
  void* workspace;
};
constexpr int kRouteMaxExperts = 1024, kRouteMaxK = 32, kRouteMaxGroups = 64;
size_t token_route_workspace(int64_t n, int experts, int k);
void token_route(const RouteArgs& a, hipStream_t stream);
void token_route_empty(int32_t* offsets, int experts, hipStream_t stream);

// Packed weights: per layer ceil(n / 32) strips of 32 outputs; a strip is
// ceil(k / 64) * 2 steps of 32 inputs; a step is 2 (gated: 4) blocks of 16
// outputs x 32 inputs, each the 64 lanes' 16-byte operands of
// v_mfma_f32_16x16x32_bf16 in lane order.
constexpr int kStrip = 32;
inline int strips_of(int n) { return (n + kStrip - 1) / kStrip; }
inline int steps_of(int k) { return (k + 63) / 64 * 2; }
inline size_t packed_elements(int experts, int n, int k, int gated) {
  return static_cast<size_t>(experts) * strips_of(n) * steps_of(k) * (gated ? 4 : 2) * 512;
}
void token_pack(const uint16_t* w, const uint16_t* gate, int experts, int n, int k, uint16_t* packed, hipStream_t stream);

enum TokenAct { TACT_NONE = 0, TACT_RELU = 1, TACT_GELU = 2, TACT_SILU = 3 };

// One product over all rows of one layer (offsets null), or over each
// expert's rows (rows offsets[e] .. offsets[e + 1] - 1 of the layer's output).
struct ProductArgs {
  const uint16_t* x;             // rows of K values, 16-byte aligned, pitch a multiple of 8
  int64_t ldx;
  const int32_t* order;          // null, or: row r of the product reads x row order[r] / order_k
  int order_k;
  int64_t x_rows;                // rows of x (with order)
  int far;                       // (set by token_product: offsets into x do not fit 32 bits)
  const int32_t* offsets;        // null, or [experts + 1]
  int experts;
  int64_t rows;                  // rows (with offsets: an upper bound of their number)
  int K;                         // inputs: the x row's values past K up to a multiple of 8 are 0
  const uint16_t* w;             // packed
  int N, gated;
  const float *bias, *gate_bias; // [experts][N] or null
  int act;
  const uint16_t* residual;
  int64_t ldr;
  void* y;
  int y_f32;
  int64_t ldy;
  int N_store;                   // columns written (>= N: the ones past N are 0)
};
// The shape that a product takes, by its rows, sizes and experts; -1 where none's tiles
// are as few as a launch holds.
int token_product_shape(const ProductArgs& a);
// a shape's rows and outputs per tile, and workgroups per CU
void token_product_tile(int shape, bool gated, int tile[3]);
void token_product(const ProductArgs& a, int shape, hipStream_t stream);

// rows [n][d] of any alignment to rows of pitch `ldo` (a multiple of 8), zero-padded
void token_align_rows(const uint16_t* x, int64_t ldx, int64_t n, int d, uint16_t* out, int64_t ldo, hipStream_t stream);

// out[t] = residual[t] + sum_j weights[t][j] * part[slots[t][j]]
struct CombineArgs {
  const float* part;             // rows of pitch ldp (a multiple of 8), 16-byte aligned
  int64_t ldp;
  const float* weights;
  const int32_t* slots;
  int64_t n;
  int k, d;
  const uint16_t* residual;
  int64_t ldr;
  uint16_t* out;
  int64_t ldo;
};
void token_combine(const CombineArgs& a, hipStream_t stream);

}  // namespace k
}  // namespace dycl

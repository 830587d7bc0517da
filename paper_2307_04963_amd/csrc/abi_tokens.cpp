// C entry points of the token operators (include/dycl_tokens.h): argument
// checks, workspace layout and launches.  Nothing thrown crosses them.
#include "../../include/dycl_tokens.h"

#include <string>

#include "abi.hpp"
#include "tokens.hpp"

namespace {

using dycl::fail;
using dycl::guarded;
using namespace dycl::k;

struct Bad : std::runtime_error {
  using std::runtime_error::runtime_error;
};

// throws (mapped to DYCL_E_INVALID) unless ok
void need(bool ok, const char* op, const char* what) {
  if (!ok) throw Bad(std::string(op) + ": " + what);
}

bool at(const void* p, size_t align) { return reinterpret_cast<uintptr_t>(p) % align == 0; }

bool type_ok(int t) { return t == DYCL_BF16 || t == DYCL_F32; }

size_t size_of(int t) { return t == DYCL_F32 ? 4 : 2; }

size_t pad256(size_t v) { return (v + 255) / 256 * 256; }

bool rows_aligned(const uint16_t* x, int64_t ldx, int k) { return at(x, 16) && ldx % 8 == 0 && k % 8 == 0; }

int64_t round8(int64_t v) { return (v + 7) / 8 * 8; }

constexpr int kMaxWidth = 1 << 20, kMaxLayers = 1024;

bool layers_ok(int experts, int n, int k) {
  return experts >= 1 && experts <= kMaxLayers && n >= 1 && n <= kMaxWidth && k >= 1 && k <= kMaxWidth;
}

constexpr int64_t kMaxRows = int64_t(1) << 31, kMaxPitch = int64_t(1) << 40;

const char* const kTooMany = "more tiles of results than a launch holds";

bool pitch_ok(int64_t ld, int64_t width) { return ld >= width && ld < kMaxPitch; }

}  // namespace

namespace dycl {
namespace k {

void launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) throw HipError(std::string(what) + ": launch failed: " + hipGetErrorString(e));
}

}  // namespace k
}  // namespace dycl

extern "C" {

int dycl_op_norm(const void* x, int x_type, int64_t ldx, const void* y, int y_type, int64_t ldy, const void* gate,
                 int64_t ldg, int gate_act, const float* row_gate, const float* channel_scale, float residual_scale,
                 int post, const float* post_weight, const float* post_bias, int pre, const float* pre_weight,
                 const float* pre_bias, float eps, int64_t n, int d, void* h, int64_t ldh, void* u, int u_type,
                 int64_t ldu, void* hip_stream) {
  return guarded([&] {
    const char* op = "dycl_op_norm";
    need(n >= 0 && n < kMaxRows, op, "n outside [0, 2^31)");
    need(d >= 1 && d <= kNormMaxD, op, "d outside [1, 32768]");
    need(type_ok(x_type) && (!y || type_ok(y_type)) && (!u || type_ok(u_type)), op, "unknown element type");
    need(post >= 0 && post <= DYCL_NORM_LAYER && pre >= 0 && pre <= DYCL_NORM_LAYER, op, "unknown norm");
    need(gate_act >= 0 && gate_act <= 2, op, "unknown gate activation");
    need(eps >= 0.f, op, "negative or NaN eps");
    if (n == 0) return static_cast<int>(DYCL_OK);   // (empty tensors' pointers are null)
    need(y || (post == DYCL_NORM_NONE && !gate && !row_gate && !channel_scale && !post_weight && !post_bias), op,
         "a post norm or a gate without y");
    need(post != DYCL_NORM_NONE || (!post_weight && !post_bias), op, "post weights without a post norm");
    need(u || pre == DYCL_NORM_NONE, op, "a pre norm without u");
    need(pre != DYCL_NORM_NONE || (!pre_weight && !pre_bias), op, "pre weights without a pre norm");
    need(h || u, op, "neither h nor u");
    need(x, op, "null x");
    need(pitch_ok(ldx, d) && (!y || pitch_ok(ldy, d)) && (!gate || pitch_ok(ldg, d)) && (!h || pitch_ok(ldh, d)) &&
             (!u || pitch_ok(ldu, d)),
         op, "a row pitch below d");
    const int yt = y ? y_type : DYCL_BF16;
    need(at(x, size_of(x_type)) && at(h, size_of(x_type)) && at(y, size_of(yt)) && at(gate, size_of(yt)) &&
             (!u || at(u, size_of(u_type))) && at(row_gate, 4) && at(channel_scale, 4) && at(post_weight, 4) &&
             at(post_bias, 4) && at(pre_weight, 4) && at(pre_bias, 4),
         op, "a pointer not aligned to its element");
    need(h != x || ldh == ldx, op, "h is x with another pitch");
    need(!h || h != y || (ldh == ldy && yt == x_type), op, "h is y with another pitch or type");
    need(!u || (u != x && u != y && u != gate && u != h), op, "u is another of the tensors");
    need(!h || h != gate, op, "h is the gate");
    NormArgs a;
    a.x = x;
    a.y = y;
    a.gate = gate;
    a.x_f32 = x_type == DYCL_F32;
    a.y_f32 = yt == DYCL_F32;
    a.ldx = ldx;
    a.ldy = ldy;
    a.ldg = ldg;
    a.gate_act = gate_act;
    a.row_gate = row_gate;
    a.channel_scale = channel_scale;
    a.residual_scale = residual_scale;
    a.post = post;
    a.pre = pre;
    a.post_w = post_weight;
    a.post_b = post_bias;
    a.pre_w = pre_weight;
    a.pre_b = pre_bias;
    a.eps = eps;
    a.n = n;
    a.d = d;
    a.h = h;
    a.u = u;
    a.u_f32 = u && u_type == DYCL_F32;
    a.ldh = ldh;
    a.ldu = ldu;
    token_norm(a, static_cast<hipStream_t>(hip_stream));
    return static_cast<int>(DYCL_OK);
  });
}

size_t dycl_op_route_workspace(int64_t n, int experts, int k) {
  if (n < 1 || n >= kMaxRows || experts < 1 || experts > kRouteMaxExperts || k < 1) return 0;
  return token_route_workspace(n, experts, k);
}

int dycl_op_route(const void* logits, int logits_type, int64_t ldl, const float* bias, const uint8_t* mask, int64_t n,
                  int experts, int groups, int top_groups, int k, int score, int renormalise, float scale, int32_t* ids,
                  float* weights, int32_t* offsets, int32_t* order, int32_t* slots, void* workspace,
                  size_t workspace_bytes, void* hip_stream) {
  return guarded([&] {
    const char* op = "dycl_op_route";
    need(experts >= 1 && experts <= kRouteMaxExperts, op, "experts outside [1, 1024]");
    need(k >= 1 && k <= experts && k <= kRouteMaxK, op, "k outside [1, min(experts, 32)]");
    need(groups >= 1 && groups <= kRouteMaxGroups && experts % groups == 0, op,
         "groups outside [1, 64] or not dividing experts");
    need(top_groups >= 1 && top_groups <= groups, op, "top_groups outside [1, groups]");
    need(score == 0 || score == 1, op, "unknown score");
    need(type_ok(logits_type), op, "unknown element type");
    need(n >= 0 && n < kMaxRows && n * k < kMaxRows, op, "n * k outside [0, 2^31)");
    need((!offsets && !order && !slots) || (offsets && (n == 0 || (order && slots))), op,
         "offsets, order and slots are given together");
    need(at(offsets, 4) && at(order, 4) && at(slots, 4) && at(ids, 4) && at(weights, 4) && at(bias, 4) &&
             at(logits, size_of(logits_type)) && at(workspace, 8),
         op, "a pointer not aligned to its element");
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (n == 0) {
      if (offsets) token_route_empty(offsets, experts, s);
      return static_cast<int>(DYCL_OK);
    }
    need(logits && ids && weights, op, "null logits, ids or weights");
    need(pitch_ok(ldl, experts), op, "a row pitch below experts");
    const size_t bytes = offsets ? token_route_workspace(n, experts, k) : 0;
    need(bytes == 0 || (workspace && workspace_bytes >= bytes), op, "workspace too small");
    RouteArgs a;
    a.logits = logits;
    a.logits_f32 = logits_type == DYCL_F32;
    a.ldl = ldl;
    a.bias = bias;
    a.mask = mask;
    a.n = n;
    a.experts = experts;
    a.groups = groups;
    a.top_groups = top_groups;
    a.k = k;
    a.sigmoid = score;
    a.renormalise = renormalise != 0;
    a.scale = scale;
    a.ids = ids;
    a.weights = weights;
    a.offsets = offsets;
    a.order = order;
    a.slots = slots;
    a.workspace = workspace;
    token_route(a, s);
    return static_cast<int>(DYCL_OK);
  });
}

size_t dycl_op_linear_packed_bytes(int experts, int n, int k, int gated) {
  return layers_ok(experts, n, k) ? packed_elements(experts, n, k, gated) * 2 : 0;
}

int dycl_op_linear_tile(int64_t rows, int n, int k, int gated, int experts, int32_t tile[3]) {
  return guarded([&] {
    const char* op = "dycl_op_linear_tile";
    need(layers_ok(experts ? experts : 1, n, k), op, "experts outside [0, 1024], or n or k outside [1, 2^20]");
    need(rows >= 1 && rows < kMaxRows, op, "rows outside [1, 2^31)");
    need(tile, op, "null tile");
    ProductArgs a{};
    const int32_t some = 0;
    a.offsets = experts ? &some : nullptr;   // (only whether there are any)
    a.experts = experts ? experts : 1;
    a.rows = rows;
    a.K = k;
    a.N = n;
    a.gated = gated != 0;
    const int shape = token_product_shape(a);
    need(shape >= 0, op, kTooMany);
    token_product_tile(shape, gated != 0, tile);
    return static_cast<int>(DYCL_OK);
  });
}

int dycl_op_linear_pack(const uint16_t* w, const uint16_t* gate, int experts, int n, int k, uint16_t* packed,
                        size_t packed_bytes, void* hip_stream) {
  return guarded([&] {
    const char* op = "dycl_op_linear_pack";
    need(layers_ok(experts, n, k), op, "experts outside [1, 1024], or n or k outside [1, 2^20]");
    need(w && packed, op, "null weights or output");
    need(at(w, 2) && at(gate, 2) && at(packed, 16), op, "a pointer not aligned (packed: 16 bytes)");
    need(packed_bytes >= packed_elements(experts, n, k, gate != nullptr) * 2, op, "output too small");
    token_pack(w, gate, experts, n, k, packed, static_cast<hipStream_t>(hip_stream));
    return static_cast<int>(DYCL_OK);
  });
}

size_t dycl_op_linear_workspace(const uint16_t* x, int64_t ldx, int64_t m, int k, int n, int gated) {
  (void)n;
  (void)gated;
  if (m < 1 || m >= kMaxRows || k < 1 || k > kMaxWidth) return 0;
  return rows_aligned(x, ldx, k) ? 0 : static_cast<size_t>(m) * round8(k) * 2;
}

int dycl_op_linear(const uint16_t* x, int64_t ldx, int64_t m, int k, const uint16_t* packed, int n, int gated,
                   const float* bias, const float* gate_bias, int act, const uint16_t* residual, int64_t ldr, void* y,
                   int y_type, int64_t ldy, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return guarded([&] {
    const char* op = "dycl_op_linear";
    need(layers_ok(1, n, k), op, "n or k outside [1, 2^20]");
    need(m >= 0 && m < kMaxRows, op, "m outside [0, 2^31)");
    need(act >= 0 && act <= TACT_SILU, op, "unknown activation");
    need(type_ok(y_type), op, "unknown element type");
    need(gated || !gate_bias, op, "a gate bias without a gate");
    if (m == 0) return static_cast<int>(DYCL_OK);
    need(x && packed && y, op, "null x, packed weights or y");
    need(pitch_ok(ldx, k) && pitch_ok(ldy, n) && (!residual || pitch_ok(ldr, n)), op, "a row pitch below the row");
    need(at(x, 2) && at(packed, 16) && at(bias, 4) && at(gate_bias, 4) && at(residual, 2) && at(y, size_of(y_type)) &&
             at(workspace, 16),
         op, "a pointer not aligned to its element (packed, workspace: 16 bytes)");
    need(y != x, op, "y is x");
    need(y != residual || (y_type == DYCL_BF16 && ldy == ldr), op, "y is the residual with another pitch or type");
    const size_t bytes = dycl_op_linear_workspace(x, ldx, m, k, n, gated);
    need(bytes == 0 || (workspace && workspace_bytes >= bytes), op, "workspace too small");
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    ProductArgs a{};
    a.x = x;
    a.ldx = ldx;
    a.order_k = 1;
    a.experts = 1;
    a.rows = m;
    a.K = k;
    a.w = packed;
    a.N = n;
    a.gated = gated != 0;
    a.bias = bias;
    a.gate_bias = gate_bias;
    a.act = act;
    a.residual = residual;
    a.ldr = ldr;
    a.y = y;
    a.y_f32 = y_type == DYCL_F32;
    a.ldy = ldy;
    a.N_store = n;
    const int shape = token_product_shape(a);
    need(shape >= 0, op, kTooMany);
    if (!rows_aligned(x, ldx, k)) {
      uint16_t* rows = static_cast<uint16_t*>(workspace);
      token_align_rows(x, ldx, m, k, rows, round8(k), s);
      a.x = rows;
      a.ldx = round8(k);
    }
    token_product(a, shape, s);
    return static_cast<int>(DYCL_OK);
  });
}

size_t dycl_op_experts_workspace(const uint16_t* x, int64_t ldx, int64_t n, int experts, int k, int d, int f) {
  if (n < 1 || k < 1 || n >= kMaxRows || n * k >= kMaxRows || !layers_ok(experts, d, f)) return 0;
  const size_t pairs = static_cast<size_t>(n) * k;
  const size_t rows = rows_aligned(x, ldx, d) ? 0 : pad256(static_cast<size_t>(n) * round8(d) * 2);
  return rows + pad256(pairs * strips_of(f) * kStrip * 2) + pad256(pairs * strips_of(d) * kStrip * 4);
}

int dycl_op_experts(const uint16_t* x, int64_t ldx, int64_t n, int d, int f, int experts, int k,
                    const uint16_t* packed1, int gated, const float* bias1, const float* gate_bias1, int act,
                    const uint16_t* packed2, const float* bias2, const float* weights, const int32_t* offsets,
                    const int32_t* order, const int32_t* slots, const uint16_t* residual, int64_t ldr, uint16_t* out,
                    int64_t ldo, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return guarded([&] {
    const char* op = "dycl_op_experts";
    need(layers_ok(experts, d, f), op, "experts outside [1, 1024], or d or f outside [1, 2^20]");
    need(k >= 1 && k <= experts && k <= kRouteMaxK, op, "k outside [1, min(experts, 32)]");
    need(n >= 0 && n < kMaxRows && n * k < kMaxRows, op, "n * k outside [0, 2^31)");
    need(act >= 0 && act <= TACT_SILU, op, "unknown activation");
    need(gated || !gate_bias1, op, "a gate bias without a gate");
    if (n == 0) return static_cast<int>(DYCL_OK);
    need(x && packed1 && packed2 && weights && offsets && order && slots && out, op, "a null tensor, list or weights");
    need(pitch_ok(ldx, d) && pitch_ok(ldo, d) && (!residual || pitch_ok(ldr, d)), op, "a row pitch below d");
    need(at(x, 2) && at(packed1, 16) && at(packed2, 16) && at(bias1, 4) && at(gate_bias1, 4) && at(bias2, 4) &&
             at(weights, 4) && at(offsets, 4) && at(order, 4) && at(slots, 4) && at(residual, 2) && at(out, 2) &&
             at(workspace, 16),
         op, "a pointer not aligned to its element (packed, workspace: 16 bytes)");
    need(out != residual || ldo == ldr, op, "out is the residual with another pitch");
    need(workspace && workspace_bytes >= dycl_op_experts_workspace(x, ldx, n, experts, k, d, f), op,
         "workspace too small");
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const size_t pairs = static_cast<size_t>(n) * k;
    const int64_t fp = static_cast<int64_t>(strips_of(f)) * kStrip, dp = static_cast<int64_t>(strips_of(d)) * kStrip;
    char* ws = static_cast<char*>(workspace);
    uint16_t* hidden = reinterpret_cast<uint16_t*>(ws);
    ws += pad256(pairs * fp * 2);
    float* part = reinterpret_cast<float*>(ws);
    ws += pad256(pairs * dp * 4);

    ProductArgs a{};
    a.x = x;
    a.ldx = ldx;
    a.order = order;
    a.order_k = k;
    a.x_rows = n;
    a.offsets = offsets;
    a.experts = experts;
    a.rows = static_cast<int64_t>(pairs);
    a.K = d;
    a.w = packed1;
    a.N = f;
    a.gated = gated != 0;
    a.bias = bias1;
    a.gate_bias = gate_bias1;
    a.act = act;
    a.y = hidden;
    a.ldy = fp;
    a.N_store = static_cast<int>(fp);

    ProductArgs b{};
    b.x = hidden;
    b.ldx = fp;
    b.order_k = 1;
    b.offsets = offsets;
    b.experts = experts;
    b.rows = a.rows;
    b.K = f;
    b.w = packed2;
    b.N = d;
    b.bias = bias2;
    b.act = TACT_NONE;
    b.y = part;
    b.y_f32 = 1;
    b.ldy = dp;
    b.N_store = static_cast<int>(dp);

    const int first = token_product_shape(a), second = token_product_shape(b);
    need(first >= 0 && second >= 0, op, kTooMany);
    if (!rows_aligned(x, ldx, d)) {
      uint16_t* rows = reinterpret_cast<uint16_t*>(ws);
      token_align_rows(x, ldx, n, d, rows, round8(d), s);
      a.x = rows;
      a.ldx = round8(d);
    }
    token_product(a, first, s);
    token_product(b, second, s);

    CombineArgs c{};
    c.part = part;
    c.ldp = dp;
    c.weights = weights;
    c.slots = slots;
    c.n = n;
    c.k = k;
    c.d = d;
    c.residual = residual;
    c.ldr = ldr;
    c.out = out;
    c.ldo = ldo;
    token_combine(c, s);
    return static_cast<int>(DYCL_OK);
  });
}

}  // extern "C"

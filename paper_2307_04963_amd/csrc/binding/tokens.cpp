// Python entry points of the token operators (include/dycl_tokens.h): checks of
// tensors, allocation of outputs and workspaces on the current stream, one call
// of the C interface.  In Python and ctypes that took 12 to 18 us, several times
// a small operator's own time; here it takes 4 to 6.
//
// Functions take their arguments in order; experts.py gives them names and
// defaults.  Wrong tensors raise ValueError, refusals of the C interface the
// package's DyclError.
#include "tensors.hpp"

namespace {

using namespace binding;

// x, y, post, post_weight, post_bias, gate, gate_act, row_gate, channel_scale, residual_scale, pre, pre_weight, pre_bias, eps,
// h, u, u_f32 -> (h or None where x stays, u or None)
PyObject* norm(PyObject*, PyObject* const* args, Py_ssize_t count) {
  return guarded([&] {
    Args a(args, count, 17);
    const at::Tensor& x = *a.tensor("x", false);
    const at::Tensor* y = a.tensor("y");
    const int post = a.small("post");
    const at::Tensor *post_w = a.tensor("post_weight"), *post_b = a.tensor("post_bias"), *gate = a.tensor("gate");
    const int gate_act = a.small("gate_act");
    const at::Tensor *row_gate = a.tensor("row_gate"), *channel = a.tensor("channel_scale");
    const float residual_scale = a.real();
    const int pre = a.small("pre");
    const at::Tensor *pre_w = a.tensor("pre_weight"), *pre_b = a.tensor("pre_bias");
    const float eps = a.real();
    const at::Tensor *h_in = a.tensor("h"), *u_in = a.tensor("u");
    const bool u_f32 = a.integer() != 0;

    input(x, "x");
    const int64_t n = x.size(0), d = x.size(1);
    const at::Device dev = x.device();
    const int64_t ldx = matrix(x, "x", n, d, dev);
    int64_t ldy = d, ldg = d;
    if (y) ldy = matrix(*y, "y", n, d, dev);
    if (gate) {
      if (!y) refuse("a gate needs y");
      ldg = matrix(*gate, "gate", n, d, dev);
      if (gate->scalar_type() != y->scalar_type()) refuse("gate must have y's type");
    }
    const float* rg = floats(row_gate, "row_gate", {n}, dev);
    const float* cs = floats(channel, "channel_scale", {d}, dev);
    const float *pw = floats(post_w, "post_weight", {d}, dev), *pb = floats(post_b, "post_bias", {d}, dev);
    const float *qw = floats(pre_w, "pre_weight", {d}, dev), *qb = floats(pre_b, "pre_bias", {d}, dev);
    if (u_in && pre == DYCL_NORM_NONE) refuse("u needs a pre norm");
    // (as the C interface, which a call that leaves x as it is does not come to)
    if (!y && (post != DYCL_NORM_NONE || rg || cs || pw || pb)) refuse("a post norm or a gate needs y");
    if (pre == DYCL_NORM_NONE && (qw || qb)) refuse("pre weights need a pre norm");
    if (d > INT32_MAX) refuse("d out of range");
    const c10::DeviceGuard on(dev);
    at::Tensor h, u;
    if (h_in) {
      h = *h_in;
    } else if (y || residual_scale != 1.0f) {
      h = make({n, d}, x.scalar_type(), dev);
    }
    if (u_in) {
      u = *u_in;
    } else if (pre != DYCL_NORM_NONE) {
      u = make({n, d}, u_f32 ? at::kFloat : at::kBFloat16, dev);
    }
    const int64_t ldh = h_in ? matrix(h, "h", n, d, dev) : d, ldu = u_in ? matrix(u, "u", n, d, dev) : d;
    if (h.defined() && h.scalar_type() != x.scalar_type()) refuse("h must have x's type");
    if (h.defined() || u.defined())
      check(dycl_op_norm(x.data_ptr(), type_of(x), ldx, pointer(y), y ? type_of(*y) : 0, ldy, pointer(gate), ldg, gate_act, rg, cs,
                         residual_scale, post, pw, pb, pre, qw, qb, eps, n, static_cast<int>(d), h.defined() ? h.data_ptr() : nullptr, ldh,
                         u.defined() ? u.data_ptr() : nullptr, u.defined() ? type_of(u) : 0, ldu, stream_of(dev)));
    return tuple({h, u});
  });
}

// logits, k, score, bias, groups, top_groups, mask, renormalise, scale, partition, workspace, automatic
// -> (ids, weights, offsets, order, slots)
PyObject* route(PyObject*, PyObject* const* args, Py_ssize_t count) {
  return guarded([&] {
    Args a(args, count, 12);
    const at::Tensor& logits = *a.tensor("logits", false);
    const int k = a.small("k"), score = a.small("score");
    const at::Tensor* bias = a.tensor("bias");
    const int groups = a.small("groups"), top_groups = a.small("top_groups");
    const at::Tensor* mask = a.tensor("mask");
    const bool renormalise = a.integer() != 0;
    const float scale = a.real();
    const bool partition = a.integer() != 0;
    const at::Tensor* given = a.tensor("workspace");
    const bool automatic = a.integer() != 0;

    input(logits, "logits");
    const int64_t n = logits.size(0), E = logits.size(1);
    const at::Device dev = logits.device();
    const int64_t ldl = matrix(logits, "logits", n, E, dev);
    if (E > INT32_MAX) refuse("experts out of range");
    if (k < 1 || k > E) refuse("k must be between 1 and the " + std::to_string(E) + " experts");
    const float* b = floats(bias, "bias", {E}, dev);
    const uint8_t* m = nullptr;
    if (mask && mask->scalar_type() == at::kBool)
      m = vector<uint8_t>(mask, "mask", {n}, at::kBool, dev);
    else
      m = vector<uint8_t>(mask, "mask", {n}, at::kByte, dev);
    const c10::DeviceGuard on(dev);
    at::Tensor ids = make({n, k}, at::kInt, dev), weights = make({n, k}, at::kFloat, dev), offsets, order, slots, own;
    if (partition) {
      offsets = make({E + 1}, at::kInt, dev);
      order = make({n * k}, at::kInt, dev);
      slots = make({n, k}, at::kInt, dev);
    }
    size_t have;
    void* ws = workspace_of(given, automatic, partition ? dycl_op_route_workspace(n, static_cast<int>(E), k) : 0, dev, own, have);
    auto list = [](const at::Tensor& t) { return t.defined() ? static_cast<int32_t*>(t.data_ptr()) : nullptr; };
    check(dycl_op_route(logits.data_ptr(), type_of(logits), ldl, b, m, n, static_cast<int>(E), groups, top_groups, k, score, renormalise,
                        scale, list(ids), static_cast<float*>(weights.data_ptr()), list(offsets), list(order), list(slots), ws, have,
                        stream_of(dev)));
    return tuple({ids, weights, offsets, order, slots});
  });
}

struct Layer {
  const at::Tensor* data;
  long experts, n, k;
  bool gated;
  explicit Layer(Args& a) : data(a.tensor("packed", false)), experts(a.integer()), n(a.integer()), k(a.integer()), gated(a.integer() != 0) {}
  const uint16_t* check(const char* what, const at::Device& dev) const {
    if (data->device() != dev) refuse(std::string(what) + " is on another device");
    if (!data->is_contiguous() || experts > INT32_MAX || n > INT32_MAX || k > INT32_MAX ||
        data->nbytes() < dycl_op_linear_packed_bytes(static_cast<int>(experts), static_cast<int>(n), static_cast<int>(k), gated))
      refuse(std::string(what) + " is not what pack() returned");
    return static_cast<const uint16_t*>(data->data_ptr());
  }
};

// w, gate -> packed data
PyObject* pack(PyObject*, PyObject* const* args, Py_ssize_t count) {
  return guarded([&] {
    Args a(args, count, 2);
    const at::Tensor& w = *a.tensor("w", false);
    const at::Tensor* gate = a.tensor("gate");
    if ((w.dim() != 2 && w.dim() != 3) || w.scalar_type() != at::kBFloat16 || !w.is_cuda())
      refuse("w must be a bfloat16 tensor [n, k] or [experts, n, k] on a GPU");
    if (gate && (gate->sizes() != w.sizes() || gate->scalar_type() != w.scalar_type() || gate->device() != w.device()))
      refuse("gate must be like w");
    const int64_t e = w.dim() == 3 ? w.size(0) : 1, n = w.size(-2), k = w.size(-1);
    if (e > INT32_MAX || n > INT32_MAX || k > INT32_MAX) refuse("w is too large");
    const c10::DeviceGuard on(w.device());
    const at::Tensor wc = w.contiguous(), gc = gate ? gate->contiguous() : at::Tensor();
    const size_t bytes = dycl_op_linear_packed_bytes(static_cast<int>(e), static_cast<int>(n), static_cast<int>(k), gate != nullptr);
    const at::Tensor data = make({static_cast<int64_t>(bytes / 2)}, at::kShort, w.device());
    check(dycl_op_linear_pack(bits(&wc), gate ? bits(&gc) : nullptr, static_cast<int>(e), static_cast<int>(n), static_cast<int>(k),
                              bits(&data), bytes, stream_of(w.device())));
    return wrap(data);
  });
}

// x, packed (data, experts, n, k, gated), bias, gate_bias, act, residual, out, out_f32, workspace, automatic -> y
PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t count) {
  return guarded([&] {
    Args a(args, count, 14);
    const at::Tensor& x = *a.tensor("x", false);
    const Layer layer(a);
    const at::Tensor *bias = a.tensor("bias"), *gate_bias = a.tensor("gate_bias");
    const int act = a.small("act");
    const at::Tensor *residual = a.tensor("residual"), *out = a.tensor("out");
    const bool out_f32 = a.integer() != 0;
    const at::Tensor* given = a.tensor("workspace");
    const bool automatic = a.integer() != 0;

    input(x, "x");
    const int64_t m = x.size(0), k = x.size(1), n = layer.n;
    const at::Device dev = x.device();
    if (layer.experts != 1 || layer.k != k) refuse("packed must be one layer on " + std::to_string(k) + " inputs");
    const uint16_t* w = layer.check("packed", dev);
    const int64_t ldx = bf16_matrix(x, "x", m, k, dev), ldr = residual ? bf16_matrix(*residual, "residual", m, n, dev) : n;
    const float *b = floats(bias, "bias", {n}, dev), *g = floats(gate_bias, "gate_bias", {n}, dev);
    const c10::DeviceGuard on(dev);
    const at::Tensor y = out ? *out : make({m, n}, out_f32 ? at::kFloat : at::kBFloat16, dev);
    const int64_t ldy = out ? matrix(y, "out", m, n, dev) : n;
    at::Tensor own;
    size_t have;
    const int ni = static_cast<int>(n), ki = static_cast<int>(k);
    void* ws = workspace_of(given, automatic, dycl_op_linear_workspace(bits(&x), ldx, m, ki, ni, layer.gated), dev, own, have);
    check(dycl_op_linear(bits(&x), ldx, m, ki, w, ni, layer.gated, b, g, act, bits(residual), ldr, y.data_ptr(), type_of(y), ldy, ws, have,
                         stream_of(dev)));
    return wrap(y);
  });
}

// x, weights, offsets, order, slots, packed (5), packed2 (5), act, bias, gate_bias, bias2, residual, out, workspace, automatic -> y
PyObject* experts(PyObject*, PyObject* const* args, Py_ssize_t count) {
  return guarded([&] {
    Args a(args, count, 23);
    const at::Tensor& x = *a.tensor("x", false);
    const at::Tensor& weights = *a.tensor("routing.weights", false);
    const at::Tensor *offsets = a.tensor("routing.offsets"), *order = a.tensor("routing.order"), *slots = a.tensor("routing.slots");
    const Layer one(a), two(a);
    const int act = a.small("act");
    const at::Tensor *bias = a.tensor("bias"), *gate_bias = a.tensor("gate_bias"), *bias2 = a.tensor("bias2");
    const at::Tensor *residual = a.tensor("residual"), *out = a.tensor("out"), *given = a.tensor("workspace");
    const bool automatic = a.integer() != 0;

    input(x, "x");
    const int64_t n = x.size(0), d = x.size(1), E = one.experts, f = one.n;
    const at::Device dev = x.device();
    if (one.k != d || two.experts != E || two.n != d || two.k != f || two.gated)
      refuse("packed must be layers of " + std::to_string(d) + " inputs, packed2 ungated layers back of as many experts");
    const uint16_t *w1 = one.check("packed", dev), *w2 = two.check("packed2", dev);
    if (!offsets || !order || !slots || weights.dim() != 2) refuse("routing must hold a partition");
    const int64_t k = weights.size(1);
    const float* w = floats(&weights, "routing.weights", {n, k}, dev);
    const int32_t* off = vector<int32_t>(offsets, "routing.offsets", {E + 1}, at::kInt, dev);
    const int32_t* ord = vector<int32_t>(order, "routing.order", {n * k}, at::kInt, dev);
    const int32_t* slot = vector<int32_t>(slots, "routing.slots", {n, k}, at::kInt, dev);
    const int64_t ldx = bf16_matrix(x, "x", n, d, dev), ldr = residual ? bf16_matrix(*residual, "residual", n, d, dev) : d;
    const float *b1 = floats(bias, "bias", {E, f}, dev), *g1 = floats(gate_bias, "gate_bias", {E, f}, dev),
                *b2 = floats(bias2, "bias2", {E, d}, dev);
    const c10::DeviceGuard on(dev);
    const at::Tensor y = out ? *out : make({n, d}, at::kBFloat16, dev);
    const int64_t ldo = out ? bf16_matrix(y, "out", n, d, dev) : d;
    at::Tensor own;
    size_t have;
    const int Ei = static_cast<int>(E), ki = static_cast<int>(k), di = static_cast<int>(d), fi = static_cast<int>(f);
    void* ws = workspace_of(given, automatic, dycl_op_experts_workspace(bits(&x), ldx, n, Ei, ki, di, fi), dev, own, have);
    check(dycl_op_experts(bits(&x), ldx, n, di, fi, Ei, ki, w1, one.gated, b1, g1, act, w2, b2, w, off, ord, slot, bits(residual), ldr,
                          bits(&y), ldo, ws, have, stream_of(dev)));
    return wrap(y);
  });
}

PyObject* set_error(PyObject*, PyObject* type) {
  Py_XSETREF(error_type(), Py_NewRef(type));
  Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {
    {"norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(norm)), METH_FASTCALL, nullptr},
    {"route", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(route)), METH_FASTCALL, nullptr},
    {"pack", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(pack)), METH_FASTCALL, nullptr},
    {"linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear)), METH_FASTCALL, nullptr},
    {"experts", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(experts)), METH_FASTCALL, nullptr},
    {"set_error", set_error, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_tokens", "the token and decoding operators on torch tensors", -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tokens() {
  PyObject* m = PyModule_Create(&kModule);
  if (m && PyModule_AddFunctions(m, decode_methods()) < 0) Py_CLEAR(m);
  return m;
}

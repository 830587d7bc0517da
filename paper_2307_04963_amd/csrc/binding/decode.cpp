// Python entry points of the decoding operators (include/dycl_decode.h); decoding.py
// gives their arguments names and defaults.
#include <algorithm>
#include <cmath>
#include <vector>

#include "tensors.hpp"

namespace {

using namespace binding;

const int32_t* ints(const at::Tensor* t, const char* what, at::IntArrayRef shape, const at::Device& dev) {
  return vector<int32_t>(t, what, shape, at::kInt, dev);
}

// one layer's cache, and the page tables that lead to it
struct Cache {
  const at::Tensor *keys, *values;
  explicit Cache(Args& a) : keys(a.tensor("cache.keys", false)), values(a.tensor("cache.values", false)) {}
  int64_t pages = 0;
  int heads = 0, page = 0, dim = 0;
  void check(const at::Device& dev) {
    if (keys->dim() != 4 || keys->scalar_type() != at::kBFloat16 || !keys->is_contiguous())
      refuse("cache.keys must be a contiguous bfloat16 tensor [pages, heads, page, dim]");
    if (values->sizes() != keys->sizes() || values->scalar_type() != keys->scalar_type() || !values->is_contiguous())
      refuse("cache.values must be like cache.keys");
    if (keys->device() != dev || values->device() != dev) refuse("the cache is on another device");
    for (int i = 1; i < 4; ++i)
      if (keys->size(i) > INT32_MAX) refuse("the cache is too large");
    pages = keys->size(0);
    heads = static_cast<int>(keys->size(1));
    page = static_cast<int>(keys->size(2));
    dim = static_cast<int>(keys->size(3));
    if (dim < 1) refuse("the cache's dim must not be 0");
  }
};

struct Tables {
  const int32_t* data;
  int64_t sequences, ld;
  int max_pages;
  Tables(const at::Tensor& t, const at::Device& dev) {
    if (t.dim() != 2 || t.scalar_type() != at::kInt || t.device() != dev || t.size(1) < 1 || t.size(1) > INT32_MAX ||
        (t.size(1) > 1 && t.stride(1) != 1) || (t.size(0) > 1 && t.stride(0) < t.size(1)))
      refuse("tables must be int32 [sequences, max_pages] on the cache's device, the last dimension contiguous");
    data = static_cast<const int32_t*>(t.data_ptr());
    sequences = t.size(0);
    max_pages = static_cast<int>(t.size(1));
    ld = sequences > 1 ? t.stride(0) : std::max<int64_t>(max_pages, t.stride(0));
  }
};

const double* frequencies_of(const at::Tensor* f, int& pairs, const at::Device& dev) {
  pairs = 0;
  if (!f) return nullptr;
  if (f->dim() != 1 || f->scalar_type() != at::kDouble || !f->is_contiguous() || f->device() != dev || f->size(0) > INT32_MAX)
    refuse("frequencies must be a contiguous float64 tensor [pairs] on the rows' device");
  pairs = static_cast<int>(f->size(0));
  return static_cast<const double*>(f->data_ptr());
}

// the number of heads of `dim` values in a row
int heads_of(const at::Tensor& t, const char* what, int64_t dim) {
  if (dim < 1 || t.size(1) % dim || t.size(1) / dim > INT32_MAX) refuse(std::string(what) + ": a row must be whole heads of dim values");
  return static_cast<int>(t.size(1) / dim);
}

// x, positions, frequencies, dim, layout, magnitude, adjoint, out -> y
PyObject* rotate(PyObject*, PyObject* const* args, Py_ssize_t count) {
  return guarded([&] {
    Args a(args, count, 8);
    const at::Tensor& x = *a.tensor("x", false);
    const at::Tensor *positions = a.tensor("positions", false), *frequencies = a.tensor("frequencies", false);
    const int dim = a.small("dim"), layout = a.small("layout");
    const float magnitude = a.real();
    const bool adjoint = a.integer() != 0;
    const at::Tensor* out = a.tensor("out");

    input(x, "x");
    const int64_t n = x.size(0), width = x.size(1);
    const at::Device dev = x.device();
    const int64_t ldx = matrix(x, "x", n, width, dev);
    const int heads = heads_of(x, "x", dim);
    const int32_t* at_ = ints(positions, "positions", {n}, dev);
    int pairs;
    const double* f = frequencies_of(frequencies, pairs, dev);
    const c10::DeviceGuard on(dev);
    const at::Tensor y = out ? *out : make({n, width}, x.scalar_type(), dev);
    const int64_t ldy = out ? matrix(y, "out", n, width, dev) : width;
    if (y.scalar_type() != x.scalar_type()) refuse("out must have x's type");
    check(dycl_op_rotate(x.data_ptr(), type_of(x), ldx, at_, f, pairs, layout, magnitude, adjoint, n, heads, dim, y.data_ptr(), ldy,
                         stream_of(dev)));
    return wrap(y);
  });
}

// keys, values, k, v, positions, tables, sequence, frequencies, layout, magnitude, q, q_out -> q_out or None
PyObject* append(PyObject*, PyObject* const* args, Py_ssize_t count) {
  return guarded([&] {
    Args a(args, count, 12);
    Cache cache(a);
    const at::Tensor &k = *a.tensor("k", false), &v = *a.tensor("v", false);
    const at::Tensor *positions = a.tensor("positions", false), *tables = a.tensor("tables", false), *sequence = a.tensor("sequence");
    const at::Tensor* frequencies = a.tensor("frequencies");
    const int layout = a.small("layout");
    const float magnitude = a.real();
    const at::Tensor *q = a.tensor("q"), *q_out = a.tensor("q_out");

    input(k, "k");
    const at::Device dev = k.device();
    cache.check(dev);
    const int64_t n = k.size(0), width = static_cast<int64_t>(cache.heads) * cache.dim;
    const int64_t ldk = matrix(k, "k", n, width, dev), ldv = matrix(v, "v", n, width, dev);
    if (v.scalar_type() != k.scalar_type()) refuse("v must have k's type");
    const int32_t* at_ = ints(positions, "positions", {n}, dev);
    const int32_t* seq = ints(sequence, "sequence", {n}, dev);
    const Tables table(*tables, dev);
    int pairs, q_heads = 0;
    const double* f = frequencies_of(frequencies, pairs, dev);
    const c10::DeviceGuard on(dev);
    int64_t ldq = 0, ldo = 0;
    at::Tensor turned;
    if (q) {
      input(*q, "q");
      q_heads = heads_of(*q, "q", cache.dim);
      ldq = matrix(*q, "q", n, q->size(1), dev);
      turned = q_out ? *q_out : make({n, q->size(1)}, q->scalar_type(), dev);
      ldo = matrix(turned, "q_out", n, q->size(1), dev);
      if (q->scalar_type() != k.scalar_type() || turned.scalar_type() != k.scalar_type()) refuse("q and q_out must have k's type");
    } else if (q_out) {
      refuse("q_out needs q");
    }
    // (an empty tensor's pointer is null)
    const bool turn = q && n > 0;
    check(dycl_op_append(k.data_ptr(), ldk, v.data_ptr(), ldv, turn ? q->data_ptr() : nullptr, ldq, turn ? turned.data_ptr() : nullptr, ldo,
                         type_of(k), at_, seq, f, pairs, layout, magnitude, n, q_heads, cache.heads, cache.dim, table.data, table.ld,
                         table.sequences, table.max_pages, bits(cache.keys), bits(cache.values), cache.pages, cache.page, stream_of(dev)));
    return wrap(turned);
  });
}

// q, keys, values, tables, lengths, sequence, scale (NaN: 1 / sqrt(dim)), window, mask, max_length (-1: the tables'), out, workspace,
// automatic -> out
PyObject* attend(PyObject*, PyObject* const* args, Py_ssize_t count) {
  return guarded([&] {
    Args a(args, count, 13);
    const at::Tensor& q = *a.tensor("q", false);
    Cache cache(a);
    const at::Tensor *tables = a.tensor("tables", false), *lengths = a.tensor("lengths", false), *sequence = a.tensor("sequence");
    PyObject* given_scale = a.next();
    float scale = 0.f;
    if (given_scale != Py_None) {
      const double v = PyFloat_AsDouble(given_scale);
      if (v == -1.0 && PyErr_Occurred()) throw Refused{};
      scale = static_cast<float>(v);
    }
    const long window = a.integer();
    const at::Tensor* mask = a.tensor("mask");
    long max_length = a.integer();
    const at::Tensor *out = a.tensor("out"), *given = a.tensor("workspace");
    const bool automatic = a.integer() != 0;

    input(q, "q");
    const at::Device dev = q.device();
    cache.check(dev);
    const int64_t n = q.size(0), width = q.size(1);
    const int64_t ldq = bf16_matrix(q, "q", n, width, dev);
    const int q_heads = heads_of(q, "q", cache.dim);
    if (given_scale == Py_None) scale = static_cast<float>(1.0 / std::sqrt(static_cast<double>(cache.dim)));
    const Tables table(*tables, dev);
    const int32_t* seen = ints(lengths, "lengths", {n}, dev);
    const int32_t* seq = ints(sequence, "sequence", {n}, dev);
    if (max_length < 0) max_length = static_cast<long>(table.max_pages) * cache.page;
    const uint8_t* m = nullptr;
    int64_t ldm = 0;
    if (mask) {
      if (mask->dim() != 2 || mask->size(0) != n || mask->size(1) < max_length || mask->device() != dev ||
          (mask->scalar_type() != at::kBool && mask->scalar_type() != at::kByte) || (mask->size(1) > 1 && mask->stride(1) != 1) ||
          (n > 1 && mask->stride(0) < mask->size(1)))
        refuse("mask must be bool or uint8 [" + std::to_string(n) + ", at least " + std::to_string(max_length) +
               "] on the rows' device, the last dimension contiguous");
      m = static_cast<const uint8_t*>(mask->data_ptr());
      ldm = n > 1 ? mask->stride(0) : std::max<int64_t>(mask->size(1), mask->stride(0));
    }
    const c10::DeviceGuard on(dev);
    const at::Tensor y = out ? *out : make({n, width}, at::kBFloat16, dev);
    const int64_t ldo = out ? bf16_matrix(y, "out", n, width, dev) : width;
    at::Tensor own;
    size_t have;
    void* ws = workspace_of(given, automatic, dycl_op_attend_workspace(n, q_heads, cache.heads, cache.dim, max_length, window), dev, own, have);
    check(dycl_op_attend(bits(&q), ldq, n, q_heads, cache.heads, cache.dim, scale, bits(cache.keys), bits(cache.values), cache.pages,
                         cache.page, table.data, table.ld, table.sequences, table.max_pages, seen, seq, max_length, window, m, ldm, bits(&y),
                         ldo, ws, have, stream_of(dev)));
    return wrap(y);
  });
}

// logits, scores, beams, k, ended, end, workspace, automatic -> (parents, tokens, scores, ended)
PyObject* beam(PyObject*, PyObject* const* args, Py_ssize_t count) {
  return guarded([&] {
    Args a(args, count, 8);
    const at::Tensor& logits = *a.tensor("logits", false);
    const at::Tensor* scores = a.tensor("scores", false);
    const int beams = a.small("beams"), k = a.small("k");
    const at::Tensor* ended = a.tensor("ended");
    const int end = a.small("end");
    const at::Tensor* given = a.tensor("workspace");
    const bool automatic = a.integer() != 0;

    input(logits, "logits");
    const int64_t rows = logits.size(0), words = logits.size(1);
    const at::Device dev = logits.device();
    const int64_t ldl = matrix(logits, "logits", rows, words, dev);
    if (words > INT32_MAX) refuse("words out of range");
    if (beams < 1 || rows % beams) refuse("logits must have whole sequences of " + std::to_string(beams) + " beams");
    if (k < 1) refuse("k must be at least 1");
    const float* s = floats(scores, "scores", {rows}, dev);
    const uint8_t* e = ended && ended->scalar_type() == at::kBool ? vector<uint8_t>(ended, "ended", {rows}, at::kBool, dev)
                                                                  : vector<uint8_t>(ended, "ended", {rows}, at::kByte, dev);
    const int64_t sequences = rows / beams;
    const c10::DeviceGuard on(dev);
    const int v = static_cast<int>(words);
    const size_t bytes = dycl_op_beam_workspace(sequences, beams, v, k);
    at::Tensor parents, tokens, next, over, own;
    if (bytes || !sequences) {           // (else the sizes are refused: nothing is allocated for them)
      parents = make({sequences, k}, at::kInt, dev), tokens = make({sequences, k}, at::kInt, dev);
      next = make({sequences, k}, at::kFloat, dev), over = make({sequences, k}, at::kByte, dev);
    }
    auto data = [](const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; };
    size_t have;
    void* ws = workspace_of(given, automatic, bytes, dev, own, have);
    check(dycl_op_beam(logits.data_ptr(), type_of(logits), ldl, s, e, end, sequences, beams, v, k, static_cast<int32_t*>(data(parents)),
                       static_cast<int32_t*>(data(tokens)), static_cast<float*>(data(next)), static_cast<uint8_t*>(data(over)), ws, have,
                       stream_of(dev)));
    return tuple({parents, tokens, next, over});
  });
}

// tables, lengths, parents, fresh, page or None, out_tables, out_lengths, then each layer's keys and values -> (tables, lengths).
// Everything about every layer is checked before the first layer's launch.
PyObject* fork(PyObject*, PyObject* const* args, Py_ssize_t count) {
  return guarded([&] {
    Args a(args, count, std::max<Py_ssize_t>(count, 7));
    const at::Tensor &tables = *a.tensor("tables", false), &lengths = *a.tensor("lengths", false);
    const at::Tensor &parents = *a.tensor("parents", false), &fresh = *a.tensor("fresh", false);
    const bool has_page = *a.a != Py_None;
    int page = has_page ? a.small("page") : (a.next(), 0);
    const at::Tensor *out_tables = a.tensor("out_tables"), *out_lengths = a.tensor("out_lengths");
    std::vector<Cache> layers;
    if (a.left % 2) refuse("a layer's cache must be its keys and values");
    while (a.left) layers.emplace_back(a);

    if (!tables.is_cuda()) refuse("tables must be on a GPU");
    const at::Device dev = tables.device();
    const Tables table(tables, dev);
    const int64_t n = parents.numel();
    if (parents.scalar_type() != at::kInt || !parents.is_contiguous() || parents.device() != dev)
      refuse("parents must be a contiguous int32 tensor on the tables' device");
    const int32_t* len = ints(&lengths, "lengths", {table.sequences}, dev);
    if (fresh.numel() != n || fresh.scalar_type() != at::kInt || !fresh.is_contiguous() || fresh.device() != dev)
      refuse("fresh must be a contiguous int32 tensor like parents");
    for (Cache& c : layers) {
      c.check(dev);
      // (its pointers would be null, which to the C interface is no cache)
      if (!c.keys->numel()) refuse("the cache is empty");
      if (has_page && c.page != page) refuse("page is not the cache's");
      if (c.page != layers[0].page) refuse("the layers' pages must hold the same number of tokens");
    }
    if (!layers.empty()) page = layers[0].page;
    const c10::DeviceGuard on(dev);
    at::Tensor t = out_tables ? *out_tables : make({n, table.max_pages}, at::kInt, dev);
    at::Tensor l = out_lengths ? *out_lengths : make({n}, at::kInt, dev);
    const Tables next(t, dev);
    if (t.size(0) != n || next.max_pages != table.max_pages) refuse("out_tables must be " + sizes(n, table.max_pages));
    ints(&l, "out_lengths", {n}, dev);
    auto call = [&](const Cache* c, int64_t rows, bool write) {
      check(dycl_op_fork(table.data, table.ld, len, table.sequences, table.max_pages, static_cast<const int32_t*>(parents.data_ptr()),
                         static_cast<const int32_t*>(fresh.data_ptr()), rows, write ? static_cast<int32_t*>(t.data_ptr()) : nullptr, next.ld,
                         write ? static_cast<int32_t*>(l.data_ptr()) : nullptr, c ? bits(c->keys) : nullptr, c ? bits(c->values) : nullptr,
                         c ? c->pages : 0, c ? c->heads : 0, page, c ? c->dim : 0, stream_of(dev)));
    };
    for (size_t i = 1; i < layers.size(); ++i) call(&layers[i], 0, false);     // (no rows: only its checks)
    call(layers.empty() ? nullptr : &layers[0], n, true);
    for (size_t i = 1; i < layers.size(); ++i) call(&layers[i], n, false);
    return tuple({t, l});
  });
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyCFunction fast() {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F));
}

}  // namespace

PyMethodDef* decode_methods() {
  static PyMethodDef methods[] = {{"rotate", fast<rotate>(), METH_FASTCALL, nullptr}, {"append", fast<append>(), METH_FASTCALL, nullptr},
                                  {"attend", fast<attend>(), METH_FASTCALL, nullptr}, {"beam", fast<beam>(), METH_FASTCALL, nullptr},
                                  {"fork", fast<fork>(), METH_FASTCALL, nullptr},     {nullptr, nullptr, 0, nullptr}};
  return methods;
}

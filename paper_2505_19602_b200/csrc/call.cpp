// The hot calls of the C ABI for Python callers: tensors are read through PyTorch's C++ interface and handed to the function
// whose address the binding passes, in one native call.  A step of a small map costs the host 5.9 us this way; with four ctypes
// structures built for every call (and the launches and events that a step made then) it was 14.5 us, twice what the GPU takes.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <exception>
#include <initializer_list>
#include <vector>

#include "../../include/scalekv.h"

namespace {

// A C++ exception (a sparse tensor has no strides, a wrapped one no memory) becomes the Python one that the tensor's own method
// raises: none may cross the interpreter's C frames.
template <typename F> bool guarded(F read) {
  try {
    return read();
  } catch (...) {
    torch::translate_exception_to_python(std::current_exception());
    return false;
  }
}

// obj.name() or, with an index, obj.name(index)
bool ask(PyObject *obj, const char *name, int index, long long *out) {
  PyObject *r = index < 0 ? PyObject_CallMethod(obj, name, nullptr) : PyObject_CallMethod(obj, name, "i", index);
  if (!r) return false;
  *out = (long long)(intptr_t)PyLong_AsVoidPtr(r);
  Py_DECREF(r);
  return !PyErr_Occurred();
}

bool bad_shape() {
  PyErr_SetString(PyExc_AssertionError, "expected [B, H, n, d] with contiguous head_dim");
  return false;
}

// [B, H, n, d] tensor -> view with element strides; the last axis must be contiguous.  Anything else that has a tensor's dim(),
// stride(i) and data_ptr() is asked for them (a subclass of Tensor may have its own).
bool view(PyObject *obj, scalekv_tensor *out) {
  if (!THPVariable_CheckExact(obj)) {
    long long dim, last, ptr, sb, sh, st;
    if (!ask(obj, "dim", -1, &dim)) return false;
    if (dim != 4) return bad_shape();
    if (!ask(obj, "stride", 3, &last)) return false;
    if (last != 1) return bad_shape();
    if (!ask(obj, "data_ptr", -1, &ptr) || !ask(obj, "stride", 0, &sb) || !ask(obj, "stride", 1, &sh) || !ask(obj, "stride", 2, &st)) return false;
    *out = {reinterpret_cast<const void *>((intptr_t)ptr), sb, sh, st};
    return true;
  }
  return guarded([&] {
    const at::Tensor &t = THPVariable_Unpack(obj);
    if (t.dim() != 4 || t.stride(3) != 1) return bad_shape();
    out->ptr = t.data_ptr();
    out->stride_b = t.stride(0);
    out->stride_h = t.stride(1);
    out->stride_t = t.stride(2);
    return true;
  });
}

// None or a tensor of floats
bool floats(PyObject *obj, float **out) {
  *out = nullptr;
  if (obj == Py_None) return true;
  if (!THPVariable_CheckExact(obj)) {
    long long ptr;
    if (!ask(obj, "data_ptr", -1, &ptr)) return false;
    *out = reinterpret_cast<float *>((intptr_t)ptr);
    return true;
  }
  return guarded([&] {
    *out = static_cast<float *>(THPVariable_Unpack(obj).data_ptr());
    return true;
  });
}

template <typename T> T address(PyObject *obj) { return reinterpret_cast<T>(PyLong_AsVoidPtr(obj)); }

bool arguments(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
  return false;
}

// A whole number.  One beyond 32 bits becomes the limit that it lies beyond, which no call takes for a layer or a scale; its low half might be one.
int number(PyObject *obj) { return (int)std::min<long>(std::max<long>(PyLong_AsLong(obj), INT32_MIN), INT32_MAX); }

// A factor of products, as 32 bits hold it.  0 stands for another, so what only becomes 0 there is refused.
float factor(PyObject *obj) {
  const double x = PyFloat_AsDouble(obj);
  if (x != 0. && (float)x == 0.f && !PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "softmax_scale is below what 32 bits hold");
  return (float)x;
}

#define CALL(expr)            \
  int st;                     \
  if (PyErr_Occurred()) return nullptr; \
  Py_BEGIN_ALLOW_THREADS      \
  st = (int)(expr);           \
  Py_END_ALLOW_THREADS        \
  return PyLong_FromLong(st)

// step(function, ctx, layer, scale, Q, K, V, O, lse, w, window address)
PyObject *step(PyObject *, PyObject *const *a, Py_ssize_t n) {
  scalekv_tensor q, k, v, o;
  float *lse;
  if (!arguments(n, 11) || !view(a[4], &q) || !view(a[5], &k) || !view(a[6], &v) || !view(a[7], &o) || !floats(a[8], &lse)) return nullptr;
  const auto fn = address<decltype(&scalekv_step)>(a[0]);
  const auto ctx = address<scalekv_ctx *>(a[1]);
  const int layer = number(a[2]), scale = number(a[3]), w = number(a[9]);
  const auto window = address<const int32_t *>(a[10]);
  CALL(fn(ctx, layer, scale, q, k, v, o, lse, w, window));
}

// step_ex(function, ctx, layer, scale, Q, K, V, O, lse, compress, w, window address, options address)
PyObject *step_ex(PyObject *, PyObject *const *a, Py_ssize_t n) {
  scalekv_tensor q, k, v, o;
  float *lse;
  if (!arguments(n, 13) || !view(a[4], &q) || !view(a[5], &k) || !view(a[6], &v) || !view(a[7], &o) || !floats(a[8], &lse)) return nullptr;
  const auto fn = address<decltype(&scalekv_step_ex)>(a[0]);
  const auto ctx = address<scalekv_ctx *>(a[1]);
  const int layer = number(a[2]), scale = number(a[3]), compress = number(a[9]), w = number(a[10]);
  const auto window = address<const int32_t *>(a[11]);
  const auto opts = address<const scalekv_select_opts *>(a[12]);
  CALL(fn(ctx, layer, scale, q, k, v, o, lse, compress, w, window, opts));
}

// append(function, ctx, layer, scale, K, V)
PyObject *append(PyObject *, PyObject *const *a, Py_ssize_t n) {
  scalekv_tensor k, v;
  if (!arguments(n, 6) || !view(a[4], &k) || !view(a[5], &v)) return nullptr;
  const auto fn = address<decltype(&scalekv_append)>(a[0]);
  const auto ctx = address<scalekv_ctx *>(a[1]);
  const int layer = number(a[2]), scale = number(a[3]);
  CALL(fn(ctx, layer, scale, k, v));
}

// attend(function, ctx, layer, Q, O, lse)
PyObject *attend(PyObject *, PyObject *const *a, Py_ssize_t n) {
  scalekv_tensor q, o;
  float *lse;
  if (!arguments(n, 6) || !view(a[3], &q) || !view(a[4], &o) || !floats(a[5], &lse)) return nullptr;
  const auto fn = address<decltype(&scalekv_attend)>(a[0]);
  const auto ctx = address<scalekv_ctx *>(a[1]);
  const int layer = number(a[2]);
  CALL(fn(ctx, layer, q, o, lse));
}

// compress_ex(function, ctx, layer, Qw or None, w, window address, full map, options address)
PyObject *compress_ex(PyObject *, PyObject *const *a, Py_ssize_t n) {
  scalekv_tensor q = {nullptr, 0, 0, 0};
  if (!arguments(n, 8) || (a[3] != Py_None && !view(a[3], &q))) return nullptr;
  const auto fn = address<decltype(&scalekv_compress_ex)>(a[0]);
  const auto ctx = address<scalekv_ctx *>(a[1]);
  const int layer = number(a[2]), w = number(a[4]), full = number(a[6]);
  const auto window = address<const int32_t *>(a[5]);
  const auto opts = address<const scalekv_select_opts *>(a[7]);
  CALL(fn(ctx, layer, q, w, window, full, opts));
}

// [batch][heads] of floats, as lists of lists
PyObject *lists(const std::vector<double> &x, Py_ssize_t batch, Py_ssize_t heads) {
  PyObject *out = PyList_New(batch);
  for (Py_ssize_t b = 0; out && b < batch; ++b) {
    PyObject *row = PyList_New(heads);
    for (Py_ssize_t h = 0; row && h < heads; ++h) {
      PyObject *v = PyFloat_FromDouble(x[(size_t)(b * heads + h)]);
      if (!v) Py_CLEAR(row);
      else PyList_SET_ITEM(row, h, v);
    }
    if (!row) Py_CLEAR(out);
    else PyList_SET_ITEM(out, b, row);
  }
  return out;
}

// layer_stats_ex(function, ctx, layer, Q, topk_prime, query_stride, batch, heads) -> (status, car, htk and the three per slice)
PyObject *layer_stats_ex(PyObject *, PyObject *const *a, Py_ssize_t n) {
  scalekv_tensor q;
  if (!arguments(n, 8) || !view(a[3], &q)) return nullptr;
  const auto fn = address<decltype(&scalekv_layer_stats_ex)>(a[0]);
  const auto ctx = address<scalekv_ctx *>(a[1]);
  const int layer = number(a[2]), topk = number(a[4]), stride = number(a[5]);
  const Py_ssize_t batch = PyLong_AsSsize_t(a[6]), heads = PyLong_AsSsize_t(a[7]);
  if (PyErr_Occurred()) return nullptr;
  double car = 0.0, htk = 0.0;
  int st = 0;
  std::vector<double> cs, ts, ns;
  if (!guarded([&] {
        cs.resize((size_t)(batch * heads)); ts.resize(cs.size()); ns.resize(cs.size());
        return true;
      })) return nullptr;
  Py_BEGIN_ALLOW_THREADS
  st = (int)fn(ctx, layer, q, topk, stride, &car, &htk, cs.data(), ts.data(), ns.data());
  Py_END_ALLOW_THREADS
  PyObject *c = lists(cs, batch, heads), *t = lists(ts, batch, heads), *m = lists(ns, batch, heads);
  if (c && t && m) return Py_BuildValue("(iddNNN)", st, car, htk, c, t, m);
  Py_XDECREF(c); Py_XDECREF(t); Py_XDECREF(m);
  return nullptr;
}

// ---- the paged token cache: [tokens][heads][head_dim] tensors, whose type, device and sizes are checked here, since the library sees addresses
// only.  What does not fit is a ValueError that names the argument.
bool rows(PyObject *obj, const char *name, long tokens, long heads, long dim, int device, scalekv_rows *out, at::ScalarType *type, long *got_heads) {
  if (!THPVariable_Check(obj)) {
    PyErr_Format(PyExc_TypeError, "%s: expected a tensor, got %s", name, Py_TYPE(obj)->tp_name);
    return false;
  }
  return guarded([&] {
    const at::Tensor &t = THPVariable_Unpack(obj);
    const char *wrong = nullptr;
    if (t.dim() != 3 || t.size(0) != tokens || (heads > 0 && t.size(1) != heads) || t.size(2) != dim) wrong = "has another shape than [tokens, heads, head_dim]";
    else if (!t.is_cuda() || t.get_device() != device) wrong = "is not on the cache's device";
    else if (t.scalar_type() != at::kBFloat16 && t.scalar_type() != at::kFloat) wrong = "is neither bfloat16 nor float32";
    else if (*type != at::ScalarType::Undefined && t.scalar_type() != *type) wrong = "has another type than it should";
    else if (t.numel() > 0 && t.stride(2) != 1) wrong = "must have contiguous head_dim";
    if (wrong) {
      PyErr_Format(PyExc_ValueError, "%s %s", name, wrong);
      return false;
    }
    *type = t.scalar_type();
    if (got_heads) *got_heads = t.size(1);
    *out = {t.data_ptr(), t.stride(0), t.stride(1)};
    // (the stride of an axis of one entry says nothing and need not keep rows on 16 bytes)
    if (t.size(0) <= 1) out->stride_t = 0;
    if (t.size(1) <= 1) out->stride_h = 0;
    return true;
  });
}

// move(function, handle, layer, batch address, tokens, kv heads, head_dim, device, K, V, stream): paged_write and paged_read
PyObject *paged_move(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arguments(n, 11)) return nullptr;
  const auto fn = address<decltype(&scalekv_paged_write)>(a[0]);
  const auto kv = address<scalekv_paged *>(a[1]);
  const int layer = number(a[2]);
  const auto batch = address<const scalekv_paged_batch *>(a[3]);
  const long tokens = PyLong_AsLong(a[4]), heads = PyLong_AsLong(a[5]), dim = PyLong_AsLong(a[6]), device = PyLong_AsLong(a[7]);
  const auto stream = address<void *>(a[10]);
  if (PyErr_Occurred()) return nullptr;
  scalekv_rows k, v;
  at::ScalarType type = at::ScalarType::Undefined;
  if (!rows(a[8], "K", tokens, heads, dim, (int)device, &k, &type, nullptr) || !rows(a[9], "V", tokens, heads, dim, (int)device, &v, &type, nullptr)) return nullptr;
  CALL(fn(kv, layer, batch, k, v, type == at::kFloat ? SCALEKV_F32 : SCALEKV_BF16, stream));
}

// paged_attend(function, handle, layer, batch address, tokens, head_dim, device, Q, O, lse or None, causal, window, sinks, scale, stream)
PyObject *paged_attend(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arguments(n, 15)) return nullptr;
  const auto fn = address<decltype(&scalekv_paged_attend)>(a[0]);
  const auto kv = address<scalekv_paged *>(a[1]);
  const int layer = number(a[2]);
  const auto batch = address<const scalekv_paged_batch *>(a[3]);
  const long tokens = PyLong_AsLong(a[4]), dim = PyLong_AsLong(a[5]), device = PyLong_AsLong(a[6]);
  const long window = PyLong_AsLong(a[11]), sinks = PyLong_AsLong(a[12]);
  const int causal = PyObject_IsTrue(a[10]);
  const float scale = factor(a[13]);
  const auto stream = address<void *>(a[14]);
  if (PyErr_Occurred()) return nullptr;
  if (window > 0x7fffffff || sinks > 0x7fffffff || window < 0 || sinks < 0) {
    PyErr_SetString(PyExc_ValueError, "window and n_sink must lie in [0, 2^31)");
    return nullptr;
  }
  const scalekv_paged_mask mask = {causal, (int32_t)window, (int32_t)sinks};
  scalekv_rows q, o;
  at::ScalarType type = at::kBFloat16;
  long heads = 0;
  float *lse = nullptr;
  if (!rows(a[7], "Q", tokens, 0, dim, (int)device, &q, &type, &heads) || !rows(a[8], "O", tokens, heads, dim, (int)device, &o, &type, nullptr)) return nullptr;
  if (a[9] != Py_None) {
    if (!THPVariable_Check(a[9])) {
      PyErr_SetString(PyExc_TypeError, "lse: expected a tensor");
      return nullptr;
    }
    if (!guarded([&] {
          const at::Tensor &t = THPVariable_Unpack(a[9]);
          if (t.dim() != 2 || t.size(0) != tokens || t.size(1) != heads || t.scalar_type() != at::kFloat || !t.is_contiguous() || !t.is_cuda() ||
              t.get_device() != device) {
            PyErr_SetString(PyExc_ValueError, "lse must be a contiguous float32 [tokens, heads] on the cache's device");
            return false;
          }
          lse = static_cast<float *>(t.data_ptr());
          return true;
        })) return nullptr;
  }
  CALL(fn(kv, layer, batch, (int32_t)std::min<long>(heads, INT32_MAX), q, o, lse, &mask, scale, stream));
}

// A dense tensor of one type whose sizes are known but for those that are given as -1; the last axis is contiguous, and the one before it too where `strided` is null, which
// otherwise receives its stride.
bool dense(PyObject *obj, const char *name, at::ScalarType type, std::initializer_list<long> sizes, int device, void **out, long long *strided = nullptr) {
  if (!THPVariable_Check(obj)) {
    PyErr_Format(PyExc_TypeError, "%s: expected a tensor, got %s", name, Py_TYPE(obj)->tp_name);
    return false;
  }
  return guarded([&] {
    const at::Tensor &t = THPVariable_Unpack(obj);
    const char *wrong = nullptr;
    if (t.dim() != (int64_t)sizes.size()) wrong = "has another number of axes than it should";
    for (size_t i = 0; !wrong && i < sizes.size(); ++i)
      if (sizes.begin()[i] >= 0 && t.size(i) != sizes.begin()[i]) wrong = "has another shape than it should";
    if (!wrong && (!t.is_cuda() || t.get_device() != device)) wrong = "is not on the cache's device";
    if (!wrong && t.scalar_type() != type) wrong = type == at::kInt ? "is not int32" : "is not float32";
    const int64_t n = t.dim();
    if (!wrong && t.numel() > 0) {
      if (!strided) {
        if (!t.is_contiguous()) wrong = "must be contiguous";
      } else {
        if (t.stride(n - 1) != 1 && t.size(n - 1) > 1) wrong = "must have a contiguous last axis";
        else if (t.size(n - 2) > 1 && (t.stride(n - 2) < 0 || t.stride(n - 2) > INT32_MAX)) wrong = "has a stride beyond 32 bits";
        else if (n == 3 && t.size(0) > 1 && t.stride(0) != t.size(1) * t.stride(1)) wrong = "must have contiguous leading axes";
      }
    }
    if (wrong) {
      PyErr_Format(PyExc_ValueError, "%s %s", name, wrong);
      return false;
    }
    *out = t.data_ptr();
    if (strided) *strided = t.size(n - 2) > 1 || (n == 3 && t.size(0) > 1) ? t.stride(n - 2) : t.size(n - 1);
    return true;
  });
}

// A size or a number of entries within 32 bits.
bool size(PyObject *obj, const char *name, int32_t *out) {
  const long x = PyLong_AsLong(obj);
  if (PyErr_Occurred()) return false;
  if (x < 0 || x > INT32_MAX) {
    PyErr_Format(PyExc_ValueError, "%s must lie in [0, 2^31)", name);
    return false;
  }
  *out = (int32_t)x;
  return true;
}

// paged_write_rotated(function, handle, layer, batch address, tokens, kv heads, head_dim, device, Q or None, Q_out or None, K, V, rotary address, axes, positions, stream)
PyObject *paged_write_rotated(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arguments(n, 16)) return nullptr;
  const auto fn = address<decltype(&scalekv_paged_write_rotated)>(a[0]);
  const auto kv = address<scalekv_paged *>(a[1]);
  const int layer = number(a[2]);
  const auto batch = address<const scalekv_paged_batch *>(a[3]);
  const long tokens = PyLong_AsLong(a[4]), kv_heads = PyLong_AsLong(a[5]), dim = PyLong_AsLong(a[6]), device = PyLong_AsLong(a[7]), axes = PyLong_AsLong(a[13]);
  const auto rotary = address<const scalekv_rotary *>(a[12]);
  const auto stream = address<void *>(a[15]);
  if (PyErr_Occurred()) return nullptr;
  scalekv_rows q = {}, q_out = {}, k, v;
  at::ScalarType type = at::ScalarType::Undefined, out_type = at::kBFloat16;
  long heads = 0;
  void *positions;
  long long axis_stride;
  if (!rows(a[10], "K", tokens, kv_heads, dim, (int)device, &k, &type, nullptr) || !rows(a[11], "V", tokens, kv_heads, dim, (int)device, &v, &type, nullptr)) return nullptr;
  if (a[8] != Py_None && (!rows(a[8], "Q", tokens, 0, dim, (int)device, &q, &type, &heads) || !rows(a[9], "Q_out", tokens, heads, dim, (int)device, &q_out, &out_type, nullptr))) return nullptr;
  if (!dense(a[14], "positions", at::kInt, {axes, tokens}, (int)device, &positions, &axis_stride)) return nullptr;
  CALL(fn(kv, layer, batch, (int32_t)std::min<long>(heads, INT32_MAX), q, q_out, k, v, type == at::kFloat ? SCALEKV_F32 : SCALEKV_BF16, rotary, static_cast<const int32_t *>(positions), axis_stride,
          stream));
}

// paged_attend_tree(function, handle, layer, batch address, tokens, head_dim, device, Q, O, lse or None, tree, scale, stream)
PyObject *paged_attend_tree(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arguments(n, 13)) return nullptr;
  const auto fn = address<decltype(&scalekv_paged_attend_tree)>(a[0]);
  const auto kv = address<scalekv_paged *>(a[1]);
  const int layer = number(a[2]);
  const auto batch = address<const scalekv_paged_batch *>(a[3]);
  const long tokens = PyLong_AsLong(a[4]), dim = PyLong_AsLong(a[5]), device = PyLong_AsLong(a[6]);
  const float scale = factor(a[11]);
  const auto stream = address<void *>(a[12]);
  if (PyErr_Occurred()) return nullptr;
  scalekv_rows q, o;
  at::ScalarType type = at::kBFloat16;
  long heads = 0;
  void *lse = nullptr, *tree;
  if (!rows(a[7], "Q", tokens, 0, dim, (int)device, &q, &type, &heads) || !rows(a[8], "O", tokens, heads, dim, (int)device, &o, &type, nullptr)) return nullptr;
  if (a[9] != Py_None && !dense(a[9], "lse", at::kFloat, {tokens, heads}, (int)device, &lse)) return nullptr;
  if (!dense(a[10], "tree", at::kInt, {tokens, -1}, (int)device, &tree)) return nullptr;
  const long words = THPVariable_Unpack(a[10]).size(1);
  CALL(fn(kv, layer, batch, (int32_t)std::min<long>(heads, INT32_MAX), q, o, static_cast<float *>(lse), static_cast<const int32_t *>(tree), (int32_t)std::min<long>(words, INT32_MAX), scale, stream));
}

// paged_accept(function, handle, layer, batch address, sequences, device, path, counts, stream)
PyObject *paged_accept(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arguments(n, 9)) return nullptr;
  const auto fn = address<decltype(&scalekv_paged_accept)>(a[0]);
  const auto kv = address<scalekv_paged *>(a[1]);
  const int layer = number(a[2]);
  const auto batch = address<const scalekv_paged_batch *>(a[3]);
  const long seqs = PyLong_AsLong(a[4]), device = PyLong_AsLong(a[5]);
  const auto stream = address<void *>(a[8]);
  if (PyErr_Occurred()) return nullptr;
  void *path, *counts;
  long long stride;
  if (!dense(a[6], "path", at::kInt, {seqs, -1}, (int)device, &path, &stride) || !dense(a[7], "counts", at::kInt, {seqs}, (int)device, &counts)) return nullptr;
  const long len = THPVariable_Unpack(a[6]).size(1);
  CALL(fn(kv, layer, batch, static_cast<const int32_t *>(path), (int32_t)stride, (int32_t)std::min<long>(len, INT32_MAX), static_cast<const int32_t *>(counts), stream));
}

// paged_weigh(function, handle, layer, batch address, tokens, head_dim, device, Q, lse, weights, pages, kv heads, page_tokens, causal, window, sinks, decay, scale, stream)
PyObject *paged_weigh(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arguments(n, 19)) return nullptr;
  const auto fn = address<decltype(&scalekv_paged_weigh)>(a[0]);
  const auto kv = address<scalekv_paged *>(a[1]);
  const int layer = number(a[2]);
  const auto batch = address<const scalekv_paged_batch *>(a[3]);
  const long tokens = PyLong_AsLong(a[4]), dim = PyLong_AsLong(a[5]), device = PyLong_AsLong(a[6]);
  const long pages = PyLong_AsLong(a[10]), kv_heads = PyLong_AsLong(a[11]), page_tokens = PyLong_AsLong(a[12]);
  const int causal = PyObject_IsTrue(a[13]);
  const double decay = PyFloat_AsDouble(a[16]);
  const float scale = factor(a[17]);
  const auto stream = address<void *>(a[18]);
  scalekv_paged_mask mask = {causal, 0, 0};
  if (PyErr_Occurred() || !size(a[14], "window", &mask.window) || !size(a[15], "n_sink", &mask.n_sink)) return nullptr;
  scalekv_rows q;
  at::ScalarType type = at::kBFloat16;
  long heads = 0;
  void *lse, *weights;
  if (!rows(a[7], "Q", tokens, 0, dim, (int)device, &q, &type, &heads) || !dense(a[8], "lse", at::kFloat, {tokens, heads}, (int)device, &lse) ||
      !dense(a[9], "weights", at::kFloat, {pages, kv_heads, page_tokens}, (int)device, &weights)) return nullptr;
  CALL(fn(kv, layer, batch, (int32_t)std::min<long>(heads, INT32_MAX), q, static_cast<const float *>(lse), &mask, scale, static_cast<float *>(weights), (float)decay, stream));
}

// paged_fade(function, handle, layer, batch address, device, weights, pages, kv heads, page_tokens, window, n_sink, decay, stream)
PyObject *paged_fade(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arguments(n, 13)) return nullptr;
  const auto fn = address<decltype(&scalekv_paged_fade)>(a[0]);
  const auto kv = address<scalekv_paged *>(a[1]);
  const int layer = number(a[2]);
  const auto batch = address<const scalekv_paged_batch *>(a[3]);
  const long device = PyLong_AsLong(a[4]), pages = PyLong_AsLong(a[6]), kv_heads = PyLong_AsLong(a[7]), page_tokens = PyLong_AsLong(a[8]);
  const double decay = PyFloat_AsDouble(a[11]);
  const auto stream = address<void *>(a[12]);
  scalekv_paged_mask mask = {1, 0, 0};
  if (PyErr_Occurred() || !size(a[9], "window", &mask.window) || !size(a[10], "n_sink", &mask.n_sink)) return nullptr;
  void *weights;
  if (!dense(a[5], "weights", at::kFloat, {pages, kv_heads, page_tokens}, (int)device, &weights)) return nullptr;
  CALL(fn(kv, layer, batch, &mask, static_cast<float *>(weights), (float)decay, stream));
}

// paged_evict(function, handle, layer, batch address, sequences, device, to_table, keep, weights, pages, kv heads, page_tokens, sinks, recent, kept, stream)
PyObject *paged_evict(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arguments(n, 16)) return nullptr;
  const auto fn = address<decltype(&scalekv_paged_evict)>(a[0]);
  const auto kv = address<scalekv_paged *>(a[1]);
  const int layer = number(a[2]);
  const auto batch = address<const scalekv_paged_batch *>(a[3]);
  const long seqs = PyLong_AsLong(a[4]), device = PyLong_AsLong(a[5]), pages = PyLong_AsLong(a[9]), kv_heads = PyLong_AsLong(a[10]), page_tokens = PyLong_AsLong(a[11]);
  const auto stream = address<void *>(a[15]);
  int32_t sinks, recent;
  if (PyErr_Occurred() || !size(a[12], "n_sink", &sinks) || !size(a[13], "n_recent", &recent)) return nullptr;
  void *to, *keep, *weights, *kept;
  long long to_stride, kept_stride;
  if (!dense(a[6], "to_table", at::kInt, {seqs, -1}, (int)device, &to, &to_stride) || !dense(a[7], "keep", at::kInt, {seqs}, (int)device, &keep) ||
      !dense(a[8], "weights", at::kFloat, {pages, kv_heads, page_tokens}, (int)device, &weights) ||
      !dense(a[14], "kept", at::kInt, {seqs, kv_heads, -1}, (int)device, &kept, &kept_stride)) return nullptr;
  const long to_pages = THPVariable_Unpack(a[6]).size(1), len = THPVariable_Unpack(a[14]).size(2);
  CALL(fn(kv, layer, batch, static_cast<const int32_t *>(to), (int32_t)to_stride, (int32_t)std::min<long>(to_pages, INT32_MAX), static_cast<const int32_t *>(keep), static_cast<float *>(weights),
          sinks, recent, static_cast<int32_t *>(kept), (int32_t)kept_stride, (int32_t)std::min<long>(len, INT32_MAX), stream));
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(step), METHOD(step_ex), METHOD(append), METHOD(attend), METHOD(compress_ex), METHOD(layer_stats_ex), METHOD(paged_move),
                         METHOD(paged_attend), METHOD(paged_write_rotated), METHOD(paged_attend_tree), METHOD(paged_accept), METHOD(paged_weigh), METHOD(paged_fade),
                         METHOD(paged_evict),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_scalekv_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__scalekv_call() { return PyModule_Create(&module); }

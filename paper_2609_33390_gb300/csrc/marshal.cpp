// Marshalling of the calls on caches in 4 bits in their usual form: results allocated here, the current stream.
//
// A call of one of them on a few rows takes the GPU 4 to 16 us, and took the interpreter, which looks at up to ten
// tensors' shapes, types, places and strides, 9 to 25 us a call. With the checks here a call takes the host 4 to
// 12 us, its launches among them (reading back 15.8 -> 6.5, attention 25 -> 12). What they do not pass, and results
// given or another stream, goes the interpreter's way, which has a word for each refusal.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/brisk.h"

namespace {

using Sizes = at::IntArrayRef;

// The arguments of one call, as far as they pass: tensors on the current device, as the workspace.
struct Checks {
  const brisk_cache_dims* d;
  void* ws = nullptr;
  int device = -1;
  bool ok = false;

  Checks(PyObject* dims, PyObject* workspace) : d(static_cast<const brisk_cache_dims*>(PyLong_AsVoidPtr(dims))) {
    if (!THPVariable_CheckExact(workspace)) return;
    const at::Tensor& t = THPVariable_Unpack(workspace);
    if (!t.is_cuda()) return;
    device = t.device().index();
    ok = device == c10::cuda::current_device();
    ws = t.mutable_data_ptr();
  }
  at::ScalarType dtype() const { return d->dtype == BRISK_DT_BF16 ? at::kBFloat16 : at::kFloat; }

  const at::Tensor* tensor(PyObject* o, at::ScalarType type, Sizes shape) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.is_cuda() && t.device().index() == device && t.scalar_type() == type && t.sizes() == shape ? &t : nullptr;
  }
  // A strided tensor, the last dimension contiguous; nothing where a size is zero.
  brisk_view view(PyObject* o, Sizes shape) {
    brisk_view v{};
    for (int64_t n : shape)
      if (n == 0 && o == Py_None) return v;
    const at::Tensor* t = tensor(o, dtype(), shape);
    if (!t || t->strides().back() != 1) {
      ok = false;
      return v;
    }
    const Sizes s = t->strides();
    const size_t i = shape.size() - 3;             // (of the prefix: no sequences)
    v.ptr = t->const_data_ptr();
    v.seq = i > 0 ? s[0] : 0;
    v.tok = s[i];
    v.head = s[i + 1];
    return v;
  }
  const void* plain(PyObject* o, at::ScalarType type, Sizes shape, bool may_miss = false) {
    if (may_miss && o == Py_None) return nullptr;
    const at::Tensor* t = tensor(o, type, shape);
    if (t && t->is_contiguous()) return t->const_data_ptr();
    ok = false;
    return nullptr;
  }
  // codes and scales under `name` and `scales`. `written`: asked for as memory to write, which a tensor that shares its
  // memory with the one it is a lazy clone of gets a copy for.
  brisk_packed packed(PyObject* cache, const char* name, const char* scales, bool written = false) {
    brisk_packed p{};
    if (d->S == 0) return p;
    const at::Tensor* t[2] = {};
    if (PyDict_CheckExact(cache)) {
      const char* names[2] = {name, scales};
      const int64_t last[2] = {d->D / 2, d->D <= 64 ? 4 : 8};
      for (int i = 0; i < 2; ++i) {
        PyObject* o = PyDict_GetItemString(cache, names[i]);   // (borrowed)
        if (o) t[i] = tensor(o, at::kByte, {d->B, d->S, d->Hkv, last[i]});
      }
    }
    if (!t[0] || !t[1] || t[0]->strides()[3] != 1 || t[1]->strides()[3] != 1) {
      ok = false;
      return p;
    }
    const Sizes c = t[0]->strides(), s = t[1]->strides();
    auto at = [&](const at::Tensor& x) { return written ? x.mutable_data_ptr() : const_cast<void*>(x.const_data_ptr()); };
    return brisk_packed{at(*t[0]), at(*t[1]), c[0], c[1], c[2], s[0], s[1], s[2]};
  }
  at::Tensor make(at::ScalarType type, Sizes shape) const {
    return at::empty(shape, at::TensorOptions().dtype(type).device(at::kCUDA, device));
  }
  void* stream() const { return c10::cuda::getCurrentCUDAStream(device).stream(); }
};

// The entry point of type F at `address`; other threads run meanwhile, as they do in any call of the library.
template <typename F, typename... A>
brisk_status call(PyObject* address, A... args) {
  const F f = reinterpret_cast<F>(PyLong_AsVoidPtr(address));
  brisk_status s;
  Py_BEGIN_ALLOW_THREADS
  s = f(args...);
  Py_END_ALLOW_THREADS
  return s;
}

// {a: x, b: y}, or the status where the call was refused.
PyObject* results(brisk_status s, const char* a, const at::Tensor& x, const char* b, const at::Tensor& y) {
  if (s != BRISK_OK) return PyLong_FromLong(s);
  PyObject *r = PyDict_New(), *px = THPVariable_Wrap(x), *py = THPVariable_Wrap(y);
  if (!r || !px || !py || PyDict_SetItemString(r, a, px) < 0 || PyDict_SetItemString(r, b, py) < 0) Py_CLEAR(r);
  Py_XDECREF(px);
  Py_XDECREF(py);
  return r;
}

// (function, dims, workspace, scale, q, k_prefix, v_prefix, cache, own_len, visible)
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 10) return PyErr_Format(PyExc_TypeError, "10 arguments, not %zd", n);
  Checks c(a[1], a[2]);
  if (!c.ok) Py_RETURN_NONE;
  const brisk_cache_dims* d = c.d;
  if (!PyFloat_CheckExact(a[3])) Py_RETURN_NONE;
  const float scale = (float)PyFloat_AsDouble(a[3]);
  const int64_t shape[4] = {d->B, d->L, d->Hq, d->D};
  const brisk_view q = c.view(a[4], shape), kp = c.view(a[5], {d->P, d->Hkv, d->D}), vp = c.view(a[6], {d->P, d->Hkv, d->D});
  const brisk_packed k = c.packed(a[7], "k", "k_scales"), v = c.packed(a[7], "v", "v_scales");
  const void* len = c.plain(a[8], at::kInt, {d->B});
  const void* visible = c.plain(a[9], at::kInt, {d->B, d->L}, true);
  if (!c.ok) Py_RETURN_NONE;
  const at::Tensor out = c.make(c.dtype(), shape), lse = c.make(at::kFloat, {d->B, d->L, d->Hq});
  const brisk_status s = call<decltype(&brisk_packed_attend)>(
      a[0], d, &q, &kp, &vp, &k, &v, static_cast<const int32_t*>(len), static_cast<const int32_t*>(visible), scale,
      out.mutable_data_ptr(), static_cast<float*>(lse.mutable_data_ptr()), c.ws, c.stream());
  return results(s, "out", out, "lse", lse);
  END_HANDLE_TH_ERRORS
}

// (function, dims, workspace, cache, k, v, start, count)
PyObject* store(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 8) return PyErr_Format(PyExc_TypeError, "8 arguments, not %zd", n);
  Checks c(a[1], a[2]);
  if (!c.ok) Py_RETURN_NONE;
  const brisk_cache_dims* d = c.d;
  if (!THPVariable_CheckExact(a[4]) || THPVariable_Unpack(a[4]).dim() != 4) Py_RETURN_NONE;
  const int64_t T = THPVariable_Unpack(a[4]).size(1);
  if (T < 1 || T > 1 << 30) Py_RETURN_NONE;
  const int64_t shape[4] = {d->B, T, d->Hkv, d->D};
  const brisk_view k = c.view(a[4], shape), v = c.view(a[5], shape);
  const brisk_packed kp = c.packed(a[3], "k", "k_scales", true), vp = c.packed(a[3], "v", "v_scales", true);
  const void* start = c.plain(a[6], at::kInt, {d->B});
  const void* count = c.plain(a[7], at::kInt, {d->B}, true);
  if (!c.ok) Py_RETURN_NONE;
  return PyLong_FromLong(call<decltype(&brisk_packed_store)>(
      a[0], d, (int32_t)T, &k, &v, static_cast<const int32_t*>(start), static_cast<const int32_t*>(count), &kp, &vp,
      c.ws, c.stream()));
  END_HANDLE_TH_ERRORS
}

// (function, dims, workspace, cache, T, start, count)
PyObject* load(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 7) return PyErr_Format(PyExc_TypeError, "7 arguments, not %zd", n);
  Checks c(a[1], a[2]);
  if (!c.ok) Py_RETURN_NONE;
  const brisk_cache_dims* d = c.d;
  if (!PyLong_CheckExact(a[4])) Py_RETURN_NONE;
  const long long T = PyLong_AsLongLong(a[4]);
  if (PyErr_Occurred()) return nullptr;
  if (T < 1 || T > 1 << 30) Py_RETURN_NONE;
  const brisk_packed kp = c.packed(a[3], "k", "k_scales"), vp = c.packed(a[3], "v", "v_scales");
  const void* start = c.plain(a[5], at::kInt, {d->B});
  const void* count = c.plain(a[6], at::kInt, {d->B}, true);
  if (!c.ok) Py_RETURN_NONE;
  const int64_t shape[4] = {d->B, T, d->Hkv, d->D};
  const at::Tensor k = c.make(c.dtype(), shape), v = c.make(c.dtype(), shape);
  const brisk_view kv{k.mutable_data_ptr(), T * d->Hkv * d->D, (int64_t)d->Hkv * d->D, d->D};
  brisk_view vv = kv;
  vv.ptr = v.mutable_data_ptr();
  const brisk_status s = call<decltype(&brisk_packed_load)>(
      a[0], d, (int32_t)T, &kp, &vp, static_cast<const int32_t*>(start), static_cast<const int32_t*>(count), &kv, &vv,
      c.ws, c.stream());
  return results(s, "k", k, "v", v);
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"attend", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(attend)), METH_FASTCALL, nullptr},
    {"store", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(store)), METH_FASTCALL, nullptr},
    {"load", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(load)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }

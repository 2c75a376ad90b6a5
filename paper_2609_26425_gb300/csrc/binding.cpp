// binding.cpp -- Python calls of the rotary and paged entry points.
//
// Only marshalling, like the ctypes binding of the other entry points: dtypes,
// shapes, strides and devices are checked, outputs that the caller does not
// give are allocated by PyTorch, and raw pointers and the current stream go to
// the C ABI of include/qwm.h.  A rotation that autograd has to record is left to
// paged.py.  It is compiled because a single token's call is
// as long as its binding: through ctypes 12 to 17 us a call, of which the launch
// is 3.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <utility>

#include "../../include/qwm.h"

namespace {

PyObject* g_error = nullptr;  // QwmError(function, status)

PyObject* fail(const char* fn, qwm_status st) {
  PyObject* e = g_error ? PyObject_CallFunction(g_error, "si", fn, (int)st) : nullptr;
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  } else if (!PyErr_Occurred()) {
    PyErr_Format(PyExc_RuntimeError, "%s failed: %d", fn, (int)st);
  }
  return nullptr;
}

// The functions below return null or false with a Python error set.
const at::Tensor* tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_ValueError, "%s must be a CUDA tensor", name);
    return nullptr;
  }
  return &THPVariable_Unpack(o);
}

// A reference that is given back on every way out, an exception's too.
struct Ref {
  PyObject* p = nullptr;
  ~Ref() { Py_XDECREF(p); }
  PyObject* release() { return std::exchange(p, nullptr); }
};

// The result of one output or of two.
PyObject* result(Ref& a, Ref& b) {
  if (!b.p) return a.release();
  PyObject* both = PyTuple_New(2);
  if (!both) return nullptr;
  PyTuple_SET_ITEM(both, 0, a.release());
  PyTuple_SET_ITEM(both, 1, b.release());
  return both;
}

const char* type_name(at::ScalarType t) { return t == at::kHalf ? "torch.float16" : "torch.bfloat16"; }

// A [tokens][heads][head_dim] tensor (any strides of tokens and heads); n, d < 0:
// any.
bool rows(const at::Tensor& t, at::ScalarType type, int device, const char* name, int64_t n, int64_t d, qwm_rows* r) {
  if (!t.is_cuda() || t.scalar_type() != type || (device >= 0 && t.get_device() != device)) {
    PyErr_Format(PyExc_ValueError, "%s must be a %s CUDA tensor of one device with the others", name, type_name(type));
    return false;
  }
  if (t.dim() != 3 || (n >= 0 && t.size(0) != n) || (d >= 0 && t.size(2) != d)) {
    PyErr_Format(PyExc_ValueError, "%s must be [tokens][heads][head_dim] with %lld tokens of %lld channels (-1: any)", name,
                 (long long)n, (long long)d);
    return false;
  }
  if (t.size(2) > 1 && t.stride(2) != 1) {
    PyErr_Format(PyExc_ValueError, "%s must have contiguous channels", name);
    return false;
  }
  r->data = t.data_ptr();
  r->token_stride = t.size(0) > 1 ? t.stride(0) : 0;  // the stride of a dimension of one is never used
  r->head_stride = t.size(1) > 1 ? t.stride(1) : 0;
  r->heads = (int32_t)t.size(1);
  return true;
}

// A caller's tensor that the call writes: autograd notices where it was saved.
void written(const at::Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// The output for `like`: the caller's tensor `o`, or a new contiguous one.
bool output(PyObject* o, const at::Tensor& like, int device, const char* name, qwm_rows* r, Ref* ret) {
  if (o != Py_None) {
    const at::Tensor* t = tensor(o, name);
    if (!t) return false;
    if (t->sizes() != like.sizes()) {
      PyErr_Format(PyExc_ValueError, "%s must have the shape of its input", name);
      return false;
    }
    if (!rows(*t, like.scalar_type(), device, name, -1, -1, r)) return false;
    written(*t);
    ret->p = Py_NewRef(o);
    return true;
  }
  const at::Tensor t = at::empty(like.sizes(), like.options().memory_format(at::MemoryFormat::Contiguous));
  r->data = t.data_ptr();
  r->head_stride = t.size(2);
  r->token_stride = t.size(1) * t.size(2);
  r->heads = (int32_t)t.size(1);
  ret->p = THPVariable_Wrap(t);
  return ret->p != nullptr;
}

bool positions(PyObject* o, int64_t n, int device, const int32_t** p) {
  const at::Tensor* t = tensor(o, "pos");
  if (!t) return false;
  if (!t->is_cuda() || t->scalar_type() != at::kInt || !t->is_contiguous() || t->dim() != 2 || t->size(0) != n ||
      t->size(1) != 3 || t->get_device() != device) {
    PyErr_Format(PyExc_ValueError, "pos must be a contiguous int32 CUDA tensor [%lld][3]", (long long)n);
    return false;
  }
  *p = static_cast<const int32_t*>(t->data_ptr());
  return true;
}

bool integer(PyObject* o, const char* name, int64_t lo, int64_t hi, int64_t* v) {
  *v = PyLong_AsLongLong(o);
  if (*v == -1 && PyErr_Occurred()) return false;
  if (*v < lo || *v > hi) {
    PyErr_Format(PyExc_ValueError, "%s is out of range", name);
    return false;
  }
  return true;
}

// What a rotation, a cache or a batch keeps for its calls: integers, the last of them
// the device of what they stand for, which has to be the tensors' (kAnyDevice: it tells
// the device).
constexpr int kAnyDevice = -2;
template <int N>
bool key(PyObject* o, const char* name, int device, int64_t (&v)[N]) {
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != N) {
    PyErr_Format(PyExc_ValueError, "not a %s", name);
    return false;
  }
  for (int i = 0; i < N; ++i)
    if (!integer(PyTuple_GET_ITEM(o, i), name, INT64_MIN, INT64_MAX, &v[i])) return false;
  if (device != kAnyDevice && v[N - 1] != device) {
    PyErr_Format(PyExc_ValueError, "the %s is on another device (%lld) than the tensors (%d)", name, (long long)v[N - 1], device);
    return false;
  }
  return true;
}

// (frequencies' address, time, height, width pairs, interleaved, device) of a rotation
bool rotation(PyObject* o, int64_t d, at::ScalarType type, int device, qwm_rope_config* c, const float** freq) {
  int64_t v[6];
  if (!key(o, "rotation", device, v)) return false;
  c->head_dim = (int32_t)d;
  c->dtype = type == at::kHalf ? QWM_F16 : QWM_BF16;
  for (int i = 0; i < 3; ++i) c->pairs[i] = (int32_t)v[1 + i];
  c->interleaved = (int32_t)v[4];
  *freq = reinterpret_cast<const float*>(v[0]);
  return true;
}

bool count(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) PyErr_Format(PyExc_TypeError, "%zd arguments, %zd wanted", n, want);
  return n == want;
}

bool tracked(PyObject* o) { return THPVariable_Check(o) && THPVariable_Unpack(o).requires_grad(); }

// turn(backward, rotation, q, pos, k or None, q_out or None, k_out or None); None, with
// nothing done, if autograd has to record the call
PyObject* turn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 7)) return nullptr;
  if (c10::GradMode::is_enabled() && (tracked(a[2]) || tracked(a[4]) || tracked(a[5]) || tracked(a[6]))) Py_RETURN_NONE;
  const bool backward = a[0] == Py_True;
  const at::Tensor* q = tensor(a[2], "q");
  if (!q) return nullptr;
  if (q->scalar_type() != at::kBFloat16 && q->scalar_type() != at::kHalf) {
    PyErr_SetString(PyExc_ValueError, "the rotation takes bf16 or fp16 CUDA tensors");
    return nullptr;
  }
  qwm_rope_config cfg;
  const float* freq;
  const int32_t* pos;
  qwm_rows qr, qo, kr, ko;
  if (!rows(*q, q->scalar_type(), -1, "q", -1, -1, &qr)) return nullptr;
  const int dev = q->get_device();
  const int64_t N = q->size(0), d = q->size(2);
  if (!rotation(a[1], d, q->scalar_type(), dev, &cfg, &freq) || !positions(a[3], N, dev, &pos)) return nullptr;
  const bool has_k = a[4] != Py_None;
  const at::Tensor* k = has_k ? tensor(a[4], "k") : nullptr;
  if (has_k && (!k || !rows(*k, q->scalar_type(), dev, "k", N, d, &kr))) return nullptr;
  Ref q_out, k_out;
  if (!output(a[5], *q, dev, "q_out", &qo, &q_out) || (has_k && !output(a[6], *k, dev, "k_out", &ko, &k_out))) return nullptr;
  qwm_status st;
  {
    const c10::cuda::CUDAGuard guard(dev);
    void* s = c10::cuda::getCurrentCUDAStream(dev).stream();
    Py_BEGIN_ALLOW_THREADS
    st = (backward ? qwm_rope_backward : qwm_rope)(&cfg, freq, pos, N, &qr, &qo, has_k ? &kr : nullptr, has_k ? &ko : nullptr, s);
    Py_END_ALLOW_THREADS
  }
  if (st != QWM_OK) return fail(backward ? "qwm_rope_backward" : "qwm_rope", st);
  return result(q_out, k_out);
}

// A cache is (descriptor's address, head_dim, qwm_dtype, device), a batch
// (qwm_paged_batch's address, rows or -1 for any, device).
struct Cache {
  qwm_paged* handle;
  int64_t d;
  at::ScalarType type;
};
// The cache, for tensors of `device`; kAnyDevice, and `own` tells the cache's.
bool cache_on(PyObject* o, int device, Cache* c, int* own = nullptr) {
  int64_t v[4];
  if (!key(o, "paged cache", device, v)) return false;
  c->handle = reinterpret_cast<qwm_paged*>(v[0]);
  c->d = v[1];
  c->type = v[2] == QWM_F16 ? at::kHalf : at::kBFloat16;
  if (own) *own = (int)v[3];
  return true;
}
// The cache for tensors of `like`'s device.
bool cache_of(PyObject* o, const at::Tensor& like, Cache* c) { return cache_on(o, like.is_cuda() ? like.get_device() : -1, c); }
bool batch_of(PyObject* o, int64_t n, int device, qwm_paged_batch* b) {
  int64_t v[3];
  if (!key(o, "paged batch", device, v)) return false;
  if (v[1] >= 0 && v[1] != n) {
    PyErr_Format(PyExc_ValueError, "the batch has %lld rows, the tensor %lld", (long long)v[1], (long long)n);
    return false;
  }
  *b = *reinterpret_cast<const qwm_paged_batch*>(v[0]);
  b->tokens = n;
  return true;
}

// append(cache, batch, k, v, rotation or None, pos or None, q or None, q_out or None)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Cache c;
  if (!count(n, 8)) return nullptr;
  const at::Tensor *k = tensor(a[2], "k"), *v = k ? tensor(a[3], "v") : nullptr;
  qwm_rows kr, vr, qr, qo;
  if (!v || !cache_of(a[0], *k, &c) || !rows(*k, c.type, -1, "k", -1, c.d, &kr)) return nullptr;
  const int64_t N = k->size(0);
  const int dev = k->get_device();
  qwm_paged_batch b;
  if (!rows(*v, c.type, dev, "v", N, c.d, &vr) || !batch_of(a[1], N, dev, &b)) return nullptr;
  qwm_rope_config cfg;
  const float* freq = nullptr;
  const int32_t* pos = nullptr;
  const bool turned = a[4] != Py_None, has_q = a[6] != Py_None;
  if (turned && (!rotation(a[4], c.d, c.type, dev, &cfg, &freq) || !positions(a[5], N, dev, &pos))) return nullptr;
  Ref q_out;
  if (has_q) {
    const at::Tensor* q = tensor(a[6], "q");
    if (!q || !rows(*q, c.type, dev, "q", N, c.d, &qr) || !output(a[7], *q, dev, "q_out", &qo, &q_out)) return nullptr;
  }
  qwm_status st;
  {
    const c10::cuda::CUDAGuard guard(dev);
    void* s = c10::cuda::getCurrentCUDAStream(dev).stream();
    Py_BEGIN_ALLOW_THREADS
    st = qwm_paged_append(c.handle, &b, &kr, &vr, turned ? &cfg : nullptr, freq, pos, has_q ? &qr : nullptr,
                          has_q ? &qo : nullptr, s);
    Py_END_ALLOW_THREADS
  }
  if (st != QWM_OK) return fail("qwm_paged_append", st);
  return has_q ? q_out.release() : Py_NewRef(Py_None);
}

// read(cache, batch, kv_heads, rows or -1, k_out or None or False, v_out or None or False);
// None: a new tensor, False: not wanted (None in its place)
PyObject* read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Cache c;
  int dev;
  int64_t H, N, v[3];
  if (!count(n, 6) || !cache_on(a[0], kAnyDevice, &c, &dev) || !integer(a[2], "kv_heads", 1, 4096, &H) ||
      !integer(a[3], "tokens", -1, INT32_MAX, &N))
    return nullptr;
  const at::Tensor* given[2] = {nullptr, nullptr};
  for (int i = 0; i < 2; ++i) {
    PyObject* o = a[4 + i];
    if (o == Py_None || o == Py_False) continue;
    if (!(given[i] = tensor(o, i ? "v_out" : "k_out"))) return nullptr;
    if (N < 0 && given[i]->dim() == 3) N = given[i]->size(0);
  }
  if (!key(a[1], "paged batch", dev, v)) return nullptr;
  if (N < 0) N = v[1];
  if (N < 0) {
    PyErr_SetString(PyExc_ValueError, "the number of tokens to read is not known: give it, an output, or a batch made with it");
    return nullptr;
  }
  qwm_paged_batch b;
  if (!batch_of(a[1], N, dev, &b)) return nullptr;
  qwm_rows r[2];
  Ref ret[2];
  for (int i = 0; i < 2; ++i) {
    if (a[4 + i] == Py_False) {
      ret[i].p = Py_NewRef(Py_None);
    } else if (given[i]) {
      if (!rows(*given[i], c.type, dev, i ? "v_out" : "k_out", N, c.d, &r[i])) return nullptr;
      ret[i].p = Py_NewRef(a[4 + i]);
    } else {
      const at::Tensor t = at::empty({N, H, c.d}, at::TensorOptions().dtype(c.type).device(at::kCUDA, (c10::DeviceIndex)dev));
      r[i] = qwm_rows{t.data_ptr(), H * c.d, c.d, (int32_t)H};
      ret[i].p = THPVariable_Wrap(t);
      if (!ret[i].p) return nullptr;
    }
  }
  for (const at::Tensor* t : given)
    if (t) written(*t);
  qwm_status st;
  {
    const c10::cuda::CUDAGuard guard(dev);
    void* s = c10::cuda::getCurrentCUDAStream(dev).stream();
    Py_BEGIN_ALLOW_THREADS
    st = qwm_paged_read(c.handle, &b, a[4] == Py_False ? nullptr : &r[0], a[5] == Py_False ? nullptr : &r[1], s);
    Py_END_ALLOW_THREADS
  }
  if (st != QWM_OK) return fail("qwm_paged_read", st);
  return result(ret[0], ret[1]);
}

// attend(cache, batch, q, block, window, sinks, sm_scale, out or None, lse or None, want_lse, workspace or None)
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Cache c;
  if (!count(n, 11)) return nullptr;
  const at::Tensor* q = tensor(a[2], "q");
  qwm_rows qr, orows;
  if (!q || !cache_of(a[0], *q, &c) || !rows(*q, c.type, -1, "q", -1, c.d, &qr)) return nullptr;
  const int64_t N = q->size(0), H = q->size(1);
  const int dev = q->get_device();
  qwm_paged_batch b;
  int64_t block, window, sinks;
  if (!batch_of(a[1], N, dev, &b) || !integer(a[3], "block", INT32_MIN, INT32_MAX, &block) ||
      !integer(a[4], "window", INT32_MIN, INT32_MAX, &window) || !integer(a[5], "sinks", INT32_MIN, INT32_MAX, &sinks))
    return nullptr;
  const qwm_mask mask{(int32_t)block, (int32_t)window, (int32_t)sinks};
  const double scale = PyFloat_AsDouble(a[6]);
  if (scale == -1.0 && PyErr_Occurred()) return nullptr;
  void* ws = nullptr;
  size_t ws_bytes = 0;
  if (a[10] != Py_None) {
    const at::Tensor* t = tensor(a[10], "workspace");
    if (!t) return nullptr;
    if (!t->is_cuda() || t->get_device() != dev || !t->is_contiguous()) {
      PyErr_SetString(PyExc_ValueError, "workspace must be a contiguous CUDA tensor of q's device");
      return nullptr;
    }
    ws = t->data_ptr();
    ws_bytes = t->nbytes();
  }
  Ref out, lse;
  float* lse_data = nullptr;
  if (a[8] != Py_None) {
    const at::Tensor* t = tensor(a[8], "lse");
    if (!t) return nullptr;
    if (!t->is_cuda() || t->get_device() != dev || t->scalar_type() != at::kFloat || !t->is_contiguous() || t->dim() != 2 ||
        t->size(0) != H || t->size(1) != N) {
      PyErr_SetString(PyExc_ValueError, "lse must be a contiguous fp32 CUDA tensor [heads][tokens]");
      return nullptr;
    }
    lse_data = static_cast<float*>(t->data_ptr());
    written(*t);
    lse.p = Py_NewRef(a[8]);
  } else if (PyObject_IsTrue(a[9]) == 1) {
    const at::Tensor t = at::empty({H, N}, q->options().dtype(at::kFloat).memory_format(at::MemoryFormat::Contiguous));
    lse_data = static_cast<float*>(t.data_ptr());
    lse.p = THPVariable_Wrap(t);
    if (!lse.p) return nullptr;
  }
  if (!output(a[7], *q, dev, "out", &orows, &out)) return nullptr;
  qwm_status st;
  {
    const c10::cuda::CUDAGuard guard(dev);
    void* s = c10::cuda::getCurrentCUDAStream(dev).stream();
    Py_BEGIN_ALLOW_THREADS
    st = qwm_paged_attend(c.handle, &b, &qr, &mask, (float)scale, &orows, lse_data, ws, ws_bytes, s);
    Py_END_ALLOW_THREADS
  }
  if (st != QWM_OK) return fail("qwm_paged_attend", st);
  return result(out, lse);
}

// set_error(class): what a status other than QWM_OK raises
PyObject* set_error(PyObject*, PyObject* cls) {
  Py_XDECREF(g_error);
  g_error = Py_NewRef(cls);
  Py_RETURN_NONE;
}

// A C++ exception (out of memory, say) becomes a Python one.
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  try {
    return F(self, a, n);
  } catch (const c10::OutOfMemoryError& e) {
    PyErr_SetString(PyExc_MemoryError, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyCFunction fast() {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<F>));
}

PyMethodDef methods[] = {
    {"turn", fast<turn>(), METH_FASTCALL, nullptr},
    {"append", fast<append>(), METH_FASTCALL, nullptr},
    {"read", fast<read>(), METH_FASTCALL, nullptr},
    {"attend", fast<attend>(), METH_FASTCALL, nullptr},
    {"set_error", set_error, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "qwm_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit_qwm_binding() { return PyModule_Create(&module); }

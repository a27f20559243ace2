// The common path of the Python binding of the training operators, natively:
// tensors are looked at, outputs allocated and the C entry point called
// without a Python object per check.  A call on a handful of tensors takes 6
// us of host time instead of 16; a step of 300 tensors, six of them checked
// each, 42 us instead of 960 (14 of them behind its launches), where its kernels
// take 70.
//
// Every function returns None where an argument is not plainly what it takes:
// the caller's Python code then says what is wrong with it (or handles it).
// An int is the status of the C call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/EmptyTensor.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/autograd/variable.h>

#include <vector>

#include "acdc_train.h"
#include "acdc_train_lm.h"

namespace {

using at::Tensor;

// The tensor behind a Python object; null for None; `bad` for anything else.
struct Args {
  PyObject* const* a;
  bool bad = false;
  const Tensor* may(int i) {
    if (a[i] == Py_None) return nullptr;
    if (!THPVariable_Check(a[i])) {
      bad = true;
      return nullptr;
    }
    return &THPVariable_Unpack(a[i]);
  }
  const Tensor* must(int i) {
    const Tensor* t = may(i);
    if (t == nullptr) bad = true;
    return t;
  }
  double number(int i) {
    const double v = PyFloat_AsDouble(a[i]);
    if (v == -1.0 && PyErr_Occurred()) {
      PyErr_Clear();
      bad = true;
    }
    return v;
  }
  bool flag(int i) {  // (what has no truth value raises in the caller's Python code)
    const int v = PyObject_IsTrue(a[i]);
    if (v < 0) {
      PyErr_Clear();
      bad = true;
    }
    return v == 1;
  }
  acdc_stream_t stream(int i) {
    void* p = PyLong_AsVoidPtr(a[i]);
    if (p == nullptr && PyErr_Occurred()) {
      PyErr_Clear();
      bad = true;
    }
    return static_cast<acdc_stream_t>(p);
  }
};

int32_t type_of(const Tensor& t) {
  const auto s = t.scalar_type();
  return s == at::kFloat ? ACDC_F32 : s == at::kBFloat16 ? ACDC_BF16 : -1;
}
// A view marked as conjugated or negated: its memory does not hold its values.
bool lazy(const Tensor& t) { return t.is_conj() || t.is_neg(); }
// A tensor that its storage does not hold (any more): its address is null, which the
// library would take for an argument left out, or stands for nothing.
bool gone(const Tensor& t) {
  return t.numel() > 0 &&
         at::detail::computeStorageNbytes(t.sizes(), t.strides(), t.itemsize(), size_t(t.storage_offset())) > t.storage().nbytes();
}
bool readable(const Tensor& t) { return !lazy(t) && !gone(t); }
// The same of a contiguous tensor of n elements, of which a step has a thousand.
bool whole(const Tensor& t, int64_t n) {
  return !lazy(t) && (n == 0 || size_t(t.storage_offset() + n) * t.itemsize() <= t.storage().nbytes());
}
bool vector_of(const Tensor* t, int64_t n, const at::Device& device, at::ScalarType type) {
  return t == nullptr || (t->dim() == 1 && t->size(0) == n && t->scalar_type() == type && t->device() == device &&
                          t->is_contiguous() && readable(*t));
}
bool floats(const Tensor* t, int64_t n, const at::Device& device) { return vector_of(t, n, device, at::kFloat); }
int32_t index_bits(const Tensor& t, int64_t n, const at::Device& device) {
  const auto s = t.scalar_type();
  if (s != at::kInt && s != at::kLong) return 0;
  return vector_of(&t, n, device, s) ? (s == at::kInt ? 32 : 64) : 0;
}

struct Logits {
  const Tensor* x = nullptr;
  int64_t rows = 0, stride = 0;
  int32_t classes = 0, dtype = 0, bits = 0;
  bool read(const Tensor* t, const Tensor* targets) {
    if (t == nullptr || targets == nullptr || !plain(*t)) return false;
    x = t;
    rows = t->size(0);
    classes = int32_t(t->size(1));
    stride = step(*t);
    dtype = type_of(*t);
    bits = index_bits(*targets, rows, t->device());
    return bits != 0;
  }
  static int64_t step(const Tensor& t) { return t.size(0) <= 1 ? std::max(t.stride(0), t.size(1)) : t.stride(0); }
  static bool plain(const Tensor& t) {
    return t.dim() == 2 && t.is_cuda() && type_of(t) >= 0 && t.size(1) >= 1 && t.size(1) <= 0x7fffffff &&
           (t.size(1) == 1 || t.stride(1) == 1) && step(t) >= t.size(1) && readable(t);
  }
  Tensor make(at::IntArrayRef size) const { return at::empty(size, x->options().dtype(at::kFloat)); }
  // the gradient's tensor: `out`, or a new one
  bool gradient(const Tensor* out, Tensor* g, int64_t* g_stride) const {
    if (out == nullptr) {
      *g = at::empty({rows, int64_t(classes)}, x->options());
      *g_stride = classes;
      return true;
    }
    if (!plain(*out) || out->sizes() != x->sizes() || out->scalar_type() != x->scalar_type() || out->device() != x->device())
      return false;
    *g = *out;
    *g_stride = step(*out);
    return true;
  }
  bool workspace(const Tensor* given, size_t need, Tensor* ws) const {
    if (given == nullptr) {
      *ws = at::empty({int64_t(std::max<size_t>(need, 1))}, x->options().dtype(at::kByte));
      return true;
    }
    if (given->scalar_type() != at::kByte || given->dim() != 1 || size_t(given->numel()) < need ||
        given->device() != x->device() || !given->is_contiguous() || gone(*given))
      return false;
    *ws = *given;
    return true;
  }
};

template <class T = float>
T* ptr(const Tensor* t) {
  return t == nullptr ? nullptr : static_cast<T*>(t->data_ptr());
}
template <class T = float>
T* ptr(const Tensor& t) {
  return t.defined() ? static_cast<T*>(t.data_ptr()) : nullptr;
}
// A caller's tensor that a kernel writes: torch is told, so that autograd refuses
// a backward pass over what it saved of the old values.
void wrote(const Tensor* t) {
  if (t != nullptr && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}
PyObject* wrap(const Tensor& t) {
  if (t.defined()) return THPVariable_Wrap(t);
  Py_RETURN_NONE;
}
PyObject* tuple_of(std::initializer_list<Tensor> ts) {
  PyObject* r = PyTuple_New(Py_ssize_t(ts.size()));
  if (r == nullptr) return nullptr;
  Py_ssize_t i = 0;
  for (const Tensor& t : ts) {
    PyObject* o = wrap(t);
    if (o == nullptr) {
      Py_DECREF(r);
      return nullptr;
    }
    PyTuple_SET_ITEM(r, i++, o);
  }
  return r;
}
// No C++ exception leaves an entry point: an allocation that fails raises in Python.
template <class F>
PyObject* guarded(Py_ssize_t given, Py_ssize_t wanted, F&& f) {
  if (given != wanted) {
    PyErr_Format(PyExc_TypeError, "takes %zd arguments, got %zd", wanted, given);
    return nullptr;
  }
  try {
    return f();
  } catch (const c10::OutOfMemoryError& e) {
    PyObject* torch = PyImport_ImportModule("torch");
    PyObject* type = torch != nullptr ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
    PyErr_Clear();
    PyErr_SetString(type != nullptr ? type : PyExc_MemoryError, e.what());
    Py_XDECREF(type);
    Py_XDECREF(torch);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// (logits, targets, entropy, save, workspace, stream) -> (logp, entropy, saved)
PyObject* logprobs(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject* {
    Args a{args};
    const Tensor *x = a.must(0), *t = a.must(1), *given = a.may(4);
    const bool want_entropy = a.flag(2), save = a.flag(3);
    const acdc_stream_t stream = a.stream(5);
    Logits l;
    Tensor ws;
    if (a.bad || !l.read(x, t)) Py_RETURN_NONE;
    const size_t need = acdc_logprob_workspace_size(l.rows, l.classes, l.dtype);
    if (!l.workspace(given, need, &ws)) Py_RETURN_NONE;
    Tensor logp = l.make({l.rows}), entropy, saved;
    if (want_entropy) entropy = l.make({l.rows});
    if (save) saved = l.make({l.rows, 4});
    const int rc = acdc_logprob_forward(x->data_ptr(), l.dtype, l.stride, t->data_ptr(), l.bits, l.rows, l.classes,
                                        ptr(logp), ptr(entropy), ptr(saved), ws.data_ptr(), need, stream);
    if (rc != ACDC_OK) return PyLong_FromLong(rc);
    return tuple_of({logp, entropy, saved});
  });
}

// (logits, targets, saved, grad_logp, grad_entropy, scale, out, stream) -> grad_logits
PyObject* logprobs_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    Args a{args};
    const Tensor *x = a.must(0), *t = a.must(1), *saved = a.must(2), *g = a.must(3), *h = a.may(4), *scale = a.may(5),
                 *out = a.may(6);
    const acdc_stream_t stream = a.stream(7);
    Logits l;
    if (a.bad || !l.read(x, t)) Py_RETURN_NONE;
    const at::Device device = x->device();
    if (saved->dim() != 2 || saved->size(0) != l.rows || saved->size(1) != 4 || saved->scalar_type() != at::kFloat ||
        saved->device() != device || !saved->is_contiguous() || !readable(*saved) || !floats(g, l.rows, device) ||
        !floats(h, l.rows, device) || !floats(scale, 1, device))
      Py_RETURN_NONE;
    Tensor grad;
    int64_t grad_stride = 0;
    if (!l.gradient(out, &grad, &grad_stride)) Py_RETURN_NONE;
    const int rc = acdc_logprob_backward(x->data_ptr(), l.dtype, l.stride, t->data_ptr(), l.bits, ptr(saved), ptr(g), ptr(h),
                                         ptr(scale), grad.data_ptr(), grad_stride, l.rows, l.classes, stream);
    if (rc != ACDC_OK) return PyLong_FromLong(rc);
    wrote(out);
    return wrap(grad);
  });
}

// (logits, actions, logp_old, advantages, logp_ref, weights, clip_low, clip_high, kl_coef, entropy_coef, grad_scale,
//  mean, grad, save, out, workspace, stream) -> (stats, logp, grad_logits, saved, row_grads)
PyObject* policy(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(n, 17, [&]() -> PyObject* {
    Args a{args};
    const Tensor *x = a.must(0), *t = a.must(1), *old = a.must(2), *adv = a.must(3), *ref = a.may(4), *w = a.may(5),
                 *out = a.may(14), *given = a.may(15);
    acdc_policy_params p;
    p.clip_low = float(a.number(6));
    p.clip_high = float(a.number(7));
    p.kl_coef = float(a.number(8));
    p.entropy_coef = float(a.number(9));
    p.grad_scale = float(a.number(10));
    p.mean = a.flag(11) ? 1 : 0;
    const bool want_grad = a.flag(12), save = a.flag(13);
    const acdc_stream_t stream = a.stream(16);
    Logits l;
    if (a.bad || !l.read(x, t)) Py_RETURN_NONE;
    const at::Device device = x->device();
    for (const Tensor* v : {old, adv, ref, w})
      if (!floats(v, l.rows, device)) Py_RETURN_NONE;
    if (!(p.clip_low >= 0.f) || !(p.clip_high >= 0.f) || (p.kl_coef != 0.f && ref == nullptr)) Py_RETURN_NONE;
    Tensor grad, saved, row_grads, ws;
    int64_t grad_stride = l.classes;
    if (want_grad && !l.gradient(out, &grad, &grad_stride)) Py_RETURN_NONE;
    const size_t need = acdc_policy_workspace_size(l.rows, l.classes, l.dtype);
    if (!l.workspace(given, need, &ws)) Py_RETURN_NONE;
    Tensor stats = l.make({6}), logp = l.make({l.rows});
    if (save) {
      saved = l.make({l.rows, 4});
      row_grads = l.make({2, l.rows});
    }
    const int rc = acdc_policy_loss(x->data_ptr(), l.dtype, l.stride, t->data_ptr(), l.bits, ptr(old), ptr(ref), ptr(adv),
                                    ptr(w), l.rows, l.classes, &p, ptr(stats), ptr(logp), ptr<void>(grad), grad_stride,
                                    ptr(saved), ptr(row_grads), ws.data_ptr(), need, stream);
    if (rc != ACDC_OK) return PyLong_FromLong(rc);
    if (grad.defined()) wrote(out);
    return tuple_of({stats, logp, grad, saved, row_grads});
  });
}

// (logits, targets, offsets, logp_ref, beta, label_smoothing, grad_scale, grad, save, out, workspace, stream)
//  -> (stats, logp, grad_logits, saved, row_grads)
PyObject* preference(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(n, 12, [&]() -> PyObject* {
    Args a{args};
    const Tensor *x = a.must(0), *t = a.must(1), *off = a.must(2), *ref = a.must(3), *out = a.may(9), *given = a.may(10);
    acdc_preference_params p;
    p.beta = float(a.number(4));
    p.label_smoothing = float(a.number(5));
    p.grad_scale = float(a.number(6));
    const bool want_grad = a.flag(7), save = a.flag(8);
    const acdc_stream_t stream = a.stream(11);
    Logits l;
    if (a.bad || !l.read(x, t)) Py_RETURN_NONE;
    const at::Device device = x->device();
    if (off->dim() != 1 || off->size(0) % 2 != 1) Py_RETURN_NONE;
    const int32_t off_bits = index_bits(*off, off->size(0), device);
    const int64_t pairs = off->size(0) / 2;
    if (off_bits == 0 || !floats(ref, l.rows, device) || !(p.label_smoothing >= 0.f && p.label_smoothing <= 1.f))
      Py_RETURN_NONE;
    Tensor grad, saved, row_grads, ws;
    int64_t grad_stride = l.classes;
    if (want_grad && !l.gradient(out, &grad, &grad_stride)) Py_RETURN_NONE;
    const size_t need = acdc_preference_workspace_size(l.rows, l.classes, l.dtype, pairs);
    if (!l.workspace(given, need, &ws)) Py_RETURN_NONE;
    Tensor stats = l.make({5}), logp = l.make({l.rows});
    if (save) {
      saved = l.make({l.rows, 4});
      row_grads = l.make({2, l.rows});
    }
    const int rc = acdc_preference_loss(x->data_ptr(), l.dtype, l.stride, t->data_ptr(), l.bits, off->data_ptr(), off_bits,
                                        ptr(ref), l.rows, l.classes, pairs, &p, ptr(stats), ptr(logp), ptr<void>(grad),
                                        grad_stride, ptr(saved), ptr(row_grads), ws.data_ptr(), need, stream);
    if (rc != ACDC_OK) return PyLong_FromLong(rc);
    if (grad.defined()) wrote(out);
    return tuple_of({stats, logp, grad, saved, row_grads});
  });
}

// ---------------------------------------------------------------- the optimiser

// The items of a list or tuple; null for anything else.
struct Items {
  PyObject** at = nullptr;
  Py_ssize_t count = -1;
  explicit Items(PyObject* o) {
    if (PyList_Check(o)) {
      count = PyList_GET_SIZE(o);
      at = ((PyListObject*)o)->ob_item;
    } else if (PyTuple_Check(o)) {
      count = PyTuple_GET_SIZE(o);
      at = ((PyTupleObject*)o)->ob_item;
    }
  }
  const Tensor* tensor(Py_ssize_t i) const { return THPVariable_Check(at[i]) ? &THPVariable_Unpack(at[i]) : nullptr; }
};
// One number for all tensors, or a list of one each.
struct Numbers {
  Items items;
  double one = 0.0;
  bool ok = true;
  Numbers(PyObject* o, Py_ssize_t count) : items(o) {
    if (items.count >= 0) {
      ok = items.count == count;
    } else {
      ok = PyFloat_Check(o) || PyLong_Check(o);
      if (ok) one = value(o);
    }
  }
  double value(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
      PyErr_Clear();
      ok = false;
    }
    return v;
  }
  float of(Py_ssize_t i) { return float(items.count >= 0 ? value(items.at[i]) : one); }
};

bool plain(const Tensor* t, int64_t numel, const at::Device& device, at::ScalarType type) {
  return t != nullptr && t->scalar_type() == type && t->numel() == numel && t->device() == device && t->is_contiguous() &&
         whole(*t, numel);
}

// (params, grads, moments, masters, lr, weight_decay, beta1, beta2, eps, step, grad_scale, stream) -> status
PyObject* adamw(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(n, 12, [&]() -> PyObject* {
    Args a{args};
    const Items params(args[0]), grads(args[1]), moments(args[2]);
    const Py_ssize_t count = params.count;
    if (count < 1 || count > 0x7fffffff || grads.count != count || moments.count != count) Py_RETURN_NONE;
    const bool with_masters = args[3] != Py_None;
    const Items masters(with_masters ? args[3] : args[0]);
    Numbers lr(args[4], count), decay(args[5], count);
    if (masters.count != count || !lr.ok || !decay.ok) Py_RETURN_NONE;
    const double beta1 = a.number(6), beta2 = a.number(7), eps = a.number(8);
    if (!PyLong_Check(args[9])) Py_RETURN_NONE;
    const long long step = PyLong_AsLongLong(args[9]);
    const Tensor* scale = a.may(10);
    const acdc_stream_t stream = a.stream(11);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      a.bad = true;
    }
    const Tensor* first = params.tensor(0);
    if (a.bad || first == nullptr || !first->is_cuda()) Py_RETURN_NONE;
    const at::Device device = first->device();
    if (scale != nullptr && !plain(scale, 1, device, at::kFloat)) Py_RETURN_NONE;
    std::vector<acdc_adamw_tensor> records(static_cast<size_t>(count));
    for (Py_ssize_t i = 0; i < count; ++i) {
      const Tensor *p = params.tensor(i), *g = grads.tensor(i);
      if (p == nullptr || g == nullptr || type_of(*p) < 0 || type_of(*g) < 0 || !p->is_contiguous() ||
          p->device() != device || g->sizes() != p->sizes() || g->device() != device || !g->is_contiguous())
        Py_RETURN_NONE;
      const int64_t numel = p->numel();
      if (!whole(*p, numel) || !whole(*g, numel)) Py_RETURN_NONE;
      acdc_adamw_tensor& r = records[size_t(i)];
      r = acdc_adamw_tensor{p->data_ptr(), nullptr, g->data_ptr(), nullptr, nullptr, nullptr, nullptr, numel,
                            lr.of(i), decay.of(i), type_of(*p), type_of(*g)};
      const Items m(moments.at[i]);
      if (m.count != 2 && m.count != 4) Py_RETURN_NONE;
      const auto type = m.count == 2 ? at::kFloat : at::kFloat8_e4m3fn;
      if (!plain(m.tensor(0), numel, device, type) || !plain(m.tensor(1), numel, device, type)) Py_RETURN_NONE;
      r.m = m.tensor(0)->data_ptr();
      r.v = m.tensor(1)->data_ptr();
      if (m.count == 4) {
        const int64_t blocks = (numel + 255) / 256;
        if (!plain(m.tensor(2), blocks, device, at::kFloat) || !plain(m.tensor(3), blocks, device, at::kFloat))
          Py_RETURN_NONE;
        r.m_scale = ptr(m.tensor(2));
        r.v_scale = ptr(m.tensor(3));
      }
      if (with_masters && masters.at[i] != Py_None) {
        const Tensor* w = masters.tensor(i);
        if (r.param_type != ACDC_BF16 || !plain(w, numel, device, at::kFloat)) Py_RETURN_NONE;
        r.master = ptr(w);
      }
    }
    if (!lr.ok || !decay.ok) Py_RETURN_NONE;
    const int rc = acdc_adamw_step(records.data(), int32_t(count), beta1, beta2, eps, step, ptr(scale), stream);
    if (rc == ACDC_OK) {
      for (Py_ssize_t i = 0; i < count; ++i) {
        wrote(params.tensor(i));
        if (records[size_t(i)].master != nullptr) wrote(masters.tensor(i));
        const Items m(moments.at[i]);
        for (Py_ssize_t k = 0; k < m.count; ++k) wrote(m.tensor(k));
      }
    }
    return PyLong_FromLong(rc);
  });
}

// (grads, max_norm, out, stream) -> [norm, scale]
PyObject* grad_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(n, 4, [&]() -> PyObject* {
    Args a{args};
    const Items grads(args[0]);
    const Py_ssize_t count = grads.count;
    if (count < 1 || count > 0x7fffffff) Py_RETURN_NONE;
    const float most = float(a.number(1));
    const Tensor* out = a.may(2);
    const acdc_stream_t stream = a.stream(3);
    const Tensor* first = grads.tensor(0);
    if (a.bad || first == nullptr || !first->is_cuda()) Py_RETURN_NONE;
    const at::Device device = first->device();
    std::vector<const void*> ptrs(static_cast<size_t>(count));
    std::vector<int64_t> sizes(static_cast<size_t>(count));
    std::vector<int32_t> types(static_cast<size_t>(count));
    for (Py_ssize_t i = 0; i < count; ++i) {
      const Tensor* g = grads.tensor(i);
      if (g == nullptr || type_of(*g) < 0 || !g->is_contiguous() || g->device() != device || gone(*g)) Py_RETURN_NONE;
      ptrs[size_t(i)] = g->data_ptr();
      sizes[size_t(i)] = g->numel();
      types[size_t(i)] = type_of(*g);
    }
    if (!floats(out, 2, device)) Py_RETURN_NONE;
    const size_t need = acdc_grad_norm_workspace_size(sizes.data(), int32_t(count));
    Tensor ws = at::empty({int64_t(std::max<size_t>(need, 1))}, first->options().dtype(at::kByte));
    Tensor result = out != nullptr ? *out : at::empty({2}, first->options().dtype(at::kFloat));
    const int rc = acdc_grad_norm(ptrs.data(), sizes.data(), types.data(), int32_t(count), most, ptr(result), ws.data_ptr(),
                                  need, stream);
    if (rc != ACDC_OK) return PyLong_FromLong(rc);
    wrote(out);
    return wrap(result);
  });
}

// ------------------------------------------------ the language-model operators

// Rows of float32 or bfloat16 values on one device; `bad` where something is not plain.
struct Matrix {
  const Tensor* t = nullptr;
  int64_t rows = 0, width = 0, stride = 0;
  int32_t dtype = 0;
  bool read(const Tensor* m) {
    if (m == nullptr || !Logits::plain(*m)) return false;
    t = m;
    rows = m->size(0);
    width = m->size(1);
    stride = Logits::step(*m);
    dtype = type_of(*m);
    return true;
  }
  bool like(const Matrix& m) const { return rows == m.rows && width == m.width && t->device() == m.t->device(); }
  at::Device device() const { return t->device(); }
  Tensor make(at::IntArrayRef size, at::ScalarType type) const { return at::empty(size, t->options().dtype(type)); }
  Tensor floats(at::IntArrayRef size) const { return make(size, at::kFloat); }
  // a workspace of `need` bytes that begins at a multiple of 256
  bool workspace(const Tensor* given, size_t need, Tensor* ws) const {
    if (given == nullptr) {
      *ws = make({int64_t(std::max<size_t>(need, 1))}, at::kByte);
      return true;
    }
    if (given->scalar_type() != at::kByte || given->dim() != 1 || size_t(given->numel()) < need ||
        given->device() != t->device() || !given->is_contiguous() || gone(*given) ||
        reinterpret_cast<uintptr_t>(given->data_ptr()) % 256 != 0)
      return false;
    *ws = *given;
    return true;
  }
};
at::ScalarType scalar(int32_t dtype) { return dtype == ACDC_F32 ? at::kFloat : at::kBFloat16; }
// A tensor that the call writes: the caller's, or a new one.
bool target_matrix(const Tensor* given, const Matrix& like, int64_t rows, int64_t width, at::ScalarType type, bool any_type,
                   Tensor* out, Matrix* m) {
  if (given == nullptr) *out = like.make({rows, width}, type);
  else *out = *given;
  if (given != nullptr && (!m->read(given) || (!any_type && given->scalar_type() != type))) return false;
  if (given == nullptr) {
    m->t = out;
    m->rows = rows;
    m->width = width;
    m->stride = width;
    m->dtype = type == at::kFloat ? ACDC_F32 : ACDC_BF16;
  }
  return m->rows == rows && m->width == width && out->device() == like.device();
}
// weights and biases: a vector of either type
bool width_vector(const Tensor* t, int64_t n, const at::Device& device) {
  return t == nullptr || (type_of(*t) >= 0 && vector_of(t, n, device, t->scalar_type()));
}
// What the C entry point refuses, the caller's Python code puts into words.
bool refused(int rc) { return rc == ACDC_ERR_INVALID_ARG; }

struct Head {
  Matrix hidden, weight;
  acdc_vocab_head h;
  size_t need = 0;
  Tensor ws;
  bool read(const Tensor* x, const Tensor* w, const Tensor* targets, bool gradient, const Tensor* given) {
    if (!hidden.read(x) || !weight.read(w) || targets == nullptr || hidden.width != weight.width || weight.rows < 1 ||
        weight.rows > 0x7fffffff || hidden.dtype != weight.dtype || hidden.device() != weight.device())
      return false;
    const int32_t bits = index_bits(*targets, hidden.rows, hidden.device());
    if (bits == 0) return false;
    h = acdc_vocab_head{x->data_ptr(), w->data_ptr(), targets->data_ptr(), hidden.stride, weight.stride, hidden.rows,
                        int32_t(hidden.width), int32_t(weight.rows), hidden.dtype, bits};
    need = acdc_vocab_workspace_size(h.rows, h.width, h.classes, h.dtype, gradient ? 1 : 0);
    return need != 0 && hidden.workspace(given, need, &ws);
  }
  bool grads(const Tensor* out, const Tensor* grad_weight, bool accumulate, bool want_hidden, bool want_weight, Tensor* gh,
             Tensor* gw, acdc_vocab_grads* g) const {
    *g = acdc_vocab_grads{nullptr, nullptr, 0, 0, 0, accumulate ? 1 : 0};
    Matrix m;
    if (want_hidden) {
      if (!target_matrix(out, hidden, h.rows, h.width, scalar(h.dtype), false, gh, &m)) return false;
      g->hidden = gh->data_ptr();
      g->hidden_stride = m.stride;
    }
    if (want_weight) {
      if (accumulate && grad_weight == nullptr) return false;
      if (!target_matrix(grad_weight, hidden, h.classes, h.width, scalar(h.dtype), true, gw, &m)) return false;
      if (m.dtype != h.dtype && m.dtype != ACDC_F32) return false;
      g->weight = gw->data_ptr();
      g->weight_stride = m.stride;
      g->weight_type = m.dtype;
    }
    return true;
  }
};

// (hidden, weight, targets, save, workspace, stream) -> (logp, saved)
PyObject* vocab_logprobs(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject* {
    Args a{args};
    const Tensor *x = a.must(0), *w = a.must(1), *t = a.must(2), *given = a.may(4);
    const bool save = a.flag(3);
    const acdc_stream_t stream = a.stream(5);
    Head head;
    if (a.bad || !head.read(x, w, t, false, given)) Py_RETURN_NONE;
    Tensor logp = head.hidden.floats({head.h.rows}), saved;
    if (save) saved = head.hidden.floats({head.h.rows, 2});
    const int rc = acdc_vocab_logprob(&head.h, ptr(logp), ptr(saved), head.ws.data_ptr(), head.need, stream);
    if (refused(rc)) Py_RETURN_NONE;
    if (rc != ACDC_OK) return PyLong_FromLong(rc);
    return tuple_of({logp, saved});
  });
}

// (hidden, weight, targets, saved, grad_logp, scale, want_hidden, want_weight, out, grad_weight, accumulate, workspace,
//  stream) -> (grad_hidden, grad_weight)
PyObject* vocab_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(n, 13, [&]() -> PyObject* {
    Args a{args};
    const Tensor *x = a.must(0), *w = a.must(1), *t = a.must(2), *saved = a.must(3), *g = a.must(4), *scale = a.may(5),
                 *out = a.may(8), *gw_given = a.may(9), *given = a.may(11);
    const bool want_hidden = a.flag(6), want_weight = a.flag(7), accumulate = a.flag(10);
    const acdc_stream_t stream = a.stream(12);
    Head head;
    if (a.bad || !head.read(x, w, t, true, given)) Py_RETURN_NONE;
    const at::Device device = head.hidden.device();
    if (saved->dim() != 2 || saved->size(0) != head.h.rows || saved->size(1) != 2 || saved->scalar_type() != at::kFloat ||
        saved->device() != device || !saved->is_contiguous() || !readable(*saved) || !floats(g, head.h.rows, device) ||
        !floats(scale, 1, device))
      Py_RETURN_NONE;
    Tensor gh, gw;
    acdc_vocab_grads grads;
    if (!head.grads(out, gw_given, accumulate, want_hidden, want_weight, &gh, &gw, &grads)) Py_RETURN_NONE;
    const int rc = acdc_vocab_backward(&head.h, ptr(saved), ptr(g), ptr(scale), &grads, head.ws.data_ptr(), head.need, stream);
    if (refused(rc)) Py_RETURN_NONE;
    if (rc != ACDC_OK) return PyLong_FromLong(rc);
    if (want_hidden) wrote(out);
    if (want_weight) wrote(gw_given);
    return tuple_of({gh, gw});
  });
}

// (hidden, weight, targets, weights, mean, grad_scale, want_hidden, want_weight, save, out, grad_weight, accumulate,
//  workspace, stream) -> (stats, logp, grad_hidden, grad_weight, saved, row_grads)
PyObject* vocab_loss(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(n, 14, [&]() -> PyObject* {
    Args a{args};
    const Tensor *x = a.must(0), *w = a.must(1), *t = a.must(2), *weights = a.may(3), *out = a.may(9), *gw_given = a.may(10),
                 *given = a.may(12);
    acdc_vocab_params p;
    p.mean = a.flag(4) ? 1 : 0;
    p.grad_scale = float(a.number(5));
    const bool want_hidden = a.flag(6), want_weight = a.flag(7), save = a.flag(8), accumulate = a.flag(11);
    const acdc_stream_t stream = a.stream(13);
    Head head;
    if (a.bad || !head.read(x, w, t, want_hidden || want_weight, given)) Py_RETURN_NONE;
    if (!floats(weights, head.h.rows, head.hidden.device())) Py_RETURN_NONE;
    Tensor gh, gw, saved, row_grads;
    acdc_vocab_grads grads;
    if (!head.grads(out, gw_given, accumulate, want_hidden, want_weight, &gh, &gw, &grads)) Py_RETURN_NONE;
    Tensor stats = head.hidden.floats({2}), logp = head.hidden.floats({head.h.rows});
    if (save) {
      saved = head.hidden.floats({head.h.rows, 2});
      row_grads = head.hidden.floats({head.h.rows});
    }
    const int rc = acdc_vocab_loss(&head.h, ptr(weights), &p, ptr(stats), ptr(logp), ptr(saved), ptr(row_grads), &grads,
                                   head.ws.data_ptr(), head.need, stream);
    if (refused(rc)) Py_RETURN_NONE;
    if (rc != ACDC_OK) return PyLong_FromLong(rc);
    if (want_hidden) wrote(out);
    if (want_weight) wrote(gw_given);
    return tuple_of({stats, logp, gh, gw, saved, row_grads});
  });
}

// dtype: 0 or 1, or -1 for `otherwise`
at::ScalarType type_or(double dtype, at::ScalarType otherwise) { return dtype < 0 ? otherwise : scalar(int32_t(dtype)); }

// (x, weight, bias, eps, dtype, save, out, stream) -> (y, saved)
PyObject* norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    Args a{args};
    const Tensor *x = a.must(0), *weight = a.may(1), *bias = a.may(2), *out = a.may(6);
    const double eps = a.number(3), dtype = a.number(4);
    const bool save = a.flag(5);
    const acdc_stream_t stream = a.stream(7);
    Matrix m, to;
    if (a.bad || !m.read(x) || !width_vector(weight, m.width, m.device()) || !width_vector(bias, m.width, m.device()) ||
        (weight != nullptr && bias != nullptr && weight->scalar_type() != bias->scalar_type()))
      Py_RETURN_NONE;
    Tensor y, saved;
    if (!target_matrix(out, m, m.rows, m.width, type_or(dtype, out != nullptr ? out->scalar_type() : x->scalar_type()), false, &y, &to))
      Py_RETURN_NONE;
    if (save) saved = m.floats({m.rows, 2});
    const Tensor* v = weight != nullptr ? weight : bias;
    const int rc = acdc_norm_forward(x->data_ptr(), m.dtype, m.stride, ptr<void>(weight), ptr<void>(bias), v != nullptr ? type_of(*v) : 0,
                                     float(eps), y.data_ptr(), to.dtype, to.stride, ptr(saved), m.rows, int32_t(m.width), stream);
    if (refused(rc)) Py_RETURN_NONE;
    if (rc != ACDC_OK) return PyLong_FromLong(rc);
    wrote(out);
    return tuple_of({y, saved});
  });
}

// (x, grad_y, weight, saved, out, grad_weight, grad_bias, given, accumulate, want_x, want_weight, want_bias, dtype, workspace,
//  stream) -> (grad_x, grad_weight, grad_bias); given: the two sums go into grad_weight and grad_bias (None: not wanted)
PyObject* norm_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(n, 15, [&]() -> PyObject* {
    Args a{args};
    const Tensor *x = a.must(0), *gy = a.must(1), *weight = a.may(2), *saved = a.must(3), *out = a.may(4), *gw_in = a.may(5),
                 *gb_in = a.may(6), *ws_in = a.may(13);
    const bool given = a.flag(7), accumulate = a.flag(8), want_x = a.flag(9), want_w = a.flag(10), want_b = a.flag(11);
    const double dtype = a.number(12);
    const acdc_stream_t stream = a.stream(14);
    Matrix m, g, to;
    if (a.bad || !m.read(x) || !g.read(gy) || !g.like(m) || !width_vector(weight, m.width, m.device())) Py_RETURN_NONE;
    const at::Device device = m.device();
    if (saved->dim() != 2 || saved->size(0) != m.rows || saved->size(1) != 2 || saved->scalar_type() != at::kFloat ||
        saved->device() != device || !saved->is_contiguous() || !readable(*saved) || (accumulate && !given))
      Py_RETURN_NONE;
    Tensor gx, gw, gb;
    if (want_x && !target_matrix(out, m, m.rows, m.width, x->scalar_type(), false, &gx, &to)) Py_RETURN_NONE;
    if (given) {
      if (!width_vector(gw_in, m.width, device) || !width_vector(gb_in, m.width, device)) Py_RETURN_NONE;
      if (want_w && gw_in != nullptr) gw = *gw_in;
      if (want_b && gb_in != nullptr) gb = *gb_in;
      if (gw.defined() && gb.defined() && gw.scalar_type() != gb.scalar_type()) Py_RETURN_NONE;
    } else {
      const at::ScalarType type = type_or(dtype, weight != nullptr ? weight->scalar_type() : at::kFloat);
      if (want_w) gw = m.make({m.width}, type);
      if (want_b) gb = m.make({m.width}, type);
    }
    const int32_t type = gw.defined() ? type_of(gw) : gb.defined() ? type_of(gb) : 0;
    const size_t need = acdc_norm_workspace_size(m.rows, int32_t(std::min<int64_t>(m.width, 0x7fffffff)));
    Tensor ws;
    if (need == 0 || ((need > 256 || ws_in != nullptr) && !m.workspace(ws_in, need, &ws))) Py_RETURN_NONE;
    const int rc = acdc_norm_backward(x->data_ptr(), m.dtype, m.stride, gy->data_ptr(), g.dtype, g.stride, ptr<void>(weight),
                                      weight != nullptr ? type_of(*weight) : 0, ptr(saved), ptr<void>(gx), to.stride, ptr<void>(gw),
                                      ptr<void>(gb), type, accumulate ? 1 : 0, m.rows, int32_t(m.width), ptr<void>(ws), need, stream);
    if (refused(rc)) Py_RETURN_NONE;
    if (rc != ACDC_OK) return PyLong_FromLong(rc);
    if (want_x) wrote(out);
    if (given) {
      if (gw.defined()) wrote(gw_in);
      if (gb.defined()) wrote(gb_in);
    }
    return tuple_of({gx, gw, gb});
  });
}

// (tokens, weight, scale, dtype, out, stream) -> rows
PyObject* embedding(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject* {
    Args a{args};
    const Tensor *t = a.must(0), *w = a.must(1), *out = a.may(4);
    const double scale = a.number(2), dtype = a.number(3);
    const acdc_stream_t stream = a.stream(5);
    Matrix m, to;
    if (a.bad || !m.read(w) || t->dim() != 1 || m.rows > 0x7fffffff) Py_RETURN_NONE;
    const int64_t rows = t->size(0);
    const int32_t bits = index_bits(*t, rows, m.device());
    Tensor y;
    if (bits == 0 || !target_matrix(out, m, rows, m.width, type_or(dtype, out != nullptr ? out->scalar_type() : w->scalar_type()), false, &y, &to))
      Py_RETURN_NONE;
    const int rc = acdc_embedding_forward(t->data_ptr(), bits, w->data_ptr(), m.dtype, m.stride, float(scale), y.data_ptr(), to.dtype,
                                          to.stride, rows, int32_t(m.width), int32_t(m.rows), stream);
    if (refused(rc)) Py_RETURN_NONE;
    if (rc != ACDC_OK) return PyLong_FromLong(rc);
    wrote(out);
    return wrap(y);
  });
}

// (tokens, grad_rows, classes, scale, dtype, grad_weight, accumulate, workspace, stream) -> grad_weight
PyObject* embedding_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(n, 9, [&]() -> PyObject* {
    Args a{args};
    const Tensor *t = a.must(0), *g = a.must(1), *given = a.may(5), *ws_in = a.may(7);
    if (!PyLong_Check(args[2])) Py_RETURN_NONE;
    const long long classes = PyLong_AsLongLong(args[2]);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      Py_RETURN_NONE;
    }
    const double scale = a.number(3), dtype = a.number(4);
    const bool accumulate = a.flag(6);
    const acdc_stream_t stream = a.stream(8);
    Matrix m, to;
    if (a.bad || !m.read(g) || classes < 1 || classes > 0x7fffffff || (accumulate && given == nullptr)) Py_RETURN_NONE;
    const int32_t bits = t->dim() == 1 ? index_bits(*t, m.rows, m.device()) : 0;
    Tensor gw, ws;
    if (bits == 0 ||
        !target_matrix(given, m, classes, m.width, type_or(dtype, given != nullptr ? given->scalar_type() : g->scalar_type()), false, &gw, &to))
      Py_RETURN_NONE;
    const size_t need = acdc_embedding_workspace_size(m.rows, int32_t(std::min<int64_t>(m.width, 0x7fffffff)), int32_t(classes));
    if (need == 0 || !m.workspace(ws_in, need, &ws)) Py_RETURN_NONE;
    const int rc = acdc_embedding_backward(t->data_ptr(), bits, g->data_ptr(), m.dtype, m.stride, float(scale), gw.data_ptr(), to.dtype,
                                           to.stride, accumulate ? 1 : 0, m.rows, int32_t(m.width), int32_t(classes), ws.data_ptr(),
                                           need, stream);
    if (refused(rc)) Py_RETURN_NONE;
    if (rc != ACDC_OK) return PyLong_FromLong(rc);
    wrote(given);
    return wrap(gw);
  });
}

// (tensors...) -> whether a node that computes one of them, or sums up its gradient, was
// made on the default stream
PyObject* made_on_default_stream(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(n, n, [&]() -> PyObject* {
    Args a{args};
    for (Py_ssize_t i = 0; i < n; ++i) {
      const Tensor* t = a.may(int(i));
      if (t == nullptr || !t->requires_grad()) continue;
      const auto node = t->grad_fn() ? t->grad_fn() : torch::autograd::impl::try_get_grad_accumulator(*t);
      if (!node) continue;
      const auto stream = node->stream();
      if (stream && stream->id() == 0) Py_RETURN_TRUE;
    }
    Py_RETURN_FALSE;
  });
}

#define ENTRY(name) {#name, (PyCFunction)(void*)name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(logprobs), ENTRY(logprobs_backward), ENTRY(policy),     ENTRY(preference),
                         ENTRY(adamw),    ENTRY(grad_norm),         ENTRY(vocab_logprobs), ENTRY(vocab_backward),
                         ENTRY(vocab_loss), ENTRY(norm), ENTRY(norm_backward), ENTRY(embedding), ENTRY(embedding_backward),
                         ENTRY(made_on_default_stream),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_train_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__train_binding() { return PyModule_Create(&module); }

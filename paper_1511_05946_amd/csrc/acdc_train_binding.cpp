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
#include <torch/csrc/autograd/python_variable.h>

#include <vector>

#include "acdc_train.h"

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

#define ENTRY(name) {#name, (PyCFunction)(void*)name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(logprobs), ENTRY(logprobs_backward), ENTRY(policy),     ENTRY(preference),
                         ENTRY(adamw),    ENTRY(grad_norm),         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_train_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__train_binding() { return PyModule_Create(&module); }

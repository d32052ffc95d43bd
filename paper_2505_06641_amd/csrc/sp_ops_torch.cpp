// The operators that train the heads, for Python: checks of tensors' types, shapes, strides and devices (which the C entry points of
// sneakpeek.h cannot see), then the call.  The same checks written in Python take longer than the launch that they guard: 3.7 us a
// call of layer norm, beside 3.3 us for the launch.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <memory>
#include <new>
#include <sstream>
#include <string>
#include <vector>

#include "sneakpeek.h"

namespace {

PyObject* g_error = nullptr;                    // the binding's SneakPeekError(status, where, detail)

// One call in the making: who it is, and whether something has been refused.  After a refusal the Python error is set.
struct Call {
  const char* where;
  int device;
  bool bad = false;

  void refuse(const std::string& detail) {
    if (bad) return;
    bad = true;
    if (PyErr_Occurred()) return;
    PyObject* e = g_error ? PyObject_CallFunction(g_error, "iss", (int)SP_EINVAL, where, detail.c_str()) : nullptr;
    if (e) {
      PyErr_SetObject(g_error, e);
      Py_DECREF(e);
    } else if (!PyErr_Occurred()) {
      PyErr_SetString(PyExc_ValueError, detail.c_str());
    }
  }

  const at::Tensor* tensor(PyObject* o, const char* name) {
    if (!o || o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) {
      refuse(std::string(name) + " is no tensor");
      return nullptr;
    }
    return &THPVariable_Unpack(o);
  }
  const at::Tensor* needed(PyObject* o, const char* name) {
    const at::Tensor* t = tensor(o, name);
    if (!t && !bad) refuse(std::string(name) + " is missing");
    return t;
  }
  // A matrix that says what the others have to fit.
  const at::Tensor* matrix(PyObject* o, const char* name, int64_t* rows, int64_t* cols) {
    const at::Tensor* t = needed(o, name);
    if (!t) return nullptr;
    if (t->dim() != 2) {
      refuse(std::string(name) + " is no matrix");
      return nullptr;
    }
    *rows = t->size(0);
    *cols = t->size(1);
    return t;
  }
  int32_t dtype(const at::Tensor* t, const char* name) {
    if (t && t->scalar_type() == at::kFloat) return SP_F32;
    if (t && t->scalar_type() == at::kBFloat16) return SP_BF16;
    if (t) refuse(std::string(name) + " is neither float32 nor bfloat16");
    return SP_F32;
  }
  bool basics(const at::Tensor& t, at::ScalarType type, at::IntArrayRef shape) {
    return t.scalar_type() == type && t.layout() == at::kStrided && t.sizes() == shape && t.is_cuda() && t.device().index() == device;
  }
  void misfit(const at::Tensor& t, const char* name, at::ScalarType type, at::IntArrayRef shape) {
    std::ostringstream s;
    s << name << ": " << t.scalar_type() << " " << t.sizes() << " on " << t.device();
    if (t.layout() == at::kStrided) s << " with strides " << t.strides();
    s << ", where " << type << " " << shape << " with contiguous rows on device " << device << " is asked for";
    refuse(s.str());
  }
  // Address of a contiguous tensor, of an absent one null.
  void* whole(const at::Tensor* t, const char* name, at::ScalarType type, at::IntArrayRef shape) {
    if (!t || bad) return nullptr;
    if (basics(*t, type, shape) && t->is_contiguous()) return t->data_ptr();
    misfit(*t, name, type, shape);
    return nullptr;
  }
  void* whole(PyObject* o, const char* name, at::ScalarType type, at::IntArrayRef shape) { return whole(tensor(o, name), name, type, shape); }
  // Address and row stride of a matrix with contiguous rows.
  void* rows(const at::Tensor* t, const char* name, at::ScalarType type, int64_t n, int64_t width, int64_t* stride) {
    *stride = width;
    if (!t || bad) return nullptr;
    if (basics(*t, type, {n, width}) && (t->stride(1) == 1 || width <= 1) && (t->stride(0) >= width || n <= 1)) {
      if (t->stride(0) > width) *stride = t->stride(0);
      return t->data_ptr();
    }
    misfit(*t, name, type, {n, width});
    return nullptr;
  }
  void* rows(PyObject* o, const char* name, at::ScalarType type, int64_t n, int64_t width, int64_t* stride) {
    return rows(tensor(o, name), name, type, n, width, stride);
  }
  int32_t count(int64_t v, const char* name) {
    if (v > INT32_MAX) refuse(std::string(name) + " is beyond 2^31 - 1");
    return (int32_t)v;
  }
  double number(PyObject* o, double otherwise) {
    if (!o) return otherwise;
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) refuse("");
    return v;
  }
  bool truth(PyObject* o) {
    const int v = o ? PyObject_IsTrue(o) : 0;
    if (v < 0) refuse("");
    return v > 0;
  }
  // The stream's handle; by default that of the device's current stream.
  void* stream(PyObject* o) {
    if (bad) return nullptr;
    if (!o || o == Py_None) return (void*)c10::hip::getCurrentHIPStream((c10::DeviceIndex)device).stream();
    PyObject* h = PyObject_GetAttrString(o, "cuda_stream");
    void* s = h ? PyLong_AsVoidPtr(h) : nullptr;
    Py_XDECREF(h);
    if (PyErr_Occurred()) refuse("");
    return s;
  }
};

// Arguments of a method by position or name: names[i] goes to out[i], those not given stay null.
template <size_t N>
struct Names {
  const char* text[N];
  PyObject* word[N];
  explicit Names(const char* const (&t)[N]) {
    for (size_t i = 0; i < N; ++i) {
      text[i] = t[i];
      word[i] = PyUnicode_InternFromString(t[i]);
    }
  }
  bool parse(Call& c, PyObject* const* args, Py_ssize_t n, PyObject* kw, PyObject* (&out)[N]) const {
    for (size_t i = 0; i < N; ++i) out[i] = nullptr;
    if (n > (Py_ssize_t)N) {
      PyErr_Format(PyExc_TypeError, "%s takes %d arguments, %d were given", c.where, (int)N, (int)n);
      c.bad = true;
      return false;
    }
    for (Py_ssize_t i = 0; i < n; ++i) out[i] = args[i];
    const Py_ssize_t more = kw ? PyTuple_GET_SIZE(kw) : 0;
    for (Py_ssize_t j = 0; j < more; ++j) {
      PyObject* key = PyTuple_GET_ITEM(kw, j);
      size_t i = 0;
      while (i < N && word[i] != key) ++i;
      if (i == N)
        for (i = 0; i < N && PyUnicode_Compare(word[i], key) != 0; ++i) {}
      if (i == N || out[i]) {
        PyErr_Format(PyExc_TypeError, i == N ? "%s has no argument %R" : "%s got argument %R twice", c.where, key);
        c.bad = true;
        return false;
      }
      out[i] = args[n + j];
    }
    return true;
  }
};

struct OpsObject {
  PyObject_HEAD
  sp_ops* handle;
  int device;
};

PyObject* finish(OpsObject* self, const Call& c, sp_status rc) {
  if (rc == SP_OK) Py_RETURN_NONE;
  const std::string detail = std::string(sp_strerror(rc)) + " " + sp_ops_last_hip_error(self->handle);
  PyObject* e = g_error ? PyObject_CallFunction(g_error, "iss", (int)rc, c.where, detail.c_str()) : nullptr;
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  } else if (!PyErr_Occurred()) {
    PyErr_SetString(PyExc_RuntimeError, detail.c_str());
  }
  return nullptr;
}

PyObject* layer_norm(OpsObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  static const Names<8> names({"x", "y", "gamma", "beta", "eps", "mean", "rstd", "stream"});
  Call c{"sp_layer_norm", self->device};
  PyObject* v[8];
  if (!names.parse(c, args, nargs, kw, v)) return nullptr;
  int64_t n = 0, d = 0, xs, ys;
  const at::Tensor *x = c.matrix(v[0], "x", &n, &d), *y = c.needed(v[1], "y");
  if (c.bad) return nullptr;
  const int32_t dt = c.dtype(x, "x");
  const auto type = x->scalar_type();
  void *px = c.rows(x, "x", type, n, d, &xs), *py = c.rows(y, "y", type, n, d, &ys);
  void *gamma = c.whole(v[2], "gamma", at::kFloat, {d}), *beta = c.whole(v[3], "beta", at::kFloat, {d});
  void *mean = c.whole(v[5], "mean", at::kFloat, {n}), *rstd = c.whole(v[6], "rstd", at::kFloat, {n});
  const float eps = (float)c.number(v[4], 1e-5);
  const int32_t rows = c.count(n, "x's rows"), width = c.count(d, "x's width");
  void* s = c.stream(v[7]);
  if (c.bad) return nullptr;
  return finish(self, c, sp_layer_norm(self->handle, rows, width, dt, px, xs, (float*)gamma, (float*)beta, eps, py, ys, (float*)mean,
                                       (float*)rstd, s));
}

PyObject* layer_norm_backward(OpsObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  static const Names<9> names({"dy", "x", "mean", "rstd", "gamma", "dx", "dgamma", "dbeta", "stream"});
  Call c{"sp_layer_norm_backward", self->device};
  PyObject* v[9];
  if (!names.parse(c, args, nargs, kw, v)) return nullptr;
  int64_t n = 0, d = 0, dys, xs, dxs;
  const at::Tensor *x = c.matrix(v[1], "x", &n, &d), *dy = c.needed(v[0], "dy"), *mean = c.needed(v[2], "mean"),
                   *rstd = c.needed(v[3], "rstd");
  if (c.bad) return nullptr;
  const int32_t dt = c.dtype(x, "x");
  const auto type = x->scalar_type();
  void *pdy = c.rows(dy, "dy", type, n, d, &dys), *px = c.rows(x, "x", type, n, d, &xs), *pdx = c.rows(v[5], "dx", type, n, d, &dxs);
  void *pm = c.whole(mean, "mean", at::kFloat, {n}), *pr = c.whole(rstd, "rstd", at::kFloat, {n});
  void *gamma = c.whole(v[4], "gamma", at::kFloat, {d}), *dg = c.whole(v[6], "dgamma", at::kFloat, {d}),
       *db = c.whole(v[7], "dbeta", at::kFloat, {d});
  const int32_t rows = c.count(n, "x's rows"), width = c.count(d, "x's width");
  void* s = c.stream(v[8]);
  if (c.bad) return nullptr;
  return finish(self, c, sp_layer_norm_backward(self->handle, rows, width, dt, pdy, dys, px, xs, (float*)gamma, (float*)pm, (float*)pr,
                                                pdx, dxs, (float*)dg, (float*)db, s));
}

// Weights [groups, k, m] and the offsets of their groups.
bool weights(Call& c, PyObject* w_, PyObject* offsets_, at::ScalarType type, int64_t k, int64_t* groups, int64_t* m, void** w,
             void** offsets) {
  const at::Tensor *t = c.needed(w_, "w"), *o = c.needed(offsets_, "offsets");
  if (c.bad) return false;
  if (t->dim() != 3) {
    c.refuse("w is not [groups, inputs, outputs]");
    return false;
  }
  *groups = t->size(0);
  *m = t->size(2);
  *w = c.whole(t, "w", type, {*groups, k, *m});
  *offsets = c.whole(o, "offsets", at::kInt, {*groups + 1});
  return !c.bad;
}

PyObject* grouped_linear(OpsObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  static const Names<9> names({"x", "offsets", "w", "y", "bias", "relu", "residual", "act_out", "stream"});
  Call c{"sp_grouped_linear", self->device};
  PyObject* v[9];
  if (!names.parse(c, args, nargs, kw, v)) return nullptr;
  int64_t n = 0, k = 0, groups = 0, m = 0, xs, ys, rs, as;
  const at::Tensor *x = c.matrix(v[0], "x", &n, &k), *y = c.needed(v[3], "y");
  if (c.bad) return nullptr;
  const int32_t dt = c.dtype(x, "x"), ot = c.dtype(y, "y");
  void *w = nullptr, *offsets = nullptr;
  if (!weights(c, v[2], v[1], x->scalar_type(), k, &groups, &m, &w, &offsets)) return nullptr;
  const auto out = y->scalar_type();
  void *px = c.rows(x, "x", x->scalar_type(), n, k, &xs), *py = c.rows(y, "y", out, n, m, &ys);
  void *pr = c.rows(v[6], "residual", out, n, m, &rs), *pa = c.rows(v[7], "act_out", out, n, m, &as);
  void* bias = c.whole(v[4], "bias", at::kFloat, {groups, m});
  const int32_t act = c.truth(v[5]) ? SP_ACT_RELU : SP_ACT_NONE;
  const int32_t rows = c.count(n, "x's rows"), ki = c.count(k, "inputs"), mo = c.count(m, "outputs"), g = c.count(groups, "groups");
  void* s = c.stream(v[8]);
  if (c.bad) return nullptr;
  return finish(self, c, sp_grouped_linear(self->handle, rows, ki, mo, g, dt, px, xs, (int32_t*)offsets, w, (float*)bias, act, ot, pr, rs,
                                           py, ys, pa, as, s));
}

PyObject* grouped_linear_backward(OpsObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  static const Names<9> names({"dy", "x", "offsets", "w", "act", "dx", "dw", "db", "stream"});
  Call c{"sp_grouped_linear_backward", self->device};
  PyObject* v[9];
  if (!names.parse(c, args, nargs, kw, v)) return nullptr;
  int64_t n = 0, k = 0, groups = 0, m = 0, dys, as, xs, dxs;
  const at::Tensor *x = c.matrix(v[1], "x", &n, &k), *dy = c.needed(v[0], "dy");
  if (c.bad) return nullptr;
  const int32_t dt = c.dtype(x, "x");
  const auto type = x->scalar_type();
  void *w = nullptr, *offsets = nullptr;
  if (!weights(c, v[3], v[2], type, k, &groups, &m, &w, &offsets)) return nullptr;
  void *pdy = c.rows(dy, "dy", type, n, m, &dys), *pa = c.rows(v[4], "act", type, n, m, &as), *px = c.rows(x, "x", type, n, k, &xs),
       *pdx = c.rows(v[5], "dx", type, n, k, &dxs);
  void *dw = c.whole(v[6], "dw", at::kFloat, {groups, k, m}), *db = c.whole(v[7], "db", at::kFloat, {groups, m});
  const int32_t rows = c.count(n, "x's rows"), ki = c.count(k, "inputs"), mo = c.count(m, "outputs"), g = c.count(groups, "groups");
  void* s = c.stream(v[8]);
  if (c.bad) return nullptr;
  return finish(self, c, sp_grouped_linear_backward(self->handle, rows, ki, mo, g, dt, pdy, dys, pa, as, px, xs, (int32_t*)offsets, w, pdx,
                                                    dxs, (float*)dw, (float*)db, s));
}

PyObject* cross_entropy(OpsObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  static const Names<9> names({"logits", "label", "loss", "app", "n_classes", "weight", "scale", "dlogits", "stream"});
  Call c{"sp_cross_entropy", self->device};
  PyObject* v[9];
  if (!names.parse(c, args, nargs, kw, v)) return nullptr;
  int64_t n = 0, width = 0, zs, ds;
  const at::Tensor *z = c.matrix(v[0], "logits", &n, &width), *label = c.needed(v[1], "label"), *loss = c.needed(v[2], "loss"),
                   *classes = c.tensor(v[4], "n_classes"), *dz = c.tensor(v[7], "dlogits");
  if (c.bad) return nullptr;
  const int32_t dt = c.dtype(z, "logits"), gt = dz ? c.dtype(dz, "dlogits") : dt;
  const int64_t apps = classes ? classes->numel() : 0;
  void *pz = c.rows(z, "logits", z->scalar_type(), n, width, &zs);
  void *pd = c.rows(dz, "dlogits", dz ? dz->scalar_type() : at::kFloat, n, width, &ds);
  void *pl = c.whole(label, "label", at::kInt, {n}), *po = c.whole(loss, "loss", at::kFloat, {n});
  void *app = c.whole(v[3], "app", at::kInt, {n}), *pc = c.whole(classes, "n_classes", at::kInt, {apps}),
       *weight = c.whole(v[5], "weight", at::kFloat, {n});
  const float scale = (float)c.number(v[6], 1.0);
  const int32_t rows = c.count(n, "logits' rows"), wide = c.count(width, "logits' width"), na = c.count(apps, "n_classes");
  void* s = c.stream(v[8]);
  if (c.bad) return nullptr;
  return finish(self, c, sp_cross_entropy(self->handle, rows, wide, dt, pz, zs, na, (int32_t*)app, (int32_t*)pc, (int32_t*)pl,
                                          (float*)weight, scale, (float*)po, gt, pd, ds, s));
}

// A list of tensors as sp_clip_grad_norm takes them.  What is kept is the tensors: one that gets other storage (assignment to .data, set_,
// resize_) is found where it is at the time of the call, and checked anew.
struct Packed {
  std::vector<at::Tensor> tensors, outs;        // outs empty: in place
  std::vector<const void*> grads;               // of the call that is being made
  std::vector<void*> out;
  std::vector<int64_t> sizes;
  bool in_place = true;
  int32_t dtype = SP_F32;
  int device = -1;                              // -1: no tensors

  void collect(Call& c) {
    grads.clear();
    out.clear();
    sizes.clear();
    device = -1;
    for (size_t i = 0; i < tensors.size(); ++i) {
      const at::Tensor &g = tensors[i], &o = in_place ? g : outs[i];
      if (i == 0) {
        dtype = c.dtype(&g, "a gradient");
        device = g.is_cuda() ? g.device().index() : -2;
      }
      for (const at::Tensor* t : {&g, &o})
        if (t->layout() != at::kStrided || !t->is_contiguous() || !t->is_cuda() || t->device().index() != device ||
            t->scalar_type() != tensors[0].scalar_type())
          c.refuse("contiguous tensors of one type on one device are asked for");
      if (!c.bad && g.numel() != o.numel()) c.refuse("a gradient and its output differ in size");
      if (c.bad) return;
      grads.push_back(g.data_ptr());
      out.push_back(o.data_ptr());
      sizes.push_back(g.numel());
    }
  }
};
constexpr const char* kPacked = "sneakpeek.packed_tensors";

void free_packed(PyObject* capsule) { delete (Packed*)PyCapsule_GetPointer(capsule, kPacked); }

PyObject* pack_tensors(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  Call c{"TensorList", 0};
  if (nargs != 2 || !PyList_Check(args[0]) || (args[1] != Py_None && !PyList_Check(args[1]))) {
    PyErr_SetString(PyExc_TypeError, "pack_tensors(list, list or None)");
    return nullptr;
  }
  const Py_ssize_t n = PyList_GET_SIZE(args[0]);
  const bool in_place = args[1] == Py_None;
  if (!in_place && PyList_GET_SIZE(args[1]) != n) {
    c.refuse("as many outputs as gradients are asked for");
    return nullptr;
  }
  std::unique_ptr<Packed> p(new Packed);
  p->in_place = in_place;
  for (Py_ssize_t i = 0; i < n && !c.bad; ++i) {
    const at::Tensor* g = c.needed(PyList_GET_ITEM(args[0], i), "a gradient");
    const at::Tensor* o = in_place ? g : c.needed(PyList_GET_ITEM(args[1], i), "an output");
    if (c.bad) break;
    p->tensors.push_back(*g);
    if (!in_place) p->outs.push_back(*o);
  }
  if (!c.bad) p->collect(c);
  if (c.bad) return nullptr;
  PyObject* capsule = PyCapsule_New(p.get(), kPacked, free_packed);
  if (capsule) p.release();
  return capsule;
}

PyObject* clip_packed(OpsObject* self, PyObject* const* args, Py_ssize_t nargs) {
  Call c{"sp_clip_grad_norm", self->device};
  if (nargs != 4) {
    PyErr_SetString(PyExc_TypeError, "clip_packed(packed, max_norm, norm, stream)");
    return nullptr;
  }
  Packed* p = (Packed*)PyCapsule_GetPointer(args[0], kPacked);
  if (!p) return nullptr;
  p->collect(c);
  if (!c.bad && p->device != -1 && p->device != self->device) c.refuse("the tensors are on another device than the operators");
  if (c.bad) return nullptr;
  const float max_norm = (float)c.number(args[1], 0.0);
  void* norm = c.whole(c.bad ? nullptr : c.needed(args[2], "norm"), "norm", at::kFloat, {1});
  void* s = c.stream(args[3]);
  if (c.bad) return nullptr;
  return finish(self, c, sp_clip_grad_norm(self->handle, (int32_t)p->grads.size(), p->dtype, p->grads.data(), p->sizes.data(), max_norm,
                                           p->in_place ? nullptr : p->out.data(), (float*)norm, s));
}

PyObject* set_handle(OpsObject* self, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != 2) {
    PyErr_SetString(PyExc_TypeError, "set_handle(handle, device)");
    return nullptr;
  }
  void* h = PyLong_AsVoidPtr(args[0]);
  const long d = PyLong_AsLong(args[1]);
  if (PyErr_Occurred()) return nullptr;
  self->handle = (sp_ops*)h;
  self->device = (int)d;
  Py_RETURN_NONE;
}

// No C++ exception leaves a method (torch throws for tensors without storage, for instance).
template <auto F, typename S>
PyObject* guarded(S* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  try {
    return F(self, args, nargs, kw);
  } catch (const std::bad_alloc&) {
    PyErr_NoMemory();
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}
template <auto F, typename S>
PyObject* guarded_positional(S* self, PyObject* const* args, Py_ssize_t nargs) {
  return guarded<[](S* s, PyObject* const* a, Py_ssize_t n, PyObject*) { return F(s, a, n); }>(self, args, nargs, nullptr);
}
template <auto F> PyCFunction with_names() { return (PyCFunction)(void (*)(void))(&guarded<F, OpsObject>); }
template <auto F, typename S> PyCFunction positional() { return (PyCFunction)(void (*)(void))(&guarded_positional<F, S>); }

PyMethodDef ops_methods[] = {
    {"set_handle", positional<set_handle, OpsObject>(), METH_FASTCALL, "set_handle(handle, device): the sp_ops that the methods work on; 0 for none"},
    {"sp_layer_norm", with_names<layer_norm>(), METH_FASTCALL | METH_KEYWORDS,
     "sp_layer_norm(x, y, gamma=None, beta=None, eps=1e-5, mean=None, rstd=None, stream=None)\n\n"
     "y = layer norm of x's rows; mean and rstd (float32 [n]) receive the statistics."},
    {"sp_layer_norm_backward", with_names<layer_norm_backward>(), METH_FASTCALL | METH_KEYWORDS,
     "sp_layer_norm_backward(dy, x, mean, rstd, gamma=None, dx=None, dgamma=None, dbeta=None, stream=None)\n\n"
     "Gradients of sp_layer_norm with the statistics that it handed out; dgamma and dbeta are float32 [d]."},
    {"sp_grouped_linear", with_names<grouped_linear>(), METH_FASTCALL | METH_KEYWORDS,
     "sp_grouped_linear(x, offsets, w, y, bias=None, relu=False, residual=None, act_out=None, stream=None)\n\n"
     "y = act(x W_g + b_g) + residual; x [n, k], offsets int32 [groups + 1], w [groups, k, m], bias float32 [groups, m]."},
    {"sp_grouped_linear_backward", with_names<grouped_linear_backward>(), METH_FASTCALL | METH_KEYWORDS,
     "sp_grouped_linear_backward(dy, x, offsets, w, act=None, dx=None, dw=None, db=None, stream=None)\n\n"
     "Gradients of sp_grouped_linear; act: its y (act_out, if it had a residual) where it had relu=True.  dw, db: float32."},
    {"sp_cross_entropy", with_names<cross_entropy>(), METH_FASTCALL | METH_KEYWORDS,
     "sp_cross_entropy(logits, label, loss, app=None, n_classes=None, weight=None, scale=1.0, dlogits=None, stream=None)\n\n"
     "loss [n] and dlogits of softmax cross entropy over the first n_classes[app[i]] columns (all of them without app)."},
    {"clip_packed", positional<clip_packed, OpsObject>(), METH_FASTCALL, "clip_packed(packed, max_norm, norm, stream): sp_clip_grad_norm of packed tensors"},
    {nullptr, nullptr, 0, nullptr}};

PyType_Slot ops_slots[] = {{Py_tp_methods, ops_methods}, {Py_tp_doc, (void*)"Calls on one sp_ops, checked."}, {0, nullptr}};
PyType_Spec ops_spec = {"paper_2505_06641_amd._ops_native.OpsBase", sizeof(OpsObject), 0, Py_TPFLAGS_DEFAULT | Py_TPFLAGS_BASETYPE, ops_slots};

PyObject* set_error(PyObject*, PyObject* cls) {
  Py_INCREF(cls);
  Py_XDECREF(g_error);
  g_error = cls;
  Py_RETURN_NONE;
}

PyMethodDef module_methods[] = {
    {"set_error", set_error, METH_O, "set_error(cls): refusals and failures raise cls(status, where, detail)"},
    {"pack_tensors", positional<pack_tensors, PyObject>(), METH_FASTCALL, "pack_tensors(grads, out or None): the tensors, as clip_packed takes them"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_ops_native", "Checked calls of the operators that train the heads.", -1, module_methods,
                          nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ops_native() {
  PyObject* m = PyModule_Create(&module_def);
  PyObject* type = m ? PyType_FromSpec(&ops_spec) : nullptr;
  if (!type || PyModule_AddObject(m, "OpsBase", type) != 0) {
    Py_XDECREF(type);
    Py_XDECREF(m);
    return nullptr;
  }
  return m;
}

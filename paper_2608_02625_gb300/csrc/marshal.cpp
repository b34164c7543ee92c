// Native marshalling of the Python binding: torch tensors to dlm_tensor
// descriptors, torch's current stream to dlm_set_stream, and the call.
//
// Every function takes the arguments of its Python entry point and returns the
// library's status, or None when it has done nothing because an argument is
// not of the ordinary form (a plain CUDA tensor of a supported type with
// storage, on the current device; a Python int; a RefineParams): the caller
// then takes the general path in Python, which marshals what can be marshalled
// and raises what has to be raised. What it is for: through ctypes, building
// the descriptors in Python took longer on a GB300's Grace host than the work on
// the GPU of a small call (calls issued one after another: the update of 8 x 2048
// 17.6 us, of which 8.7 on the GPU, now 10.3; one sequence's attention 13.9, now
// 12.3; a first call on new tensors about 20 us shorter).
#include <Python.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <vector>

#include "dlmrefine.h"

namespace {

constexpr int kMaxTensors = 12;

PyObject* g_params_type = nullptr;  // RefineParams
PyObject* g_adamw_type = nullptr;   // AdamwParams
PyObject *s_threshold, *s_k, *s_frac, *s_mask_id, *s_prompt, *s_seq;
PyObject *s_beta1, *s_beta2, *s_eps, *s_decay, *s_max_norm, *s_lr, *s_step, *s_norm;

// The tensors of one call. Every method returns false where the general path
// has to decide.
class Call {
 public:
  // Descriptor of `o` as argument slot n (null for None when `optional`).
  bool add(PyObject* o, bool optional = false) {
    if (optional && o == Py_None) {
      ptr_[n_++] = nullptr;
      return true;
    }
    at::Tensor* t = nullptr;
    if (!plain(o, &t)) return false;
    dlm_tensor& d = desc_[n_];
    if (!describe(*t, &d)) return false;
    ptr_[n_++] = &d;
    return true;
  }

  // Device memory the call works in: any type, contiguous.
  bool workspace(PyObject* o, void** data, size_t* bytes) {
    at::Tensor* t = nullptr;
    if (!plain(o, &t) || !t->is_contiguous()) return false;
    *bytes = static_cast<size_t>(t->numel()) * t->itemsize();
    *data = *bytes ? t->data_ptr() : nullptr;
    return true;
  }

  bool params(PyObject* o, dlm_refine_params* p) {
    if (reinterpret_cast<PyObject*>(Py_TYPE(o)) != g_params_type) return false;
    double threshold, frac;
    long k, mask_id;
    if (!number(o, s_threshold, &threshold) || !number(o, s_frac, &frac) || !integer(o, s_k, &k) ||
        !integer(o, s_mask_id, &mask_id))
      return false;
    p->edit_threshold = static_cast<float>(threshold);
    p->remask_frac = static_cast<float>(frac);
    p->remask_k = static_cast<int32_t>(k);
    p->mask_id = static_cast<int32_t>(mask_id);
    return lengths(o, s_prompt, &p->prompt_lens) && lengths(o, s_seq, &p->seq_lens);
  }

  bool adamw(PyObject* o, dlm_adamw_params* p) {
    if (reinterpret_cast<PyObject*>(Py_TYPE(o)) != g_adamw_type) return false;
    const void *lr, *step, *norm;
    if (!number(o, s_beta1, &p->beta1) || !number(o, s_beta2, &p->beta2) || !number(o, s_eps, &p->eps) ||
        !number(o, s_decay, &p->weight_decay) || !number(o, s_max_norm, &p->max_norm) || !scalar(o, s_lr, at::kFloat, false, &lr) ||
        !scalar(o, s_step, at::kInt, false, &step) || !scalar(o, s_norm, at::kFloat, true, &norm))
      return false;
    p->lr = static_cast<const float*>(lr);
    p->step = static_cast<const int32_t*>(step);
    p->norm = static_cast<const float*>(norm);
    return true;
  }

  // The current stream of the tensors' device, for the library.
  bool stream() {
    if (device_ < 0 || c10::cuda::current_device() != device_) return false;
    return dlm_set_stream(c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device_)).stream()) == DLM_OK;
  }

  dlm_tensor* operator[](int i) { return ptr_[i]; }

  // Descriptors of a list or tuple of tensors.
  bool list(PyObject* o, std::vector<dlm_tensor>* out) {
    if (!PyList_CheckExact(o) && !PyTuple_CheckExact(o)) return false;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(o);
    out->resize(static_cast<size_t>(n));
    for (Py_ssize_t i = 0; i < n; ++i) {
      at::Tensor* t = nullptr;
      if (!plain(PySequence_Fast_GET_ITEM(o, i), &t) || !describe(*t, &(*out)[static_cast<size_t>(i)])) return false;
    }
    return true;
  }

 private:
  static bool describe(const at::Tensor& t, dlm_tensor* d) {
    switch (t.scalar_type()) {
      case at::kBFloat16: d->dtype = DLM_BF16; break;
      case at::kFloat: d->dtype = DLM_F32; break;
      case at::kInt: d->dtype = DLM_I32; break;
      case at::kByte: d->dtype = DLM_U8; break;
      default: return false;
    }
    const int64_t nd = t.dim();
    if (nd < 1 || nd > 4) return false;
    d->data = t.numel() ? t.data_ptr() : nullptr;
    d->ndim = static_cast<int32_t>(nd);
    for (int i = 0; i < 4; ++i) {
      d->shape[i] = i < nd ? t.size(i) : 0;
      d->stride[i] = i < nd ? t.stride(i) : 0;
    }
    return true;
  }

  bool plain(PyObject* o, at::Tensor** out) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage()) return false;
    const int dev = t.get_device();
    if (device_ >= 0 && dev != device_) return false;
    device_ = dev;
    *out = const_cast<at::Tensor*>(&t);
    return true;
  }

  static bool number(PyObject* o, PyObject* name, double* v) {
    PyObject* x = PyObject_GetAttr(o, name);
    if (!x) return false;
    const bool ok = PyFloat_CheckExact(x) || PyLong_CheckExact(x);
    if (ok) *v = PyFloat_AsDouble(x);
    Py_DECREF(x);
    return ok && !PyErr_Occurred();
  }

  static bool integer(PyObject* o, PyObject* name, long* v) {
    PyObject* x = PyObject_GetAttr(o, name);
    if (!x) return false;
    const bool ok = PyLong_CheckExact(x);
    if (ok) *v = PyLong_AsLong(x);
    Py_DECREF(x);
    return ok && !PyErr_Occurred() && *v >= INT32_MIN && *v <= INT32_MAX;
  }

  bool lengths(PyObject* o, PyObject* name, const int32_t** v) {
    PyObject* x = PyObject_GetAttr(o, name);
    if (!x) return false;
    at::Tensor* t = nullptr;
    const bool ok = plain(x, &t) && t->scalar_type() == at::kInt && t->is_contiguous();
    if (ok) *v = static_cast<const int32_t*>(t->data_ptr());
    Py_DECREF(x);  // the RefineParams keeps it
    return ok;
  }

  // The address of a one-element tensor (null for None where `optional`).
  bool scalar(PyObject* o, PyObject* name, at::ScalarType type, bool optional, const void** v) {
    PyObject* x = PyObject_GetAttr(o, name);
    if (!x) return false;
    at::Tensor* t = nullptr;
    bool ok = optional && x == Py_None;
    *v = nullptr;
    if (!ok && plain(x, &t) && t->scalar_type() == type && t->numel() == 1) {
      *v = t->data_ptr();
      ok = true;
    }
    Py_DECREF(x);  // the AdamwParams keeps it
    return ok;
  }

  dlm_tensor desc_[kMaxTensors];
  dlm_tensor* ptr_[kMaxTensors];
  int n_ = 0, device_ = -1;
};

bool as_int32(PyObject* o, int32_t* v) {
  if (!PyLong_CheckExact(o)) return false;
  const long x = PyLong_AsLong(o);
  if (PyErr_Occurred() || x < INT32_MIN || x > INT32_MAX) return false;
  *v = static_cast<int32_t>(x);
  return true;
}

bool as_float(PyObject* o, float* v) {
  if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) return false;
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) return false;
  *v = static_cast<float>(x);
  return true;
}

PyObject* general_path() {
  PyErr_Clear();
  Py_RETURN_NONE;
}

// body(call, status): false for the general path. No C++ exception leaves.
template <typename Body>
PyObject* run(Py_ssize_t n, Py_ssize_t want, Body body) {
  if (n != want) return general_path();
  int status = 0;
  try {
    Call c;
    if (!body(c, &status)) return general_path();
  } catch (...) {
    return general_path();
  }
  return PyLong_FromLong(status);
}

// The library call without the interpreter lock (a launch may wait for queue space).
template <typename F>
int unlocked(F f) {
  int status;
  Py_BEGIN_ALLOW_THREADS status = f();
  Py_END_ALLOW_THREADS return status;
}

bool add_all(Call& c, PyObject* const* a, int first, int last) {
  for (int i = first; i < last; ++i)
    if (!c.add(a[i])) return false;
  return true;
}

PyObject* bidir_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 5, [&](Call& c, int* st) {
    if (!add_all(c, a, 0, 3) || !c.add(a[3], true) || !c.add(a[4]) || !c.stream()) return false;
    *st = unlocked([&] { return dlm_bidir_attn(c[0], c[1], c[2], c[3], c[4]); });
    return true;
  });
}

PyObject* attn_masked(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 8, [&](Call& c, int* st) {
    int32_t mode, block;
    if (!add_all(c, a, 0, 3) || !c.add(a[3], true) || !c.add(a[4], true) || !as_int32(a[5], &mode) ||
        !as_int32(a[6], &block) || !c.add(a[7]) || !c.stream())
      return false;
    *st = unlocked([&] { return dlm_attn_masked(c[0], c[1], c[2], c[3], c[4], mode, block, c[5]); });
    return true;
  });
}

PyObject* vocab_confidence(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 4, [&](Call& c, int* st) {
    if (!add_all(c, a, 0, 4) || !c.stream()) return false;
    *st = unlocked([&] { return dlm_vocab_confidence(c[0], c[1], c[2], c[3]); });
    return true;
  });
}

PyObject* token_prob(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 4, [&](Call& c, int* st) {
    if (!add_all(c, a, 0, 4) || !c.stream()) return false;
    *st = unlocked([&] { return dlm_token_prob(c[0], c[1], c[2], c[3]); });
    return true;
  });
}

// tokens, mask, argmax, conf, params, new_tokens, new_mask, n_edits
PyObject* refine_update(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 8, [&](Call& c, int* st) {
    dlm_refine_params p;
    if (!add_all(c, a, 0, 4) || !c.params(a[4], &p) || !add_all(c, a, 5, 8) || !c.stream()) return false;
    *st = unlocked([&] { return dlm_refine_update(c[0], c[1], c[2], c[3], &p, c[4], c[5], c[6]); });
    return true;
  });
}

// tokens, mask, argmax, conf, tok_prob, params, new_tokens, new_mask, n_edits
PyObject* refine_update_ranked(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 9, [&](Call& c, int* st) {
    dlm_refine_params p;
    if (!add_all(c, a, 0, 5) || !c.params(a[5], &p) || !add_all(c, a, 6, 9) || !c.stream()) return false;
    *st = unlocked([&] { return dlm_refine_update_ranked(c[0], c[1], c[2], c[3], c[4], &p, c[5], c[6], c[7]); });
    return true;
  });
}

// logits, tokens, mask, params, argmax, conf, lse, new_tokens, new_mask, n_edits, workspace
PyObject* refine_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 11, [&](Call& c, int* st) {
    dlm_refine_params p;
    void* ws;
    size_t bytes;
    if (!add_all(c, a, 0, 3) || !c.params(a[3], &p) || !add_all(c, a, 4, 10) || !c.workspace(a[10], &ws, &bytes) ||
        !c.stream())
      return false;
    *st = unlocked([&] {
      return dlm_refine_step(c[0], c[1], c[2], &p, c[3], c[4], c[5], c[6], c[7], c[8], ws, bytes);
    });
    return true;
  });
}

// logits, tokens, mask, params, argmax, conf, lse, new_tokens, new_mask, n_edits
PyObject* refine_step_static(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 10, [&](Call& c, int* st) {
    dlm_refine_params p;
    if (!add_all(c, a, 0, 3) || !c.params(a[3], &p) || !add_all(c, a, 4, 10) || !c.stream()) return false;
    *st = unlocked([&] { return dlm_refine_step_static(c[0], c[1], c[2], &p, c[3], c[4], c[5], c[6], c[7], c[8]); });
    return true;
  });
}

// hidden, weight, argmax, conf, lse, workspace
PyObject* lmhead_confidence(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 6, [&](Call& c, int* st) {
    void* ws;
    size_t bytes;
    if (!add_all(c, a, 0, 5) || !c.workspace(a[5], &ws, &bytes) || !c.stream()) return false;
    *st = unlocked([&] { return dlm_lmhead_confidence(c[0], c[1], c[2], c[3], c[4], ws, bytes); });
    return true;
  });
}

// hidden, weight, targets, loss, lse, workspace
PyObject* lmhead_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 6, [&](Call& c, int* st) {
    void* ws;
    size_t bytes;
    if (!add_all(c, a, 0, 5) || !c.workspace(a[5], &ws, &bytes) || !c.stream()) return false;
    *st = unlocked([&] { return dlm_lmhead_loss(c[0], c[1], c[2], c[3], c[4], ws, bytes); });
    return true;
  });
}

// hidden, weight, targets, lse, dloss, d_hidden, d_weight, workspace
PyObject* lmhead_loss_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 8, [&](Call& c, int* st) {
    void* ws;
    size_t bytes;
    if (!add_all(c, a, 0, 5) || !c.add(a[5], true) || !c.add(a[6], true) || !c.workspace(a[7], &ws, &bytes) || !c.stream())
      return false;
    *st = unlocked([&] { return dlm_lmhead_loss_grad(c[0], c[1], c[2], c[3], c[4], c[5], c[6], ws, bytes); });
    return true;
  });
}

// x, weight, bias, eps, out, mean, rstd
PyObject* layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 7, [&](Call& c, int* st) {
    float eps;
    if (!add_all(c, a, 0, 2) || !c.add(a[2], true) || !as_float(a[3], &eps) || !c.add(a[4]) || !c.add(a[5], true) ||
        !c.add(a[6], true) || !c.stream())
      return false;
    *st = unlocked([&] { return dlm_layer_norm(c[0], c[1], c[2], eps, c[3], c[4], c[5]); });
    return true;
  });
}

// dout, x, weight, mean, rstd, dx, dweight, dbias, workspace (None where nothing needs it)
PyObject* layer_norm_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 9, [&](Call& c, int* st) {
    void* ws = nullptr;
    size_t bytes = 0;
    if (!add_all(c, a, 0, 6) || !c.add(a[6], true) || !c.add(a[7], true) ||
        (a[8] != Py_None && !c.workspace(a[8], &ws, &bytes)) || !c.stream())
      return false;
    *st = unlocked([&] { return dlm_layer_norm_grad(c[0], c[1], c[2], c[3], c[4], c[5], c[6], c[7], ws, bytes); });
    return true;
  });
}

// grads, outs (None: the norm alone), max_norm, norm, workspace
PyObject* clip_grad_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 5, [&](Call& c, int* st) {
    std::vector<dlm_tensor> grads, outs;
    float max_norm;
    void* ws;
    size_t bytes;
    const bool scale = a[1] != Py_None;
    if (!c.list(a[0], &grads) || (scale && (!c.list(a[1], &outs) || outs.size() != grads.size())) ||
        grads.size() > INT32_MAX || !as_float(a[2], &max_norm) || !c.add(a[3]) || !c.workspace(a[4], &ws, &bytes) || !c.stream())
      return false;
    // An empty list has no descriptors, but still outputs.
    dlm_tensor none;
    *st = unlocked([&] {
      return dlm_clip_grad_norm(grads.empty() ? &none : grads.data(), !scale ? nullptr : outs.empty() ? &none : outs.data(),
                                static_cast<int32_t>(grads.size()), max_norm, c[0], ws, bytes);
    });
    return true;
  });
}

// x, w_gate, w_up, act, out, gate, up
PyObject* gated_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 7, [&](Call& c, int* st) {
    int32_t act;
    if (!add_all(c, a, 0, 3) || !as_int32(a[3], &act) || !c.add(a[4]) || !c.add(a[5], true) || !c.add(a[6], true) || !c.stream())
      return false;
    *st = unlocked([&] { return dlm_gated_linear(c[0], c[1], c[2], act, c[3], c[4], c[5]); });
    return true;
  });
}

// dout, x, w_gate, w_up, gate, up, act, add, dx, dw_gate, dw_up, workspace
PyObject* gated_linear_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 12, [&](Call& c, int* st) {
    int32_t act;
    void* ws;
    size_t bytes;
    if (!add_all(c, a, 0, 6) || !as_int32(a[6], &act)) return false;
    for (int i = 7; i < 11; ++i)
      if (!c.add(a[i], true)) return false;
    if (!c.workspace(a[11], &ws, &bytes) || !c.stream()) return false;
    *st = unlocked([&] { return dlm_gated_linear_grad(c[0], c[1], c[2], c[3], c[4], c[5], act, c[6], c[7], c[8], c[9], ws, bytes); });
    return true;
  });
}

// x, weight, bias, act, residual, out, pre, workspace (None where nothing needs it)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 8, [&](Call& c, int* st) {
    int32_t act;
    void* ws = nullptr;
    size_t bytes = 0;
    if (!add_all(c, a, 0, 2) || !c.add(a[2], true) || !as_int32(a[3], &act) || !c.add(a[4], true) || !c.add(a[5]) ||
        !c.add(a[6], true) || (a[7] != Py_None && !c.workspace(a[7], &ws, &bytes)) || !c.stream())
      return false;
    *st = unlocked([&] { return dlm_linear(c[0], c[1], c[2], act, c[3], c[4], c[5], ws, bytes); });
    return true;
  });
}

// dout, x, weight, pre, act, add, dx, dweight, dbias, workspace
PyObject* linear_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 10, [&](Call& c, int* st) {
    int32_t act;
    void* ws;
    size_t bytes;
    if (!add_all(c, a, 0, 3) || !c.add(a[3], true) || !as_int32(a[4], &act)) return false;
    for (int i = 5; i < 9; ++i)
      if (!c.add(a[i], true)) return false;
    if (!c.workspace(a[9], &ws, &bytes) || !c.stream()) return false;
    *st = unlocked([&] { return dlm_linear_grad(c[0], c[1], c[2], c[3], act, c[4], c[5], c[6], c[7], ws, bytes); });
    return true;
  });
}

// params, masters (or None), grads, m, v, m_scales, v_scales (None: states in 32 bits), hyper
PyObject* adamw(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 8, [&](Call& c, int* st) {
    std::vector<dlm_tensor> t[7];
    dlm_tensor none;
    dlm_tensor* p[7];
    dlm_adamw_params hyper;
    for (int i = 0; i < 7; ++i) {
      const bool optional = i == 1 || i >= 5;
      p[i] = nullptr;
      if (optional && a[i] == Py_None) continue;
      if (!c.list(a[i], &t[i]) || t[i].size() != t[0].size() || t[i].size() > INT32_MAX) return false;
      p[i] = t[i].empty() ? &none : t[i].data();
    }
    if (!c.adamw(a[7], &hyper) || !c.stream()) return false;
    *st = unlocked([&] { return dlm_adamw(p[0], p[1], p[2], p[3], p[4], p[5], p[6], static_cast<int32_t>(t[0].size()), &hyper); });
    return true;
  });
}

// handle (a non-zero int), device index
PyObject* loop_launch(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(n, 2, [&](Call&, int* st) {
    int32_t dev;
    if (!PyLong_CheckExact(a[0]) || !as_int32(a[1], &dev)) return false;
    void* handle = PyLong_AsVoidPtr(a[0]);
    if (!handle || c10::cuda::current_device() != dev ||
        dlm_set_stream(c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(dev)).stream()) != DLM_OK)
      return false;
    *st = unlocked([&] { return dlm_loop_launch(static_cast<dlm_loop*>(handle)); });
    return true;
  });
}

PyObject* set_params_type(PyObject*, PyObject* type) {
  Py_XDECREF(g_params_type);
  g_params_type = Py_NewRef(type);
  Py_RETURN_NONE;
}

PyObject* set_adamw_type(PyObject*, PyObject* type) {
  Py_XDECREF(g_adamw_type);
  g_adamw_type = Py_NewRef(type);
  Py_RETURN_NONE;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(bidir_attn),
                         FAST(attn_masked),
                         FAST(vocab_confidence),
                         FAST(token_prob),
                         FAST(refine_update),
                         FAST(refine_update_ranked),
                         FAST(refine_step),
                         FAST(refine_step_static),
                         FAST(lmhead_confidence),
                         FAST(lmhead_loss),
                         FAST(lmhead_loss_grad),
                         FAST(layer_norm),
                         FAST(layer_norm_grad),
                         FAST(clip_grad_norm),
                         FAST(gated_linear),
                         FAST(gated_linear_grad),
                         FAST(linear),
                         FAST(linear_grad),
                         FAST(adamw),
                         FAST(loop_launch),
                         {"set_params_type", set_params_type, METH_O, nullptr},
                         {"set_adamw_type", set_adamw_type, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) {
  s_threshold = PyUnicode_InternFromString("edit_threshold");
  s_k = PyUnicode_InternFromString("remask_k");
  s_frac = PyUnicode_InternFromString("remask_frac");
  s_mask_id = PyUnicode_InternFromString("mask_id");
  s_prompt = PyUnicode_InternFromString("prompt_lens");
  s_seq = PyUnicode_InternFromString("seq_lens");
  s_beta1 = PyUnicode_InternFromString("beta1");
  s_beta2 = PyUnicode_InternFromString("beta2");
  s_eps = PyUnicode_InternFromString("eps");
  s_decay = PyUnicode_InternFromString("weight_decay");
  s_max_norm = PyUnicode_InternFromString("max_norm");
  s_lr = PyUnicode_InternFromString("lr");
  s_step = PyUnicode_InternFromString("step");
  s_norm = PyUnicode_InternFromString("norm");
  return PyModule_Create(&module);
}

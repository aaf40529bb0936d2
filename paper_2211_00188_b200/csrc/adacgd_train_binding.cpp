// Python binding of the training operators: checks torch tensors, fills the argument records of adacgd_train.h and calls the
// entry points.  A call through ctypes spends 0.5 us on every tensor it checks, which is most of what a small call takes; here
// the whole of it is about one.
//
// Every function takes the handle first and returns the entry point's status, or RETRY when another stream or device is
// current (the Python side orders the streams and calls again with the handle's `force` set).  Wrong arguments raise ValueError.
//
// The calls are not recorded by autograd.  So an output that requires a gradient is refused while gradients are recorded, and the
// version of what a call has written moves on, as after any other modification in place.
#include <Python.h>

#include <string>

#include <ATen/core/Tensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "adacgd_train.h"

namespace {

constexpr long RETRY = -1;

struct Handle {
  adacgd_train* ctx;
  int index;
  void* stream;
  bool force;
};

struct Refused {
  std::string what;
};
[[noreturn]] void refuse(const char* name, const std::string& what) { throw Refused{std::string(name) + " " + what}; }

int type_code(at::ScalarType t) {
  switch (t) {
    case at::kFloat: return ADACGD_F32;
    case at::kHalf: return ADACGD_F16;
    case at::kBFloat16: return ADACGD_BF16;
    default: return -1;
  }
}

enum Use { IN, OUT };

const at::Tensor* tensor(PyObject* o, const char* name, bool optional) {
  if (o == Py_None && optional) return nullptr;
  if (!THPVariable_Check(o)) refuse(name, "must be a tensor");
  return &THPVariable_Unpack(o);
}

// What the matrices of a call share: set by the first.  And the call's outputs.
struct Shape {
  const Handle* h;
  const at::Tensor* written[8];
  int outputs = 0;
  int64_t rows = 0, cols = 0;
  at::ScalarType type = at::kFloat;
  int code = 0;

  explicit Shape(const Handle* handle) : h(handle) {}
  void output(const at::Tensor& t, const char* name) {
    if (t.requires_grad() && c10::GradMode::is_enabled()) refuse(name, "requires a gradient, and the call is not recorded: use torch.no_grad() or a detached tensor");
    written[outputs++] = &t;
  }
  void count_versions() const {
    for (int i = 0; i < outputs; ++i)
      if (!written[i]->is_inference()) written[i]->unsafeGetTensorImpl()->bump_version();
  }
  void lead(PyObject* o, const char* name, const void** p, int64_t* stride) {
    const at::Tensor& t = *tensor(o, name, false);
    type = t.scalar_type();
    code = type_code(type);
    if (code < 0 || t.dim() != 2) refuse(name, "must be a 2-D float32, float16 or bfloat16 tensor");
    rows = t.size(0);
    cols = t.size(1);
    place(t, name, p, stride);
  }
  void matrix(PyObject* o, const char* name, Use use, bool optional, const void** p, int64_t* stride) {
    *p = nullptr;
    *stride = 0;
    const at::Tensor* t = tensor(o, name, optional);
    if (!t) return;
    if (t->scalar_type() != type) refuse(name, "must have the type of the other matrices");
    if (t->dim() != 2 || t->size(0) != rows || t->size(1) != cols)
      refuse(name, "must have the shape (" + std::to_string(rows) + ", " + std::to_string(cols) + ")");
    place(*t, name, p, stride);
    if (use == OUT) output(*t, name);
  }
  void place(const at::Tensor& t, const char* name, const void** p, int64_t* stride) const {
    if (!t.is_cuda() || t.get_device() != h->index) refuse(name, "must be on cuda:" + std::to_string(h->index));
    if (cols > 1 && t.stride(1) != 1) refuse(name, "must have unit column stride");
    int64_t s = t.stride(0);
    if (s < cols) {
      if (rows > 1) refuse(name, "has rows that overlap");
      s = cols;
    }
    *p = t.data_ptr();
    *stride = s;
  }
  void* vector(PyObject* o, const char* name, Use use, bool optional, int64_t n, at::ScalarType want) {
    const at::Tensor* t = tensor(o, name, optional);
    if (!t) return nullptr;
    if (t->scalar_type() != want) refuse(name, std::string("must have the type ") + c10::toString(want));
    void* const p = contiguous(*t, name, n);
    if (use == OUT) output(*t, name);
    return p;
  }
  void* contiguous(const at::Tensor& t, const char* name, int64_t n) const {
    if (!t.is_cuda() || t.get_device() != h->index) refuse(name, "must be on cuda:" + std::to_string(h->index));
    if (t.numel() != n || !t.is_contiguous()) refuse(name, "must be contiguous with " + std::to_string(n) + " elements");
    return t.data_ptr();
  }
  // weight-like vectors: all of the matrices' type or all float32
  struct Param {
    PyObject* o;
    const char* name;
    Use use;
  };
  int params(std::initializer_list<Param> list, void** out) {
    at::ScalarType want = type;
    bool first = true;
    for (const Param& e : list) {
      const at::Tensor* t = tensor(e.o, e.name, true);
      *out = nullptr;
      if (t) {
        if (first) {
          want = t->scalar_type();
          if (want != type && want != at::kFloat) refuse(e.name, "must be float32 or of the matrices' type");
          first = false;
        } else if (t->scalar_type() != want) {
          refuse(e.name, "must have the type of the other weight-like arguments");
        }
        *out = contiguous(*t, e.name, cols);
        if (e.use == OUT) output(*t, e.name);
      }
      ++out;
    }
    return type_code(want);
  }
  void token_rows(adacgd_token_rows* r, PyObject* logits, PyObject* labels, PyObject* mask, PyObject* seq_start, PyObject* sequences) {
    lead(logits, "logits", &r->logits, &r->logits_stride);
    r->tokens = rows;
    r->vocab = cols;
    r->dtype = code;
    const at::Tensor& y = *tensor(labels, "labels", false);
    if (y.scalar_type() != at::kLong && y.scalar_type() != at::kInt) refuse("labels", "must be int64 or int32");
    r->label_bytes = y.scalar_type() == at::kLong ? 8 : 4;
    r->labels = contiguous(y, "labels", rows);
    r->mask = nullptr;
    if (const at::Tensor* m = tensor(mask, "mask", true)) {
      if (m->scalar_type() != at::kBool && m->scalar_type() != at::kByte) refuse("mask", "must be bool or uint8");
      r->mask = (const uint8_t*)contiguous(*m, "mask", rows);
    }
    int64_t given = -1;
    if (sequences != Py_None) {
      given = PyLong_AsLongLong(sequences);
      if (given == -1 && PyErr_Occurred()) throw Refused{""};
    }
    r->seq_start = nullptr;
    r->sequences = given < 0 && sequences == Py_None ? 1 : given;
    if (const at::Tensor* s = tensor(seq_start, "seq_start", true)) {
      if (s->scalar_type() != at::kInt) refuse("seq_start", "must be int32");
      if (sequences != Py_None && given != s->numel() - 1) refuse("sequences", "and seq_start disagree");
      r->sequences = s->numel() - 1;
      r->seq_start = (const int32_t*)contiguous(*s, "seq_start", s->numel());
    }
  }
};

double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused{""};
  return v;
}
uint64_t bits(PyObject* o) {   // any integer, modulo 2^64
  const uint64_t v = PyLong_AsUnsignedLongLongMask(o);
  if (v == (uint64_t)-1 && PyErr_Occurred()) throw Refused{""};
  return v;
}
adacgd_drop drop(PyObject* const* a) { return adacgd_drop{number(a[0]), bits(a[1]), bits(a[2])}; }
int truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Refused{""};
  return v;
}

// The frame of every call: the handle, the current stream and device, errors as exceptions.
template <typename F>
PyObject* call(PyObject* const* args, Py_ssize_t n, Py_ssize_t want, F body) {
  if (n != want) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  if (!PyCapsule_IsValid(args[0], "adacgd_train")) {
    PyErr_SetString(PyExc_RuntimeError, "the context is closed");
    return nullptr;
  }
  const Handle* h = (const Handle*)PyCapsule_GetPointer(args[0], "adacgd_train");
  try {
    Shape s{h};
    long status = RETRY;
    auto ready = [&] {
      return h->force || (c10::cuda::current_device() == h->index &&
                          (void*)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)h->index).stream() == h->stream);
    };
    status = body(s, ready);
    if (status == ADACGD_OK) s.count_versions();
    return PyLong_FromLong(status);
  } catch (const Refused& r) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, r.what.c_str());
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

#define MAT(name, i, use, optional)                                         \
  s.matrix(a[i], #name, use, optional, (const void**)&r.name, &r.name##_stride)

// (handle, x, out, residual, p, seed, offset)
PyObject* dropout(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(a, n, 7, [&](Shape& s, auto ready) -> long {
    adacgd_dropout_args r;
    s.lead(a[1], "x", &r.x, &r.x_stride);
    MAT(out, 2, OUT, false);
    MAT(residual, 3, IN, true);
    r.rows = s.rows;
    r.cols = s.cols;
    r.dtype = s.code;
    r.reserved = 0;
    r.drop = drop(a + 4);
    return ready() ? (long)adacgd_dropout(s.h->ctx, &r) : RETRY;
  });
}

// (handle, x, out, weight, bias, eps, residual, sum, mean, rstd, p, seed, offset)
PyObject* layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(a, n, 13, [&](Shape& s, auto ready) -> long {
    adacgd_norm_args r;
    s.lead(a[1], "x", &r.x, &r.x_stride);
    MAT(out, 2, OUT, false);
    MAT(residual, 6, IN, true);
    MAT(sum, 7, OUT, true);
    void* p[2];
    r.param_dtype = s.params({{a[3], "weight", IN}, {a[4], "bias", IN}}, p);
    r.weight = p[0];
    r.bias = p[1];
    r.mean = (float*)s.vector(a[8], "mean", OUT, true, s.rows, at::kFloat);
    r.rstd = (float*)s.vector(a[9], "rstd", OUT, true, s.rows, at::kFloat);
    r.rows = s.rows;
    r.cols = s.cols;
    r.dtype = s.code;
    r.eps = (float)number(a[5]);
    r.reserved = 0;
    r.drop = drop(a + 10);
    return ready() ? (long)adacgd_layer_norm(s.h->ctx, &r) : RETRY;
  });
}

// (handle, dout, s, mean, rstd, dx, weight, dweight, dbias, dsum, dresidual, p, seed, offset)
PyObject* layer_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(a, n, 14, [&](Shape& s, auto ready) -> long {
    adacgd_norm_backward_args r;
    s.lead(a[1], "dout", &r.dout, &r.dout_stride);
    MAT(s, 2, IN, false);
    MAT(dx, 5, OUT, false);
    MAT(dsum, 9, IN, true);
    MAT(dresidual, 10, OUT, true);
    r.mean = (const float*)s.vector(a[3], "mean", IN, false, s.rows, at::kFloat);
    r.rstd = (const float*)s.vector(a[4], "rstd", IN, false, s.rows, at::kFloat);
    void* p[3];
    r.param_dtype = s.params({{a[6], "weight", IN}, {a[7], "dweight", OUT}, {a[8], "dbias", OUT}}, p);
    r.weight = p[0];
    r.dweight = p[1];
    r.dbias = p[2];
    r.rows = s.rows;
    r.cols = s.cols;
    r.dtype = s.code;
    r.drop = drop(a + 11);
    return ready() ? (long)adacgd_layer_norm_backward(s.h->ctx, &r) : RETRY;
  });
}

// (handle, logits, labels, logp, mask, lse)
PyObject* token_logp(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(a, n, 6, [&](Shape& s, auto ready) -> long {
    adacgd_token_rows r;
    s.token_rows(&r, a[1], a[2], a[4], Py_None, Py_None);
    float* logp = (float*)s.vector(a[3], "logp", OUT, false, s.rows, at::kFloat);
    float* lse = (float*)s.vector(a[5], "lse", OUT, true, s.rows, at::kFloat);
    return ready() ? (long)adacgd_token_logp(s.h->ctx, &r, logp, lse) : RETRY;
  });
}

// (handle, logits, labels, ref_logp, loss, dlogits, mask, sequences, seq_start, beta, kind, label_smoothing, length_normalized,
//  grad_scale, margin, seq_logp)
PyObject* preference_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(a, n, 16, [&](Shape& s, auto ready) -> long {
    adacgd_preference_args r;
    s.token_rows(&r.rows, a[1], a[2], a[6], a[8], a[7]);
    r.ref_logp = (const float*)s.vector(a[3], "ref_logp", IN, false, s.rows, at::kFloat);
    r.loss = (float*)s.vector(a[4], "loss", OUT, false, 1, at::kFloat);
    MAT(dlogits, 5, OUT, true);
    r.beta = (float)number(a[9]);
    r.kind = (int32_t)bits(a[10]);
    r.label_smoothing = (float)number(a[11]);
    r.length_normalized = truth(a[12]);
    r.grad_scale = (float)number(a[13]);
    r.margin = (float*)s.vector(a[14], "margin", OUT, true, r.rows.sequences / 2, at::kFloat);
    r.seq_logp = (float*)s.vector(a[15], "seq_logp", OUT, true, r.rows.sequences, at::kFloat);
    r.reserved = 0;
    return ready() ? (long)adacgd_preference_loss(s.h->ctx, &r) : RETRY;
  });
}

// (handle, logits, labels, old_logp, advantages, loss, dlogits, mask, sequences, seq_start, ref_logp, clip_low, clip_high, kl_beta,
//  per_sequence, grad_scale, logp, stats)
PyObject* policy_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(a, n, 18, [&](Shape& s, auto ready) -> long {
    adacgd_policy_args r;
    s.token_rows(&r.rows, a[1], a[2], a[7], a[9], a[8]);
    r.old_logp = (const float*)s.vector(a[3], "old_logp", IN, false, s.rows, at::kFloat);
    r.advantages = (const float*)s.vector(a[4], "advantages", IN, false, s.rows, at::kFloat);
    r.loss = (float*)s.vector(a[5], "loss", OUT, false, 1, at::kFloat);
    MAT(dlogits, 6, OUT, true);
    r.ref_logp = (const float*)s.vector(a[10], "ref_logp", IN, true, s.rows, at::kFloat);
    r.clip_low = (float)number(a[11]);
    r.clip_high = (float)number(a[12]);
    r.kl_beta = (float)number(a[13]);
    r.per_sequence = truth(a[14]);
    r.grad_scale = (float)number(a[15]);
    r.logp = (float*)s.vector(a[16], "logp", OUT, true, s.rows, at::kFloat);
    r.stats = (float*)s.vector(a[17], "stats", OUT, true, 3, at::kFloat);
    r.reserved = 0;
    return ready() ? (long)adacgd_policy_loss(s.h->ctx, &r) : RETRY;
  });
}

void release(PyObject* c) { delete (Handle*)PyCapsule_GetPointer(c, "adacgd_train"); }

// bind(context, device index, stream) -> handle
PyObject* bind(PyObject*, PyObject* args) {
  unsigned long long ctx, stream;
  int index;
  if (!PyArg_ParseTuple(args, "KiK", &ctx, &index, &stream)) return nullptr;
  Handle* h = new (std::nothrow) Handle{(adacgd_train*)ctx, index, (void*)stream, false};
  if (!h) return PyErr_NoMemory();
  return PyCapsule_New(h, "adacgd_train", release);
}

// force(handle, truth value)
PyObject* force(PyObject*, PyObject* args) {
  PyObject* c;
  int on;
  if (!PyArg_ParseTuple(args, "Op", &c, &on)) return nullptr;
  Handle* h = (Handle*)PyCapsule_GetPointer(c, "adacgd_train");
  if (!h) return nullptr;
  h->force = on != 0;
  Py_RETURN_NONE;
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(dropout),         FAST(layer_norm),      FAST(layer_norm_backward), FAST(token_logp),
                         FAST(preference_loss), FAST(policy_loss),     {"bind", bind, METH_VARARGS, nullptr},
                         {"force", force, METH_VARARGS, nullptr},      {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_train_binding", "Binding of the training operators.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__train_binding() { return PyModule_Create(&module); }

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

#include <cmath>
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
    matrix_of(o, name, use, optional, rows, cols, type, p, stride);
  }
  // A matrix of its own shape and type.
  void matrix_of(PyObject* o, const char* name, Use use, bool optional, int64_t n, int64_t width, at::ScalarType want, const void** p,
                 int64_t* stride) {
    *p = nullptr;
    *stride = 0;
    const at::Tensor* t = tensor(o, name, optional);
    if (!t) return;
    if (t->scalar_type() != want) refuse(name, want == type ? "must have the type of the other matrices" : std::string("must have the type ") + c10::toString(want));
    if (t->dim() != 2 || t->size(0) != n || t->size(1) != width)
      refuse(name, "must have the shape (" + std::to_string(n) + ", " + std::to_string(width) + ")");
    place(*t, name, p, stride);
    if (use == OUT) output(*t, name);
  }
  void place(const at::Tensor& t, const char* name, const void** p, int64_t* stride) const {
    if (!t.is_cuda() || t.get_device() != h->index) refuse(name, "must be on cuda:" + std::to_string(h->index));
    if (t.size(1) > 1 && t.stride(1) != 1) refuse(name, "must have unit column stride");
    int64_t s = t.stride(0);
    if (s < t.size(1)) {
      if (t.size(0) > 1) refuse(name, "has rows that overlap");
      s = t.size(1);
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
  int params(std::initializer_list<Param> list, void** out) { return params(list, out, cols); }
  int params(std::initializer_list<Param> list, void** out, int64_t n) {
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
        *out = contiguous(*t, e.name, n);
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
    r->labels = whole_numbers(labels, "labels", rows, &r->label_bytes);
    r->mask = counted(mask, rows);
    runs(seq_start, sequences, &r->seq_start, &r->sequences);
  }
  // int64 or int32
  const void* whole_numbers(PyObject* o, const char* name, int64_t n, int32_t* bytes) {
    const at::Tensor& y = *tensor(o, name, false);
    if (y.scalar_type() != at::kLong && y.scalar_type() != at::kInt) refuse(name, "must be int64 or int32");
    *bytes = y.scalar_type() == at::kLong ? 8 : 4;
    return contiguous(y, name, n);
  }
  const uint8_t* counted(PyObject* mask, int64_t n) {
    const at::Tensor* m = tensor(mask, "mask", true);
    if (!m) return nullptr;
    if (m->scalar_type() != at::kBool && m->scalar_type() != at::kByte) refuse("mask", "must be bool or uint8");
    return (const uint8_t*)contiguous(*m, "mask", n);
  }
  void runs(PyObject* seq_start, PyObject* sequences, const int32_t** start, int64_t* count) {
    int64_t given = -1;
    if (sequences != Py_None) {
      given = PyLong_AsLongLong(sequences);
      if (given == -1 && PyErr_Occurred()) throw Refused{""};
    }
    *start = nullptr;
    *count = given < 0 && sequences == Py_None ? 1 : given;
    if (const at::Tensor* s = tensor(seq_start, "seq_start", true)) {
      if (s->scalar_type() != at::kInt) refuse("seq_start", "must be int32");
      if (sequences != Py_None && given != s->numel() - 1) refuse("sequences", "and seq_start disagree");
      *count = s->numel() - 1;
      *start = (const int32_t*)contiguous(*s, "seq_start", s->numel());
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

// (handle, tokens, table, out, scale, mask)
PyObject* embedding(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(a, n, 6, [&](Shape& s, auto ready) -> long {
    adacgd_embedding_args r;
    s.lead(a[2], "table", &r.table, &r.table_stride);
    r.vocab = s.rows;
    r.cols = s.cols;
    r.dtype = s.code;
    const at::Tensor& ids = *tensor(a[1], "tokens", false);
    r.tokens = ids.numel();
    r.ids = s.whole_numbers(a[1], "tokens", r.tokens, &r.id_bytes);
    r.mask = s.counted(a[5], r.tokens);
    s.matrix_of(a[3], "out", OUT, false, r.tokens, s.cols, s.type, (const void**)&r.out, &r.out_stride);
    r.scale = (float)number(a[4]);
    r.reserved = 0;
    return ready() ? (long)adacgd_embedding(s.h->ctx, &r) : RETRY;
  });
}

// (handle, tokens, dout, dtable, scale, mask, base)
PyObject* embedding_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(a, n, 7, [&](Shape& s, auto ready) -> long {
    adacgd_embedding_backward_args r;
    s.lead(a[2], "dout", &r.dout, &r.dout_stride);
    r.tokens = s.rows;
    r.cols = s.cols;
    r.dtype = s.code;
    r.ids = s.whole_numbers(a[1], "tokens", s.rows, &r.id_bytes);
    r.mask = s.counted(a[5], s.rows);
    const at::Tensor& d = *tensor(a[3], "dtable", false);
    if (d.dim() != 2) refuse("dtable", "must be a 2-D tensor");
    if (d.scalar_type() != s.type && d.scalar_type() != at::kFloat) refuse("dtable", "must be float32 or of dout's type");
    r.vocab = d.size(0);
    r.table_dtype = type_code(d.scalar_type());
    s.matrix_of(a[3], "dtable", OUT, false, r.vocab, s.cols, d.scalar_type(), (const void**)&r.dtable, &r.dtable_stride);
    s.matrix_of(a[6], "base", IN, true, r.vocab, s.cols, d.scalar_type(), &r.base, &r.base_stride);
    r.scale = (float)number(a[4]);
    return ready() ? (long)adacgd_embedding_backward(s.h->ctx, &r) : RETRY;
  });
}

int64_t whole(PyObject* o) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused{""};
  return v;
}

// What qk_norm and its backward pass share: q and k (the inputs), positions, freq, head_dim, eps, interleaved; the weights are the caller's.
void heads_of(Shape& s, adacgd_qk_norm_args* r, PyObject* q, PyObject* k, PyObject* positions, PyObject* freq, PyObject* head_dim, PyObject* eps,
              PyObject* interleaved) {
  s.lead(q, "q", &r->q, &r->q_stride);
  const int64_t dim = whole(head_dim);
  if (dim < 1 || dim > ADACGD_TRAIN_MAX_HEAD) refuse("head_dim", "must be in [1, " + std::to_string(ADACGD_TRAIN_MAX_HEAD) + "]");
  if (s.cols < 1 || s.cols % dim) refuse("q", "must have a multiple of head_dim columns");
  r->head_dim = (int32_t)dim;
  r->tokens = s.rows;
  r->heads = s.cols / dim;
  r->key_heads = 0;
  r->dtype = s.code;
  r->k = nullptr;
  r->k_stride = 0;
  if (const at::Tensor* t = tensor(k, "k", true)) {
    if (t->dim() != 2 || t->size(1) < 1 || t->size(1) % dim) refuse("k", "must be a 2-D tensor with a multiple of head_dim columns");
    r->key_heads = t->size(1) / dim;
    s.matrix_of(k, "k", IN, false, s.rows, t->size(1), s.type, &r->k, &r->k_stride);
  }
  r->pairs = 0;
  r->freq = nullptr;
  r->positions = nullptr;
  r->position_bytes = 8;
  if (const at::Tensor* f = tensor(freq, "freq", true)) {
    if (f->scalar_type() != at::kFloat) refuse("freq", "must have the type Float");
    if (f->numel() > dim / 2) refuse("freq", "must have at most head_dim / 2 elements");
    r->pairs = (int32_t)f->numel();
    r->freq = (const float*)s.contiguous(*f, "freq", f->numel());
    if (positions == Py_None) refuse("positions", "must be given with freq");
    r->positions = s.whole_numbers(positions, "positions", s.rows, &r->position_bytes);
  }
  r->eps = (float)number(eps);
  r->interleaved = truth(interleaved);
  r->reserved = 0;
}

// (handle, q, k, q_out, k_out, positions, freq, head_dim, q_weight, k_weight, eps, interleaved)
PyObject* qk_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(a, n, 12, [&](Shape& s, auto ready) -> long {
    adacgd_qk_norm_args r;
    heads_of(s, &r, a[1], a[2], a[5], a[6], a[7], a[10], a[11]);
    const bool keys = r.key_heads > 0;
    if (!keys && (a[4] != Py_None || a[9] != Py_None)) refuse("k_out", "and k_weight go with k");
    MAT(q_out, 3, OUT, false);
    s.matrix_of(a[4], "k_out", OUT, !keys, s.rows, r.key_heads * r.head_dim, s.type, (const void**)&r.k_out, &r.k_out_stride);
    void* p[2];
    r.param_dtype = s.params({{a[8], "q_weight", IN}, {a[9], "k_weight", IN}}, p, r.head_dim);
    r.q_weight = p[0];
    r.k_weight = p[1];
    return ready() ? (long)adacgd_qk_norm(s.h->ctx, &r) : RETRY;
  });
}

// (handle, dq_out, dk_out, q, k, dq, dk, positions, freq, head_dim, q_weight, k_weight, dq_weight, dk_weight, eps, interleaved)
PyObject* qk_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(a, n, 16, [&](Shape& s, auto ready) -> long {
    adacgd_qk_norm_backward_args r;
    heads_of(s, &r.f, a[3], a[4], a[7], a[8], a[9], a[14], a[15]);
    const bool keys = r.f.key_heads > 0;
    const int64_t kc = r.f.key_heads * r.f.head_dim;
    if (!keys && (a[2] != Py_None || a[6] != Py_None || a[11] != Py_None || a[13] != Py_None)) refuse("dk_out", "dk, k_weight and dk_weight go with k");
    s.matrix_of(a[1], "dq_out", IN, false, s.rows, s.cols, s.type, (const void**)&r.f.q_out, &r.f.q_out_stride);
    s.matrix_of(a[2], "dk_out", IN, !keys, s.rows, kc, s.type, (const void**)&r.f.k_out, &r.f.k_out_stride);
    s.matrix_of(a[5], "dq", OUT, false, s.rows, s.cols, s.type, (const void**)&r.dq, &r.dq_stride);
    s.matrix_of(a[6], "dk", OUT, !keys, s.rows, kc, s.type, (const void**)&r.dk, &r.dk_stride);
    void* p[4];
    r.f.param_dtype = s.params({{a[10], "q_weight", IN}, {a[11], "k_weight", IN}, {a[12], "dq_weight", OUT}, {a[13], "dk_weight", OUT}}, p, r.f.head_dim);
    r.f.q_weight = p[0];
    r.f.k_weight = p[1];
    r.dq_weight = p[2];
    r.dk_weight = p[3];
    return ready() ? (long)adacgd_qk_norm_backward(s.h->ctx, &r) : RETRY;
  });
}

// q, k and v, the heads they hold, and the sequences.
void attention_of(Shape& s, adacgd_attention_inputs* r, PyObject* q, PyObject* k, PyObject* v, PyObject* heads, PyObject* sequences, PyObject* seq_start,
                  PyObject* causal, PyObject* scale, PyObject* mask) {
  s.lead(q, "q", &r->q, &r->q_stride);
  const int64_t count = whole(heads);
  if (count < 1 || count > 65535 || s.cols < 1 || s.cols % count) refuse("heads", "must be in [1, 65535] and divide q's columns");
  const int64_t dim = s.cols / count;
  if (dim > ADACGD_ATTENTION_MAX_HEAD) refuse("q", "must have at most " + std::to_string(ADACGD_ATTENTION_MAX_HEAD) + " columns a head");
  const at::Tensor& kt = *tensor(k, "k", false);
  const int64_t kc = kt.dim() == 2 ? kt.size(1) : 0;
  if (kc < 1 || kc % dim || count % (kc / dim)) refuse("k", "must be a 2-D tensor of key heads whose number divides heads");
  r->heads = (int32_t)count;
  r->key_heads = (int32_t)(kc / dim);
  r->head_dim = (int32_t)dim;
  r->tokens = s.rows;
  r->dtype = s.code;
  s.matrix_of(k, "k", IN, false, s.rows, kc, s.type, &r->k, &r->k_stride);
  s.matrix_of(v, "v", IN, false, s.rows, kc, s.type, &r->v, &r->v_stride);
  s.runs(seq_start, sequences, &r->seq_start, &r->sequences);
  r->causal = truth(causal);
  r->scale = scale == Py_None ? (float)(1.0 / std::sqrt((double)dim)) : (float)number(scale);
  r->mask = s.counted(mask, s.rows);
}

// (handle, q, k, v, out, lse, heads, sequences, seq_start, causal, scale, mask)
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(a, n, 12, [&](Shape& s, auto ready) -> long {
    adacgd_attention_args r;
    attention_of(s, &r.in, a[1], a[2], a[3], a[6], a[7], a[8], a[9], a[10], a[11]);
    MAT(out, 4, OUT, false);
    r.lse = (float*)s.vector(a[5], "lse", OUT, true, s.rows * r.in.heads, at::kFloat);
    return ready() ? (long)adacgd_attention(s.h->ctx, &r) : RETRY;
  });
}

// (handle, dout, q, k, v, out, lse, row_dot, dq, dk, dv, heads, sequences, seq_start, causal, scale, mask)
PyObject* attention_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(a, n, 17, [&](Shape& s, auto ready) -> long {
    adacgd_attention_backward_args r;
    attention_of(s, &r.in, a[2], a[3], a[4], a[11], a[12], a[13], a[14], a[15], a[16]);
    const int64_t kc = (int64_t)r.in.key_heads * r.in.head_dim;
    MAT(dout, 1, IN, false);
    MAT(out, 5, IN, false);
    r.lse = (const float*)s.vector(a[6], "lse", IN, false, s.rows * r.in.heads, at::kFloat);
    r.row_dot = (float*)s.vector(a[7], "row_dot", OUT, false, s.rows * r.in.heads, at::kFloat);
    MAT(dq, 8, OUT, false);
    s.matrix_of(a[9], "dk", OUT, false, s.rows, kc, s.type, (const void**)&r.dk, &r.dk_stride);
    s.matrix_of(a[10], "dv", OUT, false, s.rows, kc, s.type, (const void**)&r.dv, &r.dv_stride);
    return ready() ? (long)adacgd_attention_backward(s.h->ctx, &r) : RETRY;
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
                         FAST(preference_loss), FAST(policy_loss),     FAST(embedding),           FAST(embedding_backward),
                         FAST(qk_norm),         FAST(qk_norm_backward), FAST(attention),          FAST(attention_backward),
                         {"bind", bind, METH_VARARGS, nullptr},
                         {"force", force, METH_VARARGS, nullptr},      {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_train_binding", "Binding of the training operators.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__train_binding() { return PyModule_Create(&module); }

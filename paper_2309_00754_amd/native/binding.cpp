// The accepted form of the Python binding's calls, in native code: checks the
// tensors (dtype, device, contiguity, shape), takes their pointers and the
// current stream, and calls libhydra.  Whatever is not the accepted form (a
// host tensor, another dtype, a sequence that is no list or tuple, a missing
// workspace, a tensor subclass, an exception on the way) returns kSlow, and
// the Python function checks the arguments itself, with its own messages.
//
// Why: at decode sizes a call's host time is its time.  In Python, one
// condition of attribute reads per tensor and ctypes took 7.6 us for the small
// linear (its kernel 6.2), 19.8 for four projections (24 tensors; 15) and 7.5
// for each call of the PPO step (kernels 2.8 to 4.8).
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

#include <vector>

#include "../../include/hydra.h"

namespace {

constexpr long kSlow = -1000;

// kAny: bf16 or fp32; kFp8: e4m3; kScale: a scale byte; kI64: 64-bit whole numbers
enum Kind { kBf16, kF32, kI32, kU8, kAny, kFp8, kScale, kI64 };

// Collects the arguments of one call; ok turns false at the first that is not
// of the accepted form.
struct Take {
  bool ok = true;
  int device = -1;           // of the tensors so far
  bool one_device = true;

  const at::Tensor* tensor(PyObject* o, Kind kind, bool rows_apart = false) {
    if (!ok || o == Py_None) return nullptr;
    if (!THPVariable_CheckExact(o)) {
      ok = false;
      return nullptr;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    const auto d = t.scalar_type();
    const bool dtype = kind == kBf16   ? d == at::kBFloat16 || d == at::kShort || d == at::kUInt16
                       : kind == kF32  ? d == at::kFloat
                       : kind == kI32  ? d == at::kInt
                       : kind == kU8   ? d == at::kByte
                       : kind == kFp8  ? d == at::kFloat8_e4m3fn || d == at::kByte
                       : kind == kScale ? d == at::kFloat8_e8m0fnu || d == at::kByte
                       : kind == kI64  ? d == at::kLong || d == at::kUInt64
                                       : d == at::kBFloat16 || d == at::kFloat || d == at::kShort || d == at::kUInt16;
    ok = t.is_cuda() && dtype && (rows_apart || t.is_contiguous());
    if (!ok) return nullptr;
    const int on = t.get_device();
    one_device = one_device && (device < 0 || device == on);
    device = on;
    return &t;
  }
  static hydra_dtype type_of(const at::Tensor* t) {
    return t && t->scalar_type() == at::kFloat ? HYDRA_F32 : HYDRA_BF16;
  }
  // None, or a tensor of bf16 or fp32 of this shape, and its type.
  void* any1(PyObject* o, int64_t n, hydra_dtype& type) {
    const at::Tensor* t = tensor(o, kAny);
    type = type_of(t);
    return ptr(t, t && t->dim() == 1 && t->size(0) == n);
  }
  void* any2(PyObject* o, int64_t n, int64_t m, hydra_dtype& type) {
    const at::Tensor* t = tensor(o, kAny);
    type = type_of(t);
    return ptr(t, t && t->dim() == 2 && t->size(0) == n && t->size(1) == m);
  }
  // A matrix of bf16 or fp32 that has to be there, its rows contiguous and
  // possibly apart: its sizes, type and row distance.
  void* rows_of(PyObject* o, int64_t& M, int64_t& V, hydra_dtype& type, int64_t& ld) {
    const at::Tensor* t = tensor(o, kAny, true);
    if (!t || t->dim() != 2) {
      ok = false;
      return nullptr;
    }
    M = t->size(0);
    V = t->size(1);
    type = type_of(t);
    ld = M > 1 ? t->stride(0) : V;
    ok = (V <= 1 || t->stride(1) == 1) && ld >= V;
    return t->data_ptr();
  }
  // None: no workspace.
  void* maybe_workspace(PyObject* o, size_t& bytes) {
    bytes = 0;
    return o == Py_None ? nullptr : workspace(o, bytes);
  }
  // The stream of a call that goes where its tensors are: they have to be on
  // the current device, and so has a given stream.
  void* stream_here(PyObject* o) {
    ok = ok && one_device && device == (int)c10::hip::current_device();
    if (ok && o != Py_None) {
      PyObject* d = PyObject_GetAttrString(o, "device_index");
      ok = d && PyLong_Check(d) && PyLong_AsLong(d) == device;
      Py_XDECREF(d);
      if (PyErr_Occurred()) {
        PyErr_Clear();
        ok = false;
      }
    }
    return stream(o);
  }
  // A matrix that has to be there: its sizes and pointer.
  const uint16_t* matrix(PyObject* o, int64_t& rows, int64_t& cols, Kind kind = kBf16) {
    const at::Tensor* t = tensor(o, kind);
    if (!t || t->dim() != 2) {
      ok = false;
      return nullptr;
    }
    rows = t->size(0);
    cols = t->size(1);
    return static_cast<const uint16_t*>(t->data_ptr());
  }
  int64_t rows(PyObject* o) {  // size(0) of a tensor, 0 for None
    if (!ok || o == Py_None) return 0;
    if (!THPVariable_CheckExact(o) || THPVariable_Unpack(o).dim() < 1) {
      ok = false;
      return 0;
    }
    return THPVariable_Unpack(o).size(0);
  }
  void* ptr(const at::Tensor* t, bool shape) {
    if (!ok || !t) return nullptr;
    if (!shape) {
      ok = false;
      return nullptr;
    }
    return t->data_ptr();
  }
  // None, or a tensor of this shape.
  template <class T>
  T* at1(PyObject* o, Kind kind, int64_t n) {
    const at::Tensor* t = tensor(o, kind);
    return static_cast<T*>(ptr(t, t && t->dim() == 1 && t->size(0) == n));
  }
  template <class T>
  T* at2(PyObject* o, Kind kind, int64_t n, int64_t m) {
    const at::Tensor* t = tensor(o, kind);
    return static_cast<T*>(ptr(t, t && t->dim() == 2 && t->size(0) == n && t->size(1) == m));
  }
  void* workspace(PyObject* o, size_t& bytes) {
    const at::Tensor* t = tensor(o, kU8);
    if (!t) {
      ok = false;
      return nullptr;
    }
    bytes = (size_t)t->numel();
    return t->data_ptr();
  }
  double number(PyObject* o) {
    if (!PyFloat_Check(o) && !PyLong_CheckExact(o)) {
      ok = false;
      return 0.0;
    }
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
      PyErr_Clear();
      ok = false;
    }
    return v;
  }
  float real(PyObject* o) { return (float)number(o); }
  int64_t whole(PyObject* o) {
    if (!PyLong_CheckExact(o)) {
      ok = false;
      return 0;
    }
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
      PyErr_Clear();
      ok = false;
    }
    return v;
  }
  void* stream(PyObject* o) {
    if (!ok) return nullptr;
    if (o == Py_None) return reinterpret_cast<void*>(c10::hip::getCurrentHIPStream().stream());
    PyObject* h = PyObject_GetAttrString(o, "cuda_stream");
    if (!h) {
      PyErr_Clear();
      ok = false;
      return nullptr;
    }
    void* p = PyLong_Check(h) ? PyLong_AsVoidPtr(h) : nullptr;
    if (PyErr_Occurred() || !PyLong_Check(h)) {
      PyErr_Clear();
      ok = false;
    }
    Py_DECREF(h);
    return p;
  }
  // n entries of a list or tuple; None (where allowed): n times None.
  PyObject* const* list(PyObject* o, int64_t n, bool may_be_none = false) {
    static PyObject* const nones[HYDRA_MAX_GROUP] = {Py_None, Py_None, Py_None, Py_None,
                                                     Py_None, Py_None, Py_None, Py_None};
    if (may_be_none && o == Py_None && n <= HYDRA_MAX_GROUP) return nones;
    if (!(PyList_CheckExact(o) || PyTuple_CheckExact(o)) || PySequence_Fast_GET_SIZE(o) != n) {
      ok = false;
      return nones;
    }
    return PySequence_Fast_ITEMS(o);
  }
};

// f(take) fills the arguments and returns the library call to make; the call
// itself runs without the interpreter's lock, as through ctypes.
template <class F>
PyObject* guarded(F&& f) {
  try {
    Take a;
    auto call = f(a);
    if (!a.ok) return PyLong_FromLong(kSlow);
    hydra_status st;
    Py_BEGIN_ALLOW_THREADS st = call();
    Py_END_ALLOW_THREADS return PyLong_FromLong((long)st);
  } catch (...) {
    PyErr_Clear();
    return PyLong_FromLong(kSlow);
  }
}

#define HYDRA_PY(name, count)                                                        \
  PyObject* name##_(PyObject* const* v);                                             \
  PyObject* name(PyObject*, PyObject* const* v, Py_ssize_t n) {                      \
    if (n != count) {                                                                \
      PyErr_SetString(PyExc_TypeError, #name ": wrong number of arguments");         \
      return nullptr;                                                                \
    }                                                                                \
    return name##_(v);                                                               \
  }                                                                                  \
  PyObject* name##_(PyObject* const* v)

// x W A B s y_off y_on workspace stream with_workspace
HYDRA_PY(lora_linear, 10) {
  return guarded([&](Take& a) {
    int64_t M = 0, K = 0, N = a.rows(v[1]), r = a.rows(v[2]);
    const uint16_t* x = a.matrix(v[0], M, K);
    const uint16_t* W = a.at2<uint16_t>(v[1], kBf16, N, K);
    const uint16_t* A = a.at2<uint16_t>(v[2], kBf16, r, K);
    const uint16_t* B = a.at2<uint16_t>(v[3], kBf16, N, r);
    const float s = a.real(v[4]);
    float* yo = a.at2<float>(v[5], kF32, M, N);
    float* yn = a.at2<float>(v[6], kF32, M, N);
    const bool with_ws = v[9] == Py_True;
    size_t bytes = 0;
    void* ws = with_ws ? a.workspace(v[7], bytes) : nullptr;
    a.ok = a.ok && W;
    void* st = a.stream(v[8]);
    return [=]() {
      return with_ws ? hydra_lora_linear_ws(x, W, A, B, s, M, N, K, r, yo, yn, ws, bytes, st)
                     : hydra_lora_linear(x, W, A, B, s, M, N, K, r, yo, yn, st);
    };
  });
}

// xs Ws As Bs ss y_offs y_ons workspace stream with_workspace
HYDRA_PY(lora_linear_group, 10) {
  struct Members {
    const uint16_t *x[HYDRA_MAX_GROUP], *W[HYDRA_MAX_GROUP], *A[HYDRA_MAX_GROUP], *B[HYDRA_MAX_GROUP];
    float *yo[HYDRA_MAX_GROUP], *yn[HYDRA_MAX_GROUP], s[HYDRA_MAX_GROUP];
  } m;
  return guarded([&](Take& a) {
    const int64_t G = PyList_CheckExact(v[1]) || PyTuple_CheckExact(v[1]) ? PySequence_Fast_GET_SIZE(v[1]) : 0;
    a.ok = G >= 1 && G <= HYDRA_MAX_GROUP;
    int64_t M = 0, K = 0, N = 0, r = 0;
    const bool with_ws = v[9] == Py_True;
    size_t bytes = 0;
    void* ws = nullptr;
    if (a.ok) {
      PyObject *const *xs = a.list(v[0], G), *const *Ws = a.list(v[1], G), *const *As = a.list(v[2], G),
                      *const *Bs = a.list(v[3], G), *const *ss = a.list(v[4], G),
                      *const *yo = a.list(v[5], G, true), *const *yn = a.list(v[6], G, true);
      if (a.ok) {
        a.matrix(xs[0], M, K);
        N = a.rows(Ws[0]);
        for (int64_t i = G - 1; i >= 0; --i)
          if (As[i] != Py_None) r = a.rows(As[i]);
        for (int64_t i = 0; i < G; ++i) {
          m.x[i] = a.at2<uint16_t>(xs[i], kBf16, M, K);
          m.W[i] = a.at2<uint16_t>(Ws[i], kBf16, N, K);
          m.A[i] = a.at2<uint16_t>(As[i], kBf16, r, K);
          m.B[i] = a.at2<uint16_t>(Bs[i], kBf16, N, r);
          m.yo[i] = a.at2<float>(yo[i], kF32, M, N);
          m.yn[i] = a.at2<float>(yn[i], kF32, M, N);
          m.s[i] = a.real(ss[i]);
        }
        if (with_ws) ws = a.workspace(v[7], bytes);
      }
    }
    void* st = a.stream(v[8]);
    return [=, &m]() {
      return with_ws ? hydra_lora_linear_group_ws(G, m.x, m.W, m.A, m.B, m.s, M, N, K, r, m.yo, m.yn, ws, bytes, st)
                     : hydra_lora_linear_group(G, m.x, m.W, m.A, m.B, m.s, M, N, K, r, m.yo, m.yn, st);
    };
  });
}

// x_off W x_ons As Bs ss y_off y_ons workspace stream with_workspace
HYDRA_PY(lora_linear_multi, 11) {
  struct Inputs {
    const uint16_t *x[HYDRA_MAX_ADAPTERS], *A[HYDRA_MAX_ADAPTERS], *B[HYDRA_MAX_ADAPTERS];
    float *yn[HYDRA_MAX_ADAPTERS], s[HYDRA_MAX_ADAPTERS];
  } m;
  return guarded([&](Take& a) {
    const int64_t n = PyList_CheckExact(v[2]) || PyTuple_CheckExact(v[2]) ? PySequence_Fast_GET_SIZE(v[2]) : -1;
    a.ok = n >= 1 && n <= HYDRA_MAX_ADAPTERS;
    int64_t M = 0, K = 0, N = 0, r = 0;
    const uint16_t *xo = nullptr, *W = nullptr;
    float* yo = nullptr;
    const bool with_ws = v[10] == Py_True;
    size_t bytes = 0;
    void* ws = nullptr;
    if (a.ok) {
      PyObject *const *xs = a.list(v[2], n), *const *As = a.list(v[3], n, true), *const *Bs = a.list(v[4], n, true),
                      *const *ss = a.list(v[5], n), *const *yn = a.list(v[7], n, true);
      if (a.ok) {
        a.matrix(v[0] != Py_None ? v[0] : xs[0], M, K);
        N = a.rows(v[1]);
        for (int64_t i = n - 1; i >= 0; --i)
          if (As[i] != Py_None) r = a.rows(As[i]);
        W = a.at2<uint16_t>(v[1], kBf16, N, K);
        xo = a.at2<uint16_t>(v[0], kBf16, M, K);
        yo = a.at2<float>(v[6], kF32, M, N);
        for (int64_t i = 0; i < n; ++i) {
          m.x[i] = a.at2<uint16_t>(xs[i], kBf16, M, K);
          m.A[i] = a.at2<uint16_t>(As[i], kBf16, r, K);
          m.B[i] = a.at2<uint16_t>(Bs[i], kBf16, N, r);
          m.yn[i] = a.at2<float>(yn[i], kF32, M, N);
          m.s[i] = a.real(ss[i]);
        }
        if (with_ws) ws = a.workspace(v[8], bytes);
      }
    }
    void* st = a.stream(v[9]);
    return [=, &m]() {
      return with_ws ? hydra_lora_linear_multi_ws(xo, W, n, m.x, m.A, m.B, m.s, M, N, K, r, yo, m.yn, ws, bytes, st)
                     : hydra_lora_linear_multi(xo, W, n, m.x, m.A, m.B, m.s, M, N, K, r, yo, m.yn, st);
    };
  });
}

// h_act h W_lm A B s tokens w_rm n_seq seq_len lp_on lp_off kl reward lse_on lse_off workspace err_flag stream
// own_scratch (h_act None: one input)
HYDRA_PY(score, 20) {
  return guarded([&](Take& a) {
    int64_t M = 0, K = 0, V = a.rows(v[2]), r = a.rows(v[3]);
    const uint16_t* h = a.matrix(v[1], M, K);
    const uint16_t* ha = a.at2<uint16_t>(v[0], kBf16, M, K);
    const uint16_t* W = a.at2<uint16_t>(v[2], kBf16, V, K);
    const uint16_t* A = a.at2<uint16_t>(v[3], kBf16, r, K);
    const uint16_t* B = a.at2<uint16_t>(v[4], kBf16, V, r);
    const float s = a.real(v[5]);
    const int32_t* tok = a.at1<int32_t>(v[6], kI32, M);
    const uint16_t* w_rm = a.at1<uint16_t>(v[7], kBf16, K);
    const int64_t n_seq = a.whole(v[8]), seq_len = a.whole(v[9]);
    float* lp_on = a.at1<float>(v[10], kF32, M);
    float* lp_off = a.at1<float>(v[11], kF32, M);
    float* kl = a.at1<float>(v[12], kF32, M);
    float* reward = a.at1<float>(v[13], kF32, n_seq);
    float* lse_on = a.at1<float>(v[14], kF32, M);
    float* lse_off = a.at1<float>(v[15], kF32, M);
    const bool own = v[19] == Py_True, two = v[0] != Py_None;
    size_t bytes = 0;
    void* ws = own ? nullptr : a.workspace(v[16], bytes);
    int32_t* err = a.at1<int32_t>(v[17], kI32, 1);
    a.ok = a.ok && W && n_seq >= 1 && seq_len >= 1 && n_seq <= M && seq_len <= M && n_seq * seq_len == M;
    void* st = a.stream(v[18]);
    return [=]() {
      if (own)
        return hydra_score_noalloc(h, W, A, B, s, tok, w_rm, n_seq, seq_len, K, V, r, lp_on, lp_off, kl, reward, lse_on,
                                   lse_off, err, st);
      if (two)
        return hydra_score_two_input(ha, h, W, A, B, s, tok, w_rm, n_seq, seq_len, K, V, r, lp_on, lp_off, kl, reward,
                                     lse_on, lse_off, ws, bytes, err, st);
      return hydra_score(h, W, A, B, s, tok, w_rm, n_seq, seq_len, K, V, r, lp_on, lp_off, kl, reward, lse_on, lse_off,
                         ws, bytes, err, st);
    };
  });
}

// logits_on logits_off tokens lp_on lp_off kl lse_on lse_off err_flag stream
HYDRA_PY(score_logits, 10) {
  return guarded([&](Take& a) {
    int64_t M = 0, V = 0;
    const void* on = a.matrix(v[0], M, V, kF32);
    const float* off = a.at2<float>(v[1], kF32, M, V);
    const int32_t* tok = a.at1<int32_t>(v[2], kI32, M);
    float* o[5];
    for (int i = 0; i < 5; ++i) o[i] = a.at1<float>(v[3 + i], kF32, M);
    int32_t* err = a.at1<int32_t>(v[8], kI32, 1);
    void* st = a.stream(v[9]);
    float *lp_on = o[0], *lp_off = o[1], *kl = o[2], *lse_on = o[3], *lse_off = o[4];
    return [=]() {
      return hydra_score_logits(static_cast<const float*>(on), off, tok, M, V, lp_on, lp_off, kl, lse_on, lse_off, err,
                                st);
    };
  });
}

// h w_v values stream
HYDRA_PY(value_head, 4) {
  return guarded([&](Take& a) {
    int64_t M = 0, K = 0;
    const uint16_t* h = a.matrix(v[0], M, K);
    const uint16_t* w = a.at1<uint16_t>(v[1], kBf16, K);
    float* values = a.at1<float>(v[2], kF32, M);
    void* st = a.stream(v[3]);
    return [=]() { return hydra_value_head(h, w, M, K, values, st); };
  });
}

// kl reward values n_seq seq_len start beta gamma lam rewards advantages returns stream
HYDRA_PY(ppo_advantages, 13) {
  return guarded([&](Take& a) {
    const int64_t n_seq = a.whole(v[3]), seq_len = a.whole(v[4]), start = a.whole(v[5]);
    a.ok = a.ok && n_seq >= 1 && seq_len >= 1 && n_seq <= (int64_t(1) << 40) / seq_len;
    const int64_t M = a.ok ? n_seq * seq_len : 0;
    const float* kl = a.at1<float>(v[0], kF32, M);
    const float* reward = a.at1<float>(v[1], kF32, n_seq);
    const float* values = a.at1<float>(v[2], kF32, M);
    const float beta = a.real(v[6]), gamma = a.real(v[7]), lam = a.real(v[8]);
    float* rewards = a.at1<float>(v[9], kF32, M);
    float* adv = a.at1<float>(v[10], kF32, M);
    float* ret = a.at1<float>(v[11], kF32, M);
    void* st = a.stream(v[12]);
    return [=]() {
      return hydra_ppo_advantages(kl, reward, values, n_seq, seq_len, start, beta, gamma, lam, rewards, adv, ret, st);
    };
  });
}

// lp_new lp_old advantages values returns n_seq seq_len start eps losses d_lp d_v stream
HYDRA_PY(ppo_loss, 13) {
  return guarded([&](Take& a) {
    const int64_t n_seq = a.whole(v[5]), seq_len = a.whole(v[6]), start = a.whole(v[7]);
    a.ok = a.ok && n_seq >= 1 && seq_len >= 1 && n_seq <= (int64_t(1) << 40) / seq_len;
    const int64_t M = a.ok ? n_seq * seq_len : 0;
    const float* in[5];
    for (int i = 0; i < 5; ++i) in[i] = a.at1<float>(v[i], kF32, M);
    const float eps = a.real(v[8]);
    float* losses = a.at1<float>(v[9], kF32, 3);
    float* d_lp = a.at1<float>(v[10], kF32, M);
    float* d_v = a.at1<float>(v[11], kF32, M);
    void* st = a.stream(v[12]);
    const float *lp_new = in[0], *lp_old = in[1], *adv = in[2], *values = in[3], *returns = in[4];
    return [=]() {
      return hydra_ppo_loss(lp_new, lp_old, adv, values, returns, n_seq, seq_len, start, eps, losses, d_lp, d_v, st);
    };
  });
}

// x Wt A B s dy dx dA dB workspace stream
HYDRA_PY(lora_linear_backward, 11) {
  return guarded([&](Take& a) {
    int64_t M = 0, N = 0, r = 0, K = 0;
    const uint16_t* dy = a.matrix(v[5], M, N);
    const uint16_t* A = a.matrix(v[2], r, K);  // (without an adapter: the Python path)
    const uint16_t* x = a.at2<uint16_t>(v[0], kBf16, M, K);
    const uint16_t* Wt = a.at2<uint16_t>(v[1], kBf16, K, N);
    const uint16_t* B = a.at2<uint16_t>(v[3], kBf16, N, r);
    const float s = a.real(v[4]);
    float* dx = a.at2<float>(v[6], kF32, M, K);
    float* dA = a.at2<float>(v[7], kF32, r, K);
    float* dB = a.at2<float>(v[8], kF32, N, r);
    size_t bytes = 0;
    void* ws = a.workspace(v[9], bytes);
    void* st = a.stream(v[10]);
    return [=]() { return hydra_lora_linear_backward(x, Wt, A, B, s, dy, M, N, K, r, dx, dA, dB, ws, bytes, st); };
  });
}

// x weight bias y mean rstd eps stream
HYDRA_PY(layer_norm, 8) {
  return guarded([&](Take& a) {
    const at::Tensor* x = a.tensor(v[0], kAny);
    a.ok = a.ok && x && x->dim() == 2;
    const int64_t M = a.ok ? x->size(0) : 0, K = a.ok ? x->size(1) : 0;
    const void* xp = a.ok ? x->data_ptr() : nullptr;
    const hydra_dtype xt = Take::type_of(x);
    hydra_dtype wt, bt, yt;
    const void* w = a.any1(v[1], K, wt);
    const void* b = a.any1(v[2], K, bt);
    a.ok = a.ok && (!w || !b || wt == bt);
    void* y = a.any2(v[3], M, K, yt);
    float* mean = a.at1<float>(v[4], kF32, M);
    float* rstd = a.at1<float>(v[5], kF32, M);
    const float eps = a.real(v[6]);
    void* st = a.stream_here(v[7]);
    return [=]() { return hydra_layer_norm(xp, xt, w, b, w ? wt : bt, eps, M, K, y, yt, mean, rstd, st); };
  });
}

// dy x weight mean rstd dx dweight dbias workspace stream
HYDRA_PY(layer_norm_backward, 10) {
  return guarded([&](Take& a) {
    const at::Tensor* x = a.tensor(v[1], kAny);
    a.ok = a.ok && x && x->dim() == 2;
    const int64_t M = a.ok ? x->size(0) : 0, K = a.ok ? x->size(1) : 0;
    const void* xp = a.ok ? x->data_ptr() : nullptr;
    const hydra_dtype xt = Take::type_of(x);
    hydra_dtype dyt, wt, dxt;
    const void* dy = a.any2(v[0], M, K, dyt);
    const void* w = a.any1(v[2], K, wt);
    const float* mean = a.at1<float>(v[3], kF32, M);
    const float* rstd = a.at1<float>(v[4], kF32, M);
    void* dx = a.any2(v[5], M, K, dxt);
    float* dw = a.at1<float>(v[6], kF32, K);
    float* db = a.at1<float>(v[7], kF32, K);
    size_t bytes = 0;
    void* ws = a.workspace(v[8], bytes);
    void* st = a.stream_here(v[9]);
    return [=]() {
      return hydra_layer_norm_backward(dy, dyt, xp, xt, w, wt, mean, rstd, M, K, dx, dxt, dw, db, ws, bytes, st);
    };
  });
}

// logits tokens lp lse entropy top_ids top_lp workspace err_flag stream
HYDRA_PY(token_logprobs, 10) {
  return guarded([&](Take& a) {
    int64_t M = 0, V = 0, ld = 0, top = 0;
    hydra_dtype zt = HYDRA_BF16;
    const void* z = a.rows_of(v[0], M, V, zt, ld);
    const int32_t* tok = a.at1<int32_t>(v[1], kI32, M);
    float* lp = a.at1<float>(v[2], kF32, M);
    float* lse = a.at1<float>(v[3], kF32, M);
    float* ent = a.at1<float>(v[4], kF32, M);
    const at::Tensor* ids = a.tensor(v[5], kI32);
    if (ids && ids->dim() == 2) top = ids->size(1);
    int32_t* idp = a.at2<int32_t>(v[5], kI32, M, top);
    float* tlp = a.at2<float>(v[6], kF32, M, top);
    size_t bytes = 0, need = 0;
    void* ws = a.maybe_workspace(v[7], bytes);
    int32_t* err = a.at1<int32_t>(v[8], kI32, 1);
    // (one that is needed and missing, or sizes that are refused: the Python path)
    a.ok = a.ok && (ws || (hydra_token_logprobs_workspace_bytes(M, V, top, &need) == HYDRA_OK && need == 0));
    void* st = a.stream_here(v[9]);
    return [=]() {
      return hydra_token_logprobs(z, zt, ld, tok, M, V, top, lp, lse, ent, idp, tlp, ws, bytes, err, st);
    };
  });
}

// logits tokens lse d_logits d_lp entropy d_entropy err_flag stream
HYDRA_PY(token_logprobs_backward, 9) {
  return guarded([&](Take& a) {
    int64_t M = 0, V = 0, ld = 0, dM = 0, dV = 0, ld_d = 0;
    hydra_dtype zt = HYDRA_BF16, dt = HYDRA_BF16;
    const void* z = a.rows_of(v[0], M, V, zt, ld);
    void* dz = a.ok ? a.rows_of(v[3], dM, dV, dt, ld_d) : nullptr;
    a.ok = a.ok && dM == M && dV == V;
    const int32_t* tok = a.at1<int32_t>(v[1], kI32, M);
    const float* lse = a.at1<float>(v[2], kF32, M);
    const float* d_lp = a.at1<float>(v[4], kF32, M);
    const float* ent = a.at1<float>(v[5], kF32, M);
    const float* d_ent = a.at1<float>(v[6], kF32, M);
    int32_t* err = a.at1<int32_t>(v[7], kI32, 1);
    void* st = a.stream_here(v[8]);
    return [=]() {
      return hydra_token_logprobs_backward(z, zt, ld, tok, lse, ent, d_lp, d_ent, M, V, dz, dt, ld_d, err, st);
    };
  });
}

// grads max_norm (None: the norm alone) norm outs workspace err_flag stream
HYDRA_PY(grad_clip, 7) {
  struct Tensors {
    std::vector<const void*> g;
    std::vector<void*> out;
    std::vector<int32_t> type, out_type;
    std::vector<int64_t> numel;
  } m;
  return guarded([&](Take& a) {
    const int64_t n = PyList_CheckExact(v[0]) || PyTuple_CheckExact(v[0]) ? PySequence_Fast_GET_SIZE(v[0]) : -1;
    a.ok = n >= 1 && n <= HYDRA_MAX_GRADS;
    const bool clip = v[1] != Py_None, own = v[3] != Py_None;
    if (a.ok) {
      PyObject *const *gs = a.list(v[0], n), *const *os = own ? a.list(v[3], n) : nullptr;
      m.g.reserve(n);
      m.type.reserve(n);
      m.numel.reserve(n);
      for (int64_t i = 0; a.ok && i < n; ++i) {
        const at::Tensor* g = a.tensor(gs[i], kAny);
        if (!g) {
          a.ok = false;
          break;
        }
        m.g.push_back(g->data_ptr());
        m.type.push_back(Take::type_of(g));
        m.numel.push_back(g->numel());
        if (!own) continue;
        const at::Tensor* o = a.tensor(os[i], kAny);
        if (!o || o->sizes() != g->sizes()) {
          a.ok = false;
          break;
        }
        m.out.push_back(o->data_ptr());
        m.out_type.push_back(Take::type_of(o));
      }
    }
    const float max_norm = clip ? a.real(v[1]) : 0.f;
    float* norm = a.at1<float>(v[2], kF32, 1);
    size_t bytes = 0;
    void* ws = a.workspace(v[4], bytes);
    int32_t* err = a.at1<int32_t>(v[5], kI32, 1);
    void* st = a.stream_here(v[6]);
    return [=, &m]() {
      if (!clip) return hydra_grad_norm(n, m.g.data(), m.type.data(), m.numel.data(), norm, ws, bytes, st);
      return hydra_grad_clip(n, m.g.data(), m.type.data(), m.numel.data(), max_norm, norm, own ? m.out.data() : nullptr,
                             own ? m.out_type.data() : nullptr, ws, bytes, err, st);
    };
  });
}

// x q scale block_rows qt scale_t stream
HYDRA_PY(fp8_quantize, 7) {
  return guarded([&](Take& a) {
    const at::Tensor* x = a.tensor(v[0], kAny);
    a.ok = a.ok && x && x->dim() == 2;
    const int64_t M = a.ok ? x->size(0) : 0, K = a.ok ? x->size(1) : 0;
    const void* xp = a.ok ? x->data_ptr() : nullptr;
    const hydra_dtype xt = Take::type_of(x);
    const int64_t rows = a.whole(v[3]);
    a.ok = a.ok && (rows == 1 || rows == 128);
    const int64_t kb = (K + 127) / 128, mb = a.ok ? (M + rows - 1) / rows : 0;
    uint8_t* q = a.at2<uint8_t>(v[1], kFp8, M, K);
    uint8_t* scale = a.at2<uint8_t>(v[2], kScale, mb, kb);
    uint8_t* qt = a.at2<uint8_t>(v[4], kFp8, K, M);
    uint8_t* st = a.at2<uint8_t>(v[5], kScale, kb, mb);
    void* stream = a.stream_here(v[6]);
    return [=]() { return hydra_fp8_quantize(xp, xt, M, K, rows, q, scale, qt, st, stream); };
  });
}

// x Wq w_scale A B s y_off y_on x_adapter xq x_scale workspace stream
HYDRA_PY(fp8_lora_linear, 13) {
  return guarded([&](Take& a) {
    const int64_t N = a.rows(v[1]), r = a.rows(v[3]);
    const at::Tensor* W = a.tensor(v[1], kFp8);
    a.ok = a.ok && W && W->dim() == 2;
    const int64_t K = a.ok ? W->size(1) : 0, kb = (K + 127) / 128;
    const uint8_t* Wp = a.ok ? static_cast<const uint8_t*>(W->data_ptr()) : nullptr;
    const int64_t M = a.rows(v[0] != Py_None ? v[0] : v[9]);
    const uint16_t* x = a.at2<uint16_t>(v[0], kBf16, M, K);
    const uint8_t* ws = a.at2<uint8_t>(v[2], kScale, (N + 127) / 128, kb);
    const uint16_t* A = a.at2<uint16_t>(v[3], kBf16, r, K);
    const uint16_t* B = a.at2<uint16_t>(v[4], kBf16, N, r);
    const float s = a.real(v[5]);
    hydra_dtype ot, nt;
    void* yo = a.any2(v[6], M, N, ot);
    void* yn = a.any2(v[7], M, N, nt);
    a.ok = a.ok && (!yo || !yn || ot == nt);
    const uint16_t* xa = a.at2<uint16_t>(v[8], kBf16, M, K);
    const uint8_t* xq = a.at2<uint8_t>(v[9], kFp8, M, K);
    const uint8_t* xs = a.at2<uint8_t>(v[10], kScale, M, kb);
    size_t bytes = 0;
    void* w = a.workspace(v[11], bytes);
    void* st = a.stream_here(v[12]);
    return [=]() {
      return hydra_fp8_lora_linear(x, xa, xq, xs, Wp, ws, A, B, s, M, N, K, r, yo, yn, yo ? ot : nt, w, bytes, st);
    };
  });
}

// x Wqt wt_scale A B s dy dx dA dB p rng workspace stream
HYDRA_PY(fp8_lora_linear_backward, 14) {
  return guarded([&](Take& a) {
    int64_t M = 0, N = 0, K = 0;
    const uint16_t* dy = a.matrix(v[6], M, N);
    const int64_t r = a.rows(v[3]);
    // K from the first of A, x and Wqt that is there
    PyObject* const from = v[3] != Py_None ? v[3] : v[0] != Py_None ? v[0] : v[1];
    a.ok = a.ok && THPVariable_CheckExact(from) && THPVariable_Unpack(from).dim() == 2;
    if (a.ok) K = THPVariable_Unpack(from).size(from == v[1] ? 0 : 1);
    const int64_t nb = (N + 127) / 128;
    const uint16_t* x = a.at2<uint16_t>(v[0], kBf16, M, K);
    const uint8_t* W = a.at2<uint8_t>(v[1], kFp8, K, N);
    const uint8_t* ws = a.at2<uint8_t>(v[2], kScale, (K + 127) / 128, nb);
    const uint16_t* A = a.at2<uint16_t>(v[3], kBf16, r, K);
    const uint16_t* B = a.at2<uint16_t>(v[4], kBf16, N, r);
    const float s = a.real(v[5]);
    hydra_dtype dt;
    void* dx = a.any2(v[7], M, K, dt);
    float* dA = a.at2<float>(v[8], kF32, r, K);
    float* dB = a.at2<float>(v[9], kF32, N, r);
    const double p = a.number(v[10]);
    const uint64_t* rng = a.at1<uint64_t>(v[11], kI64, 2);
    size_t bytes = 0;
    void* w = a.workspace(v[12], bytes);
    void* st = a.stream_here(v[13]);
    return [=]() {
      return hydra_fp8_lora_linear_backward(x, W, ws, A, B, s, dy, M, N, K, r, p, rng, dx, dt, dA, dB, w, bytes, st);
    };
  });
}

// x y p rng residual stream
HYDRA_PY(dropout, 6) {
  return guarded([&](Take& a) {
    const at::Tensor* x = a.tensor(v[0], kAny);
    const at::Tensor* y = a.tensor(v[1], kAny);
    const double p = a.number(v[2]);
    const uint64_t* rng = a.at1<uint64_t>(v[3], kI64, 2);
    const at::Tensor* res = a.tensor(v[4], kAny);
    a.ok = a.ok && x && y && y->sizes() == x->sizes() && (!res || res->sizes() == x->sizes());
    const void* xp = a.ok ? x->data_ptr() : nullptr;
    void* yp = a.ok ? y->data_ptr() : nullptr;
    const void* rp = a.ok && res ? res->data_ptr() : nullptr;
    const int64_t n = a.ok ? x->numel() : 0;
    const hydra_dtype xt = Take::type_of(x), yt = Take::type_of(y), rt = Take::type_of(res);
    void* st = a.stream_here(v[5]);
    return [=]() { return hydra_dropout(xp, xt, rp, rt, p, rng, n, yp, yt, st); };
  });
}

// target draft drafts u accepted tokens lp lens temperature workspace err_flag stream
HYDRA_PY(verify_drafts, 12) {
  return guarded([&](Take& a) {
    int64_t Mt = 0, V = 0, ld = 0, Md = 0, Vd = 0, ld_d = 0;
    hydra_dtype zt = HYDRA_BF16, dt = HYDRA_BF16;
    const void* z = a.rows_of(v[0], Mt, V, zt, ld);
    const at::Tensor* u = a.tensor(v[3], kF32);
    a.ok = a.ok && u && u->dim() == 2 && u->size(1) >= 1;
    const int64_t n = a.ok ? u->size(0) : 0, k = a.ok ? u->size(1) - 1 : 0;
    const void* zd = nullptr;
    if (a.ok && v[1] != Py_None) {
      zd = a.rows_of(v[1], Md, Vd, dt, ld_d);
      a.ok = a.ok && Md == n * k && Vd == V;
    }
    a.ok = a.ok && Mt == n * (k + 1);
    const float* up = a.at2<float>(v[3], kF32, n, k + 1);
    const int32_t* drafts = a.at2<int32_t>(v[2], kI32, n, k);
    int32_t* accepted = a.at1<int32_t>(v[4], kI32, n);
    int32_t* tokens = a.at2<int32_t>(v[5], kI32, n, k + 1);
    float* lp = a.at2<float>(v[6], kF32, n, k + 1);
    const int32_t* lens = a.at1<int32_t>(v[7], kI32, n);
    const double temperature = a.number(v[8]);
    size_t bytes = 0;
    void* w = a.workspace(v[9], bytes);
    int32_t* err = a.at1<int32_t>(v[10], kI32, 1);
    void* st = a.stream_here(v[11]);
    return [=]() {
      return hydra_verify_drafts(z, zt, ld, zd, dt, ld_d, drafts, lens, up, n, k, V, temperature, accepted, tokens, lp, w,
                                 bytes, err, st);
    };
  });
}

#define HYDRA_DEF(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {HYDRA_DEF(lora_linear),  HYDRA_DEF(lora_linear_group), HYDRA_DEF(lora_linear_multi),
                         HYDRA_DEF(score),        HYDRA_DEF(score_logits),      HYDRA_DEF(value_head),
                         HYDRA_DEF(ppo_advantages), HYDRA_DEF(ppo_loss),        HYDRA_DEF(lora_linear_backward),
                         HYDRA_DEF(layer_norm),   HYDRA_DEF(layer_norm_backward), HYDRA_DEF(token_logprobs),
                         HYDRA_DEF(token_logprobs_backward), HYDRA_DEF(grad_clip),
                         HYDRA_DEF(fp8_quantize), HYDRA_DEF(fp8_lora_linear), HYDRA_DEF(fp8_lora_linear_backward),
                         HYDRA_DEF(dropout),      HYDRA_DEF(verify_drafts),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_hydra_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__hydra_native() {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddIntConstant(m, "SLOW", kSlow) != 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}

// The calls on rows (rotary positions, norms of rows, token log probabilities,
// embedding, log probabilities from hidden rows, distillation) on torch tensors, as
// functions of a Python module.
//
// A small call's time is its binding's: looked at from Python, the tensors of
// one call cost 5 us and its ctypes arguments 2 more, where the GPU takes 4.
// Here it is 1 to 2.  Tensors are taken through their Python attributes
// (dtype, shape, stride(), data_ptr(), get_device()), so this depends on no
// torch header or library.
//
// What a call cannot describe (types, shapes, strides, places) raises TypeError
// or ValueError before an address is taken; what the C ABI refuses raises
// NspError.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <hip/hip_runtime_api.h>

#include <string>

#include "nsp.h"

namespace {

// Python objects that every call needs; set up with the module, never freed.
PyObject *g_bf16, *g_f32, *g_f64, *g_i64, *g_error, *g_raw_stream;
PyObject *s_dtype, *s_shape, *s_stride, *s_data_ptr, *s_get_device, *s_numel, *s_is_contiguous, *s_element_size, *s_cuda_stream, *s_device_index;

struct Failed {};   // a Python error is set

[[noreturn]] void fail(PyObject *type, const std::string &text) {
  PyErr_SetString(type, text.c_str());
  throw Failed();
}

struct Ref {
  PyObject *o;
  explicit Ref(PyObject *p) : o(p) {
    if (!p) throw Failed();
  }
  Ref(const Ref &) = delete;
  Ref &operator=(const Ref &) = delete;
  ~Ref() { Py_DECREF(o); }
};

long long number(PyObject *o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Failed();
  return v;
}

long long ask(PyObject *t, PyObject *method) {
  Ref r(PyObject_CallMethodNoArgs(t, method));
  return number(r.o);
}

std::string text(PyObject *o) {
  PyObject *r = o ? PyObject_Str(o) : nullptr;
  const char *c = r ? PyUnicode_AsUTF8(r) : nullptr;
  std::string s = c ? c : "?";
  Py_XDECREF(r);
  if (PyErr_Occurred()) PyErr_Clear();
  return s;
}

std::string shown(PyObject *t) {   // a tensor's type, shape and strides
  PyObject *d = PyObject_GetAttr(t, s_dtype), *h = PyObject_GetAttr(t, s_shape), *st = PyObject_CallMethodNoArgs(t, s_stride);
  const std::string s = text(d) + " " + text(h) + ", strides " + text(st);
  Py_XDECREF(d);
  Py_XDECREF(h);
  Py_XDECREF(st);
  return s;
}

struct Dims {
  int n = 0;
  long long d[3] = {0, 0, 0};
  bool operator==(const Dims &o) const { return n == o.n && d[0] == o.d[0] && d[1] == o.d[1] && d[2] == o.d[2]; }
  std::string str() const {
    std::string s = "(";
    for (int i = 0; i < n; ++i) s += (i ? ", " : "") + std::to_string(d[i]);
    return s + ")";
  }
};

// A tuple of up to three numbers (more: n is 4).
Dims dims_of(PyObject *tuple) {
  Dims r;
  const Py_ssize_t n = PyTuple_Check(tuple) ? PyTuple_GET_SIZE(tuple) : 4;
  r.n = (int)(n > 3 ? 4 : n);
  for (int i = 0; i < r.n && r.n <= 3; ++i) r.d[i] = number(PyTuple_GET_ITEM(tuple, i));
  return r;
}

bool has(PyObject *o) { return o && o != Py_None; }

void need(PyObject *t, const char *name) {
  if (!has(t)) fail(PyExc_TypeError, std::string(name) + ": a tensor is needed");
}

PyObject *dtype_of(PyObject *t, const char *name) {   // borrowed: the types live as long as torch
  need(t, name);
  PyObject *d = PyObject_GetAttr(t, s_dtype);
  if (!d) {
    PyErr_Clear();
    fail(PyExc_TypeError, std::string(name) + ": a tensor is needed");
  }
  Py_DECREF(d);
  return d;
}

nsp_dtype code(PyObject *dtype, const char *name) {
  if (dtype == g_bf16) return NSP_BF16;
  if (dtype == g_f32) return NSP_F32;
  fail(PyExc_TypeError, std::string(name) + ": unsupported dtype " + text(dtype) + " (bfloat16 or float32)");
}

Dims shape_of(PyObject *t) {
  Ref s(PyObject_GetAttr(t, s_shape));
  return dims_of(s.o);
}

// The GPU of a call's tensors (-1: none, which `launch` refuses at the end).
struct Place {
  int dev = -1;
  bool known = false;
  void add(PyObject *t, const char *name) {
    const int d = (int)ask(t, s_get_device);
    if (known && d != dev)
      fail(PyExc_TypeError, std::string(name) + ": a tensor on " + (d < 0 ? std::string("the host") : "GPU " + std::to_string(d)) + ", others on " +
                                (dev < 0 ? std::string("the host") : "GPU " + std::to_string(dev)));
    dev = d;
    known = true;
  }
};

// A [tokens, n] or [tokens, heads, n] tensor.
nsp_rows rows(PyObject *t, const Dims &shape, PyObject *dtype, Place &at, const char *name) {
  if (dtype_of(t, name) != dtype || !(shape_of(t) == shape))
    fail(PyExc_TypeError, std::string(name) + ": " + text(dtype) + " " + shape.str() + " is needed (got " + shown(t) + ")");
  at.add(t, name);
  Ref st(PyObject_CallMethodNoArgs(t, s_stride));
  const Dims s = dims_of(st.o);
  if (s.d[shape.n - 1] != 1 && shape.d[shape.n - 1] > 1)
    fail(PyExc_ValueError, std::string(name) + ": a row's elements must be contiguous (strides " + s.str() + ")");
  return nsp_rows{reinterpret_cast<void *>(ask(t, s_data_ptr)), s.d[0], shape.n == 3 ? s.d[1] : 0};
}

// The address of n contiguous elements; null for an argument left out.
void *array(PyObject *t, long long n, PyObject *dtype, Place &at, const char *name) {
  if (!has(t)) return nullptr;
  if (dtype_of(t, name) != dtype || ask(t, s_numel) != n || !ask(t, s_is_contiguous))
    fail(PyExc_TypeError, std::string(name) + ": " + std::to_string(n) + " contiguous elements of " + text(dtype) + " are needed (got " + shown(t) + ")");
  at.add(t, name);
  return reinterpret_cast<void *>(ask(t, s_data_ptr));
}

struct Workspace {
  void *data = nullptr;
  size_t bytes = 0;
  Workspace(PyObject *t, Place &at) {
    if (!has(t)) return;
    dtype_of(t, "workspace");
    if (!ask(t, s_is_contiguous)) fail(PyExc_TypeError, "workspace: contiguous memory is needed");
    at.add(t, "workspace");
    data = reinterpret_cast<void *>(ask(t, s_data_ptr));
    bytes = (size_t)(ask(t, s_numel) * ask(t, s_element_size));
  }
};

float real(PyObject *o, float none) {
  if (!o) return none;
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Failed();
  return (float)v;
}

int whole(PyObject *o, int none, const char *name) {
  if (!o) return none;
  const long long v = number(o);
  if (v != (int)v) fail(PyExc_ValueError, std::string(name) + ": " + std::to_string(v) + " is past 32 bits");
  return (int)v;
}

// call(stream) with the tensors' GPU current, on `stream` (None: that GPU's current
// one; a Stream of another GPU is refused, a handle is taken as it is).
template <class F>
PyObject *launch(const char *name, const Place &at, PyObject *stream, F call) {
  if (at.dev < 0) fail(PyExc_TypeError, std::string(name) + ": tensors must be on the GPU");
  hipStream_t s;
  if (has(stream)) {
    if (PyLong_Check(stream)) {
      s = reinterpret_cast<hipStream_t>(number(stream));
    } else {
      Ref h(PyObject_GetAttr(stream, s_cuda_stream));
      s = reinterpret_cast<hipStream_t>(number(h.o));
      PyObject *d = PyObject_GetAttr(stream, s_device_index);
      if (d) {
        Ref r(d);
        if (number(d) != at.dev)
          fail(PyExc_ValueError, "stream: of GPU " + std::to_string(number(d)) + ", the tensors are on GPU " + std::to_string(at.dev));
      } else {
        PyErr_Clear();
      }
    }
  } else {
    Ref dev(PyLong_FromLong(at.dev));
    Ref h(PyObject_CallOneArg(g_raw_stream, dev.o));
    s = reinterpret_cast<hipStream_t>(number(h.o));
  }
  int before = at.dev;
  (void)hipGetDevice(&before);
  if (before != at.dev && hipSetDevice(at.dev) != hipSuccess) fail(PyExc_RuntimeError, std::string(name) + ": hipSetDevice failed");
  const nsp_status st = call(s);
  if (before != at.dev) (void)hipSetDevice(before);
  if (st != NSP_OK) {
    Ref e(PyObject_CallFunction(g_error, "iss", (int)st, name, nsp_last_error()));
    PyErr_SetObject(g_error, e.o);
    throw Failed();
  }
  Py_RETURN_NONE;
}

// A function's parameters by name, the first `required` of them without a default.
struct Signature {
  const char *function;
  int required, n;
  const char *names[13];
  PyObject *interned[13];
};

void bind(const Signature &f, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames, PyObject **out) {
  if (nargs > f.n) fail(PyExc_TypeError, std::string(f.function) + "() takes at most " + std::to_string(f.n) + " arguments");
  for (int i = 0; i < f.n; ++i) out[i] = i < nargs ? args[i] : nullptr;
  const Py_ssize_t nkw = kwnames ? PyTuple_GET_SIZE(kwnames) : 0;
  for (Py_ssize_t k = 0; k < nkw; ++k) {
    PyObject *key = PyTuple_GET_ITEM(kwnames, k);
    int i = 0;
    while (i < f.n && f.interned[i] != key) ++i;
    if (i == f.n)
      for (i = 0; i < f.n && PyUnicode_Compare(f.interned[i], key) != 0;) ++i;
    if (i == f.n) fail(PyExc_TypeError, std::string(f.function) + "() got an unexpected argument '" + text(key) + "'");
    if (out[i]) fail(PyExc_TypeError, std::string(f.function) + "() got '" + f.names[i] + "' twice");
    out[i] = args[nargs + k];
  }
  for (int i = 0; i < f.required; ++i)
    if (!out[i]) fail(PyExc_TypeError, std::string(f.function) + "() misses '" + f.names[i] + "'");
}

Signature k_rotary_fwd = {"nsp_rotary_fwd", 4, 9, {"positions", "freqs", "q", "q_out", "k", "k_out", "scale", "layout", "stream"}, {}};
Signature k_rotary_bwd = {"nsp_rotary_bwd", 4, 9, {"positions", "freqs", "dq_out", "dq", "dk_out", "dk", "scale", "layout", "stream"}, {}};
Signature k_norm_fwd = {"nsp_norm_fwd", 4, 9, {"x", "weight", "bias", "y", "mean", "rstd", "eps", "kind", "stream"}, {}};
Signature k_norm_bwd = {"nsp_norm_bwd", 9, 11,
                        {"x", "weight", "dy", "mean", "rstd", "dx", "dweight", "dbias", "workspace", "kind", "stream"}, {}};
Signature k_logp_fwd = {"nsp_token_logp_fwd", 4, 10,
                        {"logits", "targets", "logp", "lse", "entropy", "top_logp", "top_index", "workspace", "scale", "stream"}, {}};
Signature k_logp_bwd = {"nsp_token_logp_bwd", 4, 10,
                        {"logits", "targets", "lse", "dlogits", "g_logp", "g_entropy", "entropy", "g_lse", "scale", "stream"}, {}};
Signature k_linear_fwd = {"nsp_linear_logp_fwd", 5, 9,
                          {"x", "weight", "targets", "logp", "lse", "entropy", "workspace", "scale", "stream"}, {}};
Signature k_linear_bwd = {"nsp_linear_logp_bwd", 7, 13,
                          {"x", "weight", "targets", "lse", "dx", "dweight", "workspace", "g_logp", "g_entropy", "entropy", "g_lse", "scale", "stream"},
                          {}};
Signature k_distill_fwd = {"nsp_distill_fwd", 5, 9,
                           {"logits", "index", "teacher_logp", "loss", "lse", "workspace", "kind", "scale", "stream"}, {}};
Signature k_distill_bwd = {"nsp_distill_bwd", 6, 9,
                           {"logits", "index", "teacher_logp", "lse", "g_loss", "dlogits", "kind", "scale", "stream"}, {}};
Signature k_embed_fwd = {"nsp_embedding_fwd", 3, 5, {"tokens", "weight", "y", "scale", "stream"}, {}};
Signature k_embed_bwd = {"nsp_embedding_bwd", 4, 6, {"tokens", "dy", "dweight", "workspace", "scale", "stream"}, {}};

PyObject *rotary(const Signature &f, bool bwd, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) {
  PyObject *a[9];
  bind(f, args, nargs, kwnames, a);
  const char *const *nm = f.names + 2;
  PyObject *dtype = dtype_of(a[2], nm[0]);
  const Dims d = shape_of(a[2]);
  if (d.n != 3) fail(PyExc_TypeError, std::string(nm[0]) + ": [tokens, heads, head_dim] is needed (got " + shown(a[2]) + ")");
  Place at;
  const nsp_rows q = rows(a[2], d, dtype, at, nm[0]), qo = rows(a[3], d, dtype, at, nm[1]);
  nsp_rows k{}, ko{};
  Dims dk = d;
  dk.d[1] = 0;
  if (has(a[4]) || has(a[5])) {
    if (!has(a[4]) || !has(a[5])) fail(PyExc_TypeError, std::string(nm[2]) + " and " + nm[3] + ": both are needed, or neither");
    dtype_of(a[4], nm[2]);
    const Dims s = shape_of(a[4]);
    if (s.n != 3) fail(PyExc_TypeError, std::string(nm[2]) + ": [tokens, heads, head_dim] is needed (got " + shown(a[4]) + ")");
    dk.d[1] = s.d[1];
    k = rows(a[4], dk, dtype, at, nm[2]);
    ko = rows(a[5], dk, dtype, at, nm[3]);
  }
  need(a[0], "positions");
  need(a[1], "freqs");
  dtype_of(a[1], "freqs");
  const long long half = ask(a[1], s_numel);
  const auto *pos = static_cast<const int64_t *>(array(a[0], d.d[0], g_i64, at, "positions"));
  const auto *freqs = static_cast<const double *>(array(a[1], half, g_f64, at, "freqs"));
  const nsp_dtype c = code(dtype, nm[0]);
  const float scale = real(a[6], 1.f);
  const auto layout = (nsp_rotary_layout)whole(a[7], NSP_ROTARY_HALF, "layout");
  if (d.d[1] > INT32_MAX || dk.d[1] > INT32_MAX || d.d[2] > INT32_MAX || half > INT32_MAX / 2) fail(PyExc_ValueError, "sizes past 2^31 - 1");
  const bool keys = dk.d[1] > 0;
  return launch(f.function, at, a[8], [&](hipStream_t s) {
    return (bwd ? nsp_rotary_bwd : nsp_rotary_fwd)(layout, c, d.d[0], (int32_t)d.d[2], (int32_t)(2 * half), freqs, scale, pos, (int32_t)d.d[1], &q,
                                                   &qo, (int32_t)dk.d[1], keys ? &k : nullptr, keys ? &ko : nullptr, s);
  });
}

struct NormSizes {
  Dims shape;
  long long T, H, n;
  PyObject *dtype;
  explicit NormSizes(PyObject *x) : dtype(dtype_of(x, "x")) {
    shape = shape_of(x);
    if (shape.n != 2 && shape.n != 3) fail(PyExc_TypeError, "x: [tokens, n] or [tokens, heads, n] is needed (got " + shown(x) + ")");
    T = shape.d[0];
    H = shape.n == 3 ? shape.d[1] : 1;
    n = shape.d[shape.n - 1];
    if (H > INT32_MAX || n > INT32_MAX) fail(PyExc_ValueError, "x: sizes past 2^31 - 1");
  }
};

PyObject *norm_fwd(PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) {
  PyObject *a[9];
  bind(k_norm_fwd, args, nargs, kwnames, a);
  const NormSizes z(a[0]);
  PyObject *wd = has(a[1]) ? dtype_of(a[1], "weight") : has(a[2]) ? dtype_of(a[2], "bias") : z.dtype;
  Place at;
  const nsp_rows x = rows(a[0], z.shape, z.dtype, at, "x"), y = rows(a[3], z.shape, z.dtype, at, "y");
  const void *w = array(a[1], z.n, wd, at, "weight"), *b = array(a[2], z.n, wd, at, "bias");
  auto *mean = static_cast<float *>(array(a[4], z.T * z.H, g_f32, at, "mean")), *rstd = static_cast<float *>(array(a[5], z.T * z.H, g_f32, at, "rstd"));
  const nsp_dtype c = code(z.dtype, "x"), cw = code(wd, "weight");
  const float eps = real(a[6], 1e-6f);
  const auto kind = (nsp_norm_kind)whole(a[7], NSP_NORM_LAYER, "kind");
  return launch("nsp_norm_fwd", at, a[8], [&](hipStream_t s) {
    return nsp_norm_fwd(kind, c, cw, z.T, (int32_t)z.H, (int32_t)z.n, &x, w, b, eps, &y, mean, rstd, s);
  });
}

PyObject *norm_bwd(PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) {
  PyObject *a[11];
  bind(k_norm_bwd, args, nargs, kwnames, a);
  const NormSizes z(a[0]);
  PyObject *wd = z.dtype;
  for (const int i : {1, 6, 7})
    if (has(a[i])) {
      wd = dtype_of(a[i], k_norm_bwd.names[i]);
      break;
    }
  Place at;
  const nsp_rows x = rows(a[0], z.shape, z.dtype, at, "x"), dy = rows(a[2], z.shape, z.dtype, at, "dy"),
                 dx = rows(a[5], z.shape, z.dtype, at, "dx");
  const void *w = array(a[1], z.n, wd, at, "weight");
  const auto *mean = static_cast<const float *>(array(a[3], z.T * z.H, g_f32, at, "mean")),
             *rstd = static_cast<const float *>(array(a[4], z.T * z.H, g_f32, at, "rstd"));
  void *dw = array(a[6], z.n, wd, at, "dweight"), *db = array(a[7], z.n, wd, at, "dbias");
  const Workspace ws(a[8], at);
  const nsp_dtype c = code(z.dtype, "x"), cw = code(wd, "weight");
  const auto kind = (nsp_norm_kind)whole(a[9], NSP_NORM_LAYER, "kind");
  return launch("nsp_norm_bwd", at, a[10], [&](hipStream_t s) {
    return nsp_norm_bwd(kind, c, cw, z.T, (int32_t)z.H, (int32_t)z.n, &x, w, &dy, mean, rstd, &dx, dw, db, ws.data, ws.bytes, s);
  });
}

struct LogitSizes {
  Dims shape;
  PyObject *dtype;
  explicit LogitSizes(PyObject *t) : dtype(dtype_of(t, "logits")) {
    shape = shape_of(t);
    if (shape.n != 2) fail(PyExc_TypeError, "logits: [tokens, vocab] is needed (got " + shown(t) + ")");
    if (shape.d[1] > INT32_MAX) fail(PyExc_ValueError, "logits: sizes past 2^31 - 1");
  }
};

PyObject *logp_fwd(PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) {
  PyObject *a[10];
  bind(k_logp_fwd, args, nargs, kwnames, a);
  const LogitSizes z(a[0]);
  const long long T = z.shape.d[0];
  Place at;
  const nsp_rows x = rows(a[0], z.shape, z.dtype, at, "logits");
  long long k = 0;
  if (has(a[5]) || has(a[6])) {
    if (!has(a[5]) || !has(a[6])) fail(PyExc_TypeError, "top_logp and top_index: both are needed, or neither");
    dtype_of(a[5], "top_logp");
    const Dims d = shape_of(a[5]);
    if (d.n != 2 || d.d[0] != T) fail(PyExc_TypeError, "top_logp: [tokens, top] is needed (got " + shown(a[5]) + ")");
    k = d.d[1];
  }
  need(a[3], "lse");
  const auto *y = static_cast<const int64_t *>(array(a[1], T, g_i64, at, "targets"));
  auto *logp = static_cast<float *>(array(a[2], T, g_f32, at, "logp")), *lse = static_cast<float *>(array(a[3], T, g_f32, at, "lse")),
       *ent = static_cast<float *>(array(a[4], T, g_f32, at, "entropy")), *tl = static_cast<float *>(array(a[5], T * k, g_f32, at, "top_logp"));
  auto *ti = static_cast<int64_t *>(array(a[6], T * k, g_i64, at, "top_index"));
  const Workspace ws(a[7], at);
  const nsp_dtype c = code(z.dtype, "logits");
  const float scale = real(a[8], 1.f);
  if (k > INT32_MAX) fail(PyExc_ValueError, "top_logp: sizes past 2^31 - 1");
  return launch("nsp_token_logp_fwd", at, a[9], [&](hipStream_t s) {
    return nsp_token_logp_fwd(c, T, (int32_t)z.shape.d[1], x.data, x.token_stride, y, scale, logp, lse, ent, (int32_t)k, tl, ti, ws.data, ws.bytes, s);
  });
}

PyObject *logp_bwd(PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) {
  PyObject *a[10];
  bind(k_logp_bwd, args, nargs, kwnames, a);
  const LogitSizes z(a[0]);
  const long long T = z.shape.d[0];
  Place at;
  const nsp_rows x = rows(a[0], z.shape, z.dtype, at, "logits"), d = rows(a[3], z.shape, z.dtype, at, "dlogits");
  need(a[2], "lse");
  const auto *y = static_cast<const int64_t *>(array(a[1], T, g_i64, at, "targets"));
  const auto f = [&](int i) { return static_cast<const float *>(array(a[i], T, g_f32, at, k_logp_bwd.names[i])); };
  const float *lse = f(2), *gl = f(4), *ge = f(5), *ent = f(6), *gs = f(7);
  const nsp_dtype c = code(z.dtype, "logits");
  const float scale = real(a[8], 1.f);
  return launch("nsp_token_logp_bwd", at, a[9], [&](hipStream_t s) {
    return nsp_token_logp_bwd(c, T, (int32_t)z.shape.d[1], x.data, x.token_stride, y, scale, lse, ent, gl, gs, ge, d.data, d.token_stride, s);
  });
}

// A [rows, dim] tensor's sizes and type.
struct Matrix {
  Dims shape;
  PyObject *dtype;
  Matrix(PyObject *t, const char *name, const char *wanted) : dtype(dtype_of(t, name)) {
    shape = shape_of(t);
    if (shape.n != 2) fail(PyExc_TypeError, std::string(name) + ": " + wanted + " is needed (got " + shown(t) + ")");
    if (shape.d[1] > INT32_MAX) fail(PyExc_ValueError, std::string(name) + ": sizes past 2^31 - 1");
  }
};

// Hidden rows and the vocabulary's weight.
struct LinearSizes {
  Matrix x, w;
  nsp_rows rx, rw;
  LinearSizes(PyObject *tx, PyObject *tw, Place &at) : x(tx, "x", "[tokens, dim]"), w(tw, "weight", "[vocab, dim]") {
    if (w.shape.d[1] != x.shape.d[1] || w.shape.d[0] > INT32_MAX)
      fail(PyExc_TypeError, "weight: [vocab, " + std::to_string(x.shape.d[1]) + "] is needed (got " + shown(tw) + ")");
    rx = rows(tx, x.shape, g_bf16, at, "x");
    rw = rows(tw, w.shape, g_bf16, at, "weight");
  }
  long long tokens() const { return x.shape.d[0]; }
  int32_t dim() const { return (int32_t)x.shape.d[1]; }
  int32_t vocab() const { return (int32_t)w.shape.d[0]; }
};

PyObject *linear_fwd(PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) {
  PyObject *a[9];
  bind(k_linear_fwd, args, nargs, kwnames, a);
  Place at;
  const LinearSizes z(a[0], a[1], at);
  const long long T = z.tokens();
  need(a[4], "lse");
  const auto *y = static_cast<const int64_t *>(array(a[2], T, g_i64, at, "targets"));
  auto *logp = static_cast<float *>(array(a[3], T, g_f32, at, "logp")), *lse = static_cast<float *>(array(a[4], T, g_f32, at, "lse")),
       *ent = static_cast<float *>(array(a[5], T, g_f32, at, "entropy"));
  const Workspace ws(a[6], at);
  const float scale = real(a[7], 1.f);
  return launch("nsp_linear_logp_fwd", at, a[8], [&](hipStream_t s) {
    return nsp_linear_logp_fwd(T, z.dim(), z.vocab(), &z.rx, &z.rw, y, scale, logp, lse, ent, ws.data, ws.bytes, s);
  });
}

PyObject *linear_bwd(PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) {
  PyObject *a[13];
  bind(k_linear_bwd, args, nargs, kwnames, a);
  Place at;
  const LinearSizes z(a[0], a[1], at);
  const long long T = z.tokens();
  need(a[3], "lse");
  const auto *y = static_cast<const int64_t *>(array(a[2], T, g_i64, at, "targets"));
  const auto f = [&](int i) { return static_cast<const float *>(array(a[i], T, g_f32, at, k_linear_bwd.names[i])); };
  const float *lse = f(3), *gl = f(7), *ge = f(8), *ent = f(9), *gs = f(10);
  PyObject *gd = has(a[4]) ? dtype_of(a[4], "dx") : has(a[5]) ? dtype_of(a[5], "dweight") : g_bf16;
  nsp_rows dx{}, dw{};
  if (has(a[4])) dx = rows(a[4], z.x.shape, gd, at, "dx");
  if (has(a[5])) dw = rows(a[5], z.w.shape, gd, at, "dweight");
  const Workspace ws(a[6], at);
  const nsp_dtype c = code(gd, "dx");
  const float scale = real(a[11], 1.f);
  return launch("nsp_linear_logp_bwd", at, a[12], [&](hipStream_t s) {
    return nsp_linear_logp_bwd(c, T, z.dim(), z.vocab(), &z.rx, &z.rw, y, scale, lse, ent, gl, gs, ge, has(a[4]) ? &dx : nullptr,
                               has(a[5]) ? &dw : nullptr, ws.data, ws.bytes, s);
  });
}

// A teacher's alternatives: their number a token.
long long alternatives(PyObject *index, long long T) {
  const Matrix m(index, "index", "[tokens, top]");
  if (m.shape.d[0] != T) fail(PyExc_TypeError, "index: [" + std::to_string(T) + ", top] is needed (got " + shown(index) + ")");
  return m.shape.d[1];
}

PyObject *distill_fwd(PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) {
  PyObject *a[9];
  bind(k_distill_fwd, args, nargs, kwnames, a);
  const LogitSizes z(a[0]);
  const long long T = z.shape.d[0];
  Place at;
  const nsp_rows x = rows(a[0], z.shape, z.dtype, at, "logits");
  const long long k = alternatives(a[1], T);
  need(a[2], "teacher_logp");
  need(a[4], "lse");
  const auto *index = static_cast<const int64_t *>(array(a[1], T * k, g_i64, at, "index"));
  const auto *teacher = static_cast<const float *>(array(a[2], T * k, g_f32, at, "teacher_logp"));
  auto *loss = static_cast<float *>(array(a[3], T, g_f32, at, "loss")), *lse = static_cast<float *>(array(a[4], T, g_f32, at, "lse"));
  const Workspace ws(a[5], at);
  const nsp_dtype c = code(z.dtype, "logits");
  const auto kind = (nsp_distill_kind)whole(a[6], NSP_DISTILL_GIVEN, "kind");
  const float scale = real(a[7], 1.f);
  return launch("nsp_distill_fwd", at, a[8], [&](hipStream_t s) {
    return nsp_distill_fwd(c, T, (int32_t)z.shape.d[1], x.data, x.token_stride, (int32_t)k, index, teacher, kind, scale, loss, lse, ws.data, ws.bytes, s);
  });
}

PyObject *distill_bwd(PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) {
  PyObject *a[9];
  bind(k_distill_bwd, args, nargs, kwnames, a);
  const LogitSizes z(a[0]);
  const long long T = z.shape.d[0];
  Place at;
  const nsp_rows x = rows(a[0], z.shape, z.dtype, at, "logits"), d = rows(a[5], z.shape, z.dtype, at, "dlogits");
  const long long k = alternatives(a[1], T);
  need(a[2], "teacher_logp");
  need(a[3], "lse");
  need(a[4], "g_loss");
  const auto *index = static_cast<const int64_t *>(array(a[1], T * k, g_i64, at, "index"));
  const auto f = [&](int i, long long n) { return static_cast<const float *>(array(a[i], n, g_f32, at, k_distill_bwd.names[i])); };
  const float *teacher = f(2, T * k), *lse = f(3, T), *g = f(4, T);
  const nsp_dtype c = code(z.dtype, "logits");
  const auto kind = (nsp_distill_kind)whole(a[6], NSP_DISTILL_GIVEN, "kind");
  const float scale = real(a[7], 1.f);
  return launch("nsp_distill_bwd", at, a[8], [&](hipStream_t s) {
    return nsp_distill_bwd(c, T, (int32_t)z.shape.d[1], x.data, x.token_stride, (int32_t)k, index, teacher, kind, scale, lse, g, d.data,
                           d.token_stride, s);
  });
}

// tokens, table rows, the tokens' rows
PyObject *embedding(const Signature &f, bool bwd, PyObject *tokens, PyObject *table, PyObject *out, PyObject *workspace, PyObject *scaling,
                    PyObject *stream) {
  const char *const table_name = bwd ? "dweight" : "weight", *const out_name = bwd ? "dy" : "y";
  const Matrix w(table, table_name, "[vocab, dim]"), y(out, out_name, "[tokens, dim]");
  const long long T = y.shape.d[0];
  if (w.shape.d[1] != y.shape.d[1] || w.shape.d[0] > INT32_MAX)
    fail(PyExc_TypeError, std::string(table_name) + ": [vocab, " + std::to_string(y.shape.d[1]) + "] is needed (got " + shown(table) + ")");
  Place at;
  const nsp_rows rw = rows(table, w.shape, w.dtype, at, table_name), ry = rows(out, y.shape, y.dtype, at, out_name);
  need(tokens, "tokens");
  const auto *ids = static_cast<const int64_t *>(array(tokens, T, g_i64, at, "tokens"));
  const Workspace ws(workspace, at);
  const nsp_dtype cw = code(w.dtype, table_name), cy = code(y.dtype, out_name);
  const float scale = real(scaling, 1.f);
  const int32_t dim = (int32_t)w.shape.d[1], vocab = (int32_t)w.shape.d[0];
  return launch(f.function, at, stream, [&](hipStream_t s) {
    return bwd ? nsp_embedding_bwd(cw, cy, T, dim, vocab, ids, &ry, scale, &rw, ws.data, ws.bytes, s)
               : nsp_embedding_fwd(cw, cy, T, dim, vocab, ids, &rw, scale, &ry, s);
  });
}

PyObject *embed_fwd(PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) {
  PyObject *a[5];
  bind(k_embed_fwd, args, nargs, kwnames, a);
  return embedding(k_embed_fwd, false, a[0], a[1], a[2], nullptr, a[3], a[4]);
}

PyObject *embed_bwd(PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) {
  PyObject *a[6];
  bind(k_embed_bwd, args, nargs, kwnames, a);
  return embedding(k_embed_bwd, true, a[0], a[2], a[1], a[3], a[4], a[5]);
}

// No C++ exception leaves the module.
template <class F>
PyObject *guarded(F f) {
  try {
    return f();
  } catch (const Failed &) {
    return nullptr;
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

#define FUNCTION(name, expr)                                                                             \
  PyObject *py_##name(PyObject *, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) {          \
    return guarded([&] { return expr; });                                                                \
  }
FUNCTION(rotary_fwd, rotary(k_rotary_fwd, false, args, nargs, kwnames))
FUNCTION(rotary_bwd, rotary(k_rotary_bwd, true, args, nargs, kwnames))
FUNCTION(norm_fwd, norm_fwd(args, nargs, kwnames))
FUNCTION(norm_bwd, norm_bwd(args, nargs, kwnames))
FUNCTION(logp_fwd, logp_fwd(args, nargs, kwnames))
FUNCTION(logp_bwd, logp_bwd(args, nargs, kwnames))
FUNCTION(linear_fwd, linear_fwd(args, nargs, kwnames))
FUNCTION(linear_bwd, linear_bwd(args, nargs, kwnames))
FUNCTION(distill_fwd, distill_fwd(args, nargs, kwnames))
FUNCTION(distill_bwd, distill_bwd(args, nargs, kwnames))
FUNCTION(embed_fwd, embed_fwd(args, nargs, kwnames))
FUNCTION(embed_bwd, embed_bwd(args, nargs, kwnames))

#define METHOD(name, f, doc) \
  {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL | METH_KEYWORDS, doc}
PyMethodDef g_methods[] = {
    METHOD("nsp_rotary_fwd", py_rotary_fwd,
           "nsp_rotary_fwd(positions, freqs, q, q_out, k=None, k_out=None, scale=1.0, layout=NSP_ROTARY_HALF, stream=None)\n\n"
           "Rotate the query (and key) heads [tokens, heads, head_dim] by their\npositions (int64 [tokens]); freqs: float64 [rot_dim / 2] on the "
           "GPU, as\nnsp_rotary_frequencies gives them.  q_out may be q itself (in place)."),
    METHOD("nsp_rotary_bwd", py_rotary_bwd,
           "nsp_rotary_bwd(positions, freqs, dq_out, dq, dk_out=None, dk=None, scale=1.0, layout=NSP_ROTARY_HALF, stream=None)\n\n"
           "Gradient of nsp_rotary_fwd: dq_out, dk_out into dq, dk (in place allowed)."),
    METHOD("nsp_norm_fwd", py_norm_fwd,
           "nsp_norm_fwd(x, weight, bias, y, mean=None, rstd=None, eps=1e-6, kind=NSP_NORM_LAYER, stream=None)\n\n"
           "Norm of the rows of x ([tokens, n] or [tokens, heads, n]) into y (x\nitself: in place); weight, bias: [n] of one type, or None; mean, "
           "rstd:\nfloat32 [rows], for the backward, or None."),
    METHOD("nsp_norm_bwd", py_norm_bwd,
           "nsp_norm_bwd(x, weight, dy, mean, rstd, dx, dweight, dbias, workspace, kind=NSP_NORM_LAYER, stream=None)\n\n"
           "Gradient of nsp_norm_fwd into dx, and dweight and dbias (of the\nweight's type; None: not computed)."),
    METHOD("nsp_token_logp_fwd", py_logp_fwd,
           "nsp_token_logp_fwd(logits, targets, logp, lse, entropy=None, top_logp=None, top_index=None, workspace=None, scale=1.0, stream=None)\n\n"
           "Log probabilities of the targets (int64 [tokens]; outside the vocabulary:\nignored) under logits [tokens, vocab], with their "
           "log-sum-exp, entropy\n(float32 [tokens]) and the top alternatives ([tokens, top], float32 and\nint64).  Everything but logits and lse "
           "may be None."),
    METHOD("nsp_token_logp_bwd", py_logp_bwd,
           "nsp_token_logp_bwd(logits, targets, lse, dlogits, g_logp=None, g_entropy=None, entropy=None, g_lse=None, scale=1.0, stream=None)\n\n"
           "Gradient of nsp_token_logp_fwd's logp, entropy and lse (float32\n[tokens] each, or None) with respect to the logits, into dlogits (the\n"
           "logits themselves: in place)."),
    METHOD("nsp_linear_logp_fwd", py_linear_fwd,
           "nsp_linear_logp_fwd(x, weight, targets, logp, lse, entropy=None, workspace=None, scale=1.0, stream=None)\n\n"
           "nsp_token_logp_fwd for logits x @ weight.T that are not stored: x bfloat16\n[tokens, dim], weight bfloat16 [vocab, dim]; targets int64 "
           "[tokens] (outside\nthe vocabulary: ignored), logp, lse, entropy float32 [tokens].  targets with\nlogp, and entropy, may be None."),
    METHOD("nsp_linear_logp_bwd", py_linear_bwd,
           "nsp_linear_logp_bwd(x, weight, targets, lse, dx, dweight, workspace, g_logp=None, g_entropy=None, entropy=None, g_lse=None, scale=1.0, "
           "stream=None)\n\n"
           "Gradient of nsp_linear_logp_fwd's logp, entropy and lse (float32 [tokens]\neach, or None) with respect to x and weight, into dx and "
           "dweight (both\nbfloat16 or both float32; None: not computed)."),
    METHOD("nsp_distill_fwd", py_distill_fwd,
           "nsp_distill_fwd(logits, index, teacher_logp, loss, lse, workspace=None, kind=NSP_DISTILL_GIVEN, scale=1.0, stream=None)\n\n"
           "Divergence of the rows of logits [tokens, vocab] from a teacher's top\nalternatives (index int64, teacher_logp float32, [tokens, top], as\n"
           "nsp_token_logp_fwd gives them): loss (or None) and lse, float32 [tokens]."),
    METHOD("nsp_distill_bwd", py_distill_bwd,
           "nsp_distill_bwd(logits, index, teacher_logp, lse, g_loss, dlogits, kind=NSP_DISTILL_GIVEN, scale=1.0, stream=None)\n\n"
           "Gradient of nsp_distill_fwd's loss, times g_loss (float32 [tokens]), with\nrespect to the logits, into dlogits (the logits themselves: in "
           "place)."),
    METHOD("nsp_embedding_fwd", py_embed_fwd,
           "nsp_embedding_fwd(tokens, weight, y, scale=1.0, stream=None)\n\n"
           "Rows of weight [vocab, dim] of the tokens (int64 [tokens]; outside the\nvocabulary: zeros), times scale, into y [tokens, dim]."),
    METHOD("nsp_embedding_bwd", py_embed_bwd,
           "nsp_embedding_bwd(tokens, dy, dweight, workspace, scale=1.0, stream=None)\n\n"
           "Gradient of nsp_embedding_fwd with respect to the table, into dweight\n[vocab, dim] (all rows are written)."),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_rows", "The calls on rows, on torch tensors.", -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__rows() {
  return guarded([]() -> PyObject * {
    for (auto [p, s] : {std::pair{&s_dtype, "dtype"}, {&s_shape, "shape"}, {&s_stride, "stride"}, {&s_data_ptr, "data_ptr"},
                        {&s_get_device, "get_device"}, {&s_numel, "numel"}, {&s_is_contiguous, "is_contiguous"},
                        {&s_element_size, "element_size"}, {&s_cuda_stream, "cuda_stream"}, {&s_device_index, "device_index"}})
      if (!(*p = PyUnicode_InternFromString(s))) throw Failed();
    for (Signature *f : {&k_rotary_fwd, &k_rotary_bwd, &k_norm_fwd, &k_norm_bwd, &k_logp_fwd, &k_logp_bwd, &k_linear_fwd, &k_linear_bwd, &k_distill_fwd, &k_distill_bwd,
                         &k_embed_fwd, &k_embed_bwd})
      for (int i = 0; i < f->n; ++i)
        if (!(f->interned[i] = PyUnicode_InternFromString(f->names[i]))) throw Failed();
    Ref torch(PyImport_ImportModule("torch")), nsp(PyImport_ImportModule("paper_2609_22755_amd.nsp")),
        rows(PyImport_ImportModule("paper_2609_22755_amd.rows"));
    for (auto [p, s] : {std::pair{&g_bf16, "bfloat16"}, {&g_f32, "float32"}, {&g_f64, "float64"}, {&g_i64, "int64"}})
      if (!(*p = PyObject_GetAttrString(torch.o, s))) throw Failed();
    if (!(g_error = PyObject_GetAttrString(nsp.o, "NspError"))) throw Failed();
    if (!(g_raw_stream = PyObject_GetAttrString(rows.o, "raw_stream"))) throw Failed();
    return PyModule_Create(&g_module);
  });
}

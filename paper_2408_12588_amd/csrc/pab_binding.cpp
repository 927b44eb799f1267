// CPython binding of the calls that a denoising loop makes over and over: pab_attention and pab_attention_compute, and around them
// the calls on 8-bit rows and the query / key norm.
//
// Small launches are bound by the host: a reused call, which launches nothing, took 1.75 us from Python, of which the library
// took 0.1: 0.55 for the pointers of three tensors, 0.3 for the stream, 0.45 for ctypes, the rest for the steps in between.
// (With it: a reused call 0.37, an operation of its own 5.8 - 6.2 -> 3.1 - 3.7 with its launch, a run of 60 calls over a tiny model
// 211 - 228 -> 121 - 145, three machines, each without and with it.)
// Here plain torch tensors are looked at through torch's own C++ interface and the library is called directly.  Whatever is not
// a plain dense device tensor or a plain number goes back to the Python code (NotImplemented), which has the same checks and
// raises the errors.
#include <ATen/ops/empty.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/pab.h"

namespace {

PyObject *py_check, *get_device, *get_raw_stream;   // pab._check; torch's functions for the current device and stream, or NULL

// device address of a plain dense device tensor; false: not one
bool plain_address(PyObject *o, void **p) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor &t = THPVariable_Unpack(o);
  if (!t.is_cuda() || !t.is_contiguous()) return false;
  *p = t.data_ptr();
  return true;
}

// ... or an address as such (None: 0)
bool address(PyObject *o, void **p) {
  if (plain_address(o, p)) return true;
  if (o == Py_None) *p = nullptr;
  else if (PyLong_CheckExact(o)) *p = PyLong_AsVoidPtr(o);
  else return false;
  return !PyErr_Occurred();
}

bool integer(PyObject *o, int *v) {
  if (!PyLong_CheckExact(o)) return false;
  *v = (int)PyLong_AsLong(o);
  return !PyErr_Occurred();
}

// handle of the stream argument: an address, or None for torch's current stream where a device tensor shows that torch's device
// side is up
bool stream_of(PyObject *o, bool on_device, void **st) {
  if (PyLong_CheckExact(o)) {
    *st = PyLong_AsVoidPtr(o);
    return !PyErr_Occurred();
  }
  if (o != Py_None || !on_device || !get_raw_stream) return false;
  PyObject *dev = PyObject_CallNoArgs(get_device);
  PyObject *r = dev ? PyObject_CallOneArg(get_raw_stream, dev) : nullptr;
  Py_XDECREF(dev);
  if (!r) return false;
  *st = PyLong_AsVoidPtr(r);
  Py_DECREF(r);
  return !PyErr_Occurred();
}

// what the Python code takes over: anything out of the ordinary, of which it raises the errors
PyObject *not_mine() {
  PyErr_Clear();
  Py_RETURN_NOTIMPLEMENTED;
}

// an error status: pab._check raises it
PyObject *failed(int status) {
  PyObject *r = PyObject_CallFunction(py_check, "i", status);
  Py_XDECREF(r);
  if (r) PyErr_SetString(PyExc_RuntimeError, "libpab failed");
  return nullptr;
}

// C++ exceptions end here: a tensor without storage and the like
template <typename F> PyObject *guarded(F f) {
  try {
    return f();
  } catch (const std::exception &) {
    return not_mine();
  }
}

// attention(context address, block, kind, step, q, k, v, stream) -> (decision, address of the slot or None)
PyObject *attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 8) return PyErr_Format(PyExc_TypeError, "attention takes 8 arguments, not %zd", n);
  return guarded([&]() -> PyObject * {
    void *ctx, *q, *k, *v, *st;
    const void *out = nullptr;
    int block, kind, step;
    if (!address(a[0], &ctx) || !integer(a[1], &block) || !integer(a[2], &kind) || !integer(a[3], &step) || !address(a[4], &q) ||
        !address(a[5], &k) || !address(a[6], &v) || !stream_of(a[7], THPVariable_CheckExact(a[4]), &st))
      return not_mine();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = pab_attention(static_cast<pab_ctx *>(ctx), block, kind, step, q, k, v, st, &out);
    Py_END_ALLOW_THREADS
    if (rc < 0) return failed(rc);
    return out ? Py_BuildValue("(iN)", rc, PyLong_FromVoidPtr(const_cast<void *>(out))) : Py_BuildValue("(iO)", rc, Py_None);
  });
}

// attention_compute(kind, q, k, v, out, stream) -> None
PyObject *attention_compute(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 6) return PyErr_Format(PyExc_TypeError, "attention_compute takes 6 arguments, not %zd", n);
  return guarded([&]() -> PyObject * {
    int kind;
    void *p[4], *st;
    if (!integer(a[0], &kind)) return not_mine();
    for (int i = 0; i < 4; ++i)
      if (!plain_address(a[1 + i], &p[i])) return not_mine();
    const at::Tensor &q = THPVariable_Unpack(a[1]), &k = THPVariable_Unpack(a[2]), &v = THPVariable_Unpack(a[3]);
    const auto type = q.scalar_type();
    if ((type != at::kBFloat16 && type != at::kFloat) || k.scalar_type() != type || v.scalar_type() != type || q.dim() != 4) return not_mine();
    const auto s = q.sizes();
    if (k.sizes() != v.sizes()) return not_mine();
    if (kind == PAB_CROSS ? k.dim() != 3 || k.size(1) != s[2] || k.size(2) != s[3] : k.sizes() != s) return not_mine();
    const int64_t L = kind == PAB_CROSS ? k.size(0) : 0;
    for (int64_t x : {s[0], s[1], s[2], s[3], L})
      if (x > 0x7fffffff) return not_mine();
    if (!stream_of(a[5], true, &st)) return not_mine();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = pab_attention_compute(kind, type == at::kBFloat16 ? PAB_BF16 : PAB_F32, (int)s[0], (int)s[1], (int)L, (int)s[2], (int)s[3], p[0],
                               p[1], p[2], p[3], st);
    Py_END_ALLOW_THREADS
    if (rc < 0) return failed(rc);
    Py_RETURN_NONE;
  });
}

// ---- 8-bit rows and the query / key norm.  The Python code allocates, checks and marshals in 9 to 14 us what the library launches in
//      2.5; the same here, for plain tensors on the current device and its current stream.  Per call with its
//      launch, fp32 or one token: quantise 14.1 -> 8.6 us, read back 10.2 -> 5.3, product 12.0 -> 5.5, query / key norm 17.0 -> 6.0. ----

PyObject *q8_type, *s_data, *s_scale, *s_K;   // pab.Q8 and the names of its fields

const at::Tensor *plain_tensor(PyObject *o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor &t = THPVariable_Unpack(o);
  return t.is_cuda() && t.layout() == at::kStrided ? &t : nullptr;
}

bool float_type(const at::Tensor &t, int *dtype) {
  const auto s = t.scalar_type();
  *dtype = s == at::kBFloat16 ? PAB_BF16 : PAB_F32;
  return s == at::kBFloat16 || s == at::kFloat;
}

// A matrix whose rows are dense and evenly spaced: the leading axes collapse into one row index.  `tail`: axes that make up a row
// (1: the last one, 2: heads and head dim).
bool rows_of(const at::Tensor &t, int tail, long long *rows, long long *pitch) {
  const int n = (int)t.dim();
  if (n < tail) return false;
  long long row = 1;
  for (int i = n - 1; i >= n - tail; --i) {
    if (t.size(i) < 1 || (t.size(i) > 1 && t.stride(i) != row)) return false;
    row *= t.size(i);
  }
  *rows = 1;
  *pitch = row;
  bool first = true;
  for (int i = n - tail - 1; i >= 0; --i) {
    if (t.size(i) < 1) return false;
    if (t.size(i) == 1) continue;
    if (first) *pitch = t.stride(i);
    else if (t.stride(i) != *pitch * *rows) return false;
    first = false;
    *rows *= t.size(i);
  }
  return true;
}

// a dense vector of n values of the given type, or None
bool vector_of(PyObject *o, at::ScalarType type, long long n, int device, const void **p) {
  *p = nullptr;
  if (o == Py_None) return true;
  const at::Tensor *t = plain_tensor(o);
  if (!t || t->scalar_type() != type || t->numel() != n || !t->is_contiguous() || t->get_device() != device) return false;
  *p = t->data_ptr();
  return true;
}

struct Rows {
  pab_q8 q;
  long long rows, K;
  int device;
  at::Tensor like;
};

// whether these tensors hold 8-bit rows of K columns
bool rows_in(const at::Tensor &d, const at::Tensor &s, long long K, Rows *r) {
  const auto dt = d.scalar_type(), st = s.scalar_type();
  if ((dt != at::kByte && dt != at::kFloat8_e4m3fn) || (st != at::kByte && st != at::kFloat8_e8m0fnu) || d.dim() != 2 || s.dim() != 2 ||
      d.size(0) != s.size(0) || d.size(0) < 1 || K < 1 || K > 0x7fffff00 || d.get_device() != s.get_device())
    return false;
  const long long nb = (K + 127) / 128;
  if (d.size(1) < 128 * nb || s.size(1) < nb || d.stride(1) != 1 || s.stride(1) != 1) return false;
  r->q = pab_q8{d.data_ptr(), s.data_ptr(), d.stride(0), s.stride(0)};
  r->rows = d.size(0);
  r->K = K;
  r->device = d.get_device();
  return true;
}

bool q8_of(PyObject *o, Rows *r) {
  if ((PyObject *)Py_TYPE(o) != q8_type) return false;
  PyObject *d = PyObject_GetAttr(o, s_data), *s = PyObject_GetAttr(o, s_scale), *k = PyObject_GetAttr(o, s_K);
  bool ok = d && s && k && PyLong_CheckExact(k);
  if (ok) {   // the object keeps its tensors
    const at::Tensor *td = plain_tensor(d), *ts = plain_tensor(s);
    ok = td && ts && rows_in(*td, *ts, PyLong_AsLongLong(k), r);
    if (ok) r->like = *td;
  }
  Py_XDECREF(d);
  Py_XDECREF(s);
  Py_XDECREF(k);
  return ok && !PyErr_Occurred();
}

// the current device is `device`: its current stream
bool stream_on(PyObject *stream, int device, void **st) {
  if (stream != Py_None || !get_raw_stream) return false;
  PyObject *dev = PyObject_CallNoArgs(get_device);
  const bool same = dev && PyLong_AsLong(dev) == device;
  PyObject *r = same ? PyObject_CallOneArg(get_raw_stream, dev) : nullptr;
  Py_XDECREF(dev);
  if (!r) return false;
  *st = PyLong_AsVoidPtr(r);
  Py_DECREF(r);
  return !PyErr_Occurred();
}

// q8_ok(data, scale, K) -> True for plain tensors that hold such rows
PyObject *q8_ok(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 3) return PyErr_Format(PyExc_TypeError, "q8_ok takes 3 arguments, not %zd", n);
  return guarded([&]() -> PyObject * {
    const at::Tensor *d = plain_tensor(a[0]), *s = plain_tensor(a[1]);
    Rows r;
    if (!d || !s || !PyLong_CheckExact(a[2]) || !rows_in(*d, *s, PyLong_AsLongLong(a[2]), &r) || PyErr_Occurred()) return not_mine();
    Py_RETURN_TRUE;
  });
}

// quantize(x, stream) -> (data, scale, K)
PyObject *quantize(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 2) return PyErr_Format(PyExc_TypeError, "quantize takes 2 arguments, not %zd", n);
  return guarded([&]() -> PyObject * {
    const at::Tensor *x = plain_tensor(a[0]);
    int dtype;
    long long rows, ldx;
    void *st;
    if (!x || x->dim() < 1 || !float_type(*x, &dtype) || !rows_of(*x, 1, &rows, &ldx) || x->size(-1) > 0x7fffff00 ||
        !stream_on(a[1], x->get_device(), &st))
      return not_mine();
    const long long K = x->size(-1), nb = (K + 127) / 128;
    const auto bytes = x->options().dtype(at::kByte);
    const at::Tensor d = at::empty({rows, 128 * nb}, bytes), s = at::empty({rows, (nb + 3) / 4 * 4}, bytes);
    const pab_q8 y{d.data_ptr(), s.data_ptr(), d.stride(0), s.stride(0)};
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = pab_quantize(rows, (int)K, dtype, x->data_ptr(), ldx, &y, st);
    Py_END_ALLOW_THREADS
    if (rc < 0) return failed(rc);
    return Py_BuildValue("(NNL)", THPVariable_Wrap(d), THPVariable_Wrap(s), K);
  });
}

// dequantize(y, x, gate, dtype, out, stream) -> out
PyObject *dequantize(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 6) return PyErr_Format(PyExc_TypeError, "dequantize takes 6 arguments, not %zd", n);
  return guarded([&]() -> PyObject * {
    Rows y;
    void *st;
    if (!q8_of(a[0], &y)) return not_mine();
    const at::Tensor *x = a[1] == Py_None ? nullptr : plain_tensor(a[1]), *given = a[4] == Py_None ? nullptr : plain_tensor(a[4]);
    if ((a[1] != Py_None && !x) || (a[4] != Py_None && !given)) return not_mine();
    at::ScalarType type = at::kBFloat16;
    if (a[3] != Py_None) {
      if (!THPDtype_Check(a[3])) return not_mine();
      type = reinterpret_cast<THPDtype *>(a[3])->scalar_type;
    } else if (x) {
      type = x->scalar_type();
    } else if (given) {
      type = given->scalar_type();
    }
    if (type != at::kBFloat16 && type != at::kFloat) return not_mine();
    long long rows = 0, ldx = 0, ldo = 0;
    if (x && (x->scalar_type() != type || !rows_of(*x, 1, &rows, &ldx) || rows != y.rows || x->size(-1) != y.K || x->get_device() != y.device))
      return not_mine();
    const void *gate;
    if (!vector_of(a[2], type, y.K, y.device, &gate) || !stream_on(a[5], y.device, &st)) return not_mine();
    at::Tensor out;
    if (given) out = *given;
    else if (x) out = at::empty(x->sizes(), x->options());
    else out = at::empty({y.rows, y.K}, y.like.options().dtype(type));
    if (out.scalar_type() != type || !rows_of(out, 1, &rows, &ldo) || rows != y.rows || out.size(-1) != y.K || out.get_device() != y.device)
      return not_mine();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = pab_dequantize(y.rows, (int)y.K, type == at::kBFloat16 ? PAB_BF16 : PAB_F32, &y.q, x ? x->data_ptr() : nullptr, ldx, gate, out.data_ptr(),
                        ldo, st);
    Py_END_ALLOW_THREADS
    if (rc < 0) return failed(rc);
    return THPVariable_Wrap(out);
  });
}

// linear_quantized(a, w, bias, act, out, stream) -> out
PyObject *linear_quantized(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 6) return PyErr_Format(PyExc_TypeError, "linear_quantized takes 6 arguments, not %zd", n);
  return guarded([&]() -> PyObject * {
    Rows x, w, r;
    int act;
    const void *bias;
    void *st;
    if (!q8_of(a[0], &x) || !q8_of(a[1], &w) || x.K != w.K || x.device != w.device || x.rows > 0x7fffff00 || w.rows > 0x7fffff00 ||
        !integer(a[3], &act) || !vector_of(a[2], at::kBFloat16, w.rows, x.device, &bias))
      return not_mine();
    const bool rows8 = (PyObject *)Py_TYPE(a[4]) == q8_type;
    const at::Tensor *given = a[4] == Py_None || rows8 ? nullptr : plain_tensor(a[4]);
    if (rows8 ? !q8_of(a[4], &r) || r.rows != x.rows || r.K != w.rows || r.device != x.device : a[4] != Py_None && !given) return not_mine();
    if (!stream_on(a[5], x.device, &st)) return not_mine();
    at::Tensor out;
    long long rows = 0, ldc = 0;
    if (!rows8) {
      out = given ? *given : at::empty({x.rows, w.rows}, x.like.options().dtype(at::kBFloat16));
      if (out.scalar_type() != at::kBFloat16 || !rows_of(out, 1, &rows, &ldc) || rows != x.rows || out.size(-1) != w.rows || out.get_device() != x.device)
        return not_mine();
    }
    void *c = rows8 ? nullptr : out.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = pab_linear_quantized((int)x.rows, (int)w.rows, (int)x.K, &x.q, &w.q, bias, act, c, ldc, rows8 ? &r.q : nullptr, st);
    Py_END_ALLOW_THREADS
    if (rc < 0) return failed(rc);
    return rows8 ? Py_NewRef(a[4]) : THPVariable_Wrap(out);
  });
}

bool three_of(PyObject *o, int v[3]) {
  if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != 3) return false;
  for (int i = 0; i < 3; ++i) {
    int overflow;
    PyObject *x = PyTuple_GET_ITEM(o, i);
    if (!PyLong_CheckExact(x)) return false;
    const long k = PyLong_AsLongAndOverflow(x, &overflow);
    if (overflow || k < 0 || k > 0x7fffff00) return false;
    v[i] = (int)k;
  }
  return true;
}

// qk_norm_rope(q, k, places, axis_dim, factors, norm, gamma_q, beta_q, gamma_k, beta_k, eps, q_out, k_out, stream) -> (q_out, k_out)
PyObject *qk_norm_rope(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 14) return PyErr_Format(PyExc_TypeError, "qk_norm_rope takes 14 arguments, not %zd", n);
  return guarded([&]() -> PyObject * {
    const at::Tensor *q = plain_tensor(a[0]), *k = a[1] == Py_None ? nullptr : plain_tensor(a[1]);
    pab_qk_norm d{};
    void *st;
    long long rows = 0, m = 0;
    if (!q || (a[1] != Py_None && !k) || q->dim() < 3 || !float_type(*q, &d.dtype) || !three_of(a[2], d.places) || !three_of(a[3], d.axis_dim) ||
        !integer(a[5], &d.norm) || !PyFloat_CheckExact(a[10]) || !rows_of(*q, 2, &rows, &d.ld_q))
      return not_mine();
    const int device = q->get_device();
    const auto type = q->scalar_type();
    const int64_t H = q->size(-2), D = q->size(-1);
    if (H > 0x7fffff00 || D > 0x7fffff00) return not_mine();
    const __int128 grid = (__int128)d.places[0] * d.places[1] * d.places[2];
    if (grid < 1 || grid > rows || rows % (long long)grid || rows > 0x7fffffffLL) return not_mine();
    d.n_batch = (int)(rows / (long long)grid);
    d.heads_q = (int)H;
    d.head_dim = (int)D;
    d.eps = (float)PyFloat_AS_DOUBLE(a[10]);
    long long pairs = 0;
    for (int i = 0; i < 3; ++i) pairs += (long long)d.places[i] * (d.axis_dim[i] / 2);
    if (!vector_of(a[4], at::kFloat, 2 * pairs, device, &d.factors) || !vector_of(a[6], type, D, device, &d.gamma_q) ||
        !vector_of(a[7], type, D, device, &d.beta_q) || !vector_of(a[8], type, D, device, &d.gamma_k) || !vector_of(a[9], type, D, device, &d.beta_k))
      return not_mine();
    const at::Tensor *given[2] = {a[11] == Py_None ? nullptr : plain_tensor(a[11]), a[12] == Py_None ? nullptr : plain_tensor(a[12])};
    if ((a[11] != Py_None && !given[0]) || (a[12] != Py_None && !given[1]) || (!k && a[12] != Py_None)) return not_mine();
    if (k && (k->dim() < 3 || k->scalar_type() != type || k->get_device() != device || !rows_of(*k, 2, &m, &d.ld_k) || m != rows || k->size(-1) != D ||
              k->size(-2) > 0x7fffff00))
      return not_mine();
    if (!stream_on(a[13], device, &st)) return not_mine();
    const at::Tensor q_out = given[0] ? *given[0] : at::empty(q->sizes(), q->options());
    at::Tensor k_out;
    if (k) k_out = given[1] ? *given[1] : at::empty(k->sizes(), k->options());
    auto fits = [&](const at::Tensor &out, const at::Tensor &in, long long *ld) {
      return out.scalar_type() == type && out.sizes() == in.sizes() && out.get_device() == device && rows_of(out, 2, &m, ld);
    };
    if (!fits(q_out, *q, &d.ld_q_out) || (k && !fits(k_out, *k, &d.ld_k_out))) return not_mine();
    d.q = q->data_ptr();
    d.q_out = q_out.data_ptr();
    if (k) {
      d.heads_k = (int)k->size(-2);
      d.k = k->data_ptr();
      d.k_out = k_out.data_ptr();
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = pab_qk_norm_rope(&d, st);
    Py_END_ALLOW_THREADS
    if (rc < 0) return failed(rc);
    if (!k) return Py_BuildValue("(NO)", THPVariable_Wrap(q_out), Py_None);
    return Py_BuildValue("(NN)", THPVariable_Wrap(q_out), THPVariable_Wrap(k_out));
  });
}

// bind_q8(pab.Q8)
PyObject *bind_q8(PyObject *, PyObject *type) {
  PyObject *old = q8_type;
  q8_type = Py_NewRef(type);
  Py_XDECREF(old);
  if (!s_data) s_data = PyUnicode_InternFromString("data");
  if (!s_scale) s_scale = PyUnicode_InternFromString("scale");
  if (!s_K) s_K = PyUnicode_InternFromString("K");
  if (!s_data || !s_scale || !s_K) return nullptr;
  Py_RETURN_NONE;
}

// bind(pab._check, torch's current device function, its raw stream function; None where there is none)
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 3) return PyErr_Format(PyExc_TypeError, "bind takes 3 arguments, not %zd", n);
  PyObject **slot[3] = {&py_check, &get_device, &get_raw_stream};
  for (int i = 0; i < 3; ++i) {
    PyObject *old = *slot[i];
    *slot[i] = a[i] == Py_None ? nullptr : Py_NewRef(a[i]);
    Py_XDECREF(old);
  }
  if (!get_device) Py_CLEAR(get_raw_stream);
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"attention", (PyCFunction)(void (*)(void))attention, METH_FASTCALL, nullptr},
                         {"attention_compute", (PyCFunction)(void (*)(void))attention_compute, METH_FASTCALL, nullptr},
                         {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
                         {"bind_q8", (PyCFunction)bind_q8, METH_O, nullptr},
                         {"q8_ok", (PyCFunction)(void (*)(void))q8_ok, METH_FASTCALL, nullptr},
                         {"quantize", (PyCFunction)(void (*)(void))quantize, METH_FASTCALL, nullptr},
                         {"dequantize", (PyCFunction)(void (*)(void))dequantize, METH_FASTCALL, nullptr},
                         {"linear_quantized", (PyCFunction)(void (*)(void))linear_quantized, METH_FASTCALL, nullptr},
                         {"qk_norm_rope", (PyCFunction)(void (*)(void))qk_norm_rope, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }

// Python module _call: entry points of the C ABI called with torch tensors: those of Scan and Delta, the block's
// group norm and the windowed convolution.
//
// A decode step is one kernel of some 4 us, and handing its sixteen arguments over through ctypes took
// 2.5 us of host time (on a slower host 6), beside a launch of 3.5.  Here the addresses are taken from the
// tensors directly and the options are put on the stack: 0.2 us (0.4).  The library is the one
// that ctypes has loaded; its entry points come in as addresses.
#include <Python.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/m2rnn.h"

namespace {

decltype(&m2rnn_fwd_opt) fwd_opt = nullptr;
decltype(&m2rnn_bwd_opt) bwd_opt = nullptr;
decltype(&m2rnn_delta_fwd) delta_fwd = nullptr;
decltype(&m2rnn_delta_bwd) delta_bwd = nullptr;
decltype(&m2rnn_delta_ckpt_bytes) delta_ckpt_bytes = nullptr;
decltype(&m2rnn_group_norm_fwd) group_norm_fwd = nullptr;
decltype(&m2rnn_group_norm_bwd) group_norm_bwd = nullptr;
decltype(&m2rnn_conv_silu_window_fwd) window_fwd = nullptr;

// None -> NULL, an int as it is, a tensor -> its address, anything else -> what its data_ptr() says (a
// subclass of the tensor may have its own); false with a Python error set otherwise
bool address(PyObject *o, void *&p) {
  if (o == Py_None) {
    p = nullptr;
  } else if (THPVariable_CheckExact(o)) {
    p = THPVariable_Unpack(o).data_ptr();
  } else if (PyLong_Check(o)) {
    p = PyLong_AsVoidPtr(o);
    return !(p == nullptr && PyErr_Occurred());
  } else {
    PyObject *method = PyObject_GetAttrString(o, "data_ptr");
    if (!method) {
      if (PyErr_ExceptionMatches(PyExc_AttributeError))
        PyErr_SetString(PyExc_TypeError, "expected a tensor, an address or None");
      return false;
    }
    PyObject *number = PyObject_CallNoArgs(method);
    Py_DECREF(method);
    if (!number) return false;
    p = PyLong_AsVoidPtr(number);
    Py_DECREF(number);
    return !(p == nullptr && PyErr_Occurred());
  }
  return true;
}

// the addresses of the positional arguments a0 .. a0 + n - 1
template <size_t n>
bool addresses(PyObject *const *args, void *(&p)[n]) {
  try {
    for (size_t i = 0; i < n; ++i)
      if (!address(args[i], p[i])) return false;
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return false;
  }
  return true;
}

bool ready(const void *entry) {
  if (!entry) PyErr_SetString(PyExc_RuntimeError, "init has not been called");
  return entry != nullptr;
}

bool arity(Py_ssize_t have, Py_ssize_t want) {
  if (have != want) PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, have);
  return have == want;
}

PyObject *init(PyObject *, PyObject *const *args, Py_ssize_t n) {
  void *p[2];
  if (!arity(n, 2) || !addresses(args, p)) return nullptr;
  if (!p[0] || !p[1]) {
    PyErr_SetString(PyExc_ValueError, "an entry point is NULL");
    return nullptr;
  }
  fwd_opt = (decltype(fwd_opt))p[0];
  bwd_opt = (decltype(bwd_opt))p[1];
  Py_RETURN_NONE;
}

// fwd(desc, w_r, gate_alpha, gate_beta, q, k, v, f, W, H0, y, HT, ckpt, workspace, stream, bytes) -> status
PyObject *fwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  void *p[15];
  if (!ready((const void *)fwd_opt) || !arity(n, 16) || !addresses(args, p)) return nullptr;
  const size_t bytes = PyLong_AsSize_t(args[15]);
  if (bytes == (size_t)-1 && PyErr_Occurred()) return nullptr;
  m2rnn_opts o = {};
  o.w_r = p[1];
  o.gate_alpha = (const float *)p[2];
  o.gate_beta = (const float *)p[3];
  m2rnn_status st;
  Py_BEGIN_ALLOW_THREADS
  st = fwd_opt((const m2rnn_desc *)p[0], &o, p[4], p[5], p[6], (const float *)p[7], p[8], (const float *)p[9], p[10],
               (float *)p[11], (float *)p[12], p[13], bytes, p[14]);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// bwd(desc, w_r, dw_r, gate_alpha, gate_beta, dgate_alpha, dgate_beta, q, k, v, f, W, H0, ckpt, dy, dHT,
//     dq, dk, dv, df, dW, dH0, workspace, stream, bytes, grad_clip) -> status
PyObject *bwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  void *p[24];
  if (!ready((const void *)bwd_opt) || !arity(n, 26) || !addresses(args, p)) return nullptr;
  const size_t bytes = PyLong_AsSize_t(args[24]);
  const double clip = PyFloat_AsDouble(args[25]);
  if (PyErr_Occurred()) return nullptr;
  m2rnn_opts o = {};
  o.w_r = p[1];
  o.dw_r = (float *)p[2];
  o.grad_clip = (float)clip;
  o.gate_alpha = (const float *)p[3];
  o.gate_beta = (const float *)p[4];
  o.dgate_alpha = (float *)p[5];
  o.dgate_beta = (float *)p[6];
  m2rnn_status st;
  Py_BEGIN_ALLOW_THREADS
  st = bwd_opt((const m2rnn_desc *)p[0], &o, p[7], p[8], p[9], (const float *)p[10], p[11], (const float *)p[12],
               (const float *)p[13], p[14], (const float *)p[15], p[16], p[17], p[18], (float *)p[19], (float *)p[20],
               (float *)p[21], p[22], bytes, p[23]);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

PyObject *init_layer(PyObject *, PyObject *const *args, Py_ssize_t n) {
  void *p[6];
  if (!arity(n, 6) || !addresses(args, p)) return nullptr;
  for (const void *entry : p)
    if (!entry) {
      PyErr_SetString(PyExc_ValueError, "an entry point is NULL");
      return nullptr;
    }
  delta_fwd = (decltype(delta_fwd))p[0];
  delta_bwd = (decltype(delta_bwd))p[1];
  delta_ckpt_bytes = (decltype(delta_ckpt_bytes))p[2];
  group_norm_fwd = (decltype(group_norm_fwd))p[3];
  group_norm_bwd = (decltype(group_norm_bwd))p[4];
  window_fwd = (decltype(window_fwd))p[5];
  Py_RETURN_NONE;
}

// An operand as `address` takes it; of a tensor also what the kernels assume of it: its type, its number of
// elements, dense, on the GPU `device` that the call's stream belongs to (device < 0: any).
bool operand(PyObject *o, const char *name, at::ScalarType type, int64_t count, long device, void *&p) {
  if (!THPVariable_Check(o)) return address(o, p);
  try {
    const at::Tensor &t = THPVariable_Unpack(o);
    const char *bad = !t.is_cuda() ? "is not on the GPU"
                      : device >= 0 && t.get_device() != device ? "is on another GPU than the current one"
                      : t.scalar_type() != type ? "has another dtype than the call takes"
                      : t.numel() != count ? "has another size than the call takes"
                      : !t.is_contiguous() ? "is not contiguous"
                                           : nullptr;
    if (bad) {
      PyErr_Format(PyExc_ValueError, "%s %s", name, bad);
      return false;
    }
    p = t.data_ptr();
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return false;
  }
  return true;
}
// Room of at least `bytes` bytes, as a tensor of any type, an address or None.
bool room(PyObject *o, const char *name, size_t bytes, long device, void *&p) {
  if (THPVariable_Check(o)) {
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!operand(o, name, t.scalar_type(), t.numel(), device, p)) return false;
    if (t.nbytes() < bytes) {
      PyErr_Format(PyExc_ValueError, "%s has fewer bytes than the call takes", name);
      return false;
    }
    return true;
  }
  return address(o, p);
}
at::ScalarType io_type(int32_t io) { return io == M2RNN_BF16 ? at::kBFloat16 : at::kFloat; }

struct DeltaSizes {
  int64_t qk, v, gates, state;
  explicit DeltaSizes(const m2rnn_desc *d) {
    const int64_t bt = (int64_t)d->B * d->T;
    qk = bt * d->Nqk * d->K;
    v = bt * d->N * d->V;
    gates = bt * d->N;
    state = (int64_t)d->B * d->N * d->K * d->V;
  }
};

// delta_fwd(desc, q, k, v, g, beta, H0, y, HT, ckpt, workspace, stream, bytes, device) -> status
PyObject *call_delta_fwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (!ready((const void *)delta_fwd) || !arity(n, 14)) return nullptr;
  void *d, *q, *k, *v, *g, *beta, *H0, *y, *HT, *ckpt, *ws, *stream;
  const size_t bytes = PyLong_AsSize_t(args[12]);
  const long dev = PyLong_AsLong(args[13]);
  if (PyErr_Occurred() || !address(args[0], d)) return nullptr;
  const m2rnn_desc *desc = (const m2rnn_desc *)d;
  const DeltaSizes z(desc);
  const at::ScalarType io = io_type(desc->io), f = at::kFloat;
  if (!operand(args[1], "q", io, z.qk, dev, q) || !operand(args[2], "k", io, z.qk, dev, k) ||
      !operand(args[3], "v", io, z.v, dev, v) || !operand(args[4], "g", f, z.gates, dev, g) ||
      !operand(args[5], "beta", f, z.gates, dev, beta) || !operand(args[6], "H0", f, z.state, dev, H0) ||
      !operand(args[7], "y", io, z.v, dev, y) || !operand(args[8], "HT", f, z.state, dev, HT) ||
      !room(args[9], "ckpt", args[9] == Py_None ? 0 : delta_ckpt_bytes(desc), dev, ckpt) ||
      !room(args[10], "workspace", bytes, dev, ws) || !address(args[11], stream))
    return nullptr;
  m2rnn_status st;
  Py_BEGIN_ALLOW_THREADS
  st = delta_fwd(desc, q, k, v, (const float *)g, (const float *)beta, (const float *)H0, y, (float *)HT, ckpt,
                 ws, bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// delta_bwd(desc, q, k, v, g, beta, H0, ckpt, dy, dHT, dq, dk, dv, dg, dbeta, dH0, workspace, stream, bytes, device)
// -> status
PyObject *call_delta_bwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (!ready((const void *)delta_bwd) || !arity(n, 20)) return nullptr;
  void *d, *q, *k, *v, *g, *beta, *H0, *ckpt, *dy, *dHT, *dq, *dk, *dv, *dg, *dbeta, *dH0, *ws, *stream;
  const size_t bytes = PyLong_AsSize_t(args[18]);
  const long dev = PyLong_AsLong(args[19]);
  if (PyErr_Occurred() || !address(args[0], d)) return nullptr;
  const m2rnn_desc *desc = (const m2rnn_desc *)d;
  const DeltaSizes z(desc);
  const at::ScalarType io = io_type(desc->io), f = at::kFloat;
  if (!operand(args[1], "q", io, z.qk, dev, q) || !operand(args[2], "k", io, z.qk, dev, k) ||
      !operand(args[3], "v", io, z.v, dev, v) || !operand(args[4], "g", f, z.gates, dev, g) ||
      !operand(args[5], "beta", f, z.gates, dev, beta) || !operand(args[6], "H0", f, z.state, dev, H0) ||
      !room(args[7], "ckpt", args[7] == Py_None ? 0 : delta_ckpt_bytes(desc), dev, ckpt) ||
      !operand(args[8], "dy", io, z.v, dev, dy) || !operand(args[9], "dHT", f, z.state, dev, dHT) ||
      !operand(args[10], "dq", io, z.qk, dev, dq) || !operand(args[11], "dk", io, z.qk, dev, dk) ||
      !operand(args[12], "dv", io, z.v, dev, dv) || !operand(args[13], "dg", io, z.gates, dev, dg) ||
      !operand(args[14], "dbeta", io, z.gates, dev, dbeta) || !operand(args[15], "dH0", f, z.state, dev, dH0) ||
      !room(args[16], "workspace", bytes, dev, ws) || !address(args[17], stream))
    return nullptr;
  m2rnn_status st;
  Py_BEGIN_ALLOW_THREADS
  st = delta_bwd(desc, q, k, v, (const float *)g, (const float *)beta, (const float *)H0, ckpt, dy, (const float *)dHT,
                 dq, dk, dv, dg, dbeta, (float *)dH0, ws, bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// The sizes and the type of x [B,T,D], and the current GPU, which all tensors have to be on (a stream belongs to it);
// false with a Python error set
bool shape_of(PyObject *o, int32_t (&size)[3], int32_t &io, long &device) {
  if (!THPVariable_Check(o)) {
    PyErr_SetString(PyExc_TypeError, "x: expected a tensor");
    return false;
  }
  const at::Tensor &t = THPVariable_Unpack(o);
  if (t.dim() != 3 || (t.scalar_type() != at::kBFloat16 && t.scalar_type() != at::kFloat)) {
    PyErr_SetString(PyExc_ValueError, "x: expected three dimensions, float32 or bfloat16");
    return false;
  }
  for (int i = 0; i < 3; ++i) {
    if (t.size(i) > INT32_MAX) {
      PyErr_SetString(PyExc_ValueError, "x: a dimension is too large");
      return false;
    }
    size[i] = (int32_t)t.size(i);
  }
  io = t.scalar_type() == at::kBFloat16 ? M2RNN_BF16 : M2RNN_F32;
  device = -1;
  try {
    if (t.is_cuda()) device = c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice().index();
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return false;
  }
  return true;
}
// groups, eps and mode
bool norm_of(PyObject *const *args, int32_t &groups, float &eps, int32_t &mode) {
  const long g = PyLong_AsLong(args[0]), m = PyLong_AsLong(args[2]);
  eps = (float)PyFloat_AsDouble(args[1]);
  if (PyErr_Occurred()) return false;
  groups = (int32_t)g;
  mode = (int32_t)m;
  if (groups != g || mode != m) PyErr_SetString(PyExc_ValueError, "groups or mode is too large");
  return groups == g && mode == m;
}

// group_norm_fwd(x, a, w, b, groups, eps, mode, out, stream) -> status
PyObject *call_group_norm_fwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  int32_t s[3], io;
  long dev;
  if (!ready((const void *)group_norm_fwd) || !arity(n, 9) || !shape_of(args[0], s, io, dev)) return nullptr;
  int32_t groups, mode;
  float eps;
  void *x, *a, *w, *b, *out, *stream;
  const int64_t all = (int64_t)s[0] * s[1] * s[2];
  const at::ScalarType t = io_type(io);
  if (!norm_of(args + 4, groups, eps, mode) || !operand(args[0], "x", t, all, dev, x) || !operand(args[1], "a", t, all, dev, a) ||
      !operand(args[2], "w", t, s[2], dev, w) || !operand(args[3], "b", t, s[2], dev, b) ||
      !operand(args[7], "out", t, all, dev, out) || !address(args[8], stream))
    return nullptr;
  m2rnn_status st;
  Py_BEGIN_ALLOW_THREADS
  st = group_norm_fwd(s[0], s[1], s[2], groups, io, mode, x, a, w, b, eps, out, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// group_norm_bwd(x, a, w, b, groups, eps, mode, dout, dx, da, dw, db, workspace, stream, bytes) -> status
PyObject *call_group_norm_bwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  int32_t s[3], io;
  long dev;
  if (!ready((const void *)group_norm_bwd) || !arity(n, 15) || !shape_of(args[0], s, io, dev)) return nullptr;
  int32_t groups, mode;
  float eps;
  const size_t bytes = PyLong_AsSize_t(args[14]);
  if (PyErr_Occurred()) return nullptr;
  void *x, *a, *w, *b, *dout, *dx, *da, *dw, *db, *ws, *stream;
  const int64_t all = (int64_t)s[0] * s[1] * s[2];
  const at::ScalarType t = io_type(io), f = at::kFloat;
  if (!norm_of(args + 4, groups, eps, mode) || !operand(args[0], "x", t, all, dev, x) ||
      !operand(args[1], "a", t, all, dev, a) || !operand(args[2], "w", t, s[2], dev, w) ||
      !operand(args[3], "b", t, s[2], dev, b) || !operand(args[7], "dout", t, all, dev, dout) ||
      !operand(args[8], "dx", t, all, dev, dx) || !operand(args[9], "da", t, all, dev, da) ||
      !operand(args[10], "dw", f, s[2], dev, dw) || !operand(args[11], "db", f, s[2], dev, db) ||
      !room(args[12], "workspace", bytes, dev, ws) || !address(args[13], stream))
    return nullptr;
  m2rnn_status st;
  Py_BEGIN_ALLOW_THREADS
  st = group_norm_bwd(s[0], s[1], s[2], groups, io, mode, x, a, w, b, eps, dout, dx, da, (float *)dw, (float *)db, ws,
                      bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// window_fwd(x, w, bias, win, out, win_out, stream) -> status
PyObject *call_window_fwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
  int32_t s[3], io;
  long dev;
  if (!ready((const void *)window_fwd) || !arity(n, 7) || !shape_of(args[0], s, io, dev)) return nullptr;
  void *x, *w, *bias, *win, *out, *win_out, *stream;
  const int64_t all = (int64_t)s[0] * s[1] * s[2], rows = (int64_t)s[0] * 3 * s[2];
  const at::ScalarType t = io_type(io);
  if (!operand(args[0], "x", t, all, dev, x) || !operand(args[1], "w", t, 4 * (int64_t)s[2], dev, w) ||
      !operand(args[2], "bias", t, s[2], dev, bias) || !operand(args[3], "win", t, rows, dev, win) ||
      !operand(args[4], "out", t, all, dev, out) || !operand(args[5], "win_out", t, rows, dev, win_out) ||
      !address(args[6], stream))
    return nullptr;
  m2rnn_status st;
  Py_BEGIN_ALLOW_THREADS
  st = window_fwd(s[0], s[1], s[2], io, x, w, bias, win, out, win_out, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

PyMethodDef methods[] = {{"init", (PyCFunction)(void (*)(void))init, METH_FASTCALL, nullptr},
                         {"init_layer", (PyCFunction)(void (*)(void))init_layer, METH_FASTCALL, nullptr},
                         {"group_norm_fwd", (PyCFunction)(void (*)(void))call_group_norm_fwd, METH_FASTCALL, nullptr},
                         {"group_norm_bwd", (PyCFunction)(void (*)(void))call_group_norm_bwd, METH_FASTCALL, nullptr},
                         {"window_fwd", (PyCFunction)(void (*)(void))call_window_fwd, METH_FASTCALL, nullptr},
                         {"delta_fwd", (PyCFunction)(void (*)(void))call_delta_fwd, METH_FASTCALL, nullptr},
                         {"delta_bwd", (PyCFunction)(void (*)(void))call_delta_bwd, METH_FASTCALL, nullptr},
                         {"fwd", (PyCFunction)(void (*)(void))fwd, METH_FASTCALL, nullptr},
                         {"bwd", (PyCFunction)(void (*)(void))bwd, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject *PyInit__call() {
  PyObject *m = PyModule_Create(&module);
  // (a tensor is read through torch's own headers: under another torch its layout may be another one)
  if (m && PyModule_AddStringConstant(m, "torch_version", M2RNN_TORCH_VERSION) < 0) Py_CLEAR(m);
  return m;
}

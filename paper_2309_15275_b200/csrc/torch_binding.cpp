// Native part of the Python binding: the calls of binding.py and autograd.py that a
// training step makes, with tensor checks, output allocation and argument marshalling
// in C++ (a call through ctypes cost 15-40 us of host time, several times what the
// kernels of a small layer take), and the autograd function behind LbpLinear, whose
// backward pass then runs without the interpreter.
//
// Conventions of the module functions: positional arguments as binding.py passes them.
// They return the call's result; an int, the lbp_status, where the library refused; None
// where an argument is not what they expect.  In that case nothing has been done, and
// binding.py goes through its own checks, which name the error.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/autocast_mode.h>
#include <ATen/cuda/CUDAGeneratorImpl.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <dlfcn.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/python_cpp_function.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/pybind.h>

#include <mutex>
#include <optional>
#include <string>
#include <vector>

#include "lbp.h"

namespace {

using at::Tensor;

// ---- the C library, resolved from the file binding.py has loaded ----
struct Library {
  decltype(&lbp_status_string) status_string;
  decltype(&lbp_status_bytes) status_bytes;
  decltype(&lbp_workspace_bytes) workspace_bytes;
  decltype(&lbp_workspace_bytes_ex) workspace_bytes_ex;
  decltype(&lbp_workspace_bytes_projected) workspace_bytes_projected;
  decltype(&lbp_spectrum_workspace_bytes) spectrum_workspace_bytes;
  decltype(&lbp_project) project;
  decltype(&lbp_spectrum) spectrum;
  decltype(&lbp_backward) backward;
  decltype(&lbp_backward_ex) backward_ex;
  decltype(&lbp_backward_batch) backward_batch;
  decltype(&lbp_backward_fullrank) backward_fullrank;
  decltype(&lbp_linear_workspace_bytes) linear_workspace_bytes;
  decltype(&lbp_linear) linear;
  decltype(&lbp_linear_grad) linear_grad;
  decltype(&lbp_dropout) dropout;
  decltype(&lbp_project_grad_workspace_bytes) project_grad_workspace_bytes;
  decltype(&lbp_project_grad) project_grad;
  decltype(&lbp_workspace_bytes_act) workspace_bytes_act;
  decltype(&lbp_backward_act) backward_act;
} lib;
PyObject* error_type = nullptr;   // binding.LbpError

template <class F>
bool resolve(void* handle, const char* name, F* fn) {
  *fn = reinterpret_cast<F>(dlsym(handle, name));
  return *fn != nullptr;
}

// ---- arguments ----
struct Bases {
  lbp_basis v[256];
  int r = 0;
};
// int(o), where that is an int32; false otherwise (no error is left behind).
bool index_of(PyObject* o, int32_t* v) {
  int over = 0;
  long l = 0;
  if (PyLong_Check(o)) {
    l = PyLong_AsLongAndOverflow(o, &over);
  } else {   // a numpy or torch scalar, a float
    PyObject* n = PyNumber_Long(o);
    if (n == nullptr) {
      PyErr_Clear();
      return false;
    }
    l = PyLong_AsLongAndOverflow(n, &over);
    Py_DECREF(n);
  }
  *v = static_cast<int32_t>(l);
  return over == 0 && *v == l;
}
// A sequence of pairs; whether a pair is a basis is the library's to say.
bool parse_pair(PyObject* p, lbp_basis* out) {
  if (PyTuple_Check(p) && PyTuple_GET_SIZE(p) == 2)
    return index_of(PyTuple_GET_ITEM(p, 0), &out->i) && index_of(PyTuple_GET_ITEM(p, 1), &out->j);
  PyObject* t = PySequence_Check(p) ? PySequence_Tuple(p) : nullptr;   // a list, a row of an array
  const bool ok = t != nullptr && PyTuple_GET_SIZE(t) == 2 && index_of(PyTuple_GET_ITEM(t, 0), &out->i) &&
                  index_of(PyTuple_GET_ITEM(t, 1), &out->j);
  Py_XDECREF(t);
  PyErr_Clear();
  return ok;
}
bool parse_bases(PyObject* o, Bases* out) {
  if (!PySequence_Check(o)) return false;
  PyObject* s = PySequence_Fast(o, "");
  if (s == nullptr) {
    PyErr_Clear();
    return false;
  }
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(s);
  bool ok = n <= 256;
  for (Py_ssize_t q = 0; q < n && ok; ++q) ok = parse_pair(PySequence_Fast_GET_ITEM(s, q), &out->v[q]);
  Py_DECREF(s);
  out->r = static_cast<int>(n);
  return ok;
}

bool parse_int(PyObject* o, int* v) {
  int32_t a = 0;
  if (!PyIndex_Check(o) || !index_of(o, &a) || a < 0 || a > (1 << 30)) return false;   // no floats
  *v = a;
  return true;
}

// A tensor, or an undefined one for None; false: neither.
bool parse_tensor(PyObject* o, Tensor* t) {
  if (o == Py_None) return true;
  if (!THPVariable_Check(o)) return false;
  *t = THPVariable_Unpack(o);
  return true;
}

int dtype_code(at::ScalarType t) {
  if (t == at::kFloat) return LBP_F32;
  if (t == at::kBFloat16) return LBP_BF16;
  return -1;
}
int parse_dtype(PyObject* o) {
  return THPDtype_Check(o) ? dtype_code(reinterpret_cast<THPDtype*>(o)->scalar_type) : -1;
}

bool int_size(int64_t v) { return v >= 0 && v <= (1ll << 30); }

// On the current CUDA device, and contiguous.
bool dense_on(const Tensor& t, int dev) {
  return t.is_cuda() && t.get_device() == dev && t.is_contiguous();
}

bool has_shape(const Tensor& t, at::IntArrayRef want) { return t.sizes() == want; }

// Strides of a (B,H,W,C) tensor as the library takes them (all zero: dense).
bool view_of(const Tensor& t, int dev, lbp_view* v) {
  *v = lbp_view{0, 0, 0};
  if (!t.is_cuda() || t.get_device() != dev) return false;
  if (t.is_contiguous()) return true;
  const int64_t B = t.size(0), H = t.size(1), W = t.size(2), C = t.size(3);
  if (C > 1 && t.stride(3) != 1) return false;
  const int64_t tok = W > 1 ? t.stride(2) : C;
  const int64_t row = H > 1 ? t.stride(1) : W * tok;
  const int64_t img = B > 1 ? t.stride(0) : H * row;
  *v = lbp_view{img, row, tok};
  return img != 0 || row != 0 || tok != 0;   // (an expanded tensor would read as dense)
}
// Row pitch of an (n, C) matrix (0: dense).
bool rows_of(const Tensor& t, int dev, int64_t* pitch) {
  *pitch = 0;
  if (!t.is_cuda() || t.get_device() != dev) return false;
  if (t.is_contiguous()) return true;
  if (t.size(1) > 1 && t.stride(1) != 1) return false;
  *pitch = t.size(0) > 1 ? t.stride(0) : 0;
  return t.size(0) <= 1 || *pitch != 0;   // (an expanded tensor would read as dense)
}

Tensor bytes_on(const Tensor& like, size_t n) {
  return at::empty({static_cast<int64_t>(n)}, like.options().dtype(at::kByte));
}
// A new tensor like another, past the dispatcher (which takes 1 to 2 us of a call's 6).
Tensor fresh(at::IntArrayRef shape, at::ScalarType dtype, const Tensor& like) {
  return at::detail::empty_cuda(shape, dtype, like.device(), std::nullopt);
}
void* current_stream(int dev) { return c10::cuda::getCurrentCUDAStream(dev).stream(); }

PyObject* pair(const Tensor& a, const Tensor& b) {
  PyObject* t = PyTuple_New(2);
  if (t == nullptr) return nullptr;
  PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(a));
  PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(b));
  return t;
}
PyObject* not_handled() { Py_RETURN_NONE; }

// A call into the library: other Python threads run meanwhile (it may search a tile plan, wait
// for the batch section of another thread, or for room in a full launch queue).
template <class F>
auto without_gil(F call) {
  pybind11::gil_scoped_release no_gil;
  return call();
}

// One problem's shapes, dtypes and devices, as binding._check_layer_tensors has them.
struct Problem {
  lbp_layer L;
  int dev;
};
bool layer_of(const Tensor& g_y, const Tensor& W, const Tensor& x, int k, Problem* p) {
  if (!g_y.defined() || !W.defined() || g_y.dim() != 4 || W.dim() != 2 || !g_y.is_cuda()) return false;
  const int dt = dtype_code(g_y.scalar_type());
  if (dt < 0 || W.scalar_type() != g_y.scalar_type()) return false;
  const int64_t B = g_y.size(0), H = g_y.size(1), Wd = g_y.size(2), Cout = g_y.size(3), Cin = W.size(1);
  if (W.size(0) != Cout || !int_size(B) || !int_size(H) || !int_size(Wd) || !int_size(Cout) || !int_size(Cin))
    return false;
  p->dev = g_y.get_device();
  if (p->dev != c10::cuda::current_device() || !dense_on(W, p->dev)) return false;
  if (x.defined() && (!has_shape(x, {B, H, Wd, Cin}) || x.scalar_type() != g_y.scalar_type())) return false;
  p->L = lbp_layer{static_cast<int32_t>(B), static_cast<int32_t>(H), static_cast<int32_t>(Wd),
                   static_cast<int32_t>(Cin), static_cast<int32_t>(Cout), k, dt, LBP_F32};
  return true;
}
// The given output, checked, or a new one.
bool grad_x(Tensor* g_x, const Tensor& g_y, const lbp_layer& L) {
  if (!g_x->defined()) {
    *g_x = at::empty({L.B, L.H, L.W, L.Cin}, g_y.options());
    return true;
  }
  return has_shape(*g_x, {L.B, L.H, L.W, L.Cin}) && g_x->scalar_type() == g_y.scalar_type();
}
bool grad_w(Tensor* g_W, const Tensor& g_y, lbp_layer* L, int gw_code, int dev) {
  if (!g_W->defined()) {
    if (gw_code < 0) return false;
    *g_W = at::empty({L->Cout, L->Cin}, g_y.options().dtype(gw_code == LBP_BF16 ? at::kBFloat16 : at::kFloat));
  } else if (!has_shape(*g_W, {L->Cout, L->Cin}) || !dense_on(*g_W, dev)) {
    return false;
  }
  L->gw_dtype = dtype_code(g_W->scalar_type());
  return L->gw_dtype >= 0;
}

// project(t, k, bases, out, ws)
PyObject* py_project(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Tensor t, out, ws;
  int k = 0;
  Bases b;
  if (n != 5 || !parse_tensor(a[0], &t) || !parse_int(a[1], &k) || !parse_bases(a[2], &b) ||
      !parse_tensor(a[3], &out) || !parse_tensor(a[4], &ws) || !t.defined() || t.dim() != 4 || k < 1 || !t.is_cuda())
    return not_handled();
  const int dt = dtype_code(t.scalar_type()), dev = t.get_device();
  if (dt < 0 || dev != c10::cuda::current_device() || !t.is_contiguous()) return not_handled();
  for (int i = 0; i < 4; ++i)
    if (!int_size(t.size(i))) return not_handled();
  const int64_t shape[5] = {t.size(0), (t.size(1) + k - 1) / k, (t.size(2) + k - 1) / k, b.r, t.size(3)};
  if (!out.defined())
    out = at::empty(shape, t.options());
  else if (!has_shape(out, shape) || out.scalar_type() != t.scalar_type() || !dense_on(out, dev))
    return not_handled();
  if (!ws.defined()) ws = bytes_on(t, lib.status_bytes());
  if (!dense_on(ws, dev)) return not_handled();
  const int e = without_gil([&] {
    return lib.project(t.data_ptr(), out.data_ptr(), t.size(0), t.size(1), t.size(2), t.size(3), k, b.v, b.r, dt,
                       ws.data_ptr(), ws.numel(), current_stream(dev));
  });
  return e != LBP_OK ? PyLong_FromLong(e) : THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

// spectrum(t, k, out, ws)
PyObject* py_spectrum(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Tensor t, out, ws;
  int k = 0;
  if (n != 4 || !parse_tensor(a[0], &t) || !parse_int(a[1], &k) || !parse_tensor(a[2], &out) ||
      !parse_tensor(a[3], &ws) || !t.defined() || t.dim() != 4 || !t.is_cuda())
    return not_handled();
  const int dt = dtype_code(t.scalar_type()), dev = t.get_device();
  if (dt < 0 || dev != c10::cuda::current_device() || !t.is_contiguous()) return not_handled();
  for (int i = 0; i < 4; ++i)
    if (!int_size(t.size(i))) return not_handled();
  if (!out.defined())
    out = at::empty({k, k}, t.options().dtype(at::kDouble));
  else if (!has_shape(out, {k, k}) || out.scalar_type() != at::kDouble || !dense_on(out, dev))
    return not_handled();
  if (!ws.defined()) {
    const size_t bytes = lib.spectrum_workspace_bytes(t.size(0), t.size(1), t.size(2), t.size(3), k, dt);
    if (bytes == 0) return not_handled();
    ws = bytes_on(t, bytes);
  }
  if (!dense_on(ws, dev)) return not_handled();
  const int e = without_gil([&] {
    return lib.spectrum(t.data_ptr(), out.data_ptr<double>(), t.size(0), t.size(1), t.size(2), t.size(3), k, dt,
                        ws.data_ptr(), ws.numel(), current_stream(dev));
  });
  return e != LBP_OK ? PyLong_FromLong(e) : THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

// backward(x, g_y, W, k, bases | None, gw_dtype, g_x, g_W, ws); bases None: exact backpropagation
PyObject* py_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Tensor x, g_y, W, g_x, g_W, ws;
  int k = 0;
  Bases b;
  Problem p;
  if (n != 9 || !parse_tensor(a[0], &x) || !parse_tensor(a[1], &g_y) || !parse_tensor(a[2], &W) ||
      !parse_int(a[3], &k) || (a[4] != Py_None && !parse_bases(a[4], &b)) || !parse_tensor(a[6], &g_x) ||
      !parse_tensor(a[7], &g_W) || !parse_tensor(a[8], &ws) || !x.defined() || !layer_of(g_y, W, x, k, &p))
    return not_handled();
  const int dev = p.dev, r = a[4] == Py_None ? k * k : b.r;
  if (!dense_on(x, dev) || !dense_on(g_y, dev) || !grad_x(&g_x, g_y, p.L) || !dense_on(g_x, dev) ||
      !grad_w(&g_W, g_y, &p.L, parse_dtype(a[5]), dev))
    return not_handled();
  if (!ws.defined()) {
    const size_t bytes = lib.workspace_bytes(&p.L, r);
    if (bytes == 0) return not_handled();
    ws = bytes_on(g_y, bytes);
  }
  if (!dense_on(ws, dev)) return not_handled();
  const bool exact = a[4] == Py_None;
  const int e = without_gil([&] {
    return exact ? lib.backward_fullrank(x.data_ptr(), g_y.data_ptr(), W.data_ptr(), g_x.data_ptr(), g_W.data_ptr(),
                                         &p.L, ws.data_ptr(), ws.numel(), current_stream(dev))
                 : lib.backward(x.data_ptr(), g_y.data_ptr(), W.data_ptr(), g_x.data_ptr(), g_W.data_ptr(), &p.L, b.v,
                                b.r, ws.data_ptr(), ws.numel(), current_stream(dev));
  });
  return e != LBP_OK ? PyLong_FromLong(e) : pair(g_x, g_W);
  END_HANDLE_TH_ERRORS
}

// What lbp_backward_ex takes, as tensors; the optional ones may be undefined.
struct ExCall {
  Tensor x, x_hat, g_y, W, g_bias, x_extra, gy_extra, gx_extra, g_x, g_W, ws;
  double beta = 0.0;
  int k = 0, gw_code = LBP_F32;
  const lbp_layer_grad* grad = nullptr;   // lbp_backward_act
};
// Returns the library's status, or -1 where a check does not hold (nothing done).
int run_ex(ExCall* c, const lbp_basis* set, int r) {
  Problem p;
  if (c->x.defined() == c->x_hat.defined() || !layer_of(c->g_y, c->W, c->x, c->k, &p) || c->k < 1) return -1;
  lbp_layer& L = p.L;
  const int dev = p.dev;
  const at::ScalarType dt = c->g_y.scalar_type();
  if (c->x_hat.defined()) {
    const int64_t shape[5] = {L.B, (L.H + c->k - 1) / c->k, (L.W + c->k - 1) / c->k, r, L.Cin};
    if (!has_shape(c->x_hat, shape) || c->x_hat.scalar_type() != dt || !dense_on(c->x_hat, dev)) return -1;
  }
  if (!c->g_W.defined() && c->beta != 0.0) return -1;
  if (!grad_x(&c->g_x, c->g_y, L) || !grad_w(&c->g_W, c->g_y, &L, c->gw_code, dev)) return -1;
  lbp_extras ex{};
  ex.beta = static_cast<float>(c->beta);
  if (c->g_bias.defined()) {
    const at::ScalarType bt = c->g_bias.scalar_type();
    if ((bt != at::kFloat && bt != dt) || !has_shape(c->g_bias, {L.Cout}) || !dense_on(c->g_bias, dev)) return -1;
    ex.g_bias = c->g_bias.data_ptr();
    ex.g_bias_dtype = dtype_code(bt);
  }
  if (c->x_extra.defined() || c->gy_extra.defined()) {
    if (!c->x_extra.defined() || !c->gy_extra.defined() || !c->gx_extra.defined() || c->x_extra.dim() != 2) return -1;
    const int64_t n = c->x_extra.size(0);
    if (!int_size(n) || !has_shape(c->x_extra, {n, L.Cin}) || !has_shape(c->gy_extra, {n, L.Cout}) ||
        !has_shape(c->gx_extra, {n, L.Cin}) || c->x_extra.scalar_type() != dt || c->gy_extra.scalar_type() != dt ||
        c->gx_extra.scalar_type() != dt)
      return -1;
    if (n > 0) {
      if (!rows_of(c->x_extra, dev, &ex.x_extra_pitch) || !rows_of(c->gy_extra, dev, &ex.gy_extra_pitch) ||
          !rows_of(c->gx_extra, dev, &ex.gx_extra_pitch))
        return -1;
      ex.x_extra = c->x_extra.data_ptr();
      ex.gy_extra = c->gy_extra.data_ptr();
      ex.gx_extra = c->gx_extra.data_ptr();
      ex.n_extra = static_cast<int32_t>(n);
    }
  }
  if ((c->x.defined() && !view_of(c->x, dev, &ex.x_view)) || !view_of(c->g_y, dev, &ex.gy_view) ||
      !view_of(c->g_x, dev, &ex.gx_view))
    return -1;
  if (!c->ws.defined()) {
    const size_t bytes = c->grad != nullptr ? lib.workspace_bytes_act(&L, r, &ex, c->x_hat.defined() ? 1 : 0)
                         : c->x_hat.defined() ? lib.workspace_bytes_projected(&L, r, &ex)
                                              : lib.workspace_bytes_ex(&L, r, &ex);
    if (bytes == 0) return -1;
    c->ws = bytes_on(c->g_y, bytes);
  }
  if (!dense_on(c->ws, dev)) return -1;
  if (c->grad != nullptr)
    return lib.backward_act(c->x.defined() ? c->x.data_ptr() : nullptr,
                            c->x_hat.defined() ? c->x_hat.data_ptr() : nullptr, c->g_y.data_ptr(), c->W.data_ptr(),
                            c->g_x.data_ptr(), c->g_W.data_ptr(), &L, set, r, &ex, c->grad, c->ws.data_ptr(),
                            c->ws.numel(), current_stream(dev));
  return lib.backward_ex(c->x.defined() ? c->x.data_ptr() : nullptr,
                         c->x_hat.defined() ? c->x_hat.data_ptr() : nullptr, c->g_y.data_ptr(), c->W.data_ptr(),
                         c->g_x.data_ptr(), c->g_W.data_ptr(), &L, set, r, &ex, c->ws.data_ptr(), c->ws.numel(),
                         current_stream(dev));
}

// backward_ex(x, x_hat, g_y, W, k, bases, beta, g_bias, x_extra, gy_extra, gx_extra, gw_dtype, g_x, g_W, ws)
bool parse_ex(PyObject* const* a, ExCall* c, Bases* b) {
  if (!parse_tensor(a[0], &c->x) || !parse_tensor(a[1], &c->x_hat) || !parse_tensor(a[2], &c->g_y) ||
      !parse_tensor(a[3], &c->W) || !parse_int(a[4], &c->k) || !parse_bases(a[5], b) || !PyFloat_Check(a[6]) ||
      !parse_tensor(a[7], &c->g_bias) || !parse_tensor(a[8], &c->x_extra) || !parse_tensor(a[9], &c->gy_extra) ||
      !parse_tensor(a[10], &c->gx_extra) || !parse_tensor(a[12], &c->g_x) || !parse_tensor(a[13], &c->g_W) ||
      !parse_tensor(a[14], &c->ws) || (c->g_bias.defined() && c->g_bias.scalar_type() != at::kFloat))
    return false;
  c->beta = PyFloat_AS_DOUBLE(a[6]);
  c->gw_code = parse_dtype(a[11]);
  return true;
}
PyObject* py_backward_ex(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  ExCall c;
  Bases b;
  if (n != 15 || !parse_ex(a, &c, &b)) return not_handled();
  const int e = without_gil([&] { return run_ex(&c, b.v, b.r); });
  if (e < 0) return not_handled();
  return e != LBP_OK ? PyLong_FromLong(e) : pair(c.g_x, c.g_W);
  END_HANDLE_TH_ERRORS
}

// backward_batch(xs, g_ys, Ws, k, bases, g_xs, g_Ws, wss) -> 0 or a status
PyObject* py_backward_batch(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  int k = 0;
  Bases b;
  if (n != 8 || !parse_int(a[3], &k) || !parse_bases(a[4], &b)) return not_handled();
  PyObject* lists[6] = {a[0], a[1], a[2], a[5], a[6], a[7]};
  Py_ssize_t count = -1;
  for (PyObject* l : lists) {
    if (!PyList_Check(l) && !PyTuple_Check(l)) return not_handled();
    const Py_ssize_t m = PySequence_Fast_GET_SIZE(l);
    if (count >= 0 && m != count) return not_handled();
    count = m;
  }
  if (count < 1 || count > 64) return not_handled();
  std::vector<Tensor> held;   // the lists are the caller's to change once the lock is released
  held.reserve(6 * count);
  void* ptr[6][64];
  lbp_layer layers[64];
  size_t sizes[64];
  int dev = 0;
  for (Py_ssize_t i = 0; i < count; ++i) {
    Tensor t[6];
    for (int l = 0; l < 6; ++l)
      if (!parse_tensor(PySequence_Fast_GET_ITEM(lists[l], i), &t[l]) || !t[l].defined()) return not_handled();
    Problem p;
    if (!layer_of(t[1], t[2], t[0], k, &p)) return not_handled();
    dev = p.dev;
    if (!grad_x(&t[3], t[1], p.L) || !grad_w(&t[4], t[1], &p.L, -1, dev)) return not_handled();
    for (int l = 0; l < 6; ++l) {
      if (!dense_on(t[l], dev)) return not_handled();
      ptr[l][i] = t[l].data_ptr();
      held.push_back(t[l]);
    }
    layers[i] = p.L;
    sizes[i] = static_cast<size_t>(t[5].numel());
  }
  const int e = without_gil([&] {
    return lib.backward_batch(static_cast<int>(count), ptr[0], ptr[1], ptr[2], ptr[3], ptr[4], layers, b.v, b.r, ptr[5],
                              sizes, nullptr, current_stream(dev));
  });
  return PyLong_FromLong(e);
  END_HANDLE_TH_ERRORS
}

// Raises binding.LbpError(status, where) from any thread.
[[noreturn]] void raise_status(int status, const char* where) {
  pybind11::gil_scoped_acquire gil;
  PyObject* e = PyObject_CallFunction(error_type, "is", status, where);
  if (e != nullptr) {
    PyErr_SetObject(error_type, e);
    Py_DECREF(e);
  }
  python_error err;
  err.persist();
  throw err;
}

// y = x W^T (+ b);  backward: Algorithm 1 on the selected bases.  H, W: the token grid of
// a (B, n + H*W, Cin) sequence, 0: x is (B, H, W, Cin).  With save_projected the
// forward pass keeps x_hat = p(x) (Eq. 3) instead of x.
struct LinearFunction : public torch::autograd::Function<LinearFunction> {
  static Tensor forward(torch::autograd::AutogradContext* ctx, const Tensor& x, const Tensor& weight,
                        const std::optional<Tensor>& bias, int64_t k, const std::vector<int64_t>& bases,
                        bool save_projected, int64_t H, int64_t W) {
    auto& saved = ctx->saved_data;
    saved["k"] = k;
    saved["bases"] = bases;
    saved["bias"] = bias.has_value();
    saved["H"] = H;
    saved["W"] = W;
    bool projected = false;
    if (H > 0) {
      TORCH_CHECK_VALUE(x.dim() == 3 && x.size(1) >= H * W, "with a grid, x must be (B, n + H*W, Cin)");
    } else {
      TORCH_CHECK_VALUE(x.dim() == 4, "x must be (B, H, W, Cin)");
      projected = save_projected && x.is_cuda();
    }
    saved["projected"] = projected;
    if (projected) {
      const Tensor xc = x.contiguous();
      const int dt = dtype_code(xc.scalar_type()), dev = xc.get_device();
      TORCH_CHECK_TYPE(dt >= 0, "unsupported dtype ", xc.scalar_type());
      const std::vector<lbp_basis> set = unpack(bases);
      Tensor x_hat = at::empty({xc.size(0), (xc.size(1) + k - 1) / k, (xc.size(2) + k - 1) / k,
                                static_cast<int64_t>(set.size()), xc.size(3)},
                               xc.options());
      Tensor ws = bytes_on(xc, lib.status_bytes());
      const int e = lib.project(xc.data_ptr(), x_hat.data_ptr(), xc.size(0), xc.size(1), xc.size(2), xc.size(3),
                                static_cast<int>(k), set.data(), static_cast<int>(set.size()), dt, ws.data_ptr(),
                                ws.numel(), current_stream(dev));
      if (e != LBP_OK) raise_status(e, "lbp_project");
      ctx->save_for_backward({x_hat, weight});
    } else {
      ctx->save_for_backward({x, weight});
    }
    // The bias rides in the product's epilogue where that is all one type.  Otherwise (a bias
    // of another type, autocast, which casts the product's operands but not the sum's) torch's
    // rules for the two operations decide the type of y.
    const at::ScalarType dt = x.scalar_type();
    if (!bias.has_value() || (weight.scalar_type() == dt && bias->scalar_type() == dt &&
                              !at::autocast::is_autocast_enabled(x.device().type())))
      return at::linear(x, weight, bias);
    return at::matmul(x, weight.t()) + *bias;
  }

  static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx,
                                                 torch::autograd::variable_list grads) {
    at::AutoGradMode no_grad(false);
    auto& saved = ctx->saved_data;
    const auto vars = ctx->get_saved_variables();
    const std::vector<int64_t> flat = saved["bases"].toIntVector();
    const std::vector<lbp_basis> set = unpack(flat);
    const int64_t H = saved["H"].toInt(), W = saved["W"].toInt();
    const Tensor g_y = grads[0].contiguous();
    ExCall c;
    c.k = static_cast<int>(saved["k"].toInt());
    c.W = vars[1].contiguous();
    c.gw_code = dtype_code(c.W.scalar_type());
    TORCH_CHECK_TYPE(c.gw_code >= 0, "unsupported dtype ", c.W.scalar_type());
    TORCH_CHECK_VALUE(g_y.is_cuda(), "g_y must be a CUDA tensor (the library has no CPU path)");
    if (saved["bias"].toBool()) c.g_bias = at::empty({c.W.size(0)}, c.W.options());
    Tensor g_x, cls;
    int64_t n = 0;
    if (H > 0) {
      const Tensor x = vars[0].contiguous();
      const int64_t B = x.size(0);
      n = x.size(1) - H * W;
      g_x = at::empty_like(x);
      auto tokens = [&](const Tensor& t) {
        return t.as_strided({B, H, W, t.size(2)}, {t.stride(0), W * t.size(2), t.size(2), 1},
                            t.storage_offset() + n * t.size(2));
      };
      c.x = tokens(x);
      c.g_y = tokens(g_y);
      c.g_x = tokens(g_x);
      if (n == 1) {   // one class token per image: rows with the sequence's pitch, in place
        c.x_extra = x.select(1, 0);
        c.gy_extra = g_y.select(1, 0);
        c.gx_extra = g_x.select(1, 0);
      } else if (n > 1) {   // several: gathered (a few rows)
        c.x_extra = x.narrow(1, 0, n).reshape({B * n, x.size(2)});
        c.gy_extra = g_y.narrow(1, 0, n).reshape({B * n, g_y.size(2)});
        c.gx_extra = cls = at::empty({B * n, x.size(2)}, x.options());
      }
    } else {
      c.g_y = g_y;
      (saved["projected"].toBool() ? c.x_hat : c.x) = vars[0].contiguous();
    }
    const int e = run_ex(&c, set.data(), static_cast<int>(set.size()));
    TORCH_CHECK_VALUE(e >= 0, "LbpLinear: gradient, activation and weight do not fit together (shapes ",
                      g_y.sizes(), ", ", vars[0].sizes(), ", ", c.W.sizes(), "; one dtype, the current device)");
    if (e != LBP_OK) raise_status(e, "lbp_backward_ex");
    if (n > 1) g_x.narrow(1, 0, n).copy_(cls.view({g_x.size(0), n, g_x.size(2)}));
    return {H > 0 ? g_x : c.g_x, c.g_W, c.g_bias, Tensor(), Tensor(), Tensor(), Tensor(), Tensor()};
  }

  static std::vector<lbp_basis> unpack(const std::vector<int64_t>& flat) {
    std::vector<lbp_basis> v(flat.size() / 2);
    for (size_t q = 0; q < v.size(); ++q)
      v[q] = lbp_basis{static_cast<int32_t>(flat[2 * q]), static_cast<int32_t>(flat[2 * q + 1])};
    return v;
  }
};

// Whether torch's functions on a tensor of this type give tensors of it (unless the class has
// switched that off).
bool makes_subclasses(PyTypeObject* type) {
  const pybind11::object off = pybind11::module_::import("torch._C").attr("_disabled_torch_function_impl");
  return !pybind11::getattr(reinterpret_cast<PyObject*>(type), "__torch_function__", off).is(off);
}

// y, as a subclass where one is among the n operands, as under torch's own functions.
PyObject* wrap_like(const Tensor& y, PyObject* const* a, int n) {
  PyObject* out = THPVariable_Wrap(y);
  for (int i = 0; i < n && out != nullptr && THPVariable_CheckExact(out); ++i)
    if (THPVariable_Check(a[i]) && !THPVariable_CheckExact(a[i]) && makes_subclasses(Py_TYPE(a[i]))) {
      PyObject* as = PyObject_CallMethod(out, "as_subclass", "O", Py_TYPE(a[i]));
      Py_DECREF(out);
      out = as;
    }
  return out;
}

// LinearFunction under autocast too: the backward pass wants x, weight and g_y of one type, which is that of y, so where
// one is to follow x and weight are brought to it first.  (The product rounds them to autocast's type either way.  Not by
// autocast's cache, whose entry may have been made under no_grad.)
Tensor plain_layer(Tensor x, Tensor weight, const Tensor& bias, int k, const std::vector<int64_t>& bases, bool projected, int H,
                   int W) {
  const bool backward = at::GradMode::is_enabled() && (x.requires_grad() || weight.requires_grad() || (bias.defined() && bias.requires_grad()));
  if (backward && x.is_cuda() && at::autocast::is_autocast_enabled(at::kCUDA)) {
    const at::ScalarType t = at::autocast::get_autocast_dtype(at::kCUDA);
    const at::ScalarType of_y = bias.defined() ? c10::promoteTypes(t, bias.scalar_type()) : t;
    if (dtype_code(of_y) >= 0)
      for (Tensor* v : {&x, &weight})
        if (v->is_floating_point() && v->scalar_type() != at::kDouble) *v = v->to(of_y);   // (autocast passes doubles over)
  }
  return LinearFunction::apply(x, weight, bias.defined() ? std::optional<Tensor>(bias) : std::nullopt, static_cast<int64_t>(k),
                               bases, projected, static_cast<int64_t>(H), static_cast<int64_t>(W));
}

// linear(x, weight, bias | None, k, bases, save_projected, H, W) -> y
PyObject* py_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Tensor x, weight, bias;
  int k = 0, H = 0, W = 0;
  Bases b;
  if (n != 8 || !parse_tensor(a[0], &x) || !parse_tensor(a[1], &weight) || !parse_tensor(a[2], &bias) ||
      !parse_int(a[3], &k) || k < 1 || !parse_bases(a[4], &b) || !parse_int(a[6], &H) || !parse_int(a[7], &W) ||
      !x.defined() || !weight.defined() || (H > 0) != (W > 0)) {
    PyErr_SetString(PyExc_ValueError,
                    "linear: x and weight are tensors, bases a list of (i, j) pairs, k and the grid positive");
    return nullptr;
  }
  std::vector<int64_t> flat(2 * b.r);
  for (int q = 0; q < b.r; ++q) {
    flat[2 * q] = b.v[q].i;
    flat[2 * q + 1] = b.v[q].j;
  }
  const bool projected = PyObject_IsTrue(a[5]) == 1;
  Tensor y;
  {
    pybind11::gil_scoped_release no_gil;
    y = plain_layer(x, weight, bias, k, flat, projected, H, W);
  }
  return wrap_like(y, a, 3);
  END_HANDLE_TH_ERRORS
}

// ---- what a layer does around its product ----
bool parse_act(PyObject* o, int32_t* act) {
  static const char* const names[] = {"none", "relu", "gelu", "gelu_tanh", "silu"};
  *act = LBP_ACT_NONE;
  if (o == Py_None) return true;
  if (!PyUnicode_Check(o)) return false;
  for (int i = 0; i < 5; ++i)
    if (PyUnicode_CompareWithASCIIString(o, names[i]) == 0) {
      *act = i;
      return true;
    }
  return false;
}
bool parse_u64(PyObject* o, uint64_t* v) {
  if (!PyLong_Check(o)) return false;
  *v = PyLong_AsUnsignedLongLong(o);
  if (PyErr_Occurred() == nullptr) return true;
  PyErr_Clear();
  return false;
}
// p, seed, offset, rng (the last an undefined tensor for None; it has to outlive the call)
bool parse_drop(PyObject* const* a, lbp_epilogue* e, Tensor* rng) {
  if (PyFloat_Check(a[0]))
    e->p = static_cast<float>(PyFloat_AS_DOUBLE(a[0]));
  else if (PyLong_CheckExact(a[0]))
    e->p = static_cast<float>(PyLong_AsDouble(a[0]));
  else
    return false;
  if (PyErr_Occurred() != nullptr) {
    PyErr_Clear();
    return false;
  }
  return e->p >= 0.f && e->p <= 1.f && parse_u64(a[1], &e->seed) && parse_u64(a[2], &e->offset) && parse_tensor(a[3], rng);
}
// The numbers' state in device memory, {seed, offset}.
bool use_rng(const Tensor& rng, int dev, lbp_epilogue* e) {
  if (!rng.defined()) return true;
  if (rng.scalar_type() != at::kLong || rng.numel() != 2 || !dense_on(rng, dev) || e->seed != 0) return false;
  e->seed_dev = static_cast<const uint64_t*>(rng.data_ptr());
  e->offset_dev = e->seed_dev + 1;
  return true;
}
// Rows of the last dimension at one distance (0: dense).
bool matrix_of(const Tensor& t, int dev, int64_t* pitch) {
  *pitch = 0;
  if (!t.is_cuda() || t.get_device() != dev || t.dim() < 1) return false;
  if (t.is_contiguous()) return true;
  const int64_t last = t.dim() - 1, C = t.size(last);
  if (C > 1 && t.stride(last) != 1) return false;
  int64_t after = -1;
  for (int64_t d = last - 1; d >= 0; --d) {
    const int64_t n = t.size(d);
    if (n == 1) continue;
    if (after < 0)
      *pitch = t.stride(d);
    else if (t.stride(d) != after)
      return false;
    after = t.stride(d) * n;
  }
  return after < 0 || *pitch >= C;
}
// A matrix like another: its pitch, 0 for an undefined one.
bool matrix_like(const Tensor& t, const Tensor& like, at::IntArrayRef shape, int dev, int64_t* pitch) {
  *pitch = 0;
  return !t.defined() || (t.scalar_type() == like.scalar_type() && t.sizes() == shape && matrix_of(t, dev, pitch));
}
void* data_or_null(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
bool on_current_device(const Tensor& t) { return t.defined() && t.is_cuda() && t.get_device() == c10::cuda::current_device(); }

// A workspace for calls that need no more than a status block and whose caller has not given one, so that nobody polls
// it: one for each device, which is written to only where a wait expires (an allocation takes a fifth of such a call).
// Inside a stream capture a block of its own: memory of a capture's pool is the graph's.
Tensor status_block(const Tensor& like) {
  static std::mutex mu;
  static auto* const blocks = new std::vector<Tensor>(64);   // (never freed: the driver may be gone at exit)
  const int dev = like.get_device();
  const int64_t bytes = static_cast<int64_t>(lib.status_bytes());
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  const bool free_to = dev < 64 && cudaStreamIsCapturing(c10::cuda::getCurrentCUDAStream(dev).stream(), &capture) == cudaSuccess &&
                       capture == cudaStreamCaptureStatusNone;
  std::lock_guard<std::mutex> lock(mu);
  if (dev < 64 && (*blocks)[dev].defined()) return (*blocks)[dev];
  Tensor block = fresh({bytes}, at::kByte, like);
  if (free_to) (*blocks)[dev] = block;
  return block;
}

struct LinearArgs {
  Tensor x, W, bias, residual, out, z, ws;
  bool save_z = false;
};
// Returns the library's status, or -1 where a check does not hold (nothing done).
int run_linear(LinearArgs* c, const lbp_epilogue& e) {
  if (!on_current_device(c->x) || !c->W.defined() || c->W.dim() != 2 || c->x.dim() < 1) return -1;
  const int dt = dtype_code(c->x.scalar_type()), dev = c->x.get_device();
  const int64_t Cout = c->W.size(0), Cin = c->W.size(1);
  if (dt < 0 || c->x.size(-1) != Cin || Cin < 1 || !int_size(Cin) || !int_size(Cout) ||
      c->W.scalar_type() != c->x.scalar_type() || !dense_on(c->W, dev))
    return -1;
  if (c->bias.defined() && (c->bias.scalar_type() != c->x.scalar_type() || !has_shape(c->bias, {Cout}) || !dense_on(c->bias, dev)))
    return -1;
  c10::SmallVector<int64_t, 8> shape(c->x.sizes().begin(), c->x.sizes().end());
  shape.back() = Cout;
  const int64_t rows = c->x.numel() / Cin;
  if (!c->out.defined()) c->out = fresh(shape, c->x.scalar_type(), c->x);
  if (!c->z.defined() && c->save_z) c->z = fresh(shape, c->x.scalar_type(), c->x);
  lbp_pitches p{};
  if (!matrix_of(c->x, dev, &p.x) || !matrix_like(c->residual, c->x, shape, dev, &p.residual) ||
      !matrix_like(c->out, c->x, shape, dev, &p.y) || !matrix_like(c->z, c->x, shape, dev, &p.z))
    return -1;
  if (!c->ws.defined()) {
    const size_t bytes = lib.linear_workspace_bytes(rows, static_cast<int>(Cin), static_cast<int>(Cout), dt);
    if (bytes == 0) return -1;
    c->ws = bytes <= lib.status_bytes() ? status_block(c->x) : fresh({static_cast<int64_t>(bytes)}, at::kByte, c->x);
  }
  if (!dense_on(c->ws, dev)) return -1;
  return lib.linear(c->x.data_ptr(), c->W.data_ptr(), data_or_null(c->bias), data_or_null(c->residual), c->out.data_ptr(),
                    data_or_null(c->z), rows, static_cast<int>(Cin), static_cast<int>(Cout), dt, &p, &e, c->ws.data_ptr(),
                    c->ws.nbytes(), current_stream(dev));
}

// linear_forward(x, W, bias, activation, residual, p, seed, offset, rng, save_z, out, z, ws)
PyObject* py_linear_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  LinearArgs c;
  lbp_epilogue e{};
  Tensor rng;
  if (n != 13 || !parse_tensor(a[0], &c.x) || !parse_tensor(a[1], &c.W) || !parse_tensor(a[2], &c.bias) ||
      !parse_act(a[3], &e.act) || !parse_tensor(a[4], &c.residual) || !parse_drop(a + 5, &e, &rng) ||
      !parse_tensor(a[10], &c.out) || !parse_tensor(a[11], &c.z) || !parse_tensor(a[12], &c.ws) ||
      !on_current_device(c.x) || !use_rng(rng, c.x.get_device(), &e))
    return not_handled();
  const int save_z = PyObject_IsTrue(a[9]);
  if (save_z < 0) return nullptr;
  c.save_z = save_z == 1;
  const int s = without_gil([&] { return run_linear(&c, e); });
  if (s < 0) return not_handled();
  return s != LBP_OK ? PyLong_FromLong(s) : c.z.defined() ? pair(c.out, c.z) : THPVariable_Wrap(c.out);
  END_HANDLE_TH_ERRORS
}

// The pointwise calls: drop(a) with act'(b) or + b.  -1: not handled.
int run_pointwise(const Tensor& a, const Tensor& b, Tensor* out, const lbp_epilogue& e, bool grad) {
  if (!on_current_device(a) || a.dim() < 1) return -1;
  const int dt = dtype_code(a.scalar_type()), dev = a.get_device();
  const int64_t C = a.size(-1);
  if (dt < 0 || C < 1 || !int_size(C)) return -1;
  if (!out->defined()) *out = fresh(a.sizes(), a.scalar_type(), a);
  int64_t pa, pb, po;
  if (!matrix_of(a, dev, &pa) || !matrix_like(b, a, a.sizes(), dev, &pb) || !matrix_like(*out, a, a.sizes(), dev, &po))
    return -1;
  const int64_t rows = a.numel() / C;
  if (grad) {
    if (e.act != LBP_ACT_NONE && !b.defined()) return -1;
    const lbp_pitches p{po, 0, pa, pb};
    return lib.linear_grad(a.data_ptr(), data_or_null(b), out->data_ptr(), rows, static_cast<int>(C), dt, &p, &e,
                           current_stream(dev));
  }
  const lbp_pitches p{pa, pb, po, 0};
  return lib.dropout(a.data_ptr(), data_or_null(b), out->data_ptr(), rows, static_cast<int>(C), dt, &p, &e,
                     current_stream(dev));
}

// linear_grad(g_y, z, activation, p, seed, offset, rng, out)
PyObject* py_linear_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Tensor g_y, z, out, rng;
  lbp_epilogue e{};
  if (n != 8 || !parse_tensor(a[0], &g_y) || !parse_tensor(a[1], &z) || !parse_act(a[2], &e.act) ||
      !parse_drop(a + 3, &e, &rng) || !parse_tensor(a[7], &out) || !on_current_device(g_y) ||
      !use_rng(rng, g_y.get_device(), &e))
    return not_handled();
  const int s = without_gil([&] { return run_pointwise(g_y, z, &out, e, true); });
  if (s < 0) return not_handled();
  return s != LBP_OK ? PyLong_FromLong(s) : THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

// dropout(x, p, seed, offset, rng, residual, out)
PyObject* py_dropout(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Tensor x, residual, out, rng;
  lbp_epilogue e{};
  if (n != 7 || !parse_tensor(a[0], &x) || !parse_drop(a + 1, &e, &rng) || !parse_tensor(a[5], &residual) ||
      !parse_tensor(a[6], &out) || !on_current_device(x) || !use_rng(rng, x.get_device(), &e))
    return not_handled();
  const int s = without_gil([&] { return run_pointwise(x, residual, &out, e, false); });
  if (s < 0) return not_handled();
  return s != LBP_OK ? PyLong_FromLong(s) : THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

// project_grad(g_y, z, k, bases, activation, p, seed, offset, rng, out, ws)
PyObject* py_project_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Tensor g_y, z, rng, out, ws;
  int k = 0;
  Bases b;
  lbp_epilogue e{};
  lbp_view v, vz;
  if (n != 11 || !parse_tensor(a[0], &g_y) || !parse_tensor(a[1], &z) || !parse_int(a[2], &k) || !parse_bases(a[3], &b) ||
      !parse_act(a[4], &e.act) || !parse_drop(a + 5, &e, &rng) || !parse_tensor(a[9], &out) || !parse_tensor(a[10], &ws) ||
      !on_current_device(g_y) || g_y.dim() != 4 || k < 1)
    return not_handled();
  const int dt = dtype_code(g_y.scalar_type()), dev = g_y.get_device();
  if (dt < 0 || !view_of(g_y, dev, &v) || !use_rng(rng, dev, &e)) return not_handled();
  for (int i = 0; i < 4; ++i)
    if (!int_size(g_y.size(i))) return not_handled();
  if (z.defined() ? z.scalar_type() != g_y.scalar_type() || z.sizes() != g_y.sizes() || !view_of(z, dev, &vz) ||
                        vz.image != v.image || vz.row != v.row || vz.token != v.token
                  : e.act != LBP_ACT_NONE)
    return not_handled();
  const int64_t shape[5] = {g_y.size(0), (g_y.size(1) + k - 1) / k, (g_y.size(2) + k - 1) / k, b.r, g_y.size(3)};
  if (!out.defined())
    out = fresh(shape, g_y.scalar_type(), g_y);
  else if (!has_shape(out, shape) || out.scalar_type() != g_y.scalar_type() || !dense_on(out, dev))
    return not_handled();
  if (!ws.defined()) {
    const size_t bytes = lib.project_grad_workspace_bytes(g_y.size(0), g_y.size(1), g_y.size(2), g_y.size(3), k, b.r, dt);
    if (bytes == 0) return not_handled();
    ws = fresh({static_cast<int64_t>(bytes)}, at::kByte, g_y);
  }
  if (!dense_on(ws, dev)) return not_handled();
  const int s = without_gil([&] {
    return lib.project_grad(g_y.data_ptr(), data_or_null(z), out.data_ptr(), g_y.size(0), g_y.size(1), g_y.size(2),
                            g_y.size(3), k, b.v, b.r, dt, &v, &e, ws.data_ptr(), ws.nbytes(), current_stream(dev));
  });
  return s != LBP_OK ? PyLong_FromLong(s) : THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

bool parse_i64(PyObject* o, int64_t* v) {
  if (!PyLong_Check(o)) return false;
  *v = PyLong_AsLongLong(o);
  if (PyErr_Occurred() == nullptr) return true;
  PyErr_Clear();
  return false;
}

// backward_act(the fifteen of backward_ex, z, activation, p, seed, offset, rng, z_extra, first, number, first_extra,
//              number_extra)
PyObject* py_backward_act(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  ExCall c;
  Bases b;
  Tensor z, z_extra, rng;
  lbp_layer_grad g{};
  lbp_epilogue& e = g.epilogue;
  if (n != 26 || !parse_ex(a, &c, &b) || !parse_tensor(a[15], &z) || !parse_act(a[16], &e.act) ||
      !parse_drop(a + 17, &e, &rng) || !parse_tensor(a[21], &z_extra) || !parse_i64(a[22], &e.first) ||
      !parse_i64(a[24], &g.first_extra) || !parse_i64(a[25], &g.number_extra) || !on_current_device(c.g_y) ||
      !use_rng(rng, c.g_y.get_device(), &e))
    return not_handled();
  if (a[23] != Py_None) {
    if (!PyTuple_Check(a[23]) || PyTuple_GET_SIZE(a[23]) != 3 || !parse_i64(PyTuple_GET_ITEM(a[23], 0), &e.number.image) ||
        !parse_i64(PyTuple_GET_ITEM(a[23], 1), &e.number.row) || !parse_i64(PyTuple_GET_ITEM(a[23], 2), &e.number.token))
      return not_handled();
  }
  const int dev = c.g_y.get_device();
  if (z.defined()) {
    lbp_view v, vz;
    if (z.scalar_type() != c.g_y.scalar_type() || z.sizes() != c.g_y.sizes() || !view_of(c.g_y, dev, &v) ||
        !view_of(z, dev, &vz) || vz.image != v.image || vz.row != v.row || vz.token != v.token)
      return not_handled();
    g.z = z.data_ptr();
  } else if (e.act != LBP_ACT_NONE) {
    return not_handled();
  }
  if (z_extra.defined()) {
    int64_t pitch, pz;
    if (!c.gy_extra.defined() || z_extra.scalar_type() != c.g_y.scalar_type() || z_extra.sizes() != c.gy_extra.sizes() ||
        z_extra.dim() != 2 || !rows_of(c.gy_extra, dev, &pitch) || !rows_of(z_extra, dev, &pz) || pz != pitch)
      return not_handled();
    g.z_extra = z_extra.data_ptr();
  }
  c.grad = &g;
  const int s = without_gil([&] { return run_ex(&c, b.v, b.r); });
  if (s < 0) return not_handled();
  return s != LBP_OK ? PyLong_FromLong(s) : pair(c.g_x, c.g_W);
  END_HANDLE_TH_ERRORS
}

// The state that one forward pass draws its numbers from: torch's generator of the device, so
// that torch.manual_seed and a captured graph's replays have the meaning they have for torch's
// own dropout.
struct Drawn {
  bool captured = false;
  uint64_t seed = 0, offset = 0;
  const uint64_t *seed_dev = nullptr, *offset_dev = nullptr;
};
Drawn draw_state(int dev) {
  at::Generator gen = at::cuda::detail::getDefaultCUDAGenerator(static_cast<c10::DeviceIndex>(dev));
  at::PhiloxCudaState s;
  {
    std::lock_guard<std::mutex> lock(gen.mutex());
    s = at::check_generator<at::CUDAGeneratorImpl>(gen)->philox_cuda_state(4);
  }
  Drawn d;
  d.captured = s.captured_;
  if (s.captured_) {
    d.seed_dev = reinterpret_cast<const uint64_t*>(s.seed_.ptr);
    d.offset_dev = reinterpret_cast<const uint64_t*>(s.offset_.ptr);
    d.offset = s.offset_intragraph_;
  } else {
    d.seed = s.seed_.val;
    d.offset = s.offset_.val;
  }
  return d;
}

// y = residual + drop(act(x W^T + b)) with the gradient of the product by Algorithm 1: LinearFunction
// with an epilogue.  The forward product is the library's too.
struct LayerFunction : public torch::autograd::Function<LayerFunction> {
  // What the forward pass computes; z is kept where a backward pass is to follow and needs it.
  static Tensor compute(const Tensor& x, const Tensor& weight, const std::optional<Tensor>& bias,
                        const std::optional<Tensor>& residual, int64_t act, double p, const Drawn& d, Tensor* z,
                        Tensor* used) {
    LinearArgs c;
    lbp_epilogue e{};
    e.act = static_cast<int32_t>(act);
    e.p = static_cast<float>(p);
    e.seed = d.seed;
    e.offset = d.offset;
    e.seed_dev = d.seed_dev;
    e.offset_dev = d.offset_dev;
    if (used != nullptr && d.captured) {
      *used = at::empty({2}, x.options().dtype(at::kLong));
      e.used = static_cast<uint64_t*>(used->data_ptr());
    }
    c.x = x.contiguous();
    c.W = weight.contiguous();
    if (bias.has_value()) c.bias = bias->contiguous();
    if (residual.has_value()) c.residual = residual->contiguous();
    c.save_z = z != nullptr && act != LBP_ACT_NONE;
    const int s = run_linear(&c, e);
    TORCH_CHECK_VALUE(s >= 0, "LbpLinear: x ", x.sizes(), " ", x.scalar_type(), ", weight ", weight.sizes(), " ",
                      weight.scalar_type(), ", bias and residual do not fit together (CUDA tensors of one dtype, "
                      "fp32 or bf16, on the current device; residual of the output's shape)");
    if (s != LBP_OK) raise_status(s, "lbp_linear");
    if (z != nullptr) *z = c.z;
    return c.out;
  }

  static Tensor forward(torch::autograd::AutogradContext* ctx, const Tensor& x, const Tensor& weight,
                        const std::optional<Tensor>& bias, const std::optional<Tensor>& residual, int64_t k,
                        const std::vector<int64_t>& bases, bool save_projected, int64_t H, int64_t W, int64_t act,
                        double p) {
    auto& saved = ctx->saved_data;
    saved["k"] = k;
    saved["bases"] = bases;
    saved["bias"] = bias.has_value();
    saved["residual"] = residual.has_value();
    saved["H"] = H;
    saved["W"] = W;
    saved["act"] = act;
    saved["p"] = p;
    const Drawn d = p > 0.0 ? draw_state(x.get_device()) : Drawn{};
    saved["seed"] = static_cast<int64_t>(d.seed);
    saved["offset"] = static_cast<int64_t>(d.offset);
    Tensor z, used, kept = x;
    const Tensor y = compute(x, weight, bias, residual, act, p, d, &z, &used);
    const bool projected = H <= 0 && save_projected;
    if (projected) {
      const Tensor xc = x.contiguous();
      const std::vector<lbp_basis> set = LinearFunction::unpack(bases);
      kept = at::empty({xc.size(0), (xc.size(1) + k - 1) / k, (xc.size(2) + k - 1) / k, static_cast<int64_t>(set.size()),
                        xc.size(3)},
                       xc.options());
      Tensor ws = bytes_on(xc, lib.status_bytes());
      const int s = lib.project(xc.data_ptr(), kept.data_ptr(), xc.size(0), xc.size(1), xc.size(2), xc.size(3),
                                static_cast<int>(k), set.data(), static_cast<int>(set.size()),
                                dtype_code(xc.scalar_type()), ws.data_ptr(), ws.numel(), current_stream(xc.get_device()));
      if (s != LBP_OK) raise_status(s, "lbp_project");
    }
    saved["projected"] = projected;
    ctx->save_for_backward({kept, weight, z, used});
    return y;
  }

  static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx,
                                                 torch::autograd::variable_list grads) {
    at::AutoGradMode no_grad(false);
    auto& saved = ctx->saved_data;
    const auto vars = ctx->get_saved_variables();
    const std::vector<lbp_basis> set = LinearFunction::unpack(saved["bases"].toIntVector());
    const int64_t H = saved["H"].toInt(), W = saved["W"].toInt();
    TORCH_CHECK_VALUE(grads[0].is_cuda(), "g_y must be a CUDA tensor (the library has no CPU path)");
    Tensor g_y = grads[0].contiguous();
    Tensor z = vars[2];
    const Tensor used = vars[3];
    lbp_layer_grad g{};
    g.epilogue.act = static_cast<int32_t>(saved["act"].toInt());
    g.epilogue.p = static_cast<float>(saved["p"].toDouble());
    g.epilogue.seed = static_cast<uint64_t>(saved["seed"].toInt());
    g.epilogue.offset = static_cast<uint64_t>(saved["offset"].toInt());
    if (used.defined()) {   // captured: what the forward pass has noted
      g.epilogue.seed_dev = static_cast<const uint64_t*>(used.data_ptr());
      g.epilogue.offset_dev = g.epilogue.seed_dev + 1;
      g.epilogue.offset = 0;
    }
    ExCall c;
    c.k = static_cast<int>(saved["k"].toInt());
    c.W = vars[1].contiguous();
    c.gw_code = dtype_code(c.W.scalar_type());
    if (saved["bias"].toBool()) c.g_bias = at::empty({c.W.size(0)}, c.W.options());
    Tensor g_x, cls;
    int64_t n = 0;
    const int64_t C = c.W.size(0);
    if (H > 0) {
      const Tensor x = vars[0].contiguous();
      const int64_t B = x.size(0);
      n = x.size(1) - H * W;
      g_x = at::empty_like(x);
      const bool changed = g.epilogue.act != LBP_ACT_NONE || g.epilogue.p > 0.f;
      if (n > 1 && changed) {   // numbers of the extra tokens are no arithmetic series: the whole sequence at once
        Tensor g_z;
        const int s = run_pointwise(g_y, z, &g_z, g.epilogue, true);
        TORCH_CHECK_VALUE(s >= 0, "LbpLinear: gradient and kept activation do not fit together");
        if (s != LBP_OK) raise_status(s, "lbp_linear_grad");
        g_y = g_z;
        g = lbp_layer_grad{};
        z = Tensor();
      }
      auto tokens = [&](const Tensor& t) {
        return t.as_strided({B, H, W, t.size(2)}, {t.stride(0), W * t.size(2), t.size(2), 1},
                            t.storage_offset() + n * t.size(2));
      };
      c.x = tokens(x);
      c.g_y = tokens(g_y);
      c.g_x = tokens(g_x);
      if (z.defined()) g.z = tokens(z).data_ptr();
      g.epilogue.first = n * C;
      g.epilogue.number = lbp_view{(n + H * W) * C, W * C, C};
      if (n == 1) {
        c.x_extra = x.select(1, 0);
        c.gy_extra = g_y.select(1, 0);
        c.gx_extra = g_x.select(1, 0);
        if (z.defined()) g.z_extra = z.data_ptr();
        g.number_extra = (1 + H * W) * C;
      } else if (n > 1) {
        c.x_extra = x.narrow(1, 0, n).reshape({B * n, x.size(2)});
        c.gy_extra = g_y.narrow(1, 0, n).reshape({B * n, g_y.size(2)});
        c.gx_extra = cls = at::empty({B * n, x.size(2)}, x.options());
      }
    } else {
      c.g_y = g_y;
      if (z.defined()) g.z = z.data_ptr();
      (saved["projected"].toBool() ? c.x_hat : c.x) = vars[0].contiguous();
    }
    c.grad = &g;
    const int e = run_ex(&c, set.data(), static_cast<int>(set.size()));
    TORCH_CHECK_VALUE(e >= 0, "LbpLinear: gradient, activation and weight do not fit together (shapes ", g_y.sizes(),
                      ", ", vars[0].sizes(), ", ", c.W.sizes(), "; one dtype, the current device)");
    if (e != LBP_OK) raise_status(e, "lbp_backward_act");
    if (n > 1) g_x.narrow(1, 0, n).copy_(cls.view({g_x.size(0), n, g_x.size(2)}));
    return {H > 0 ? g_x : c.g_x, c.g_W, c.g_bias, saved["residual"].toBool() ? grads[0] : Tensor(), Tensor(), Tensor(),
            Tensor(), Tensor(), Tensor(), Tensor(), Tensor()};
  }
};

// layer(x, weight, bias | None, residual | None, k, bases, save_projected, H, W, activation, p) -> y
PyObject* py_layer(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Tensor x, weight, bias, residual;
  int k = 0, H = 0, W = 0;
  int32_t act = 0;
  Bases b;
  if (n != 11 || !parse_tensor(a[0], &x) || !parse_tensor(a[1], &weight) || !parse_tensor(a[2], &bias) ||
      !parse_tensor(a[3], &residual) || !parse_int(a[4], &k) || k < 1 || !parse_bases(a[5], &b) || !parse_int(a[7], &H) ||
      !parse_int(a[8], &W) || !parse_act(a[9], &act) || !PyFloat_Check(a[10]) || !x.defined() || !weight.defined() ||
      (H > 0) != (W > 0)) {
    PyErr_SetString(PyExc_ValueError,
                    "layer: x, weight and residual are tensors, bases a list of (i, j) pairs, k and the grid positive");
    return nullptr;
  }
  const double p = PyFloat_AS_DOUBLE(a[10]);
  const bool projected = PyObject_IsTrue(a[6]) == 1;
  std::vector<int64_t> flat(2 * b.r);
  for (int q = 0; q < b.r; ++q) {
    flat[2 * q] = b.v[q].i;
    flat[2 * q + 1] = b.v[q].j;
  }
  Tensor y;
  {
    pybind11::gil_scoped_release no_gil;
    TORCH_CHECK_VALUE(x.is_cuda(), "x must be a CUDA tensor (the library has no CPU path)");
    TORCH_CHECK_VALUE(p >= 0.0 && p <= 1.0, "dropout is a probability, got ", p);
    // (the calls below that go past the autograd function would leave a tangent behind)
    for (const Tensor* v : {&x, &weight, &bias, &residual})
      TORCH_CHECK_NOT_IMPLEMENTED(!v->defined() || !v->_fw_grad(/*level=*/0).defined(),
                                  "LbpLinear has no forward-mode derivative");
    TORCH_CHECK_VALUE(H == 0 || (x.dim() == 3 && x.size(1) >= static_cast<int64_t>(H) * W),
                      "with a grid, x must be (B, n + H*W, Cin)");
    TORCH_CHECK_VALUE(H > 0 || x.dim() == 4, "x must be (B, H, W, Cin)");
    const auto opt = [](const Tensor& t) { return t.defined() ? std::optional<Tensor>(t) : std::nullopt; };
    // Under autocast the product's operands and the bias are of its type, as for torch's own linear layer.  A residual
    // stream keeps its own, and the sum with it follows torch's rules, as it does behind torch's layer.
    Tensor stream;
    if (at::autocast::is_autocast_enabled(at::kCUDA)) {
      const at::ScalarType t = at::autocast::get_autocast_dtype(at::kCUDA);
      if (residual.defined() && residual.scalar_type() != t) {
        c10::SmallVector<int64_t, 8> shape(x.sizes().begin(), x.sizes().end());
        shape.back() = weight.dim() == 2 ? weight.size(0) : -1;
        TORCH_CHECK_VALUE(residual.is_floating_point() && residual.sizes() == shape && residual.device() == x.device(),
                          "LbpLinear: residual ", residual.sizes(), " ", residual.scalar_type(), " on ", residual.device(),
                          " must have the output's shape ", at::IntArrayRef(shape), " and device");
        std::swap(stream, residual);
      }
      if (!stream.defined() || act != LBP_ACT_NONE || p > 0.0)
        for (Tensor* v : {&x, &weight, &bias})
          if (v->defined() && v->is_floating_point()) *v = v->to(t);
    }
    bool backward = false;
    if (at::GradMode::is_enabled())
      for (const Tensor* v : {&x, &weight, &bias, &residual}) backward |= v->defined() && v->requires_grad();
    if (stream.defined() && act == LBP_ACT_NONE && p == 0.0)   // nothing else follows the product: the plain layer's
      y = plain_layer(x, weight, bias, k, flat, projected, H, W);
    else if (backward)
      y = LayerFunction::apply(x, weight, opt(bias), opt(residual), static_cast<int64_t>(k), flat, projected,
                               static_cast<int64_t>(H), static_cast<int64_t>(W), static_cast<int64_t>(act), p);
    else
      y = LayerFunction::compute(x, weight, opt(bias), opt(residual), act, p, p > 0.0 ? draw_state(x.get_device()) : Drawn{},
                                 nullptr, nullptr);
    if (stream.defined()) y = stream + y;
  }
  return wrap_like(y, a, 4);
  END_HANDLE_TH_ERRORS
}

// What a Python autograd function shows of the node: y.grad_fn.saved_tensors.
PyObject* node_saved_tensors(PyObject* self, void*) {
  HANDLE_TH_ERRORS
  using Node = torch::autograd::CppNode<LinearFunction>;
  auto* node = dynamic_cast<Node*>(reinterpret_cast<torch::autograd::THPCppFunction*>(self)->cdata.get());
  if (node == nullptr) {
    PyErr_SetString(PyExc_RuntimeError, "saved_tensors: not a node of LbpLinear");
    return nullptr;
  }
  const auto vars = node->ctx_.get_saved_variables();
  PyObject* t = PyTuple_New(static_cast<Py_ssize_t>(vars.size()));
  if (t == nullptr) return nullptr;
  for (size_t i = 0; i < vars.size(); ++i) PyTuple_SET_ITEM(t, i, THPVariable_Wrap(vars[i]));
  return t;
  END_HANDLE_TH_ERRORS
}
void register_node_type() {
  using namespace torch::autograd;
  static PyTypeObject type;
  static PyGetSetDef properties[] = {
      {const_cast<char*>("saved_tensors"), node_saved_tensors, nullptr, nullptr, nullptr},
      THP_FUNCTION_DEFAULT_PROPERTIES,
      {nullptr, nullptr, nullptr, nullptr, nullptr}};
  torch::autograd::_initFunctionPyTypeObject(type, "LbpLinearBackward", properties, nullptr);
  torch::autograd::registerCppFunction(typeid(torch::autograd::CppNode<LinearFunction>), &type);
}

// load(path of liblbp.so, LbpError)
PyObject* py_load(PyObject*, PyObject* args) {
  const char* path = nullptr;
  PyObject* err = nullptr;
  if (!PyArg_ParseTuple(args, "sO", &path, &err)) return nullptr;
  void* h = dlopen(path, RTLD_NOW | RTLD_LOCAL);
  if (h == nullptr) {
    PyErr_SetString(PyExc_RuntimeError, dlerror());
    return nullptr;
  }
  const bool ok = resolve(h, "lbp_status_string", &lib.status_string) &&
                  resolve(h, "lbp_status_bytes", &lib.status_bytes) &&
                  resolve(h, "lbp_workspace_bytes", &lib.workspace_bytes) &&
                  resolve(h, "lbp_workspace_bytes_ex", &lib.workspace_bytes_ex) &&
                  resolve(h, "lbp_workspace_bytes_projected", &lib.workspace_bytes_projected) &&
                  resolve(h, "lbp_spectrum_workspace_bytes", &lib.spectrum_workspace_bytes) &&
                  resolve(h, "lbp_project", &lib.project) && resolve(h, "lbp_spectrum", &lib.spectrum) &&
                  resolve(h, "lbp_backward", &lib.backward) && resolve(h, "lbp_backward_ex", &lib.backward_ex) &&
                  resolve(h, "lbp_backward_batch", &lib.backward_batch) &&
                  resolve(h, "lbp_backward_fullrank", &lib.backward_fullrank) &&
                  resolve(h, "lbp_linear_workspace_bytes", &lib.linear_workspace_bytes) &&
                  resolve(h, "lbp_linear", &lib.linear) && resolve(h, "lbp_linear_grad", &lib.linear_grad) &&
                  resolve(h, "lbp_dropout", &lib.dropout) &&
                  resolve(h, "lbp_project_grad_workspace_bytes", &lib.project_grad_workspace_bytes) &&
                  resolve(h, "lbp_project_grad", &lib.project_grad) &&
                  resolve(h, "lbp_workspace_bytes_act", &lib.workspace_bytes_act) &&
                  resolve(h, "lbp_backward_act", &lib.backward_act);
  if (!ok) {
    PyErr_Format(PyExc_RuntimeError, "%s does not export what this binding calls", path);
    return nullptr;
  }
  if (error_type == nullptr) register_node_type();
  Py_INCREF(err);
  Py_XSETREF(error_type, err);
  Py_RETURN_NONE;
}

#define LBP_FAST(name, fn) \
  {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fn)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"load", py_load, METH_VARARGS, nullptr},
                         LBP_FAST("project", py_project),
                         LBP_FAST("spectrum", py_spectrum),
                         LBP_FAST("backward", py_backward),
                         LBP_FAST("backward_ex", py_backward_ex),
                         LBP_FAST("backward_batch", py_backward_batch),
                         LBP_FAST("linear", py_linear),
                         LBP_FAST("layer", py_layer),
                         LBP_FAST("linear_forward", py_linear_forward),
                         LBP_FAST("linear_grad", py_linear_grad),
                         LBP_FAST("dropout", py_dropout),
                         LBP_FAST("project_grad", py_project_grad),
                         LBP_FAST("backward_act", py_backward_act),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lbp_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lbp_torch() { return PyModule_Create(&module); }

// Argument checks of the expert-layer calls (include/taccl.h) on torch tensors,
// and the calls. In Python the checks took longer than the launch: 4.2 us of a
// 7.7 us call for the norm of one token (3.5 the launch); with them here a call
// takes 4.0 us.
//
// Functions take positional arguments; None leaves an optional tensor out. The
// last argument is a hipStream_t, or None for the device's current stream. They
// raise ValueError for tensors that do not fit and return the library's status.
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <initializer_list>
#include <limits>
#include <sstream>
#include <stdexcept>
#include <string>

#include "taccl.h"

namespace {

using at::ScalarType;
using at::Tensor;

// torch's functions for the current device and its current stream
PyObject *current_device = nullptr, *current_stream = nullptr;

// the library's calls
template <class A>
using Fn = taccl_status_t (*)(const A *, taccl_stream_t);
Fn<taccl_norm_t> norm_fn;
Fn<taccl_norm_backward_t> norm_backward_fn;
Fn<taccl_route_t> route_fn;
Fn<taccl_route_backward_t> route_backward_fn;
Fn<taccl_dispatch_t> dispatch_fn;
Fn<taccl_combine_t> combine_fn;
Fn<taccl_combine_backward_t> combine_backward_fn;

// a Python error that is set already
struct Raised {};

// one of the tensors does not fit
struct Misfit : std::runtime_error {
  using std::runtime_error::runtime_error;
};

const Tensor &tensor(PyObject *o, const char *name) {
  if (!THPVariable_Check(o)) throw Misfit(std::string(name) + " must be a CUDA tensor");
  return THPVariable_Unpack(o);
}

std::string shown(const Tensor &t) {
  std::ostringstream s;
  s << t.sizes() << " of " << t.scalar_type() << " with strides " << t.strides() << " on "
    << t.device();
  return s.str();
}

[[noreturn]] void misfit(const Tensor &t, const char *name, const std::string &what) {
  throw Misfit(std::string(name) + " must be " + what + ", got " + shown(t));
}

[[noreturn]] void misfit(const Tensor &t, const char *name, const char *what, at::IntArrayRef shape,
                         ScalarType type) {
  std::ostringstream s;
  s << "a " << what << " " << shape << " of " << type << " on the call's device";
  misfit(t, name, s.str());
}

int32_t dtype_code(const Tensor &t, const char *name, bool matrix) {
  if (!matrix || t.dim() == 2) {
    if (t.scalar_type() == at::kFloat) return TACCL_F32;
    if (t.scalar_type() == at::kBFloat16) return TACCL_BF16;
    if (t.scalar_type() == at::kHalf) return TACCL_F16;
  }
  misfit(t, name,
         std::string(matrix ? "a matrix" : "a tensor") + " of float32, bfloat16 or float16");
}

// A size in the call's 32 bits. One that does not fit stays past every limit
// there instead of coming out as another size.
int32_t size32(int64_t n) {
  return (int32_t)std::min<int64_t>(n, std::numeric_limits<int32_t>::max());
}

// The call's device and stream, by the tensor that its others go by
struct At {
  int device;
  taccl_stream_t stream;

  At(const Tensor &t, const char *name, PyObject *s) : device((int)t.get_device()) {
    if (device < 0) misfit(t, name, "a CUDA tensor");
    PyObject *now = PyObject_CallNoArgs(current_device);
    if (!now) throw Raised();
    const long index = PyLong_AsLong(now);
    if (index != device) {
      Py_DECREF(now);
      misfit(t, name, "a CUDA tensor on the current device");
    }
    if (s == Py_None) {
      PyObject *handle = PyObject_CallOneArg(current_stream, now);
      Py_DECREF(now);
      if (!handle) throw Raised();
      stream = PyLong_AsVoidPtr(handle);
      Py_DECREF(handle);
    } else {
      Py_DECREF(now);
      stream = PyLong_AsVoidPtr(s);
    }
    if (PyErr_Occurred()) throw Raised();
  }

  // rows [n][d] with a contiguous last axis
  template <class P>
  void rows(const Tensor &t, const char *name, int64_t n, int64_t d, ScalarType type, P *&p,
            int64_t &stride) const {
    if (t.scalar_type() != type || t.dim() != 2 || t.size(0) != n || t.size(1) != d ||
        t.get_device() != device || (t.stride(1) != 1 && d > 1))
      misfit(t, name, "CUDA tensor with contiguous rows", {n, d}, type);
    p = (P *)t.data_ptr();
    stride = t.stride(0);
  }
  template <class P>
  void rows(PyObject *o, const char *name, int64_t n, int64_t d, ScalarType type, P *&p,
            int64_t &stride) const {
    if (o != Py_None) rows(tensor(o, name), name, n, d, type, p, stride);
  }

  // a contiguous tensor
  template <class P>
  void flat(PyObject *o, const char *name, std::initializer_list<int64_t> shape, ScalarType type,
            P *&p) const {
    if (o == Py_None) return;
    const Tensor &t = tensor(o, name);
    const at::IntArrayRef want(shape);
    if (t.scalar_type() != type || t.sizes() != want || t.get_device() != device ||
        !t.is_contiguous())
      misfit(t, name, "contiguous CUDA tensor", want, type);
    p = (P *)t.data_ptr();
  }

  // a mask: a byte per token, or a truth value
  void mask(PyObject *o, int64_t n, const uint8_t *&p) const {
    const bool truth = THPVariable_Check(o) && THPVariable_Unpack(o).scalar_type() == at::kBool;
    flat(o, "mask", {n}, truth ? at::kBool : at::kByte, p);
  }

  void workspace(PyObject *o, void *&p, int64_t &bytes) const {
    const Tensor &t = tensor(o, "workspace");
    if (t.get_device() != device || !t.is_contiguous())
      misfit(t, "workspace", "a contiguous CUDA tensor on the call's device");
    p = t.data_ptr();
    bytes = (int64_t)t.nbytes();
  }
};

// experts and slots [tokens][k], and tokens and k by them
template <class A>
void choices(A &a, const At &at, PyObject *experts, PyObject *slots) {
  const Tensor &e = tensor(experts, "experts");
  if (e.dim() != 2) misfit(e, "experts", "a matrix [tokens, k]");
  a.tokens = e.size(0);
  a.k = size32(e.size(1));
  at.flat(experts, "experts", {a.tokens, a.k}, at::kInt, a.experts);
  at.flat(slots, "slots", {a.tokens, a.k}, at::kInt, a.slots);
}

const Tensor &buffer(PyObject *o, const char *name) {
  const Tensor &t = tensor(o, name);
  if (t.dim() != 3 || !t.is_contiguous() || t.get_device() < 0)
    misfit(t, name, "a contiguous CUDA tensor [experts, capacity, dim]");
  return t;
}
template <class A>
void buffer_sizes(A &a, const Tensor &t) {
  a.num_experts = size32(t.size(0));
  a.capacity = t.size(1);
  a.cols = size32(t.size(2));
}

double real(PyObject *o) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) throw Raised();
  return x;
}
int64_t whole(PyObject *o) {
  const int64_t x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) throw Raised();
  return x;
}
int32_t small(PyObject *o, const char *name) {
  const int64_t x = whole(o);
  if (x != (int32_t)x) throw Misfit(std::string(name) + " does not fit 32 bits");
  return (int32_t)x;
}

template <class A>
PyObject *run(Fn<A> fn, const A &a, const At &at) {
  taccl_status_t st;
  Py_BEGIN_ALLOW_THREADS;
  st = fn(&a, at.stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(st);
}

// x, weight, out, eps, residual, total, q, scale, group, stream
PyObject *norm(PyObject *const *o) {
  const Tensor &x = tensor(o[0], "x");
  taccl_norm_t a{};
  a.dtype = dtype_code(x, "x", true);
  const ScalarType type = x.scalar_type();
  const At at(x, "x", o[9]);
  const int64_t n = a.rows = x.size(0), d = x.size(1);
  a.cols = size32(d);
  a.eps = (float)real(o[3]);
  a.group = small(o[8], "group");
  at.rows(x, "x", n, d, type, a.x, a.x_stride);
  at.flat(o[1], "weight", {d}, type, a.weight);
  at.rows(o[2], "out", n, d, type, a.out, a.out_stride);
  at.rows(o[4], "residual", n, d, type, a.residual, a.residual_stride);
  at.rows(o[5], "total", n, d, type, a.total, a.total_stride);
  at.rows(o[6], "q", n, d, at::kFloat8_e4m3fn, a.q, a.q_stride);
  at.rows(o[7], "scale", n, a.group > 0 ? (d + a.group - 1) / a.group : 1, at::kFloat, a.scale,
          a.scale_stride);
  return run(norm_fn, a, at);
}

// dout, h, weight, dx, dweight, workspace, eps, dtotal, stream
PyObject *norm_backward(PyObject *const *o) {
  const Tensor &h = tensor(o[1], "h");
  taccl_norm_backward_t a{};
  a.dtype = dtype_code(h, "h", true);
  const ScalarType type = h.scalar_type();
  const At at(h, "h", o[8]);
  const int64_t n = a.rows = h.size(0), d = h.size(1);
  a.cols = size32(d);
  a.eps = (float)real(o[6]);
  at.rows(h, "h", n, d, type, a.h, a.h_stride);
  at.rows(o[0], "dout", n, d, type, a.dout, a.dout_stride);
  at.flat(o[2], "weight", {d}, type, a.weight);
  at.rows(o[3], "dx", n, d, type, a.dx, a.dx_stride);
  at.flat(o[4], "dweight", {d}, at::kFloat, a.dweight);
  at.workspace(o[5], a.workspace, a.workspace_bytes);
  at.rows(o[7], "dtotal", n, d, type, a.dtotal, a.dtotal_stride);
  return run(norm_backward_fn, a, at);
}

// logits, experts, weights, slots, counts, prob_sums, loss, rows, workspace, mask, capacity, coef,
// renorm, stream
PyObject *route(PyObject *const *o) {
  const Tensor &l = tensor(o[0], "logits");
  taccl_route_t a{};
  a.dtype = dtype_code(l, "logits", true);
  const At at(l, "logits", o[13]);
  const int64_t n = l.size(0), e = l.size(1);
  a.num_experts = size32(e);
  choices(a, at, o[1], o[3]);
  a.tokens = n;
  at.rows(l, "logits", n, e, l.scalar_type(), a.logits, a.logits_stride);
  at.flat(o[1], "experts", {n, a.k}, at::kInt, a.experts);
  at.flat(o[2], "weights", {n, a.k}, at::kFloat, a.weights);
  at.flat(o[4], "counts", {e}, at::kInt, a.counts);
  at.flat(o[5], "prob_sums", {e}, at::kFloat, a.prob_sums);
  at.flat(o[6], "loss", {1}, at::kFloat, a.loss);
  at.flat(o[7], "rows", {1}, at::kInt, a.rows);
  at.workspace(o[8], a.workspace, a.workspace_bytes);
  at.mask(o[9], n, a.mask);
  a.capacity = whole(o[10]);
  a.coef = (float)real(o[11]);
  a.renorm = PyObject_IsTrue(o[12]);
  return run(route_fn, a, at);
}

// logits, experts, counts, rows, dlogits, dweights, dloss, mask, coef, renorm, stream
PyObject *route_backward(PyObject *const *o) {
  const Tensor &l = tensor(o[0], "logits");
  taccl_route_backward_t a{};
  a.dtype = dtype_code(l, "logits", true);
  const At at(l, "logits", o[10]);
  const int64_t n = a.tokens = l.size(0), e = l.size(1);
  a.num_experts = size32(e);
  const Tensor &experts = tensor(o[1], "experts");
  if (experts.dim() != 2) misfit(experts, "experts", "a matrix [tokens, k]");
  const int64_t k = experts.size(1);
  a.k = size32(k);
  at.rows(l, "logits", n, e, l.scalar_type(), a.logits, a.logits_stride);
  at.flat(o[1], "experts", {n, k}, at::kInt, a.experts);
  at.flat(o[2], "counts", {e}, at::kInt, a.counts);
  at.flat(o[3], "rows", {1}, at::kInt, a.rows);
  at.rows(o[4], "dlogits", n, e, l.scalar_type(), a.dlogits, a.dlogits_stride);
  at.flat(o[5], "dweights", {n, k}, at::kFloat, a.dweights);
  at.flat(o[6], "dloss", {1}, at::kFloat, a.dloss);
  at.mask(o[7], n, a.mask);
  a.coef = (float)real(o[8]);
  a.renorm = PyObject_IsTrue(o[9]);
  return run(route_backward_fn, a, at);
}

// x, experts, slots, counts, out, scale, out_scale, stream
PyObject *dispatch(PyObject *const *o) {
  const Tensor &out = buffer(o[4], "out");
  taccl_dispatch_t a{};
  const At at(out, "out", o[7]);
  buffer_sizes(a, out);
  choices(a, at, o[1], o[2]);
  at.rows(o[0], "x", a.tokens, a.cols, out.scalar_type(), a.x, a.x_stride);
  a.element_bytes = (int32_t)out.element_size();
  at.flat(o[3], "counts", {a.num_experts}, at::kInt, a.counts);
  a.out = out.data_ptr();
  if (o[5] != Py_None || o[6] != Py_None) {
    const Tensor &scale = tensor(o[5], "scale");
    if (scale.dim() != 2) misfit(scale, "scale", "a matrix [tokens, n]");
    tensor(o[6], "out_scale");
    a.scale_cols = size32(scale.size(1));
    at.rows(scale, "scale", a.tokens, a.scale_cols, at::kFloat, a.scale, a.scale_stride);
    at.flat(o[6], "out_scale", {a.num_experts, a.capacity, a.scale_cols}, at::kFloat, a.out_scale);
  }
  return run(dispatch_fn, a, at);
}

// buffer, experts, slots, out, weights, stream
PyObject *combine(PyObject *const *o) {
  const Tensor &b = buffer(o[0], "buffer");
  taccl_combine_t a{};
  a.dtype = dtype_code(b, "buffer", false);
  const At at(b, "buffer", o[5]);
  buffer_sizes(a, b);
  choices(a, at, o[1], o[2]);
  a.buffer = b.data_ptr();
  at.rows(o[3], "out", a.tokens, a.cols, b.scalar_type(), a.out, a.out_stride);
  at.flat(o[4], "weights", {a.tokens, a.k}, at::kFloat, a.weights);
  return run(combine_fn, a, at);
}

// dout, buffer, experts, slots, counts, weights, dbuffer, dweights, stream
PyObject *combine_backward(PyObject *const *o) {
  const Tensor &b = buffer(o[1], "buffer");
  taccl_combine_backward_t a{};
  a.dtype = dtype_code(b, "buffer", false);
  const At at(b, "buffer", o[8]);
  buffer_sizes(a, b);
  choices(a, at, o[2], o[3]);
  at.rows(o[0], "dout", a.tokens, a.cols, b.scalar_type(), a.dout, a.dout_stride);
  a.buffer = b.data_ptr();
  at.flat(o[4], "counts", {a.num_experts}, at::kInt, a.counts);
  at.flat(o[5], "weights", {a.tokens, a.k}, at::kFloat, a.weights);
  at.flat(o[6], "dbuffer", {a.num_experts, a.capacity, a.cols}, b.scalar_type(), a.dbuffer);
  at.flat(o[7], "dweights", {a.tokens, a.k}, at::kFloat, a.dweights);
  return run(combine_backward_fn, a, at);
}

template <PyObject *(*kCall)(PyObject *const *), int kArgs>
PyObject *checked(PyObject *, PyObject *const *o, Py_ssize_t n) {
  if (n != kArgs) {
    PyErr_Format(PyExc_TypeError, "takes %d arguments, got %zd", kArgs, n);
    return nullptr;
  }
  try {
    return kCall(o);
  } catch (const Raised &) {
  } catch (const Misfit &e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::exception &e) {  // torch's own errors
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// bind(current device, current stream, addresses of the library's calls)
PyObject *bind(PyObject *, PyObject *args) {
  PyObject *device, *stream;
  unsigned long long f[7];
  if (!PyArg_ParseTuple(args, "OOKKKKKKK", &device, &stream, f, f + 1, f + 2, f + 3, f + 4, f + 5,
                        f + 6))
    return nullptr;
  Py_INCREF(device);
  Py_INCREF(stream);
  Py_XDECREF(current_device);
  Py_XDECREF(current_stream);
  current_device = device;
  current_stream = stream;
  norm_fn = (Fn<taccl_norm_t>)f[0];
  norm_backward_fn = (Fn<taccl_norm_backward_t>)f[1];
  route_fn = (Fn<taccl_route_t>)f[2];
  route_backward_fn = (Fn<taccl_route_backward_t>)f[3];
  dispatch_fn = (Fn<taccl_dispatch_t>)f[4];
  combine_fn = (Fn<taccl_combine_t>)f[5];
  combine_backward_fn = (Fn<taccl_combine_backward_t>)f[6];
  Py_RETURN_NONE;
}

#define CALL(NAME, ARGS) \
  { #NAME, (PyCFunction)(void (*)())checked<NAME, ARGS>, METH_FASTCALL, nullptr }
PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, nullptr},
                         CALL(norm, 10),
                         CALL(norm_backward, 9),
                         CALL(route, 14),
                         CALL(route_backward, 11),
                         CALL(dispatch, 8),
                         CALL(combine, 6),
                         CALL(combine_backward, 9),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_experts", nullptr, -1, methods,
                      nullptr,               nullptr,    nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__experts() { return PyModule_Create(&module); }

// Argument marshalling of Shampoo.step in native code: checks the parameter and gradient
// tensors of a step (device, dtype, contiguity, shape) and hands their addresses to
// shampoo_step on the current stream.  Ten attribute look-ups per tensor cost a millisecond in
// Python on a few hundred parameters, more than the step itself; here they cost some tens of
// nanoseconds per tensor.  What the tensor library throws (a tensor without storage, no device, no memory) leaves here
// as the Python exception that the same call raises from Python.
//
// The operators of a training pass likewise: checks, outputs and workspaces from torch's allocator, the call on the current
// stream of the tensors' device.  (16 x 512 residual norms: 12.7 us a call in Python, of which the kernel's launch is four.)  They return
// their tensors, or the library's error code.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/ATen.h>
#include <c10/hip/HIPGuard.h>
#include <c10/hip/HIPStream.h>
#include <pybind11/pybind11.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <cstdint>
#include <memory>
#include <optional>
#include <vector>

#include "../../include/shampoo.h"

namespace {

using StepFn = int (*)(void *, void *const *, const void *const *, float, int64_t, void *);

struct Stepper {
  StepFn fn;
  void *handle;
  c10::Device device{c10::DeviceType::CUDA, 0};
  at::ScalarType grad_dtype;
  std::vector<std::vector<int64_t>> shapes;
  std::vector<void *> w;
  std::vector<const void *> g;
};

constexpr const char *CAPSULE = "shampoo.stepper";

void stepper_free(PyObject *cap) { delete static_cast<Stepper *>(PyCapsule_GetPointer(cap, CAPSULE)); }

// make(address of shampoo_step, handle, device index, gradients are bf16, [shape tuples])
PyObject *make(PyObject *, PyObject *args) {
  HANDLE_TH_ERRORS
  unsigned long long fn, handle;
  int device, bf16;
  PyObject *shapes;
  if (!PyArg_ParseTuple(args, "KKipO!", &fn, &handle, &device, &bf16, &PyList_Type, &shapes)) return nullptr;
  auto s = std::make_unique<Stepper>();
  s->fn = reinterpret_cast<StepFn>(fn);
  s->handle = reinterpret_cast<void *>(handle);
  s->device = c10::Device(c10::DeviceType::CUDA, static_cast<c10::DeviceIndex>(device));
  s->grad_dtype = bf16 ? at::kBFloat16 : at::kFloat;
  for (Py_ssize_t i = 0; i < PyList_GET_SIZE(shapes); ++i) {
    PyObject *t = PyList_GET_ITEM(shapes, i);
    std::vector<int64_t> dims;
    for (Py_ssize_t k = 0; PyTuple_Check(t) && k < PyTuple_GET_SIZE(t); ++k) dims.push_back(PyLong_AsLongLong(PyTuple_GET_ITEM(t, k)));
    if (!PyTuple_Check(t) || PyErr_Occurred()) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "shapes are tuples of integers");
      return nullptr;
    }
    s->shapes.push_back(std::move(dims));
  }
  s->w.resize(s->shapes.size());
  s->g.resize(s->shapes.size());
  PyObject *cap = PyCapsule_New(s.get(), CAPSULE, stepper_free);
  if (cap) (void)s.release();
  return cap;
  END_HANDLE_TH_ERRORS
}

// step(stepper, params, grads, lr, step number) -> return code of shampoo_step
PyObject *step(PyObject *, PyObject *args) {
  HANDLE_TH_ERRORS
  PyObject *cap, *params, *grads;
  float lr;
  long long t;
  if (!PyArg_ParseTuple(args, "OOOfL", &cap, &params, &grads, &lr, &t)) return nullptr;
  auto *s = static_cast<Stepper *>(PyCapsule_GetPointer(cap, CAPSULE));
  if (!s) return nullptr;
  THPObjectPtr ps(PySequence_Fast(params, "params is a sequence of tensors"));
  if (!ps) return nullptr;
  THPObjectPtr gs(PySequence_Fast(grads, "grads is a sequence of tensors"));
  if (!gs) return nullptr;
  const Py_ssize_t n = static_cast<Py_ssize_t>(s->shapes.size());
  if (PySequence_Fast_GET_SIZE(ps.get()) != n || PySequence_Fast_GET_SIZE(gs.get()) != n) {
    PyErr_SetString(PyExc_ValueError, "one parameter and one gradient tensor per declared parameter");
    return nullptr;
  }
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject *po = PySequence_Fast_GET_ITEM(ps.get(), i), *go = PySequence_Fast_GET_ITEM(gs.get(), i);
    const char *bad = nullptr;
    if (!THPVariable_Check(po) || !THPVariable_Check(go)) {
      bad = "parameters and gradients are tensors";
    } else {
      const at::Tensor &w = THPVariable_Unpack(po), &g = THPVariable_Unpack(go);
      const c10::IntArrayRef shape(s->shapes[i]);
      if (w.device() != s->device || g.device() != s->device) bad = "tensors must live on the optimizer's device";
      else if (w.scalar_type() != at::kFloat || g.scalar_type() != s->grad_dtype)
        bad = s->grad_dtype == at::kFloat ? "parameters are float32, gradients torch.float32" : "parameters are float32, gradients torch.bfloat16";
      else if (!w.is_contiguous() || !g.is_contiguous()) bad = "tensors must be contiguous";
      else if (w.sizes() != shape || g.sizes() != shape) bad = "shape differs from the one given at creation";
      else { s->w[i] = w.data_ptr(); s->g[i] = g.data_ptr(); }
    }
    if (bad) { PyErr_Format(PyExc_ValueError, "parameter %zd: %s", i, bad); return nullptr; }
  }
  void *stream = c10::hip::getCurrentHIPStream().stream();
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    rc = s->fn(s->handle, s->w.data(), s->g.data(), lr, static_cast<int64_t>(t), stream);
  }
  return PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------------------------------
// Operators of a training pass
// ---------------------------------------------------------------------------
struct Library {
  decltype(&shampoo_linear_cross_entropy_workspace_bytes) cross_entropy_bytes;
  decltype(&shampoo_linear_cross_entropy) cross_entropy;
  decltype(&shampoo_checkpoint_bytes) checkpoint_bytes;
  decltype(&shampoo_checkpoint_pack) pack;
  decltype(&shampoo_checkpoint_unpack) unpack;
  decltype(&shampoo_checkpoint_activation_grad) activation_grad;
  decltype(&shampoo_checkpoint_weight_grad_workspace_bytes) weight_grad_bytes;
  decltype(&shampoo_checkpoint_weight_grad) weight_grad;
  decltype(&shampoo_residual_norm_forward) norm_forward;
  decltype(&shampoo_residual_norm_backward_workspace_bytes) norm_backward_bytes;
  decltype(&shampoo_residual_norm_backward) norm_backward;
} library;
static_assert(sizeof(Library) == 11 * sizeof(void *), "addresses only");

// use([addresses of the entry points in the order above])
PyObject *use(PyObject *, PyObject *list) {
  constexpr Py_ssize_t n = sizeof(Library) / sizeof(void *);
  if (!PyList_Check(list) || PyList_GET_SIZE(list) != n) { PyErr_SetString(PyExc_TypeError, "a list of addresses"); return nullptr; }
  void **to = reinterpret_cast<void **>(&library);
  for (Py_ssize_t i = 0; i < n; ++i) {
    to[i] = PyLong_AsVoidPtr(PyList_GET_ITEM(list, i));
    if (PyErr_Occurred()) return nullptr;
  }
  Py_RETURN_NONE;
}

struct Refused { const char *why; };      // becomes an AssertionError

const at::Tensor &tensor(PyObject *o) {
  if (!THPVariable_Check(o)) throw Refused{"a tensor is needed"};
  return THPVariable_Unpack(o);
}
int dtype_code(at::ScalarType t) {
  if (t == at::kFloat) return SHAMPOO_GRAD_F32;
  if (t == at::kBFloat16) return SHAMPOO_GRAD_BF16;
  throw Refused{"float32 or bfloat16 is needed"};
}
at::ScalarType dtype_of(int64_t code) { return code == SHAMPOO_GRAD_F32 ? at::kFloat : at::kBFloat16; }
// a CUDA matrix whose rows are contiguous, as the library reads it (a copy where it is not, or not aligned to `align` bytes)
at::Tensor rows_of(const at::Tensor &x, size_t align = 1) {
  if (!x.is_cuda() || x.dim() != 2) throw Refused{"a CUDA matrix is needed"};
  const int64_t n = x.size(0), d = x.size(1);
  at::Tensor y = (d > 1 && x.stride(1) != 1) || (n > 1 && x.stride(0) < d) ? x.contiguous() : x;
  if (reinterpret_cast<uintptr_t>(y.data_ptr()) % align != 0) y = y.clone(at::MemoryFormat::Contiguous);
  return y;
}
int64_t ld(const at::Tensor &x) { return x.size(0) > 1 ? x.stride(0) : std::max<int64_t>(x.size(1), 1); }
// a float32 operand of exactly this shape on this device, or none
std::optional<at::Tensor> vector(PyObject *o, at::IntArrayRef shape, const at::Device &device) {
  if (o == Py_None) return std::nullopt;
  const at::Tensor &x = tensor(o);
  if (x.scalar_type() != at::kFloat || x.sizes() != shape || x.device() != device) throw Refused{"a float32 tensor of the right shape is needed"};
  return x.contiguous();
}
const float *floats(const std::optional<at::Tensor> &x) { return x ? static_cast<const float *>(x->data_ptr()) : nullptr; }
void *address(const std::optional<at::Tensor> &x) { return x ? x->data_ptr() : nullptr; }
at::Tensor empty(const at::Tensor &like, at::IntArrayRef shape, at::ScalarType t) { return at::empty(shape, like.options().dtype(t)); }
at::Tensor bytes(const at::Tensor &like, size_t n) { return empty(like, {static_cast<int64_t>(std::max<size_t>(n, 256))}, at::kByte); }
void *stream_of(const at::Tensor &x) { return c10::hip::getCurrentHIPStream(x.get_device()).stream(); }
PyObject *wrap(const std::optional<at::Tensor> &x) { if (!x) Py_RETURN_NONE; return THPVariable_Wrap(*x); }
PyObject *tuple(std::initializer_list<std::optional<at::Tensor>> list) {
  THPObjectPtr out(PyTuple_New(static_cast<Py_ssize_t>(list.size())));
  if (!out) return nullptr;
  Py_ssize_t i = 0;
  for (const auto &x : list) {
    PyObject *o = wrap(x);
    if (!o) return nullptr;
    PyTuple_SET_ITEM(out.get(), i++, o);
  }
  return out.release();
}
int64_t integer(PyObject *o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw python_error();
  return v;
}
float real(PyObject *o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw python_error();
  return static_cast<float>(v);
}
// The body of an operator: what it throws becomes a Python exception; the arguments are counted.
template <typename F> PyObject *guarded(Py_ssize_t have, Py_ssize_t want, F &&body) {
  HANDLE_TH_ERRORS
  if (have != want) { PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", want, have); return nullptr; }
  try {
    return body();
  } catch (const Refused &r) {
    PyErr_SetString(PyExc_AssertionError, r.why);
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}
// the library's call, on the device of x and without the interpreter's lock
template <typename F> int call(const at::Tensor &x, F &&f) {
  const c10::hip::HIPGuard guard(x.get_device());
  void *stream = stream_of(x);
  pybind11::gil_scoped_release no_gil;
  return f(stream);
}

// (x, w, targets, bias, weight, scale, code of dw's type or None, gradients) -> (loss, dx, dw, dbias)
PyObject *cross_entropy(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  return guarded(n_args, 8, [&]() -> PyObject * {
    const at::Tensor &x0 = tensor(a[0]), &w0 = tensor(a[1]), &t0 = tensor(a[2]);
    const int code = dtype_code(x0.scalar_type());
    const at::Device device = x0.device();
    if (!x0.is_cuda() || x0.dim() != 2 || w0.dim() != 2 || w0.scalar_type() != x0.scalar_type() || w0.device() != device || w0.size(1) != x0.size(1))
      throw Refused{"x [n, d] and w [v, d] of one type on one device are needed"};
    const int64_t n = x0.size(0), d = x0.size(1), v = w0.size(0);
    if (t0.device() != device || t0.scalar_type() != at::kLong || t0.dim() != 1 || t0.size(0) != n) throw Refused{"targets are int64 [n]"};
    const bool gradients = PyObject_IsTrue(a[7]) != 0;
    const at::ScalarType grad = a[6] == Py_None ? w0.scalar_type() : dtype_of(integer(a[6]));
    const bool in_out = v > 1 && w0.stride(0) == 1 && (d > 1 || w0.stride(1) != 1);      // the view of a matrix [d, v]
    const at::Tensor x = rows_of(x0, 16), w = rows_of(in_out ? w0.t() : w0, 16), targets = t0.contiguous();
    const auto bias = vector(a[3], {v}, device), weight = vector(a[4], {n}, device);
    const at::Tensor loss = empty(x, {n}, at::kFloat);
    std::optional<at::Tensor> dx, dw, dbias;
    if (gradients) {
      dx = empty(x, {n, d}, x.scalar_type());
      dw = empty(x, w.sizes(), grad);
      if (bias) dbias = empty(x, {v}, at::kFloat);
    }
    if (d > INT32_MAX || v > INT32_MAX) return PyLong_FromLong(SHAMPOO_ERR_UNSUPPORTED);
    const shampoo_cross_entropy c = {n, static_cast<int32_t>(d), static_cast<int32_t>(v), code, dtype_code(grad), in_out ? SHAMPOO_IN_OUT : SHAMPOO_OUT_IN,
                                     bias ? 1 : 0, gradients ? 1 : 0, ld(x), ld(w), d, w.size(1)};
    const at::Tensor ws = bytes(x, library.cross_entropy_bytes(&c));
    const float scale = real(a[5]);
    const int rc = call(x, [&](void *stream) {
      return library.cross_entropy(&c, x.data_ptr(), w.data_ptr(), floats(bias), static_cast<const int64_t *>(targets.data_ptr()), floats(weight), scale,
                                   static_cast<float *>(loss.data_ptr()), address(dx), address(dw), static_cast<float *>(address(dbias)), ws.data_ptr(),
                                   static_cast<size_t>(ws.numel()), stream);
    });
    if (rc != 0) return PyLong_FromLong(rc);
    return tuple({loss, dx, dw && in_out ? std::optional<at::Tensor>(dw->t()) : dw, dbias});
  });
}

at::Tensor packed_for(const at::Tensor &x) {
  if (x.size(1) > INT32_MAX) throw Refused{"too many columns"};
  return bytes(x, library.checkpoint_bytes(x.size(0), static_cast<int32_t>(x.size(1))));
}
size_t size_of(const at::Tensor &x) { return static_cast<size_t>(x.numel()); }

// An int32 argument of the library
int32_t integer32(PyObject *o) {
  const int64_t v = integer(o);
  if (v < INT32_MIN || v > INT32_MAX) throw Refused{"an integer of 32 bits is needed"};
  return static_cast<int32_t>(v);
}
// The memory of a checkpoint of this shape: the library reads as much of it as the shape says.
const at::Tensor &checkpoint(PyObject *o, int64_t rows, int32_t cols) {
  const at::Tensor &p = tensor(o);
  if (!p.is_cuda() || p.scalar_type() != at::kByte || !p.is_contiguous()) throw Refused{"a checkpoint is contiguous bytes on a CUDA device"};
  if (rows < 0 || cols < 1 || size_of(p) < library.checkpoint_bytes(rows, cols)) throw Refused{"the checkpoint's memory does not hold its shape"};
  return p;
}

// (x) -> packed
PyObject *pack(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  return guarded(n_args, 1, [&]() -> PyObject * {
    const int code = dtype_code(tensor(a[0]).scalar_type());
    const at::Tensor x = rows_of(tensor(a[0])), p = packed_for(x);
    const int rc = call(x, [&](void *stream) {
      return library.pack(x.data_ptr(), code, x.size(0), static_cast<int32_t>(x.size(1)), ld(x), p.data_ptr(), size_of(p), stream);
    });
    return rc != 0 ? PyLong_FromLong(rc) : THPVariable_Wrap(p);
  });
}

// (packed, rows, cols, activation, code of the type) -> y
PyObject *unpack(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  return guarded(n_args, 5, [&]() -> PyObject * {
    const int64_t rows = integer(a[1]), code = integer(a[4]);
    const int32_t cols = integer32(a[2]), activation = integer32(a[3]);
    const at::Tensor &p = checkpoint(a[0], rows, cols);
    const at::Tensor y = empty(p, {rows, cols}, dtype_of(code));
    const int rc = call(p, [&](void *stream) {
      return library.unpack(p.data_ptr(), size_of(p), rows, cols, activation, y.data_ptr(), static_cast<int32_t>(code), cols, stream);
    });
    return rc != 0 ? PyLong_FromLong(rc) : THPVariable_Wrap(y);
  });
}

// (packed, rows, cols, dy, activation) -> dx
PyObject *activation_grad(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  return guarded(n_args, 5, [&]() -> PyObject * {
    const int64_t rows = integer(a[1]);
    const int32_t cols = integer32(a[2]), activation = integer32(a[4]);
    const at::Tensor &p = checkpoint(a[0], rows, cols);
    const at::Tensor dy = rows_of(tensor(a[3]));
    if (dy.size(0) != rows || dy.size(1) != cols || dy.device() != p.device()) throw Refused{"dy is not of the checkpoint's shape and device"};
    const int code = dtype_code(dy.scalar_type());
    const at::Tensor dx = empty(dy, {rows, cols}, dy.scalar_type());
    const int rc = call(dy, [&](void *stream) {
      return library.activation_grad(p.data_ptr(), size_of(p), rows, cols, activation, dy.data_ptr(), code, ld(dy), dx.data_ptr(), cols, stream);
    });
    return rc != 0 ? PyLong_FromLong(rc) : THPVariable_Wrap(dx);
  });
}

// (packed, rows, cols, dy, activation, code of dw's type or None, out_in, bias) -> (dw, db)
PyObject *weight_grad(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  return guarded(n_args, 8, [&]() -> PyObject * {
    const int64_t rows = integer(a[1]);
    const int32_t in = integer32(a[2]), activation = integer32(a[4]);
    const at::Tensor &p = checkpoint(a[0], rows, in);
    const at::Tensor dy = rows_of(tensor(a[3]), 16);
    if (dy.size(0) != rows || dy.device() != p.device()) throw Refused{"dy is not of the checkpoint's rows and device"};
    const int64_t out = dy.size(1);
    if (out > INT32_MAX) return PyLong_FromLong(SHAMPOO_ERR_UNSUPPORTED);
    const int code = dtype_code(dy.scalar_type());
    const at::ScalarType grad = a[5] == Py_None ? dy.scalar_type() : dtype_of(integer(a[5]));
    const bool out_in = PyObject_IsTrue(a[6]) != 0;
    const at::Tensor dw = out_in ? empty(dy, {out, in}, grad) : empty(dy, {in, out}, grad);
    std::optional<at::Tensor> db;
    if (PyObject_IsTrue(a[7]) != 0) db = empty(dy, {out}, at::kFloat);
    const int32_t out32 = static_cast<int32_t>(out);
    const at::Tensor ws = bytes(dy, library.weight_grad_bytes(rows, in, out32, activation, code, ld(dy), dtype_code(grad), db ? 1 : 0));
    const int rc = call(dy, [&](void *stream) {
      return library.weight_grad(p.data_ptr(), size_of(p), rows, in, activation, dy.data_ptr(), code, out32, ld(dy), dw.data_ptr(), dtype_code(grad),
                                 out_in ? SHAMPOO_OUT_IN : SHAMPOO_IN_OUT, dw.size(1), static_cast<float *>(address(db)), ws.data_ptr(), size_of(ws), stream);
    });
    return rc != 0 ? PyLong_FromLong(rc) : tuple({dw, db});
  });
}

// a: post, pre, w_post, b_post, gate, w_pre, b_pre, epsilon, scale
struct Norm {
  std::optional<at::Tensor> w_post, b_post, gate, w_pre, b_pre;
  shampoo_residual_norm c;
  Norm(int64_t rows, int64_t cols, at::ScalarType type, const at::Device &device, PyObject *const *a) {
    w_post = vector(a[2], {cols}, device); b_post = vector(a[3], {cols}, device);
    w_pre = vector(a[5], {cols}, device); b_pre = vector(a[6], {cols}, device);
    int64_t gates = 0;
    if (a[4] != Py_None) {
      const at::Tensor &g = tensor(a[4]);
      gates = g.dim() == 2 ? g.size(0) : 1;
      gate = g.dim() == 1 ? vector(a[4], {cols}, device) : vector(a[4], {gates, cols}, device);
    }
    if (cols > INT32_MAX) throw Refused{"too many columns"};
    c = {rows, static_cast<int32_t>(cols), dtype_code(type), static_cast<int32_t>(integer(a[0])), static_cast<int32_t>(integer(a[1])), gates, real(a[7]), real(a[8]),
         floats(w_post), floats(b_post), floats(gate), floats(w_pre), floats(b_pre)};
  }
};

// (r, f, post, pre, w_post, b_post, gate, w_pre, b_pre, epsilon, scale, checkpoint) -> (r_out, h, packed r, packed f)
PyObject *norm_forward(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  return guarded(n_args, 12, [&]() -> PyObject * {
    const at::Tensor r = rows_of(tensor(a[0])), f = rows_of(tensor(a[1]));
    if (r.sizes() != f.sizes() || r.scalar_type() != f.scalar_type() || r.device() != f.device()) throw Refused{"r and f of one shape, type and device are needed"};
    const int64_t rows = r.size(0), cols = r.size(1);
    const Norm k(rows, cols, r.scalar_type(), r.device(), a + 2);
    const at::Tensor r_out = empty(r, {rows, cols}, r.scalar_type());
    std::optional<at::Tensor> h, r8, f8;
    if (k.c.pre != SHAMPOO_NORM_NONE) h = empty(r, {rows, cols}, r.scalar_type());
    if (PyObject_IsTrue(a[11]) != 0) { r8 = packed_for(r); f8 = packed_for(r); }
    const int rc = call(r, [&](void *stream) {
      return library.norm_forward(&k.c, r.data_ptr(), ld(r), f.data_ptr(), ld(f), r_out.data_ptr(), cols, address(h), cols, address(r8), address(f8),
                                  r8 ? size_of(*r8) : 0, stream);
    });
    return rc != 0 ? PyLong_FromLong(rc) : tuple({r_out, h, r8, f8});
  });
}

// (r, f, rows, cols, code of their type where they are packed and otherwise None, dr_out, dh, post ... scale as above)
//   -> (dr, df, dgate, dw_post, db_post, dw_pre, db_pre)
PyObject *norm_backward(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  return guarded(n_args, 16, [&]() -> PyObject * {
    const bool packed = a[4] != Py_None;
    const auto matrix = [&](PyObject *o) { return packed ? checkpoint(o, integer(a[2]), integer32(a[3])) : rows_of(tensor(o)); };
    const at::Tensor r = matrix(a[0]), f = matrix(a[1]);
    const int64_t rows = packed ? integer(a[2]) : r.size(0), cols = packed ? integer(a[3]) : r.size(1);
    const at::ScalarType type = packed ? dtype_of(integer(a[4])) : r.scalar_type();
    const at::Device device = r.device();
    if (f.device() != device || (!packed && (f.sizes() != r.sizes() || f.scalar_type() != type))) throw Refused{"r and f of one shape, type and device are needed"};
    const Norm k(rows, cols, type, device, a + 7);
    std::optional<at::Tensor> d[2];
    for (int i = 0; i < 2; ++i) {
      if (a[5 + i] == Py_None) continue;
      d[i] = rows_of(tensor(a[5 + i]));
      if (d[i]->device() != device || d[i]->scalar_type() != type || d[i]->size(0) != rows || d[i]->size(1) != cols)
        throw Refused{"gradients of r's shape, type and device are needed"};
    }
    const at::Tensor dr = empty(r, {rows, cols}, type), df = empty(r, {rows, cols}, type);
    std::optional<at::Tensor> dgate, dw_post, db_post, dw_pre, db_pre;
    if (k.gate) dgate = empty(r, k.gate->sizes(), at::kFloat);
    if (k.c.post != SHAMPOO_NORM_NONE) dw_post = empty(r, {cols}, at::kFloat);
    if (k.c.post == SHAMPOO_NORM_LAYER && k.b_post) db_post = empty(r, {cols}, at::kFloat);
    if (k.c.pre != SHAMPOO_NORM_NONE) dw_pre = empty(r, {cols}, at::kFloat);
    if (k.c.pre == SHAMPOO_NORM_LAYER && k.b_pre) db_pre = empty(r, {cols}, at::kFloat);
    const at::Tensor ws = bytes(r, library.norm_backward_bytes(&k.c));
    auto out = [](const std::optional<at::Tensor> &x) { return static_cast<float *>(address(x)); };
    const int rc = call(r, [&](void *stream) {
      return library.norm_backward(&k.c, packed ? 1 : 0, r.data_ptr(), packed ? cols : ld(r), f.data_ptr(), packed ? cols : ld(f), address(d[0]), d[0] ? ld(*d[0]) : 0,
                                   address(d[1]), d[1] ? ld(*d[1]) : 0, dr.data_ptr(), cols, df.data_ptr(), cols, out(dgate), out(dw_post), out(db_post), out(dw_pre),
                                   out(db_pre), ws.data_ptr(), size_of(ws), stream);
    });
    return rc != 0 ? PyLong_FromLong(rc) : tuple({dr, df, dgate, dw_post, db_post, dw_pre, db_pre});
  });
}

#define OPERATOR(NAME) {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(NAME)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"make", make, METH_VARARGS, nullptr}, {"step", step, METH_VARARGS, nullptr}, {"use", use, METH_O, nullptr},
                         OPERATOR(cross_entropy), OPERATOR(pack), OPERATOR(unpack), OPERATOR(activation_grad), OPERATOR(weight_grad),
                         OPERATOR(norm_forward), OPERATOR(norm_backward), {nullptr, nullptr, 0, nullptr}};
#undef OPERATOR
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }

// The forward calls of the binding as one native function each: what a program pays on the host for a call whose kernel runs 4 us.
// Through ctypes a call of one small layer took the host 5.7 - 6.6 us (checks 0.6 - 0.75, the output 1.1 - 1.4, ctypes 0.5, the launch 2.4);
// here 4.4, of which the kernel's own 4.0 are the limit: 10 -> 8 at 1024 rows 6.0 -> 5.2 us a call, 256 -> 256 at 16 rows 6.0 -> 5.3,
// 78 -> 16 -> 2 at 256 rows 7.2 -> 6.5.
//
// A function takes the layer object(s) and x, makes the checks of binding._check_io, allocates y (and the workspace, if the call
// needs one) with torch's allocator and calls the library on the current stream, both without the interpreter's lock, as torch's own
// functions and ctypes do: an allocation may wait for the device, and the device for a thread that needs the lock.
// It returns None, having done nothing, for anything but the plain case -- a strided CUDA tensor of torch's own class with no
// dispatch or function mode active, a layer of the binding's own struct -- and for whatever the library refuses: the binding then
// takes the general path, which serves it or says what is wrong.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/Device.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <vector>

#include "lutkan.h"

namespace {

// Handed over by the binding (init): the library's entry points, the ctypes classes of the two layer structs, and torch's function
// that returns the handle of the current stream.
struct {
  decltype(&lutkan_forward_or_workspace) forward_or_workspace;
  decltype(&lutkan_forward) forward;
  decltype(&lutkan_model_forward_or_workspace) model_or_workspace;
  decltype(&lutkan_model_forward) model;
  decltype(&bspline_forward_workspace_bytes) spline_workspace_bytes;
  decltype(&bspline_kan_forward) spline;
  decltype(&lutkan_rmsnorm_fp8) rmsnorm;
  decltype(&lutkan_quantise_fp8) quantise;
  decltype(&lutkan_matmul_fp8) matmul;
  decltype(&lutkan_grouped_matmul_fp8) grouped_matmul;
  PyObject *lut_struct, *spline_struct, *current_stream;
} g;

PyObject *s_c, *s_d, *s_m, *s_device;      // attribute names of a layer object

// A layer object's fields.  `c` holds the ctypes struct's memory for as long as this lives.
struct Layer {
  Py_buffer c{};
  long d = 0, m = 0;
  c10::Device device{c10::kCPU};
  ~Layer() { if (c.obj) PyBuffer_Release(&c); }
  Layer() = default;
  Layer(const Layer &) = delete;
  Layer &operator=(const Layer &) = delete;

  bool read(PyObject *layer, PyObject *struct_type, size_t bytes) {
    PyObject *held = PyObject_GetAttr(layer, s_c);
    bool ok = held && (PyObject *)Py_TYPE(held) == struct_type && PyObject_GetBuffer(held, &c, PyBUF_SIMPLE) == 0 && (size_t)c.len == bytes;
    Py_XDECREF(held);
    ok = ok && number(layer, s_d, &d) && number(layer, s_m, &m);
    if (!ok) return false;
    PyObject *dev = PyObject_GetAttr(layer, s_device);
    ok = dev && THPDevice_Check(dev);
    if (ok) device = reinterpret_cast<THPDevice *>(dev)->device;
    Py_XDECREF(dev);
    return ok;
  }

 private:
  static bool number(PyObject *layer, PyObject *name, long *out) {
    PyObject *v = PyObject_GetAttr(layer, name);
    const bool ok = v && PyLong_CheckExact(v);
    if (ok) *out = PyLong_AsLong(v);
    Py_XDECREF(v);
    return ok && !(*out == -1 && PyErr_Occurred());
  }
};

// A strided tensor of torch's own class on one GPU, and nothing that would intercept or defer an operator on it.
const at::Tensor *plain_tensor(PyObject *x) {
  if (!THPVariable_CheckExact(x)) return nullptr;
  const at::Tensor &t = THPVariable_Unpack(x);
  const c10::DispatchKeySet plain({c10::DispatchKey::CUDA, c10::DispatchKey::ADInplaceOrView, c10::DispatchKey::AutogradCUDA, c10::DispatchKey::AutocastCUDA});
  if (!t.defined() || (t.key_set().raw_repr() & ~plain.raw_repr()) != 0 || t.layout() != c10::kStrided) return nullptr;
  if (!t.device().is_cuda() || !t.device().has_index()) return nullptr;
  return &t;
}

bool intercepted() {
  return c10::impl::dispatch_mode_enabled() || at::impl::torch_function_mode_enabled() || c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::Tracer) ||
         c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::Functionalize) || c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::FuncTorchDynamicLayerFrontMode);
}

// x as the layers' kernels take it: [B][d] contiguous fp32 on the layer's GPU.
const at::Tensor *plain_input(PyObject *x, long d, c10::Device device) {
  const at::Tensor *t = plain_tensor(x);
  if (!t || t->scalar_type() != at::kFloat || t->device() != device || t->dim() != 2 || t->size(1) != d || !t->is_contiguous()) return nullptr;
  return intercepted() ? nullptr : t;
}

bool stream_of(c10::Device device, void **out) {
  PyObject *index = PyLong_FromLong(device.index());
  PyObject *handle = index ? PyObject_CallOneArg(g.current_stream, index) : nullptr;
  Py_XDECREF(index);
  if (!handle) return false;
  *out = PyLong_AsVoidPtr(handle);
  Py_DECREF(handle);
  return !PyErr_Occurred();
}

at::Tensor workspace_of(size_t bytes, c10::Device device) {
  return at::empty({(int64_t)std::max<size_t>(bytes, 256)}, at::TensorOptions().dtype(at::kByte).device(device));
}

PyObject *not_taken() {
  PyErr_Clear();
  Py_RETURN_NONE;
}

struct WithoutLock {
  PyThreadState *state = PyEval_SaveThread();
  ~WithoutLock() { PyEval_RestoreThread(state); }
};

// once(needed): the call that runs without a workspace or says how much one takes; again(workspace, bytes): the call with one.
template <typename Once, typename Again>
PyObject *forward(const at::Tensor &x, long m, c10::Device device, const Once &once, const Again &again) {
  try {
    void *stream = nullptr;
    if (!stream_of(device, &stream)) return not_taken();
    at::Tensor y;
    int rc;
    {
      const WithoutLock unlocked;
      y = at::empty({x.size(0), m}, x.options().requires_grad(false));
      const float *in = x.const_data_ptr<float>();
      float *out = y.mutable_data_ptr<float>();
      const int64_t B = x.size(0);
      size_t needed = 0;
      rc = once(in, B, out, &needed, stream);
      if (rc == LUTKAN_OK && needed != 0) {
        const at::Tensor workspace = workspace_of(needed, device);
        rc = again(in, B, out, workspace.mutable_data_ptr(), (size_t)workspace.numel(), stream);
      }
    }
    if (rc != LUTKAN_OK) return not_taken();
    return THPVariable_Wrap(y);
  } catch (...) {                                          // no exception crosses into the interpreter: the general path reports it
    return not_taken();
  }
}

PyObject *lut_forward(PyObject *, PyObject *const *args, Py_ssize_t n) {
  Layer layer;
  if (n != 2 || !layer.read(args[0], g.lut_struct, sizeof(lutkan_dev_layer))) return not_taken();
  const at::Tensor *x = plain_input(args[1], layer.d, layer.device);
  if (!x) return not_taken();
  const auto *l = static_cast<const lutkan_dev_layer *>(layer.c.buf);
  return forward(*x, layer.m, layer.device,
                 [&](const float *in, int64_t B, float *out, size_t *needed, void *stream) { return g.forward_or_workspace(l, in, B, out, nullptr, needed, stream); },
                 [&](const float *in, int64_t B, float *out, void *ws, size_t bytes, void *stream) { return g.forward(l, in, B, out, nullptr, ws, bytes, stream); });
}

PyObject *lut_model_forward(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 2 || !(PyList_CheckExact(args[0]) || PyTuple_CheckExact(args[0]))) return not_taken();
  const Py_ssize_t count = PySequence_Fast_GET_SIZE(args[0]);
  if (count < 1 || count > LUTKAN_MAX_LAYERS) return not_taken();
  lutkan_dev_layer layers[LUTKAN_MAX_LAYERS];
  long d = 0, m = 0;
  c10::Device device(c10::kCPU);
  for (Py_ssize_t i = 0; i < count; ++i) {
    if (i >= PySequence_Fast_GET_SIZE(args[0])) return not_taken();                  // reading an attribute may run code that changes the list
    PyObject *const item = PySequence_Fast_GET_ITEM(args[0], i);
    Py_INCREF(item);
    Layer layer;
    const bool ok = layer.read(item, g.lut_struct, sizeof(lutkan_dev_layer));
    Py_DECREF(item);
    if (!ok) return not_taken();
    if (i == 0) { d = layer.d; device = layer.device; }
    if (layer.device != device) return not_taken();
    m = layer.m;
    std::memcpy(&layers[i], layer.c.buf, sizeof(lutkan_dev_layer));
  }
  const at::Tensor *x = plain_input(args[1], d, device);
  if (!x) return not_taken();
  const int32_t n_layers = (int32_t)count;
  return forward(*x, m, device,
                 [&](const float *in, int64_t B, float *out, size_t *needed, void *stream) { return g.model_or_workspace(layers, n_layers, in, B, out, nullptr, needed, stream); },
                 [&](const float *in, int64_t B, float *out, void *ws, size_t bytes, void *stream) { return g.model(layers, n_layers, in, B, out, nullptr, ws, bytes, stream); });
}

PyObject *spline_forward(PyObject *, PyObject *const *args, Py_ssize_t n) {
  Layer layer;
  if (n != 2 || !layer.read(args[0], g.spline_struct, sizeof(bspline_dev_layer))) return not_taken();
  const at::Tensor *x = plain_input(args[1], layer.d, layer.device);
  if (!x) return not_taken();
  const auto *l = static_cast<const bspline_dev_layer *>(layer.c.buf);
  return forward(*x, layer.m, layer.device,
                 [&](const float *, int64_t B, float *, size_t *needed, void *) { *needed = std::max<size_t>(g.spline_workspace_bytes(l, B), 256); return LUTKAN_OK; },
                 [&](const float *in, int64_t B, float *out, void *ws, size_t bytes, void *stream) { return g.spline(l, in, B, out, ws, bytes, stream); });
}

// ---- the 8-bit operators: arguments as the binding's functions of the same names take them, without the optional outputs
int type_of(const at::Tensor &t) {
  switch (t.scalar_type()) {
    case at::kFloat: return LUTKAN_F32;
    case at::kHalf: return LUTKAN_F16;
    case at::kBFloat16: return LUTKAN_BF16;
    default: return -1;
  }
}

int64_t blocks(int64_t n) { return (n + 127) / 128; }

// Rows of contiguous columns (the stride of a dimension of one element is arbitrary and not used).
bool is_rows(const at::Tensor &t, int64_t dims) { return t.dim() == dims && (t.size(dims - 1) <= 1 || t.stride(dims - 1) == 1); }
int64_t row_stride(const at::Tensor &t) { return t.size(-2) > 1 ? t.stride(-2) : t.size(-1); }

// Allocates and calls without the interpreter's lock, on the tensors' GPU: `work(stream)` returns the library's status.
template <typename Work>
bool on_device(const at::Tensor &x, const Work &work) {
  void *stream = nullptr;
  if (!stream_of(x.device(), &stream)) return false;
  const WithoutLock unlocked;
  const c10::DeviceGuard guard(x.device());
  return work(stream) == LUTKAN_OK;
}

// A contiguous matrix in the memory of `held` (bytes), from byte `at` on.
at::Tensor matrix_in(const at::Tensor &held, int64_t at, at::ScalarType type, int64_t rows, int64_t columns) {
  at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(held.storage()), held.key_set(), c10::scalarTypeToTypeMeta(type));
  c10::TensorImpl *impl = t.unsafeGetTensorImpl();
  impl->set_sizes_contiguous({rows, columns});
  impl->set_storage_offset(at / (int64_t)c10::elementSize(type));
  return t;
}

PyObject *none() { Py_RETURN_NONE; }

PyObject *wrapped(const at::Tensor &a, const at::Tensor &b) {
  PyObject *pair = PyTuple_New(2), *x = THPVariable_Wrap(a), *y = THPVariable_Wrap(b);
  if (!pair || !x || !y) { Py_XDECREF(pair); Py_XDECREF(x); Py_XDECREF(y); return nullptr; }
  PyTuple_SET_ITEM(pair, 0, x);
  PyTuple_SET_ITEM(pair, 1, y);
  return pair;
}

// rmsnorm_fp8(x, weight, residual or None, eps)
PyObject *rmsnorm_fp8(PyObject *, PyObject *const *args, Py_ssize_t n) {
  try {
    if (n != 4 || !PyFloat_CheckExact(args[3])) return not_taken();
    const at::Tensor *x = plain_tensor(args[0]), *w = plain_tensor(args[1]), *r = args[2] == Py_None ? nullptr : plain_tensor(args[2]);
    if (!x || !w || (args[2] != Py_None && !r) || intercepted()) return not_taken();
    if (!is_rows(*x, 2) || !is_rows(*w, 1) || type_of(*x) < 0 || type_of(*w) < 0 || w->size(0) != x->size(1) || w->device() != x->device()) return not_taken();
    if (r && (!is_rows(*r, 2) || type_of(*r) < 0 || r->size(0) != x->size(0) || r->size(1) != x->size(1) || r->device() != x->device())) return not_taken();
    const int64_t rows = x->size(0), width = x->size(1);
    if (width > INT32_MAX) return not_taken();
    lutkan_rmsnorm_fp8_args a{};
    at::Tensor codes, scales, out;
    const bool ok = on_device(*x, [&](void *stream) {
      const auto options = x->options().requires_grad(false);
      const int64_t scales_at = (rows * width + 255) / 256 * 256;            // codes and scales go together: one allocation, 0.5 us less
      const at::Tensor held = at::empty({scales_at + rows * blocks(width) * 4}, options.dtype(at::kByte));
      codes = matrix_in(held, 0, at::kFloat8_e4m3fn, rows, width);
      scales = matrix_in(held, scales_at, at::kFloat, rows, blocks(width));
      a.x = x->const_data_ptr(); a.weight = w->const_data_ptr();
      a.codes = codes.mutable_data_ptr(); a.scales = scales.mutable_data_ptr<float>();
      a.x_stride = row_stride(*x); a.codes_stride = width; a.scales_stride = blocks(width);
      a.rows = rows; a.width = (int32_t)width; a.x_type = type_of(*x); a.weight_type = type_of(*w); a.eps = (float)PyFloat_AS_DOUBLE(args[3]);
      if (r) {
        out = at::empty({rows, width}, r->options().requires_grad(false));
        a.residual = r->const_data_ptr(); a.residual_type = type_of(*r); a.residual_stride = row_stride(*r);
        a.residual_out = out.mutable_data_ptr(); a.residual_out_stride = width;
      }
      return g.rmsnorm(&a, stream);
    });
    if (!ok) return not_taken();
    PyObject *three = PyTuple_New(3), *c = THPVariable_Wrap(codes), *s = THPVariable_Wrap(scales), *o = r ? THPVariable_Wrap(out) : none();
    if (!three || !c || !s || !o) { Py_XDECREF(three); Py_XDECREF(c); Py_XDECREF(s); Py_XDECREF(o); return nullptr; }
    PyTuple_SET_ITEM(three, 0, c);
    PyTuple_SET_ITEM(three, 1, s);
    PyTuple_SET_ITEM(three, 2, o);
    return three;
  } catch (...) {
    return not_taken();
  }
}

// quantise_fp8(weight)
PyObject *quantise_fp8(PyObject *, PyObject *const *args, Py_ssize_t n) {
  try {
    const at::Tensor *w = n == 1 ? plain_tensor(args[0]) : nullptr;
    if (!w || intercepted() || type_of(*w) < 0 || !(is_rows(*w, 2) || is_rows(*w, 3))) return not_taken();
    const int64_t rows = w->size(-2), k = w->size(-1);
    if (rows > INT32_MAX || k > INT32_MAX) return not_taken();
    const bool several = w->dim() == 3;
    at::Tensor codes, scales;
    const bool ok = on_device(*w, [&](void *stream) {
      const auto options = w->options().requires_grad(false);
      codes = at::empty(w->sizes(), options.dtype(at::kFloat8_e4m3fn));
      scales = several ? at::empty({w->size(0), blocks(rows), blocks(k)}, options.dtype(at::kFloat)) : at::empty({blocks(rows), blocks(k)}, options.dtype(at::kFloat));
      return g.quantise(w->const_data_ptr(), type_of(*w), several ? w->size(0) : 1, (int32_t)rows, (int32_t)k, row_stride(*w), several ? w->stride(0) : 0,
                        codes.mutable_data_ptr(), scales.mutable_data_ptr<float>(), stream);
    });
    return ok ? wrapped(codes, scales) : not_taken();
  } catch (...) {
    return not_taken();
  }
}

bool is_whole_numbers(const at::Tensor &t) { return t.dim() == 1 && t.is_contiguous() && (t.scalar_type() == at::kInt || t.scalar_type() == at::kLong); }

// matmul_fp8(x, x_scales, weight, weight_scales, dtype) and, with two more, group_sizes and rows or None
PyObject *matmul_fp8(PyObject *, PyObject *const *args, Py_ssize_t n) {
  try {
    const bool grouped = n == 7;
    if ((n != 5 && n != 7) || !THPDtype_Check(args[4])) return not_taken();
    const at::Tensor *x = plain_tensor(args[0]), *xs = plain_tensor(args[1]), *w = plain_tensor(args[2]), *ws = plain_tensor(args[3]);
    const at::Tensor *sizes = grouped ? plain_tensor(args[5]) : nullptr, *index = grouped && args[6] != Py_None ? plain_tensor(args[6]) : nullptr;
    if (!x || !xs || !w || !ws || (grouped && (!sizes || (args[6] != Py_None && !index))) || intercepted()) return not_taken();
    const int64_t dims = grouped ? 3 : 2;
    if (!is_rows(*x, 2) || !is_rows(*xs, 2) || !is_rows(*w, dims) || ws->dim() != dims || !ws->is_contiguous()) return not_taken();
    if (x->scalar_type() != at::kFloat8_e4m3fn || w->scalar_type() != at::kFloat8_e4m3fn || xs->scalar_type() != at::kFloat || ws->scalar_type() != at::kFloat) return not_taken();
    const int64_t k = x->size(1), columns = w->size(-2);
    if (w->size(-1) != k || xs->size(0) != x->size(0) || xs->size(1) != blocks(k) || ws->size(-2) != blocks(columns) || ws->size(-1) != blocks(k)) return not_taken();
    if (xs->device() != x->device() || w->device() != x->device() || ws->device() != x->device() || k > INT32_MAX || columns > INT32_MAX) return not_taken();
    if (grouped) {
      if (ws->size(0) != w->size(0) || w->size(0) > INT32_MAX || !is_whole_numbers(*sizes) || sizes->size(0) != w->size(0) || sizes->device() != x->device()) return not_taken();
      if (index && (!is_whole_numbers(*index) || index->device() != x->device())) return not_taken();
    }
    lutkan_matmul_fp8_args a{};
    a.rows = index ? index->size(0) : x->size(0);
    at::Tensor y;
    const bool ok = on_device(*x, [&](void *stream) {
      y = at::empty({a.rows, columns}, x->options().requires_grad(false).dtype(reinterpret_cast<THPDtype *>(args[4])->scalar_type));
      a.x = x->const_data_ptr(); a.x_scales = xs->const_data_ptr<float>(); a.weight = w->const_data_ptr(); a.weight_scales = ws->const_data_ptr<float>();
      a.y = y.mutable_data_ptr();
      a.x_rows = x->size(0); a.x_stride = row_stride(*x); a.x_scales_stride = row_stride(*xs); a.weight_stride = row_stride(*w); a.y_stride = columns;
      a.weight_matrix_stride = grouped ? w->stride(0) : 0;
      a.k = (int32_t)k; a.n = (int32_t)columns; a.y_type = type_of(y);
      if (grouped) {
        a.groups = (int32_t)w->size(0);
        a.group_sizes = sizes->const_data_ptr(); a.group_sizes_bytes = (int32_t)sizes->element_size();
        if (index) { a.row_index = index->const_data_ptr(); a.row_index_bytes = (int32_t)index->element_size(); }
      }
      return grouped ? g.grouped_matmul(&a, stream) : g.matmul(&a, stream);
    });
    return ok ? THPVariable_Wrap(y) : not_taken();
  } catch (...) {
    return not_taken();
  }
}

// init(addresses of the ten entry points, the two struct classes, the stream function)
PyObject *init(PyObject *, PyObject *args) {
  unsigned long long p[10];
  PyObject *lut_struct, *spline_struct, *current_stream;
  if (!PyArg_ParseTuple(args, "KKKKKKKKKKOOO", &p[0], &p[1], &p[2], &p[3], &p[4], &p[5], &p[6], &p[7], &p[8], &p[9], &lut_struct, &spline_struct, &current_stream)) return nullptr;
  g.forward_or_workspace = reinterpret_cast<decltype(g.forward_or_workspace)>(p[0]);
  g.forward = reinterpret_cast<decltype(g.forward)>(p[1]);
  g.model_or_workspace = reinterpret_cast<decltype(g.model_or_workspace)>(p[2]);
  g.model = reinterpret_cast<decltype(g.model)>(p[3]);
  g.spline_workspace_bytes = reinterpret_cast<decltype(g.spline_workspace_bytes)>(p[4]);
  g.spline = reinterpret_cast<decltype(g.spline)>(p[5]);
  g.rmsnorm = reinterpret_cast<decltype(g.rmsnorm)>(p[6]);
  g.quantise = reinterpret_cast<decltype(g.quantise)>(p[7]);
  g.matmul = reinterpret_cast<decltype(g.matmul)>(p[8]);
  g.grouped_matmul = reinterpret_cast<decltype(g.grouped_matmul)>(p[9]);
  Py_INCREF(lut_struct); Py_INCREF(spline_struct); Py_INCREF(current_stream);
  g.lut_struct = lut_struct; g.spline_struct = spline_struct; g.current_stream = current_stream;
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"init", init, METH_VARARGS, nullptr},
                         {"lut_forward", (PyCFunction)(void (*)())lut_forward, METH_FASTCALL, nullptr},
                         {"lut_model_forward", (PyCFunction)(void (*)())lut_model_forward, METH_FASTCALL, nullptr},
                         {"spline_forward", (PyCFunction)(void (*)())spline_forward, METH_FASTCALL, nullptr},
                         {"rmsnorm_fp8", (PyCFunction)(void (*)())rmsnorm_fp8, METH_FASTCALL, nullptr},
                         {"quantise_fp8", (PyCFunction)(void (*)())quantise_fp8, METH_FASTCALL, nullptr},
                         {"matmul_fp8", (PyCFunction)(void (*)())matmul_fp8, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lutkan_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lutkan_call() {
  s_c = PyUnicode_InternFromString("c");
  s_d = PyUnicode_InternFromString("d");
  s_m = PyUnicode_InternFromString("m");
  s_device = PyUnicode_InternFromString("device");
  return (s_c && s_d && s_m && s_device) ? PyModule_Create(&module) : nullptr;
}

// The Python binding's common calls in native code: operand checks, output
// and workspace allocation, and the library call, for tensors on the current
// stream of their device.
//
// Each function takes its operands as positional arguments (None where the
// caller gave none) and returns the call's result, a nonzero status as an
// int, or None when it does not take the call: any operand that is not
// exactly what the C-ABI expects, a tensor subclass, a tensor without
// storage.  The caller then runs the same call through the Python checks,
// which raise the error or handle the general case, so nothing is decided
// here but the plain valid call.
//
// What it saves is host time on small layers, whose kernels take a few
// microseconds: the 128-token 1152 -> 1152 linear took 33.7 us a call with
// the checks and allocations in Python (two of them under a stream context)
// for 10 us of kernels, and 13.6 here (9.4 since its quantizer is one launch);
// with a kept output and workspace, in MXFP4, 14.5 -> 8.2.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/Context.h>
#include <ATen/hip/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/impl/LocalDispatchKeySet.h>

#include "solfp4.h"

namespace {

using at::Tensor;

PyObject* current_raw_stream = nullptr;   // torch._C._cuda_getCurrentRawStream

// Thrown (and caught at the entry) when the native path does not take a call.
struct NotTaken {};

const Tensor& tensor(PyObject* o) {
  if (!THPVariable_CheckExact(o)) throw NotTaken{};
  return THPVariable_Unpack(o);
}

void need(bool ok) {
  if (!ok) throw NotTaken{};
}

// A contiguous GPU tensor of this type and shape (on `dev`, when given).
void need_tensor(const Tensor& t, at::ScalarType type, at::IntArrayRef shape, const at::Device* dev) {
  need(t.is_cuda() && t.scalar_type() == type && t.layout() == at::kStrided && t.sizes() == shape &&
       t.is_contiguous() && (!dev || t.device() == *dev));
}

void need_matrix(const Tensor& t) { need(t.layout() == at::kStrided && t.dim() == 2); }

// The device's allocation itself, without the dispatcher's way to it (0.3 us
// an output), unless a dispatch mode looks on or torch is asked to fill fresh
// memory.
Tensor make(at::IntArrayRef shape, at::ScalarType type, const at::Device& dev) {
  const at::Context& context = at::globalContext();
  if (c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::Python) ||
      (context.deterministicAlgorithms() && context.deterministicFillUninitializedMemory()))
    return at::empty(shape, at::TensorOptions().dtype(type).device(dev));
  return at::detail::empty_cuda(shape, type, dev, std::nullopt);
}

// An operand that the caller gives or leaves to the call, and its Python object.
struct Operand {
  Tensor t;
  PyObject* given = nullptr;   // borrowed
  Operand(PyObject* o, at::ScalarType type, at::IntArrayRef shape, const at::Device& dev) {
    if (o != Py_None) {
      t = tensor(o);
      need_tensor(t, type, shape, &dev);
      given = o;
    }
  }
  void allocate(at::ScalarType type, at::IntArrayRef shape, const at::Device& dev) {
    if (!given) t = make(shape, type, dev);
  }
  PyObject* object() const {
    if (!given) return THPVariable_Wrap(t);
    Py_INCREF(given);
    return given;
  }
};

Tensor workspace_arg(PyObject* o, size_t bytes, const at::Device& dev) {
  if (o == Py_None) return Tensor();
  const Tensor& t = tensor(o);
  need(t.is_cuda() && t.scalar_type() == at::kByte && t.layout() == at::kStrided && t.dim() == 1 &&
       t.is_contiguous() && t.device() == dev && t.numel() >= (int64_t)bytes);
  return t;
}

void* ptr(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
uint8_t* u8(const Tensor& t) { return static_cast<uint8_t*>(ptr(t)); }
uint16_t* u16(const Tensor& t) { return static_cast<uint16_t*>(ptr(t)); }
float* f32(const Tensor& t) { return static_cast<float*>(ptr(t)); }

// The current stream of `dev`, as the C-ABI takes it.
void* stream_of(const at::Device& dev) {
  PyObject* index = PyLong_FromLong(dev.index());
  PyObject* r = index ? PyObject_CallOneArg(current_raw_stream, index) : nullptr;
  Py_XDECREF(index);
  void* s = r ? PyLong_AsVoidPtr(r) : nullptr;
  Py_XDECREF(r);
  if (PyErr_Occurred()) throw NotTaken{};
  return s;
}

struct NoGil {
  PyThreadState* state = PyEval_SaveThread();
  ~NoGil() { PyEval_RestoreThread(state); }
};

template <typename F>
int call(F&& f) {
  NoGil released;
  return f();
}

template <typename F>
PyObject* entry(Py_ssize_t got, Py_ssize_t want, F&& f) {
  if (got != want) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return f();
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

PyObject* failed(int status) { return PyLong_FromLong(status); }

// (x, codes, scales, global_scale, workspace) -> (codes, scales, global_scale)
PyObject* nvfp4_quantize_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 5, [&]() -> PyObject* {
    const Tensor& x = tensor(a[0]);
    need_matrix(x);
    const int64_t rows = x.size(0), K = x.size(1);
    need(K % 16 == 0);
    need_tensor(x, at::kBFloat16, {rows, K}, nullptr);
    const at::Device dev = x.device();
    Operand codes(a[1], at::kByte, {rows, K / 2}, dev), scales(a[2], at::kByte, {rows, K / 16}, dev);
    Operand gs(a[3], at::kFloat, {1}, dev);
    const size_t bytes = nvfp4_quantize_workspace_bytes(rows, K);
    Tensor ws = workspace_arg(a[4], bytes, dev);
    void* stream = stream_of(dev);
    codes.allocate(at::kByte, {rows, K / 2}, dev);
    scales.allocate(at::kByte, {rows, K / 16}, dev);
    gs.allocate(at::kFloat, {1}, dev);
    if (!ws.defined()) ws = make({(int64_t)std::max<size_t>(bytes, 256)}, at::kByte, dev);
    const int rc = call([&] {
      return nvfp4_quantize(u16(x), rows, K, u8(codes.t), u8(scales.t), f32(gs.t), ptr(ws),
                            (size_t)ws.numel(), stream);
    });
    if (rc) return failed(rc);
    return Py_BuildValue("(NNN)", codes.object(), scales.object(), gs.object());
  });
}

// (x, codes, scales) -> (codes, scales)
PyObject* mxfp4_quantize_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 3, [&]() -> PyObject* {
    const Tensor& x = tensor(a[0]);
    need_matrix(x);
    const int64_t rows = x.size(0), K = x.size(1);
    need(K % 32 == 0);
    need_tensor(x, at::kBFloat16, {rows, K}, nullptr);
    const at::Device dev = x.device();
    Operand codes(a[1], at::kByte, {rows, K / 2}, dev), scales(a[2], at::kByte, {rows, K / 32}, dev);
    void* stream = stream_of(dev);
    codes.allocate(at::kByte, {rows, K / 2}, dev);
    scales.allocate(at::kByte, {rows, K / 32}, dev);
    const int rc = call([&] { return mxfp4_quantize(u16(x), rows, K, u8(codes.t), u8(scales.t), stream); });
    if (rc) return failed(rc);
    return Py_BuildValue("(NN)", codes.object(), scales.object());
  });
}

// (a_codes, a_scales, a_gs, b_codes, b_scales, b_gs, bias, out, workspace) -> out
PyObject* nvfp4_gemm_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 9, [&]() -> PyObject* {
    const Tensor &ac = tensor(a[0]), &as = tensor(a[1]), &ag = tensor(a[2]);
    const Tensor &bc = tensor(a[3]), &bs = tensor(a[4]), &bg = tensor(a[5]);
    need_matrix(ac);
    need_matrix(bc);
    const int64_t M = ac.size(0), N = bc.size(0), K = 2 * ac.size(1);
    need(K % 16 == 0);
    need_tensor(ac, at::kByte, {M, K / 2}, nullptr);
    const at::Device dev = ac.device();
    need_tensor(as, at::kByte, {M, K / 16}, &dev);
    need_tensor(ag, at::kFloat, {1}, &dev);
    need_tensor(bc, at::kByte, {N, K / 2}, &dev);
    need_tensor(bs, at::kByte, {N, K / 16}, &dev);
    need_tensor(bg, at::kFloat, {1}, &dev);
    Operand bias(a[6], at::kBFloat16, {N}, dev), out(a[7], at::kBFloat16, {M, N}, dev);
    const size_t bytes = nvfp4_gemm_workspace_bytes(M, N, K);
    Tensor ws = workspace_arg(a[8], bytes, dev);
    void* stream = stream_of(dev);
    out.allocate(at::kBFloat16, {M, N}, dev);
    if (!ws.defined() && bytes) ws = make({(int64_t)bytes}, at::kByte, dev);
    const int rc = call([&] {
      return nvfp4_gemm(u8(ac), u8(as), f32(ag), u8(bc), u8(bs), f32(bg), u16(bias.t), u16(out.t), ptr(ws),
                        ws.defined() ? (size_t)ws.numel() : 0, M, N, K, stream);
    });
    return rc ? failed(rc) : out.object();
  });
}

// (a_codes, a_scales, b_codes, b_scales, bias, out) -> out
PyObject* mxfp4_gemm_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 6, [&]() -> PyObject* {
    const Tensor &ac = tensor(a[0]), &as = tensor(a[1]), &bc = tensor(a[2]), &bs = tensor(a[3]);
    need_matrix(ac);
    need_matrix(bc);
    const int64_t M = ac.size(0), N = bc.size(0), K = 2 * ac.size(1);
    need(K % 32 == 0);
    need_tensor(ac, at::kByte, {M, K / 2}, nullptr);
    const at::Device dev = ac.device();
    need_tensor(as, at::kByte, {M, K / 32}, &dev);
    need_tensor(bc, at::kByte, {N, K / 2}, &dev);
    need_tensor(bs, at::kByte, {N, K / 32}, &dev);
    Operand bias(a[4], at::kBFloat16, {N}, dev), out(a[5], at::kBFloat16, {M, N}, dev);
    void* stream = stream_of(dev);
    out.allocate(at::kBFloat16, {M, N}, dev);
    const int rc = call([&] {
      return mxfp4_gemm(u8(ac), u8(as), u8(bc), u8(bs), u16(bias.t), u16(out.t), M, N, K, stream);
    });
    return rc ? failed(rc) : out.object();
  });
}

// (x, w_codes, w_scales, w_gs, bias, out, workspace) -> out
PyObject* nvfp4_linear_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 7, [&]() -> PyObject* {
    const Tensor &x = tensor(a[0]), &wc = tensor(a[1]), &ws_ = tensor(a[2]), &wg = tensor(a[3]);
    need_matrix(x);
    need_matrix(wc);
    const int64_t M = x.size(0), K = x.size(1), N = wc.size(0);
    need(K % 16 == 0);
    need_tensor(x, at::kBFloat16, {M, K}, nullptr);
    const at::Device dev = x.device();
    need_tensor(wc, at::kByte, {N, K / 2}, &dev);
    need_tensor(ws_, at::kByte, {N, K / 16}, &dev);
    need_tensor(wg, at::kFloat, {1}, &dev);
    Operand bias(a[4], at::kBFloat16, {N}, dev), out(a[5], at::kBFloat16, {M, N}, dev);
    const size_t bytes = nvfp4_linear_workspace_bytes(M, N, K);
    Tensor ws = workspace_arg(a[6], bytes, dev);
    void* stream = stream_of(dev);
    out.allocate(at::kBFloat16, {M, N}, dev);
    if (!ws.defined()) ws = make({(int64_t)bytes}, at::kByte, dev);
    const int rc = call([&] {
      return nvfp4_linear(u16(x), u8(wc), u8(ws_), f32(wg), u16(bias.t), u16(out.t), ptr(ws),
                          (size_t)ws.numel(), M, N, K, stream);
    });
    return rc ? failed(rc) : out.object();
  });
}

// (x, w_codes, w_scales, bias, out, workspace) -> out
PyObject* mxfp4_linear_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 6, [&]() -> PyObject* {
    const Tensor &x = tensor(a[0]), &wc = tensor(a[1]), &ws_ = tensor(a[2]);
    need_matrix(x);
    need_matrix(wc);
    const int64_t M = x.size(0), K = x.size(1), N = wc.size(0);
    need(K % 32 == 0);
    need_tensor(x, at::kBFloat16, {M, K}, nullptr);
    const at::Device dev = x.device();
    need_tensor(wc, at::kByte, {N, K / 2}, &dev);
    need_tensor(ws_, at::kByte, {N, K / 32}, &dev);
    Operand bias(a[3], at::kBFloat16, {N}, dev), out(a[4], at::kBFloat16, {M, N}, dev);
    const size_t bytes = mxfp4_linear_workspace_bytes(M, K);
    Tensor ws = workspace_arg(a[5], bytes, dev);
    void* stream = stream_of(dev);
    out.allocate(at::kBFloat16, {M, N}, dev);
    if (!ws.defined()) ws = make({(int64_t)bytes}, at::kByte, dev);
    const int rc = call([&] {
      return mxfp4_linear(u16(x), u8(wc), u8(ws_), u16(bias.t), u16(out.t), ptr(ws), (size_t)ws.numel(), M,
                          N, K, stream);
    });
    return rc ? failed(rc) : out.object();
  });
}

// ---- operators around the linears -----------------------------------------

int type_of(const Tensor& t) {
  switch (t.scalar_type()) {
    case at::kBFloat16: return SOLFP4_BF16;
    case at::kHalf: return SOLFP4_F16;
    case at::kFloat: return SOLFP4_F32;
    default: throw NotTaken{};
  }
}

// A GPU tensor like `like` in type and device, of this shape, whose last
// dimension is contiguous.
void need_strided(const Tensor& t, const Tensor& like, at::IntArrayRef shape) {
  need(t.is_cuda() && t.layout() == at::kStrided && t.scalar_type() == like.scalar_type() && t.sizes() == shape &&
       t.device() == like.device() && (shape.back() <= 1 || t.stride(-1) == 1));
}

// An operand with strides that the caller may leave out.
struct Strided {
  Tensor t;
  PyObject* given = nullptr;   // borrowed
  Strided(PyObject* o, const Tensor& like, at::IntArrayRef shape) {
    if (o == Py_None) return;
    t = tensor(o);
    need_strided(t, like, shape);
    given = o;
  }
  int64_t stride(int64_t d) const { return t.defined() ? t.stride(d) : 0; }
  void allocate(const Tensor& like, at::IntArrayRef shape) {
    if (!given) t = make(shape, like.scalar_type(), like.device());
  }
  PyObject* object() const {
    if (!t.defined()) Py_RETURN_NONE;
    if (!given) return THPVariable_Wrap(t);
    Py_INCREF(given);
    return given;
  }
};

double number(PyObject* o) {
  need(PyFloat_CheckExact(o) || PyLong_CheckExact(o));
  const double v = PyFloat_AsDouble(o);
  need(!PyErr_Occurred());
  return v;
}

struct Gain {
  Tensor t;
  int64_t groups = 1, stride = 0;
  Gain(PyObject* o, const Tensor& x, int64_t rows, int64_t width) {
    if (o == Py_None) return;
    t = tensor(o);
    need(t.layout() == at::kStrided && (t.dim() == 1 || t.dim() == 2));
    if (t.dim() == 1) {
      need_strided(t, x, {width});
    } else {
      groups = t.size(0);
      need_strided(t, x, {groups, width});
      stride = t.stride(0);
    }
    need(groups >= 1 && rows % groups == 0);
  }
};

// The shift beside the gain: its shape where there is one.
struct Shift : Gain {
  Shift(PyObject* o, const Gain& gain, const Tensor& x, int64_t rows, int64_t width) : Gain(o, x, rows, width) {
    need(!t.defined() || !gain.t.defined() || t.sizes() == gain.t.sizes());
    if (!t.defined()) groups = gain.groups;
  }
};

const Tensor& matrix_operand(PyObject* o) {
  const Tensor& x = tensor(o);
  need_matrix(x);
  type_of(x);
  need_strided(x, x, x.sizes());
  return x;
}

// (x, residual, gain, eps, out, sum_out) -> (out, sum)
PyObject* add_rmsnorm_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 6, [&]() -> PyObject* {
    const Tensor& x = matrix_operand(a[0]);
    const int64_t rows = x.size(0), width = x.size(1);
    Strided r(a[1], x, {rows, width}), out(a[4], x, {rows, width}), sum(a[5], x, {rows, width});
    Gain g(a[2], x, rows, width);
    const double eps = number(a[3]);
    need(eps >= 0);
    need(r.given || !sum.given);
    void* stream = stream_of(x.device());
    out.allocate(x, {rows, width});
    if (r.given) sum.allocate(x, {rows, width});
    const int rc = call([&] {
      return solfp4_add_rmsnorm(type_of(x), ptr(x), x.stride(0), ptr(r.t), r.stride(0), ptr(g.t), g.stride, g.groups,
                                (float)eps, ptr(sum.t), sum.stride(0), ptr(out.t), out.stride(0), rows, width, stream);
    });
    if (rc) return failed(rc);
    return Py_BuildValue("(NN)", out.object(), sum.object());
  });
}

// (x, residual, gain, eps, codes, scales, sum_out) -> (codes, scales, sum)
template <typename F>
PyObject* quantized_norm(PyObject* const* a, Py_ssize_t n, int pack, F f) {
  return entry(n, 7, [&]() -> PyObject* {
    const Tensor& x = matrix_operand(a[0]);
    const int64_t rows = x.size(0), width = x.size(1);
    need(width % 32 == 0);
    const at::Device dev = x.device();
    Strided r(a[1], x, {rows, width}), sum(a[6], x, {rows, width});
    Gain g(a[2], x, rows, width);
    const double eps = number(a[3]);
    need(eps >= 0);
    Operand codes(a[4], at::kByte, {rows, width / pack}, dev), scales(a[5], at::kByte, {rows, width / 32}, dev);
    need(r.given || !sum.given);
    void* stream = stream_of(dev);
    codes.allocate(at::kByte, {rows, width / pack}, dev);
    scales.allocate(at::kByte, {rows, width / 32}, dev);
    if (r.given) sum.allocate(x, {rows, width});
    const int rc = call([&] {
      return f(type_of(x), ptr(x), x.stride(0), ptr(r.t), r.stride(0), ptr(g.t), g.stride, g.groups, (float)eps,
               ptr(sum.t), sum.stride(0), u8(codes.t), u8(scales.t), rows, width, stream);
    });
    if (rc) return failed(rc);
    return Py_BuildValue("(NNN)", codes.object(), scales.object(), sum.object());
  });
}

PyObject* mxfp8_add_rmsnorm_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return quantized_norm(a, n, 1, mxfp8_add_rmsnorm);
}
PyObject* mxfp4_add_rmsnorm_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return quantized_norm(a, n, 2, mxfp4_add_rmsnorm);
}

// (dy, x, gain, dsum, eps, dx, dgain, workspace) -> (dx, dgain)
PyObject* rmsnorm_backward_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 8, [&]() -> PyObject* {
    const Tensor& x = matrix_operand(a[1]);
    const int64_t rows = x.size(0), width = x.size(1);
    const Tensor& dy = tensor(a[0]);
    need_strided(dy, x, {rows, width});
    Gain g(a[2], x, rows, width);
    Strided dsum(a[3], x, {rows, width}), dx(a[5], x, {rows, width});
    const double eps = number(a[4]);
    need(eps >= 0);
    const at::Device dev = x.device();
    const at::IntArrayRef shape = g.t.defined() ? g.t.sizes() : at::IntArrayRef();
    need(g.t.defined() || a[6] == Py_None);
    Operand dgain(a[6], at::kFloat, shape, dev);
    const size_t bytes = g.t.defined() ? solfp4_rmsnorm_backward_workspace_bytes(rows, width, g.groups) : 0;
    Tensor ws = g.t.defined() ? workspace_arg(a[7], bytes, dev) : Tensor();
    void* stream = stream_of(dev);
    dx.allocate(x, {rows, width});
    if (g.t.defined()) {
      dgain.allocate(at::kFloat, shape, dev);
      if (!ws.defined()) ws = make({(int64_t)std::max<size_t>(bytes, 256)}, at::kByte, dev);
    }
    const int rc = call([&] {
      return solfp4_rmsnorm_backward(type_of(x), ptr(dy), dy.stride(0), ptr(x), x.stride(0), ptr(g.t), g.stride,
                                     g.groups, ptr(dsum.t), dsum.stride(0), (float)eps, ptr(dx.t), dx.stride(0),
                                     f32(dgain.t), ptr(ws), ws.defined() ? (size_t)ws.numel() : 0, rows, width, stream);
    });
    if (rc) return failed(rc);
    if (g.t.defined()) return Py_BuildValue("(NN)", dx.object(), dgain.object());
    return Py_BuildValue("(NO)", dx.object(), Py_None);
  });
}

// (x, residual, gain, shift, eps, out, sum_out) -> (out, sum)
PyObject* add_layernorm_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 7, [&]() -> PyObject* {
    const Tensor& x = matrix_operand(a[0]);
    const int64_t rows = x.size(0), width = x.size(1);
    Strided r(a[1], x, {rows, width}), out(a[5], x, {rows, width}), sum(a[6], x, {rows, width});
    Gain g(a[2], x, rows, width);
    Shift t(a[3], g, x, rows, width);
    const double eps = number(a[4]);
    need(eps >= 0);
    need(r.given || !sum.given);
    void* stream = stream_of(x.device());
    out.allocate(x, {rows, width});
    if (r.given) sum.allocate(x, {rows, width});
    const int rc = call([&] {
      return solfp4_add_layernorm(type_of(x), ptr(x), x.stride(0), ptr(r.t), r.stride(0), ptr(g.t), g.stride, ptr(t.t),
                                  t.stride, t.groups, (float)eps, ptr(sum.t), sum.stride(0), ptr(out.t), out.stride(0),
                                  rows, width, stream);
    });
    if (rc) return failed(rc);
    return Py_BuildValue("(NN)", out.object(), sum.object());
  });
}

// (x, residual, gain, shift, eps, codes, scales, sum_out) -> (codes, scales, sum)
template <typename F>
PyObject* quantized_layernorm(PyObject* const* a, Py_ssize_t n, int pack, F f) {
  return entry(n, 8, [&]() -> PyObject* {
    const Tensor& x = matrix_operand(a[0]);
    const int64_t rows = x.size(0), width = x.size(1);
    need(width % 32 == 0);
    const at::Device dev = x.device();
    Strided r(a[1], x, {rows, width}), sum(a[7], x, {rows, width});
    Gain g(a[2], x, rows, width);
    Shift t(a[3], g, x, rows, width);
    const double eps = number(a[4]);
    need(eps >= 0);
    Operand codes(a[5], at::kByte, {rows, width / pack}, dev), scales(a[6], at::kByte, {rows, width / 32}, dev);
    need(r.given || !sum.given);
    void* stream = stream_of(dev);
    codes.allocate(at::kByte, {rows, width / pack}, dev);
    scales.allocate(at::kByte, {rows, width / 32}, dev);
    if (r.given) sum.allocate(x, {rows, width});
    const int rc = call([&] {
      return f(type_of(x), ptr(x), x.stride(0), ptr(r.t), r.stride(0), ptr(g.t), g.stride, ptr(t.t), t.stride, t.groups,
               (float)eps, ptr(sum.t), sum.stride(0), u8(codes.t), u8(scales.t), rows, width, stream);
    });
    if (rc) return failed(rc);
    return Py_BuildValue("(NNN)", codes.object(), scales.object(), sum.object());
  });
}

PyObject* mxfp8_add_layernorm_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return quantized_layernorm(a, n, 1, mxfp8_add_layernorm);
}
PyObject* mxfp4_add_layernorm_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return quantized_layernorm(a, n, 2, mxfp4_add_layernorm);
}

// An output that the call has or has not; None where it has not.
PyObject* object_or_none(const Operand& o) {
  if (o.t.defined()) return o.object();
  Py_RETURN_NONE;
}

// (dy, x, gain, shift, dsum, eps, dx, dgain, dshift, workspace) -> (dx, dgain, dshift)
PyObject* layernorm_backward_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 10, [&]() -> PyObject* {
    const Tensor& x = matrix_operand(a[1]);
    const int64_t rows = x.size(0), width = x.size(1);
    const Tensor& dy = tensor(a[0]);
    need_strided(dy, x, {rows, width});
    Gain g(a[2], x, rows, width);
    Shift t(a[3], g, x, rows, width);
    Strided dsum(a[4], x, {rows, width}), dx(a[6], x, {rows, width});
    const double eps = number(a[5]);
    need(eps >= 0);
    const at::Device dev = x.device();
    need((g.t.defined() || a[7] == Py_None) && (t.t.defined() || a[8] == Py_None));
    const at::IntArrayRef gain_shape = g.t.defined() ? g.t.sizes() : at::IntArrayRef();
    const at::IntArrayRef shift_shape = t.t.defined() ? t.t.sizes() : at::IntArrayRef();
    Operand dgain(a[7], at::kFloat, gain_shape, dev), dshift(a[8], at::kFloat, shift_shape, dev);
    const bool sums = g.t.defined() || t.t.defined();
    const size_t bytes = sums ? solfp4_layernorm_backward_workspace_bytes(rows, width, t.groups) : 0;
    Tensor ws = sums ? workspace_arg(a[9], bytes, dev) : Tensor();
    void* stream = stream_of(dev);
    dx.allocate(x, {rows, width});
    if (g.t.defined()) dgain.allocate(at::kFloat, gain_shape, dev);
    if (t.t.defined()) dshift.allocate(at::kFloat, shift_shape, dev);
    if (sums && !ws.defined()) ws = make({(int64_t)std::max<size_t>(bytes, 256)}, at::kByte, dev);
    const int rc = call([&] {
      return solfp4_layernorm_backward(type_of(x), ptr(dy), dy.stride(0), ptr(x), x.stride(0), ptr(g.t), g.stride,
                                       t.groups, ptr(dsum.t), dsum.stride(0), (float)eps, ptr(dx.t), dx.stride(0),
                                       f32(dgain.t), f32(dshift.t), ptr(ws), ws.defined() ? (size_t)ws.numel() : 0, rows,
                                       width, stream);
    });
    if (rc) return failed(rc);
    return Py_BuildValue("(NNN)", dx.object(), object_or_none(dgain), object_or_none(dshift));
  });
}

// (q, k, table, positions, layout, inverse, q_out, k_out) -> (q, k)
PyObject* rotary_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 8, [&]() -> PyObject* {
    const Tensor& q = tensor(a[0]);
    need(q.layout() == at::kStrided && q.dim() == 3);
    type_of(q);
    need_strided(q, q, q.sizes());
    const int64_t tokens = q.size(0), heads = q.size(1), dim = q.size(2);
    const at::Device dev = q.device();
    Tensor k;
    int64_t k_heads = 0;
    if (a[1] != Py_None) {
      k = tensor(a[1]);
      need(k.layout() == at::kStrided && k.dim() == 3);
      k_heads = k.size(1);
      need_strided(k, q, {tokens, k_heads, dim});
    }
    const Tensor& table = tensor(a[2]);
    need_matrix(table);
    const int64_t table_rows = table.size(0), rotated = table.size(1);
    need_tensor(table, at::kFloat, {table_rows, rotated}, &dev);
    need(rotated % 2 == 0 && rotated <= dim && (table_rows > 0 || tokens == 0));
    Tensor at_;
    int position_bytes = 0;
    if (a[3] != Py_None) {
      at_ = tensor(a[3]);
      need(at_.scalar_type() == at::kInt || at_.scalar_type() == at::kLong);
      need_tensor(at_, at_.scalar_type(), {tokens}, &dev);
      position_bytes = at_.scalar_type() == at::kInt ? 4 : 8;
    }
    need(PyLong_CheckExact(a[4]) && (PyBool_Check(a[5]) || PyLong_CheckExact(a[5])));
    const long layout = PyLong_AsLong(a[4]);
    need(layout == SOLFP4_ROTARY_HALF || layout == SOLFP4_ROTARY_INTERLEAVED);
    const int inverse = PyObject_IsTrue(a[5]);
    need(k.defined() || a[7] == Py_None);
    Strided q_out(a[6], q, {tokens, heads, dim}), k_out(a[7], q, {tokens, k_heads, dim});
    void* stream = stream_of(dev);
    q_out.allocate(q, {tokens, heads, dim});
    if (k.defined()) k_out.allocate(q, {tokens, k_heads, dim});
    const int rc = call([&] {
      return solfp4_rotary(type_of(q), (int)layout, inverse, ptr(q), q.stride(0), q.stride(1), ptr(q_out.t),
                           q_out.stride(0), q_out.stride(1), heads, ptr(k), k.defined() ? k.stride(0) : 0,
                           k.defined() ? k.stride(1) : 0, ptr(k_out.t), k_out.stride(0), k_out.stride(1), k_heads,
                           f32(table), table_rows, ptr(at_), position_bytes, tokens, dim, rotated, stream);
    });
    if (rc) return failed(rc);
    return Py_BuildValue("(NN)", q_out.object(), k_out.object());
  });
}

// (x, w_codes, w_scales, w_gs, bias, out) -> out
PyObject* nvfp4_weight_linear_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 6, [&]() -> PyObject* {
    const Tensor &x = tensor(a[0]), &wc = tensor(a[1]), &ws = tensor(a[2]), &wg = tensor(a[3]);
    need_matrix(x);
    need_matrix(wc);
    const int64_t M = x.size(0), K = x.size(1), N = wc.size(0);
    need(K % 16 == 0);
    need_tensor(x, at::kBFloat16, {M, K}, nullptr);
    const at::Device dev = x.device();
    need_tensor(wc, at::kByte, {N, K / 2}, &dev);
    need_tensor(ws, at::kByte, {N, K / 16}, &dev);
    need_tensor(wg, at::kFloat, {1}, &dev);
    Operand bias(a[4], at::kBFloat16, {N}, dev), out(a[5], at::kBFloat16, {M, N}, dev);
    void* stream = stream_of(dev);
    out.allocate(at::kBFloat16, {M, N}, dev);
    const int rc = call([&] {
      return nvfp4_weight_linear(u16(x), u8(wc), u8(ws), f32(wg), u16(bias.t), u16(out.t), M, N, K, stream);
    });
    return rc ? failed(rc) : out.object();
  });
}

// (x, w_codes, w_scales, bias, out) -> out
PyObject* mxfp4_weight_linear_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 5, [&]() -> PyObject* {
    const Tensor &x = tensor(a[0]), &wc = tensor(a[1]), &ws = tensor(a[2]);
    need_matrix(x);
    need_matrix(wc);
    const int64_t M = x.size(0), K = x.size(1), N = wc.size(0);
    need(K % 32 == 0);
    need_tensor(x, at::kBFloat16, {M, K}, nullptr);
    const at::Device dev = x.device();
    need_tensor(wc, at::kByte, {N, K / 2}, &dev);
    need_tensor(ws, at::kByte, {N, K / 32}, &dev);
    Operand bias(a[3], at::kBFloat16, {N}, dev), out(a[4], at::kBFloat16, {M, N}, dev);
    void* stream = stream_of(dev);
    out.allocate(at::kBFloat16, {M, N}, dev);
    const int rc = call([&] {
      return mxfp4_weight_linear(u16(x), u8(wc), u8(ws), u16(bias.t), u16(out.t), M, N, K, stream);
    });
    return rc ? failed(rc) : out.object();
  });
}

// (x_codes, x_scales, w_codes, w_scales, bias, out) -> out
PyObject* mxfp8_linear_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 6, [&]() -> PyObject* {
    const Tensor &xc = tensor(a[0]), &xs = tensor(a[1]), &wc = tensor(a[2]), &ws = tensor(a[3]);
    need_matrix(xc);
    need_matrix(wc);
    const int64_t M = xc.size(0), K = xc.size(1), N = wc.size(0);
    need(K % 32 == 0);
    need_tensor(xc, at::kByte, {M, K}, nullptr);
    const at::Device dev = xc.device();
    need_tensor(xs, at::kByte, {M, K / 32}, &dev);
    need_tensor(wc, at::kByte, {N, K / 2}, &dev);
    need_tensor(ws, at::kByte, {N, K / 32}, &dev);
    Operand bias(a[4], at::kBFloat16, {N}, dev), out(a[5], at::kBFloat16, {M, N}, dev);
    void* stream = stream_of(dev);
    out.allocate(at::kBFloat16, {M, N}, dev);
    const int rc = call([&] {
      return mxfp8_linear(u8(xc), u8(xs), u8(wc), u8(ws), u16(bias.t), u16(out.t), M, N, K, stream);
    });
    return rc ? failed(rc) : out.object();
  });
}

// ---- low-rank adapters ----------------------------------------------------

// The operands that both passes have: t [tokens][N], x, a, b, scales, and the
// plan (buffer, tokens, adapters).
struct Adapters {
  const Tensor &t, &x, &a, &b;
  Tensor scales, plan;
  int64_t tokens, N, K, rank, adapters;
  at::Device dev;
  static const Tensor& of(PyObject* o, int64_t dims) {
    const Tensor& v = tensor(o);
    need(v.layout() == at::kStrided && v.dim() == dims);
    return v;
  }
  Adapters(PyObject* t_, PyObject* x_, PyObject* a_, PyObject* b_, PyObject* scales_, PyObject* plan_,
           PyObject* plan_tokens, PyObject* plan_adapters)
      : t(of(t_, 2)), x(of(x_, 2)), a(of(a_, 3)), b(of(b_, 3)), tokens(t.size(0)), N(t.size(1)), K(x.size(1)),
        rank(a.size(1)), adapters(a.size(0)), dev(x.device()) {
    need(x.scalar_type() == at::kBFloat16);
    need_strided(x, x, {tokens, K});
    need_strided(t, x, {tokens, N});
    need_tensor(a, at::kBFloat16, {adapters, rank, K}, &dev);
    need_tensor(b, at::kBFloat16, {adapters, N, rank}, &dev);
    if (scales_ != Py_None) {
      scales = tensor(scales_);
      need_tensor(scales, at::kFloat, {adapters}, &dev);
    }
    need(rank >= 1 && rank <= 128);
    if (plan_ == Py_None) {
      need(adapters == 1);
    } else {
      plan = tensor(plan_);
      need(PyLong_CheckExact(plan_tokens) && PyLong_CheckExact(plan_adapters));
      need(PyLong_AsLongLong(plan_tokens) == tokens && PyLong_AsLongLong(plan_adapters) == adapters);
      need_tensor(plan, at::kInt, {(int64_t)solfp4_adapter_plan_bytes(tokens, adapters) / 4}, &dev);
    }
  }
};

// (y, x, a, b, scales, plan, plan_tokens, plan_adapters, hidden, out, workspace) -> (out, hidden)
PyObject* add_adapters_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 11, [&]() -> PyObject* {
    const Adapters o(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7]);
    const bool fresh = a[8] == Py_True;
    Operand hidden(fresh ? Py_None : a[8], at::kFloat, {o.tokens, o.rank}, o.dev);
    Strided out(a[9], o.x, {o.tokens, o.N});
    const size_t bytes = solfp4_add_adapters_workspace_bytes(o.tokens, o.adapters, o.plan.defined(), o.N, o.K, o.rank);
    Tensor ws = workspace_arg(a[10], bytes, o.dev);
    void* stream = stream_of(o.dev);
    out.allocate(o.x, {o.tokens, o.N});
    if (fresh) hidden.allocate(at::kFloat, {o.tokens, o.rank}, o.dev);
    if (!ws.defined() && bytes) ws = make({(int64_t)bytes}, at::kByte, o.dev);
    const int rc = call([&] {
      return solfp4_add_adapters(u16(o.t), o.t.stride(0), u16(o.x), o.x.stride(0), u16(o.a), u16(o.b), f32(o.scales),
                                 o.adapters, ptr(o.plan), u16(out.t), out.stride(0), f32(hidden.t), ptr(ws),
                                 ws.defined() ? (size_t)ws.numel() : 0, o.tokens, o.N, o.K, o.rank, stream);
    });
    if (rc) return failed(rc);
    return Py_BuildValue("(NN)", out.object(), object_or_none(hidden));
  });
}

// (dy, x, hidden, a, b, scales, plan, plan_tokens, plan_adapters, past, dx, da, db, workspace) -> (dx, da, db)
PyObject* adapters_backward_(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 14, [&]() -> PyObject* {
    const Adapters o(a[0], a[1], a[3], a[4], a[5], a[6], a[7], a[8]);
    const Tensor& hidden = tensor(a[2]);
    need_tensor(hidden, at::kFloat, {o.tokens, o.rank}, &o.dev);
    Strided past(a[9], o.x, {o.tokens, o.K}), dx(a[10], o.x, {o.tokens, o.K});
    Operand da(a[11], at::kFloat, o.a.sizes(), o.dev), db(a[12], at::kFloat, o.b.sizes(), o.dev);
    const size_t bytes =
        solfp4_adapters_backward_workspace_bytes(o.tokens, o.adapters, o.plan.defined(), o.N, o.K, o.rank);
    Tensor ws = workspace_arg(a[13], bytes, o.dev);
    void* stream = stream_of(o.dev);
    dx.allocate(o.x, {o.tokens, o.K});
    da.allocate(at::kFloat, o.a.sizes(), o.dev);
    db.allocate(at::kFloat, o.b.sizes(), o.dev);
    if (!ws.defined()) ws = make({(int64_t)std::max<size_t>(bytes, 256)}, at::kByte, o.dev);
    const int rc = call([&] {
      return solfp4_adapters_backward(u16(o.t), o.t.stride(0), u16(o.x), o.x.stride(0), f32(hidden), u16(o.a), u16(o.b),
                                      f32(o.scales), o.adapters, ptr(o.plan), u16(past.t), past.stride(0), u16(dx.t),
                                      dx.stride(0), f32(da.t), f32(db.t), ptr(ws), (size_t)ws.numel(), o.tokens, o.N,
                                      o.K, o.rank, stream);
    });
    if (rc) return failed(rc);
    return Py_BuildValue("(NNN)", dx.object(), da.object(), db.object());
  });
}

PyMethodDef methods[] = {
    {"nvfp4_quantize", (PyCFunction)(void*)nvfp4_quantize_, METH_FASTCALL, nullptr},
    {"mxfp4_quantize", (PyCFunction)(void*)mxfp4_quantize_, METH_FASTCALL, nullptr},
    {"nvfp4_gemm", (PyCFunction)(void*)nvfp4_gemm_, METH_FASTCALL, nullptr},
    {"mxfp4_gemm", (PyCFunction)(void*)mxfp4_gemm_, METH_FASTCALL, nullptr},
    {"nvfp4_linear", (PyCFunction)(void*)nvfp4_linear_, METH_FASTCALL, nullptr},
    {"mxfp4_linear", (PyCFunction)(void*)mxfp4_linear_, METH_FASTCALL, nullptr},
    {"add_rmsnorm", (PyCFunction)(void*)add_rmsnorm_, METH_FASTCALL, nullptr},
    {"mxfp8_add_rmsnorm", (PyCFunction)(void*)mxfp8_add_rmsnorm_, METH_FASTCALL, nullptr},
    {"mxfp4_add_rmsnorm", (PyCFunction)(void*)mxfp4_add_rmsnorm_, METH_FASTCALL, nullptr},
    {"rmsnorm_backward", (PyCFunction)(void*)rmsnorm_backward_, METH_FASTCALL, nullptr},
    {"add_layernorm", (PyCFunction)(void*)add_layernorm_, METH_FASTCALL, nullptr},
    {"mxfp8_add_layernorm", (PyCFunction)(void*)mxfp8_add_layernorm_, METH_FASTCALL, nullptr},
    {"mxfp4_add_layernorm", (PyCFunction)(void*)mxfp4_add_layernorm_, METH_FASTCALL, nullptr},
    {"layernorm_backward", (PyCFunction)(void*)layernorm_backward_, METH_FASTCALL, nullptr},
    {"rotary", (PyCFunction)(void*)rotary_, METH_FASTCALL, nullptr},
    {"nvfp4_weight_linear", (PyCFunction)(void*)nvfp4_weight_linear_, METH_FASTCALL, nullptr},
    {"mxfp4_weight_linear", (PyCFunction)(void*)mxfp4_weight_linear_, METH_FASTCALL, nullptr},
    {"mxfp8_linear", (PyCFunction)(void*)mxfp8_linear_, METH_FASTCALL, nullptr},
    {"adapters_backward", (PyCFunction)(void*)adapters_backward_, METH_FASTCALL, nullptr},
    {"add_adapters", (PyCFunction)(void*)add_adapters_, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", "Native checks, allocation and calls of the binding.",
                      -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host() {
  PyObject* c = PyImport_ImportModule("torch._C");
  if (!c) return nullptr;
  current_raw_stream = PyObject_GetAttrString(c, "_cuda_getCurrentRawStream");
  Py_DECREF(c);
  if (!current_raw_stream) return nullptr;
  return PyModule_Create(&module);
}

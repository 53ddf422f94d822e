// Argument marshalling of the calls around the layer: torch tensors in, one C call of include/pw.h out.  These calls take
// a few microseconds on the GPU, and marshalled in Python (ctypes, five or six tensors to look at) they took 8 to 14
// microseconds of the host's time.  Here the marshalling is 0.3 to 0.5 of them, and a call from Python with its launch 2.4
// (three tensors) to 4.3 (five).
//
// Every function gets the context, its device index, a stream (None: the device's current one) and the arguments of the
// Python method, and returns 0 or  status | (number of the argument that is wrong) << 8.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <string.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/pw.h"

namespace {

constexpr int64_t kGroup = 128;

// A tensor argument; `bad` collects the first thing that is wrong with any of them.
struct Call {
  pw_ctx* ctx;
  int index;
  pw_stream stream;
  int bad = 0;

  Call(PyObject* const* a) {
    ctx = static_cast<pw_ctx*>(PyLong_AsVoidPtr(a[0]));
    index = (int)PyLong_AsLong(a[1]);
    if (a[2] == Py_None) stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)index).stream();
    else stream = static_cast<pw_stream>(PyLong_AsVoidPtr(a[2]));
  }
  void fail(int status, int arg) {
    if (!bad) bad = status | arg << 8;
  }
  // Arguments that are no tensors.  What is not of the kind leaves Python's error set and the call not made; what does
  // not fit the C type is an invalid argument, never another one.
  int integer(PyObject* o, int arg) {
    int overflow = 0;
    const long v = PyLong_AsLongAndOverflow(o, &overflow);
    if (overflow || v < INT32_MIN || v > INT32_MAX || (v == -1 && PyErr_Occurred())) return fail(PW_ERR_INVALID_ARG, arg), -1;
    return (int)v;
  }
  float number(PyObject* o, int arg) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) fail(PW_ERR_INVALID_ARG, arg);
    return (float)v;
  }
  int truth(PyObject* o, int arg) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) fail(PW_ERR_INVALID_ARG, arg);
    return v;
  }
};

struct Matrix {
  void* data = nullptr;
  int64_t rows = 0, cols = 0, stride = 0;
  int type = -1;                                   // pw_type, or kCodes / kWords for the other kinds
};
constexpr int kCodes = 16, kWords = 17;            // 8-bit codes, int32

int type_of(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return PW_F32;
    case at::kHalf: return PW_F16;
    case at::kBFloat16: return PW_BF16;
    case at::kFloat8_e4m3fn:
    case at::kByte: return kCodes;
    case at::kInt: return kWords;
    default: return -1;
  }
}

// A 2-D tensor on the call's device whose rows are contiguous.  kind: a type, or -1 for any of f32 / f16 / bf16.
Matrix matrix(Call& c, PyObject* o, int arg, int kind, int64_t rows = -1, int64_t cols = -1, bool whole = false) {
  Matrix m;
  if (!THPVariable_Check(o)) return c.fail(PW_ERR_INVALID_ARG, arg), m;
  const at::Tensor& t = THPVariable_Unpack(o);
  m.type = type_of(t);
  const bool kind_ok = kind < 0 ? m.type >= PW_F32 && m.type <= PW_BF16 : m.type == kind;
  if (!kind_ok || !t.is_cuda() || t.is_neg() || t.get_device() != c.index) return c.fail(PW_ERR_INVALID_ARG, arg), m;
  if (t.dim() != 2) return c.fail(PW_ERR_SHAPE, arg), m;
  m.rows = t.size(0);
  m.cols = t.size(1);
  m.stride = t.stride(0);
  if ((m.cols > 1 && t.stride(1) != 1) || (rows >= 0 && m.rows != rows) || (cols >= 0 && m.cols != cols) || (whole && !t.is_contiguous()) ||
      m.rows > INT32_MAX || m.cols > INT32_MAX)
    return c.fail(PW_ERR_SHAPE, arg), m;
  m.data = m.rows && m.cols ? t.data_ptr() : nullptr;
  return m;
}

// A contiguous 1-D tensor of `n`.
Matrix vector(Call& c, PyObject* o, int arg, int kind, int64_t n) {
  Matrix m;
  if (!THPVariable_Check(o)) return c.fail(PW_ERR_INVALID_ARG, arg), m;
  const at::Tensor& t = THPVariable_Unpack(o);
  m.type = type_of(t);
  const bool kind_ok = kind < 0 ? m.type >= PW_F32 && m.type <= PW_BF16 : m.type == kind;
  if (!kind_ok || !t.is_cuda() || t.is_neg() || t.get_device() != c.index) return c.fail(PW_ERR_INVALID_ARG, arg), m;
  if (t.dim() != 1 || t.size(0) != n || !t.is_contiguous()) return c.fail(PW_ERR_SHAPE, arg), m;
  m.data = t.data_ptr();
  return m;
}

Matrix scales(Call& c, PyObject* o, int arg, int64_t rows, int64_t cols, int64_t block_rows) {
  return matrix(c, o, arg, PW_F32, (rows + block_rows - 1) / block_rows, (cols + kGroup - 1) / kGroup, true);
}

// Around a call of the library, once all arguments are read: the call's device current and the interpreter released.  A
// launch waits when the stream's queue is full, and for a host function in it that wants the interpreter it would wait for
// good.  (The caller's frame holds the tensors.)
struct Released {
  PyThreadState* state = PyEval_SaveThread();
  ~Released() { PyEval_RestoreThread(state); }
};
struct Outside {
  Released released;
  c10::cuda::CUDAGuard device;
  explicit Outside(const Call& c) : device((c10::DeviceIndex)c.index) {}
};

// Runs the marshalling of one call; a C++ exception of torch's (a tensor without storage, say) is an invalid argument.
template <class F>
PyObject* guarded(PyObject* const* args, Py_ssize_t n, Py_ssize_t want, F f) {
  if (n != want) {
    PyErr_Format(PyExc_TypeError, "%zd arguments, %zd wanted", n, want);
    return nullptr;
  }
  try {
    Call c(args);
    if (PyErr_Occurred()) return nullptr;
    const int status = f(c, args + 3);
    if (PyErr_Occurred()) return nullptr;
    return PyLong_FromLong(status);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// x, block_rows, q, scales
PyObject* quantize_scaled(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(args, n, 7, [](Call& c, PyObject* const* a) -> int {
    const Matrix x = matrix(c, a[0], 1, -1);
    const int block = c.integer(a[1], 2);
    if (block != 1 && block != kGroup) c.fail(PW_ERR_INVALID_ARG, 2);
    if (c.bad) return c.bad;
    const Matrix q = matrix(c, a[2], 3, kCodes, x.rows, x.cols), s = scales(c, a[3], 4, x.rows, x.cols, block);
    if (c.bad) return c.bad;
    Outside outside(c);
    return pw_quantize_scaled(c.ctx, x.data, x.type, (int)x.rows, (int)x.cols, x.stride, block, q.data, q.stride,
                              static_cast<float*>(s.data), c.stream);
  });
}

// x, weight, eps, residual, residual_out, y, q, q_scales
PyObject* add_rmsnorm(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(args, n, 11, [](Call& c, PyObject* const* a) -> int {
    const Matrix x = matrix(c, a[0], 1, -1);
    const Matrix w = vector(c, a[1], 2, -1, x.cols);
    const float eps = c.number(a[2], 3);
    Matrix r, ro, y, q, s;
    if (a[3] != Py_None) r = matrix(c, a[3], 4, -1, x.rows, x.cols);
    if (a[4] != Py_None) {
      if (a[3] == Py_None) c.fail(PW_ERR_INVALID_ARG, 5);
      ro = matrix(c, a[4], 5, r.type, x.rows, x.cols);
    }
    if (a[5] != Py_None) y = matrix(c, a[5], 6, -1, x.rows, x.cols);
    if ((a[6] == Py_None) != (a[7] == Py_None)) c.fail(PW_ERR_INVALID_ARG, 8);
    if (a[6] != Py_None) {
      q = matrix(c, a[6], 7, kCodes, x.rows, x.cols);
      s = scales(c, a[7], 8, x.rows, x.cols, 1);
    }
    if (c.bad) return c.bad;
    Outside outside(c);
    return pw_add_rmsnorm(c.ctx, (int)x.rows, (int)x.cols, x.data, x.type, x.stride, r.data, r.type, r.stride, w.data, w.type, eps, ro.data, ro.stride,
                          y.data, y.type, y.stride, q.data, q.stride, static_cast<float*>(s.data), c.stream);
  });
}

// a, a_scales, w, w_scales, out
PyObject* scaled_linear(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(args, n, 8, [](Call& c, PyObject* const* a) -> int {
    const Matrix x = matrix(c, a[0], 1, kCodes);
    const Matrix w = matrix(c, a[2], 3, kCodes, -1, x.cols);
    const Matrix sx = scales(c, a[1], 2, x.rows, x.cols, 1), sw = scales(c, a[3], 4, w.rows, x.cols, kGroup);
    const Matrix out = matrix(c, a[4], 5, -1, x.rows, w.rows);
    if (c.bad) return c.bad;
    Outside outside(c);
    return pw_scaled_linear(c.ctx, (int)x.rows, (int)w.rows, (int)x.cols, x.data, x.stride, static_cast<float*>(sx.data), w.data, w.stride,
                            static_cast<float*>(sw.data), out.data, out.type, out.stride, c.stream);
  });
}

// router_logits, top_k, score, bias, n_groups, top_groups, group_best, renormalize, scale, ids, gates
PyObject* route_tokens(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(args, n, 14, [](Call& c, PyObject* const* a) -> int {
    const Matrix l = matrix(c, a[0], 1, -1);
    pw_routing r;
    r.n_experts = (int32_t)l.cols;
    r.top_k = c.integer(a[1], 2);
    r.score = c.integer(a[2], 3);
    r.n_groups = c.integer(a[4], 5);
    r.top_groups = c.integer(a[5], 6);
    r.group_best = c.integer(a[6], 7);
    r.renormalize = c.truth(a[7], 8);
    r.scale = c.number(a[8], 9);
    Matrix b;
    if (a[3] != Py_None) b = vector(c, a[3], 4, PW_F32, l.cols);
    const Matrix ids = matrix(c, a[9], 10, kWords, l.rows, r.top_k, true), gates = matrix(c, a[10], 11, PW_F32, l.rows, r.top_k, true);
    if (c.bad) return c.bad;
    Outside outside(c);
    return pw_route_tokens(c.ctx, &r, l.data, l.type, l.stride, static_cast<float*>(b.data), (int)l.rows, static_cast<int32_t*>(ids.data),
                           static_cast<float*>(gates.data), c.stream);
  });
}

// layer, hidden, topk_ids, gates, out, mode, H
PyObject* moe_forward_routed(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(args, n, 10, [](Call& c, PyObject* const* a) -> int {
    const int layer = c.integer(a[0], 1);
    const Matrix h = matrix(c, a[1], 2, PW_F16, -1, PyLong_AsLongLong(a[6]), true);
    const Matrix ids = matrix(c, a[2], 3, kWords, h.rows, -1, true), gates = matrix(c, a[3], 4, PW_F32, h.rows, ids.cols, true);
    const Matrix out = matrix(c, a[4], 5, PW_F32, h.rows, h.cols, true);
    const pw_mode mode = (pw_mode)c.integer(a[5], 6);
    if (c.bad) return c.bad;
    Outside outside(c);
    return pw_moe_forward_routed(c.ctx, layer, h.data, static_cast<int32_t*>(ids.data), static_cast<float*>(gates.data), (int)h.rows, (int)ids.cols, nullptr,
                                 static_cast<float*>(out.data), mode, c.stream);
  });
}

// layer, hidden, router_logits, top_k, out, H, E
PyObject* moe_forward_few(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(args, n, 10, [](Call& c, PyObject* const* a) -> int {
    const int layer = c.integer(a[0], 1);
    const Matrix h = matrix(c, a[1], 2, PW_F16, -1, PyLong_AsLongLong(a[5]), true);
    const Matrix l = matrix(c, a[2], 3, PW_F32, h.rows, PyLong_AsLongLong(a[6]), true);
    const int k = c.integer(a[3], 4);
    const Matrix out = matrix(c, a[4], 5, -1, h.rows, h.cols, true);
    if (c.bad) return c.bad;
    Outside outside(c);
    return pw_moe_forward_few(c.ctx, layer, h.data, static_cast<float*>(l.data), (int)h.rows, k, nullptr, out.data, out.type, c.stream);
  });
}

// layer, hidden, topk_ids, gates, out, H
PyObject* moe_forward_few_routed(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(args, n, 9, [](Call& c, PyObject* const* a) -> int {
    const int layer = c.integer(a[0], 1);
    const Matrix h = matrix(c, a[1], 2, PW_F16, -1, PyLong_AsLongLong(a[5]), true);
    const Matrix ids = matrix(c, a[2], 3, kWords, h.rows, -1, true), gates = matrix(c, a[3], 4, PW_F32, h.rows, ids.cols, true);
    const Matrix out = matrix(c, a[4], 5, -1, h.rows, h.cols, true);
    if (c.bad) return c.bad;
    Outside outside(c);
    return pw_moe_forward_few_routed(c.ctx, layer, h.data, static_cast<int32_t*>(ids.data), static_cast<float*>(gates.data), (int)h.rows, (int)ids.cols,
                                     nullptr, out.data, out.type, c.stream);
  });
}

// A Python reference that is given back.
struct Ref {
  PyObject* o;
  explicit Ref(PyObject* p) : o(p) {}
  ~Ref() { Py_XDECREF(o); }
  Ref(const Ref&) = delete;
};

// The header of a Page or PlanePage (its ctypes structure) whose buffer is on the call's device.
bool page_header(Call& c, PyObject* o, int arg, pw_page* out) {
  Ref head(PyObject_GetAttrString(o, "c")), codes(head.o ? PyObject_GetAttrString(o, "codes") : nullptr);
  if (!codes.o) return false;                      // Python's error is set
  Py_buffer b;
  if (PyObject_GetBuffer(head.o, &b, PyBUF_SIMPLE) < 0) return false;
  const bool whole = b.len == (Py_ssize_t)sizeof(pw_page);
  if (whole) memcpy(out, b.buf, sizeof(pw_page));
  PyBuffer_Release(&b);
  if (!whole) return c.fail(PW_ERR_INVALID_ARG, arg), false;
  if (codes.o == Py_None) return true;             // a page without a buffer: the library says what is wrong with it
  if (!THPVariable_Check(codes.o) || !THPVariable_Unpack(codes.o).is_cuda() || THPVariable_Unpack(codes.o).get_device() != c.index)
    return c.fail(PW_ERR_INVALID_ARG, arg), false;
  return true;
}

// x, pages, out_features, bias, out, and a function that makes a workspace of so many bytes
PyObject* page_linear(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(args, n, 9, [](Call& c, PyObject* const* a) -> int {
    const Matrix x = matrix(c, a[0], 1, PW_F16);
    pw_page page[PW_LINEAR_PAGES];
    int32_t features[PW_LINEAR_PAGES];
    Ref pages(PySequence_Fast(a[1], "pages: a sequence of pages"));
    if (!pages.o) return 0;
    const Py_ssize_t count = PySequence_Fast_GET_SIZE(pages.o);
    if (count < 1 || count > PW_LINEAR_PAGES) c.fail(PW_ERR_INVALID_ARG, 2);
    if (c.bad) return c.bad;
    int64_t total = 0;
    for (Py_ssize_t i = 0; i < count; ++i) {
      if (!page_header(c, PySequence_Fast_GET_ITEM(pages.o, i), 2, &page[i])) return c.bad;
      features[i] = (int32_t)page[i].rows;
      if (page[i].rows > INT32_MAX) return c.fail(PW_ERR_SHAPE, 2), c.bad;
    }
    if (a[2] != Py_None) {
      Ref f(PySequence_Fast(a[2], "out_features: a sequence of numbers"));
      if (!f.o) return 0;
      if (PySequence_Fast_GET_SIZE(f.o) != count) c.fail(PW_ERR_SHAPE, 3);
      for (Py_ssize_t i = 0; i < count && !c.bad; ++i) {
        features[i] = c.integer(PySequence_Fast_GET_ITEM(f.o, i), 3);
        if (features[i] < 1) c.fail(PW_ERR_INVALID_ARG, 3);
      }
    }
    for (Py_ssize_t i = 0; i < count; ++i) total += features[i];
    Matrix bias;
    if (a[3] != Py_None) bias = vector(c, a[3], 4, -1, total);
    const Matrix out = matrix(c, a[4], 5, -1, x.rows, total);
    if (c.bad) return c.bad;
    const size_t bytes = pw_page_linear_workspace(c.ctx, (int)x.rows, (int)x.cols, page, features, (int)count, out.type);
    Ref made(nullptr);
    void* workspace = nullptr;
    if (bytes) {
      made.o = PyObject_CallFunction(a[5], "n", (Py_ssize_t)bytes);
      if (!made.o) return 0;
      workspace = THPVariable_Unpack(made.o).data_ptr();
    }
    Outside outside(c);
    return pw_page_linear(c.ctx, (int)x.rows, (int)x.cols, x.data, x.stride, page, features, (int)count, bias.data, bias.type, out.data, out.type, out.stride,
                          workspace, bytes, c.stream);
  });
}

#define PW_METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {PW_METHOD(quantize_scaled), PW_METHOD(add_rmsnorm), PW_METHOD(scaled_linear), PW_METHOD(route_tokens),
                         PW_METHOD(moe_forward_routed), PW_METHOD(page_linear), PW_METHOD(moe_forward_few), PW_METHOD(moe_forward_few_routed), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pwtorch", "Argument marshalling for torch tensors.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pwtorch(void) {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "built_for", PW_BUILT_FOR) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}

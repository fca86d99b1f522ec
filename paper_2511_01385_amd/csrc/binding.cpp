// binding.cpp -- the operators around the adapter, called with torch tensors (Python module _binding).
//
// Small calls are bound by the host: looking at a tensor from Python (type, shape, device, layout, pointer) takes
// half a microsecond, a launch about three.  Each function here looks at its tensors, fills the C struct and
// calls the C entry, which makes its own checks.  It returns the entry's status, or None when a tensor is not what
// the call needs (its type, shape, device or layout, or no tensor at all): api.py then says what is wrong.
//
// Arguments are positional, None for a tensor that is left out; the last two are the current device and its
// stream as integers.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>

#include <algorithm>
#include <initializer_list>

#include "rdfft.h"

namespace {

// raised when the arguments are not plainly right
struct NotPlain {};

struct Call {
  PyObject* const* args;
  c10::DeviceIndex device;
  rdfft_stream_t stream;
  at::ScalarType type = at::kFloat;
  rdfft_dtype_t code = RDFFT_F32;

  Call(PyObject* const* a, Py_ssize_t given, Py_ssize_t want) : args(a) {
    if (given != want) throw NotPlain{};
    device = (c10::DeviceIndex)integer(want - 2);
    stream = reinterpret_cast<rdfft_stream_t>(static_cast<uintptr_t>(integer(want - 1)));
  }
  int64_t integer(Py_ssize_t i) const {
    if (!PyLong_Check(args[i])) throw NotPlain{};
    const long long v = PyLong_AsLongLong(args[i]);
    if (v == -1 && PyErr_Occurred()) {
      PyErr_Clear();
      throw NotPlain{};
    }
    return v;
  }
  double number(Py_ssize_t i) const {
    if (!PyFloat_Check(args[i])) throw NotPlain{};
    return PyFloat_AS_DOUBLE(args[i]);
  }
  bool has(Py_ssize_t i) const { return args[i] != Py_None; }
  const at::Tensor& tensor(Py_ssize_t i, at::ScalarType want) const {
    if (!THPVariable_Check(args[i])) throw NotPlain{};
    const at::Tensor& t = THPVariable_Unpack(args[i]);
    if (!t.is_cuda() || t.get_device() != device || t.scalar_type() != want || t.layout() != at::kStrided)
      throw NotPlain{};
    return t;
  }
  // the tensor that sets the call's storage type and (rows, n)
  void first(Py_ssize_t i, int64_t* rows, int64_t* n) {
    if (!THPVariable_Check(args[i])) throw NotPlain{};
    const at::Tensor& t = THPVariable_Unpack(args[i]);
    if (t.dim() != 2) throw NotPlain{};
    type = t.scalar_type();
    if (type == at::kFloat) code = RDFFT_F32;
    else if (type == at::kBFloat16) code = RDFFT_BF16;
    else if (type == at::kHalf) code = RDFFT_F16;
    else throw NotPlain{};
    *rows = t.size(0);
    *n = t.size(1);
  }
  // (rows, n) of the storage type, rows of consecutive elements; null for None
  template <class T>
  void rows(Py_ssize_t i, int64_t r, int64_t n, T** p, int64_t* ld) const {
    *p = nullptr;
    *ld = 0;
    if (!has(i)) return;
    const at::Tensor& t = tensor(i, type);
    if (t.dim() != 2 || t.size(0) != r || t.size(1) != n) throw NotPlain{};
    if ((t.stride(1) != 1 && n > 1) || (t.stride(0) < n && r > 1)) throw NotPlain{};
    *p = static_cast<T*>(t.data_ptr());
    *ld = std::max(t.stride(0), n);
  }
  void* vector(Py_ssize_t i, at::ScalarType want, int64_t n) const {
    if (!has(i)) return nullptr;
    const at::Tensor& t = tensor(i, want);
    if (t.dim() != 1 || t.size(0) != n || !t.is_contiguous()) throw NotPlain{};
    return t.data_ptr();
  }
  float* floats(Py_ssize_t i, int64_t n) const { return static_cast<float*>(vector(i, at::kFloat, n)); }
  // codes at i and scales at i + 1
  act8_t held(Py_ssize_t i, int64_t r, int64_t n) const {
    if (!has(i)) {
      if (has(i + 1)) throw NotPlain{};  // half a checkpoint
      return {nullptr, nullptr};
    }
    const at::Tensor &c = tensor(i, at::kChar), &s = tensor(i + 1, at::kByte);
    if (c.dim() != 2 || c.size(0) != r || c.size(1) != n || !c.is_contiguous()) throw NotPlain{};
    if (s.dim() != 2 || s.size(0) != r || s.size(1) != (n + 31) / 32 || !s.is_contiguous()) throw NotPlain{};
    return {static_cast<int8_t*>(c.data_ptr()), static_cast<uint8_t*>(s.data_ptr())};
  }
  // (rows, n) in 8-bit floating point: codes at i and scales at i + 1, by rows or in tiles
  fp8_t held8(Py_ssize_t i, int64_t r, int64_t n) const {
    if (!has(i)) {
      if (has(i + 1)) throw NotPlain{};
      return fp8_t{};
    }
    const at::Tensor &c = tensor(i, at::kFloat8_e4m3fn), &s = tensor(i + 1, at::kByte);
    const int64_t blocks = (n + 127) / 128, bands = (r + 127) / 128;
    if (c.dim() != 2 || c.size(0) != r || c.size(1) != n || s.dim() != 2 || s.size(1) != blocks) throw NotPlain{};
    if (s.size(0) != r && s.size(0) != bands) throw NotPlain{};
    for (const at::Tensor* t : {&c, &s})
      if ((t->stride(1) != 1 && t->size(1) > 1) || (t->stride(0) < t->size(1) && t->size(0) > 1)) throw NotPlain{};
    return {static_cast<uint8_t*>(c.data_ptr()), std::max(c.stride(0), n), static_cast<uint8_t*>(s.data_ptr()),
            std::max(s.stride(0), blocks), s.size(0) == r ? 1 : 128};
  }
  // (rows, columns) of a matrix in 8-bit floating point
  void size8(Py_ssize_t i, int64_t* rows, int64_t* n) const {
    if (!THPVariable_Check(args[i])) throw NotPlain{};
    const at::Tensor& t = THPVariable_Unpack(args[i]);
    if (t.dim() != 2) throw NotPlain{};
    *rows = t.size(0);
    *n = t.size(1);
  }
  // a workspace of `need` bytes: the caller's at i, or one allocated here; `keep` holds it until the call is made
  void workspace(Py_ssize_t i, int64_t need, at::Tensor* keep, void** p, int64_t* bytes) const {
    *p = nullptr;
    *bytes = 0;
    if (need <= 0) return;  // (a negative status: the call itself will say so)
    if (has(i)) {
      if (!THPVariable_Check(args[i])) throw NotPlain{};
      *keep = THPVariable_Unpack(args[i]);
      if (!keep->is_cuda() || keep->get_device() != device || !keep->is_contiguous()) throw NotPlain{};
      if ((int64_t)keep->nbytes() < need) throw NotPlain{};
    } else {
      *keep = at::empty({need}, at::TensorOptions().dtype(at::kByte).device(at::kCUDA, device));
    }
    *p = keep->data_ptr();
    *bytes = (int64_t)keep->nbytes();
  }
  void needs(std::initializer_list<Py_ssize_t> which) const {
    for (Py_ssize_t i : which)
      if (!has(i)) throw NotPlain{};
  }
};

template <class F>
PyObject* guarded(F&& fn) {
  int status = 0;
  try {
    status = fn();
  } catch (const NotPlain&) {
    Py_RETURN_NONE;
  } catch (const std::exception&) {  // a tensor without storage, no memory for the workspace: the long way raises its own
    Py_RETURN_NONE;
  }
  return PyLong_FromLong(status);
}

// the C call, which may wait for room in the queue, runs without the interpreter's lock (the caller's frame holds
// the tensors)
template <class F>
int unlocked(F&& fn) {
  PyThreadState* const state = PyEval_SaveThread();
  const int status = fn();  // (C entries: nothing is thrown)
  PyEval_RestoreThread(state);
  return status;
}

// x codes scales
PyObject* quantize(PyObject*, PyObject* const* args, Py_ssize_t given) {
  return guarded([&] {
    Call c(args, given, 5);
    int64_t rows, n, ld;
    void* x;
    c.first(0, &rows, &n);
    c.needs({1, 2});
    c.rows(0, rows, n, &x, &ld);
    const act8_t to = c.held(1, rows, n);
    return unlocked([&] { return act8_quantize(x, ld, &to, rows, n, c.code, c.stream); });
  });
}

// codes scales out
PyObject* dequantize(PyObject*, PyObject* const* args, Py_ssize_t given) {
  return guarded([&] {
    Call c(args, given, 5);
    int64_t rows, n, ld;
    void* out;
    c.first(2, &rows, &n);
    c.needs({0, 1});
    c.rows(2, rows, n, &out, &ld);
    const act8_t from = c.held(0, rows, n);
    return unlocked([&] { return act8_dequantize(&from, out, ld, rows, n, c.code, c.stream); });
  });
}

// x residual weight bias y mean rstd codes scales eps
PyObject* norm_forward(PyObject*, PyObject* const* args, Py_ssize_t given) {
  return guarded([&] {
    Call c(args, given, 12);
    int64_t rows, n;
    c.first(0, &rows, &n);
    c.needs({2, 4});
    layer_norm_forward_t a{};
    c.rows(0, rows, n, &a.x, &a.ldx);
    c.rows(1, rows, n, &a.residual, &a.ldr);
    a.weight = c.floats(2, n);
    a.bias = c.floats(3, n);
    c.rows(4, rows, n, &a.y, &a.ldy);
    a.mean = c.floats(5, rows);
    a.rstd = c.floats(6, rows);
    a.checkpoint = c.held(7, rows, n);
    const float eps = (float)c.number(9);
    return unlocked([&] { return layer_norm_forward(&a, rows, n, eps, c.code, c.stream); });
  });
}

// dy x residual codes scales weight mean rstd dx dweight dbias workspace
PyObject* norm_backward(PyObject*, PyObject* const* args, Py_ssize_t given) {
  return guarded([&] {
    Call c(args, given, 14);
    int64_t rows, n;
    c.first(0, &rows, &n);
    c.needs({5, 6, 7, 8, 9, 10});
    layer_norm_backward_t a{};
    c.rows(0, rows, n, &a.dy, &a.ldg);
    c.rows(1, rows, n, &a.x, &a.ldx);
    c.rows(2, rows, n, &a.residual, &a.ldr);
    a.checkpoint = c.held(3, rows, n);
    a.weight = c.floats(5, n);
    a.mean = c.floats(6, rows);
    a.rstd = c.floats(7, rows);
    c.rows(8, rows, n, &a.dx, &a.ldd);
    a.dweight = c.floats(9, n);
    a.dbias = c.floats(10, n);
    at::Tensor keep;
    c.workspace(11, layer_norm_backward_workspace(rows, n), &keep, &a.workspace, &a.workspace_bytes);
    return unlocked([&] { return layer_norm_backward(&a, rows, n, c.code, c.stream); });
  });
}

// x w bias residual y codes scales act workspace
PyObject* product_forward(PyObject*, PyObject* const* args, Py_ssize_t given) {
  return guarded([&] {
    Call c(args, given, 11);
    int64_t tokens, d_in, d_out, same;
    c.first(1, &d_out, &same);
    c.first(0, &tokens, &d_in);
    c.needs({4});
    const auto act = (rdfft_activation_t)c.integer(7);
    linear_forward_t a{};
    c.rows(0, tokens, d_in, &a.x, &a.ldx);
    c.rows(1, d_out, d_in, &a.w, &a.ldw);
    a.bias = c.vector(2, c.type, d_out);
    c.rows(3, tokens, d_out, &a.residual, &a.ldr);
    c.rows(4, tokens, d_out, &a.y, &a.ldy);
    a.checkpoint = c.held(5, tokens, d_out);
    at::Tensor keep;
    c.workspace(8, linear_forward_workspace(d_in, d_out, tokens, c.code), &keep, &a.workspace, &a.workspace_bytes);
    return unlocked([&] { return linear_forward(&a, d_in, d_out, tokens, act, c.code, c.stream); });
  });
}

// dy x w dx dw db add codes scales act workspace
PyObject* product_backward(PyObject*, PyObject* const* args, Py_ssize_t given) {
  return guarded([&] {
    Call c(args, given, 13);
    int64_t tokens, d_in = 1, d_out, other;
    const bool dx = c.has(3), dw = c.has(4), db = c.has(5);
    if (dx) c.first(3, &other, &d_in);
    if (dw) c.first(4, &other, &d_in);
    c.first(0, &tokens, &d_out);
    const auto act = (rdfft_activation_t)c.integer(9);
    linear_backward_t a{};
    c.rows(0, tokens, d_out, &a.dy, &a.ldg);
    if (dw) {
      c.needs({1});
      c.rows(1, tokens, d_in, &a.x, &a.ldx);
      c.rows(4, d_out, d_in, &a.dw, &a.lddw);
    }
    if (dx) {
      c.needs({2});
      c.rows(2, d_out, d_in, &a.w, &a.ldw);
      c.rows(3, tokens, d_in, &a.dx, &a.ldd);
      c.rows(6, tokens, d_in, &a.add, &a.lda);
    }
    a.db = c.vector(5, c.type, d_out);
    if (act != RDFFT_ACT_NONE) {
      c.needs({7, 8});
      a.checkpoint = c.held(7, tokens, d_out);
    }
    at::Tensor keep;
    c.workspace(10, linear_backward_workspace(d_in, d_out, tokens, dx, dw, db, act, c.code), &keep, &a.workspace,
                &a.workspace_bytes);
    return unlocked([&] { return linear_backward(&a, d_in, d_out, tokens, act, c.code, c.stream); });
  });
}

// x codes scales column_codes column_scales
PyObject* quantize8(PyObject*, PyObject* const* args, Py_ssize_t given) {
  return guarded([&] {
    Call c(args, given, 7);
    int64_t rows, n, ld;
    void* x;
    c.first(0, &rows, &n);
    c.rows(0, rows, n, &x, &ld);
    const fp8_t held = c.held8(1, rows, n), columns = c.held8(3, n, rows);
    return unlocked([&] {
      return fp8_quantize(x, ld, held.codes ? &held : nullptr, columns.codes ? &columns : nullptr, rows, n, c.code, c.stream);
    });
  });
}

// codes scales out
PyObject* dequantize8(PyObject*, PyObject* const* args, Py_ssize_t given) {
  return guarded([&] {
    Call c(args, given, 5);
    int64_t rows, n, ld;
    void* out;
    c.first(2, &rows, &n);
    c.needs({0, 1});
    c.rows(2, rows, n, &out, &ld);
    const fp8_t from = c.held8(0, rows, n);
    return unlocked([&] { return fp8_dequantize(&from, out, ld, rows, n, c.code, c.stream); });
  });
}

// x residual weight y summed rstd codes scales codes8 scales8 eps
PyObject* rms_forward(PyObject*, PyObject* const* args, Py_ssize_t given) {
  return guarded([&] {
    Call c(args, given, 13);
    int64_t rows, n;
    c.first(0, &rows, &n);
    c.needs({2});
    rms_norm_forward_t a{};
    c.rows(0, rows, n, &a.x, &a.ldx);
    c.rows(1, rows, n, &a.residual, &a.ldr);
    a.weight = c.floats(2, n);
    c.rows(3, rows, n, &a.y, &a.ldy);
    c.rows(4, rows, n, &a.summed, &a.lds);
    a.rstd = c.floats(5, rows);
    a.checkpoint = c.held(6, rows, n);
    a.y8 = c.held8(8, rows, n);
    const float eps = (float)c.number(10);
    return unlocked([&] { return rms_norm_forward(&a, rows, n, eps, c.code, c.stream); });
  });
}

// dy u codes scales weight rstd add dx dweight workspace
PyObject* rms_backward(PyObject*, PyObject* const* args, Py_ssize_t given) {
  return guarded([&] {
    Call c(args, given, 12);
    int64_t rows, n;
    c.first(0, &rows, &n);
    c.needs({4, 5, 7});
    rms_norm_backward_t a{};
    c.rows(0, rows, n, &a.dy, &a.ldg);
    c.rows(1, rows, n, &a.u, &a.ldu);
    a.checkpoint = c.held(2, rows, n);
    a.weight = c.floats(4, n);
    a.rstd = c.floats(5, rows);
    c.rows(6, rows, n, &a.add, &a.lda);
    c.rows(7, rows, n, &a.dx, &a.ldd);
    a.dweight = c.floats(8, n);
    at::Tensor keep;
    if (c.has(8)) c.workspace(9, rms_norm_backward_workspace(rows, n), &keep, &a.workspace, &a.workspace_bytes);
    return unlocked([&] { return rms_norm_backward(&a, rows, n, c.code, c.stream); });
  });
}

// x_codes x_scales w_codes w_scales bias residual y codes scales act workspace
PyObject* product8_forward(PyObject*, PyObject* const* args, Py_ssize_t given) {
  return guarded([&] {
    Call c(args, given, 13);
    int64_t tokens, d_in, d_out;
    c.needs({0, 2, 6});
    c.first(6, &tokens, &d_out);
    c.size8(2, &d_out, &d_in);
    const auto act = (rdfft_activation_t)c.integer(9);
    linear_fp8_forward_t a{};
    a.x = c.held8(0, tokens, d_in);
    a.w = c.held8(2, d_out, d_in);
    a.bias = c.vector(4, c.type, d_out);
    c.rows(5, tokens, d_out, &a.residual, &a.ldr);
    c.rows(6, tokens, d_out, &a.y, &a.ldy);
    a.checkpoint = c.held(7, tokens, d_out);
    at::Tensor keep;
    c.workspace(10, linear_fp8_forward_workspace(d_in, d_out, tokens, c.code), &keep, &a.workspace, &a.workspace_bytes);
    return unlocked([&] { return linear_fp8_forward(&a, d_in, d_out, tokens, act, c.code, c.stream); });
  });
}

// dy x_codes x_scales w_codes w_scales dx dw db add codes scales act workspace
PyObject* product8_backward(PyObject*, PyObject* const* args, Py_ssize_t given) {
  return guarded([&] {
    Call c(args, given, 15);
    int64_t tokens, d_in = 1, d_out, other;
    const bool dx = c.has(5), dw = c.has(6), db = c.has(7);
    if (dx) c.first(5, &other, &d_in);
    if (dw) c.first(6, &other, &d_in);
    c.first(0, &tokens, &d_out);
    const auto act = (rdfft_activation_t)c.integer(11);
    linear_fp8_backward_t a{};
    c.rows(0, tokens, d_out, &a.dy, &a.ldg);
    if (dw) {
      c.needs({1});
      a.x = c.held8(1, d_in, tokens);
      c.rows(6, d_out, d_in, &a.dw, &a.lddw);
    }
    if (dx) {
      c.needs({3});
      a.w = c.held8(3, d_in, d_out);
      c.rows(5, tokens, d_in, &a.dx, &a.ldd);
      c.rows(8, tokens, d_in, &a.add, &a.lda);
    }
    a.db = c.vector(7, c.type, d_out);
    if (act != RDFFT_ACT_NONE) {
      c.needs({9, 10});
      a.checkpoint = c.held(9, tokens, d_out);
    }
    at::Tensor keep;
    c.workspace(12, linear_fp8_backward_workspace(d_in, d_out, tokens, dx, dw, db, c.code), &keep, &a.workspace,
                &a.workspace_bytes);
    return unlocked([&] { return linear_fp8_backward(&a, d_in, d_out, tokens, act, c.code, c.stream); });
  });
}

#define FAST(name, fn) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fn)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST("act8_quantize", quantize),
                         FAST("act8_dequantize", dequantize),
                         FAST("layer_norm_forward", norm_forward),
                         FAST("layer_norm_backward", norm_backward),
                         FAST("linear_forward", product_forward),
                         FAST("linear_backward", product_backward),
                         FAST("fp8_quantize", quantize8),
                         FAST("fp8_dequantize", dequantize8),
                         FAST("rms_norm_forward", rms_forward),
                         FAST("rms_norm_backward", rms_backward),
                         FAST("linear_fp8_forward", product8_forward),
                         FAST("linear_fp8_backward", product8_backward),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }

// The operators that a program calls once per answer, called with torch tensors.  Such a call is a few microseconds of GPU
// time; reading sizes, types, strides and addresses of up to seven tensors in Python takes as long again (8.1 us a
// call where this takes 2.8, two of them the launch: vgg19_logprobs of one row).
//
// Every function takes the arguments of its namesake in binding.py, by position, and returns the library's code, or None
// where an argument is not what it has to be or the tensors are not on the current device: then binding.py, which makes
// the same checks one at a time, says what is wrong, or makes the call on their device.
#include <Python.h>
#include <c10/cuda/CUDAFunctions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>

#include "../../include/vgg19_b200.h"

namespace {

struct Unfit {};  // thrown for what binding.py has to look at

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) throw Unfit();
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.layout() != at::kStrided) throw Unfit();
  return t;
}

// A matrix whose rows are dense and do not overlap, on the current device.
struct Rows {
  void* data;
  int dtype, dev;
  int64_t rows, cols, ld;
  at::ScalarType type;
  explicit Rows(PyObject* o) {
    const at::Tensor& t = tensor(o);
    type = t.scalar_type();
    dtype = type == at::kFloat ? VGG19_FP32 : type == at::kBFloat16 ? VGG19_BF16 : -1;
    if (dtype < 0 || t.dim() != 2 || !t.is_cuda()) throw Unfit();
    dev = t.get_device();
    rows = t.size(0);
    cols = t.size(1);
    ld = t.is_contiguous() || rows <= 1 ? cols : t.stride(0);
    if (cols > INT_MAX || ld < cols || (!t.is_contiguous() && cols > 1 && t.stride(1) != 1)) throw Unfit();
    if (dev != c10::cuda::current_device()) throw Unfit();
    data = t.data_ptr();
  }
};

// The address of a dense tensor of that type and those sizes (b < 0: of one dimension) on the device; None is null.
void* dense(PyObject* o, at::ScalarType type, int dev, int64_t a, int64_t b = -1) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  if (t.scalar_type() != type || !t.is_cuda() || t.get_device() != dev || !t.is_contiguous() || t.dim() != (b < 0 ? 1 : 2) || t.size(0) != a ||
      (b >= 0 && t.size(1) != b))
    throw Unfit();
  return t.data_ptr();
}
template <typename T> T* dense_as(PyObject* o, at::ScalarType type, int dev, int64_t a, int64_t b = -1) {
  return static_cast<T*>(dense(o, type, dev, a, b));
}

// How many columns a list has; 0 for None.
int columns(PyObject* o) {
  if (o == Py_None) return 0;
  const at::Tensor& t = tensor(o);
  if (t.dim() != 2 || t.size(1) > INT_MAX) throw Unfit();
  return (int)t.size(1);
}

int integer(PyObject* o) {
  const long v = PyLong_AsLong(o);  // (-1 for what is no integer)
  if (v < 0 || v > INT_MAX) throw Unfit();
  return (int)v;
}

void* stream_of(PyObject* o) {
  static PyObject* const name = PyUnicode_InternFromString("cuda_stream");
  if (o == Py_None) return nullptr;
  PyObject* v = PyLong_Check(o) ? Py_NewRef(o) : PyObject_GetAttr(o, name);
  if (!v) throw Unfit();
  const unsigned long long s = PyLong_AsUnsignedLongLong(v);
  Py_DECREF(v);
  if (PyErr_Occurred()) throw Unfit();
  return reinterpret_cast<void*>(s);
}

// f's code as a Python integer; None if it throws.
template <typename F> PyObject* answer(Py_ssize_t given, Py_ssize_t wanted, F f) {
  if (given == wanted) {
    try {
      return PyLong_FromLong(f());
    } catch (...) {
    }
    PyErr_Clear();
  }
  Py_RETURN_NONE;
}

// The library's call without the interpreter's lock: a launch waits while the queue of launches is full.
template <typename F> int unlocked(F f) {
  PyThreadState* s = PyEval_SaveThread();
  const int rc = f();  // (a C entry point: it throws nothing)
  PyEval_RestoreThread(s);
  return rc;
}

PyObject* logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return answer(n, 8, [&] {
    const Rows z(a[0]);
    if ((a[1] == Py_None) != (a[2] == Py_None) || (a[5] == Py_None) != (a[6] == Py_None)) throw Unfit();
    const int ids = columns(a[1]), top = columns(a[5]), dev = z.dev;
    auto* id = dense_as<int32_t>(a[1], at::kInt, dev, z.rows, ids);
    auto* logprob = dense_as<float>(a[2], at::kFloat, dev, z.rows, ids);
    auto* lse = dense_as<float>(a[3], at::kFloat, dev, z.rows);
    auto* entropy = dense_as<float>(a[4], at::kFloat, dev, z.rows);
    auto* top_id = dense_as<int32_t>(a[5], at::kInt, dev, z.rows, top);
    auto* top_logprob = dense_as<float>(a[6], at::kFloat, dev, z.rows, top);
    void* stream = stream_of(a[7]);
    return unlocked([&] {
      return vgg19_logprobs(z.data, z.dtype, z.rows, (int)z.cols, z.ld, id, ids, top, logprob, lse, entropy, top_id, top_logprob, stream);
    });
  });
}

PyObject* logprobs_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return answer(n, 8, [&] {
    const Rows z(a[0]), d(a[6]);
    if (d.dtype != z.dtype || d.rows != z.rows || d.cols != z.cols || a[2] == Py_None || (a[1] == Py_None) != (a[4] == Py_None)) throw Unfit();
    const int ids = columns(a[1]), dev = z.dev;
    auto* id = dense_as<int32_t>(a[1], at::kInt, dev, z.rows, ids);
    auto* lse = dense_as<float>(a[2], at::kFloat, dev, z.rows);
    auto* entropy = dense_as<float>(a[3], at::kFloat, dev, z.rows);
    auto* d_logprob = dense_as<float>(a[4], at::kFloat, dev, z.rows, ids);
    auto* d_entropy = dense_as<float>(a[5], at::kFloat, dev, z.rows);
    void* stream = stream_of(a[7]);
    return unlocked([&] {
      return vgg19_logprobs_backward(z.data, z.dtype, z.rows, (int)z.cols, z.ld, id, ids, lse, entropy, d_logprob, d_entropy, d.data, d.ld, stream);
    });
  });
}

// x, codes, scales, out, group, bias, relu, y, y_f32, stream
PyObject* q4_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return answer(n, 10, [&] {
    const Rows x(a[0]);
    const int out = integer(a[3]), group = integer(a[4]), in = (int)x.cols, dev = x.dev;
    auto buffer = [&](PyObject* o, size_t need) {
      const at::Tensor& t = tensor(o);
      if (!t.is_cuda() || t.get_device() != dev || !t.is_contiguous() || need == 0 || t.nbytes() < need) throw Unfit();
      return t.data_ptr();
    };
    const void* codes = buffer(a[1], vgg19_q4_code_bytes(out, in));
    const void* scales = buffer(a[2], vgg19_q4_scale_bytes(out, in, group));
    auto* bias = dense_as<float>(a[5], at::kFloat, dev, out);
    const int relu = PyObject_IsTrue(a[6]);
    if (relu < 0) throw Unfit();
    void* y = dense(a[7], x.type, dev, x.rows, out);
    auto* y_f32 = dense_as<float>(a[8], at::kFloat, dev, x.rows, out);
    void* stream = stream_of(a[9]);
    return unlocked([&] { return vgg19_q4_linear(x.data, x.dtype, x.rows, in, x.ld, codes, scales, out, group, bias, relu, y, y_f32, stream); });
  });
}

uint64_t word64(PyObject* o) {
  const unsigned long long v = PyLong_AsUnsignedLongLong(o);
  if (PyErr_Occurred()) throw Unfit();
  return v;
}

// x, y, rate, seed, step, step_counter, first, stream
template <typename F> PyObject* any_dropout(F f, PyObject* const* a, Py_ssize_t n) {
  return answer(n, 8, [&] {
    const Rows x(a[0]), y(a[1]);
    if (y.dtype != x.dtype || y.rows != x.rows || y.cols != x.cols) throw Unfit();
    const double rate = PyFloat_AsDouble(a[2]);
    if (PyErr_Occurred()) throw Unfit();
    const uint64_t seed = word64(a[3]), step = word64(a[4]), first = word64(a[6]);
    const auto* counter = static_cast<const uint64_t*>(dense(a[5], at::kLong, x.dev, 1));
    void* stream = stream_of(a[7]);
    return unlocked([&] { return f(x.data, x.dtype, x.rows, (int)x.cols, x.ld, (float)rate, seed, step, counter, first, y.data, y.ld, stream); });
  });
}
PyObject* dropout(PyObject*, PyObject* const* a, Py_ssize_t n) { return any_dropout(vgg19_dropout, a, n); }
PyObject* dropout_backward(PyObject*, PyObject* const* a, Py_ssize_t n) { return any_dropout(vgg19_dropout_backward, a, n); }

vgg19_linear_loss layer_of(const Rows& x, const Rows& w, PyObject* bias, PyObject* labels) {
  if (w.dtype != x.dtype || w.cols != x.cols || w.rows > INT_MAX || labels == Py_None) throw Unfit();
  return vgg19_linear_loss{x.data, x.ld, w.data, w.ld, dense_as<float>(bias, at::kFloat, x.dev, w.rows), dense_as<int32_t>(labels, at::kInt, x.dev, x.rows),
                           x.rows, (int)x.cols, (int)w.rows, x.dtype};
}
struct Bytes {
  void* data;
  size_t size;
  Bytes(PyObject* o, int dev) {
    const at::Tensor& t = tensor(o);
    if (!t.is_cuda() || t.get_device() != dev || !t.is_contiguous()) throw Unfit();
    data = t.data_ptr();
    size = t.nbytes();
  }
};

// x, w, bias, labels, loss, lse, workspace, stream
PyObject* linear_cross_entropy(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return answer(n, 8, [&] {
    const Rows x(a[0]), w(a[1]);
    const vgg19_linear_loss layer = layer_of(x, w, a[2], a[3]);
    auto* loss = dense_as<float>(a[4], at::kFloat, x.dev, x.rows);
    auto* lse = dense_as<float>(a[5], at::kFloat, x.dev, x.rows);
    const Bytes ws(a[6], x.dev);
    void* stream = stream_of(a[7]);
    return unlocked([&] { return vgg19_linear_cross_entropy(&layer, loss, lse, ws.data, ws.size, stream); });
  });
}

// x, w, bias, labels, lse, d_loss, dx, dw, db, workspace, stream
PyObject* linear_cross_entropy_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return answer(n, 11, [&] {
    const Rows x(a[0]), w(a[1]);
    const vgg19_linear_loss layer = layer_of(x, w, a[2], a[3]);
    if (a[4] == Py_None || a[5] == Py_None) throw Unfit();
    auto* lse = dense_as<float>(a[4], at::kFloat, x.dev, x.rows);
    auto* d_loss = dense_as<float>(a[5], at::kFloat, x.dev, x.rows);
    void *dx = nullptr, *dw = nullptr;
    int64_t lddx = x.cols, lddw = x.cols;
    int dw_dtype = x.dtype;
    if (a[6] != Py_None) {
      const Rows d(a[6]);
      if (d.dtype != x.dtype || d.rows != x.rows || d.cols != x.cols) throw Unfit();
      dx = d.data;
      lddx = d.ld;
    }
    if (a[7] != Py_None) {
      const Rows d(a[7]);
      if (d.rows != w.rows || d.cols != x.cols) throw Unfit();
      dw = d.data;
      lddw = d.ld;
      dw_dtype = d.dtype;
    }
    auto* db = dense_as<float>(a[8], at::kFloat, x.dev, w.rows);
    const Bytes ws(a[9], x.dev);
    void* stream = stream_of(a[10]);
    return unlocked([&] { return vgg19_linear_cross_entropy_backward(&layer, lse, d_loss, dx, lddx, dw, dw_dtype, lddw, db, ws.data, ws.size, stream); });
  });
}

PyMethodDef methods[] = {
    {"logprobs", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(logprobs)), METH_FASTCALL, nullptr},
    {"logprobs_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(logprobs_backward)), METH_FASTCALL, nullptr},
    {"q4_linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(q4_linear)), METH_FASTCALL, nullptr},
    {"dropout", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(dropout)), METH_FASTCALL, nullptr},
    {"dropout_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(dropout_backward)), METH_FASTCALL, nullptr},
    {"linear_cross_entropy", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear_cross_entropy)), METH_FASTCALL, nullptr},
    {"linear_cross_entropy_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear_cross_entropy_backward)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensor_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensor_calls() { return PyModule_Create(&module); }

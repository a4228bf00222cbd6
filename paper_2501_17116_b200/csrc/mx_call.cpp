// The fp4_mx_* calls for Python: a module that takes tensors as they are and calls the library.  At the smallest sizes marshalling is most of a call's
// time (SwiGLU of 1 x 11008: 3.5 us on the device, 5.9 a call through ctypes with its tensors asked from Python for their address, shape, stride, type and
// device, 4.0 through this).  Knows nothing of the library but the prototypes: it is given the functions' addresses.
//
// Every function: (address of the entry point, context, stream, status word, device, the entry point's own arguments); matrices are two-dimensional
// tensors of the shape that the other arguments say, or None, operands addresses of their structures or None, all else integers.  The result
// is the entry point's.
#include <torch/csrc/autograd/python_variable.h>

#include "fp4_linear.h"

namespace {

// What a call is made from; `ok` false: a Python exception is set.
struct Call {
  static constexpr int HEAD = 5;
  PyObject* const* args;
  bool ok = true;
  int64_t device = 0;
  fp4_mx_matrix space[4];
  int used = 0;

  Call(PyObject* const* a, Py_ssize_t n, int own) : args(a) {
    if (n != HEAD + own) {
      PyErr_Format(PyExc_TypeError, "%zd arguments instead of %d", n, HEAD + own);
      ok = false;
    } else {
      device = integer(args[4]);
    }
  }
  int64_t integer(PyObject* o) {
    if (!ok) return 0;
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) ok = false;
    return v;
  }
  int64_t number(int i) { return ok ? integer(args[HEAD + i]) : 0; }
  void* address(PyObject* o) {
    if (!ok || o == Py_None) return nullptr;
    void* p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) ok = false;
    return p;
  }
  fp4_mx_tensor* operand(int i) { return ok ? static_cast<fp4_mx_tensor*>(address(args[HEAD + i])) : nullptr; }
  fp4_mx_matrix* matrix(int i, int64_t rows, int64_t cols) {
    if (!ok || args[HEAD + i] == Py_None) return nullptr;
    fp4_mx_matrix* m = &space[used++];
    try {
      ok = read(args[HEAD + i], rows, cols, m);
    } catch (const std::exception& e) {    // (a tensor without memory, say)
      PyErr_SetString(PyExc_RuntimeError, e.what());
      ok = false;
    }
    return m;
  }
  static bool refuse(const char* what) {
    PyErr_SetString(PyExc_AssertionError, what);
    return false;
  }
  // `rows` x `cols` (checked): the shape the call is about.
  bool read(PyObject* o, int64_t rows, int64_t cols, fp4_mx_matrix* m) const {
    if (!THPVariable_Check(o)) return refuse("a matrix is a tensor");
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.layout() != at::kStrided || t.dim() != 2 || t.size(0) != rows || t.size(1) != cols) {
      PyErr_Format(PyExc_AssertionError, "a matrix is not of %lld x %lld elements", (long long)rows, (long long)cols);
      return false;
    }
    if (!t.is_cuda() || t.device().index() != device) {
      PyErr_Format(PyExc_AssertionError, "a matrix on device %d, the context on device %lld", t.is_cuda() ? int(t.device().index()) : -1, (long long)device);
      return false;
    }
    if (t.stride(1) != 1 && cols > 1) return refuse("a matrix's rows are contiguous");
    const at::ScalarType type = t.scalar_type();
    if (type != at::kBFloat16 && type != at::kHalf && type != at::kFloat) {
      PyErr_Format(PyExc_AssertionError, "%s: a matrix is of torch.bfloat16, torch.float16 or torch.float32", c10::toString(type));
      return false;
    }
    m->data = t.data_ptr();
    m->ld = t.stride(0);
    m->dtype = type == at::kBFloat16 ? FP4_DTYPE_BF16 : type == at::kHalf ? FP4_DTYPE_FP16 : FP4_DTYPE_FP32;
    m->reserved = 0;
    return true;
  }

  // The call, with other threads let run meanwhile (host threads take turns on a context).
  template <class F, class... A>
  PyObject* make(F* /* its type */, A... a) {
    F* f = reinterpret_cast<F*>(address(args[0]));
    fp4_ctx* ctx = static_cast<fp4_ctx*>(address(args[1]));
    void* stream = address(args[2]);
    int32_t* status = static_cast<int32_t*>(address(args[3]));
    if (!ok) return nullptr;
    if (!f) {
      PyErr_SetString(PyExc_ValueError, "no entry point");
      return nullptr;
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f(ctx, stream, a..., status);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  }
};

PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Call c(a, n, 2);
  fp4_mx_tensor* out = c.operand(1);
  fp4_mx_matrix* x = out ? c.matrix(0, out->rows, out->cols) : nullptr;
  return c.ok ? c.make(static_cast<decltype(&fp4_mx_quantize)>(nullptr), x, out) : nullptr;
}
PyObject* dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Call c(a, n, 3);
  fp4_mx_tensor* q = c.operand(0);
  const int transposed = int(c.number(1));
  fp4_mx_matrix* out = q ? c.matrix(2, transposed ? q->cols : q->rows, transposed ? q->rows : q->cols) : nullptr;
  return c.ok ? c.make(static_cast<decltype(&fp4_mx_dequantize)>(nullptr), q, transposed, out) : nullptr;
}
PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Call c(a, n, 4);
  fp4_mx_tensor *x = c.operand(0), *w = c.operand(1);
  const int flags = int(c.number(2));
  fp4_mx_matrix* out = x && w ? c.matrix(3, flags & FP4_MX_A_T ? x->cols : x->rows, flags & FP4_MX_B_T ? w->cols : w->rows) : nullptr;
  return c.ok ? c.make(static_cast<decltype(&fp4_mx_gemm)>(nullptr), x, w, flags, out) : nullptr;
}
PyObject* linear_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Call c(a, n, 9);
  const int64_t M = c.number(2), K = c.number(3), N = c.number(4);
  const int reuse = int(c.number(5));
  fp4_mx_matrix *x = c.matrix(0, M, K), *w = c.matrix(1, K, N), *y = c.matrix(6, M, N);
  fp4_mx_tensor *sx = c.operand(7), *sw = c.operand(8);
  return c.ok ? c.make(static_cast<decltype(&fp4_mx_linear_fwd)>(nullptr), x, w, M, K, N, reuse, y, sx, sw) : nullptr;
}
PyObject* linear_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Call c(a, n, 9);
  fp4_mx_tensor *sx = c.operand(1), *sw = c.operand(2);
  const int64_t M = c.number(3), K = c.number(4), N = c.number(5);
  const int flags = int(c.number(6));
  fp4_mx_matrix *dy = c.matrix(0, M, N), *dx = c.matrix(7, M, K), *dw = c.matrix(8, K, N);
  return c.ok ? c.make(static_cast<decltype(&fp4_mx_linear_bwd)>(nullptr), dy, sx, sw, M, K, N, flags, dx, dw) : nullptr;
}
PyObject* swiglu_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Call c(a, n, 8);
  const int64_t rows = c.number(2), cols = c.number(3);
  fp4_mx_matrix *gate = c.matrix(0, rows, cols), *up = c.matrix(1, rows, cols), *h = c.matrix(4, rows, cols);
  fp4_mx_tensor *g = c.operand(5), *u = c.operand(6), *q = c.operand(7);
  return c.ok ? c.make(static_cast<decltype(&fp4_mx_swiglu_fwd)>(nullptr), gate, up, rows, cols, h, g, u, q) : nullptr;
}
PyObject* swiglu_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Call c(a, n, 9);
  fp4_mx_tensor *g = c.operand(1), *u = c.operand(2);
  const int64_t rows = c.number(3), cols = c.number(4);
  fp4_mx_matrix *dh = c.matrix(0, rows, cols), *dgate = c.matrix(5, rows, cols), *dup = c.matrix(6, rows, cols), *h = c.matrix(7, rows, cols);
  fp4_mx_tensor* q = c.operand(8);
  return c.ok ? c.make(static_cast<decltype(&fp4_mx_swiglu_bwd)>(nullptr), dh, g, u, rows, cols, dgate, dup, h, q) : nullptr;
}

#define CALL(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CALL(quantize), CALL(dequantize), CALL(gemm), CALL(linear_fwd), CALL(linear_bwd), CALL(swiglu_fwd), CALL(swiglu_bwd),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_mx_call", "The fp4_mx_* calls on tensors.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__mx_call() { return PyModule_Create(&module); }

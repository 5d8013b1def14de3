// CPython entry to the launch calls of the C ABI (no Python types beyond integers and floats, no HIP).
//
// A launch on small inputs is bound by the host: of 7.2 us for one tw_gemm issued from Python, 0.7 us were the
// ctypes call and the wrappers around it.  Here the arguments are read straight from the vector call
// (0.2 us).  Anything but plain integers (floats) in range returns None, and the caller takes the ctypes route,
// which converts or refuses as it always has.  The functions are bound by address, so that they are those
// of the library that the process has loaded.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <climits>
#include <cstdint>

namespace {

typedef int (*gemm_fn)(const void*, int, int, int, void*, void*, int, void*);
typedef int (*gemm_i8_fn)(const void*, int, int, void*, void*, int, int, float, void*);
typedef int (*conv_fn)(const void*, void*, void*, int, void*);
typedef int (*conv_i8_fn)(const void*, void*, void*, int, int, float, void*);
typedef int (*rmsnorm_fn)(const void*, const void*, const void*, float, int, int, int, void*, void*, void*, int, float*, void*);
typedef int (*quant_i8_fn)(const void*, int, int, int, void*, int, float*, void*);
typedef int (*gemm_i8_scaled_fn)(const void*, int, int, void*, const float*, const float*, void*, int, void*);
typedef int (*quant_mx4_fn)(const void*, int, int, int, int, void*, void*, int, void*);
typedef int (*gemm_mx4_fn)(const void*, const void*, int, int, void*, void*, int, void*);
typedef int (*gemm_mx4_grouped_fn)(const void*, const void*, int, int, const int*, void*, void*, int, void*);
gemm_fn f_gemm = nullptr;
gemm_i8_fn f_gemm_i8 = nullptr;
conv_fn f_conv = nullptr;
conv_i8_fn f_conv_i8 = nullptr;
rmsnorm_fn f_rmsnorm = nullptr;
quant_i8_fn f_quant_i8 = nullptr;
gemm_i8_scaled_fn f_gemm_i8_scaled = nullptr;
quant_mx4_fn f_quant_mx4 = nullptr;
gemm_mx4_fn f_gemm_mx4 = nullptr;
gemm_mx4_grouped_fn f_gemm_mx4_grouped = nullptr;
constexpr int N_FUNCTIONS = 10;

// Each sets `ok` to false when the object is not a plain number that the C type holds.
void* ptr(PyObject* o, bool& ok) {
  if (!PyLong_CheckExact(o)) { ok = false; return nullptr; }
  const unsigned long long v = PyLong_AsUnsignedLongLong(o);
  if (v == ~0ull && PyErr_Occurred()) { PyErr_Clear(); ok = false; }
  return (void*)(uintptr_t)v;
}
void* ptr_or_none(PyObject* o, bool& ok) { return o == Py_None ? nullptr : ptr(o, ok); }
int num(PyObject* o, bool& ok) {
  if (!PyLong_CheckExact(o)) { ok = false; return 0; }
  int over = 0;
  const long v = PyLong_AsLongAndOverflow(o, &over);
  if (over || v < INT_MIN || v > INT_MAX) { ok = false; return 0; }
  return (int)v;
}
float real(PyObject* o, bool& ok) {
  if (!PyFloat_CheckExact(o)) { ok = false; return 0.f; }
  return (float)PyFloat_AS_DOUBLE(o);
}
template <class F>
PyObject* run(F f) {
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = f();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  bool ok = n == N_FUNCTIONS;
  void* p[N_FUNCTIONS] = {};
  for (int i = 0; ok && i < N_FUNCTIONS; ++i) p[i] = ptr(a[i], ok);
  if (!ok) { PyErr_SetString(PyExc_TypeError, "ten function addresses expected"); return nullptr; }
  f_gemm = (gemm_fn)p[0]; f_gemm_i8 = (gemm_i8_fn)p[1]; f_conv = (conv_fn)p[2]; f_conv_i8 = (conv_i8_fn)p[3];
  f_rmsnorm = (rmsnorm_fn)p[4]; f_quant_i8 = (quant_i8_fn)p[5]; f_gemm_i8_scaled = (gemm_i8_scaled_fn)p[6];
  f_quant_mx4 = (quant_mx4_fn)p[7]; f_gemm_mx4 = (gemm_mx4_fn)p[8]; f_gemm_mx4_grouped = (gemm_mx4_grouped_fn)p[9];
  Py_RETURN_NONE;
}
PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {      // A, M, lda, layout, handle, C, ldc, stream
  bool ok = n == 8 && f_gemm;
  if (!ok) Py_RETURN_NONE;
  void* A = ptr(a[0], ok); const int M = num(a[1], ok), lda = num(a[2], ok), layout = num(a[3], ok);
  void* h = ptr(a[4], ok); void* C = ptr(a[5], ok); const int ldc = num(a[6], ok); void* s = ptr(a[7], ok);
  if (!ok) Py_RETURN_NONE;
  return run([&] { return f_gemm(A, M, lda, layout, h, C, ldc, s); });
}
PyObject* gemm_i8(PyObject*, PyObject* const* a, Py_ssize_t n) {   // A, M, lda, handle, C, ldc, c_dtype, scale, stream
  bool ok = n == 9 && f_gemm_i8;
  if (!ok) Py_RETURN_NONE;
  void* A = ptr(a[0], ok); const int M = num(a[1], ok), lda = num(a[2], ok);
  void* h = ptr(a[3], ok); void* C = ptr(a[4], ok); const int ldc = num(a[5], ok), dt = num(a[6], ok);
  const float scale = real(a[7], ok); void* s = ptr(a[8], ok);
  if (!ok) Py_RETURN_NONE;
  return run([&] { return f_gemm_i8(A, M, lda, h, C, ldc, dt, scale, s); });
}
PyObject* conv(PyObject*, PyObject* const* a, Py_ssize_t n) {      // X, binding, C, ldc, stream
  bool ok = n == 5 && f_conv;
  if (!ok) Py_RETURN_NONE;
  void* X = ptr(a[0], ok); void* b = ptr(a[1], ok); void* C = ptr(a[2], ok); const int ldc = num(a[3], ok);
  void* s = ptr(a[4], ok);
  if (!ok) Py_RETURN_NONE;
  return run([&] { return f_conv(X, b, C, ldc, s); });
}
PyObject* conv_i8(PyObject*, PyObject* const* a, Py_ssize_t n) {   // X, binding, C, ldc, c_dtype, scale, stream
  bool ok = n == 7 && f_conv_i8;
  if (!ok) Py_RETURN_NONE;
  void* X = ptr(a[0], ok); void* b = ptr(a[1], ok); void* C = ptr(a[2], ok);
  const int ldc = num(a[3], ok), dt = num(a[4], ok); const float scale = real(a[5], ok); void* s = ptr(a[6], ok);
  if (!ok) Py_RETURN_NONE;
  return run([&] { return f_conv_i8(X, b, C, ldc, dt, scale, s); });
}

PyObject* rmsnorm(PyObject*, PyObject* const* a, Py_ssize_t n) {   // X, R, gamma, eps, M, K, ld, H, Y, Q, ldq, scale, stream
  bool ok = n == 13 && f_rmsnorm;
  if (!ok) Py_RETURN_NONE;
  void *X = ptr(a[0], ok), *R = ptr_or_none(a[1], ok), *gamma = ptr_or_none(a[2], ok); const float eps = real(a[3], ok);
  const int M = num(a[4], ok), K = num(a[5], ok), ld = num(a[6], ok);
  void *H = ptr_or_none(a[7], ok), *Y = ptr_or_none(a[8], ok), *Q = ptr_or_none(a[9], ok); const int ldq = num(a[10], ok);
  float* scale = (float*)ptr_or_none(a[11], ok); void* s = ptr(a[12], ok);
  if (!ok) Py_RETURN_NONE;
  return run([&] { return f_rmsnorm(X, R, gamma, eps, M, K, ld, H, Y, Q, ldq, scale, s); });
}
PyObject* quant_i8(PyObject*, PyObject* const* a, Py_ssize_t n) {  // X, M, K, ldx, Q, ldq, scale, stream
  bool ok = n == 8 && f_quant_i8;
  if (!ok) Py_RETURN_NONE;
  void* X = ptr(a[0], ok); const int M = num(a[1], ok), K = num(a[2], ok), ldx = num(a[3], ok);
  void* Q = ptr(a[4], ok); const int ldq = num(a[5], ok); float* scale = (float*)ptr(a[6], ok); void* s = ptr(a[7], ok);
  if (!ok) Py_RETURN_NONE;
  return run([&] { return f_quant_i8(X, M, K, ldx, Q, ldq, scale, s); });
}
PyObject* gemm_i8_scaled(PyObject*, PyObject* const* a, Py_ssize_t n) {   // A, M, lda, handle, a_scale, w_scale, C, ldc, stream
  bool ok = n == 9 && f_gemm_i8_scaled;
  if (!ok) Py_RETURN_NONE;
  void* A = ptr(a[0], ok); const int M = num(a[1], ok), lda = num(a[2], ok); void* h = ptr(a[3], ok);
  const float *as = (const float*)ptr(a[4], ok), *ws = (const float*)ptr(a[5], ok);
  void* C = ptr(a[6], ok); const int ldc = num(a[7], ok); void* s = ptr(a[8], ok);
  if (!ok) Py_RETURN_NONE;
  return run([&] { return f_gemm_i8_scaled(A, M, lda, h, as, ws, C, ldc, s); });
}
PyObject* quant_mx4(PyObject*, PyObject* const* a, Py_ssize_t n) { // X, M, K, ldx, layout, Q, S, ldq, stream
  bool ok = n == 9 && f_quant_mx4;
  if (!ok) Py_RETURN_NONE;
  void* X = ptr(a[0], ok); const int M = num(a[1], ok), K = num(a[2], ok), ldx = num(a[3], ok), layout = num(a[4], ok);
  void *Q = ptr(a[5], ok), *S = ptr(a[6], ok); const int ldq = num(a[7], ok); void* s = ptr(a[8], ok);
  if (!ok) Py_RETURN_NONE;
  return run([&] { return f_quant_mx4(X, M, K, ldx, layout, Q, S, ldq, s); });
}
PyObject* gemm_mx4(PyObject*, PyObject* const* a, Py_ssize_t n) {  // Q, S, M, ldq, handle, C, ldc, stream
  bool ok = n == 8 && f_gemm_mx4;
  if (!ok) Py_RETURN_NONE;
  void *Q = ptr(a[0], ok), *S = ptr(a[1], ok); const int M = num(a[2], ok), ldq = num(a[3], ok);
  void *h = ptr(a[4], ok), *C = ptr(a[5], ok); const int ldc = num(a[6], ok); void* s = ptr(a[7], ok);
  if (!ok) Py_RETURN_NONE;
  return run([&] { return f_gemm_mx4(Q, S, M, ldq, h, C, ldc, s); });
}
PyObject* gemm_mx4_grouped(PyObject*, PyObject* const* a, Py_ssize_t n) { // Q, S, M, ldq, offsets, handle, C, ldc, stream
  bool ok = n == 9 && f_gemm_mx4_grouped;
  if (!ok) Py_RETURN_NONE;
  void *Q = ptr(a[0], ok), *S = ptr(a[1], ok); const int M = num(a[2], ok), ldq = num(a[3], ok);
  const int* off = (const int*)ptr(a[4], ok); void *h = ptr(a[5], ok), *C = ptr(a[6], ok);
  const int ldc = num(a[7], ok); void* s = ptr(a[8], ok);
  if (!ok) Py_RETURN_NONE;
  return run([&] { return f_gemm_mx4_grouped(Q, S, M, ldq, off, h, C, ldc, s); });
}

#define METHOD(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
                         {"gemm", (PyCFunction)(void (*)(void))gemm, METH_FASTCALL, nullptr},
                         {"gemm_i8", (PyCFunction)(void (*)(void))gemm_i8, METH_FASTCALL, nullptr},
                         {"conv", (PyCFunction)(void (*)(void))conv, METH_FASTCALL, nullptr},
                         {"conv_i8", (PyCFunction)(void (*)(void))conv_i8, METH_FASTCALL, nullptr},
                         METHOD(rmsnorm), METHOD(quant_i8), METHOD(gemm_i8_scaled), METHOD(quant_mx4), METHOD(gemm_mx4),
                         METHOD(gemm_mx4_grouped),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_twcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__twcall() { return PyModule_Create(&module); }

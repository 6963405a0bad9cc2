// Compiled argument marshalling of the 16-bit and 8-bit products, the norms and dropout: the Python names of
// include/hgemm.h, qgemm.h, layernorm.h, rmsnorm.h and dropout.h as builtins that unpack torch tensors, check shapes, types,
// strides and device, and call the C ABI. No arithmetic and no CUDA kernels here. Reached through the
// interpreter, the same checks cost 8 to 15 us per call, more than the kernels of a single token take.
//
// The C functions are handed over as addresses by binding.py, which loads libdgemm.so, together with the
// function that raises DgemmError.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstdint>
#include <cstring>
#include <exception>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/dropout.h"
#include "../../include/hgemm.h"
#include "../../include/layernorm.h"
#include "../../include/qgemm.h"
#include "../../include/rmsnorm.h"

namespace {

decltype(&hgemm_epilogue) f_epilogue = nullptr;
decltype(&hgemm_epilogue_bwd) f_epilogue_bwd = nullptr;
decltype(&hgemm_gated) f_gated = nullptr;
decltype(&hgemm_gated_bwd) f_gated_bwd = nullptr;
decltype(&layernorm_fwd) f_ln_fwd = nullptr;
decltype(&layernorm_bwd) f_ln_bwd = nullptr;
decltype(&rmsnorm_fwd) f_rms_fwd = nullptr;
decltype(&rmsnorm_fwd_e4m3) f_rms_e4m3 = nullptr;
decltype(&quantize_rows_e4m3) f_rows_e4m3 = nullptr;
decltype(&rmsnorm_bwd) f_rms_bwd = nullptr;
decltype(&dropout_fwd) f_drop_fwd = nullptr;
decltype(&dropout_bwd) f_drop_bwd = nullptr;
decltype(&qgemm_epilogue) f_q_epilogue = nullptr;
decltype(&qgemm_gated) f_q_gated = nullptr;
PyObject* on_error = nullptr;

// Arguments by position or name. `names` ends with nullptr; the first `required` must be given.
struct Args {
  PyObject* v[24];
  bool parse(const char* fn, const char* const* names, PyObject* const* keys, int required, PyObject* const* args, Py_ssize_t nargs,
             PyObject* kwnames) {
    int n = 0;
    while (names[n]) v[n++] = nullptr;
    if (nargs > n) {
      PyErr_Format(PyExc_TypeError, "%s: takes at most %d arguments", fn, n);
      return false;
    }
    for (Py_ssize_t i = 0; i < nargs; ++i) v[i] = args[i];
    const Py_ssize_t nk = kwnames ? PyTuple_GET_SIZE(kwnames) : 0;
    for (Py_ssize_t k = 0; k < nk; ++k) {
      PyObject* key = PyTuple_GET_ITEM(kwnames, k);
      int at = -1;
      for (int i = 0; i < n && at < 0; ++i)
        if (keys[i] == key) at = i;
      for (int i = 0; i < n && at < 0; ++i)
        if (PyUnicode_CompareWithASCIIString(key, names[i]) == 0) at = i;
      if (at < 0) {
        PyErr_Format(PyExc_TypeError, "%s: unexpected argument '%U'", fn, key);
        return false;
      }
      if (v[at]) {
        PyErr_Format(PyExc_TypeError, "%s: '%s' given twice", fn, names[at]);
        return false;
      }
      v[at] = args[nargs + k];
    }
    for (int i = 0; i < required; ++i)
      if (!v[i]) {
        PyErr_Format(PyExc_TypeError, "%s: missing argument '%s'", fn, names[i]);
        return false;
      }
    return true;
  }
};

// Interned names of one function's arguments, made once.
struct Names {
  const char* const* names;
  PyObject* keys[24];
  explicit Names(const char* const* n) : names(n) {
    for (int i = 0; n[i]; ++i) keys[i] = PyUnicode_InternFromString(n[i]);
  }
};

const at::Tensor* tensor(PyObject* o, const char* name, bool optional) {
  if (!o || o == Py_None) {
    if (!optional) PyErr_Format(PyExc_TypeError, "%s: expected a torch.Tensor", name);
    return nullptr;
  }
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s: expected a torch.Tensor", name);
    return nullptr;
  }
  return &THPVariable_Unpack(o);
}

int type_code(at::ScalarType t) {
  switch (t) {
    case at::kFloat: return HGEMM_TYPE_F32;
    case at::kHalf: return HGEMM_TYPE_F16;
    case at::kBFloat16: return HGEMM_TYPE_BF16;
    default: return -1;
  }
}

struct Call {
  const char* fn;
  at::ScalarType type = at::kFloat;
  int code = 0;
  int device = 0;
  void* stream = nullptr;
  bool check = true;
  const char* others = "the type of the first operand";  // what the other operands have to be of

  // Element type from the first operand; device and stream; the check flag.
  bool begin(const at::Tensor& first, const char* name, PyObject* stream_arg, PyObject* check_arg) {
    type = first.scalar_type();
    code = type_code(type);
    if (code < 0) {
      PyErr_Format(PyExc_TypeError, "%s: unsupported element type", name);
      return false;
    }
    device = (int)c10::cuda::current_device();
    if (!stream_arg || stream_arg == Py_None) {
      stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    } else if (PyLong_Check(stream_arg)) {
      stream = PyLong_AsVoidPtr(stream_arg);
    } else {
      PyObject* h = PyObject_GetAttrString(stream_arg, "cuda_stream");
      if (!h) return false;
      stream = PyLong_AsVoidPtr(h);
      Py_DECREF(h);
    }
    if (PyErr_Occurred()) return false;
    if (check_arg) {
      const int t = PyObject_IsTrue(check_arg);
      if (t < 0) return false;
      check = t != 0;
    }
    return true;
  }

  bool on_device(const at::Tensor& x, const char* name) const {
    if (x.is_cuda() && x.get_device() == device) return true;
    PyErr_Format(PyExc_ValueError, "%s: expected a CUDA tensor on the current device", name);
    return false;
  }

  // Address and leading dimension of a rows x cols matrix of the call's type.
  bool matrix(PyObject* o, const char* name, int64_t rows, int64_t cols, bool optional, void** ptr, int64_t* ld) const {
    return matrix_of(type, others, o, name, rows, cols, optional, ptr, ld);
  }
  // ... of 8-bit values.
  bool matrix8(PyObject* o, const char* name, int64_t rows, int64_t cols, void** ptr, int64_t* ld) const {
    return matrix_of(at::kFloat8_e4m3fn, "float8_e4m3fn", o, name, rows, cols, false, ptr, ld);
  }
  bool matrix_of(at::ScalarType t, const char* what, PyObject* o, const char* name, int64_t rows, int64_t cols, bool optional, void** ptr,
                 int64_t* ld) const {
    *ptr = nullptr;
    *ld = cols > 0 ? cols : 1;
    const at::Tensor* x = tensor(o, name, optional);
    if (!x) return !PyErr_Occurred();
    if (x->scalar_type() != t || x->dim() != 2) {
      PyErr_Format(PyExc_TypeError, "%s: need a 2-D tensor of %s", name, what);
      return false;
    }
    if (!on_device(*x, name)) return false;
    if (x->size(0) != rows || x->size(1) != cols) {
      PyErr_Format(PyExc_ValueError, "%s: shape (%lld, %lld), expected (%lld, %lld)", name, (long long)x->size(0), (long long)x->size(1),
                   (long long)rows, (long long)cols);
      return false;
    }
    if (rows > 0 && cols > 1 && x->stride(1) != 1) {
      PyErr_Format(PyExc_ValueError, "%s: columns must be contiguous (row-major)", name);
      return false;
    }
    if (rows > 1) {
      if (x->stride(0) < cols) {
        PyErr_Format(PyExc_ValueError, "%s: rows overlap (row stride %lld, %lld columns)", name, (long long)x->stride(0), (long long)cols);
        return false;
      }
      *ld = x->stride(0) > 0 ? x->stride(0) : 1;
    }
    *ptr = x->data_ptr();
    return true;
  }

  // Address of n contiguous values of `t`.
  bool vector(PyObject* o, const char* name, at::ScalarType t, int64_t n, bool optional, void** ptr) const {
    *ptr = nullptr;
    const at::Tensor* x = tensor(o, name, optional);
    if (!x) return !PyErr_Occurred();
    if (x->scalar_type() != t || x->dim() != 1) {
      PyErr_Format(PyExc_TypeError, "%s: need a 1-D tensor of %s", name, t == at::kFloat ? "float32" : others);
      return false;
    }
    if (!on_device(*x, name)) return false;
    if (x->size(0) != n || (n > 1 && x->stride(0) != 1)) {
      PyErr_Format(PyExc_ValueError, "%s: expected %lld contiguous values", name, (long long)n);
      return false;
    }
    *ptr = x->data_ptr();
    return true;
  }

  PyObject* done(int rc) const {
    if (rc < 0 && check) return PyObject_CallFunction(on_error, "is", rc, fn);
    return PyLong_FromLong(rc);
  }
};

// Rows and columns of a required 2-D operand.
const at::Tensor* operand(PyObject* o, const char* name) {
  const at::Tensor* x = tensor(o, name, false);
  if (x && x->dim() != 2) {
    PyErr_Format(PyExc_TypeError, "%s: need a 2-D tensor", name);
    return nullptr;
  }
  return x;
}

bool flag(PyObject* o, bool* out) {
  *out = false;
  if (!o) return true;
  const int t = PyObject_IsTrue(o);
  *out = t > 0;
  return t >= 0;
}
bool integer(PyObject* o, int fallback, int* out) {
  *out = fallback;
  if (!o) return true;
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) return false;
  *out = v < -1000 ? -1000 : v > 1000 ? 1000 : (int)v;
  return true;
}

// A 64-bit word from any integer (its two's complement, modulo 2^64).
bool word64(PyObject* o, uint64_t* out) {
  *out = 0;
  if (!o) return true;
  PyObject* n = PyNumber_Index(o);
  if (!n) return false;
  *out = PyLong_AsUnsignedLongLongMask(n);
  Py_DECREF(n);
  return !PyErr_Occurred();
}
bool real(PyObject* o, double fallback, double* out) {
  *out = fallback;
  return !o || (*out = PyFloat_AsDouble(o)) != -1.0 || !PyErr_Occurred();
}

// Runs `body`, turning a C++ exception (from torch) into a Python one.
template <typename F>
PyObject* guarded(F body) {
  try {
    return body();
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

PyObject* py_epilogue(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"A", "B", "D", "bias", "act", "residual", "preact", "transa", "transb", "stream", "check", nullptr};
  static Names keys(names);
  Args a;
  if (!a.parse("hgemm_epilogue", names, keys.keys, 3, args, nargs, kwnames)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor *A = operand(a.v[0], "A"), *B = A ? operand(a.v[1], "B") : nullptr;
    bool ta, tb;
    int act;
    if (!A || !B || !flag(a.v[7], &ta) || !flag(a.v[8], &tb) || !integer(a.v[4], HGEMM_ACT_NONE, &act)) return nullptr;
    Call c{"hgemm_epilogue"};
    if (!c.begin(*A, "A", a.v[9], a.v[10])) return nullptr;
    const int64_t M = A->size(ta ? 1 : 0), K = A->size(ta ? 0 : 1), N = B->size(tb ? 0 : 1);
    void *pa, *pb, *pd, *pr, *pz, *bias;
    int64_t lda, ldb, ldd, ldr, ldz;
    if (!c.matrix(a.v[0], "A", ta ? K : M, ta ? M : K, false, &pa, &lda) || !c.matrix(a.v[1], "B", tb ? N : K, tb ? K : N, false, &pb, &ldb) ||
        !c.matrix(a.v[2], "D", M, N, false, &pd, &ldd) || !c.vector(a.v[3], "bias", c.type, N, true, &bias) ||
        !c.matrix(a.v[5], "residual", M, N, true, &pr, &ldr) || !c.matrix(a.v[6], "preact", M, N, true, &pz, &ldz))
      return nullptr;
    return c.done(f_epilogue(c.code, ta, tb, M, N, K, pa, lda, pb, ldb, bias, act, pr, ldr, pd, ldd, pz, ldz, c.stream));
  });
}

PyObject* py_epilogue_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"A", "B", "dD", "act", "preact", "dA", "dB", "dbias", "transa", "transb", "stream", "check", nullptr};
  static Names keys(names);
  Args a;
  if (!a.parse("hgemm_epilogue_bwd", names, keys.keys, 3, args, nargs, kwnames)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor *A = operand(a.v[0], "A"), *B = A ? operand(a.v[1], "B") : nullptr;
    bool ta, tb;
    int act;
    if (!A || !B || !flag(a.v[8], &ta) || !flag(a.v[9], &tb) || !integer(a.v[3], HGEMM_ACT_NONE, &act)) return nullptr;
    Call c{"hgemm_epilogue_bwd"};
    if (!c.begin(*A, "A", a.v[10], a.v[11])) return nullptr;
    const int64_t M = A->size(ta ? 1 : 0), K = A->size(ta ? 0 : 1), N = B->size(tb ? 0 : 1);
    const int64_t ar = ta ? K : M, ac = ta ? M : K, br = tb ? N : K, bc = tb ? K : N;
    void *pa, *pb, *pd, *pz, *pda, *pdb, *db;
    int64_t lda, ldb, ldd, ldz, ldda, lddb;
    if (!c.matrix(a.v[0], "A", ar, ac, false, &pa, &lda) || !c.matrix(a.v[1], "B", br, bc, false, &pb, &ldb) ||
        !c.matrix(a.v[2], "dD", M, N, false, &pd, &ldd) || !c.matrix(a.v[4], "preact", M, N, true, &pz, &ldz) ||
        !c.matrix(a.v[5], "dA", ar, ac, true, &pda, &ldda) || !c.matrix(a.v[6], "dB", br, bc, true, &pdb, &lddb) ||
        !c.vector(a.v[7], "dbias", at::kFloat, N, true, &db))
      return nullptr;
    return c.done(f_epilogue_bwd(c.code, ta, tb, M, N, K, pa, lda, pb, ldb, act, pz, ldz, pd, ldd, pda, ldda, pdb, lddb,
                                 static_cast<float*>(db), c.stream));
  });
}

PyObject* py_gated(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"X", "Wg", "Wu", "H", "act", "gate", "up", "transw", "stream", "check", nullptr};
  static Names keys(names);
  Args a;
  if (!a.parse("hgemm_gated", names, keys.keys, 4, args, nargs, kwnames)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor *X = operand(a.v[0], "X"), *W = X ? operand(a.v[1], "Wg") : nullptr;
    bool tw;
    int act;
    if (!X || !W || !flag(a.v[7], &tw) || !integer(a.v[4], HGEMM_ACT_SILU, &act)) return nullptr;
    Call c{"hgemm_gated"};
    if (!c.begin(*X, "X", a.v[8], a.v[9])) return nullptr;
    const int64_t M = X->size(0), K = X->size(1), F = W->size(tw ? 0 : 1), wr = tw ? F : K, wc = tw ? K : F;
    void *px, *pg, *pu, *ph, *og, *ou;
    int64_t ldx, ldwg, ldwu, ldh, ldg, ldu;
    if (!c.matrix(a.v[0], "X", M, K, false, &px, &ldx) || !c.matrix(a.v[1], "Wg", wr, wc, false, &pg, &ldwg) ||
        !c.matrix(a.v[2], "Wu", wr, wc, false, &pu, &ldwu) || !c.matrix(a.v[3], "H", M, F, false, &ph, &ldh) ||
        !c.matrix(a.v[5], "gate", M, F, true, &og, &ldg) || !c.matrix(a.v[6], "up", M, F, true, &ou, &ldu))
      return nullptr;
    return c.done(f_gated(c.code, tw, M, F, K, px, ldx, pg, ldwg, pu, ldwu, act, ph, ldh, og, ldg, ou, ldu, c.stream));
  });
}

PyObject* py_gated_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"X", "Wg", "Wu", "gate", "up", "dH", "act", "dX", "dWg", "dWu", "transw", "stream", "check", nullptr};
  static Names keys(names);
  Args a;
  if (!a.parse("hgemm_gated_bwd", names, keys.keys, 6, args, nargs, kwnames)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor *X = operand(a.v[0], "X"), *W = X ? operand(a.v[1], "Wg") : nullptr;
    bool tw;
    int act;
    if (!X || !W || !flag(a.v[10], &tw) || !integer(a.v[6], HGEMM_ACT_SILU, &act)) return nullptr;
    Call c{"hgemm_gated_bwd"};
    if (!c.begin(*X, "X", a.v[11], a.v[12])) return nullptr;
    const int64_t M = X->size(0), K = X->size(1), F = W->size(tw ? 0 : 1), wr = tw ? F : K, wc = tw ? K : F;
    void *px, *pwg, *pwu, *pg, *pu, *pd, *dx, *dwg, *dwu;
    int64_t ldx, ldwg, ldwu, ldg, ldu, lddh, lddx, lddwg, lddwu;
    if (!c.matrix(a.v[0], "X", M, K, false, &px, &ldx) || !c.matrix(a.v[1], "Wg", wr, wc, false, &pwg, &ldwg) ||
        !c.matrix(a.v[2], "Wu", wr, wc, false, &pwu, &ldwu) || !c.matrix(a.v[3], "gate", M, F, false, &pg, &ldg) ||
        !c.matrix(a.v[4], "up", M, F, false, &pu, &ldu) || !c.matrix(a.v[5], "dH", M, F, false, &pd, &lddh) ||
        !c.matrix(a.v[7], "dX", M, K, true, &dx, &lddx) || !c.matrix(a.v[8], "dWg", wr, wc, true, &dwg, &lddwg) ||
        !c.matrix(a.v[9], "dWu", wr, wc, true, &dwu, &lddwu))
      return nullptr;
    return c.done(f_gated_bwd(c.code, tw, M, F, K, px, ldx, pwg, ldwg, pwu, ldwu, act, pg, ldg, pu, ldu, pd, lddh, dx, lddx, dwg, lddwg, dwu,
                              lddwu, c.stream));
  });
}

PyObject* py_ln_fwd(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"X", "gamma", "beta", "Y", "eps", "mean", "rstd", "stream", "check", nullptr};
  static Names keys(names);
  Args a;
  if (!a.parse("layernorm_fwd", names, keys.keys, 4, args, nargs, kwnames)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor* X = operand(a.v[0], "X");
    if (!X) return nullptr;
    Call c{"layernorm_fwd"};
    if (!c.begin(*X, "X", a.v[7], a.v[8])) return nullptr;
    double eps = 1e-5;
    if (a.v[4] && (eps = PyFloat_AsDouble(a.v[4])) == -1.0 && PyErr_Occurred()) return nullptr;
    const int64_t rows = X->size(0), cols = X->size(1);
    void *px, *py, *g, *b, *mean, *rstd;
    int64_t ldx, ldy;
    if (!c.matrix(a.v[0], "X", rows, cols, false, &px, &ldx) || !c.vector(a.v[1], "gamma", c.type, cols, true, &g) ||
        !c.vector(a.v[2], "beta", c.type, cols, true, &b) || !c.matrix(a.v[3], "Y", rows, cols, false, &py, &ldy) ||
        !c.vector(a.v[5], "mean", at::kFloat, rows, true, &mean) || !c.vector(a.v[6], "rstd", at::kFloat, rows, true, &rstd))
      return nullptr;
    return c.done(f_ln_fwd(c.code, rows, cols, px, ldx, g, b, (float)eps, py, ldy, static_cast<float*>(mean), static_cast<float*>(rstd), c.stream));
  });
}

PyObject* py_ln_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"X", "gamma", "mean", "rstd", "dY", "dX", "dgamma", "dbeta", "stream", "check", nullptr};
  static Names keys(names);
  Args a;
  if (!a.parse("layernorm_bwd", names, keys.keys, 5, args, nargs, kwnames)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor* X = operand(a.v[0], "X");
    if (!X) return nullptr;
    Call c{"layernorm_bwd"};
    if (!c.begin(*X, "X", a.v[8], a.v[9])) return nullptr;
    const int64_t rows = X->size(0), cols = X->size(1);
    void *px, *g, *mean, *rstd, *pd, *dx, *dg, *db;
    int64_t ldx, lddy, lddx;
    if (!c.matrix(a.v[0], "X", rows, cols, false, &px, &ldx) || !c.vector(a.v[1], "gamma", c.type, cols, true, &g) ||
        !c.vector(a.v[2], "mean", at::kFloat, rows, true, &mean) || !c.vector(a.v[3], "rstd", at::kFloat, rows, true, &rstd) ||
        !c.matrix(a.v[4], "dY", rows, cols, false, &pd, &lddy) || !c.matrix(a.v[5], "dX", rows, cols, true, &dx, &lddx) ||
        !c.vector(a.v[6], "dgamma", at::kFloat, cols, true, &dg) || !c.vector(a.v[7], "dbeta", at::kFloat, cols, true, &db))
      return nullptr;
    return c.done(f_ln_bwd(c.code, rows, cols, px, ldx, g, static_cast<float*>(mean), static_cast<float*>(rstd), pd, lddy, dx, lddx,
                           static_cast<float*>(dg), static_cast<float*>(db), c.stream));
  });
}

PyObject* py_rms_fwd(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"X", "gamma", "Y", "eps", "residual", "sum", "rstd", "stream", "check", nullptr};
  static Names keys(names);
  Args a;
  if (!a.parse("rmsnorm_fwd", names, keys.keys, 3, args, nargs, kwnames)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor* X = operand(a.v[0], "X");
    if (!X) return nullptr;
    Call c{"rmsnorm_fwd"};
    double eps;
    if (!c.begin(*X, "X", a.v[7], a.v[8]) || !real(a.v[3], 1e-5, &eps)) return nullptr;
    const int64_t rows = X->size(0), cols = X->size(1);
    void *px, *g, *py, *pr, *ps, *rstd;
    int64_t ldx, ldy, ldr, lds;
    if (!c.matrix(a.v[0], "X", rows, cols, false, &px, &ldx) || !c.vector(a.v[1], "gamma", c.type, cols, true, &g) ||
        !c.matrix(a.v[2], "Y", rows, cols, false, &py, &ldy) || !c.matrix(a.v[4], "residual", rows, cols, true, &pr, &ldr) ||
        !c.matrix(a.v[5], "sum", rows, cols, true, &ps, &lds) || !c.vector(a.v[6], "rstd", at::kFloat, rows, true, &rstd))
      return nullptr;
    return c.done(f_rms_fwd(c.code, rows, cols, px, ldx, pr, ldr, g, (float)eps, ps, lds, py, ldy, static_cast<float*>(rstd), c.stream));
  });
}

PyObject* py_rms_e4m3(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"X", "gamma", "Q", "scale", "eps", "residual", "sum", "rstd", "stream", "check", nullptr};
  static Names keys(names);
  Args a;
  if (!a.parse("rmsnorm_fwd_e4m3", names, keys.keys, 4, args, nargs, kwnames)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor* X = operand(a.v[0], "X");
    if (!X) return nullptr;
    Call c{"rmsnorm_fwd_e4m3"};
    double eps;
    if (!c.begin(*X, "X", a.v[8], a.v[9]) || !real(a.v[4], 1e-5, &eps)) return nullptr;
    const int64_t rows = X->size(0), cols = X->size(1);
    void *px, *g, *pq, *scale, *pr, *ps, *rstd;
    int64_t ldx, ldq, ldr, lds;
    if (!c.matrix(a.v[0], "X", rows, cols, false, &px, &ldx) || !c.vector(a.v[1], "gamma", c.type, cols, true, &g) ||
        !c.matrix8(a.v[2], "Q", rows, cols, &pq, &ldq) || !c.vector(a.v[3], "scale", at::kFloat, rows, false, &scale) ||
        !c.matrix(a.v[5], "residual", rows, cols, true, &pr, &ldr) || !c.matrix(a.v[6], "sum", rows, cols, true, &ps, &lds) ||
        !c.vector(a.v[7], "rstd", at::kFloat, rows, true, &rstd))
      return nullptr;
    return c.done(f_rms_e4m3(c.code, rows, cols, px, ldx, pr, ldr, g, (float)eps, ps, lds, pq, ldq, static_cast<float*>(scale),
                             static_cast<float*>(rstd), c.stream));
  });
}

PyObject* py_rows_e4m3(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"X", "Q", "scale", "stream", "check", nullptr};
  static Names keys(names);
  Args a;
  if (!a.parse("quantize_rows_e4m3", names, keys.keys, 3, args, nargs, kwnames)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor* X = operand(a.v[0], "X");
    if (!X) return nullptr;
    Call c{"quantize_rows_e4m3"};
    if (!c.begin(*X, "X", a.v[3], a.v[4])) return nullptr;
    const int64_t rows = X->size(0), cols = X->size(1);
    void *px, *pq, *scale;
    int64_t ldx, ldq;
    if (!c.matrix(a.v[0], "X", rows, cols, false, &px, &ldx) || !c.matrix8(a.v[1], "Q", rows, cols, &pq, &ldq) ||
        !c.vector(a.v[2], "scale", at::kFloat, rows, false, &scale))
      return nullptr;
    return c.done(f_rows_e4m3(c.code, rows, cols, px, ldx, pq, ldq, static_cast<float*>(scale), c.stream));
  });
}

PyObject* py_rms_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"S", "gamma", "rstd", "dY", "dsum", "dX", "dgamma", "stream", "check", nullptr};
  static Names keys(names);
  Args a;
  if (!a.parse("rmsnorm_bwd", names, keys.keys, 4, args, nargs, kwnames)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor* S = operand(a.v[0], "S");
    if (!S) return nullptr;
    Call c{"rmsnorm_bwd"};
    if (!c.begin(*S, "S", a.v[7], a.v[8])) return nullptr;
    const int64_t rows = S->size(0), cols = S->size(1);
    void *ps, *g, *rstd, *pd, *pr, *dx, *dg;
    int64_t lds, lddy, ldds, lddx;
    if (!c.matrix(a.v[0], "S", rows, cols, false, &ps, &lds) || !c.vector(a.v[1], "gamma", c.type, cols, true, &g) ||
        !c.vector(a.v[2], "rstd", at::kFloat, rows, true, &rstd) || !c.matrix(a.v[3], "dY", rows, cols, false, &pd, &lddy) ||
        !c.matrix(a.v[4], "dsum", rows, cols, true, &pr, &ldds) || !c.matrix(a.v[5], "dX", rows, cols, true, &dx, &lddx) ||
        !c.vector(a.v[6], "dgamma", at::kFloat, cols, true, &dg))
      return nullptr;
    return c.done(f_rms_bwd(c.code, rows, cols, ps, lds, g, static_cast<float*>(rstd), pd, lddy, pr, ldds, dx, lddx, static_cast<float*>(dg),
                            c.stream));
  });
}

// The device address of dropout's counter of uses: one int64 value, or None.
bool counter(const Call& c, PyObject* o, int64_t** ptr) {
  *ptr = nullptr;
  const at::Tensor* x = tensor(o, "step", true);
  if (!x) return !PyErr_Occurred();
  if (x->scalar_type() != at::kLong || x->numel() != 1) {
    PyErr_SetString(PyExc_TypeError, "step: need a tensor of one int64 value");
    return false;
  }
  if (!c.on_device(*x, "step")) return false;
  *ptr = static_cast<int64_t*>(x->data_ptr());
  return true;
}

PyObject* py_drop_fwd(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"X", "Y", "p", "seed", "offset", "residual", "step", "stream", "check", nullptr};
  static Names keys(names);
  Args a;
  if (!a.parse("dropout_fwd", names, keys.keys, 4, args, nargs, kwnames)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor* X = operand(a.v[0], "X");
    if (!X) return nullptr;
    Call c{"dropout_fwd"};
    double p;
    uint64_t seed, offset;
    if (!c.begin(*X, "X", a.v[7], a.v[8]) || !real(a.v[2], 0.0, &p) || !word64(a.v[3], &seed) || !word64(a.v[4], &offset)) return nullptr;
    const int64_t rows = X->size(0), cols = X->size(1);
    void *px, *py, *pr;
    int64_t ldx, ldy, ldr, *step;
    if (!c.matrix(a.v[0], "X", rows, cols, false, &px, &ldx) || !c.matrix(a.v[1], "Y", rows, cols, false, &py, &ldy) ||
        !c.matrix(a.v[5], "residual", rows, cols, true, &pr, &ldr) || !counter(c, a.v[6], &step))
      return nullptr;
    return c.done(f_drop_fwd(c.code, rows, cols, px, ldx, pr, ldr, p, seed, offset, step, py, ldy, c.stream));
  });
}

PyObject* py_drop_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"dY", "dX", "p", "seed", "offset", "step", "stream", "check", nullptr};
  static Names keys(names);
  Args a;
  if (!a.parse("dropout_bwd", names, keys.keys, 4, args, nargs, kwnames)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor* D = operand(a.v[0], "dY");
    if (!D) return nullptr;
    Call c{"dropout_bwd"};
    double p;
    uint64_t seed, offset;
    if (!c.begin(*D, "dY", a.v[6], a.v[7]) || !real(a.v[2], 0.0, &p) || !word64(a.v[3], &seed) || !word64(a.v[4], &offset)) return nullptr;
    const int64_t rows = D->size(0), cols = D->size(1);
    void *pd, *px;
    int64_t ldd, ldx, *step;
    if (!c.matrix(a.v[0], "dY", rows, cols, false, &pd, &ldd) || !c.matrix(a.v[1], "dX", rows, cols, false, &px, &ldx) ||
        !counter(c, a.v[5], &step))
      return nullptr;
    return c.done(f_drop_bwd(c.code, rows, cols, pd, ldd, p, seed, offset, step, px, ldx, c.stream));
  });
}

PyObject* py_q_epilogue(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"A", "B", "D", "a_scale", "b_scale", "bias", "act", "residual", "preact", "stream", "check", nullptr};
  static Names keys(names);
  Args a;
  if (!a.parse("qgemm_epilogue", names, keys.keys, 3, args, nargs, kwnames)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor *A = operand(a.v[0], "A"), *B = A ? operand(a.v[1], "B") : nullptr, *D = B ? operand(a.v[2], "D") : nullptr;
    int act;
    if (!D || !integer(a.v[6], HGEMM_ACT_NONE, &act)) return nullptr;
    Call c{"qgemm_epilogue"};
    c.others = "the type of the output";
    if (!c.begin(*D, "D", a.v[9], a.v[10])) return nullptr;
    const int64_t M = A->size(0), K = A->size(1), N = B->size(0);
    void *pa, *pb, *pd, *pr, *pz, *sa, *sb, *bias;
    int64_t lda, ldb, ldd, ldr, ldz;
    if (!c.matrix8(a.v[0], "A", M, K, &pa, &lda) || !c.matrix8(a.v[1], "B", N, K, &pb, &ldb) || !c.matrix(a.v[2], "D", M, N, false, &pd, &ldd) ||
        !c.vector(a.v[3], "a_scale", at::kFloat, M, true, &sa) || !c.vector(a.v[4], "b_scale", at::kFloat, N, true, &sb) ||
        !c.vector(a.v[5], "bias", c.type, N, true, &bias) || !c.matrix(a.v[7], "residual", M, N, true, &pr, &ldr) ||
        !c.matrix(a.v[8], "preact", M, N, true, &pz, &ldz))
      return nullptr;
    return c.done(f_q_epilogue(c.code, M, N, K, pa, lda, static_cast<float*>(sa), pb, ldb, static_cast<float*>(sb), bias, act, pr, ldr, pd, ldd,
                               pz, ldz, c.stream));
  });
}

PyObject* py_q_gated(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"X", "Wg", "Wu", "H", "x_scale", "g_scale", "u_scale", "act", "gate", "up", "stream", "check", nullptr};
  static Names keys(names);
  Args a;
  if (!a.parse("qgemm_gated", names, keys.keys, 4, args, nargs, kwnames)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor *X = operand(a.v[0], "X"), *W = X ? operand(a.v[1], "Wg") : nullptr, *H = W ? operand(a.v[3], "H") : nullptr;
    int act;
    if (!H || !integer(a.v[7], HGEMM_ACT_SILU, &act)) return nullptr;
    Call c{"qgemm_gated"};
    c.others = "the type of the output";
    if (!c.begin(*H, "H", a.v[10], a.v[11])) return nullptr;
    const int64_t M = X->size(0), K = X->size(1), F = W->size(0);
    void *px, *pg, *pu, *ph, *og, *ou, *sx, *sg, *su;
    int64_t ldx, ldwg, ldwu, ldh, ldg, ldu;
    if (!c.matrix8(a.v[0], "X", M, K, &px, &ldx) || !c.matrix8(a.v[1], "Wg", F, K, &pg, &ldwg) || !c.matrix8(a.v[2], "Wu", F, K, &pu, &ldwu) ||
        !c.matrix(a.v[3], "H", M, F, false, &ph, &ldh) || !c.vector(a.v[4], "x_scale", at::kFloat, M, true, &sx) ||
        !c.vector(a.v[5], "g_scale", at::kFloat, F, true, &sg) || !c.vector(a.v[6], "u_scale", at::kFloat, F, true, &su) ||
        !c.matrix(a.v[8], "gate", M, F, true, &og, &ldg) || !c.matrix(a.v[9], "up", M, F, true, &ou, &ldu))
      return nullptr;
    return c.done(f_q_gated(c.code, M, F, K, px, ldx, static_cast<float*>(sx), pg, ldwg, static_cast<float*>(sg), pu, ldwu,
                            static_cast<float*>(su), act, ph, ldh, og, ldg, ou, ldu, c.stream));
  });
}

// connect(addresses of the C functions in this order, error function)
PyObject* py_connect(PyObject*, PyObject* args) {
  void** const slots[] = {reinterpret_cast<void**>(&f_epilogue),  reinterpret_cast<void**>(&f_epilogue_bwd), reinterpret_cast<void**>(&f_gated),
                          reinterpret_cast<void**>(&f_gated_bwd), reinterpret_cast<void**>(&f_ln_fwd),       reinterpret_cast<void**>(&f_ln_bwd),
                          reinterpret_cast<void**>(&f_rms_fwd),   reinterpret_cast<void**>(&f_rms_e4m3),     reinterpret_cast<void**>(&f_rows_e4m3),
                          reinterpret_cast<void**>(&f_rms_bwd),   reinterpret_cast<void**>(&f_drop_fwd),     reinterpret_cast<void**>(&f_drop_bwd),
                          reinterpret_cast<void**>(&f_q_epilogue), reinterpret_cast<void**>(&f_q_gated)};
  constexpr Py_ssize_t n = sizeof(slots) / sizeof(slots[0]);
  if (PyTuple_GET_SIZE(args) != n + 1) {
    PyErr_Format(PyExc_TypeError, "connect: takes %zd addresses and a function", n);
    return nullptr;
  }
  void* p[n];
  for (Py_ssize_t i = 0; i < n; ++i) {
    p[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(args, i));
    if (PyErr_Occurred()) return nullptr;
  }
  for (Py_ssize_t i = 0; i < n; ++i) *slots[i] = p[i];
  PyObject* handler = PyTuple_GET_ITEM(args, n);
  Py_INCREF(handler);
  Py_XSETREF(on_error, handler);
  Py_RETURN_NONE;
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL | METH_KEYWORDS

PyMethodDef methods[] = {
    {"hgemm_epilogue", FAST(py_epilogue),
     "hgemm_epilogue(A, B, D, bias=None, act=0, residual=None, preact=None, transa=False, transb=False, stream=None, check=True)\n--\n\n"
     "``Z = op(A) @ op(B) + bias``, ``D = act(Z) + residual`` on the current CUDA device, asynchronously.\n\n"
     "``A``, ``B``, ``D`` and the optional ``bias`` (N), ``residual`` and ``preact`` (M x N; receives ``Z``) are CUDA tensors of\n"
     "one type, ``float16`` or ``bfloat16``; matrices have unit column stride. ``A`` and ``B`` are passed as stored (K x M\n"
     "when ``transa``, N x K when ``transb``). ``residual`` may be ``D``. ``act``: ``HGEMM_ACT_*``. Sums are binary32 and each\n"
     "output is rounded once. ``stream``: a ``torch.cuda.Stream``, a raw ``cudaStream_t`` integer, or ``None`` for torch's\n"
     "current stream. Returns the status; raises ``DgemmError`` on a negative one unless ``check=False``."},
    {"hgemm_epilogue_bwd", FAST(py_epilogue_bwd),
     "hgemm_epilogue_bwd(A, B, dD, act=0, preact=None, dA=None, dB=None, dbias=None, transa=False, transb=False, stream=None, check=True)\n--\n\n"
     "Gradients of :func:`hgemm_epilogue` for the incoming ``dD``: ``dA`` and ``dB`` (stored as ``A`` and ``B`` are) and\n"
     "``dbias`` (N, ``float32``), each written if given. ``preact`` is the forward pass's and may be ``None`` for\n"
     "``HGEMM_ACT_NONE``. The residual's gradient is ``dD`` itself."},
    {"hgemm_gated", FAST(py_gated),
     "hgemm_gated(X, Wg, Wu, H, act=4, gate=None, up=None, transw=False, stream=None, check=True)\n--\n\n"
     "Gated projections ``H = act(X @ op(Wg)) * (X @ op(Wu))`` in one kernel, asynchronously.\n\n"
     "``X`` (M x K), ``Wg`` and ``Wu`` (K x F, or F x K when ``transw``), ``H`` (M x F): CUDA tensors of one type, ``float16`` or\n"
     "``bfloat16``. ``gate`` and ``up`` (both or neither) receive the two products, which :func:`hgemm_gated_bwd` needs."},
    {"hgemm_gated_bwd", FAST(py_gated_bwd),
     "hgemm_gated_bwd(X, Wg, Wu, gate, up, dH, act=4, dX=None, dWg=None, dWu=None, transw=False, stream=None, check=True)\n--\n\n"
     "Gradients of :func:`hgemm_gated` for the incoming ``dH`` (M x F): ``dX``, ``dWg`` and ``dWu`` (stored as ``Wg`` and\n"
     "``Wu`` are), each written if given."},
    {"layernorm_fwd", FAST(py_ln_fwd),
     "layernorm_fwd(X, gamma, beta, Y, eps=1e-05, mean=None, rstd=None, stream=None, check=True)\n--\n\n"
     "``Y = (X - mean) * rstd * gamma + beta`` over the rows of ``X``, asynchronously.\n\n"
     "``X``, ``Y`` (rows x cols) and ``gamma``, ``beta`` (cols, each may be ``None``): CUDA tensors of one type, ``float32``,\n"
     "``float16`` or ``bfloat16``. ``mean`` and ``rstd`` (rows, ``float32``) are written if given."},
    {"layernorm_bwd", FAST(py_ln_bwd),
     "layernorm_bwd(X, gamma, mean, rstd, dY, dX=None, dgamma=None, dbeta=None, stream=None, check=True)\n--\n\n"
     "Gradients of :func:`layernorm_fwd` for the incoming ``dY``: ``dX`` (type of ``X``), ``dgamma`` and ``dbeta`` (cols,\n"
     "``float32``), each written if given. ``mean`` and ``rstd`` are the forward pass's."},
    {"rmsnorm_fwd", FAST(py_rms_fwd),
     "rmsnorm_fwd(X, gamma, Y, eps=1e-05, residual=None, sum=None, rstd=None, stream=None, check=True)\n--\n\n"
     "``s = X + residual``, ``Y = s * rstd * gamma`` over the rows, ``rstd = 1 / sqrt(mean(s^2) + eps)``, asynchronously.\n\n"
     "``X``, ``Y``, ``residual``, ``sum`` (rows x cols) and ``gamma`` (cols, or ``None``): CUDA tensors of one type, ``float32``,\n"
     "``float16`` or ``bfloat16``. ``sum`` (receives ``s``; it may be ``X`` or ``residual`` itself) and ``rstd`` (rows, ``float32``)\n"
     "are written if given. ``Y`` and ``rstd`` are computed from ``s`` before it is rounded."},
    {"rmsnorm_fwd_e4m3", FAST(py_rms_e4m3),
     "rmsnorm_fwd_e4m3(X, gamma, Q, scale, eps=1e-05, residual=None, sum=None, rstd=None, stream=None, check=True)\n--\n\n"
     ":func:`rmsnorm_fwd` with its output in 8 bits: ``scale = max(max|y|, 2^-100) / 448`` for each row (``float32``) and ``Q``\n"
     "(rows x cols, ``float8_e4m3fn``) the nearest values to ``y / scale``."},
    {"quantize_rows_e4m3", FAST(py_rows_e4m3),
     "quantize_rows_e4m3(X, Q, scale, stream=None, check=True)\n--\n\n"
     "The rows of ``X`` in 8 bits, as :func:`rmsnorm_fwd_e4m3` brings its output there."},
    {"rmsnorm_bwd", FAST(py_rms_bwd),
     "rmsnorm_bwd(S, gamma, rstd, dY, dsum=None, dX=None, dgamma=None, stream=None, check=True)\n--\n\n"
     "Gradients of :func:`rmsnorm_fwd` for the incoming ``dY`` and, where the sum goes on, ``dsum``: ``dX`` (of ``X`` and of the\n"
     "residual; it may be ``dsum`` itself) and ``dgamma`` (cols, ``float32``), each written if given. ``S`` is the forward pass's sum\n"
     "(``X`` where there was no residual), ``rstd`` its statistics."},
    {"dropout_fwd", FAST(py_drop_fwd),
     "dropout_fwd(X, Y, p, seed, offset=0, residual=None, step=None, stream=None, check=True)\n--\n\n"
     "``Y = residual + (keep ? X / (1 - p) : 0)``, asynchronously, with a mask that is a function of ``seed`` and ``offset`` (64 bits each),\n"
     "row and column, and is never stored.\n\n"
     "``X``, ``Y``, ``residual`` (rows x cols): CUDA tensors of one type, ``float32``, ``float16`` or ``bfloat16``; ``Y`` may be ``X`` or\n"
     "``residual`` itself. ``step``: a CUDA tensor of one ``int64`` value that is added to ``offset`` when the kernel runs, so that a\n"
     "captured call can have another mask in each replay."},
    {"dropout_bwd", FAST(py_drop_bwd),
     "dropout_bwd(dY, dX, p, seed, offset=0, step=None, stream=None, check=True)\n--\n\n"
     "The gradient of :func:`dropout_fwd` with the same ``p``, ``seed``, ``offset`` and ``step``: ``dX = keep ? dY / (1 - p) : 0``. ``dX`` may\n"
     "be ``dY`` itself. (The residual's gradient is ``dY``.)"},
    {"qgemm_epilogue", FAST(py_q_epilogue),
     "qgemm_epilogue(A, B, D, a_scale=None, b_scale=None, bias=None, act=0, residual=None, preact=None, stream=None, check=True)\n--\n\n"
     "``Z = a_scale[:, None] * b_scale * (A @ B.T) + bias``, ``D = act(Z) + residual`` with operands of 8 bits, asynchronously.\n\n"
     "``A`` (M x K) and ``B`` (N x K): CUDA tensors of ``float8_e4m3fn``; ``a_scale`` (M) and ``b_scale`` (N): ``float32``, ones if not\n"
     "given; ``D`` and the optional ``bias``, ``residual`` and ``preact`` as in :func:`hgemm_epilogue`."},
    {"qgemm_gated", FAST(py_q_gated),
     "qgemm_gated(X, Wg, Wu, H, x_scale=None, g_scale=None, u_scale=None, act=4, gate=None, up=None, stream=None, check=True)\n--\n\n"
     "Gated projections of 8-bit operands: ``H = act(G) * U`` with ``G = x_scale[:, None] * g_scale * (X @ Wg.T)`` and ``U`` alike.\n\n"
     "``X`` (M x K), ``Wg`` and ``Wu`` (F x K): CUDA tensors of ``float8_e4m3fn``; scales ``float32``; ``H`` and the optional ``gate`` and\n"
     "``up`` (both or neither) as in :func:`hgemm_gated`."},
    {"connect", py_connect, METH_VARARGS, "Addresses of the C functions and the function that raises on an error status."},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Compiled argument marshalling of libdgemm's 16-bit and 8-bit products, norms and dropout.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }

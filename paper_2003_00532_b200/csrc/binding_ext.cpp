// Compiled argument marshalling of the 16-bit products and layer norm: the Python names of
// include/hgemm.h and include/layernorm.h as builtins that unpack torch tensors, check shapes, types,
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

#include "../../include/hgemm.h"
#include "../../include/layernorm.h"

namespace {

decltype(&hgemm_epilogue) f_epilogue = nullptr;
decltype(&hgemm_epilogue_bwd) f_epilogue_bwd = nullptr;
decltype(&hgemm_gated) f_gated = nullptr;
decltype(&hgemm_gated_bwd) f_gated_bwd = nullptr;
decltype(&layernorm_fwd) f_ln_fwd = nullptr;
decltype(&layernorm_bwd) f_ln_bwd = nullptr;
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
    *ptr = nullptr;
    *ld = cols > 0 ? cols : 1;
    const at::Tensor* x = tensor(o, name, optional);
    if (!x) return !PyErr_Occurred();
    if (x->scalar_type() != type || x->dim() != 2) {
      PyErr_Format(PyExc_TypeError, "%s: need a 2-D tensor of the type of the first operand", name);
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
      PyErr_Format(PyExc_TypeError, "%s: need a 1-D tensor of %s", name, t == at::kFloat ? "float32" : "the type of the first operand");
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

// connect(addresses of the six C functions in the order below, error function)
PyObject* py_connect(PyObject*, PyObject* args) {
  unsigned long long p[6];
  PyObject* handler;
  if (!PyArg_ParseTuple(args, "KKKKKKO", &p[0], &p[1], &p[2], &p[3], &p[4], &p[5], &handler)) return nullptr;
  f_epilogue = reinterpret_cast<decltype(f_epilogue)>(p[0]);
  f_epilogue_bwd = reinterpret_cast<decltype(f_epilogue_bwd)>(p[1]);
  f_gated = reinterpret_cast<decltype(f_gated)>(p[2]);
  f_gated_bwd = reinterpret_cast<decltype(f_gated_bwd)>(p[3]);
  f_ln_fwd = reinterpret_cast<decltype(f_ln_fwd)>(p[4]);
  f_ln_bwd = reinterpret_cast<decltype(f_ln_bwd)>(p[5]);
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
    {"connect", py_connect, METH_VARARGS, "Addresses of the C functions and the function that raises on an error status."},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Compiled argument marshalling of libdgemm's 16-bit products and layer norm.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }

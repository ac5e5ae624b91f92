// Argument marshalling of the library's short calls (ratio / accept, resampling, mixtures) for Python.  Each of them is one
// kernel of a few microseconds, and through ctypes the binding itself - one Python call per tensor for the contiguity check
// and one for the address, then a conversion per argument - took longer than the launch (measured at 64 sequences:
// csd_accept_scan 5.3 us of host time, 2.4 us of it in the library).  Here a tensor costs a type check and two field reads.
// No arithmetic and no policy: pointers and sizes go to the C ABI as they are, the status code comes back.  The calls of categorical
// heads and 8-bit matrices take strided views and several types; for those the tensors' types, sizes and device are checked here,
// since the C ABI sees addresses only.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <exception>
#include <stdexcept>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/csd.h"

namespace {

PyObject* g_ptr_of = nullptr;   // the binding's address function for anything that is not a tensor (NumPy arrays)

struct Args {
  PyObject* const* a;
  bool ok = true;
  template <typename T> T* ptr(PyObject* o) {
    if (!ok || o == Py_None) return nullptr;
    if (THPVariable_Check(o)) {
      // a tensor without strides or storage (nested, sparse, vmapped) throws: that stays a Python error
      try {
        const at::Tensor& t = THPVariable_Unpack(o);
        if (t.is_contiguous()) return static_cast<T*>(t.data_ptr());
        PyErr_SetString(PyExc_AssertionError, "tensor must be contiguous");
      } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
      }
      ok = false;
      return nullptr;
    }
    PyObject* r = PyObject_CallOneArg(g_ptr_of, o);
    void* v = r ? PyLong_AsVoidPtr(r) : nullptr;
    Py_XDECREF(r);
    if (PyErr_Occurred()) ok = false;
    return static_cast<T*>(v);
  }
  template <typename T> T* p(int i) { return ptr<T>(a[i]); }
  int n(int i) {
    const long v = ok ? PyLong_AsLong(a[i]) : 0;
    if (v == -1 && PyErr_Occurred()) ok = false;
    if (v != static_cast<int>(v)) { if (ok) PyErr_SetString(PyExc_OverflowError, "size exceeds a C int"); ok = false; }
    return static_cast<int>(v);
  }
  double d(int i) {
    const double v = ok ? PyFloat_AsDouble(a[i]) : 0.0;
    if (v == -1.0 && PyErr_Occurred()) ok = false;
    return v;
  }
  csd_ctx* ctx() {
    csd_ctx* c = ok ? static_cast<csd_ctx*>(PyLong_AsVoidPtr(a[0])) : nullptr;
    if (PyErr_Occurred()) ok = false;
    return c;
  }
  // (logw [rows, K], mu [rows, K, C], log_sigma [rows, K, C])
  csd_gmm gmm(int i) {
    csd_gmm m{};
    PyObject* s = ok ? PySequence_Fast(a[i], "a mixture is (logw, mu, log_sigma)") : nullptr;
    if (!s) { ok = false; return m; }
    if (PySequence_Fast_GET_SIZE(s) != 3) {
      PyErr_SetString(PyExc_ValueError, "a mixture is (logw, mu, log_sigma)");
      ok = false;
    } else {
      PyObject** it = PySequence_Fast_ITEMS(s);
      m.logw = ptr<const float>(it[0]); m.mu = ptr<const float>(it[1]); m.log_sigma = ptr<const float>(it[2]);
      if (ok) {
        PyObject* sh = PyObject_GetAttrString(it[0], "shape");
        PyObject* k = sh ? PySequence_GetItem(sh, 1) : nullptr;
        m.K = k ? static_cast<int>(PyLong_AsLong(k)) : 0;
        Py_XDECREF(k); Py_XDECREF(sh);
        if (PyErr_Occurred()) ok = false;
      }
    }
    Py_DECREF(s);
    return m;
  }

  // ---- calls that check their tensors: argument 1 is the context's device
  int device = -1;
  const at::Tensor* tensor(PyObject* o, const char* name, bool optional = false) {
    if (!ok || (optional && o == Py_None)) return nullptr;
    if (!THPVariable_Check(o)) { PyErr_Format(PyExc_TypeError, "%s must be a tensor", name); ok = false; return nullptr; }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != device) {
      PyErr_Format(PyExc_ValueError, "%s must be on cuda:%d, the context's device", name, device);
      ok = false;
      return nullptr;
    }
    return &t;
  }
  template <typename F> void guarded(F f) {
    if (!ok) return;
    try { f(); } catch (const std::exception& e) { PyErr_SetString(PyExc_ValueError, e.what()); ok = false; }
  }
  static int dtype_of(const at::Tensor& t, const char* name) {
    switch (t.scalar_type()) {
      case at::kFloat: return CSD_F32;
      case at::kBFloat16: return CSD_BF16;
      case at::kHalf: return CSD_F16;
      default: throw std::runtime_error(std::string(name) + " must be float32, bfloat16 or float16");
    }
  }
  // a dense array of at least n elements of the given type
  template <typename T> T* dense(PyObject* o, const char* name, at::ScalarType type, int64_t n, bool optional = false) {
    const at::Tensor* t = tensor(o, name, optional);
    T* p = nullptr;
    if (t) guarded([&] {
      const bool u32 = type == at::kInt && t->scalar_type() == at::kUInt32;   // masks may be either
      if (t->scalar_type() != type && !u32) throw std::runtime_error(std::string(name) + " must be " + at::toString(type));
      if (!t->is_contiguous() || t->numel() < n) throw std::runtime_error(std::string(name) + " must be contiguous with at least " + std::to_string(n) + " elements");
      p = static_cast<T*>(t->data_ptr());
    });
    return p;
  }
  // rows of `cols` adjacent elements, any row stride: [rows or more, cols] (or contiguous with that many rows in its leading dimensions)
  void* rows_of(PyObject* o, const char* name, int64_t rows, int64_t cols, int* dtype, int64_t* ld, bool optional = false) {
    const at::Tensor* t = tensor(o, name, optional);
    void* p = nullptr;
    *ld = cols;
    if (t) guarded([&] {
      const int d = dtype_of(*t, name);
      if (*dtype >= 0 && d != *dtype) throw std::runtime_error(std::string(name) + " has another type than the arrays beside it");
      *dtype = d;
      if (t->dim() < 1 || t->size(-1) != cols) throw std::runtime_error(std::string(name) + " must have rows of " + std::to_string(cols) + " elements");
      if (t->dim() == 2) {
        if (t->size(0) < rows) throw std::runtime_error(std::string(name) + " must have " + std::to_string(rows) + " rows");
        if (cols > 1 && t->stride(1) != 1) throw std::runtime_error(std::string(name) + " must have adjacent elements along its rows");
        if (rows > 1) *ld = t->stride(0);
      } else if (!t->is_contiguous() || t->numel() < rows * cols) {
        throw std::runtime_error(std::string(name) + " must be two-dimensional, or contiguous with " + std::to_string(rows) + " rows");
      }
      p = t->data_ptr();
    });
    return p;
  }
  csd_logits logits(PyObject* o, const char* name, int64_t rows, int64_t V) {
    csd_logits l{};
    l.dtype = -1;
    l.data = rows_of(o, name, rows, V, &l.dtype, &l.ld);
    return l;
  }
  PyObject* item(PyObject* s, Py_ssize_t i, Py_ssize_t n, const char* what) {   // borrowed
    if (!ok) return nullptr;
    if (!PyTuple_Check(s) || PyTuple_GET_SIZE(s) != n) { PyErr_Format(PyExc_TypeError, "%s", what); ok = false; return nullptr; }
    return PyTuple_GET_ITEM(s, i);
  }
  // (temperature, top_k, top_p, min_p), each a tensor of one value a row or None; None: all off
  csd_cat_params cat_params(PyObject* o, int64_t rows) {
    csd_cat_params f{};
    if (!ok || o == Py_None) return f;
    const char* what = "parameters are a tuple (temperature, top_k, top_p, min_p)";
    if (!item(o, 0, 4, what)) return f;
    f.temperature = dense<const float>(PyTuple_GET_ITEM(o, 0), "temperature", at::kFloat, rows, true);
    f.top_k = dense<const int32_t>(PyTuple_GET_ITEM(o, 1), "top_k", at::kInt, rows, true);
    f.top_p = dense<const float>(PyTuple_GET_ITEM(o, 2), "top_p", at::kFloat, rows, true);
    f.min_p = dense<const float>(PyTuple_GET_ITEM(o, 3), "min_p", at::kFloat, rows, true);
    return f;
  }
  // (data, scale) of an 8-bit matrix [rows, K]
  csd_quant quant(PyObject* o, const char* name, int64_t rows, int K) {
    csd_quant q{};
    if (!item(o, 0, 2, "an 8-bit matrix is a tuple (data, scale)")) return q;
    int ld = 0, ls = 0;
    if (csd_quant_pitch(K, &ld, &ls) != CSD_OK) return q;   // (the call refuses K)
    q.data = dense<uint8_t>(PyTuple_GET_ITEM(o, 0), name, at::kByte, rows * ld);
    q.scale = dense<uint8_t>(PyTuple_GET_ITEM(o, 1), name, at::kByte, rows * ls);
    return q;
  }
};

bool count_is(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
  return false;
}

#define CSD_MARSHAL(NAME, COUNT, ...)                                                 \
  PyObject* NAME(PyObject*, PyObject* const* args, Py_ssize_t nargs) {                 \
    if (!count_is(nargs, COUNT)) return nullptr;                                       \
    Args x{args};                                                                      \
    csd_ctx* ctx = x.ctx();                                                            \
    int rc = CSD_OK;                                                                   \
    __VA_ARGS__                                                                               \
    return x.ok ? PyLong_FromLong(rc) : nullptr;                                       \
  }
#define CSD_RUN(EXPR) if (x.ok) { Py_BEGIN_ALLOW_THREADS rc = (EXPR); Py_END_ALLOW_THREADS }

CSD_MARSHAL(accept_scan, 14, {
  const int B = x.n(1), gamma = x.n(2), C = x.n(3);
  const double ls = x.d(4), sp = x.d(5), sq = x.d(6);
  const float *x0 = x.p<const float>(7), *mq = x.p<const float>(8), *mp = x.p<const float>(9), *u = x.p<const float>(10);
  float* lr = x.p<float>(11);
  int32_t* na = x.p<int32_t>(12);
  uint32_t* mask = x.p<uint32_t>(13);
  CSD_RUN(csd_accept_scan(ctx, B, gamma, C, ls, static_cast<float>(sp), static_cast<float>(sq), x0, mq, mp, u, lr, na, mask))
})

CSD_MARSHAL(resample, 17, {
  const int B = x.n(1), gamma = x.n(2), C = x.n(3), cap = x.n(4);
  const double ls = x.d(5), sp = x.d(6), sq = x.d(7);
  const int32_t* na = x.p<const int32_t>(8);
  const float *mp = x.p<const float>(9), *mq = x.p<const float>(10), *xi = x.p<const float>(11), *v = x.p<const float>(12);
  float* xn = x.p<float>(13);
  int32_t* np = x.p<int32_t>(14);
  uint32_t* fl = x.p<uint32_t>(15);
  int32_t* ch = x.p<int32_t>(16);
  CSD_RUN(csd_resample(ctx, B, gamma, C, cap, ls, static_cast<float>(sp), static_cast<float>(sq), na, mp, mq, xi, v, xn, np, fl, ch))
})

CSD_MARSHAL(resample_lv, 17, {
  const int B = x.n(1), gamma = x.n(2), C = x.n(3), cap = x.n(4);
  const float* ls = x.p<const float>(5);
  const int32_t* na = x.p<const int32_t>(6);
  const float *mp = x.p<const float>(7), *lp = x.p<const float>(8), *mq = x.p<const float>(9), *lq = x.p<const float>(10),
              *xi = x.p<const float>(11), *v = x.p<const float>(12);
  float* xn = x.p<float>(13);
  int32_t* np = x.p<int32_t>(14);
  uint32_t* fl = x.p<uint32_t>(15);
  int32_t* ch = x.p<int32_t>(16);
  CSD_RUN(csd_resample_lv(ctx, B, gamma, C, cap, ls, na, mp, lp, mq, lq, xi, v, xn, np, fl, ch))
})

CSD_MARSHAL(gmm_draft_sample, 8, {
  const int R = x.n(1), C = x.n(2);
  const csd_gmm q = x.gmm(3);
  const float *u = x.p<const float>(4), *nz = x.p<const float>(5);
  float* xo = x.p<float>(6);
  int32_t* comp = x.p<int32_t>(7);
  CSD_RUN(csd_gmm_draft_sample(ctx, R, C, &q, u, nz, xo, comp))
})

CSD_MARSHAL(gmm_verify, 11, {
  const int B = x.n(1), gamma = x.n(2), C = x.n(3);
  const csd_gmm q = x.gmm(4), p = x.gmm(5);
  const float *xi = x.p<const float>(6), *u = x.p<const float>(7);
  float* lr = x.p<float>(8);
  int32_t* na = x.p<int32_t>(9);
  uint32_t* mask = x.p<uint32_t>(10);
  CSD_RUN(csd_gmm_verify(ctx, B, gamma, C, &q, &p, xi, u, lr, na, mask))
})

CSD_MARSHAL(gmm_resample, 15, {
  const int B = x.n(1), gamma = x.n(2), C = x.n(3), cap = x.n(4);
  const csd_gmm q = x.gmm(5), p = x.gmm(6);
  const int32_t* na = x.p<const int32_t>(7);
  const float *w = x.p<const float>(8), *xi = x.p<const float>(9), *v = x.p<const float>(10);
  float* xn = x.p<float>(11);
  int32_t* np = x.p<int32_t>(12);
  uint32_t* fl = x.p<uint32_t>(13);
  int32_t* ch = x.p<int32_t>(14);
  CSD_RUN(csd_gmm_resample(ctx, B, gamma, C, cap, &q, &p, na, w, xi, v, xn, np, fl, ch))
})

// (context, device, ...)
#define CSD_DEVICE_OF const int64_t dv = x.n(1); x.device = static_cast<int>(dv);

CSD_MARSHAL(cat_filter, 7, {
  CSD_DEVICE_OF
  const int R = x.n(2), V = x.n(3);
  const csd_logits l = x.logits(args[4], "logits", R, V);
  const csd_cat_params f = x.cat_params(args[5], R);
  double* dist = x.dense<double>(args[6], "dist", at::kDouble, 5 * static_cast<int64_t>(R));
  CSD_RUN(csd_cat_filter(ctx, R, V, &l, &f, dist))
})

CSD_MARSHAL(cat_draft_sample, 10, {
  CSD_DEVICE_OF
  const int R = x.n(2), V = x.n(3);
  const csd_logits l = x.logits(args[4], "logits", R, V);
  const csd_cat_params f = x.cat_params(args[5], R);
  const float* u = x.dense<const float>(args[6], "u", at::kFloat, R);
  int32_t* token = x.dense<int32_t>(args[7], "token", at::kInt, R);
  float* logp = x.dense<float>(args[8], "logp", at::kFloat, R, true);
  double* dist = x.dense<double>(args[9], "dist", at::kDouble, 5 * static_cast<int64_t>(R), true);
  CSD_RUN(csd_cat_draft_sample(ctx, R, V, &l, &f, u, token, logp, dist))
})

CSD_MARSHAL(cat_verify, 16, {
  CSD_DEVICE_OF
  const int B = x.n(2), gamma = x.n(3), rows = x.n(4), V = x.n(5);
  const int64_t Rq = static_cast<int64_t>(B) * gamma, Rp = static_cast<int64_t>(B) * rows;
  const csd_logits q = x.logits(args[6], "logits_q", Rq, V);
  const double* dq = x.dense<const double>(args[7], "dist_q", at::kDouble, 5 * Rq);
  const csd_logits p = x.logits(args[8], "logits_p", Rp, V);
  const csd_cat_params f = x.cat_params(args[9], Rp);
  const int32_t* token = x.dense<const int32_t>(args[10], "token", at::kInt, Rq);
  const float* u = x.dense<const float>(args[11], "u", at::kFloat, Rq);
  double* dp = x.dense<double>(args[12], "dist_p", at::kDouble, 5 * Rp);
  float* lr = x.dense<float>(args[13], "logratio", at::kFloat, Rq);
  int32_t* na = x.dense<int32_t>(args[14], "n_accept", at::kInt, B);
  uint32_t* mask = x.dense<uint32_t>(args[15], "accept_mask", at::kInt, B, true);
  CSD_RUN(csd_cat_verify(ctx, B, gamma, rows, V, &q, dq, &p, &f, token, u, dp, lr, na, mask))
})

CSD_MARSHAL(cat_resample, 13, {
  CSD_DEVICE_OF
  const int B = x.n(2), gamma = x.n(3), rows = x.n(4), V = x.n(5);
  const int64_t Rq = static_cast<int64_t>(B) * gamma, Rp = static_cast<int64_t>(B) * rows;
  const csd_logits q = x.logits(args[6], "logits_q", Rq, V);
  const double* dq = x.dense<const double>(args[7], "dist_q", at::kDouble, 5 * Rq);
  const csd_logits p = x.logits(args[8], "logits_p", Rp, V);
  const double* dp = x.dense<const double>(args[9], "dist_p", at::kDouble, 5 * Rp);
  const int32_t* na = x.dense<const int32_t>(args[10], "n_accept", at::kInt, B);
  const float* w = x.dense<const float>(args[11], "w", at::kFloat, B);
  int32_t* xn = x.dense<int32_t>(args[12], "x_new", at::kInt, B);
  CSD_RUN(csd_cat_resample(ctx, B, gamma, rows, V, &q, dq, &p, dp, na, w, xn))
})

CSD_MARSHAL(quantize, 7, {
  CSD_DEVICE_OF
  const int M = x.n(2), K = x.n(3);
  int dtype = -1;
  int64_t ldx = 0;
  const void* in = x.rows_of(args[4], "x", M, K, &dtype, &ldx);
  int ld = 0, ls = 0;
  csd_quant_pitch(K, &ld, &ls);
  uint8_t* data = x.dense<uint8_t>(args[5], "data", at::kByte, static_cast<int64_t>(M) * ld);
  uint8_t* scale = x.dense<uint8_t>(args[6], "scale", at::kByte, static_cast<int64_t>(M) * ls);
  CSD_RUN(csd_quantize(ctx, M, K, dtype, in, ldx, data, scale))
})

CSD_MARSHAL(norm_quantize, 11, {
  CSD_DEVICE_OF
  const int M = x.n(2), K = x.n(3);
  int dtype = -1;
  int64_t ldx = 0;
  int64_t ldr = 0;
  int64_t lds = 0;
  int64_t ldw = 0;
  const void* in = x.rows_of(args[4], "x", M, K, &dtype, &ldx);
  const void* res = x.rows_of(args[5], "residual", M, K, &dtype, &ldr, true);
  const void* weight = x.rows_of(args[6], "weight", 1, K, &dtype, &ldw, true);
  const double eps = x.d(7);
  void* sum = x.rows_of(args[8], "sum", M, K, &dtype, &lds, true);
  int ld = 0, ls = 0;
  csd_quant_pitch(K, &ld, &ls);
  uint8_t* data = x.dense<uint8_t>(args[9], "data", at::kByte, static_cast<int64_t>(M) * ld);
  uint8_t* scale = x.dense<uint8_t>(args[10], "scale", at::kByte, static_cast<int64_t>(M) * ls);
  CSD_RUN(csd_norm_quantize(ctx, M, K, dtype, in, ldx, res, ldr, weight, static_cast<float>(eps), sum, lds, data, scale))
})

CSD_MARSHAL(quant_matmul, 8, {
  CSD_DEVICE_OF
  const int M = x.n(2), N = x.n(3), K = x.n(4);
  const csd_quant a = x.quant(args[5], "the left matrix", M, K);
  const csd_quant w = x.quant(args[6], "the right matrix", N, K);
  int dtype = -1;
  int64_t ldo = 0;
  void* out = x.rows_of(args[7], "out", M, N, &dtype, &ldo);
  CSD_RUN(csd_quant_matmul(ctx, M, N, K, &a, &w, dtype, out, ldo))
})

PyObject* set_ptr_of(PyObject*, PyObject* f) {
  Py_INCREF(f);
  Py_XSETREF(g_ptr_of, f);
  Py_RETURN_NONE;
}

#define CSD_METHOD(NAME) {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(NAME)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {CSD_METHOD(accept_scan), CSD_METHOD(resample), CSD_METHOD(resample_lv), CSD_METHOD(gmm_draft_sample),
                          CSD_METHOD(gmm_verify), CSD_METHOD(gmm_resample), CSD_METHOD(cat_filter), CSD_METHOD(cat_draft_sample),
                          CSD_METHOD(cat_verify), CSD_METHOD(cat_resample), CSD_METHOD(quantize), CSD_METHOD(norm_quantize),
                          CSD_METHOD(quant_matmul), {"set_ptr_of", set_ptr_of, METH_O, nullptr},
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&kModule); }

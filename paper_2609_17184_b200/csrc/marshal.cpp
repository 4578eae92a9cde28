// Argument marshalling of the operators between the linear maps: torch tensors in, calls of the C ABI out (see include/loopspec.h and
// operators.py, which documents the arguments).  Nothing is computed here.  The smallest of these calls take 3 us on the device, and asking eight
// tensors for type, shape, strides and device through Python took 12 to 25 on the host; here it takes 2 to 5.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "../../include/loopspec.h"

namespace {

PyObject* g_error = nullptr;  // LoopSpecError(code, message)

struct Refused {
  int code;
  std::string what;
};
[[noreturn]] void refuse(std::string what) { throw Refused{LOOPSPEC_EINVAL, std::move(what)}; }

const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) refuse(std::string(what) + ": a tensor is needed");
  return THPVariable_Unpack(o);
}
int32_t int32_of(int64_t x, const char* what) {
  if (x < INT32_MIN || x > INT32_MAX) refuse(std::string(what) + ": out of range");
  return (int32_t)x;
}
int32_t int_arg(PyObject* o, const char* what) {
  const long long x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) throw Refused{0, ""};  // (Python's own error)
  return int32_of(x, what);
}
float float_arg(PyObject* o) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) throw Refused{0, ""};
  return (float)x;
}
int code_of(at::ScalarType t) { return t == at::kFloat ? 0 : t == at::kBFloat16 ? 1 : t == at::kHalf ? 2 : -1; }
bool on(const at::Tensor& t, at::Device dev) { return t.device() == dev; }

// a contiguous vector of n elements (None: null)
void* vec(PyObject* o, const char* what, at::ScalarType type, int64_t n, at::Device dev, bool optional = false) {
  if (o == Py_None && optional) return nullptr;
  const at::Tensor& t = tensor(o, what);
  if (t.scalar_type() != type || t.dim() != 1 || t.size(0) != n || !on(t, dev) || !t.is_contiguous())
    refuse(std::string(what) + ": a contiguous vector of " + std::to_string(n) + " " + c10::toString(type) + " elements on " + dev.str() + " is needed");
  return t.data_ptr();
}
struct Table {
  const int32_t* ptr;
  int64_t ld;
  int32_t rows, width;
};
Table table(PyObject* o, at::Device dev) {
  const at::Tensor& t = tensor(o, "page_table");
  if (t.scalar_type() != at::kInt || t.dim() != 2 || !on(t, dev)) refuse("page_table: [sequences, pages] int32 on " + dev.str() + " is needed");
  const int64_t rows = t.size(0), width = t.size(1), ld = t.stride(0);
  if ((t.stride(1) != 1 && width > 1) || (ld < width && rows > 1)) refuse("page_table: contiguous rows that do not overlap are needed");
  return {static_cast<const int32_t*>(t.data_ptr()), ld > width ? ld : width, int32_of(rows, "page_table"), int32_of(width, "page_table")};
}
// [page][head][slot][d] views of one shape and one set of strides
loopspec_paged_kv paged(PyObject* ko, PyObject* vo, at::Device dev) {
  const at::Tensor &k = tensor(ko, "k_cache"), &v = tensor(vo, "v_cache");
  const at::ScalarType type = k.scalar_type();
  if ((type != at::kBFloat16 && type != at::kHalf) || v.scalar_type() != type || k.dim() != 4 || v.dim() != 4 || !on(k, dev) || !on(v, dev))
    refuse("k_cache, v_cache: [pages, heads, page_size, head_dim] bf16 or fp16 on " + dev.str() + " are needed");
  bool alike = v.sizes() == k.sizes() && (k.stride(3) == 1 || k.size(3) <= 1);
  int64_t stride[3];  // (of a dimension of one element any stride will do)
  for (int i = 0; alike && i < 3; ++i) {
    stride[i] = k.size(i) > 1 ? k.stride(i) : k.size(3);
    alike = k.size(i) <= 1 || v.stride(i) == stride[i];
  }
  if (!alike) refuse("k_cache, v_cache: one shape and one set of strides are needed, the last dimension contiguous");
  loopspec_paged_kv c;
  c.k = k.data_ptr(), c.v = v.data_ptr(), c.page_stride = stride[0], c.head_stride = stride[1], c.slot_stride = stride[2];
  c.n_pages = int32_of(k.size(0), "k_cache"), c.n_kv_heads = int32_of(k.size(1), "k_cache"), c.page_size = int32_of(k.size(2), "k_cache");
  c.head_dim = int32_of(k.size(3), "k_cache"), c.dtype = code_of(type);
  return c;
}
// the row stride of [rows, heads, d] with contiguous heads
int64_t heads(const at::Tensor& t, const char* what, at::ScalarType type, int64_t rows, int64_t n, int64_t d, at::Device dev) {
  if (t.scalar_type() != type || t.dim() != 3 || t.size(0) != rows || t.size(1) != n || t.size(2) != d || !on(t, dev) ||
      (t.numel() && ((t.stride(2) != 1 && d > 1) || (t.stride(1) != d && n > 1))))
    refuse(std::string(what) + ": [" + std::to_string(rows) + ", " + std::to_string(n) + ", " + std::to_string(d) + "] " + c10::toString(type) + " on " + dev.str() +
           " with contiguous heads is needed");
  return rows > 1 ? t.stride(0) : n * d;
}
void done(int rc, const char* what) {
  if (rc) throw Refused{rc, what};
}
// the call with the tensors' device current, on that device's current stream
template <typename F>
void call(at::Device dev, const char* what, F f) {
  c10::cuda::OptionalCUDAGuard guard;
  if (c10::cuda::current_device() != dev.index()) guard.set_device(dev);
  done(f((void*)c10::cuda::getCurrentCUDAStream(dev.index()).stream()), what);
}
at::Tensor made(at::IntArrayRef shape, at::ScalarType type, at::Device dev) { return at::empty(shape, at::TensorOptions().dtype(type).device(dev)); }

// f with its refusals and errors as Python's
template <typename F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (const Refused& r) {
    if (r.code) {
      PyObject* e = PyObject_CallFunction(g_error, "is", r.code, r.what.c_str());
      if (e) PyErr_SetObject(g_error, e), Py_DECREF(e);
    }
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}
bool count_is(Py_ssize_t got, Py_ssize_t want) {
  if (got != want) PyErr_Format(PyExc_TypeError, "%zd arguments are needed", want);
  return got == want;
}
PyObject* pair(const at::Tensor& a, const at::Tensor& b) {
  PyObject *x = THPVariable_Wrap(a), *y = THPVariable_Wrap(b), *t = x && y ? PyTuple_Pack(2, x, y) : nullptr;
  Py_XDECREF(x), Py_XDECREF(y);
  return t;
}

PyObject* append_kv(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count_is(n, 14)) return nullptr;
  return guarded([&] {
    const at::Tensor& qkv = tensor(a[0], "qkv");
    const int code = code_of(qkv.scalar_type());
    if (code < 0 || !qkv.is_cuda() || qkv.dim() != 2) refuse("qkv: [rows, (n_q_heads + 2 n_kv_heads) head_dim] fp32, bf16 or fp16 on a CUDA device is needed");
    const at::Device dev = qkv.device();
    const loopspec_paged_kv kv = paged(a[1], a[2], dev);
    const Table pt = table(a[3], dev);
    const int32_t nq = int_arg(a[6], "n_q_heads"), T = int32_of(qkv.size(0), "qkv");
    if (nq < 0 || qkv.size(1) != ((int64_t)nq + 2 * (int64_t)kv.n_kv_heads) * kv.head_dim || (qkv.stride(1) != 1 && qkv.size(1) > 1 && T))
      refuse("qkv: contiguous rows of (n_q_heads + 2 n_kv_heads) * head_dim elements are needed");
    const at::ScalarType type = kv.dtype == 1 ? at::kBFloat16 : at::kHalf;
    const at::Tensor out = a[12] == Py_None ? made({T, nq, kv.head_dim}, type, dev) : tensor(a[12], "out");
    const int64_t q_ld = heads(out, "out", type, T, nq, kv.head_dim, dev), half = a[7] == Py_None ? 0 : tensor(a[7], "inv_freq").numel();
    const int32_t* cached = static_cast<int32_t*>(vec(a[4], "cached", at::kInt, pt.rows, dev));
    const int32_t* cu = static_cast<int32_t*>(vec(a[5], "cu_rows", at::kInt, (int64_t)pt.rows + 1, dev));
    const double* freq = static_cast<double*>(vec(a[7], "inv_freq", at::kDouble, half, dev, true));
    const float *qn = static_cast<float*>(vec(a[8], "q_norm", at::kFloat, kv.head_dim, dev, true)), *kn = static_cast<float*>(vec(a[9], "k_norm", at::kFloat, kv.head_dim, dev, true));
    const int32_t* off = static_cast<int32_t*>(vec(a[11], "pos_offset", at::kInt, pt.rows, dev, true));
    int32_t* flag = static_cast<int32_t*>(vec(a[13], "flag", at::kInt, 1, dev, true));
    const float eps = float_arg(a[10]);
    call(dev, "append_kv", [&](void* st) {
      return loopspec_op_append_kv(qkv.data_ptr(), code, T > 1 ? qkv.stride(0) : qkv.size(1), T, nq, &kv, pt.ptr, pt.ld, pt.width, cached, cu, pt.rows, off, freq, int32_of(2 * half, "inv_freq"), qn, kn,
                                   eps, out.data_ptr(), q_ld, flag, st);
    });
    if (a[12] != Py_None) return Py_INCREF(a[12]), a[12];
    return THPVariable_Wrap(out);
  });
}

PyObject* prefix_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count_is(n, 13)) return nullptr;
  return guarded([&] {
    const at::Tensor& q = tensor(a[0], "q");
    if (!q.is_cuda() || q.dim() != 3) refuse("q: [rows, n_q_heads, head_dim] on a CUDA device is needed");
    const at::Device dev = q.device();
    const loopspec_paged_kv kv = paged(a[1], a[2], dev);
    const Table pt = table(a[5], dev);
    const at::ScalarType type = kv.dtype == 1 ? at::kBFloat16 : at::kHalf;
    const int32_t T = int32_of(q.size(0), "q"), nq = int32_of(q.size(1), "q"), P = int_arg(a[4], "prefix_len");
    const int64_t q_ld = heads(q, "q", type, T, nq, kv.head_dim, dev);
    const at::Tensor out = a[9] == Py_None ? made({T, nq, kv.head_dim}, type, dev) : tensor(a[9], "out");
    const int64_t out_ld = heads(out, "out", type, T, nq, kv.head_dim, dev);
    const at::Tensor lse = a[10] == Py_None ? made({T, nq}, at::kFloat, dev) : tensor(a[10], "lse");
    if (lse.scalar_type() != at::kFloat || lse.dim() != 2 || lse.size(0) != T || lse.size(1) != nq || !on(lse, dev) || !lse.is_contiguous())
      refuse("lse: [rows, n_q_heads] fp32, contiguous, is needed");
    const int32_t* pages = nullptr;
    if (P > 0) {
      const int64_t have = a[3] == Py_None ? 0 : tensor(a[3], "prefix_pages").numel();
      if (have * kv.page_size < P) refuse("prefix_pages: ceil(prefix_len / page_size) entries are needed");
      pages = static_cast<int32_t*>(vec(a[3], "prefix_pages", at::kInt, have, dev));
    }
    const int32_t* lens = static_cast<int32_t*>(vec(a[6], "lens", at::kInt, pt.rows, dev));
    const int32_t* cu = static_cast<int32_t*>(vec(a[7], "cu_rows", at::kInt, (int64_t)pt.rows + 1, dev));
    const float scale = a[8] == Py_None ? 0.f : float_arg(a[8]);
    if (a[8] != Py_None && scale == 0.f) refuse("scale: a positive number is needed (None: 1 / sqrt(head_dim))");
    int32_t* flag = static_cast<int32_t*>(vec(a[12], "flag", at::kInt, 1, dev, true));
    const size_t need = loopspec_prefix_attention_scratch_bytes(T, pt.rows, nq, kv.n_kv_heads, kv.head_dim, P);
    if (need == 0) refuse("prefix_attention: head_dim 64 or 128, n_q_heads a multiple of the key heads, at most 2048 sequences");
    const at::Tensor scratch = a[11] == Py_None ? made({(int64_t)need}, at::kByte, dev) : tensor(a[11], "scratch");
    if (scratch.scalar_type() != at::kByte || !on(scratch, dev) || !scratch.is_contiguous()) refuse("scratch: contiguous uint8 on q's device is needed");
    call(dev, "prefix_attention", [&](void* st) {
      return loopspec_op_prefix_attention(q.data_ptr(), q_ld, T, nq, &kv, pages, P, pt.ptr, pt.ld, pt.width, lens, cu, pt.rows, scale, out.data_ptr(), out_ld,
                                          static_cast<float*>(lse.data_ptr()), flag, scratch.data_ptr(), (size_t)scratch.numel(), st);
    });
    if (a[9] != Py_None && a[10] != Py_None) return PyTuple_Pack(2, a[9], a[10]);
    return pair(out, lse);
  });
}

PyObject* sample(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count_is(n, 8)) return nullptr;
  return guarded([&] {
    const at::Tensor& z = tensor(a[0], "logits");
    const int code = code_of(z.scalar_type());
    if (code < 0 || !z.is_cuda() || z.dim() != 2) refuse("logits: [rows, vocabulary] fp32, bf16 or fp16 on a CUDA device is needed");
    const at::Device dev = z.device();
    const int32_t rows = int32_of(z.size(0), "logits"), V = int32_of(z.size(1), "logits");
    if (z.stride(1) != 1 && V > 1 && rows) refuse("logits: contiguous rows are needed");
    const float* u = static_cast<float*>(vec(a[1], "uniforms", at::kFloat, rows, dev));
    const float* t = static_cast<float*>(vec(a[2], "temperature", at::kFloat, rows, dev, true));
    const int32_t* k = static_cast<int32_t*>(vec(a[3], "top_k", at::kInt, rows, dev, true));
    const float *p = static_cast<float*>(vec(a[4], "top_p", at::kFloat, rows, dev, true)), *m = static_cast<float*>(vec(a[5], "min_p", at::kFloat, rows, dev, true));
    at::Tensor out, probs;
    if (a[6] == Py_None) out = made({rows}, at::kInt, dev);
    if (a[7] == Py_None) probs = made({rows}, at::kFloat, dev);
    int32_t* tok = a[6] == Py_None ? static_cast<int32_t*>(out.data_ptr()) : static_cast<int32_t*>(vec(a[6], "out", at::kInt, rows, dev));
    float* pr = a[7] == Py_None ? static_cast<float*>(probs.data_ptr()) : static_cast<float*>(vec(a[7], "probs", at::kFloat, rows, dev));
    call(dev, "sample", [&](void* st) { return loopspec_op_sample(z.data_ptr(), code, z.stride(0), rows, V, u, t, k, p, m, tok, pr, st); });
    if (a[6] != Py_None) out = tensor(a[6], "out");
    if (a[7] != Py_None) probs = tensor(a[7], "probs");
    return pair(out, probs);
  });
}

PyObject* set_error(PyObject*, PyObject* cls) {
  Py_INCREF(cls);
  Py_XSETREF(g_error, cls);
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"append_kv", (PyCFunction)(void*)append_kv, METH_FASTCALL, nullptr},
                         {"prefix_attention", (PyCFunction)(void*)prefix_attention, METH_FASTCALL, nullptr},
                         {"sample", (PyCFunction)(void*)sample, METH_FASTCALL, nullptr},
                         {"set_error", set_error, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }

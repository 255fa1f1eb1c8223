// binding.cpp -- the calls of the attention step from Python, where a call's time on
// the host is what counts: sss_page_plan takes ten tensors, and to look at one from
// Python (its type, place, layout, size, address) costs 0.3 us, while the kernel
// takes 2.  Each function here looks at its arguments as the Python binding does
// and, if all are in order, makes the call of the C ABI; it returns the call's
// status, or -1 if something is not plain: the Python binding then goes through its
// checks one by one, for the error to raise or the general way to call.
//
// The library's functions come as addresses (init), so this module links to torch
// alone.
#include <Python.h>

#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "sss.h"

namespace {

decltype(&sss_page_plan) g_page_plan = nullptr;
decltype(&sss_qk_norm_rope) g_qk_norm_rope = nullptr;
decltype(&sss_attention) g_attention = nullptr;

const at::Tensor* tensor(PyObject* o) {
  return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr;
}
// a dense CUDA tensor of that type with n elements (n < 0: any number)
bool dense(const at::Tensor* t, at::ScalarType type, int64_t n) {
  return t != nullptr && t->scalar_type() == type && t->is_cuda() && t->is_contiguous() &&
         (n < 0 || t->numel() == n);
}
bool int32s(const at::Tensor* t, int64_t n) { return dense(t, at::kInt, n); }
const int32_t* ints(const at::Tensor* t) {
  return t == nullptr ? nullptr : static_cast<const int32_t*>(t->data_ptr());
}
// None, or one int32 at least
bool status_word(PyObject* o, uint32_t** to) {
  *to = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = tensor(o);
  if (!int32s(t, -1) || t->numel() < 1) return false;
  *to = static_cast<uint32_t*>(t->data_ptr());
  return true;
}
at::ScalarType type_of(int32_t dtype) {
  return dtype == SSS_OUT_F16 ? at::kHalf : dtype == SSS_OUT_BF16 ? at::kBFloat16 : at::kFloat;
}
int32_t code_of(at::ScalarType t) {
  return t == at::kFloat ? SSS_OUT_F32 : t == at::kHalf ? SSS_OUT_F16
         : t == at::kBFloat16 ? SSS_OUT_BF16 : -1;
}
// rows of `width` elements, dense but for the distance between them
bool rows(const at::Tensor* t, int64_t tokens, int64_t width, int64_t* stride) {
  if (t == nullptr || !t->is_cuda() || t->dim() != 2 || t->size(0) != tokens ||
      t->size(1) != width || t->stride(1) != 1)
    return false;
  *stride = tokens > 1 ? t->stride(0) : width;
  return true;
}
void* current_stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

template <typename F>
PyObject* guarded(F f) {  // no C++ exception leaves into the interpreter
  try {
    const int st = f();
    if (PyErr_Occurred()) return nullptr;
    return PyLong_FromLong(st);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 3) {
    PyErr_SetString(PyExc_TypeError, "init takes three addresses");
    return nullptr;
  }
  g_page_plan = reinterpret_cast<decltype(g_page_plan)>(PyLong_AsVoidPtr(a[0]));
  g_qk_norm_rope = reinterpret_cast<decltype(g_qk_norm_rope)>(PyLong_AsVoidPtr(a[1]));
  g_attention = reinterpret_cast<decltype(g_attention)>(PyLong_AsVoidPtr(a[2]));
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NONE;
}

// past, fresh, page_size, free_pages, block_table, cu_q, kv_len, positions, slots, used,
// dev_status
PyObject* page_plan(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> int {
    if (n != 11) return -1;
    const at::Tensor* t[10];
    for (int i = 0; i < 10; ++i)
      if (i != 2) {
        t[i] = tensor(a[i]);
        if (t[i] == nullptr) return -1;
      }
    const int64_t batch = t[0]->numel(), tokens = t[7]->numel();
    uint32_t* status;
    if (!PyLong_Check(a[2]) || t[4]->dim() != 2 || t[4]->size(0) != batch) return -1;
    if (!int32s(t[0], batch) || !int32s(t[1], batch) || !int32s(t[3], -1) || !int32s(t[4], -1) ||
        !int32s(t[5], batch + 1) || !int32s(t[6], batch) || !int32s(t[7], tokens) ||
        !int32s(t[8], tokens) || !int32s(t[9], 1) || !status_word(a[10], &status))
      return -1;
    const long page = PyLong_AsLong(a[2]);
    if (PyErr_Occurred()) return -1;
    if (batch > INT32_MAX || t[3]->numel() > INT32_MAX || t[4]->size(1) > INT32_MAX ||
        page < 0 || page > INT32_MAX)
      return -1;
    const auto out = [&](int i) { return static_cast<int32_t*>(t[i]->data_ptr()); };
    return g_page_plan(ints(t[0]), ints(t[1]), static_cast<int32_t>(batch),
                       static_cast<int32_t>(page), ints(t[3]), static_cast<int32_t>(t[3]->numel()),
                       out(4), static_cast<int32_t>(t[4]->size(1)), out(5), out(6), out(7), out(8),
                       tokens, out(9), status, current_stream());
  });
}

// q, k, v, rope (address), norm weights (their number, 0: none), positions, cache
// (address), slots, q_out, dev_status
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> int {
    if (n != 10) return -1;
    const auto* rope = static_cast<const sss_rope_t*>(PyLong_AsVoidPtr(a[3]));
    const long weights = PyLong_AsLong(a[4]);
    const auto* cache = static_cast<const sss_kv_cache_t*>(PyLong_AsVoidPtr(a[6]));
    if (PyErr_Occurred() || rope == nullptr || cache == nullptr) return -1;
    const at::Tensor *q = tensor(a[0]), *k = tensor(a[1]), *v = tensor(a[2]), *out = tensor(a[8]);
    if (q == nullptr || k == nullptr || v == nullptr || q->dim() != 2) return -1;
    const int64_t tokens = q->size(0), width = q->size(1), dim = cache->dim;
    const int32_t in = code_of(q->scalar_type());
    int64_t qs, ks, vs;
    uint32_t* status;
    if (tokens == 0 || in < 0 || k->scalar_type() != q->scalar_type() ||
        v->scalar_type() != q->scalar_type() || dim <= 0 || width % dim != 0 ||
        (weights != 0 && weights != dim))
      return -1;
    if (!rows(q, tokens, width, &qs) || !rows(k, tokens, cache->heads * dim, &ks) ||
        !rows(v, tokens, cache->heads * dim, &vs) ||
        !dense(out, type_of(cache->dtype), tokens * width) || !status_word(a[9], &status))
      return -1;
    const at::Tensor *positions = tensor(a[5]), *slots = tensor(a[7]);
    if ((a[5] != Py_None || rope->rot_dim > 0) && !int32s(positions, tokens)) return -1;
    if (a[7] != Py_None && !int32s(slots, tokens)) return -1;
    return g_qk_norm_rope(q->data_ptr(), qs, k->data_ptr(), ks, v->data_ptr(), vs, in, tokens,
                          static_cast<int32_t>(width / dim), rope, ints(positions),
                          out->data_ptr(), cache, ints(slots), status, current_stream());
  });
}

// q, cache (address), cu_q, kv_len, max_q, max_kv, block_table, scale, out, workspace,
// dev_status
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> int {
    if (n != 11) return -1;
    const auto* cache = static_cast<const sss_kv_cache_t*>(PyLong_AsVoidPtr(a[1]));
    const long long max_q = PyLong_AsLongLong(a[4]), max_kv = PyLong_AsLongLong(a[5]);
    const double scale = PyFloat_AsDouble(a[7]);
    if (PyErr_Occurred()) {  // (the general way says what is wrong)
      PyErr_Clear();
      return -1;
    }
    const at::Tensor *q = tensor(a[0]), *cu = tensor(a[2]), *kv = tensor(a[3]),
                     *table = tensor(a[6]), *out = tensor(a[8]), *ws = tensor(a[9]);
    uint32_t* status;
    if (cache == nullptr || q == nullptr || q->dim() != 3 || !int32s(cu, -1) || cu->numel() < 1)
      return -1;
    const int64_t tokens = q->size(0), heads = q->size(1), batch = cu->numel() - 1;
    const at::ScalarType type = type_of(cache->dtype);
    if (q->size(2) != cache->dim || !dense(q, type, -1) || !dense(out, type, q->numel())) return -1;
    if (a[3] != Py_None && !int32s(kv, batch)) return -1;
    if (a[6] != Py_None && (!int32s(table, -1) || table->dim() != 2 || table->size(0) != batch))
      return -1;
    if (a[9] != Py_None && !dense(ws, at::kByte, -1)) return -1;
    if (!status_word(a[10], &status) || heads > INT32_MAX || batch > INT32_MAX || max_q < 0 ||
        max_q > INT32_MAX || (table && table->size(1) > INT32_MAX))
      return -1;
    return g_attention(q->data_ptr(), heads * cache->dim, static_cast<int32_t>(heads), cache,
                       ints(cu), ints(kv), ints(table),
                       table ? static_cast<int32_t>(table->size(1)) : 0,
                       static_cast<int32_t>(batch), tokens, static_cast<int32_t>(max_q), max_kv,
                       static_cast<float>(scale), out->data_ptr(), ws ? ws->data_ptr() : nullptr,
                       ws ? static_cast<size_t>(ws->numel()) : 0, status, current_stream());
  });
}

template <typename F>
PyCFunction fast(F* f) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}
PyMethodDef g_methods[] = {
    {"init", fast(init), METH_FASTCALL, nullptr},
    {"page_plan", fast(page_plan), METH_FASTCALL, nullptr},
    {"qk_norm_rope", fast(qk_norm_rope), METH_FASTCALL, nullptr},
    {"attention", fast(attention), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, g_methods,
                        nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&g_module); }

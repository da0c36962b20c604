// Marshalling of the calls on 4-bit caches and of reads: one C++ call looks at a call's tensors and enters the library.
//
// Looking at a tensor from Python - its type, shape, strides, device and address - takes 0.4 us, seven of them as long as the GPU
// takes for a small call; here all of them take 0.1 us.  A function returns the library's status, or None where an argument is not
// what the call needs: the binding's own checks then say what is wrong.  Nothing is kept between calls.
//
// It reads tensors through torch's headers, whose layouts belong to one build of torch: `built_for` names that and the Python, and
// the binding does without where they are others.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/peagle.h"

namespace {

decltype(&peagle_cache_append_block_scaled) g_append = nullptr;
decltype(&peagle_cache_read) g_read = nullptr;
decltype(&peagle_draft_decode_block_scaled) g_draft = nullptr;
PyObject *s_n_tokens, *s_Hkv, *s_D, *s_n_pages, *s_C, *s_K, *s_Hq, *s_scale, *s_max_pages, *s_device_index, *s_cuda_stream;

struct Wrong {};  // an argument that the binding's checks have to look at

int64_t whole(PyObject* of, PyObject* name) {
  PyObject* v = PyObject_GetAttr(of, name);
  if (!v || !PyLong_CheckExact(v)) {
    Py_XDECREF(v);
    throw Wrong();
  }
  const long long x = PyLong_AsLongLong(v);
  Py_DECREF(v);
  if (x < INT32_MIN || x > INT32_MAX || (x == -1 && PyErr_Occurred())) throw Wrong();
  return x;
}

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) throw Wrong();
  return THPVariable_Unpack(o);
}

// The tensors of one call, all on the current device.
struct Call {
  int device;
  void* stream;
  explicit Call(PyObject* stream_or_none) : device(c10::hip::current_device()) {
    if (stream_or_none == Py_None) {
      stream = (void*)c10::hip::getCurrentHIPStream((c10::DeviceIndex)device).stream();
    } else {
      if (whole(stream_or_none, s_device_index) != device) throw Wrong();
      PyObject* v = PyObject_GetAttr(stream_or_none, s_cuda_stream);
      if (!v) throw Wrong();
      stream = PyLong_AsVoidPtr(v);
      Py_DECREF(v);
      if (PyErr_Occurred()) throw Wrong();
    }
  }
  const at::Tensor& of(PyObject* o, at::ScalarType type, c10::IntArrayRef shape) const {
    const at::Tensor& t = tensor(o);
    if (t.scalar_type() != type || t.sizes() != shape || !t.is_cuda() || t.get_device() != device) throw Wrong();
    return t;
  }
  void* whole_of(PyObject* o, at::ScalarType type, c10::IntArrayRef shape) const {
    const at::Tensor& t = of(o, type, shape);
    if (!t.is_contiguous()) throw Wrong();
    return t.data_ptr();
  }
  // Rows that may stand apart.
  void* rows(PyObject* o, c10::IntArrayRef shape, int64_t* stride) const {
    const at::Tensor& t = of(o, at::kBFloat16, shape);
    if ((shape[2] > 1 && t.stride(2) != 1) || (shape[1] > 1 && t.stride(1) != shape[2])) throw Wrong();
    *stride = shape[0] > 1 ? t.stride(0) : shape[1] * shape[2];
    return t.data_ptr();
  }
};

struct Pools {
  int32_t format;
  void *k, *v, *ks, *vs;
  Pools(const Call& call, PyObject* const* a, int64_t n_pages, int64_t Hkv, int64_t D, bool any_format) {
    const at::ScalarType type = tensor(a[0]).scalar_type(), e8 = at::kFloat8_e8m0fnu;
    if (type == at::kFloat4_e2m1fn_x2) format = PEAGLE_CACHE_E2M1;
    else if (any_format && type == at::kFloat8_e4m3fn) format = PEAGLE_CACHE_E4M3;
    else if (any_format && type == at::kFloat8_e5m2) format = PEAGLE_CACHE_E5M2;
    else throw Wrong();
    const bool four = format == PEAGLE_CACHE_E2M1;
    const int64_t pool[] = {n_pages, Hkv, 64, four ? D / 2 : D}, scales[] = {n_pages, Hkv, 64, D / 32};
    const c10::IntArrayRef scale_shape(scales, four ? 4 : 2);
    k = call.whole_of(a[0], type, pool);
    v = call.whole_of(a[1], type, pool);
    ks = call.whole_of(a[2], e8, scale_shape);
    vs = call.whole_of(a[3], e8, scale_shape);
  }
};

// The library's entry points throw nothing; other threads may run meanwhile (a launch waits where the stream's queue is full).
template <class F>
int without_lock(F f) {
  PyThreadState* const state = PyEval_SaveThread();
  const int rc = f();
  PyEval_RestoreThread(state);
  return rc;
}

template <class F>
PyObject* guarded(F f) {
  try {
    return PyLong_FromLong(f());
  } catch (...) {  // (torch's own errors among them)
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

peagle_cache_shape_t cache_shape(PyObject* o) {
  peagle_cache_shape_t s{};
  s.n_tokens = (int32_t)whole(o, s_n_tokens);
  s.Hkv = (int32_t)whole(o, s_Hkv);
  s.D = (int32_t)whole(o, s_D);
  s.n_pages = (int32_t)whole(o, s_n_pages);
  return s;
}

// cache_append(shape, k_new, v_new, slots, k_pages, v_pages, k_scale, v_scale, stream)
PyObject* cache_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&] {
    if (n != 9 || !g_append) throw Wrong();
    peagle_cache_shape_t s = cache_shape(a[0]);
    const Call call(a[8]);
    const Pools p(call, a + 4, s.n_pages, s.Hkv, s.D, false);
    const int64_t shape[] = {s.n_tokens, s.Hkv, s.D}, slots[] = {s.n_tokens};
    s.format = p.format;
    void* k = call.rows(a[1], shape, &s.k_stride);
    void* v = call.rows(a[2], shape, &s.v_stride);
    const int64_t* at = (const int64_t*)call.whole_of(a[3], at::kLong, slots);
    return without_lock([&] { return g_append(&s, k, v, at, p.k, p.v, p.ks, p.vs, call.stream); });
  });
}

// cache_read(shape, slots, k_pages, v_pages, k_scale, v_scale, k_out, v_out, stream)
PyObject* cache_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&] {
    if (n != 9 || !g_read) throw Wrong();
    peagle_cache_shape_t s = cache_shape(a[0]);
    const Call call(a[8]);
    const Pools p(call, a + 2, s.n_pages, s.Hkv, s.D, true);
    const int64_t shape[] = {s.n_tokens, s.Hkv, s.D}, slots[] = {s.n_tokens};
    s.format = p.format;
    void* k = call.rows(a[6], shape, &s.k_stride);
    void* v = call.rows(a[7], shape, &s.v_stride);
    const int64_t* at = (const int64_t*)call.whole_of(a[1], at::kLong, slots);
    return without_lock([&] { return g_read(&s, at, p.k, p.v, p.ks, p.vs, k, v, call.stream); });
  });
}

// draft_decode(shape, q_new, k_new, v_new, k_pages, v_pages, k_scale, v_scale, block_table, ctx_len, o, lse, status, workspace, stream)
PyObject* draft_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&] {
    if (n != 15 || !g_draft) throw Wrong();
    peagle_decode_shape_t s{};
    s.C = (int32_t)whole(a[0], s_C);
    s.K = (int32_t)whole(a[0], s_K);
    s.Hq = (int32_t)whole(a[0], s_Hq);
    s.Hkv = (int32_t)whole(a[0], s_Hkv);
    s.D = (int32_t)whole(a[0], s_D);
    s.n_pages = (int32_t)whole(a[0], s_n_pages);
    s.max_pages = (int32_t)whole(a[0], s_max_pages);
    PyObject* scale = PyObject_GetAttr(a[0], s_scale);
    if (!scale || !PyFloat_CheckExact(scale)) {
      Py_XDECREF(scale);
      throw Wrong();
    }
    s.scale = (float)PyFloat_AS_DOUBLE(scale);
    Py_DECREF(scale);
    const Call call(a[14]);
    const Pools p(call, a + 4, s.n_pages, s.Hkv, s.D, false);
    const int64_t q[] = {s.C, s.K, s.Hq, s.D}, kv[] = {s.C, s.K, s.Hkv, s.D}, table[] = {s.C, s.max_pages}, each[] = {s.C}, lse[] = {s.C, s.Hq, s.K};
    const at::ScalarType bf = at::kBFloat16, i32 = at::kInt;
    const at::Tensor& ws = tensor(a[13]);
    if (ws.scalar_type() != at::kByte || !ws.is_cuda() || ws.get_device() != call.device || !ws.is_contiguous()) throw Wrong();
    const void *q_new = call.whole_of(a[1], bf, q), *k_new = call.whole_of(a[2], bf, kv), *v_new = call.whole_of(a[3], bf, kv);
    const int32_t *block_table = (const int32_t*)call.whole_of(a[8], i32, table), *ctx_len = (const int32_t*)call.whole_of(a[9], i32, each);
    void *o = call.whole_of(a[10], bf, q), *sums = call.whole_of(a[11], at::kFloat, lse);
    int32_t* status = a[12] == Py_None ? nullptr : (int32_t*)call.whole_of(a[12], i32, each);
    void* workspace = ws.data_ptr();
    const size_t ws_bytes = (size_t)ws.numel();
    return without_lock([&] {
      return g_draft(&s, q_new, k_new, v_new, p.k, p.v, p.ks, p.vs, block_table, ctx_len, o, (float*)sums, status, workspace, ws_bytes, call.stream);
    });
  });
}

// bind(append, read, draft): addresses of the library's entry points
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 3) {
    PyErr_SetString(PyExc_TypeError, "bind takes three addresses");
    return nullptr;
  }
  void* p[3];
  for (int i = 0; i < 3; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  g_append = (decltype(g_append))p[0];
  g_read = (decltype(g_read))p[1];
  g_draft = (decltype(g_draft))p[2];
  Py_RETURN_NONE;
}

#define FAST(f) (PyCFunction)(void (*)(void))(f), METH_FASTCALL
PyMethodDef methods[] = {{"cache_append", FAST(cache_append), nullptr},
                         {"cache_read", FAST(cache_read), nullptr},
                         {"draft_decode", FAST(draft_decode), nullptr},
                         {"bind", FAST(bind), nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) {
  const struct {
    PyObject** to;
    const char* name;
  } names[] = {{&s_n_tokens, "n_tokens"}, {&s_Hkv, "Hkv"}, {&s_D, "D"},   {&s_n_pages, "n_pages"}, {&s_C, "C"},
               {&s_K, "K"},               {&s_Hq, "Hq"},   {&s_scale, "scale"}, {&s_max_pages, "max_pages"},
               {&s_device_index, "device_index"}, {&s_cuda_stream, "cuda_stream"}};
  for (const auto& x : names)
    if (!(*x.to = PyUnicode_InternFromString(x.name))) return nullptr;
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "built_for", PEAGLE_BUILT_FOR) != 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}

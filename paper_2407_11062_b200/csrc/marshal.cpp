// Argument marshalling of the calls that a decoding step makes for every block and token: tensors to the device pointers of
// the C ABI, in one call into compiled code.  The interpreter took 6 of the 9 to 13 us of host time of such a call to ask
// nine to eleven tensors for their addresses, more than the kernels run for one user's step.
//
// Nothing is computed here.  The addresses of the library's entry points are handed over by the binding (bind), so this
// module links against neither library; statuses go back as they are.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "eqat.h"

namespace {

decltype(&eqat_cache_append) g_append = nullptr;
decltype(&eqat_cache_read) g_read = nullptr;
decltype(&eqat_cache_attention) g_attention = nullptr;

struct Refused {};                                   // the Python error is set

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) {
    PyErr_SetString(PyExc_TypeError, "expected a tensor");
    throw Refused();
  }
  return THPVariable_Unpack(o);
}

// Of a type, and with as many elements as the descriptors say (counted in double: they have not been checked yet).
void has(const at::Tensor& t, at::ScalarType type, double least) {
  if (t.scalar_type() != type) {
    PyErr_Format(PyExc_TypeError, "expected a tensor of type %s", c10::toString(type));
    throw Refused();
  }
  if ((double)t.numel() < least) {
    PyErr_SetString(PyExc_ValueError, "a tensor has fewer elements than the descriptors say");
    throw Refused();
  }
}

// The launch goes to the current device and its current stream: so must every tensor of the call.  (Asked for once a call, and
// only where there is a CUDA tensor.)
thread_local int t_device = -1;
void here(const at::Tensor& t) {
  if (t_device < 0) t_device = c10::cuda::current_device();
  if (t.get_device() != t_device) {
    PyErr_Format(PyExc_ValueError, "a tensor is on cuda:%d, the current device is cuda:%d", (int)t.get_device(), t_device);
    throw Refused();
  }
}

// Address of a contiguous CUDA tensor; None: NULL.
void* pointer(PyObject* o, at::ScalarType type, double least) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  has(t, type, least);
  if (!t.is_cuda() || !t.is_contiguous()) {
    PyErr_SetString(PyExc_ValueError, "expected a contiguous CUDA tensor");
    throw Refused();
  }
  here(t);
  return t.data_ptr();
}

// Any type, e.g. a workspace.
void* bytes_of(PyObject* o, size_t* bytes) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  *bytes = t.nbytes();
  return pointer(o, t.scalar_type(), 0.0);
}

// Address and row pitch of a [rows, heads, head_dim] tensor whose heads and elements are dense.
eqat_bf16* rows_of(PyObject* o, const eqat_cache_desc& d, int64_t heads, int64_t* pitch) {
  const at::Tensor& t = tensor(o);
  has(t, at::kBFloat16, 0.0);
  if (t.dim() != 3 || t.size(0) < d.rows || t.size(1) != heads || t.size(2) != d.head_dim) {
    PyErr_SetString(PyExc_ValueError, "a row tensor's shape is not the descriptors' [rows, heads, head_dim]");
    throw Refused();
  }
  if (!t.is_cuda() || t.stride(2) != 1 || t.stride(1) != t.size(2)) {
    PyErr_SetString(PyExc_ValueError, "expected a CUDA tensor [rows, heads, head_dim] with dense heads");
    throw Refused();
  }
  here(t);
  const int64_t least = t.size(1) * t.size(2);
  *pitch = t.size(0) > 1 ? t.stride(0) : least;      // of a single row a stride says nothing
  return static_cast<eqat_bf16*>(t.data_ptr());
}

// A descriptor of the binding (a ctypes structure).
template <typename T>
T structure(PyObject* o) {
  Py_buffer view;
  if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw Refused();
  T value;
  const bool fits = view.len == (Py_ssize_t)sizeof(T);
  if (fits) memcpy(&value, view.buf, sizeof(T));
  PyBuffer_Release(&view);
  if (!fits) {
    PyErr_SetString(PyExc_TypeError, "expected another descriptor");
    throw Refused();
  }
  return value;
}

eqat_cache pool(PyObject* o, const eqat_cache_desc& d) {
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) {
    PyErr_SetString(PyExc_TypeError, "expected a cache: (k_codes, k_params, v_codes, v_params)");
    throw Refused();
  }
  const double tokens = (double)d.pages * d.kv_heads * d.page_size, codes = tokens * d.head_dim / 2;
  const double params = d.group > 0 ? tokens * (d.head_dim / d.group) * 2 : 0.0;
  void* p[4];
  for (int i = 0; i < 4; ++i)
    p[i] = pointer(PyTuple_GET_ITEM(o, i), i & 1 ? at::kBFloat16 : at::kByte, i & 1 ? params : codes);
  return eqat_cache{static_cast<uint8_t*>(p[0]), static_cast<eqat_bf16*>(p[1]), static_cast<uint8_t*>(p[2]), static_cast<eqat_bf16*>(p[3])};
}

template <typename F>
PyObject* call(Py_ssize_t given, Py_ssize_t wanted, F&& f) {
  if (given != wanted || g_append == nullptr) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments, or called before bind()");
    return nullptr;
  }
  t_device = -1;
  try {
    return PyLong_FromLong(f());
  } catch (const Refused&) {
    return nullptr;
  } catch (const std::exception& e) {                // a tensor without storage, no CUDA device
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

template <typename F>
int launch(F&& f) {
  void* stream = c10::cuda::getCurrentCUDAStream().stream();
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f(stream);
  Py_END_ALLOW_THREADS
  return rc;
}

const int32_t* index_of(PyObject* o, double least) { return static_cast<const int32_t*>(pointer(o, at::kInt, least)); }
eqat_bf16* values_of(PyObject* o, const eqat_cache_desc& d) {
  return static_cast<eqat_bf16*>(pointer(o, at::kBFloat16, (double)d.rows * d.kv_heads * d.head_dim));
}

struct Places {
  const int32_t *offsets, *lengths, *table;
  Places(PyObject* const* a, const eqat_cache_desc& d)
      : offsets(index_of(a[0], d.sequences + 1.0)), lengths(index_of(a[1], d.sequences)), table(index_of(a[2], (double)d.sequences * d.max_pages)) {}
};

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 3) {
    PyErr_SetString(PyExc_TypeError, "bind(append, read, attention)");
    return nullptr;
  }
  void* p[3];
  for (int i = 0; i < 3; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (p[i] == nullptr) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an address is 0");
      return nullptr;
    }
  }
  g_read = reinterpret_cast<decltype(g_read)>(p[1]);
  g_attention = reinterpret_cast<decltype(g_attention)>(p[2]);
  g_append = reinterpret_cast<decltype(g_append)>(p[0]);
  Py_RETURN_NONE;
}

// desc, K, V, row_offsets, lengths, page_table, cache, K_hat, V_hat
PyObject* cache_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 9, [&] {
    const auto d = structure<eqat_cache_desc>(a[0]);
    int64_t kp, vp;
    const auto *K = rows_of(a[1], d, d.kv_heads, &kp), *V = rows_of(a[2], d, d.kv_heads, &vp);
    const Places place(a + 3, d);
    const eqat_cache c = pool(a[6], d);
    eqat_bf16 *kh = values_of(a[7], d), *vh = values_of(a[8], d);
    return launch([&](void* s) { return g_append(&d, K, kp, V, vp, place.offsets, place.lengths, place.table, &c, kh, vh, s); });
  });
}

// desc, row_offsets, lengths, page_table, cache, K_hat, V_hat
PyObject* cache_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 7, [&] {
    const auto d = structure<eqat_cache_desc>(a[0]);
    const Places place(a + 1, d);
    const eqat_cache c = pool(a[4], d);
    eqat_bf16 *kh = values_of(a[5], d), *vh = values_of(a[6], d);
    return launch([&](void* s) { return g_read(&d, place.offsets, place.lengths, place.table, &c, kh, vh, s); });
  });
}

// desc, attn, Q, row_offsets, lengths, page_table, cache, O, lse, workspace
PyObject* cache_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 10, [&] {
    const auto d = structure<eqat_cache_desc>(a[0]);
    const auto t = structure<eqat_attention_desc>(a[1]);
    int64_t qp, op;
    const auto* Q = rows_of(a[2], d, t.q_heads, &qp);
    const Places place(a + 3, d);
    const eqat_cache c = pool(a[6], d);
    auto* O = rows_of(a[7], d, t.q_heads, &op);
    float* lse = static_cast<float*>(pointer(a[8], at::kFloat, (double)d.rows * t.q_heads));
    size_t bytes = 0;
    void* ws = bytes_of(a[9], &bytes);
    return launch([&](void* s) { return g_attention(&d, &t, Q, qp, place.offsets, place.lengths, place.table, &c, O, op, lse, ws, bytes, s); });
  });
}

PyMethodDef g_methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(bind)), METH_FASTCALL, "addresses of the library's entry points"},
    {"cache_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_append)), METH_FASTCALL, "eqat_cache_append"},
    {"cache_read", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_read)), METH_FASTCALL, "eqat_cache_read"},
    {"cache_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_attention)), METH_FASTCALL, "eqat_cache_attention"},
    {nullptr, nullptr, 0, nullptr}};
// (EQAT_BUILT_FOR: Python and torch; the build looks for it)
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_marshal", "argument marshalling of the cache's calls, " EQAT_BUILT_FOR, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&g_module); }

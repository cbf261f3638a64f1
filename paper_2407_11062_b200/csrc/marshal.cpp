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
decltype(&eqat_rms_norm_fwd) g_norm_fwd = nullptr;
decltype(&eqat_rms_norm_bwd) g_norm_bwd = nullptr;
decltype(&eqat_rotary_fwd) g_rotary_fwd = nullptr;
decltype(&eqat_rotary_bwd) g_rotary_bwd = nullptr;
decltype(&eqat_gated_fwd) g_gated_fwd = nullptr;
decltype(&eqat_gated_bwd) g_gated_bwd = nullptr;
decltype(&qlinear_packed_gated_fwd) g_packed_gated_fwd = nullptr;
decltype(&qlinear_packed_gated_bwd) g_packed_gated_bwd = nullptr;

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
eqat_bf16* rows_of(PyObject* o, int64_t rows, int64_t heads, int64_t head_dim, int64_t* pitch) {
  const at::Tensor& t = tensor(o);
  has(t, at::kBFloat16, 0.0);
  if (t.dim() != 3 || t.size(0) < rows || t.size(1) != heads || t.size(2) != head_dim) {
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
eqat_bf16* rows_of(PyObject* o, const eqat_cache_desc& d, int64_t heads, int64_t* pitch) {
  return rows_of(o, d.rows, heads, d.head_dim, pitch);
}

// The same of a [rows, features] tensor whose elements are dense.
eqat_bf16* rows_of(PyObject* o, const eqat_gated_desc& d, int64_t* pitch) {
  const at::Tensor& t = tensor(o);
  has(t, at::kBFloat16, 0.0);
  if (t.dim() != 2 || t.size(0) < d.rows || t.size(1) != d.features) {
    PyErr_SetString(PyExc_ValueError, "a tensor's shape is not the descriptor's [rows, features]");
    throw Refused();
  }
  if (!t.is_cuda() || t.stride(1) != 1) {
    PyErr_SetString(PyExc_ValueError, "expected a CUDA tensor [rows, features] with dense rows");
    throw Refused();
  }
  here(t);
  *pitch = t.size(0) > 1 ? t.stride(0) : t.size(1);
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
  constexpr int kCalls = 11;
  if (n != kCalls) {
    PyErr_SetString(PyExc_TypeError, "bind() takes the address of every call");
    return nullptr;
  }
  void* p[kCalls];
  for (int i = 0; i < kCalls; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (p[i] == nullptr) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an address is 0");
      return nullptr;
    }
  }
  g_read = reinterpret_cast<decltype(g_read)>(p[1]);
  g_attention = reinterpret_cast<decltype(g_attention)>(p[2]);
  g_norm_fwd = reinterpret_cast<decltype(g_norm_fwd)>(p[3]);
  g_norm_bwd = reinterpret_cast<decltype(g_norm_bwd)>(p[4]);
  g_rotary_fwd = reinterpret_cast<decltype(g_rotary_fwd)>(p[5]);
  g_rotary_bwd = reinterpret_cast<decltype(g_rotary_bwd)>(p[6]);
  g_gated_fwd = reinterpret_cast<decltype(g_gated_fwd)>(p[7]);
  g_gated_bwd = reinterpret_cast<decltype(g_gated_bwd)>(p[8]);
  g_packed_gated_fwd = reinterpret_cast<decltype(g_packed_gated_fwd)>(p[9]);
  g_packed_gated_bwd = reinterpret_cast<decltype(g_packed_gated_bwd)>(p[10]);
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

eqat_bf16* dense(PyObject* o, double least) { return static_cast<eqat_bf16*>(pointer(o, at::kBFloat16, least)); }

// desc, X, R, W, H, Y, codes, scales
PyObject* rms_norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 8, [&] {
    const auto d = structure<eqat_norm_desc>(a[0]);
    const double all = (double)d.rows * d.features;
    const auto *X = dense(a[1], all), *R = dense(a[2], all), *W = dense(a[3], d.features);
    auto *H = dense(a[4], all), *Y = dense(a[5], all);
    size_t bytes = 0;
    void* codes = bytes_of(a[6], &bytes);
    if (codes != nullptr && (THPVariable_Unpack(a[6]).element_size() != 1 || (double)bytes < all)) {
      PyErr_SetString(PyExc_TypeError, "expected codes of one byte, as many as the descriptor says");
      throw Refused();
    }
    float* scales = static_cast<float*>(pointer(a[7], at::kFloat, d.group > 0 ? (double)d.rows * (d.features / d.group) : 0.0));
    return launch([&](void* s) { return g_norm_fwd(&d, X, R, W, H, Y, codes, scales, s); });
  });
}

// desc, dY, H, W, dR, dX, dW, workspace
PyObject* rms_norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 8, [&] {
    const auto d = structure<eqat_norm_desc>(a[0]);
    const double all = (double)d.rows * d.features;
    const auto *dY = dense(a[1], all), *H = dense(a[2], all), *W = dense(a[3], d.features), *dR = dense(a[4], all);
    auto* dX = dense(a[5], all);
    float* dW = static_cast<float*>(pointer(a[6], at::kFloat, d.features));
    size_t bytes = 0;
    void* ws = bytes_of(a[7], &bytes);
    return launch([&](void* s) { return g_norm_bwd(&d, dY, H, W, dR, dX, dW, ws, bytes, s); });
  });
}

// desc, Q, K, turns, Q_out, K_out, positions, row_offsets, lengths
PyObject* rotary(PyObject* const* a, Py_ssize_t n, decltype(&eqat_rotary_fwd) entry) {
  return call(n, 9, [&] {
    const auto d = structure<eqat_rotary_desc>(a[0]);
    int64_t qp = 0, kp = 0, qop = 0, kop = 0;
    const auto* Q = rows_of(a[1], d.rows, d.q_heads, d.head_dim, &qp);
    auto* Q_out = rows_of(a[4], d.rows, d.q_heads, d.head_dim, &qop);
    const eqat_bf16* K = nullptr;
    eqat_bf16* K_out = nullptr;
    if (d.kv_heads > 0) {
      K = rows_of(a[2], d.rows, d.kv_heads, d.head_dim, &kp);
      K_out = rows_of(a[5], d.rows, d.kv_heads, d.head_dim, &kop);
    }
    const auto* turns = static_cast<const uint64_t*>(pointer(a[3], at::kLong, d.rotary_dim / 2));
    const int32_t *pos = index_of(a[6], d.rows), *off = index_of(a[7], d.sequences + 1.0), *len = index_of(a[8], d.sequences);
    return launch([&](void* s) { return entry(&d, Q, qp, K, kp, turns, pos, off, len, Q_out, qop, K_out, kop, s); });
  });
}
PyObject* rotary_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) { return rotary(a, n, g_rotary_fwd); }
PyObject* rotary_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) { return rotary(a, n, g_rotary_bwd); }

// desc, G, U, H
PyObject* gated_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 4, [&] {
    const auto d = structure<eqat_gated_desc>(a[0]);
    int64_t gp, up;
    const auto *G = rows_of(a[1], d, &gp), *U = rows_of(a[2], d, &up);
    auto* H = dense(a[3], (double)d.rows * d.features);
    return launch([&](void* s) { return g_gated_fwd(&d, G, gp, U, up, H, s); });
  });
}

// desc, dH, G, U, dG, dU
PyObject* gated_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 6, [&] {
    const auto d = structure<eqat_gated_desc>(a[0]);
    int64_t gp, up, dgp, dup;
    const auto* dH = dense(a[1], (double)d.rows * d.features);
    const auto *G = rows_of(a[2], d, &gp), *U = rows_of(a[3], d, &up);
    auto *dG = rows_of(a[4], d, &dgp), *dU = rows_of(a[5], d, &dup);
    return launch([&](void* s) { return g_gated_bwd(&d, dH, G, gp, U, up, dG, dgp, dU, dup, s); });
  });
}

// (Wq_packed, s16, z)
eqat_packed_weight weight_of(PyObject* o, const eqat_desc& d) {
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 3) {
    PyErr_SetString(PyExc_TypeError, "expected a weight: (Wq_packed, s16, z)");
    throw Refused();
  }
  const double all = (double)d.out_features * d.in_features, groups = d.group > 0 ? all / d.group : 0.0;
  return eqat_packed_weight{static_cast<const uint8_t*>(pointer(PyTuple_GET_ITEM(o, 0), at::kByte, all * d.bits / 8)),
                            static_cast<const eqat_fp16*>(pointer(PyTuple_GET_ITEM(o, 1), at::kHalf, groups)),
                            pointer(PyTuple_GET_ITEM(o, 2), d.zero_point_format == EQAT_ZP_FP16 ? at::kHalf : at::kByte, groups)};
}
int number(PyObject* o) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused();
  return v < 0 || v > 1000 ? -1 : (int)v;              // no activation either way
}

// desc, activation, X, gate, up, H, G, U, workspace
PyObject* packed_gated_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 9, [&] {
    const auto d = structure<eqat_desc>(a[0]);
    const int act = number(a[1]);
    const double inner = (double)d.tokens * d.out_features;
    const auto* X = dense(a[2], (double)d.tokens * d.in_features);
    const eqat_packed_weight gate = weight_of(a[3], d), up = weight_of(a[4], d);
    auto *H = dense(a[5], inner), *G = dense(a[6], inner), *U = dense(a[7], inner);
    size_t bytes = 0;
    void* ws = bytes_of(a[8], &bytes);
    return launch([&](void* s) { return g_packed_gated_fwd(&d, act, X, &gate, &up, H, G, U, ws, bytes, s); });
  });
}

// desc, activation, dH, G, U, gate, up, dX, dG, dU, workspace
PyObject* packed_gated_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 11, [&] {
    const auto d = structure<eqat_desc>(a[0]);
    const int act = number(a[1]);
    const double inner = (double)d.tokens * d.out_features;
    const auto *dH = dense(a[2], inner), *G = dense(a[3], inner), *U = dense(a[4], inner);
    const eqat_packed_weight gate = weight_of(a[5], d), up = weight_of(a[6], d);
    auto *dX = dense(a[7], (double)d.tokens * d.in_features), *dG = dense(a[8], inner), *dU = dense(a[9], inner);
    size_t bytes = 0;
    void* ws = bytes_of(a[10], &bytes);
    return launch([&](void* s) { return g_packed_gated_bwd(&d, act, dH, G, U, &gate, &up, dX, dG, dU, ws, bytes, s); });
  });
}

#define EQAT_METHOD(name, doc) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, doc}
PyMethodDef g_methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(bind)), METH_FASTCALL, "addresses of the library's entry points"},
    {"cache_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_append)), METH_FASTCALL, "eqat_cache_append"},
    {"cache_read", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_read)), METH_FASTCALL, "eqat_cache_read"},
    {"cache_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_attention)), METH_FASTCALL, "eqat_cache_attention"},
    EQAT_METHOD(rms_norm_fwd, "eqat_rms_norm_fwd"),
    EQAT_METHOD(rms_norm_bwd, "eqat_rms_norm_bwd"),
    EQAT_METHOD(rotary_fwd, "eqat_rotary_fwd"),
    EQAT_METHOD(rotary_bwd, "eqat_rotary_bwd"),
    EQAT_METHOD(gated_fwd, "eqat_gated_fwd"),
    EQAT_METHOD(gated_bwd, "eqat_gated_bwd"),
    EQAT_METHOD(packed_gated_fwd, "qlinear_packed_gated_fwd"),
    EQAT_METHOD(packed_gated_bwd, "qlinear_packed_gated_bwd"),
    {nullptr, nullptr, 0, nullptr}};
// (EQAT_BUILT_FOR: Python and torch; the build looks for it)
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_marshal", "argument marshalling of a decoding step's calls, " EQAT_BUILT_FOR, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&g_module); }

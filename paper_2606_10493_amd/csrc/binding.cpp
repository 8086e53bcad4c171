// The attention calls' Python binding: checks of the tensors and the call of the
// C ABI in one native function each.  A decode step makes these calls for every
// layer and is bound by the host: moe_rope_cache takes 3 us of it here, most of
// them the launch, and 9 with the same checks in Python and ctypes.
//
// Every function takes what its namesake in attention.py passes, in order, and
// returns the status of the C call; the stream is always the last.  Tensors are read
// through torch's C++ objects; nothing of a call is kept.
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <type_traits>

#include "moe.h"

namespace {

struct Bad {};  // a Python error is set

[[noreturn]] void bad_value(const char* format, const char* name) {
  PyErr_Format(PyExc_ValueError, format, name);
  throw Bad{};
}

int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Bad{};
  return v;
}

int64_t attribute(PyObject* o, const char* name) {
  PyObject* value = PyObject_GetAttrString(o, name);
  if (!value) throw Bad{};
  const long long v = PyLong_AsLongLong(value);
  Py_DECREF(value);
  if (v == -1 && PyErr_Occurred()) throw Bad{};
  return v;
}

// The stream of the call that runs and its device: the caller's torch stream, or the current device's current one.
// Taken once, by the first tensor.  An argument may be an object whose attributes are Python code, which may make calls
// of its own and let other threads run: each thread has its own, and a call puts back what it found.
struct Stream {
  PyObject* given = nullptr;
  hipStream_t handle = nullptr;
  int64_t device = -1;
  void take() {
    if (device >= 0) return;
    if (given == Py_None) {
      const auto current = c10::hip::getCurrentHIPStream();
      handle = current.stream();
      device = current.device_index();
    } else {
      handle = reinterpret_cast<hipStream_t>(attribute(given, "cuda_stream"));
      // an object that has a handle alone stands for a stream of the current device
      device = PyObject_HasAttrString(given, "device_index") ? attribute(given, "device_index")
                                                             : c10::hip::getCurrentHIPStream().device_index();
    }
  }
};

thread_local Stream call_stream;

struct OwnStream {
  const Stream before = call_stream;
  explicit OwnStream(PyObject* given) { call_stream = Stream{given}; }
  ~OwnStream() { call_stream = before; }
};

void on_call_device(int64_t index, const char* name) {
  call_stream.take();
  if (index != call_stream.device) bad_value("%s is on another device than the call's stream", name);
}

hipStream_t stream() {
  call_stream.take();
  return call_stream.handle;
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
    throw Bad{};
  }
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) bad_value("%s must be a device tensor", name);
  on_call_device(t.device().index(), name);
  return t;
}

// The address of a contiguous device tensor, NULL for None.  Integers and fp32 numbers have that type; bytes
// (workspaces) and 16-bit words, whose type bf16_rows looks at, have that size.
template <typename T>
T* address(PyObject* o, const char* name, int64_t* count = nullptr) {
  if (o == Py_None) {
    if (count) *count = 0;
    return nullptr;
  }
  const at::Tensor& t = tensor(o, name);
  if (!t.is_contiguous()) bad_value("%s must be contiguous", name);
  if (std::is_same_v<T, int32_t> && t.scalar_type() != at::kInt) bad_value("%s must be int32", name);
  if (std::is_same_v<T, float> && t.scalar_type() != at::kFloat) bad_value("%s must be fp32", name);
  if ((size_t)t.element_size() != sizeof(T)) bad_value("%s has elements of another size", name);
  if (count) *count = t.numel();
  return static_cast<T*>(t.data_ptr());
}

template <typename T>
T* matrix(PyObject* o, const char* name, int64_t& rows, int64_t& cols) {
  T* p = address<T>(o, name);
  if (!p && o == Py_None) bad_value("%s must not be None", name);
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.dim() != 2) bad_value("%s must have two dimensions", name);
  rows = t.size(0);
  cols = t.size(1);
  return p;
}

void bf16_rows(const at::Tensor& t, int64_t heads, int64_t dim, const char* name) {
  const at::ScalarType type = t.scalar_type();
  if (type != at::kBFloat16 && type != at::kShort && type != at::kUInt16) bad_value("%s must be bf16 or its bits", name);
  if (t.dim() != 3 || t.size(1) != heads || t.size(2) != dim) {
    PyErr_Format(PyExc_ValueError, "%s must be [tokens, %lld, %lld]", name, (long long)heads, (long long)dim);
    throw Bad{};
  }
}

// bf16 rows [tokens, heads, dim] whose heads are contiguous.
struct Rows {
  const uint16_t* p = nullptr;
  int64_t stride = 0, n = 0;
  Rows(PyObject* o, int64_t heads, int64_t dim, const char* name) {
    const at::Tensor& t = tensor(o, name);
    bf16_rows(t, heads, dim, name);
    p = static_cast<const uint16_t*>(t.data_ptr());
    n = t.size(0);
    stride = heads * dim;  // that of a single token is arbitrary
    if (n == 0) return;
    if (t.stride(2) != 1 || (t.stride(1) != dim && heads != 1)) bad_value("%s: a token's heads must be contiguous", name);
    if (n > 1) stride = t.stride(0);
  }
  Rows() = default;
};

uint16_t* out_rows(PyObject* o, int64_t tokens, int64_t heads, int64_t dim, const char* name) {
  uint16_t* p = address<uint16_t>(o, name);
  if (o == Py_None) bad_value("%s must not be None", name);
  const at::Tensor& t = THPVariable_Unpack(o);
  bf16_rows(t, heads, dim, name);
  if (t.size(0) != tokens) bad_value("%s has another number of tokens", name);
  return p;
}

void same(int64_t a, int64_t b, const char* name) {
  if (a != b) bad_value("%s has another number of entries", name);
}

int32_t to_int32(int64_t n, const char* name) {
  if (n > INT32_MAX) bad_value("%s has over 2^31 entries", name);
  return (int32_t)n;
}

// A ctypes structure, by its bytes.
template <typename T>
T structure(PyObject* o, const char* name) {
  Py_buffer view;
  if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw Bad{};
  T r;
  const bool fits = view.len == (Py_ssize_t)sizeof(T);
  if (fits) memcpy(&r, view.buf, sizeof(T));
  PyBuffer_Release(&view);
  if (!fits) bad_value("%s is another structure", name);
  return r;
}

// A cache as KVCache gives it, its tensors' device behind it.
struct DeviceCache {
  moe_kv_cache_t cache;
  int64_t device;
};

moe_kv_cache_t kv_cache(PyObject* o) {
  const auto c = structure<DeviceCache>(o, "cache");
  on_call_device(c.device, "cache");
  return c.cache;
}

int32_t integer32(PyObject* o, const char* name) {
  const int64_t v = integer(o);
  if (v < INT32_MIN || v > INT32_MAX) bad_value("%s does not fit 32 bits", name);
  return (int32_t)v;
}

float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Bad{};
  return (float)v;
}

bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Bad{};
  return v != 0;
}

int32_t* status_of(PyObject* o) { return address<int32_t>(o, "dev_status"); }

// The functions proper, and their entries for Python: the number of arguments is
// checked, and no C++ exception passes.
template <moe_status_t (*kCall)(PyObject* const*), int kArgs>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != kArgs) {
    PyErr_Format(PyExc_TypeError, "%d arguments expected, %zd given", kArgs, n);
    return nullptr;
  }
  const OwnStream own(a[kArgs - 1]);
  try {
    return PyLong_FromLong(kCall(a));
  } catch (const Bad&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}

// dims, q, k, positions, table, layout, q_out, k_out, dev_status, stream
moe_status_t rope(PyObject* const* a) {
  const auto d = structure<moe_attn_dims_t>(a[0], "dims");
  int64_t n, n_pos, rot;
  const int32_t* positions = address<int32_t>(a[3], "positions", &n);
  const float* table = matrix<float>(a[4], "table", n_pos, rot);
  Rows q, k;
  uint16_t *qo = nullptr, *ko = nullptr;
  // an output without its input is passed on, for the call to refuse
  if (a[1] != Py_None) {
    q = Rows(a[1], d.q_heads, d.head_dim, "q");
    same(q.n, n, "q");
  }
  if (a[1] != Py_None || a[6] != Py_None) qo = out_rows(a[6], n, d.q_heads, d.head_dim, "q_out");
  if (a[2] != Py_None) {
    k = Rows(a[2], d.kv_heads, d.head_dim, "k");
    same(k.n, n, "k");
  }
  if (a[2] != Py_None || a[7] != Py_None) ko = out_rows(a[7], n, d.kv_heads, d.head_dim, "k_out");
  return moe_rope(d, to_int32(n, "positions"), q.p, q.stride, k.p, k.stride, positions, table, to_int32(n_pos, "table"),
                  to_int32(rot, "table"), (moe_rope_layout_t)integer32(a[5], "layout"), qo, ko, status_of(a[8]),
                  stream());
}

// dims, q, k, v, positions, table, layout, slots, cache, q_out, k_out, dev_status, stream
moe_status_t rope_cache(PyObject* const* a) {
  const auto d = structure<moe_attn_dims_t>(a[0], "dims");
  int64_t n, n_slots, n_pos, rot;
  const int32_t *positions = address<int32_t>(a[4], "positions", &n), *slots = address<int32_t>(a[7], "slots", &n_slots);
  const float* table = matrix<float>(a[5], "table", n_pos, rot);
  const Rows q(a[1], d.q_heads, d.head_dim, "q"), k(a[2], d.kv_heads, d.head_dim, "k"), v(a[3], d.kv_heads, d.head_dim, "v");
  same(q.n, n, "q");
  same(k.n, n, "k");
  same(v.n, n, "v");
  same(n_slots, n, "slots");
  uint16_t* qo = out_rows(a[9], n, d.q_heads, d.head_dim, "q_out");
  uint16_t* ko = a[10] == Py_None ? nullptr : out_rows(a[10], n, d.kv_heads, d.head_dim, "k_out");
  return moe_rope_cache(d, to_int32(n, "positions"), q.p, q.stride, k.p, k.stride, v.p, v.stride, positions, table,
                        to_int32(n_pos, "table"), to_int32(rot, "table"), (moe_rope_layout_t)integer32(a[6], "layout"), slots,
                        kv_cache(a[8]), qo, ko, status_of(a[11]), stream());
}

// dims, cache, page_table, cu, k_out, v_out, dev_status, stream
moe_status_t cache_read(PyObject* const* a) {
  const auto d = structure<moe_attn_dims_t>(a[0], "dims");
  int64_t batch, width, n;
  const int32_t* pages = matrix<int32_t>(a[2], "page_table", batch, width);
  const int32_t* cu = address<int32_t>(a[3], "cu", &n);
  same(n, batch + 1, "cu");
  const at::Tensor& k = tensor(a[4], "k_out");
  const int64_t tokens = k.dim() == 3 ? k.size(0) : -1;
  uint16_t* ko = out_rows(a[4], tokens, d.kv_heads, d.head_dim, "k_out");
  uint16_t* vo = out_rows(a[5], tokens, d.kv_heads, d.head_dim, "v_out");
  return moe_cache_read(d, kv_cache(a[1]), pages, to_int32(batch, "page_table"),
                        to_int32(width, "page_table"), cu, to_int32(tokens, "k_out"), ko, vo, status_of(a[6]), stream());
}

// dims, q, k, v, cu_q, cu_k, max_k, scale, out, ws, causal, dev_status, stream
moe_status_t attn_prefill(PyObject* const* a) {
  const auto d = structure<moe_attn_dims_t>(a[0], "dims");
  const Rows q(a[1], d.q_heads, d.head_dim, "q"), k(a[2], d.kv_heads, d.head_dim, "k"), v(a[3], d.kv_heads, d.head_dim, "v");
  same(v.n, k.n, "v");
  int64_t n, m, ws_bytes;
  const int32_t *cu_q = address<int32_t>(a[4], "cu_q", &n), *cu_k = address<int32_t>(a[5], "cu_k", &m);
  same(m, n, "cu_k");
  uint8_t* ws = address<uint8_t>(a[9], "ws", &ws_bytes);
  return moe_attn_prefill(d, to_int32(n, "cu_q") - 1, to_int32(q.n, "q"), to_int32(k.n, "k"), integer32(a[6], "max_k"), q.p,
                          q.stride, k.p, k.stride, v.p, v.stride, cu_q, cu_k, real(a[7]), truth(a[10]),
                          out_rows(a[8], q.n, d.q_heads, d.head_dim, "out"), status_of(a[11]), ws, (size_t)ws_bytes,
                          stream());
}

// dims, q, cache, page_table, lens, max_len, scale, out, ws, prefix_pages, prefix_len, dev_status, stream
moe_status_t attn_decode(PyObject* const* a) {
  const auto d = structure<moe_attn_dims_t>(a[0], "dims");
  const auto c = kv_cache(a[2]);
  int64_t batch, width, n, n_prefix, ws_bytes;
  const int32_t* pages = matrix<int32_t>(a[3], "page_table", batch, width);
  const Rows q(a[1], d.q_heads, d.head_dim, "q");
  same(q.n, batch, "q");
  const int32_t* lens = address<int32_t>(a[4], "lens", &n);
  same(n, batch, "lens");
  const int32_t* prefix = address<int32_t>(a[9], "prefix_pages", &n_prefix);
  const int32_t prefix_len = integer32(a[10], "prefix_len");
  if (prefix_len > 0 && n_prefix * c.page_size < prefix_len) bad_value("%s must hold the prefix's tokens", "prefix_pages");
  uint8_t* ws = address<uint8_t>(a[8], "ws", &ws_bytes);
  return moe_attn_decode(d, to_int32(batch, "page_table"), q.p, q.stride, c, pages, to_int32(width, "page_table"), lens,
                         integer32(a[5], "max_len"), prefix, prefix_len, real(a[6]),
                         out_rows(a[7], batch, d.q_heads, d.head_dim, "out"), status_of(a[11]), ws, (size_t)ws_bytes,
                         stream());
}

template <moe_status_t (*kCall)(PyObject* const*), int kArgs>
constexpr PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<kCall, kArgs>)), METH_FASTCALL, nullptr};
}

PyMethodDef kMethods[] = {method<rope, 10>("rope"),
                          method<rope_cache, 13>("rope_cache"),
                          method<cache_read, 8>("cache_read"),
                          method<attn_prefill, 13>("attn_prefill"),
                          method<attn_decode, 13>("attn_decode"),
                          {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_binding", "The attention calls of libmoe.so on torch tensors.", -1, kMethods};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&kModule); }

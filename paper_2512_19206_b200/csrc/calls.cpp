// The calls of a decode step without ctypes: argument marshalling for CPython, nothing else.
//
// A call on a small cache is bound by the host: its kernels take 3 to 4 us and the launch about 2.  ctypes converts ten
// arguments in 2.6 us (measured on a null handle) and the address of a tensor costs 0.4 us of Python; here both
// are a few attribute lookups in C (0.15 us on the null handle).  decode_attention on one sequence of 1024 tokens, calls
// one after the other: 6.30 -> 5.26 us; calls whose GPU work is longer than the host's are unchanged.  Only the calls that a generation loop makes per layer and token (or draft) are here; the
// others move enough data for ctypes not to matter.
//
// The calls of the paged cache and of the partial rotation take up to thirteen tensors each, whose shapes, types and devices cost 0.5 us apiece in Python: append 10.8 us
// of the host, attention 10.3, before any launch.  They read them through the tensor type's DLPack exchange table (a published C interface: one call fills in address, shape,
// strides, type and device) and check everything here.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/dlpack.h>      // (the interface's declarations alone, plain C)

#include <string>
#include <vector>

#include "../../include/mixkvq.h"

namespace {

PyObject *s_is_cuda, *s_is_contiguous, *s_data_ptr;

// Handle and stream: an int, or None for a null pointer.
bool raw(PyObject* o, void** p) {
  *p = o == Py_None ? nullptr : PyLong_AsVoidPtr(o);
  return *p || !PyErr_Occurred();
}

// The address of a contiguous CUDA tensor (None: a null pointer, which the library refuses).
bool address(PyObject* o, void** p) {
  if (o == Py_None) {
    *p = nullptr;
    return true;
  }
  PyObject* x = PyObject_GetAttr(o, s_is_cuda);
  if (!x) return false;
  int yes = PyObject_IsTrue(x);
  Py_DECREF(x);
  if (yes > 0) {
    x = PyObject_CallMethodNoArgs(o, s_is_contiguous);
    if (!x) return false;
    yes = PyObject_IsTrue(x);
    Py_DECREF(x);
  }
  if (yes < 0) return false;
  if (!yes) {
    PyErr_SetString(PyExc_AssertionError, "a contiguous CUDA tensor is needed");
    return false;
  }
  x = PyObject_CallMethodNoArgs(o, s_data_ptr);
  if (!x) return false;
  *p = PyLong_AsVoidPtr(x);
  Py_DECREF(x);
  return *p || !PyErr_Occurred();
}

bool integer(PyObject* o, int* i) {
  *i = static_cast<int>(PyLong_AsUnsignedLongMask(o));
  return !PyErr_Occurred();
}

bool size(PyObject* o, size_t* n) {
  *n = PyLong_AsSize_t(o);
  return !PyErr_Occurred();
}

bool real(PyObject* o, float* f) {
  if (PyFloat_CheckExact(o)) {
    *f = static_cast<float>(PyFloat_AS_DOUBLE(o));
    return true;
  }
  PyObject* x = PyNumber_Float(o);
  if (!x) return false;
  *f = static_cast<float>(PyFloat_AS_DOUBLE(x));
  Py_DECREF(x);
  return true;
}

bool count_is(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) PyErr_Format(PyExc_TypeError, "%zd arguments are needed, %zd were given", want, n);
  return n == want;
}

mixkvq_cache* cache_of(void* p) { return static_cast<mixkvq_cache*>(p); }

// (handle, layer, q, out, scale, workspace, workspace bytes, stream)
PyObject* decode_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *h, *q, *out, *ws, *st;
  int layer, rc;
  float scale;
  size_t bytes;
  if (!count_is(n, 8) || !raw(a[0], &h) || !integer(a[1], &layer) || !address(a[2], &q) || !address(a[3], &out) ||
      !real(a[4], &scale) || !address(a[5], &ws) || !size(a[6], &bytes) || !raw(a[7], &st))
    return nullptr;
  Py_BEGIN_ALLOW_THREADS
  rc = mixkvq_decode_attention(cache_of(h), layer, q, static_cast<float*>(out), scale, ws, bytes, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// (handle, layer, k, v, q, out, scale, workspace, workspace bytes, stream)
PyObject* decode_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *h, *k, *v, *q, *out, *ws, *st;
  int layer, rc;
  float scale;
  size_t bytes;
  if (!count_is(n, 10) || !raw(a[0], &h) || !integer(a[1], &layer) || !address(a[2], &k) || !address(a[3], &v) ||
      !address(a[4], &q) || !address(a[5], &out) || !real(a[6], &scale) || !address(a[7], &ws) || !size(a[8], &bytes) ||
      !raw(a[9], &st))
    return nullptr;
  Py_BEGIN_ALLOW_THREADS
  rc = mixkvq_decode_step(cache_of(h), layer, k, v, q, static_cast<float*>(out), scale, ws, bytes, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// (handle, layer, k, v, q, cos, sin, position, out, scale, workspace, workspace bytes, stream)
PyObject* rope_decode_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *h, *k, *v, *q, *cos, *sin, *out, *ws, *st;
  int layer, pos, rc;
  float scale;
  size_t bytes;
  if (!count_is(n, 13) || !raw(a[0], &h) || !integer(a[1], &layer) || !address(a[2], &k) || !address(a[3], &v) ||
      !address(a[4], &q) || !address(a[5], &cos) || !address(a[6], &sin) || !integer(a[7], &pos) ||
      !address(a[8], &out) || !real(a[9], &scale) || !address(a[10], &ws) || !size(a[11], &bytes) ||
      !raw(a[12], &st))
    return nullptr;
  Py_BEGIN_ALLOW_THREADS
  rc = mixkvq_rope_decode_step(cache_of(h), layer, k, v, q, static_cast<const float*>(cos), static_cast<const float*>(sin),
                               pos, static_cast<float*>(out), scale, ws, bytes, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// (handle, layer, k, v, q, tokens, stream)
PyObject* quantize_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *h, *k, *v, *q, *st;
  int layer, tokens, rc;
  if (!count_is(n, 7) || !raw(a[0], &h) || !integer(a[1], &layer) || !address(a[2], &k) || !address(a[3], &v) ||
      !address(a[4], &q) || !integer(a[5], &tokens) || !raw(a[6], &st))
    return nullptr;
  Py_BEGIN_ALLOW_THREADS
  rc = mixkvq_quantize_append(cache_of(h), layer, k, v, q, tokens, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// Whole numbers of a sequence, as Int.
template <typename Int>
bool whole_numbers(PyObject* o, std::vector<Int>* v) {
  PyObject* x = PySequence_Fast(o, "a sequence of whole numbers is needed");
  if (!x) return false;
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(x);
  bool ok = true;
  try {
    v->resize((size_t)n);
  } catch (...) {
    PyErr_NoMemory();
    ok = false;
  }
  for (Py_ssize_t i = 0; ok && i < n; ++i) {
    int over = 0;
    const long long value = PyLong_AsLongLongAndOverflow(PySequence_Fast_GET_ITEM(x, i), &over);
    if (PyErr_Occurred()) {
      ok = false;
    } else if (over || value != (long long)(Int)value) {
      PyErr_SetString(PyExc_OverflowError, "a number is out of range");
      ok = false;
    } else {
      (*v)[(size_t)i] = (Int)value;
    }
  }
  Py_DECREF(x);
  return ok;
}

// (whether the chunk is appended, handle, layer, k, v, q, tokens, counts or None, out, output type, scale, scratch, scratch bytes, stream)
PyObject* chunk(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *h, *k, *v, *q, *out, *scratch, *st;
  int append, layer, tokens, type, rc;
  float scale;
  size_t bytes;
  std::vector<int32_t> counts;
  if (!count_is(n, 14) || !integer(a[0], &append) || !raw(a[1], &h) || !integer(a[2], &layer) || !address(a[3], &k) || !address(a[4], &v) ||
      !address(a[5], &q) || !integer(a[6], &tokens) || (a[7] != Py_None && !whole_numbers(a[7], &counts)) || !address(a[8], &out) ||
      !integer(a[9], &type) || !real(a[10], &scale) || !address(a[11], &scratch) || !size(a[12], &bytes) || !raw(a[13], &st))
    return nullptr;
  const int32_t* per_sequence = a[7] != Py_None ? counts.data() : nullptr;
  Py_BEGIN_ALLOW_THREADS
  rc = append ? mixkvq_chunk_step(cache_of(h), layer, k, v, q, tokens, per_sequence, out, type, scale, scratch, bytes, st)
              : mixkvq_chunk_attention(cache_of(h), layer, k, v, q, tokens, per_sequence, out, type, scale, scratch, bytes, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// (handle, addresses of q, k, v, their nine strides, tokens, addresses of cos and sin, positions in the tables, address of the coordinates, axes, the axis
// of every pair (bytes), addresses of the outputs, stream)
PyObject* rope_axes(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *p[10], *st;
  int tokens, positions, axes, rc;
  std::vector<int64_t> strides;
  char* pairs;
  Py_ssize_t n_pairs;
  if (!count_is(n, 16) || !raw(a[0], &p[0]) || !raw(a[1], &p[1]) || !raw(a[2], &p[2]) || !raw(a[3], &p[3]) || !whole_numbers(a[4], &strides) ||
      !integer(a[5], &tokens) || !raw(a[6], &p[4]) || !raw(a[7], &p[5]) || !integer(a[8], &positions) || !raw(a[9], &p[6]) || !integer(a[10], &axes) ||
      PyBytes_AsStringAndSize(a[11], &pairs, &n_pairs) || !raw(a[12], &p[7]) || !raw(a[13], &p[8]) || !raw(a[14], &p[9]) || !raw(a[15], &st))
    return nullptr;
  if (strides.size() != 9 || n_pairs != 64) {
    PyErr_SetString(PyExc_ValueError, "nine strides and 64 channel pairs are needed");
    return nullptr;
  }
  Py_BEGIN_ALLOW_THREADS
  rc = mixkvq_rope_axes(cache_of(p[0]), p[1], p[2], p[3], strides.data(), tokens, static_cast<const float*>(p[4]), static_cast<const float*>(p[5]),
                        positions, static_cast<const int32_t*>(p[6]), axes, reinterpret_cast<const uint8_t*>(pairs), p[7], p[8], p[9], st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// ---- Tensors by the exchange table of their type.
const DLPackExchangeAPI* g_exchange;
PyTypeObject* g_tensor_type;

bool exchange() {
  if (g_exchange) return true;
  PyObject* torch = PyImport_ImportModule("torch");
  if (!torch) return false;
  PyObject* type = PyObject_GetAttrString(torch, "Tensor");
  Py_DECREF(torch);
  if (!type) return false;
  PyObject* capsule = PyObject_GetAttrString(type, "__dlpack_c_exchange_api__");
  const DLPackExchangeAPI* api = capsule ? static_cast<const DLPackExchangeAPI*>(PyCapsule_GetPointer(capsule, "dlpack_exchange_api")) : nullptr;
  Py_XDECREF(capsule);
  if (!api || api->header.version.major != DLPACK_MAJOR_VERSION || !api->dltensor_from_py_object_no_sync || !api->current_work_stream) {
    Py_DECREF(type);
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "torch's DLPack exchange table is of another version than this module was built for");
    return false;
  }
  g_tensor_type = reinterpret_cast<PyTypeObject*>(type);      // (kept)
  g_exchange = api;
  return true;
}

enum Kind { kBf16, kFloat, kInt32, kUint8, kBf16OrFloat };

struct View {
  DLTensor t{};
  bool given = false;
  void* p() const { return given ? static_cast<char*>(t.data) + t.byte_offset : nullptr; }
  int64_t stride(int i) const { return t.strides[i]; }
  bool is_float() const { return t.dtype.code == kDLFloat; }
  bool of(Kind k) const {
    const DLDataType& d = t.dtype;
    if (d.lanes != 1) return false;
    const bool bf16 = d.code == kDLBfloat && d.bits == 16, f32 = d.code == kDLFloat && d.bits == 32;
    switch (k) {
      case kBf16: return bf16;
      case kFloat: return f32;
      case kInt32: return d.code == kDLInt && d.bits == 32;
      case kUint8: return d.code == kDLUInt && d.bits == 8;
      default: return bf16 || f32;
    }
  }
  bool contiguous() const {
    for (int i = 0; i < t.ndim; ++i)
      if (t.shape[i] == 0) return true;
    int64_t n = 1;
    for (int i = t.ndim - 1; i >= 0; --i) {
      if (t.shape[i] != 1 && t.strides[i] != n) return false;
      n *= t.shape[i];
    }
    return true;
  }
};

// What a call is made on: the handle, the device of its memory and the heads.
struct Owner {
  const char* call;
  void* handle;
  DLDevice device;
  int64_t hq, hkv;
};

bool refuse(const Owner& o, const char* what, const char* must, const std::vector<int64_t>& shape = {}) {
  std::string text = std::string(o.call) + ": " + what + " must be " + must;
  if (!shape.empty()) {
    text += " [";
    for (size_t i = 0; i < shape.size(); ++i) text += (i ? ", " : "") + (shape[i] < 0 ? std::string("any") : std::to_string(shape[i]));
    text += "]";
  }
  text += o.device.device_type == kDLCUDA ? " on cuda:" + std::to_string(o.device.device_id) : std::string(" on the CPU");
  PyErr_SetString(PyExc_ValueError, text.c_str());
  return false;
}

// A tensor (None only where `optional`) of this type on the owner's device; its own type and shape errors name `must`.
bool tensor(const Owner& o, PyObject* x, View* v, Kind kind, int ndim, const char* what, const char* must, bool optional = false) {
  v->given = false;
  if (x == Py_None && optional) return true;
  if (!exchange()) return false;
  if (!PyObject_TypeCheck(x, g_tensor_type)) return refuse(o, what, must);
  if (g_exchange->dltensor_from_py_object_no_sync(x, &v->t)) return false;
  v->given = true;
  if (v->t.ndim != ndim || !v->of(kind) || v->t.device.device_type != o.device.device_type || v->t.device.device_id != o.device.device_id || (ndim && !v->t.strides))
    return refuse(o, what, must);
  return true;
}
bool shaped(const Owner& o, const View& v, const char* what, const char* must, const std::vector<int64_t>& shape) {
  for (int i = 0; i < v.t.ndim; ++i)
    if (shape[(size_t)i] >= 0 && v.t.shape[i] != shape[(size_t)i]) return refuse(o, what, must, shape);
  return true;
}

// Rows [B, heads, n, 128] of bf16 numbers, any strides with a contiguous last dimension, or contiguous ones.
bool rows(const Owner& o, PyObject* x, View* v, int64_t B, int64_t heads, int64_t n, bool packed, const char* what, bool optional = false, Kind kind = kBf16) {
  const char* must = kind == kBf16OrFloat ? "a contiguous float32 or bfloat16 tensor" : packed ? "a contiguous bfloat16 tensor" : "a bfloat16 tensor with a contiguous last dimension";
  if (!tensor(o, x, v, kind, 4, what, must, optional)) return false;
  if (!v->given) return true;
  if (!shaped(o, *v, what, must, {B, heads, n, 128})) return false;
  if (packed ? !v->contiguous() : v->stride(3) != 1) return refuse(o, what, must, {B, heads, n, 128});
  return true;
}
void strides_of(const View& v, int64_t* s) {
  for (int i = 0; i < 3; ++i) s[i] = v.given ? v.stride(i) : 0;
}

bool vector_of(const Owner& o, PyObject* x, View* v, int64_t B, const char* what, bool optional) {
  const char* must = "a contiguous int32 tensor";
  if (!tensor(o, x, v, kInt32, 1, what, must, optional)) return false;
  return !v->given || (shaped(o, *v, what, must, {B}) && (v->contiguous() || refuse(o, what, must, {B})));
}

// The sequences of a call: pages (whose rows say how many sequences), lens, counts.
bool sequences(const Owner& o, PyObject* pages, PyObject* lens, PyObject* counts, int64_t n, mixkvq_paged_sequences* s) {
  View p, l, c;
  const char* must = "an int32 [sequences, pages] tensor with contiguous rows";
  if (!tensor(o, pages, &p, kInt32, 2, "pages", must)) return false;
  const int64_t B = p.t.shape[0], P = p.t.shape[1], stride = B > 1 ? p.stride(0) : P;
  if (P < 1 || (P > 1 && p.stride(1) != 1)) return refuse(o, "pages", must);
  if (B > INT32_MAX || P > INT32_MAX || stride > INT32_MAX || stride < P || n > INT32_MAX) return refuse(o, "pages", "smaller, and its rows apart");
  if (!vector_of(o, lens, &l, B, "lens", false) || !vector_of(o, counts, &c, B, "counts", true)) return false;
  *s = mixkvq_paged_sequences{(int32_t)B, (int32_t)n, static_cast<const int32_t*>(p.p()), (int32_t)P, (int32_t)stride, static_cast<const int32_t*>(l.p()),
                              static_cast<const int32_t*>(c.p())};
  return true;
}

// cos, sin (both None: no rotation, *given null), positions (None: not given)
bool rotation(const Owner& o, PyObject* cos, PyObject* sin, PyObject* positions, PyObject* interleaved, int64_t B, int64_t n, mixkvq_rotation* r, mixkvq_rotation** given) {
  *given = nullptr;
  if ((cos == Py_None) != (sin == Py_None) || (cos == Py_None && positions != Py_None)) {
    PyErr_Format(PyExc_ValueError, "%s: cos and sin come together, positions with them", o.call);
    return false;
  }
  if (cos == Py_None) return true;
  View c, s, p;
  const char *must = "a contiguous float32 table, cos and sin alike,", *ints = "a contiguous int32 tensor";
  if (!tensor(o, cos, &c, kFloat, 2, "cos", must) || !tensor(o, sin, &s, kFloat, 2, "sin", must)) return false;
  if (!c.contiguous() || !s.contiguous() || c.t.shape[0] != s.t.shape[0] || c.t.shape[1] != s.t.shape[1] || c.t.shape[0] > INT32_MAX || c.t.shape[1] > 64)
    return refuse(o, "cos and sin", must);
  if (!tensor(o, positions, &p, kInt32, 2, "positions", ints, true)) return false;
  if (p.given && !(shaped(o, p, "positions", ints, {B, n}) && (p.contiguous() || refuse(o, "positions", ints, {B, n})))) return false;
  const int side = PyObject_IsTrue(interleaved);
  if (side < 0) return false;
  *r = mixkvq_rotation{static_cast<const float*>(c.p()), static_cast<const float*>(s.p()), static_cast<const int32_t*>(p.p()), (int32_t)c.t.shape[0], (int32_t)(2 * c.t.shape[1]), side, 0};
  *given = r;
  return true;
}

// The owner as the binding describes it: (handle or None, device type, device index, query heads, KV heads)
bool owner(PyObject* x, const char* call, Owner* o) {
  o->call = call;
  int type, index, hq, hkv;
  if (!PyTuple_Check(x) || PyTuple_GET_SIZE(x) != 5) {
    PyErr_SetString(PyExc_TypeError, "a tuple of five says what the call is made on");
    return false;
  }
  if (!raw(PyTuple_GET_ITEM(x, 0), &o->handle) || !integer(PyTuple_GET_ITEM(x, 1), &type) || !integer(PyTuple_GET_ITEM(x, 2), &index) || !integer(PyTuple_GET_ITEM(x, 3), &hq) ||
      !integer(PyTuple_GET_ITEM(x, 4), &hkv))
    return false;
  o->device = DLDevice{static_cast<DLDeviceType>(type), index};
  o->hq = hq;
  o->hkv = hkv;
  return true;
}
// The device's current stream.
bool stream_of(const Owner& o, void** st) {
  *st = nullptr;
  return o.device.device_type != kDLCUDA || (exchange() && g_exchange->current_work_stream(kDLCUDA, o.device.device_id, st) == 0);
}

mixkvq_paged* paged_of(void* p) { return static_cast<mixkvq_paged*>(p); }
int64_t tokens_of(PyObject* x) {                 // of a [B, heads, n, 128] tensor; what is none is refused later
  if (!exchange() || !PyObject_TypeCheck(x, g_tensor_type)) {
    PyErr_Clear();
    return 0;
  }
  DLTensor t{};
  if (g_exchange->dltensor_from_py_object_no_sync(x, &t)) {
    PyErr_Clear();
    return 0;
  }
  return t.ndim == 4 ? t.shape[2] : 0;
}

// (positions, rotated channels, kind, base, factor, original, low, high, attention factor, start, cos, sin, device type, device index)
PyObject* rope_tables(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count_is(n, 14)) return nullptr;
  int count, type, index, rc;
  mixkvq_rope_scaling sc{};
  Owner o{"rope_tables", nullptr, {}, 0, 0};
  if (!integer(a[0], &count) || !integer(a[1], &sc.rotary_dim) || !integer(a[2], &sc.kind) || !integer(a[12], &type) || !integer(a[13], &index)) return nullptr;
  double* real[6] = {&sc.base, &sc.factor, &sc.original, &sc.low, &sc.high, &sc.attention_factor};
  for (int i = 0; i < 6; ++i) {
    *real[i] = PyFloat_AsDouble(a[3 + i]);
    if (PyErr_Occurred()) return nullptr;
  }
  const long long start = PyLong_AsLongLong(a[9]);
  if (PyErr_Occurred()) return nullptr;
  o.device = DLDevice{static_cast<DLDeviceType>(type), index};
  View t[2];
  void* st;
  for (int i = 0; i < 2; ++i) {
    const char* must = "a contiguous float32 tensor";
    if (!tensor(o, a[10 + i], &t[i], kFloat, 2, "an output", must) || !shaped(o, t[i], "an output", must, {count, sc.rotary_dim / 2})) return nullptr;
    if (!t[i].contiguous()) {
      refuse(o, "an output", must);
      return nullptr;
    }
  }
  if (!stream_of(o, &st)) return nullptr;
  Py_BEGIN_ALLOW_THREADS
  rc = mixkvq_rope_tables(&sc, start, count, static_cast<float*>(t[0].p()), static_cast<float*>(t[1].p()), st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// (owner, batch, q, k, v or None, cos, sin, positions, interleaved, outputs of q, k, v)
PyObject* rope_partial(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Owner o;
  int batch, rc;
  if (!count_is(n, 12) || !owner(a[0], "rope_partial", &o) || !integer(a[1], &batch)) return nullptr;
  const int64_t tokens = tokens_of(a[2]);
  if ((a[4] == Py_None) != (a[11] == Py_None)) {
    PyErr_SetString(PyExc_ValueError, "rope_partial: an input and its output come together");
    return nullptr;
  }
  View in[3], out[3];
  const char *names[3] = {"q", "k", "v"}, *outs[3] = {"the output of q", "the output of k", "the output of v"};
  int64_t strides[9];
  for (int i = 0; i < 3; ++i) {
    const int64_t heads = i == 0 ? o.hq : o.hkv;
    if (!rows(o, a[2 + i], &in[i], batch, heads, tokens, false, names[i], i == 2) || !rows(o, a[9 + i], &out[i], batch, heads, tokens, true, outs[i], i == 2)) return nullptr;
    strides_of(in[i], strides + 3 * i);
  }
  mixkvq_rotation r, *turn;
  void* st;
  if (a[7] == Py_None) {
    PyErr_SetString(PyExc_ValueError, "rope_partial: positions are needed");
    return nullptr;
  }
  if (!rotation(o, a[5], a[6], a[7], a[8], batch, tokens, &r, &turn) || !stream_of(o, &st)) return nullptr;
  Py_BEGIN_ALLOW_THREADS
  rc = mixkvq_rope_partial(cache_of(o.handle), in[0].p(), in[1].p(), in[2].p(), strides, (int)tokens, turn, out[0].p(), out[1].p(), out[2].p(), st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// What append and step share: k, v, q or None, pages, lens, counts, cos, sin, positions, interleaved, the rotated queries or None
struct Append {
  View k, v, q, q_out;
  int64_t strides[9];
  mixkvq_paged_sequences s;
  mixkvq_rotation r, *turn;
  void* st;
};
bool append_arguments(const Owner& o, PyObject* const* a, Append* x) {
  const int64_t n = tokens_of(a[0]);
  if (!sequences(o, a[3], a[4], a[5], n, &x->s)) return false;
  if ((a[2] == Py_None) != (a[10] == Py_None)) {
    PyErr_Format(PyExc_ValueError, "%s: q and q_out come together", o.call);
    return false;
  }
  if (!rows(o, a[0], &x->k, x->s.batch, o.hkv, n, false, "k") || !rows(o, a[1], &x->v, x->s.batch, o.hkv, n, false, "v") ||
      !rows(o, a[2], &x->q, x->s.batch, o.hq, n, false, "q", true) || !rows(o, a[10], &x->q_out, x->s.batch, o.hq, n, true, "q_out", true) ||
      !rotation(o, a[6], a[7], a[8], a[9], x->s.batch, n, &x->r, &x->turn) || !stream_of(o, &x->st))
    return false;
  strides_of(x->q, x->strides);
  strides_of(x->k, x->strides + 3);
  strides_of(x->v, x->strides + 6);
  return true;
}
// Output and workspace of an attention.
bool results(const Owner& o, PyObject* out, PyObject* ws, int64_t B, int64_t n, View* y, View* w) {
  if (!rows(o, out, y, B, o.hq, n, true, "out", false, kBf16OrFloat) || !tensor(o, ws, w, kUint8, 1, "the workspace", "a contiguous uint8 tensor")) return false;
  return w->contiguous() || refuse(o, "the workspace", "a contiguous uint8 tensor");
}

// (owner, layer, k, v, q, pages, lens, counts, cos, sin, positions, interleaved, q_out)
PyObject* paged_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Owner o;
  Append x;
  int layer, rc;
  if (!count_is(n, 13) || !owner(a[0], "append", &o) || !integer(a[1], &layer) || !append_arguments(o, a + 2, &x)) return nullptr;
  Py_BEGIN_ALLOW_THREADS
  rc = mixkvq_paged_append(paged_of(o.handle), layer, &x.s, x.k.p(), x.v.p(), x.q.p(), x.strides, x.turn, x.q_out.p(), x.st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// (owner, layer, pages, lens, tokens, counts, keys, values)
PyObject* paged_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Owner o;
  mixkvq_paged_sequences s;
  View k, v;
  void* st;
  int layer, tokens, rc;
  if (!count_is(n, 8) || !owner(a[0], "read", &o) || !integer(a[1], &layer) || !integer(a[4], &tokens) || !sequences(o, a[2], a[3], a[5], tokens, &s) ||
      !rows(o, a[6], &k, s.batch, o.hkv, tokens, true, "the keys' output") || !rows(o, a[7], &v, s.batch, o.hkv, tokens, true, "the values' output") || !stream_of(o, &st))
    return nullptr;
  Py_BEGIN_ALLOW_THREADS
  rc = mixkvq_paged_read(paged_of(o.handle), layer, &s, k.p(), v.p(), st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// (owner, layer, q, pages, lens, scale, counts, out, workspace)
PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Owner o;
  mixkvq_paged_sequences s;
  View q, y, w;
  void* st;
  int layer, rc;
  float scale;
  if (!count_is(n, 9) || !owner(a[0], "attention", &o) || !integer(a[1], &layer)) return nullptr;
  const int64_t tokens = tokens_of(a[2]);
  if (!sequences(o, a[3], a[4], a[6], tokens, &s) || !rows(o, a[2], &q, s.batch, o.hq, tokens, true, "q") || !real(a[5], &scale) ||
      !results(o, a[7], a[8], s.batch, tokens, &y, &w) || !stream_of(o, &st))
    return nullptr;
  Py_BEGIN_ALLOW_THREADS
  rc = mixkvq_paged_attention(paged_of(o.handle), layer, &s, q.p(), y.p(), y.is_float() ? MIXKVQ_OUT_FLOAT : MIXKVQ_OUT_BF16, scale, w.p(), (size_t)w.t.shape[0], st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// (owner, layer, k, v, q, pages, lens, counts, cos, sin, positions, interleaved, q_out, scale, out, workspace)
PyObject* paged_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Owner o;
  Append x;
  View y, w;
  int layer, rc;
  float scale;
  if (!count_is(n, 16) || !owner(a[0], "step", &o) || !integer(a[1], &layer) || !append_arguments(o, a + 2, &x) || !real(a[13], &scale) ||
      !results(o, a[14], a[15], x.s.batch, x.s.n_tokens, &y, &w))
    return nullptr;
  Py_BEGIN_ALLOW_THREADS
  rc = mixkvq_paged_step(paged_of(o.handle), layer, &x.s, x.k.p(), x.v.p(), x.q.p(), x.strides, x.turn, x.q_out.p(), y.p(),
                         y.is_float() ? MIXKVQ_OUT_FLOAT : MIXKVQ_OUT_BF16, scale, w.p(), (size_t)w.t.shape[0], x.st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

template <typename F>
PyCFunction fast(F f) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}

PyMethodDef methods[] = {{"decode_attention", fast(decode_attention), METH_FASTCALL, nullptr},
                         {"decode_step", fast(decode_step), METH_FASTCALL, nullptr},
                         {"rope_decode_step", fast(rope_decode_step), METH_FASTCALL, nullptr},
                         {"quantize_append", fast(quantize_append), METH_FASTCALL, nullptr},
                         {"chunk", fast(chunk), METH_FASTCALL, nullptr},
                         {"rope_axes", fast(rope_axes), METH_FASTCALL, nullptr},
                         {"rope_tables", fast(rope_tables), METH_FASTCALL, nullptr},
                         {"rope_partial", fast(rope_partial), METH_FASTCALL, nullptr},
                         {"paged_append", fast(paged_append), METH_FASTCALL, nullptr},
                         {"paged_read", fast(paged_read), METH_FASTCALL, nullptr},
                         {"paged_attention", fast(paged_attention), METH_FASTCALL, nullptr},
                         {"paged_step", fast(paged_step), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
  s_is_cuda = PyUnicode_InternFromString("is_cuda");
  s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  if (!s_is_cuda || !s_is_contiguous || !s_data_ptr) return nullptr;
  return PyModule_Create(&module);
}

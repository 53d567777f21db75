// Python's way to the head norm and rotation and to the paged 8-bit cache: checks of tensors and marshalling only, compiled,
// because a call's kernel is over in a few microseconds (the same checks in Python and ctypes took 7.7 us a call on the host; 3.7 so).
// The library's functions come from the loaded libdecoquant.so by address (set_up).
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>

#include "decoquant.h"

namespace {

decltype(&dq_rotate_heads) g_rotate;
decltype(&dq_paged_append) g_append;
decltype(&dq_paged_read) g_read;
decltype(&dq_paged_attention) g_attention;
PyObject* g_error;   // DQError
PyObject* g_check;   // raises for a status

struct Refused {};   // a Python error is set

template <typename... A> [[noreturn]] void refuse(const char* format, A... a) {
  PyErr_Format(g_error, format, a...);
  throw Refused{};
}

const at::Tensor& tensor(const char* name, PyObject* o) {
  if (!THPVariable_Check(o)) refuse("%s must be a tensor", name);
  return THPVariable_Unpack(o);
}
bool none(PyObject* o) { return o == Py_None; }

long long integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused{};
  return v;
}
int32_t int32(const char* name, PyObject* o) {
  const long long v = integer(o);
  if (v < INT32_MIN || v > INT32_MAX) refuse("%s does not fit 32 bits", name);
  return (int32_t)v;
}
double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused{};
  return v;
}
void* address(PyObject* o) {
  void* p = PyLong_AsVoidPtr(o);
  if (!p && PyErr_Occurred()) throw Refused{};
  return p;
}

at::ScalarType row_type(int32_t dtype) { return dtype == DQ_BF16 ? at::kBFloat16 : at::kHalf; }
const char* type_name(int32_t dtype) { return dtype == DQ_BF16 ? "bfloat16" : "float16"; }

// [rows, heads, dim] or [batch, rows, heads, dim] with channels side by side.
struct Heads {
  dq_heads c;
  int64_t dims, batch, rows;
};
Heads heads(const char* name, PyObject* o, int32_t dtype, int64_t dim, int64_t index, bool written) {
  const at::Tensor& t = tensor(name, o);
  Heads h = {};
  h.dims = t.dim();
  if (h.dims != 3 && h.dims != 4) refuse("%s must be [rows, heads, %lld] or [batch, rows, heads, %lld]", name, (long long)dim, (long long)dim);
  const at::IntArrayRef n = t.sizes(), s = t.strides();
  const int64_t at = h.dims - 3;
  h.batch = at ? n[0] : 1;
  h.rows = n[at];
  if (t.scalar_type() != row_type(dtype) || n[at + 2] != dim || t.get_device() != index)
    refuse("%s must be a torch.%s tensor on cuda:%lld with %lld channels a head", name, type_name(dtype), (long long)index, (long long)dim);
  if (h.rows > INT32_MAX || n[at + 1] > INT32_MAX || h.batch > INT32_MAX) refuse("%s has too many rows or heads", name);
  // a stride over one entry says nothing
  h.c.batch_stride = h.batch == 1 ? 0 : s[0];
  h.c.token_stride = h.rows == 1 ? 0 : s[at];
  h.c.head_stride = n[at + 1] == 1 ? 0 : s[at + 1];
  h.c.heads = (int32_t)n[at + 1];
  h.c.data = static_cast<uint16_t*>(t.data_ptr());
  if (s[at + 2] != 1 || ((h.c.batch_stride | h.c.token_stride | h.c.head_stride) & 7) || ((uintptr_t)h.c.data & 15))
    refuse("%s: channels must be neighbours, the other strides multiples of 8 elements, the data 16-byte aligned", name);
  if (written && ((h.rows > 1 && !h.c.token_stride) || (h.c.heads > 1 && !h.c.head_stride) || (h.batch > 1 && !h.c.batch_stride)))
    refuse("%s must not be an expanded tensor", name);
  return h;
}

// rows [rows, heads, head_dim] of a cache's type; heads and rows < 0: any.
Heads packed_rows(const dq_paged_cache* cache, int64_t index, const char* name, PyObject* o, int64_t n_heads, int64_t rows, bool written) {
  const Heads h = heads(name, o, cache->dtype, cache->head_dim, index, written);
  if (h.dims != 3 || (rows >= 0 && h.rows != rows) || (n_heads >= 0 && h.c.heads != n_heads)) {
    if (rows >= 0) refuse("%s must be [rows = %lld, heads, head_dim], of the heads that belong there", name, (long long)rows);
    refuse("%s must be [rows, heads, head_dim], of the heads that belong there", name);
  }
  return h;
}

// n int32 side by side.
const int32_t* vector(const char* name, PyObject* o, int64_t n, int64_t index) {
  const at::Tensor& t = tensor(name, o);
  if (t.scalar_type() != at::kInt || t.numel() != n || !t.is_contiguous() || t.get_device() != index)
    refuse("%s must hold %lld int32, side by side on cuda:%lld", name, (long long)n, (long long)index);
  return static_cast<const int32_t*>(t.data_ptr());
}

const uint16_t* weight(const char* name, PyObject* o, int32_t dtype, int64_t dim, int64_t index) {
  if (none(o)) return nullptr;
  const at::Tensor& t = tensor(name, o);
  const uint16_t* p = static_cast<const uint16_t*>(t.data_ptr());
  if (t.scalar_type() != row_type(dtype) || t.numel() != dim || !t.is_contiguous() || ((uintptr_t)p & 15) || t.get_device() != index)
    refuse("%s must be %lld contiguous torch.%s on cuda:%lld, 16-byte aligned", name, (long long)dim, type_name(dtype), (long long)index);
  return p;
}

// Norm and rotation of a call; the pointers are null where there is none.
struct Turning {
  dq_head_norm norm;
  dq_rotary rot;
  const dq_head_norm* n;
  const dq_rotary* r;
};
void turning(Turning& t, PyObject* q_weight, PyObject* k_weight, PyObject* eps, PyObject* rotary, PyObject* positions, int32_t dtype, int64_t dim,
             int64_t rows, int64_t index) {
  t = {};
  if (!none(q_weight) || !none(k_weight)) {
    t.norm = {weight("q_weight", q_weight, dtype, dim, index), weight("k_weight", k_weight, dtype, dim, index), (float)real(eps)};
    if (!(t.norm.eps >= 0.f)) refuse("eps must not be negative");
    t.n = &t.norm;
  }
  if (none(rotary)) return;
  PyObject *freq = nullptr, *axis = nullptr;              // looked at in every call: a Rotary's tensors are the caller's
  int axes = 0, interleaved = 0;
  if (!PyArg_ParseTuple(rotary, "OOii", &freq, &axis, &axes, &interleaved)) throw Refused{};
  const at::Tensor& f = tensor("inv_freq", freq);
  if (f.scalar_type() != at::kDouble || !f.is_contiguous() || f.get_device() != index) refuse("inv_freq must be contiguous float64 on cuda:%lld", (long long)index);
  if (2 * f.numel() > dim) refuse("rot_dim is larger than head_dim");
  const int rot_dim = (int)(2 * f.numel());
  t.rot.inv_freq = static_cast<const double*>(f.data_ptr());
  if (none(axis) != (axes <= 1)) refuse("several axes need axis_of_pair");
  if (!none(axis)) {
    const at::Tensor& x = tensor("axis_of_pair", axis);
    if (x.scalar_type() != at::kByte || x.numel() != f.numel() || !x.is_contiguous() || x.get_device() != index)
      refuse("axis_of_pair must be one uint8 per pair on cuda:%lld", (long long)index);
    t.rot.axis_of_pair = static_cast<const uint8_t*>(x.data_ptr());
  }
  t.rot.position_stride = rows;
  t.rot.axes = axes;
  t.rot.rot_dim = rot_dim;
  t.rot.interleaved = interleaved;
  if (!none(positions)) t.rot.positions = vector("positions (one per row and axis)", positions, axes * rows, index);
  else if (axes > 1) refuse("several axes need positions");
  t.r = &t.rot;
}

// Sizes are checked here (the library sees pointers only).
dq_paged_batch batch_of(const dq_paged_cache* cache, int64_t index, PyObject* starts, PyObject* seq_lens, PyObject* page_table, PyObject* tail_slots,
                        int64_t rows, bool uses_starts) {
  dq_paged_batch b = {};
  const int64_t n = tensor("seq_lens", seq_lens).numel();
  if (n < 1) refuse("a batch has at least one sequence");
  if (n > INT32_MAX) refuse("a batch has too many sequences");
  const at::Tensor& table = tensor("page_table", page_table);
  if (table.dim() != 2 || table.size(0) != n || table.size(1) < 1 || table.size(1) > INT32_MAX || table.scalar_type() != at::kInt || table.get_device() != index)
    refuse("page_table must be int32 [batch, pages], on the cache's GPU");
  const int64_t width = table.size(1), stride = n == 1 ? width : table.stride(0);
  if ((width > 1 && table.stride(1) != 1) || stride < width || stride > INT32_MAX) refuse("a sequence's pages must lie side by side in page_table");
  if (none(starts) && uses_starts && rows != n) refuse("without starts there is one row per sequence");
  if (none(tail_slots) && n > cache->slots) refuse("more sequences than the cache has slots");
  b.starts = none(starts) ? nullptr : vector("starts", starts, n + 1, index);
  b.seq_lens = vector("seq_lens", seq_lens, n, index);
  b.page_table = static_cast<const int32_t*>(table.data_ptr());
  b.tail_slots = none(tail_slots) ? nullptr : vector("tail_slots", tail_slots, n, index);
  b.batch = (int32_t)n;
  b.rows = (int32_t)rows;
  b.table_width = (int32_t)width;
  b.table_stride = (int32_t)stride;
  return b;
}

// call() without the interpreter's lock (a launch may wait for room in its queue); raises for its status.
template <typename F> PyObject* launch(const char* what, F call) {
  PyThreadState* const state = PyEval_SaveThread();
  const int32_t status = call();
  PyEval_RestoreThread(state);
  if (status == DQ_OK) Py_RETURN_NONE;
  PyObject* r = PyObject_CallFunction(g_check, "is", (int)status, what);
  Py_XDECREF(r);
  if (r) refuse("%s failed", what);
  throw Refused{};
}

// No C++ exception leaves a function.
template <typename F> PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F f) {
  try {
    if (n != want) {
      PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
      return nullptr;
    }
    return f();
  } catch (const Refused&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}

PyObject* rotate_heads(PyObject*, PyObject* const* a, Py_ssize_t n) {
  // q, q_out, k, k_out, positions, rotary, q_weight, k_weight, eps, index, stream
  return guarded(n, 11, [&]() -> PyObject* {
    const int64_t index = integer(a[9]);
    const at::Tensor& first = tensor("the heads", none(a[0]) ? a[2] : a[0]);
    if ((first.scalar_type() != at::kHalf && first.scalar_type() != at::kBFloat16) || index < 0) refuse("heads must be float16 or bfloat16 on a GPU");
    if (first.dim() < 1) refuse("heads must be [rows, heads, channels] or [batch, rows, heads, channels]");
    const int32_t dtype = first.scalar_type() == at::kBFloat16 ? DQ_BF16 : DQ_F16;
    const int64_t dim = first.size(-1);
    Heads h[4] = {};
    const char* const names[4] = {"q", "q_out", "k", "k_out"};
    const Heads* rows = nullptr;
    for (int i = 0; i < 4; i += 2) {
      if (none(a[i])) continue;
      h[i] = heads(names[i], a[i], dtype, dim, index, false);
      h[i + 1] = heads(names[i + 1], a[i + 1], dtype, dim, index, true);
      if (h[i + 1].dims != h[i].dims || h[i + 1].batch != h[i].batch || h[i + 1].rows != h[i].rows || h[i + 1].c.heads != h[i].c.heads)
        refuse("%s must have the shape of %s", names[i + 1], names[i]);
      if (rows && (rows->dims != h[i].dims || rows->batch != h[i].batch || rows->rows != h[i].rows)) refuse("q and k must have the same rows");
      rows = h + i;
    }
    Turning t;
    turning(t, a[6], a[7], a[8], a[5], a[4], dtype, dim, rows->batch * rows->rows, index);
    if (t.r && none(a[4])) refuse("rotate_heads needs positions");
    if (!t.r && !t.n) refuse("rotate_heads needs a rotation or a norm");
    if (rows->batch == 0 || rows->rows == 0) Py_RETURN_NONE;
    const dq_heads* c[4];
    for (int i = 0; i < 4; ++i) c[i] = none(a[i & 2]) ? nullptr : &h[i].c;
    void* const stream = address(a[10]);
    const int32_t d = (int32_t)(dim < INT32_MAX ? dim : 0);
    return launch("dq_rotate_heads", [&] {
      return g_rotate(c[0], c[1], c[2], c[3], (int32_t)rows->batch, (int32_t)rows->rows, d, dtype, t.n, t.r, stream);
    });
  });
}

PyObject* paged_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  // cache, index, k, v, starts, seq_lens, page_table, tail_slots, q, q_out, rotary, positions, q_weight, k_weight, eps, stream
  return guarded(n, 16, [&]() -> PyObject* {
    const dq_paged_cache* const cache = static_cast<const dq_paged_cache*>(address(a[0]));
    const int64_t index = integer(a[1]);
    const Heads k = packed_rows(cache, index, "k", a[2], cache->kv_heads, -1, false);
    const Heads v = packed_rows(cache, index, "v", a[3], cache->kv_heads, k.rows, false);
    const dq_paged_batch b = batch_of(cache, index, a[4], a[5], a[6], a[7], k.rows, true);
    Heads q = {}, out = {};
    if (!none(a[8])) {
      q = packed_rows(cache, index, "q", a[8], -1, k.rows, false);
      out = packed_rows(cache, index, "q_out", a[9], q.c.heads, k.rows, true);
    }
    Turning t;
    turning(t, a[12], a[13], a[14], a[10], a[11], cache->dtype, cache->head_dim, k.rows, index);
    if (k.rows == 0) Py_RETURN_NONE;
    const bool with_q = !none(a[8]);
    void* const stream = address(a[15]);
    return launch("dq_paged_append", [&] { return g_append(cache, &b, &k.c, &v.c, with_q ? &q.c : nullptr, with_q ? &out.c : nullptr, t.n, t.r, stream); });
  });
}

PyObject* paged_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  // cache, index, first, seq_lens, out_starts, page_table, tail_slots, k_out, v_out, stream
  return guarded(n, 10, [&]() -> PyObject* {
    const dq_paged_cache* const cache = static_cast<const dq_paged_cache*>(address(a[0]));
    const int64_t index = integer(a[1]);
    const Heads k = packed_rows(cache, index, "k_out", a[7], cache->kv_heads, -1, true);
    const Heads v = packed_rows(cache, index, "v_out", a[8], cache->kv_heads, k.rows, true);
    if (none(a[4])) refuse("paged_read needs out_starts");
    const dq_paged_batch b = batch_of(cache, index, a[4], a[3], a[5], a[6], k.rows, false);
    const int32_t* const first = none(a[2]) ? nullptr : vector("first", a[2], b.batch, index);
    if (k.rows == 0) Py_RETURN_NONE;
    void* const stream = address(a[9]);
    return launch("dq_paged_read", [&] { return g_read(cache, &b, first, b.starts, &k.c, &v.c, stream); });
  });
}

PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  // cache, index, q, out, starts, seq_lens, page_table, tail_slots, max_rows, max_seq_len, softmax_scale, causal, window, splits, workspace, stream
  return guarded(n, 16, [&]() -> PyObject* {
    const dq_paged_cache* const cache = static_cast<const dq_paged_cache*>(address(a[0]));
    const int64_t index = integer(a[1]);
    const Heads q = packed_rows(cache, index, "q", a[2], -1, -1, false);
    if (q.c.heads == 0 || q.c.heads % cache->kv_heads) refuse("q_heads must be a multiple of kv_heads");
    const Heads out = packed_rows(cache, index, "out", a[3], q.c.heads, q.rows, true);
    const dq_paged_batch b = batch_of(cache, index, a[4], a[5], a[6], a[7], q.rows, true);
    const at::Tensor& ws = tensor("workspace", a[14]);
    if (ws.scalar_type() != at::kByte || !ws.is_contiguous() || ws.get_device() != index) refuse("workspace must be contiguous uint8 on the cache's GPU");
    const int32_t max_rows = int32("max_rows", a[8]), max_len = int32("max_seq_len", a[9]), window = int32("window", a[12]), splits = int32("splits", a[13]);
    const int causal = PyObject_IsTrue(a[11]);
    if (causal < 0) throw Refused{};
    if (max_rows < 0 || max_len < 0 || window < 0 || (window && !causal)) refuse("max_rows, max_seq_len and window must not be negative, and a window needs causal");
    if (splits < 0 || splits > 0x7F) refuse("splits must be 0 to 64");
    if (q.rows == 0) Py_RETURN_NONE;
    const float scale = (float)real(a[10]);
    void *const work = ws.data_ptr(), *const stream = address(a[15]);
    const uint32_t flags = (causal ? DQ_PAGED_CAUSAL : 0u) | DQ_PAGED_SPLITS(splits);
    return launch("dq_paged_attention", [&] {
      return g_attention(cache, &b, &q.c, &out.c, max_rows, max_len, scale, window, work, (size_t)ws.numel(), flags, stream);
    });
  });
}

PyObject* set_up(PyObject*, PyObject* const* a, Py_ssize_t n) {
  // DQError, check(status, what), addresses of dq_rotate_heads, dq_paged_append, dq_paged_read, dq_paged_attention
  return guarded(n, 6, [&]() -> PyObject* {
    g_rotate = reinterpret_cast<decltype(g_rotate)>(address(a[2]));
    g_append = reinterpret_cast<decltype(g_append)>(address(a[3]));
    g_read = reinterpret_cast<decltype(g_read)>(address(a[4]));
    g_attention = reinterpret_cast<decltype(g_attention)>(address(a[5]));
    Py_INCREF(a[0]);
    Py_INCREF(a[1]);
    g_error = a[0];
    g_check = a[1];
    Py_RETURN_NONE;
  });
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)> PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(F)), METH_FASTCALL, nullptr};
}
PyMethodDef g_methods[] = {method<set_up>("set_up"),           method<rotate_heads>("rotate_heads"),       method<paged_append>("paged_append"),
                           method<paged_read>("paged_read"), method<paged_attention>("paged_attention"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_paged", nullptr, -1, g_methods};

}  // namespace

PyMODINIT_FUNC PyInit__paged(void) {
  PyObject* const m = PyModule_Create(&g_module);
  if (m && PyModule_AddStringConstant(m, "stamp", DQ_BIND_STAMP)) {   // of the sources it was built from
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}

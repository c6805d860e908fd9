// Marshalling of the paged calls: torch tensors -> the C entry points of pafu.h, for binding.py, which documents the calls.
// Lengths, tables and slots are read on the device, so what the C side cannot see of them (type, size, place) is checked
// here.  A decode step calls these once per layer: through ctypes, with the checks in Python, the attention call (29
// arguments) took 9.6 us on the host and the short ones 7.3; this way they take 4.0 to 4.2, of which the marshalling and the
// checks are 0.3, the Python function around them 0.2 and the rest the library's launch.
//
// The entry points' addresses come from the library that binding.py has loaded; nothing here computes or launches by itself.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <climits>

#include "pafu.h"

namespace {

struct Refused {};  // with the Python error set

[[noreturn]] void refuse(PyObject* type, const char* format, ...) {
  va_list args;
  va_start(args, format);
  PyErr_FormatV(type, format, args);
  va_end(args);
  throw Refused{};
}

decltype(&pafu_paged_tables) call_tables = nullptr;
decltype(&pafu_paged_slots) call_slots = nullptr;
decltype(&pafu_paged_append) call_append = nullptr;
decltype(&pafu_paged_attention) call_attention = nullptr;
PyObject* current_device = nullptr;  // () -> index
PyObject* current_stream = nullptr;  // (index) -> handle

long long integer(PyObject* o, long long lo = INT_MIN, long long hi = INT_MAX) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused{};
  if (v < lo || v > hi) refuse(PyExc_OverflowError, "%lld does not fit the argument", v);
  return v;
}

// The tensors of a call: all on one GPU, the current one.
struct Call {
  int device = -2;  // of the tensors so far; -2: none yet
  const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) refuse(PyExc_TypeError, "%s must be a tensor, not %s", name, Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
  }
  void place(const at::Tensor& t) {
    const int d = t.is_cuda() ? (int)t.get_device() : -1;
    if (device != -2 && d != device) device = -3;  // told last, in stream()
    else device = d;
  }
  // a contiguous list of n int32 (n < 0: of any length)
  int* list(PyObject* o, const char* name, long long n, int* length = nullptr) {
    const at::Tensor& t = tensor(o, name);
    if (t.scalar_type() != at::kInt) refuse(PyExc_TypeError, "%s must be int32, not %s", name, c10::toString(t.scalar_type()));
    if (t.dim() != 1 || !t.is_contiguous() || (n >= 0 && t.size(0) != n))
      refuse(PyExc_ValueError, n < 0 ? "%s must be a contiguous list" : "%s must be a contiguous list of %lld", name, n);
    if (t.size(0) > INT_MAX) refuse(PyExc_ValueError, "%s is too long", name);
    place(t);
    if (length) *length = (int)t.size(0);
    return static_cast<int*>(t.data_ptr());
  }
  // [n, columns] int32 with contiguous rows
  int* table(PyObject* o, long long n, int& columns, long long& ld) {
    const at::Tensor& t = tensor(o, "the block table");
    if (t.scalar_type() != at::kInt)
      refuse(PyExc_TypeError, "the block table must be int32, not %s", c10::toString(t.scalar_type()));
    if (t.dim() != 2 || t.size(0) != n || (t.size(1) > 1 && t.stride(1) != 1) || t.size(1) > INT_MAX)
      refuse(PyExc_ValueError, "the block table must be [%lld, max_pages] with contiguous rows", n);
    place(t);
    columns = (int)t.size(1);
    ld = n > 1 ? (long long)t.stride(0) : (columns > 1 ? columns : 1);
    return static_cast<int*>(t.data_ptr());
  }
  // [rows, heads, D] with contiguous rows -> token stride
  void* rows(PyObject* o, const char* name, bool f32_too, const at::Tensor*& t_out, long long& ld) {
    const at::Tensor& t = tensor(o, name);
    if (t.scalar_type() != at::kBFloat16 && !(f32_too && t.scalar_type() == at::kFloat))
      refuse(PyExc_TypeError, "%s has the unsupported dtype %s", name, c10::toString(t.scalar_type()));
    if (t.dim() != 3) refuse(PyExc_ValueError, "%s must be [rows, heads, D]", name);
    const long long heads = t.size(1), D = t.size(2);
    if ((D > 1 && t.stride(2) != 1) || (heads > 1 && t.stride(1) != D))
      refuse(PyExc_ValueError, "%s must have contiguous rows", name);
    if (t.size(0) > INT_MAX || heads > INT_MAX || D > INT_MAX) refuse(PyExc_ValueError, "%s is too long", name);
    place(t);
    ld = t.size(0) > 1 ? (long long)t.stride(0) : heads * D;
    t_out = &t;
    return t.data_ptr();
  }
  // the stream's handle, once all tensors are known
  void* stream(PyObject* given) {
    if (device == -3) refuse(PyExc_ValueError, "the tensors are on different devices");
    if (device < 0) refuse(PyExc_ValueError, "the tensors must be on the GPU");
    PyObject* index = PyObject_CallNoArgs(current_device);
    if (!index) throw Refused{};
    const long current = PyLong_AsLong(index);
    if (current != device) {
      Py_DECREF(index);
      refuse(PyExc_ValueError, "the tensors are on GPU %d and the current device is %ld", device, current);
    }
    PyObject* handle = given;
    if (given == Py_None) handle = PyObject_CallOneArg(current_stream, index);
    Py_DECREF(index);
    if (!handle) throw Refused{};
    void* s = PyLong_AsVoidPtr(handle);
    if (given == Py_None) Py_DECREF(handle);
    if (!s && PyErr_Occurred()) throw Refused{};
    return s;
  }
};

// A page pool: both tensors [n_pages, page_size, N_kv, D], of one type, shape and stride (that of an axis of length one is not
// read), elements contiguous.
struct Pool {
  void *K, *V;
  int n_pages, page_size, N, D, dtype;
  long long ld_page, ld_token, ld_head;
  Pool(Call& call, PyObject* k_obj, PyObject* v_obj) {
    const at::Tensor &k = call.tensor(k_obj, "K_pages"), &v = call.tensor(v_obj, "V_pages");
    bool alike = k.dim() == 4 && v.sizes() == k.sizes();
    for (int i = 0; alike && i < 4; ++i) alike = k.size(i) == 1 || v.stride(i) == k.stride(i);
    if (!alike || k.stride(3) != 1)
      refuse(PyExc_ValueError, "the page tensors must be [n_pages, page_size, N_kv, D] of one shape and stride, elements contiguous");
    if (v.scalar_type() != k.scalar_type() || (k.scalar_type() != at::kBFloat16 && k.scalar_type() != at::kByte))
      refuse(PyExc_TypeError, "page tensors are bfloat16 or uint8 (E4M3 codes), not %s and %s", c10::toString(k.scalar_type()),
             c10::toString(v.scalar_type()));
    for (int i = 0; i < 4; ++i)
      if (k.size(i) > INT_MAX) refuse(PyExc_ValueError, "the page tensors are too large");
    call.place(k);
    call.place(v);
    K = k.data_ptr();
    V = v.data_ptr();
    n_pages = (int)k.size(0), page_size = (int)k.size(1), N = (int)k.size(2), D = (int)k.size(3);
    ld_page = k.stride(0), ld_token = k.stride(1), ld_head = k.stride(2);
    dtype = k.scalar_type() == at::kByte ? PAFU_FP8_E4M3 : PAFU_BF16;
  }
};

// The C call runs without the interpreter's lock: a full launch queue makes it wait.
template <typename F>
PyObject* unlocked(F f) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

template <PyObject* (*F)(PyObject* const*)>
PyObject* guarded(PyObject* const* a, Py_ssize_t n, Py_ssize_t want) {
  if (n != want) {
    PyErr_Format(PyExc_TypeError, "%zd arguments instead of %zd", n, want);
    return nullptr;
  }
  try {
    return F(a);
  } catch (const Refused&) {
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// kv_len, new_len, free_pages, page_size, block_table, slots, row_start, kv_len_out, free_end, free_start, stream
PyObject* tables_of(PyObject* const* a) {
  Call c;
  int B, n_free, max_slots, columns;
  long long ld;
  const int* kv_len = c.list(a[0], "kv_len", -1, &B);
  const int* new_len = c.list(a[1], "new_len", B);
  const int* free_pages = c.list(a[2], "free_pages", -1, &n_free);
  const int page_size = (int)integer(a[3]);
  int* table = c.table(a[4], B, columns, ld);
  int* slots = c.list(a[5], "slots", -1, &max_slots);
  int* row_start = c.list(a[6], "row_start", (long long)B + 1);
  int* kv_len_out = c.list(a[7], "kv_len_out", B);
  int* free_end = c.list(a[8], "free_end", 1);
  const int* free_start = a[9] == Py_None ? nullptr : c.list(a[9], "free_start", 1);
  void* st = c.stream(a[10]);
  return unlocked([&] {
    return call_tables(st, kv_len, new_len, B, free_pages, n_free, free_start, page_size, table, columns, ld, slots, max_slots,
                       row_start, kv_len_out, free_end);
  });
}
PyObject* tables(PyObject*, PyObject* const* a, Py_ssize_t n) { return guarded<tables_of>(a, n, 11); }

// block_table, start, count, page_size, slots, row_start, stream
PyObject* slots_of(PyObject* const* a) {
  Call c;
  int B, max_slots, columns;
  long long ld;
  const int* start = c.list(a[1], "start", -1, &B);
  const int* count = c.list(a[2], "count", B);
  const int* table = c.table(a[0], B, columns, ld);
  const int page_size = (int)integer(a[3]);
  int* out = c.list(a[4], "slots", -1, &max_slots);
  int* row_start = c.list(a[5], "row_start", (long long)B + 1);
  void* st = c.stream(a[6]);
  return unlocked([&] { return call_slots(st, table, columns, ld, start, count, B, page_size, out, max_slots, row_start); });
}
PyObject* slots(PyObject*, PyObject* const* a, Py_ssize_t n) { return guarded<slots_of>(a, n, 7); }

// K, V, slots, K_pages, V_pages, k_scale_log2, v_scale_log2, stream
PyObject* append_of(PyObject* const* a) {
  Call c;
  const at::Tensor *K, *V;
  long long ld_k, ld_v;
  const Pool p(c, a[3], a[4]);
  const void* k = c.rows(a[0], "K", false, K, ld_k);
  const void* v = c.rows(a[1], "V", false, V, ld_v);
  if (K->size(1) != p.N || K->size(2) != p.D || V->sizes() != K->sizes() || ld_v != ld_k)
    refuse(PyExc_ValueError, "K and V must be [rows, %d, %d] with one stride", p.N, p.D);
  const int rows = (int)K->size(0);
  const int* at = c.list(a[2], "slots", rows);
  const int ks = (int)integer(a[5]), vs = (int)integer(a[6]);
  void* st = c.stream(a[7]);
  return unlocked([&] {
    return call_append(st, k, v, ld_k, rows, at, p.N, p.D, p.K, p.V, p.n_pages, p.page_size, p.ld_page, p.ld_token, p.ld_head,
                       p.dtype, ks, vs);
  });
}
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) { return guarded<append_of>(a, n, 8); }

// Q, K_pages, V_pages, block_table, kv_len, O, n_pinned, window, softmax_scale, k_scale_log2, v_scale_log2, workspace, stream
PyObject* attention_of(PyObject* const* a) {
  Call c;
  const at::Tensor *Q, *O;
  long long ld_q, ld_o, ld;
  int columns;
  const Pool p(c, a[1], a[2]);
  const void* q = c.rows(a[0], "Q", false, Q, ld_q);
  void* o = c.rows(a[5], "O", true, O, ld_o);
  if (Q->size(2) != p.D || O->sizes() != Q->sizes()) refuse(PyExc_ValueError, "Q and O must be [B, N, %d]", p.D);
  const int B = (int)Q->size(0), N = (int)Q->size(1);
  const int* table = c.table(a[3], B, columns, ld);
  const int* kv_len = c.list(a[4], "kv_len", B);
  const int n_pinned = (int)integer(a[6]), window = (int)integer(a[7]), ks = (int)integer(a[9]), vs = (int)integer(a[10]);
  const double scale = PyFloat_AsDouble(a[8]);
  if (scale == -1.0 && PyErr_Occurred()) throw Refused{};
  void* ws = nullptr;
  size_t ws_bytes = 0;
  if (a[11] != Py_None) {
    const at::Tensor& w = c.tensor(a[11], "the workspace");
    if (!w.is_contiguous()) refuse(PyExc_ValueError, "the workspace must be contiguous");
    c.place(w);
    ws = w.data_ptr();
    ws_bytes = w.nbytes();
  }
  void* st = c.stream(a[12]);
  const int out_dtype = O->scalar_type() == at::kFloat ? PAFU_F32 : PAFU_BF16;
  return unlocked([&] {
    return call_attention(st, q, ld_q, p.K, p.V, p.n_pages, p.page_size, p.ld_page, p.ld_token, p.ld_head, p.dtype, ks, vs, table,
                          columns, ld, kv_len, B, N, p.N, p.D, n_pinned, window, (float)scale, o, ld_o, out_dtype, ws, ws_bytes);
  });
}
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) { return guarded<attention_of>(a, n, 13); }

// addresses of the four entry points, and the functions that tell the current device and its stream's handle
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 6) {
    PyErr_SetString(PyExc_TypeError, "6 arguments wanted");
    return nullptr;
  }
  void* f[4];
  for (int i = 0; i < 4; ++i) {
    f[i] = PyLong_AsVoidPtr(a[i]);
    if (!f[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an entry point is missing");
      return nullptr;
    }
  }
  call_tables = reinterpret_cast<decltype(call_tables)>(f[0]);
  call_slots = reinterpret_cast<decltype(call_slots)>(f[1]);
  call_append = reinterpret_cast<decltype(call_append)>(f[2]);
  call_attention = reinterpret_cast<decltype(call_attention)>(f[3]);
  Py_XSETREF(current_device, Py_NewRef(a[4]));
  Py_XSETREF(current_stream, Py_NewRef(a[5]));
  Py_RETURN_NONE;
}

template <typename F>
PyCFunction fast(F f) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}
PyMethodDef methods[] = {
    {"bind", fast(bind), METH_FASTCALL, nullptr},     {"tables", fast(tables), METH_FASTCALL, nullptr},
    {"slots", fast(slots), METH_FASTCALL, nullptr},   {"append", fast(append), METH_FASTCALL, nullptr},
    {"attention", fast(attention), METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_paged_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__paged_call() {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}

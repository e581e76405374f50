// CPython binding of the C calls in spanmerge.h: argument conversion only.
//
// A decode step is a handful of short launches, and through ctypes the
// conversion of their arguments in Python took longer than the launches (one
// step's rule check, input row and projected append: 36 us of host time for
// four calls, 30 us of kernels).  Every entry here takes the C call's
// arguments in order: a tensor (or None) for a device pointer, the ctypes
// structure for a cache or a rule table, the bytes that merge_params or
// kv_proj_params gave (or a structure's own bytes) for parameters, an int (or
// None) for a stream handle, plain numbers for the rest; it returns the
// status.  The checked entries take rows with a stride as a tensor in a tuple
// of its own, which row_stride has looked at.  Values are taken and
// refused as ctypes does for the same prototypes: integers wrap to the C
// type's width (the checked entries refuse what an int does not hold: 2^32
// rows would count as none), a ctypes number of the argument's own type counts
// as its value, and what does not fit raises ctypes.ArgumentError.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <dlfcn.h>

#include <cstring>
#include <tuple>
#include <type_traits>
#include <utility>

#include "spanmerge.h"

namespace {

// The entries, resolved by open() from the library that the program loaded.
#define SM_ENTRIES(X)                                                                                         \
  X(sm_merge_spans) X(sm_merge_token_table) X(sm_merge_spans_tabled) X(sm_pack_spans) X(sm_kv_rollback)       \
  X(sm_kv_append) X(sm_decode_attention) X(sm_decode_step) X(sm_decode_merge_step)                            \
  X(sm_decode_step_noalloc) X(sm_prefill_attention) X(sm_rules_build) X(sm_rules_lookup) X(sm_match_prompt)   \
  X(sm_match_decode) X(sm_gather_surrogates) X(sm_span_dedupe) X(sm_kv_project) X(sm_kv_append_projected)
// Entries that look at each tensor's type (of a typed pointer) and device too;
// one argument more, the current device's index, comes last.
#define SM_CHECKED(X) \
  X(sm_kv_reserve) X(sm_rotary) X(sm_kv_write_rotary) X(sm_kv_read) X(sm_block_norm) X(sm_token_logprobs)     \
  X(sm_decode_attention_shared) X(sm_sample_tokens)
#define SM_SLOT(name) decltype(&::name) p_##name;
SM_ENTRIES(SM_SLOT)
SM_CHECKED(SM_SLOT)

PyObject *g_is_cuda, *g_is_contiguous, *g_data_ptr, *g_value;  // interned names
PyObject *g_dtype, *g_get_device, *g_numel, *g_shape, *g_stride;

// What setup() is given: the exceptions for unusable tensors and for other
// unusable arguments, the structures, and the C types of plain arguments.
enum { kError, kArgumentError, kPagedCache, kRuleTable, kInt, kInt64, kFloat, kSize, kPointer, kTypes };
PyObject *g_type[kTypes];

bool is_true(PyObject *r, const char *otherwise) {
  if (!r) return false;
  const int v = PyObject_IsTrue(r);
  Py_DECREF(r);
  if (v == 0) PyErr_SetString(g_type[kError], otherwise);
  return v > 0;
}

bool tensor_address(PyObject *t, void **p) {
  *p = nullptr;
  if (t == Py_None) return true;
  if (!is_true(PyObject_GetAttr(t, g_is_cuda), "expected a GPU tensor")) return false;
  if (!is_true(PyObject_CallMethodNoArgs(t, g_is_contiguous), "expected a contiguous tensor")) return false;
  PyObject *r = PyObject_CallMethodNoArgs(t, g_data_ptr);
  if (!r) return false;
  *p = PyLong_AsVoidPtr(r);
  Py_DECREF(r);
  return !PyErr_Occurred();
}

bool is_dtype(PyObject *t, PyObject *dtype) {  // (there is one object for each type)
  PyObject *d = PyObject_GetAttr(t, g_dtype);
  Py_XDECREF(d);
  return d == dtype;
}

bool as_long(PyObject *r, long *v) {
  if (!r) return false;
  *v = PyLong_AsLong(r);
  Py_DECREF(r);
  return !(*v == -1 && PyErr_Occurred());
}

// What a tensor is, without a call per property: the DLPack standard's C
// exchange interface, version 1, which torch.Tensor offers in a capsule.  Its
// structures, as the standard lays them out (of the interface up to the one
// function used here).
struct DlVersion { uint32_t major, minor; };
struct DlTensor {
  void *data;
  int32_t device_type, device_id;  // device types 2 and 10: GPU memory (host memory has others, pinned or not)
  int32_t ndim;
  uint8_t code, bits;  // of a value: code 0 integer, 2 float, 4 bfloat16
  uint16_t lanes;
  int64_t *shape, *strides;
  uint64_t byte_offset;
};
struct DlExchange {
  DlVersion version;
  void *previous, *allocator, *managed_from_object, *managed_to_object;
  int (*tensor_from_object)(void *object, DlTensor *out);  // what it points to is the tensor's
};

const DlExchange *g_exchange;
PyObject *g_plain[2];                       // the classes that it is asked for: others may have properties of their own
PyObject *g_int32, *g_float32, *g_bf16;     // torch's types

struct View : DlTensor {
  long device() const { return device_type == 2 || device_type == 10 ? device_id : -1; }
  bool is(PyObject *dtype) const {
    return lanes == 1 && (dtype == g_int32 ? code == 0 && bits == 32 : dtype == g_float32 ? code == 2 && bits == 32
                                                                                           : code == 4 && bits == 16);
  }
  int64_t numel() const {
    int64_t n = 1;
    for (int i = 0; i < ndim; ++i) n *= shape[i];
    return n;
  }
  bool contiguous() const {
    int64_t width = 1;
    for (int i = ndim - 1; i >= 0; --i) {
      if (shape[i] != 1 && strides[i] != width) return numel() == 0;
      width *= shape[i];
    }
    return true;
  }
  char *address() const { return data ? (char *)data + byte_offset : nullptr; }
};

// Whether v is a view of t, which is to be of type `dtype` (any, if that is
// null): not for other classes and types, whose methods are called.
bool view_of(PyObject *t, PyObject *dtype, View *v) {
  PyObject *cls = (PyObject *)Py_TYPE(t);
  if (!g_exchange || (cls != g_plain[0] && cls != g_plain[1])) return false;
  if (dtype && dtype != g_int32 && dtype != g_float32 && dtype != g_bf16) return false;
  if (g_exchange->tensor_from_object(t, v) == 0 && (v->strides || v->ndim == 0)) return true;
  PyErr_Clear();
  return false;
}

// tensor_address for the checked entries: a tensor of type `dtype` (unless
// that is null) on the current device; one in a tuple of its own need not be
// contiguous.
bool checked_address(PyObject *t, PyObject *dtype, long device, void **p) {
  *p = nullptr;
  if (t == Py_None) return true;
  const bool strided = PyTuple_CheckExact(t) && PyTuple_GET_SIZE(t) == 1;
  if (strided) t = PyTuple_GET_ITEM(t, 0);
  View view;
  if (view_of(t, dtype, &view) && view.device() == device && (strided || view.contiguous()) && (!dtype || view.is(dtype))) {
    *p = view.address();
    return true;
  }
  long at;  // (what is wrong, or another class)
  if (!as_long(PyObject_CallMethodNoArgs(t, g_get_device), &at)) return false;  // (-1: host memory)
  if (at != device) {
    PyErr_Format(g_type[kError], "expected tensors on the current device %ld, got one on %ld", device, at);
    return false;
  }
  if (!strided && !is_true(PyObject_CallMethodNoArgs(t, g_is_contiguous), "expected a contiguous tensor")) return false;
  if (dtype && !is_dtype(t, dtype)) {
    if (!PyErr_Occurred()) PyErr_Format(g_type[kError], "expected a tensor of %S", dtype);
    return false;
  }
  PyObject *r = PyObject_CallMethodNoArgs(t, g_data_ptr);
  if (!r) return false;
  *p = PyLong_AsVoidPtr(r);
  Py_DECREF(r);
  return !PyErr_Occurred();
}

template <class T>
constexpr bool is_host_struct = std::is_same_v<T, sm_paged_cache> || std::is_same_v<T, sm_rule_table> ||
                                std::is_same_v<T, sm_merge_params> || std::is_same_v<T, sm_kv_proj_params> ||
                                std::is_same_v<T, sm_rope_params> || std::is_same_v<T, sm_norm>;

// the C type that a plain argument (or a stream handle) has in the prototypes
template <class A>
constexpr int plain_type = std::is_same_v<A, hipStream_t>      ? kPointer
                           : std::is_floating_point_v<A>       ? kFloat
                           : std::is_same_v<A, size_t>         ? kSize
                           : sizeof(A) == 8                    ? kInt64
                                                               : kInt;

// a new reference to o, or to its value where o is a ctypes number of type t
PyObject *plain_value(PyObject *o, int t) {
  if (!PyLong_Check(o) && !PyFloat_Check(o) && PyObject_TypeCheck(o, (PyTypeObject *)g_type[t]))
    return PyObject_GetAttr(o, g_value);
  Py_INCREF(o);
  return o;
}

template <class T>
bool get_struct(PyObject *o, T **v) {
  *v = nullptr;
  if (o == Py_None) return true;
  constexpr int t = std::is_same_v<std::remove_cv_t<T>, sm_paged_cache>  ? kPagedCache
                    : std::is_same_v<std::remove_cv_t<T>, sm_rule_table> ? kRuleTable
                                                                         : kTypes;  // the parameters: bytes
  const bool right = t == kTypes ? PyBytes_Check(o) : PyObject_TypeCheck(o, (PyTypeObject *)g_type[t % kTypes]);
  Py_buffer b;
  if (!right) {
    PyErr_SetString(PyExc_TypeError, "wrong structure");
    return false;
  }
  if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) return false;
  const bool whole = b.len >= (Py_ssize_t)sizeof(T);
  *v = (T *)b.buf;  // (the caller's object keeps it for the length of the call)
  PyBuffer_Release(&b);
  if (!whole) PyErr_SetString(PyExc_TypeError, "structure too short");
  return whole;
}

template <class A>
bool get(PyObject *o, A *v) {
  if constexpr (std::is_pointer_v<A> && !std::is_same_v<A, hipStream_t>) {
    if constexpr (is_host_struct<std::remove_cv_t<std::remove_pointer_t<A>>>) {
      return get_struct(o, v);
    } else {
      void *p;
      if (!tensor_address(o, &p)) return false;
      *v = (A)p;
      return true;
    }
  } else {
    PyObject *x = plain_value(o, plain_type<A>);
    if (!x) return false;
    if constexpr (std::is_same_v<A, hipStream_t>) {
      *v = nullptr;
      if (PyLong_Check(x)) *v = (hipStream_t)(uintptr_t)PyLong_AsUnsignedLongLongMask(x);
      else if (x != Py_None) PyErr_SetString(PyExc_TypeError, "expected a stream handle");
    } else if constexpr (std::is_floating_point_v<A>) {
      *v = (A)PyFloat_AsDouble(x);
    } else {
      *v = (A)PyLong_AsUnsignedLongLongMask(x);
    }
    Py_DECREF(x);
    return !PyErr_Occurred();
  }
}

template <class A>
bool get_checked(PyObject *o, A *v, long device) {
  if constexpr (std::is_pointer_v<A> && !std::is_same_v<A, hipStream_t>) {
    typedef std::remove_cv_t<std::remove_pointer_t<A>> T;
    if constexpr (is_host_struct<T>) {
      return get_struct(o, v);
    } else {
      void *p;
      PyObject *dtype = std::is_same_v<T, int32_t> ? g_int32 : std::is_same_v<T, float> ? g_float32 : nullptr;
      if (!checked_address(o, dtype, device, &p)) return false;
      *v = (A)p;
      return true;
    }
  } else if constexpr (std::is_same_v<A, int>) {
    PyObject *x = plain_value(o, kInt);
    if (!x) return false;
    const long value = PyLong_Check(x) ? PyLong_AsLong(x) : 0;
    const bool over = (value == -1 && PyErr_Occurred()) || value != (int)value;
    if (over) {
      PyErr_Clear();
      PyErr_Format(g_type[kError], "an argument is out of range: no int holds %S", x);
    }
    Py_DECREF(x);
    return !over && get(o, v);
  } else {
    return get(o, v);
  }
}

// A TypeError of argument `at` (from 1) as ctypes reports it.
void argument_error(int at) {
  if (!PyErr_ExceptionMatches(PyExc_TypeError)) return;
  PyObject *type, *value, *trace;
  PyErr_Fetch(&type, &value, &trace);
  PyErr_Format(g_type[kArgumentError], "argument %d: %S: %S", at, type, value ? value : Py_None);
  Py_XDECREF(type);
  Py_XDECREF(value);
  Py_XDECREF(trace);
}

template <class... A, size_t... I>
PyObject *call(sm_status (*fn)(A...), PyObject *const *args, Py_ssize_t n, std::index_sequence<I...>) {
  if (n != (Py_ssize_t)sizeof...(A)) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  std::tuple<A...> v;
  int at = 0;
  if (!((++at, get(args[I], &std::get<I>(v))) && ...)) {
    argument_error(at);
    return nullptr;
  }
  sm_status st;
  Py_BEGIN_ALLOW_THREADS;
  st = fn(std::get<I>(v)...);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(st);
}

template <class... A, size_t... I>
PyObject *call_checked(sm_status (*fn)(A...), PyObject *const *args, Py_ssize_t n, std::index_sequence<I...>) {
  if (n != (Py_ssize_t)sizeof...(A) + 1) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  const long device = PyLong_AsLong(args[n - 1]);
  if (device == -1 && PyErr_Occurred()) return nullptr;
  std::tuple<A...> v;
  int at = 0;
  if (!((++at, get_checked(args[I], &std::get<I>(v), device)) && ...)) {
    argument_error(at);
    return nullptr;
  }
  sm_status st;
  Py_BEGIN_ALLOW_THREADS;
  st = fn(std::get<I>(v)...);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(st);
}

template <bool CHECKED, class... A>
PyObject *dispatch(sm_status (*fn)(A...), PyObject *const *args, Py_ssize_t n) {
  if constexpr (CHECKED) return call_checked(fn, args, n, std::index_sequence_for<A...>{});
  else return call(fn, args, n, std::index_sequence_for<A...>{});
}

template <auto *Fn, bool CHECKED = false>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (!*Fn) {
    PyErr_SetString(g_type[kError], "the library is not open");
    return nullptr;
  }
  return dispatch<CHECKED>(*Fn, args, n);
}

// open(path): the entries of the library at `path` (kept loaded)
PyObject *open_library(PyObject *, PyObject *path) {
  PyObject *name;
  if (!PyUnicode_FSConverter(path, &name)) return nullptr;
  void *lib = dlopen(PyBytes_AS_STRING(name), RTLD_NOW | RTLD_LOCAL);
  Py_DECREF(name);
  if (!lib) {
    PyErr_SetString(g_type[kError], dlerror());
    return nullptr;
  }
#define SM_FIND(name)                                                   \
  void *const f_##name = dlsym(lib, #name);                             \
  if (!f_##name) {                                                      \
    PyErr_SetString(g_type[kError], "the library lacks the entry " #name);     \
    return nullptr;                                                     \
  }
  SM_ENTRIES(SM_FIND)
  SM_CHECKED(SM_FIND)
#define SM_STORE(name) p_##name = (decltype(&::name))f_##name;
  SM_ENTRIES(SM_STORE)
  SM_CHECKED(SM_STORE)
  Py_RETURN_NONE;
}

// merge_params(d, h, ln_eps, Q, W_kv, b_kv, g_kv, beta_kv, W_o, b_o, g_o, beta_o): the structure's bytes
PyObject *merge_params(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 12) {
    PyErr_SetString(PyExc_TypeError, "merge_params takes 12 arguments");
    return nullptr;
  }
  sm_merge_params p;
  std::memset(&p, 0, sizeof p);
  const void **field[9] = {&p.Q, &p.W_kv, &p.b_kv, &p.g_kv, &p.beta_kv, &p.W_o, &p.b_o, &p.g_o, &p.beta_o};
  if (!get(args[0], &p.d) || !get(args[1], &p.h) || !get(args[2], &p.ln_eps)) return nullptr;
  for (int i = 0; i < 9; ++i)
    if (!get(args[3 + i], field[i])) return nullptr;
  return PyBytes_FromStringAndSize((const char *)&p, sizeof p);
}

// kv_proj_params(d, W_k, W_v, rope_theta, rms_eps): the structure's bytes
PyObject *kv_proj_params(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 5) {
    PyErr_SetString(PyExc_TypeError, "kv_proj_params takes 5 arguments");
    return nullptr;
  }
  sm_kv_proj_params p;
  std::memset(&p, 0, sizeof p);
  if (!get(args[0], &p.d) || !get(args[1], &p.W_k) || !get(args[2], &p.W_v) || !get(args[3], &p.rope_theta) ||
      !get(args[4], &p.rms_eps))
    return nullptr;
  return PyBytes_FromStringAndSize((const char *)&p, sizeof p);
}

// setup(types): the objects of the enumeration above, in its order
PyObject *setup(PyObject *, PyObject *types) {
  if (!PyTuple_Check(types) || PyTuple_GET_SIZE(types) != kTypes) {
    PyErr_SetString(PyExc_TypeError, "setup takes a tuple of the types");
    return nullptr;
  }
  for (int i = 0; i < kTypes; ++i) {
    PyObject *t = PyTuple_GET_ITEM(types, i);
    if (!PyType_Check(t)) {
      PyErr_SetString(PyExc_TypeError, "setup takes a tuple of the types");
      return nullptr;
    }
    Py_INCREF(t);
    Py_XSETREF(g_type[i], t);
  }
  Py_RETURN_NONE;
}

// torch_types(int32, float32, bfloat16, Tensor, Parameter, exchange): torch's types and classes for the checked
// entries, and its exchange interface (None: its methods are called)
PyObject *torch_types(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 6) {
    PyErr_SetString(PyExc_TypeError, "torch_types takes 6 arguments");
    return nullptr;
  }
  PyObject **to[] = {&g_int32, &g_float32, &g_bf16, &g_plain[0], &g_plain[1]};
  for (int i = 0; i < 5; ++i) {
    Py_INCREF(args[i]);
    Py_XSETREF(*to[i], args[i]);
  }
  g_exchange = nullptr;
  if (args[5] != Py_None) {
    const auto *e = (const DlExchange *)PyCapsule_GetPointer(args[5], "dlpack_exchange_api");
    if (!e) return nullptr;
    if (e->version.major == 1 && e->tensor_from_object) g_exchange = e;
  }
  Py_RETURN_NONE;
}

// need(tensor, count, name): it has at least so many values
PyObject *need(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 3) {
    PyErr_SetString(PyExc_TypeError, "need takes 3 arguments");
    return nullptr;
  }
  long has, count = PyLong_AsLong(args[1]);
  if (count == -1 && PyErr_Occurred()) return nullptr;
  View view;
  if (view_of(args[0], nullptr, &view)) has = (long)view.numel();
  else if (!as_long(PyObject_CallMethodNoArgs(args[0], g_numel), &has)) return nullptr;
  if (has < count) {
    PyErr_Format(g_type[kError], "%S: expected %ld values, got %ld", args[2], count, has);
    return nullptr;
  }
  Py_RETURN_NONE;
}

// parameter(tensor, dtype, count, device, name): the address of a contiguous tensor of that type, device and number of
// values; 0 for None
PyObject *parameter(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 5) {
    PyErr_SetString(PyExc_TypeError, "parameter takes 5 arguments");
    return nullptr;
  }
  PyObject *t = args[0];
  if (t == Py_None) return PyLong_FromLong(0);
  long has, at, count = PyLong_AsLong(args[2]), device = PyLong_AsLong(args[3]);
  if (PyErr_Occurred()) return nullptr;
  View view;
  if (view_of(t, args[1], &view) && view.is(args[1]) && view.numel() == count && view.device() == device && view.contiguous())
    return PyLong_FromVoidPtr(view.address());
  if (!as_long(PyObject_CallMethodNoArgs(t, g_numel), &has) ||
      !as_long(PyObject_CallMethodNoArgs(t, g_get_device), &at))
    return nullptr;
  const bool typed = is_dtype(t, args[1]);
  if (PyErr_Occurred()) return nullptr;
  if (!typed || has != count || at != device) {
    PyErr_Format(g_type[kError], "%S: expected %ld values of %S on device %ld, got %ld on %ld%s", args[4], count, args[1], device,
                 has, at, typed ? "" : " of another type");
    return nullptr;
  }
  if (!is_true(PyObject_CallMethodNoArgs(t, g_is_contiguous), "expected a contiguous tensor")) return nullptr;
  return PyObject_CallMethodNoArgs(t, g_data_ptr);
}

// row_stride(tensor, dtype, name, rows, inner, ...): the row stride of a [rows, *inner] tensor of that type whose
// rows are contiguous (one row: its length)
PyObject *row_stride(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n < 5 || n > 7) {
    PyErr_SetString(PyExc_TypeError, "row_stride takes 5 to 7 arguments");
    return nullptr;
  }
  PyObject *t = args[0];
  const Py_ssize_t dims = n - 3;
  View view;
  if (view_of(t, args[1], &view) && view.is(args[1]) && view.ndim == dims) {
    bool right = true;
    long long width = 1, row = 0;
    for (Py_ssize_t i = dims - 1; right && i >= 0; --i) {
      const long long size = view.shape[i], s = view.strides[i];
      right = size == PyLong_AsLongLong(args[3 + i]) && (i == 0 || size == 1 || s == width);
      if (i == 0) row = size > 1 ? s : width;
      width *= size;
    }
    if (PyErr_Occurred()) return nullptr;
    if (right) return PyLong_FromLongLong(row);
  }
  const bool typed = is_dtype(t, args[1]);
  if (PyErr_Occurred()) return nullptr;
  PyObject *shape = PyObject_GetAttr(t, g_shape), *stride = shape ? PyObject_CallMethodNoArgs(t, g_stride) : nullptr;
  PyObject *answer = nullptr;
  if (stride && PyTuple_Check(shape) && PyTuple_Check(stride)) {
    bool right = typed && PyTuple_GET_SIZE(shape) == dims && PyTuple_GET_SIZE(stride) == dims;
    long long width = 1, row = 0;
    for (Py_ssize_t i = dims - 1; right && i >= 0; --i) {
      const long long size = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i)), want = PyLong_AsLongLong(args[3 + i]);
      const long long s = PyLong_AsLongLong(PyTuple_GET_ITEM(stride, i));
      right = size == want && (i == 0 || size == 1 || s == width);
      if (i == 0) row = size > 1 ? s : width;
      width *= size;
    }
    if (!PyErr_Occurred()) {
      if (right) answer = PyLong_FromLongLong(row);
      else PyErr_Format(g_type[kError], "%S: expected %S rows that are contiguous, of the other tensors' sizes; got shape %S, strides %S",
                        args[2], args[1], shape, stride);
    }
  } else if (!PyErr_Occurred()) {
    PyErr_SetString(PyExc_TypeError, "expected a tensor");
  }
  Py_XDECREF(shape);
  Py_XDECREF(stride);
  return answer;
}

#define SM_CHECKED_ENTRY(name) {#name, (PyCFunction)(void (*)(void))entry<&p_##name, true>, METH_FASTCALL, nullptr},
#define SM_ENTRY(name) {#name, (PyCFunction)(void (*)(void))entry<&p_##name>, METH_FASTCALL, nullptr},
PyMethodDef methods[] = {
    SM_ENTRIES(SM_ENTRY)
    SM_CHECKED(SM_CHECKED_ENTRY)
    {"torch_types", (PyCFunction)(void (*)(void))torch_types, METH_FASTCALL, nullptr},
    {"need", (PyCFunction)(void (*)(void))need, METH_FASTCALL, nullptr},
    {"parameter", (PyCFunction)(void (*)(void))parameter, METH_FASTCALL, nullptr},
    {"row_stride", (PyCFunction)(void (*)(void))row_stride, METH_FASTCALL, nullptr},
    {"merge_params", (PyCFunction)(void (*)(void))merge_params, METH_FASTCALL, nullptr},
    {"kv_proj_params", (PyCFunction)(void (*)(void))kv_proj_params, METH_FASTCALL, nullptr},
    {"setup", setup, METH_O, nullptr},
    {"open", open_library, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) {
  g_is_cuda = PyUnicode_InternFromString("is_cuda");
  g_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  g_data_ptr = PyUnicode_InternFromString("data_ptr");
  g_value = PyUnicode_InternFromString("value");
  if (!g_is_cuda || !g_is_contiguous || !g_data_ptr || !g_value) return nullptr;
  g_dtype = PyUnicode_InternFromString("dtype");
  g_get_device = PyUnicode_InternFromString("get_device");
  g_numel = PyUnicode_InternFromString("numel");
  g_shape = PyUnicode_InternFromString("shape");
  g_stride = PyUnicode_InternFromString("stride");
  if (!g_dtype || !g_get_device || !g_numel || !g_shape || !g_stride) return nullptr;
  for (PyObject *&t : g_type) {  // (until setup: no structure or ctypes number is of these types)
    Py_INCREF(PyExc_RuntimeError);
    t = PyExc_RuntimeError;
  }
  return PyModule_Create(&module);
}

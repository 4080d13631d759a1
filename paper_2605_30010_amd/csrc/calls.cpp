// The calls of a decoding step (the cache's, the page pool's, the rotary positions') as binding.py makes them, without Python in between:
// their host part is most of a small call.  A function here makes the call if everything about it is as it mostly is (plain tensors on the
// device, of the types and layouts asked for) and returns what it makes, or the entry point's error code; for anything else it
// returns None, and binding.py, which has all the checks and says what is wrong, goes on.  us a call of the binding, launch 2.7 included, without /
// with this: rotary positions of queries and keys 8.6 / 5.0, a pool's step 10.2 / 5.6, rows stored 7.3 / 4.3, read 8.8 / 5.8, attention 7.7 / 5.1.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <dlfcn.h>

#include <array>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "earlytom.h"

namespace {

struct {
  decltype(&et_kv_append) append;
  decltype(&et_kv_append_slots) append_slots;
  decltype(&et_kv_read) read;
  decltype(&et_attention_paged_workspace_bytes) attention_bytes;
  decltype(&et_attention_paged) attention;
  decltype(&et_kv_resize_workspace_bytes) resize_bytes;
  decltype(&et_kv_resize) resize;
  decltype(&et_rotary_apply) rotary;
} lib;

// A plain tensor of this type on that device, or null.
const at::Tensor *plain(PyObject *o, at::ScalarType type, long device) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor &t = THPVariable_Unpack(o);
  return t.layout() == at::kStrided && t.scalar_type() == type && t.is_cuda() && t.device().index() == device ? &t : nullptr;
}
const at::Tensor *ints(PyObject *o, long device, int64_t n) {
  const at::Tensor *t = plain(o, at::kInt, device);
  return t && t->dim() == 1 && t->size(0) == n && t->is_contiguous() ? t : nullptr;
}
// bf16 [rows, heads * d] or [rows, heads, d] with contiguous rows.
struct Rows {
  const at::Tensor *t = nullptr;
  int64_t n = 0, heads = 0, stride = 0;
  Rows(PyObject *o, long device, int64_t d) {
    const at::Tensor *x = plain(o, at::kBFloat16, device);
    if (!x) return;
    if (x->dim() == 2 && x->stride(1) == 1 && x->size(1) % d == 0) heads = x->size(1) / d;
    else if (x->dim() == 3 && x->size(2) == d && x->stride(2) == 1 && (x->stride(1) == d || x->size(1) == 1)) heads = x->size(1);
    else return;
    t = x;
    n = x->size(0);
    stride = n > 1 ? x->stride(0) : heads * d;
  }
  uint16_t *data() const { return static_cast<uint16_t *>(t->data_ptr()); }
};
struct Seqs {
  bool good = false;
  et_kv_seqs s{};
  Seqs(PyObject *table, PyObject *len, long device) {
    const at::Tensor *t = plain(table, at::kInt, device);
    if (!t || t->dim() != 2 || t->size(1) < 1 || (t->stride(1) != 1 && t->size(1) > 1) || t->size(0) > INT32_MAX || t->size(1) > INT32_MAX) return;
    const int64_t n = t->size(0), stride = n > 1 ? t->stride(0) : t->size(1);
    const at::Tensor *l = ints(len, device, n);
    if (!l || stride > INT32_MAX) return;
    s = {static_cast<const int32_t *>(t->data_ptr()), (int32_t)stride, (int32_t)t->size(1), static_cast<const int32_t *>(l->data_ptr()), (int32_t)n};
    good = true;
  }
};
// A whole number in [0, most]; -1: something else.
int64_t whole(PyObject *o, int64_t most) {
  if (!PyLong_CheckExact(o)) return -1;
  int over = 0;
  const int64_t v = PyLong_AsLongLongAndOverflow(o, &over);
  return over || v < 0 || v > most ? -1 : v;
}
at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type, long device) {
  return at::empty(shape, at::TensorOptions().dtype(type).device(at::Device(at::kCUDA, (c10::DeviceIndex)device)));
}
// Several tensors of a call; small ones (up to 8 MiB) in one piece of memory, which costs 0.6 us less for each but the first (the binding says so where
// it is done; what is read back from a cache is kept by callers, and is made one by one).
struct Wanted {
  at::IntArrayRef sizes;
  at::ScalarType type;
};
template <size_t N>
std::array<at::Tensor, N> fresh(const Wanted (&wanted)[N], long device) {
  std::array<at::Tensor, N> out;
  size_t at[N], bytes = 0;
  for (size_t i = 0; i < N; ++i) {
    at[i] = bytes;
    bytes += (c10::multiply_integers(wanted[i].sizes) * c10::elementSize(wanted[i].type) + 127) / 128 * 128;
  }
  if (bytes > 8 << 20) {
    for (size_t i = 0; i < N; ++i) out[i] = fresh(wanted[i].sizes, wanted[i].type, device);
    return out;
  }
  const at::Tensor all = fresh({(int64_t)bytes}, at::kByte, device);
  for (size_t i = 0; i < N; ++i) {
    out[i] = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(all.storage()), all.key_set(), c10::scalarTypeToTypeMeta(wanted[i].type));
    out[i].unsafeGetTensorImpl()->set_sizes_contiguous(wanted[i].sizes);
    out[i].unsafeGetTensorImpl()->set_storage_offset(at[i] / c10::elementSize(wanted[i].type));
  }
  return out;
}
// Makes the call without Python's lock, which is taken again whatever happens (a tensor whose address
// torch withholds throws when it is asked).
template <typename F>
int unlocked(F &&call) {
  struct Released {
    PyThreadState *state = PyEval_SaveThread();
    ~Released() { PyEval_RestoreThread(state); }
  } released;
  return call();
}
PyObject *done(int rc) { return PyLong_FromLong(rc); }
template <typename... T>
PyObject *made(int rc, const T &...tensors) {
  if (rc) return PyLong_FromLong(rc);
  if constexpr (sizeof...(T) == 1) return THPVariable_Wrap(tensors...);
  else {
    PyObject *all = PyTuple_New(sizeof...(T));
    Py_ssize_t i = 0;
    bool good = all != nullptr;
    const auto add = [&](const at::Tensor &t) {
      PyObject *o = good ? THPVariable_Wrap(t) : nullptr;
      if (o) PyTuple_SET_ITEM(all, i++, o);
      else good = false;
    };
    (add(tensors), ...);
    if (good) return all;
    Py_XDECREF(all);
    return nullptr;
  }
}
template <typename T>
T *at_address(PyObject *o) { return static_cast<T *>(PyLong_AsVoidPtr(o)); }
// The stream that an argument is (Python's numbers are asked here, with its lock); false, with Python's error: it is none.
bool stream_of(PyObject *o, void *&stream) {
  stream = PyLong_AsVoidPtr(o);
  return stream || !PyErr_Occurred();
}

#define CALL(name) PyObject *name(PyObject *, PyObject *const *arg, Py_ssize_t)

// (cache, device, k, v, page_table, kv_len, cu_rows or None, stream)
CALL(append) {
  HANDLE_TH_ERRORS
  const auto *cache = at_address<et_kv_cache>(arg[0]);
  const long device = PyLong_AsLong(arg[1]);
  const Rows k(arg[2], device, cache->head_dim), v(arg[3], device, cache->head_dim);
  const Seqs seqs(arg[4], arg[5], device);
  if (!k.t || !v.t || !seqs.good || k.n != v.n || k.n > INT32_MAX || k.heads != cache->n_kv_heads || v.heads != cache->n_kv_heads) Py_RETURN_NONE;
  const at::Tensor *cu = arg[6] == Py_None ? nullptr : ints(arg[6], device, (int64_t)seqs.s.n_seqs + 1);
  if (!cu && arg[6] != Py_None) Py_RETURN_NONE;
  const int32_t *ranges = cu ? static_cast<const int32_t *>(cu->data_ptr()) : nullptr;
  void *stream;
  if (!stream_of(arg[7], stream)) return nullptr;
  return done(unlocked([&] {
    return lib.append(cache, &seqs.s, ranges, (int32_t)k.n, k.data(), k.stride, v.data(), v.stride, stream);
  }));
  END_HANDLE_TH_ERRORS
}

// (cache, device, k, v, slots, stream)
CALL(append_at) {
  HANDLE_TH_ERRORS
  const auto *cache = at_address<et_kv_cache>(arg[0]);
  const long device = PyLong_AsLong(arg[1]);
  const Rows k(arg[2], device, cache->head_dim), v(arg[3], device, cache->head_dim);
  const at::Tensor *slots = plain(arg[4], at::kLong, device);
  if (!k.t || !v.t || !slots || k.n != v.n || k.n > INT32_MAX || k.heads != cache->n_kv_heads || v.heads != cache->n_kv_heads || slots->dim() != 1 ||
      slots->size(0) != k.n || !slots->is_contiguous())
    Py_RETURN_NONE;
  void *stream;
  if (!stream_of(arg[5], stream)) return nullptr;
  return done(unlocked([&] {
    return lib.append_slots(cache, static_cast<const int64_t *>(slots->data_ptr()), (int32_t)k.n, k.data(), k.stride, v.data(), v.stride,
                            stream);
  }));
  END_HANDLE_TH_ERRORS
}

// (cache, device, page_table, kv_len, cu_rows or None, rows or None, stream) -> (k, v)
CALL(read) {
  HANDLE_TH_ERRORS
  const auto *cache = at_address<et_kv_cache>(arg[0]);
  const long device = PyLong_AsLong(arg[1]);
  const Seqs seqs(arg[2], arg[3], device);
  if (!seqs.good) Py_RETURN_NONE;
  const at::Tensor *cu = arg[4] == Py_None ? nullptr : ints(arg[4], device, (int64_t)seqs.s.n_seqs + 1);
  if (!cu && (arg[4] != Py_None || arg[5] != Py_None)) Py_RETURN_NONE;
  const int64_t rows = cu ? whole(arg[5], INT32_MAX) : seqs.s.n_seqs, width = (int64_t)cache->n_kv_heads * cache->head_dim;
  if (rows < 0) Py_RETURN_NONE;
  const at::Tensor k = fresh({rows, width}, at::kBFloat16, device), v = fresh({rows, width}, at::kBFloat16, device);
  void *stream;
  if (!stream_of(arg[6], stream)) return nullptr;
  return made(unlocked([&] {
                return lib.read(cache, &seqs.s, cu ? static_cast<const int32_t *>(cu->data_ptr()) : nullptr, (int32_t)rows,
                                static_cast<uint16_t *>(k.data_ptr()), width, static_cast<uint16_t *>(v.data_ptr()), width, stream);
              }),
              k, v);
  END_HANDLE_TH_ERRORS
}

// (cache, device, q, page_table, kv_len, max_len, window, scale, stream) -> out
CALL(attend) {
  HANDLE_TH_ERRORS
  const auto *cache = at_address<et_kv_cache>(arg[0]);
  const long device = PyLong_AsLong(arg[1]);
  const Rows q(arg[2], device, cache->head_dim);
  const Seqs seqs(arg[3], arg[4], device);
  const int64_t most = whole(arg[5], INT32_MAX), window = whole(arg[6], INT32_MAX);
  if (!q.t || !seqs.good || q.n != seqs.s.n_seqs || q.heads > INT32_MAX || most < 0 || window < 0 || !PyFloat_CheckExact(arg[7])) Py_RETURN_NONE;
  const float scale = (float)PyFloat_AS_DOUBLE(arg[7]);
  const at::Tensor out = fresh({q.n, q.heads * cache->head_dim}, at::kBFloat16, device);
  const size_t need = lib.attention_bytes(cache, &seqs.s, (int32_t)q.heads, (int32_t)most, (int32_t)window);
  at::Tensor ws;
  if (need) ws = fresh({(int64_t)need}, at::kByte, device);
  void *stream;
  if (!stream_of(arg[8], stream)) return nullptr;
  return made(unlocked([&] {
                return lib.attention(cache, &seqs.s, q.data(), q.stride, (int32_t)q.heads, (int32_t)most, (int32_t)window, scale,
                                     need ? ws.data_ptr() : nullptr, need, static_cast<uint16_t *>(out.data_ptr()), stream);
              }),
              out);
  END_HANDLE_TH_ERRORS
}

// (pool, device, state, state_out, page_table, kv_len, new_len, rows, stream) -> (cu_rows, positions, slots)
CALL(resize) {
  HANDLE_TH_ERRORS
  const auto *pool = at_address<et_kv_pool>(arg[0]);
  const long device = PyLong_AsLong(arg[1]);
  const at::Tensor *state = ints(arg[2], device, 4), *state_out = ints(arg[3], device, 4);
  const Seqs seqs(arg[4], arg[5], device);
  if (!state || !state_out || !seqs.good) Py_RETURN_NONE;
  const at::Tensor *fresh_len = ints(arg[6], device, seqs.s.n_seqs);
  const int64_t rows = whole(arg[7], INT32_MAX);
  if (!fresh_len || rows < 0) Py_RETURN_NONE;
  const int64_t ranges = (int64_t)seqs.s.n_seqs + 1;
  const auto out = fresh({{ranges, at::kInt}, {rows, at::kInt}, {rows, at::kLong}}, device);
  const at::Tensor &cu = out[0], &positions = out[1], &slots = out[2];
  const size_t need = lib.resize_bytes(seqs.s.n_seqs);
  at::Tensor ws;
  if (need) ws = fresh({(int64_t)need}, at::kByte, device);
  void *stream;
  if (!stream_of(arg[8], stream)) return nullptr;
  return made(unlocked([&] {
                return lib.resize(pool, static_cast<const int32_t *>(state->data_ptr()), static_cast<int32_t *>(state_out->data_ptr()),
                                  const_cast<int32_t *>(seqs.s.page_table_dev), seqs.s.table_stride, seqs.s.pages_per_seq, seqs.s.kv_len_dev,
                                  static_cast<const int32_t *>(fresh_len->data_ptr()), seqs.s.n_seqs, (int32_t)rows,
                                  static_cast<int32_t *>(cu.data_ptr()), static_cast<int32_t *>(positions.data_ptr()),
                                  static_cast<int64_t *>(slots.data_ptr()), need ? ws.data_ptr() : nullptr, need, stream);
              }),
              cu, positions, slots);
  END_HANDLE_TH_ERRORS
}

// (rotary, device, q, k or None, positions, q_out or None, k_out or None, transpose, stream) -> (q, k)
CALL(rotate) {
  HANDLE_TH_ERRORS
  const auto *rotary = at_address<et_rotary>(arg[0]);
  const long device = PyLong_AsLong(arg[1]);
  PyObject *out[2] = {nullptr, nullptr};                 // (borrowed where given)
  at::Tensor made_here[2];
  const at::Tensor *wanted[2] = {nullptr, nullptr};
  et_rotary_rows rows[2]{};
  int64_t n = 0;
  for (int i = 0; i < 2; ++i) {
    if (i && arg[3] == Py_None) break;
    const Rows x(arg[2 + i], device, rotary->head_dim);
    if (!x.t || x.heads > 65536 || x.n > INT32_MAX || (i && x.n != n)) Py_RETURN_NONE;
    n = x.n;
    rows[i] = {x.data(), x.stride, nullptr, x.heads * rotary->head_dim, (int32_t)x.heads};
    if (arg[5 + i] != Py_None) {
      const Rows to(arg[5 + i], device, rotary->head_dim);
      if (!to.t || to.n != n || to.heads != x.heads) Py_RETURN_NONE;
      out[i] = arg[5 + i];
      rows[i].out_dev = to.data();
      rows[i].out_stride = to.stride;
    } else {
      wanted[i] = x.t;
    }
  }
  if (wanted[0] && wanted[1]) {
    auto both = fresh({{wanted[0]->sizes(), at::kBFloat16}, {wanted[1]->sizes(), at::kBFloat16}}, device);
    made_here[0] = std::move(both[0]), made_here[1] = std::move(both[1]);
  }
  for (int i = 0; i < 2; ++i)
    if (wanted[i]) {
      if (!made_here[i].defined()) made_here[i] = fresh(wanted[i]->sizes(), at::kBFloat16, device);
      rows[i].out_dev = static_cast<uint16_t *>(made_here[i].data_ptr());
    }
  const at::Tensor *positions = ints(arg[4], device, n);
  if (!positions) Py_RETURN_NONE;
  void *stream;
  if (!stream_of(arg[8], stream)) return nullptr;
  const int rc = unlocked([&] {
    return lib.rotary(rotary, static_cast<const int32_t *>(positions->data_ptr()), (int32_t)n, &rows[0], arg[3] == Py_None ? nullptr : &rows[1],
                      arg[7] == Py_True, stream);
  });
  if (rc) return done(rc);
  for (int i = 0; i < 2; ++i) {
    if (out[i]) Py_INCREF(out[i]);
    else if (made_here[i].defined()) out[i] = THPVariable_Wrap(made_here[i]);
    else Py_INCREF(out[i] = Py_None);
  }
  return Py_BuildValue("(NN)", out[0], out[1]);
  END_HANDLE_TH_ERRORS
}

// (path of the library): looks its entry points up.
PyObject *bind(PyObject *, PyObject *path) {
  const char *name = PyUnicode_AsUTF8(path);
  if (!name) return nullptr;
  void *so = dlopen(name, RTLD_NOW);
  bool all = so != nullptr;
  auto find = [&](auto &to, const char *symbol) {
    if (so) to = reinterpret_cast<std::remove_reference_t<decltype(to)>>(dlsym(so, symbol));
    all = all && to;
  };
  find(lib.append, "et_kv_append");
  find(lib.append_slots, "et_kv_append_slots");
  find(lib.read, "et_kv_read");
  find(lib.attention_bytes, "et_attention_paged_workspace_bytes");
  find(lib.attention, "et_attention_paged");
  find(lib.resize_bytes, "et_kv_resize_workspace_bytes");
  find(lib.resize, "et_kv_resize");
  find(lib.rotary, "et_rotary_apply");
  if (!all) {
    PyErr_Format(PyExc_ImportError, "%s: %s", name, so ? "an entry point is missing" : dlerror());
    return nullptr;
  }
  Py_RETURN_NONE;
}

#define ENTRY(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(append), ENTRY(append_at), ENTRY(read), ENTRY(attend), ENTRY(resize), ENTRY(rotate),
                         {"bind", bind, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module{PyModuleDef_HEAD_INIT, "_calls", "Calls of a decoding step, without Python in between.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }

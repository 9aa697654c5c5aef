// The binding's shortcuts in C++ (module _marshal).  What binding.py does for a call of
// mocap_cache.h -- some ten tensors checked, their addresses taken, ctypes -- costs as much
// host time in Python as the kernel's launch: a rotating append of a token takes 11.1 us
// with it, 7.1 with the tensor checks here and 4.3 with the whole call (the launch alone 3.4).
//
// Nothing is refused here.  Where an argument is not what a call takes, or only unusual,
// the answer is None, and binding.py's own path checks it, says what is wrong or makes the
// call.
//
// The library's call itself runs without the interpreter's lock, as with ctypes: a launch may wait
// for a full queue, or for a stream behind a host function that needs the lock.  The caller
// holds the arguments meanwhile; the tensors that a store or a rotation names are held here.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <limits>

#include "mocap_cache.h"

namespace {

// ---- Tensors ----

// A tensor or parameter (and no other subclass) of this type on this GPU.
const at::Tensor* plain(PyObject* o, at::ScalarType type, long device) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.scalar_type() != type || t.layout() != at::kStrided || !t.is_cuda() || t.get_device() != device) return nullptr;
  return &t;
}
// The same with this many dimensions (-1: any), contiguous.
const at::Tensor* dense(PyObject* o, at::ScalarType type, long ndim, long device) {
  const at::Tensor* t = plain(o, type, device);
  return t != nullptr && (ndim < 0 || t->dim() == ndim) && t->is_contiguous() ? t : nullptr;
}

// bf16 [tokens][heads][head_dim] whose tokens' values are contiguous.
struct Rows {
  void* at = nullptr;
  int64_t stride = 0, tokens = 0, heads = 0, dim = 0;
};
bool rows_of(PyObject* o, long device, Rows* r) {
  const at::Tensor* t = plain(o, at::kBFloat16, device);
  if (t == nullptr || t->dim() != 3) return false;
  r->tokens = t->size(0);
  r->heads = t->size(1);
  r->dim = t->size(2);
  if (t->stride(2) != 1 || (r->heads > 1 && t->stride(1) != r->dim)) return false;
  r->stride = r->tokens > 1 ? t->stride(0) : r->heads * r->dim;
  r->at = t->data_ptr();
  return true;
}

// ---- Numbers and objects ----

bool fits(int64_t x) { return x >= std::numeric_limits<int32_t>::min() && x <= std::numeric_limits<int32_t>::max(); }

bool integer(PyObject* o, int64_t* out) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  *out = PyLong_AsLongLongAndOverflow(o, &over);
  return over == 0;
}
bool integer32(PyObject* o, int32_t* out) {
  int64_t x;
  if (!integer(o, &x) || !fits(x)) return false;
  *out = (int32_t)x;
  return true;
}

// An attribute, released at the end of its scope.
struct Attr {
  PyObject* o = nullptr;
  Attr() = default;
  Attr(PyObject* from, PyObject* name) { get(from, name); }
  Attr(const Attr&) = delete;
  Attr& operator=(const Attr&) = delete;
  ~Attr() { Py_XDECREF(o); }
  void get(PyObject* from, PyObject* name) {
    Py_XSETREF(o, PyObject_GetAttr(from, name));
    if (o == nullptr) PyErr_Clear();
  }
};
PyObject *n_k_pool, *n_v_pool, *n_k_scale, *n_v_scale, *n_num_blocks, *n_block_size, *n_h_kv, *n_head_dim, *n_inv_freq,
    *n_interleaved;

bool number(PyObject* from, PyObject* name, int32_t* out) {
  const Attr a(from, name);
  return a.o != nullptr && integer32(a.o, out);
}
bool pool(PyObject* from, PyObject* name, at::ScalarType type, long ndim, long device, Attr* held, void** out) {
  held->get(from, name);
  const at::Tensor* t = held->o != nullptr ? dense(held->o, type, ndim, device) : nullptr;
  if (t == nullptr) return false;
  *out = t->data_ptr();
  return true;
}

// A KvStore or (four) a Kv4Store.
struct Store {
  mocap_kv_store b;
  mocap_kv4_store q;
  int32_t h_kv, head_dim;
  Attr held[4];
};
bool store_of(PyObject* o, bool four, long device, Store* s) {
  int32_t blocks, size;
  if (!number(o, n_num_blocks, &blocks) || !number(o, n_block_size, &size) || !number(o, n_h_kv, &s->h_kv) ||
      !number(o, n_head_dim, &s->head_dim))
    return false;
  if (!four) {
    s->b = mocap_kv_store{nullptr, nullptr, blocks, size, s->h_kv, s->head_dim};
    return pool(o, n_k_pool, at::kBFloat16, 4, device, &s->held[0], &s->b.k_pool) &&
           pool(o, n_v_pool, at::kBFloat16, 4, device, &s->held[1], &s->b.v_pool);
  }
  s->q = mocap_kv4_store{nullptr, nullptr, nullptr, nullptr, blocks, size, s->h_kv, s->head_dim};
  return pool(o, n_k_pool, at::kByte, 4, device, &s->held[0], &s->q.k_pool) &&
         pool(o, n_v_pool, at::kByte, 5, device, &s->held[1], &s->q.v_pool) &&
         pool(o, n_k_scale, at::kByte, 5, device, &s->held[2], &s->q.k_scale) &&
         pool(o, n_v_scale, at::kByte, 5, device, &s->held[3], &s->q.v_scale);
}

// A Rope or None.
bool rope_of(PyObject* o, long device, Attr* held, mocap_rope* r, const mocap_rope** out) {
  *out = nullptr;
  if (o == Py_None) return true;
  held->get(o, n_inv_freq);
  const Attr i(o, n_interleaved);
  if (held->o == nullptr || i.o == nullptr || !PyBool_Check(i.o)) return false;
  const at::Tensor* t = dense(held->o, at::kFloat, 1, device);
  if (t == nullptr || t->size(0) > (1 << 20)) return false;
  *r = mocap_rope{static_cast<const float*>(t->data_ptr()), (int32_t)(2 * t->size(0)), i.o == Py_True};
  *out = r;
  return true;
}

// What the rotating appends take: k, v, rope, q, q_out.
struct Append {
  Store store;
  Rows k, v, q;
  Attr inv_freq;
  mocap_rope rope_value;
  const mocap_rope* rope;
  void* q_out = nullptr;
};
bool append_of(PyObject* store, bool four, PyObject* k, PyObject* v, PyObject* rope, PyObject* q, PyObject* q_out,
               long device, Append* a) {
  if (!store_of(store, four, device, &a->store) || !rows_of(k, device, &a->k) || !rows_of(v, device, &a->v)) return false;
  if (a->k.tokens != a->v.tokens || a->k.heads != a->v.heads || a->k.dim != a->v.dim || a->k.heads != a->store.h_kv ||
      a->k.dim != a->store.head_dim || !fits(a->k.tokens))
    return false;
  if (q != Py_None) {
    if (!rows_of(q, device, &a->q) || a->q.tokens != a->k.tokens || a->q.dim != a->k.dim || !fits(a->q.heads)) return false;
    const at::Tensor* out = dense(q_out, at::kBFloat16, 3, device);
    if (out == nullptr || out->size(0) != a->q.tokens || out->size(1) != a->q.heads || out->size(2) != a->q.dim)
      return false;
    a->q_out = out->data_ptr();
  } else if (q_out != Py_None) {
    return false;
  }
  return rope_of(rope, device, &a->inv_freq, &a->rope_value, &a->rope);
}

// Block tables [batch][stride] and lengths [batch].
struct Batch {
  const int32_t *tables, *lens;
  int32_t batch, stride;
};
bool batch_of(PyObject* tables, PyObject* lens, long device, Batch* b) {
  const at::Tensor *t = dense(tables, at::kInt, 2, device), *n = dense(lens, at::kInt, 1, device);
  if (t == nullptr || n == nullptr || !fits(t->size(0)) || !fits(t->size(1)) || n->size(0) != t->size(0)) return false;
  *b = Batch{static_cast<const int32_t*>(t->data_ptr()), static_cast<const int32_t*>(n->data_ptr()), (int32_t)t->size(0),
             (int32_t)t->size(1)};
  return true;
}

// q, o bf16 [rows][h_q][d] and lse fp32; workspace any contiguous tensor or None.
struct Attn {
  const void* q;
  void *o, *workspace = nullptr;
  float *lse;
  size_t bytes = 0;
  int32_t rows, h_q, dim;
  float scale;
};
bool attn_of(PyObject* q, PyObject* scale, PyObject* o, PyObject* lse, PyObject* workspace, bool rows_first, long device,
             Attn* a) {
  const at::Tensor *tq = dense(q, at::kBFloat16, 3, device), *to = dense(o, at::kBFloat16, 3, device);
  const at::Tensor* tl = dense(lse, at::kFloat, 2, device);
  if (tq == nullptr || to == nullptr || tl == nullptr || !PyFloat_CheckExact(scale) || to->sizes() != tq->sizes()) return false;
  const int64_t rows = tq->size(0), h_q = tq->size(1), dim = tq->size(2);
  if (!fits(rows) || !fits(h_q) || !fits(dim) || tl->size(rows_first ? 0 : 1) != rows || tl->size(rows_first ? 1 : 0) != h_q)
    return false;
  if (workspace != Py_None) {
    if (!THPVariable_CheckExact(workspace)) return false;
    const at::Tensor* w = dense(workspace, THPVariable_Unpack(workspace).scalar_type(), -1, device);
    if (w == nullptr) return false;
    a->workspace = w->data_ptr();
    a->bytes = w->nbytes();
  }
  a->q = tq->data_ptr();
  a->o = to->data_ptr();
  a->lse = static_cast<float*>(tl->data_ptr());
  a->rows = (int32_t)rows;
  a->h_q = (int32_t)h_q;
  a->dim = (int32_t)dim;
  a->scale = (float)PyFloat_AS_DOUBLE(scale);
  return true;
}

// The handle of the stream and the current device, the last two arguments of every call.
bool place(PyObject* const* last, void** stream, long* device) {
  *stream = nullptr;
  int64_t x, h = 0;
  if (!integer(last[1], &x) || (last[0] != Py_None && !integer(last[0], &h))) return false;
  *device = (long)x;
  *stream = reinterpret_cast<void*>(h);
  return true;
}

// ---- The library's calls ----

struct {
  decltype(&mocap_rope_append) rope_append;
  decltype(&mocap_decode_rope_append) decode_rope_append;
  decltype(&mocap_kv4_append) kv4_append;
  decltype(&mocap_kv4_decode_append) kv4_decode_append;
  decltype(&mocap_kv4_load) kv4_load;
  decltype(&mocap_kv4_decode_attn) kv4_decode_attn;
  decltype(&mocap_kv4_chunk_attn) kv4_chunk_attn;
} lib;

// bind(name, address): where a call of the loaded library is.
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  const char* name = n == 2 ? PyUnicode_AsUTF8(args[0]) : nullptr;
  void* at = name != nullptr ? PyLong_AsVoidPtr(args[1]) : nullptr;
  if (PyErr_Occurred()) return nullptr;
#define MOCAP_BIND(call) \
  if (name != nullptr && std::strcmp(name, "mocap_" #call) == 0) return lib.call = reinterpret_cast<decltype(lib.call)>(at), Py_NewRef(Py_None);
  MOCAP_BIND(rope_append)
  MOCAP_BIND(decode_rope_append)
  MOCAP_BIND(kv4_append)
  MOCAP_BIND(kv4_decode_append)
  MOCAP_BIND(kv4_load)
  MOCAP_BIND(kv4_decode_attn)
  MOCAP_BIND(kv4_chunk_attn)
#undef MOCAP_BIND
  PyErr_SetString(PyExc_ValueError, "bind(name, address)");
  return nullptr;
}

// Makes a call without the interpreter's lock.
struct Unlocked {
  PyThreadState* state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};
template <typename... P, typename... A>
PyObject* made(mocap_status (*call)(P...), A... args) {
  mocap_status st;
  {
    const Unlocked u;
    st = call(args...);
  }
  return PyLong_FromLong(st);
}

// append_chunk(store, table, start_pos, k, v, rope, position, q, q_out, stream, device)
template <bool FOUR>
PyObject* append_chunk(PyObject* const* a) {
  void* stream;
  long device;
  Append p;
  int64_t start, position;
  if (!place(a + 9, &stream, &device) || !integer(a[2], &start)) return nullptr;
  position = start;
  if (a[6] != Py_None && !integer(a[6], &position)) return nullptr;
  const at::Tensor* table = dense(a[1], at::kInt, 1, device);
  if (table == nullptr || !fits(table->size(0)) || !append_of(a[0], FOUR, a[3], a[4], a[5], a[7], a[8], device, &p))
    return nullptr;
  const int32_t* t = static_cast<const int32_t*>(table->data_ptr());
  const int32_t n = (int32_t)table->size(0), tokens = (int32_t)p.k.tokens, h_q = (int32_t)p.q.heads;
  if (FOUR)
    return made(lib.kv4_append, &p.store.q, t, n, start, tokens, p.rope, position, p.q.at, p.q.stride, h_q, p.k.at,
                p.k.stride, p.v.at, p.v.stride, p.q_out, stream);
  return made(lib.rope_append, &p.store.b, t, n, start, tokens, p.rope, position, p.q.at, p.q.stride, h_q, p.k.at,
              p.k.stride, p.v.at, p.v.stride, p.q_out, stream);
}

// append_batch(store, tables, lens, k, v, rope, positions, q, q_out, stream, device)
template <bool FOUR>
PyObject* append_batch(PyObject* const* a) {
  void* stream;
  long device;
  Append p;
  Batch b;
  const int32_t* positions = nullptr;
  if (!place(a + 9, &stream, &device) || !batch_of(a[1], a[2], device, &b) ||
      !append_of(a[0], FOUR, a[3], a[4], a[5], a[7], a[8], device, &p) || p.k.tokens != b.batch)
    return nullptr;
  if (a[6] != Py_None) {
    const at::Tensor* t = dense(a[6], at::kInt, 1, device);
    if (t == nullptr || t->size(0) != b.batch) return nullptr;
    positions = static_cast<const int32_t*>(t->data_ptr());
  }
  const int32_t h_q = (int32_t)p.q.heads;
  if (FOUR)
    return made(lib.kv4_decode_append, &p.store.q, b.tables, b.stride, b.lens, b.batch, p.rope, positions, p.q.at,
                p.q.stride, h_q, p.k.at, p.k.stride, p.v.at, p.v.stride, p.q_out, stream);
  return made(lib.decode_rope_append, &p.store.b, b.tables, b.stride, b.lens, b.batch, p.rope, positions, p.q.at,
              p.q.stride, h_q, p.k.at, p.k.stride, p.v.at, p.v.stride, p.q_out, stream);
}

// load(store, tables, ends, k, v, stream, device)
PyObject* load(PyObject* const* a) {
  void* stream;
  long device;
  Store s;
  Batch b;
  if (!place(a + 5, &stream, &device) || !store_of(a[0], true, device, &s) || !batch_of(a[1], a[2], device, &b))
    return nullptr;
  const at::Tensor *k = dense(a[3], at::kBFloat16, 4, device), *v = dense(a[4], at::kBFloat16, 4, device);
  if (k == nullptr || v == nullptr || k->sizes() != v->sizes() || k->size(0) != b.batch || !fits(k->size(1)) ||
      k->size(2) != s.h_kv || k->size(3) != s.head_dim)
    return nullptr;
  return made(lib.kv4_load, &s.q, b.tables, b.stride, b.lens, b.batch, (int32_t)k->size(1), k->data_ptr(), v->data_ptr(),
              stream);
}

// decode_attn(store, tables, lens, q, max_len, scale, o, lse, workspace, window, sinks, stream, device)
PyObject* decode_attn(PyObject* const* a) {
  void* stream;
  long device;
  Store s;
  Batch b;
  Attn t;
  int64_t max_len, window, sinks;
  if (!place(a + 11, &stream, &device) || !integer(a[4], &max_len) || !integer(a[9], &window) || !integer(a[10], &sinks) ||
      !store_of(a[0], true, device, &s) || !batch_of(a[1], a[2], device, &b) ||
      !attn_of(a[3], a[5], a[6], a[7], a[8], true, device, &t) || t.rows != b.batch)
    return nullptr;
  return made(lib.kv4_decode_attn, &s.q, b.tables, b.stride, b.lens, b.batch, max_len, t.q, t.h_q, s.h_kv, t.dim, t.scale,
              window, sinks, t.o, t.lse, t.workspace, t.bytes, stream);
}

// chunk_attn(store, table, q, prefix_len, scale, o, lse, workspace, window, sinks, num_splits, stream, device)
PyObject* chunk_attn(PyObject* const* a) {
  void* stream;
  long device;
  Store s;
  Attn t;
  int64_t prefix, window, sinks;
  int32_t splits;
  if (!place(a + 11, &stream, &device) || !integer(a[3], &prefix) || !integer(a[8], &window) || !integer(a[9], &sinks) ||
      !integer32(a[10], &splits) || !store_of(a[0], true, device, &s) ||
      !attn_of(a[2], a[4], a[5], a[6], a[7], false, device, &t))
    return nullptr;
  const at::Tensor* table = dense(a[1], at::kInt, 1, device);
  if (table == nullptr || !fits(table->size(0))) return nullptr;
  return made(lib.kv4_chunk_attn, &s.q, static_cast<const int32_t*>(table->data_ptr()), (int32_t)table->size(0), t.q, prefix,
              t.rows, t.h_q, s.h_kv, t.dim, t.scale, window, sinks, t.o, t.lse, t.workspace, t.bytes,
              splits, stream);
}

// A call with N arguments: its status, or None.  (Calls whose library is not loaded too.)
template <PyObject* (*CALL)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments", N);
    return nullptr;
  }
  if (lib.kv4_chunk_attn == nullptr) Py_RETURN_NONE;
  try {
    PyObject* r = CALL(args);
    if (r == nullptr && !PyErr_Occurred()) Py_RETURN_NONE;
    return r;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// ---- For the calls that binding.py makes itself ----

// address(tensor, dtype, ndim or -1, device): the address of a contiguous tensor, or None.
PyObject* address(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 4 || !THPDtype_Check(args[1])) {
    PyErr_SetString(PyExc_TypeError, "address(tensor, dtype, ndim, device)");
    return nullptr;
  }
  const long ndim = PyLong_AsLong(args[2]), device = PyLong_AsLong(args[3]);
  if (PyErr_Occurred()) return nullptr;
  try {
    const at::Tensor* t = dense(args[0], reinterpret_cast<THPDtype*>(args[1])->scalar_type, ndim, device);
    if (t == nullptr) Py_RETURN_NONE;
    return PyLong_FromVoidPtr(t->data_ptr());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// rows(tensor, device): (address, stride, tokens, heads, head_dim), or None.
PyObject* rows(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 2) {
    PyErr_SetString(PyExc_TypeError, "rows(tensor, device)");
    return nullptr;
  }
  const long device = PyLong_AsLong(args[1]);
  if (PyErr_Occurred()) return nullptr;
  try {
    Rows r;
    if (!rows_of(args[0], device, &r)) Py_RETURN_NONE;
    return Py_BuildValue("(KLLLL)", (unsigned long long)reinterpret_cast<uintptr_t>(r.at), (long long)r.stride,
                         (long long)r.tokens, (long long)r.heads, (long long)r.dim);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

template <typename F>
PyMethodDef method(const char* name, F f) {
  return PyMethodDef{name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL, nullptr};
}
PyMethodDef methods[] = {method("bind", bind),
                         method("address", address),
                         method("rows", rows),
                         method("mocap_rope_append", entry<append_chunk<false>, 11>),
                         method("mocap_kv4_append", entry<append_chunk<true>, 11>),
                         method("mocap_decode_rope_append", entry<append_batch<false>, 11>),
                         method("mocap_kv4_decode_append", entry<append_batch<true>, 11>),
                         method("mocap_kv4_load", entry<load, 7>),
                         method("mocap_kv4_decode_attn", entry<decode_attn, 13>),
                         method("mocap_kv4_chunk_attn", entry<chunk_attn, 13>),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
  const struct {
    PyObject** at;
    const char* name;
  } names[] = {{&n_k_pool, "k_pool"},         {&n_v_pool, "v_pool"},     {&n_k_scale, "k_scale"},
               {&n_v_scale, "v_scale"},       {&n_num_blocks, "num_blocks"}, {&n_block_size, "block_size"},
               {&n_h_kv, "h_kv"},             {&n_head_dim, "head_dim"}, {&n_inv_freq, "inv_freq"},
               {&n_interleaved, "interleaved"}};
  for (const auto& x : names)
    if ((*x.at = PyUnicode_InternFromString(x.name)) == nullptr) return nullptr;
  PyObject* m = PyModule_Create(&module);
  if (m != nullptr && PyModule_AddStringConstant(m, "torch_version", MOCAP_TORCH) < 0) Py_CLEAR(m);
  return m;
}

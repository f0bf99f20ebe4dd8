// Regular calls of the cache's C ABI (include/mars_cache.h) from Python: checks the tensors and takes their addresses in native code, for
// the reason that marshal.cpp gives -- a step makes several such calls per layer, the smallest of which take the GPU 2 to 8 us, and through
// ctypes each costs the host about 8.
//
// A function here handles a call only if all of it is as the binding asks for.  For anything else it returns None, having done nothing, and the binding
// goes its general way, which says what is wrong.
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>

#include "../../include/mars_cache.h"

namespace {

using at::Tensor;
struct Irregular {};

decltype(&mars_kv_append) f_append;
decltype(&mars_kv_read) f_read;
decltype(&mars_tree_mask) f_mask;
decltype(&mars_kv_attention) f_attention;
decltype(&mars_kv_commit) f_commit;
decltype(&mars_kv_reserve) f_reserve;
decltype(&mars_kv_fork) f_fork;
decltype(&mars_kv_release) f_release;
bool g_on_gpu = true;  // (tests of this file alone look at tensors that are not)

void require(bool ok) { if (!ok) throw Irregular(); }
// A plain tensor (no subclass, whose own ways Python knows), on the GPU.
const Tensor& tensor(PyObject* o) {
  require(THPVariable_CheckExact(o));
  const Tensor& t = THPVariable_Unpack(o);
  require(t.is_cuda() || !g_on_gpu);
  return t;
}
int narrow(int64_t x) {
  require(x >= 0 && x <= 0x7FFFFFFF);
  return static_cast<int>(x);
}
int integer(PyObject* o) {
  require(PyLong_CheckExact(o));
  int over = 0;
  const long x = PyLong_AsLongAndOverflow(o, &over);
  require(!over && x >= -0x7FFFFFFFL - 1 && x <= 0x7FFFFFFFL);
  return static_cast<int>(x);
}
int code(const Tensor& t) {
  const auto s = t.scalar_type();
  if (s == at::kFloat) return MARS_F32;
  require(s == at::kBFloat16 || s == at::kUInt16 || s == at::kShort);
  return MARS_BF16;
}
// [n] int32; NULL for None.
int32_t* numbers(PyObject* o, int64_t n) {
  if (o == Py_None) return nullptr;
  const Tensor& t = tensor(o);
  require(t.scalar_type() == at::kInt && t.dim() == 1 && t.size(0) == n && t.is_contiguous());
  return static_cast<int32_t*>(t.data_ptr());
}
int32_t* there(int32_t* p) {
  require(p != nullptr);
  return p;
}
// [a, b] int32.
int32_t* grid(PyObject* o, int64_t a, int64_t b) {
  const Tensor& t = tensor(o);
  require(t.scalar_type() == at::kInt && t.dim() == 2 && t.size(0) == a && t.size(1) == b && t.is_contiguous());
  return static_cast<int32_t*>(t.data_ptr());
}
mars_kv_rows rows(const Tensor& t, int64_t B, int64_t N, int64_t heads, int64_t D) {
  require(t.dim() == 4 && t.size(0) == B && t.size(1) == N && t.size(2) == heads && t.size(3) == D && t.stride(3) == 1);
  return {t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)};
}
// (asked for last, when everything else is as it should be)
void* stream_of(PyObject* ask) {
  PyObject* o = PyObject_CallNoArgs(ask);
  require(o != nullptr);
  void* s = PyLong_AsVoidPtr(o);
  Py_DECREF(o);
  require(!PyErr_Occurred());
  return s;
}
template <typename Call> PyObject* regular(Call call) {
  try {
    return PyLong_FromLong(call());
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}
template <typename Run> int unlocked(Run run) {
  PyThreadState* s = PyEval_SaveThread();
  const int rc = run();
  PyEval_RestoreThread(s);
  return rc;
}

// The cache of a call; head_dim and page_size: one of them is given, the other follows from the bytes of a head.
mars_kv_cache cache_of(PyObject* pool, PyObject* table, int64_t head_dim, int64_t page_size) {
  const Tensor &p = tensor(pool), &t = tensor(table);
  require(p.scalar_type() == at::kByte && p.dim() == 4 && p.is_contiguous());
  require(t.scalar_type() == at::kInt && t.dim() == 2 && t.is_contiguous());
  const int64_t blk = p.size(3);
  if (page_size > 0 && head_dim == 0) head_dim = blk * 16 / (17 * page_size);
  else if (head_dim > 0) page_size = blk * 16 / (17 * head_dim);
  require(head_dim > 0 && page_size > 0 && page_size * (head_dim + head_dim / 16) == blk);
  mars_kv_cache c = {};
  c.pool = p.data_ptr();
  c.page_table = static_cast<int32_t*>(t.data_ptr());
  c.layers = narrow(p.size(0)); c.pages = narrow(p.size(1)); c.heads = narrow(p.size(2));
  c.dim = narrow(head_dim); c.page = narrow(page_size);
  c.sequences = narrow(t.size(0)); c.width = narrow(t.size(1));
  return c;
}
// The tables alone (the calls that move no rows): the pool's part of the sizes is made up.
mars_kv_cache tables_of(PyObject* table, PyObject* lens, PyObject* held, PyObject* refs, int page_size) {
  const Tensor &t = tensor(table), &r = tensor(refs);
  require(t.scalar_type() == at::kInt && t.dim() == 2 && t.is_contiguous());
  require(r.scalar_type() == at::kInt && r.dim() == 1 && r.is_contiguous());
  mars_kv_cache c = {};
  c.page_table = static_cast<int32_t*>(t.data_ptr());
  c.layers = c.heads = 1; c.dim = 64; c.page = page_size;
  c.pages = narrow(r.size(0)); c.sequences = narrow(t.size(0)); c.width = narrow(t.size(1));
  c.lens = there(numbers(lens, c.sequences)); c.held = there(numbers(held, c.sequences)); c.refs = static_cast<int32_t*>(r.data_ptr());
  return c;
}
// Requests of a call are those of seqs, or the first sequences.
int32_t* sequences(PyObject* seqs, int64_t B, const mars_kv_cache& c) {
  require(seqs != Py_None || B <= c.sequences);
  return numbers(seqs, B);
}

// pool, page_table, lens, k, v, layer, seqs, n_new, status, stream
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular([&]() -> int {
    require(n == 10);
    const Tensor &k = tensor(a[3]), &v = tensor(a[4]);
    require(k.dim() == 4 && v.scalar_type() == k.scalar_type());
    const int B = narrow(k.size(0)), N = narrow(k.size(1)), dtype = code(k), layer = integer(a[5]);
    mars_kv_cache c = cache_of(a[0], a[1], k.size(3), 0);
    c.lens = there(numbers(a[2], c.sequences));
    const mars_kv_rows kr = rows(k, B, N, c.heads, c.dim), vr = rows(v, B, N, c.heads, c.dim);
    const int32_t *seqs = sequences(a[6], B, c), *n_new = numbers(a[7], B);
    int32_t* status = numbers(a[8], B);
    void* stream = stream_of(a[9]);
    return unlocked([&]() { return f_append(&c, layer, seqs, &kr, &vr, dtype, n_new, B, N, status, stream); });
  });
}
// pool, page_table, held, k, v, layer, seqs, first, stream
PyObject* read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular([&]() -> int {
    require(n == 9);
    const Tensor &k = tensor(a[3]), &v = tensor(a[4]);
    require(k.dim() == 4 && v.scalar_type() == k.scalar_type());
    const int B = narrow(k.size(0)), N = narrow(k.size(1)), dtype = code(k), layer = integer(a[5]);
    mars_kv_cache c = cache_of(a[0], a[1], k.size(3), 0);
    c.held = numbers(a[2], c.sequences);
    const mars_kv_rows kr = rows(k, B, N, c.heads, c.dim), vr = rows(v, B, N, c.heads, c.dim);
    const int32_t *seqs = sequences(a[6], B, c), *first = numbers(a[7], B);
    void* stream = stream_of(a[8]);
    return unlocked([&]() { return f_read(&c, layer, seqs, first, &kr, &vr, dtype, B, N, stream); });
  });
}
uint64_t* words(PyObject* o, int64_t B, int64_t N) {
  if (o == Py_None) return nullptr;
  const Tensor& t = tensor(o);
  require(t.scalar_type() == at::kLong && t.dim() == 3 && t.size(0) == B && t.size(1) == N && t.size(2) == (N + 63) / 64 && t.is_contiguous());
  return static_cast<uint64_t*>(t.data_ptr());
}
// tree_parent, n_new, mask, status, stream
PyObject* tree_mask(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular([&]() -> int {
    require(n == 5 && a[2] != Py_None);
    const Tensor& p = tensor(a[0]);
    require(p.dim() == 2);
    const int B = narrow(p.size(0)), N = narrow(p.size(1));
    const int32_t *parent = grid(a[0], B, N), *n_new = numbers(a[1], B);
    uint64_t* mask = words(a[2], B, N);
    int32_t* status = numbers(a[3], B);
    void* stream = stream_of(a[4]);
    return unlocked([&]() { return f_mask(parent, n_new, B, N, mask, status, stream); });
  });
}
// pool, page_table, lens, q, layer, seqs, n_new, mask, scale, max_len, out, lse, workspace, stream
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular([&]() -> int {
    require(n == 14);
    const Tensor &q = tensor(a[3]), &out = tensor(a[10]), &ws = tensor(a[12]);
    require(q.dim() == 4 && out.scalar_type() == q.scalar_type() && ws.is_contiguous() && ws.scalar_type() == at::kByte);
    const int B = narrow(q.size(0)), N = narrow(q.size(1)), q_heads = narrow(q.size(2)), dtype = code(q), layer = integer(a[4]);
    mars_kv_cache c = cache_of(a[0], a[1], q.size(3), 0);
    c.lens = there(numbers(a[2], c.sequences));
    const mars_kv_rows qr = rows(q, B, N, q_heads, c.dim), outr = rows(out, B, N, q_heads, c.dim);
    const int32_t *seqs = sequences(a[5], B, c), *n_new = numbers(a[6], B);
    const uint64_t* mask = words(a[7], B, N);
    float scale = static_cast<float>(1.0 / std::sqrt(static_cast<double>(c.dim)));
    if (a[8] != Py_None) {
      require(PyFloat_CheckExact(a[8]));
      scale = static_cast<float>(PyFloat_AS_DOUBLE(a[8]));
    }
    const int max_len = integer(a[9]);
    float* lse = nullptr;
    if (a[11] != Py_None) {
      const Tensor& t = tensor(a[11]);
      require(t.scalar_type() == at::kFloat && t.dim() == 3 && t.size(0) == B && t.size(1) == N && t.size(2) == q_heads && t.is_contiguous());
      lse = static_cast<float*>(t.data_ptr());
    }
    void *work = ws.data_ptr(), *stream = stream_of(a[13]);
    const size_t bytes = static_cast<size_t>(ws.numel());
    return unlocked([&]() {
      return f_attention(&c, layer, seqs, &qr, dtype, q_heads, n_new, mask, scale, max_len, &outr, lse, B, N, work, bytes, stream);
    });
  });
}
// pool, page_table, lens, accept_len, path_idx, page_size, seqs, new_lens, status, stream
PyObject* commit(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular([&]() -> int {
    require(n == 10);
    mars_kv_cache c = cache_of(a[0], a[1], 0, integer(a[5]));
    c.lens = there(numbers(a[2], c.sequences));
    const Tensor& p = tensor(a[4]);
    require(p.dim() == 2);
    const int B = narrow(p.size(0)), N = narrow(p.size(1));
    const int32_t *path = grid(a[4], B, N), *accept = there(numbers(a[3], B)), *seqs = sequences(a[6], B, c);
    int32_t *lens = there(numbers(a[7], c.sequences)), *status = numbers(a[8], B);
    void* stream = stream_of(a[9]);
    return unlocked([&]() { return f_commit(&c, seqs, accept, path, B, N, lens, status, stream); });
  });
}
// pool, page_table, lens, held, refs, n, page_size, seqs, status, workspace, stream
PyObject* reserve(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular([&]() -> int {
    require(n == 11);
    mars_kv_cache c = cache_of(a[0], a[1], 0, integer(a[6]));
    c.lens = there(numbers(a[2], c.sequences)); c.held = there(numbers(a[3], c.sequences)); c.refs = there(numbers(a[4], c.pages));
    const Tensor &st = tensor(a[8]), &ws = tensor(a[9]);
    require(st.dim() == 1 && ws.is_contiguous() && ws.scalar_type() == at::kByte);
    const int B = narrow(st.size(0));
    int32_t* status = numbers(a[8], B);
    const int32_t *seqs = sequences(a[7], B, c), *n_new = nullptr;
    int N = 1 << 24;
    if (PyLong_CheckExact(a[5])) N = integer(a[5]);
    else n_new = there(numbers(a[5], B));
    require(seqs || n_new || B == c.sequences);
    void *work = ws.data_ptr(), *stream = stream_of(a[10]);
    const size_t bytes = static_cast<size_t>(ws.numel());
    return unlocked([&]() { return f_reserve(&c, seqs, n_new, B, N, status, work, bytes, stream); });
  });
}
// page_table, lens, held, refs, src, dst, page_size, status, stream
PyObject* fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular([&]() -> int {
    require(n == 9);
    const mars_kv_cache c = tables_of(a[0], a[1], a[2], a[3], integer(a[6]));
    const int B = narrow(tensor(a[4]).numel());
    const int32_t *src = numbers(a[4], B), *dst = there(numbers(a[5], B));
    int32_t* status = numbers(a[7], B);
    void* stream = stream_of(a[8]);
    return unlocked([&]() { return f_fork(&c, src, dst, B, status, stream); });
  });
}
// page_table, lens, held, refs, seqs, status, stream
PyObject* release(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return regular([&]() -> int {
    require(n == 7);
    const mars_kv_cache c = tables_of(a[0], a[1], a[2], a[3], 8);
    const int B = narrow(tensor(a[4]).numel());
    const int32_t* seqs = numbers(a[4], B);
    int32_t* status = numbers(a[5], B);
    void* stream = stream_of(a[6]);
    return unlocked([&]() { return f_release(&c, seqs, B, status, stream); });
  });
}

// The addresses of the library's functions, in the order of the functions above, and whether tensors have to be on the GPU.
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* at[8];
  if (n != 9) { PyErr_SetString(PyExc_TypeError, "bind: eight addresses and a truth value"); return nullptr; }
  for (int i = 0; i < 8; ++i) {
    at[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  f_append = reinterpret_cast<decltype(f_append)>(at[0]);
  f_read = reinterpret_cast<decltype(f_read)>(at[1]);
  f_mask = reinterpret_cast<decltype(f_mask)>(at[2]);
  f_attention = reinterpret_cast<decltype(f_attention)>(at[3]);
  f_commit = reinterpret_cast<decltype(f_commit)>(at[4]);
  f_reserve = reinterpret_cast<decltype(f_reserve)>(at[5]);
  f_fork = reinterpret_cast<decltype(f_fork)>(at[6]);
  f_release = reinterpret_cast<decltype(f_release)>(at[7]);
  g_on_gpu = a[8] == Py_True;
  Py_RETURN_NONE;
}

#define MARS_METHOD(F) {#F, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(F)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {MARS_METHOD(bind),   MARS_METHOD(append),  MARS_METHOD(read), MARS_METHOD(tree_mask), MARS_METHOD(attention),
                           MARS_METHOD(commit), MARS_METHOD(reserve), MARS_METHOD(fork), MARS_METHOD(release),   {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_cache_marshal", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__cache_marshal() {
  PyObject* m = PyModule_Create(&g_module);
  // (what it was built against: the binding looks at no tensor through another version's layout)
  if (m && PyModule_AddStringConstant(m, "torch_version", MARS_TORCH_VERSION) != 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}

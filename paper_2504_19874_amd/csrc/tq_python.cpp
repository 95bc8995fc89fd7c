// The per-call half of the Python binding: reads what a call's tensors are, and calls the C ABI.
//
// A decoding step makes three calls whose kernels take 5 - 20 us each.  Marshalled in Python (attribute look-ups on a
// dozen tensors, a ctypes object per pointer, a stream object) such a call costs the host 10 - 15 us, more than the GPU
// needs for it; here the same work is a few hundred nanoseconds.
//
// Every function takes the tq_params struct as a buffer and returns the library's status, or None where an argument is
// not what the plain call has (a wrong type, dtype, device, layout or size, a workspace to be grown): nothing has been
// done then, and the caller takes its checked path, which raises the error or does the call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/turboquant.h"

namespace {

struct NotPlain {};

const tq_params* params(PyObject* o) {
  // the struct belongs to a Params object that the caller holds for the length of the call
  Py_buffer b;
  if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) {
    PyErr_Clear();
    throw NotPlain{};
  }
  const bool whole = (size_t)b.len == sizeof(tq_params);
  const tq_params* p = static_cast<const tq_params*>(b.buf);
  PyBuffer_Release(&b);
  if (!whole) throw NotPlain{};
  return p;
}

int64_t integer(PyObject* o) {
  if (!PyLong_CheckExact(o)) throw NotPlain{};
  int overflow = 0;
  const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
  if (overflow != 0) throw NotPlain{};
  return v;
}

int32_t integer32(PyObject* o) {
  const int64_t v = integer(o);
  if (v != (int32_t)v) throw NotPlain{};
  return (int32_t)v;
}

// (plain Tensor or Parameter objects only: a subclass may answer questions about itself in its own way)
const at::Tensor* tensor(PyObject* o) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_CheckExact(o)) throw NotPlain{};
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) throw NotPlain{};
  return &t;
}

// a code array: contiguous, at least `numel` elements of `type`
template <class T>
T* array(PyObject* o, c10::ScalarType type, int64_t numel) {
  const at::Tensor* t = tensor(o);
  if (t == nullptr) return nullptr;
  if (t->scalar_type() != type || t->numel() < numel || !t->is_contiguous()) throw NotPlain{};
  return static_cast<T*>(t->data_ptr());
}

// a matrix with contiguous rows, which may be padded
struct Rows {
  void* ptr;
  int64_t rows, cols, stride;
  c10::ScalarType type;
};
Rows matrix(PyObject* o) {
  const at::Tensor* t = tensor(o);
  if (t == nullptr || t->dim() != 2 || (t->size(1) > 1 && t->stride(1) != 1)) throw NotPlain{};
  return Rows{t->data_ptr(), t->size(0), t->size(1), t->stride(0), t->scalar_type()};
}

struct Codes {
  uint32_t *idx, *qjl;
  float *gamma, *norm;
};
Codes codes(const tq_params* p, PyObject* const* o, int64_t rows) {
  const int64_t words = (int64_t)(p->d_hi / 32) * p->bits_mse_hi + (int64_t)((p->d - p->d_hi) / 32) * p->bits_mse;
  const int64_t scalars = p->d_hi != 0 ? 2 : 1;
  if (rows < 0) throw NotPlain{};
  Codes c;
  c.idx = array<uint32_t>(o[0], at::kInt, rows * words);
  c.qjl = array<uint32_t>(o[1], at::kInt, rows * (p->d / 32));
  c.gamma = array<float>(o[2], at::kFloat, rows * scalars);
  c.norm = array<float>(o[3], at::kFloat, rows * scalars);
  return c;
}

int32_t vector_type(const Rows& x) {
  if (x.type == at::kFloat) return TQ_F32;
  if (x.type == at::kBFloat16) return TQ_BF16;
  throw NotPlain{};
}

void* stream() { return static_cast<void*>(c10::hip::getCurrentHIPStream().stream()); }

template <class F>
PyObject* call(Py_ssize_t got, Py_ssize_t want, F f) {
  if (got != want) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return PyLong_FromLong((long)f());
  } catch (const NotPlain&) {
    Py_RETURN_NONE;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// the library's calls run without the interpreter's lock
template <class F>
tq_status unlocked(F f) {
  tq_status st;
  Py_BEGIN_ALLOW_THREADS;
  st = f();
  Py_END_ALLOW_THREADS;
  return st;
}

// p, x, idx, norm
PyObject* quantize_mse(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 4, [&] {
    const tq_params* p = params(a[0]);
    const Rows x = matrix(a[1]);
    PyObject* const arrays[4] = {a[2], Py_None, Py_None, a[3]};
    const Codes c = codes(p, arrays, x.rows);
    const int32_t type = vector_type(x);
    void* const s = stream();
    return unlocked([&] { return tq_quantize_mse(p, x.ptr, type, x.rows, x.rows ? x.stride : p->d, c.idx, c.norm, s); });
  });
}

// p, x, idx, qjl, gamma, norm
PyObject* quantize_prod(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 6, [&] {
    const tq_params* p = params(a[0]);
    const Rows x = matrix(a[1]);
    const Codes c = codes(p, a + 2, x.rows);
    const int32_t type = vector_type(x);
    void* const s = stream();
    return unlocked(
        [&] { return tq_quantize_prod(p, x.ptr, type, x.rows, x.rows ? x.stride : p->d, c.idx, c.qjl, c.gamma, c.norm, s); });
  });
}

// p, x, idx, qjl, gamma, norm, first_row, row_step
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 8, [&] {
    const tq_params* p = params(a[0]);
    const Rows x = matrix(a[1]);
    const int64_t first = integer(a[6]), step = integer(a[7]);
    if (first < 0 || step < 1 || first > (int64_t(1) << 40) || step > (int64_t(1) << 40) || x.rows > (1 << 20)) throw NotPlain{};
    const Codes c = codes(p, a + 2, x.rows > 0 ? first + (x.rows - 1) * step + 1 : 0);
    const int32_t type = vector_type(x);
    void* const s = stream();
    return unlocked([&] {
      return tq_append(p, x.ptr, type, x.rows, x.rows ? x.stride : p->d, c.idx, c.qjl, c.gamma, c.norm, first, step, s);
    });
  });
}

// p, idx, qjl, gamma, norm, x_out
PyObject* dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 6, [&] {
    const tq_params* p = params(a[0]);
    const Rows x = matrix(a[5]);
    if (x.type != at::kFloat) throw NotPlain{};
    const Codes c = codes(p, a + 1, x.rows);
    void* const s = stream();
    return unlocked([&] {
      return tq_dequantize(p, c.idx, c.qjl, c.gamma, c.norm, x.rows, static_cast<float*>(x.ptr), x.rows ? x.stride : p->d, s);
    });
  });
}

// p, q, n_groups, q_per_group, idx, qjl, gamma, norm, n_per_group, scores, topk, topk_idx, topk_val
PyObject* score(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 13, [&] {
    const tq_params* p = params(a[0]);
    const Rows q = matrix(a[1]);
    const int32_t groups = integer32(a[2]), per_group = integer32(a[3]), topk = integer32(a[10]);
    const int64_t keys = integer(a[8]);
    if (q.type != at::kFloat || groups < 0 || per_group < 0 || topk < 0 || keys < 0 || keys > 0x7fffffff) throw NotPlain{};
    const int64_t nq = (int64_t)groups * per_group;
    if (q.rows < nq) throw NotPlain{};
    const Codes c = codes(p, a + 4, groups * keys);
    Rows s{nullptr, 0, 0, keys, at::kFloat};
    if (a[9] != Py_None) {
      s = matrix(a[9]);
      if (s.type != at::kFloat || s.rows < nq || s.cols < keys) throw NotPlain{};
      if (s.rows == 0) s.stride = keys;
    }
    int32_t* const ti = array<int32_t>(a[11], at::kInt, nq * topk);
    float* const tv = array<float>(a[12], at::kFloat, nq * topk);
    void* const st = stream();
    return unlocked([&] {
      return tq_score(p, static_cast<const float*>(q.ptr), q.rows ? q.stride : p->d, groups, per_group, c.idx, c.qjl, c.gamma, c.norm,
                      keys, static_cast<float*>(s.ptr), s.stride, topk, ti, tv, st);
    });
  });
}

// pk, pv, q, n_groups, q_per_group, k_codes, v_codes, n_per_group, scale, out, group_stride or None
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 11, [&] {
    const tq_params *pk = params(a[0]), *pv = params(a[1]);
    const Rows q = matrix(a[2]), out = matrix(a[9]);
    const int32_t groups = integer32(a[3]), per_group = integer32(a[4]);
    const int64_t keys = integer(a[7]), stride = a[10] == Py_None ? keys : integer(a[10]);
    if (q.type != at::kFloat || out.type != at::kFloat || !PyFloat_CheckExact(a[8])) throw NotPlain{};
    const float scale = (float)PyFloat_AS_DOUBLE(a[8]);
    Codes c[2];
    for (int i = 0; i < 2; ++i) {
      if (!PyTuple_CheckExact(a[5 + i]) || PyTuple_GET_SIZE(a[5 + i]) != 4) throw NotPlain{};
      PyObject* const arrays[4] = {PyTuple_GET_ITEM(a[5 + i], 0), PyTuple_GET_ITEM(a[5 + i], 1), PyTuple_GET_ITEM(a[5 + i], 2),
                                   PyTuple_GET_ITEM(a[5 + i], 3)};
      c[i] = codes(i == 0 ? pk : pv, arrays, 0);
    }
    if (pk->workspace_bytes < tq_attend_workspace_bytes(pk, pv, groups, per_group, keys)) throw NotPlain{};  // the caller grows it
    void* const s = stream();
    return unlocked([&] {
      return tq_attend_cache(pk, pv, static_cast<const float*>(q.ptr), q.rows ? q.stride : pk->d, groups, per_group, c[0].idx, c[0].qjl,
                             c[0].gamma, c[0].norm, c[1].idx, c[1].qjl, c[1].gamma, c[1].norm, keys, stride, scale,
                             static_cast<float*>(out.ptr), out.rows ? out.stride : pv->d, s);
    });
  });
}

// --- the paged cache: its struct (p.c, or p._scratch.call where scratch memory is used) and p.k, whose GPU every tensor is on and which is
// the current one -----------------------------------------------------------------------------------------------------------------

// a cache with the scratch memory of the calling thread on one stream
struct Call {
  tq_pages c;
  uint64_t stream;
};
struct Cache {
  const tq_pages* c;  // the caller holds the struct for the length of the call, and nobody changes it
  c10::Device device;
};
template <class T = tq_pages>
Cache cache(PyObject* const* o) {
  Py_buffer b;
  if (PyObject_GetBuffer(o[0], &b, PyBUF_SIMPLE) != 0) {
    PyErr_Clear();
    throw NotPlain{};
  }
  const bool whole = (size_t)b.len == sizeof(T);
  const tq_pages* c = static_cast<const tq_pages*>(b.buf);
  PyBuffer_Release(&b);
  const at::Tensor* k = tensor(o[1]);
  if (!whole || k == nullptr || k->device().index() != c10::hip::current_device()) throw NotPlain{};
  return Cache{c, k->device()};
}

const at::Tensor& there(const Cache& p, PyObject* o, c10::ScalarType type, int64_t dims) {
  const at::Tensor* t = tensor(o);
  if (t == nullptr || t->scalar_type() != type || t->dim() != dims || t->device() != p.device) throw NotPlain{};
  return *t;
}

int32_t* ints(const Cache& p, PyObject* o, int64_t n) {
  const at::Tensor& t = there(p, o, at::kInt, 1);
  if (t.size(0) != n || !t.is_contiguous()) throw NotPlain{};
  return static_cast<int32_t*>(t.data_ptr());
}

// table, lens, starts (or None): a batch of n_rows rows (-1: a call without rows)
tq_batch batch(const Cache& p, int64_t n_rows, PyObject* table, PyObject* lens, PyObject* starts, int32_t max_new) {
  const at::Tensor& t = there(p, table, at::kInt, 2);
  const int64_t n = t.size(0), width = t.size(1);
  if (n > INT32_MAX || width > INT32_MAX || max_new < 0 || (width > 1 && t.stride(1) != 1) || (n > 1 && t.stride(0) < width)) throw NotPlain{};
  if (starts == Py_None && n_rows >= 0 && n_rows < n * max_new) throw NotPlain{};
  tq_batch b;
  b.n_seqs = (int32_t)n, b.max_new = max_new, b.n_rows = n_rows < 0 ? 0 : n_rows, b.width = (int32_t)width;
  b.table_stride = n > 1 ? t.stride(0) : width;
  b.table = static_cast<int32_t*>(t.data_ptr());
  b.lens = lens == Py_None ? nullptr : ints(p, lens, n);
  b.starts = starts == Py_None ? nullptr : ints(p, starts, n + 1);
  return b;
}

struct Vectors {
  void* ptr;
  int64_t rows, heads, ld_row, ld_head;
  int32_t dtype;
};
Vectors vectors(const Cache& p, PyObject* o) {
  const at::Tensor* t = tensor(o);
  if (t == nullptr || t->dim() != 3 || t->size(2) != p.c->d || t->stride(2) != 1 || t->device() != p.device) throw NotPlain{};
  Vectors v;
  v.ptr = t->data_ptr(), v.rows = t->size(0), v.heads = t->size(1);
  v.ld_row = v.rows > 1 ? t->stride(0) : 0, v.ld_head = v.heads > 1 ? t->stride(1) : 0;
  if (v.heads > INT32_MAX) throw NotPlain{};
  if (t->scalar_type() == at::kFloat) v.dtype = TQ_F32;
  else if (t->scalar_type() == at::kBFloat16) v.dtype = TQ_BF16;
  else throw NotPlain{};
  return v;
}

void* stream_of(const Cache& p) { return static_cast<void*>(c10::hip::getCurrentHIPStream(p.device.index()).stream()); }

// the scratch memory is this stream's and large enough, and the call not captured (such a one has its own)
void scratch(const Cache& p, size_t need, void* stream) {
  if (need == 0) return;
  const Call* const call = reinterpret_cast<const Call*>(p.c);
  if (call->stream != (uint64_t)(uintptr_t)stream || p.c->workspace_bytes < need) throw NotPlain{};
  hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
  if (stream != nullptr && (hipStreamIsCapturing(static_cast<hipStream_t>(stream), &status) != hipSuccess || status != hipStreamCaptureStatusNone))
    throw NotPlain{};
}

// p.c, p.k, k, v, table, lens, starts, max_new
PyObject* pages_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 8, [&] {
    const Cache p = cache(a);
    const Vectors k = vectors(p, a[2]), v = vectors(p, a[3]);
    if (k.rows != v.rows || k.heads != v.heads || k.heads != p.c->n_heads || k.dtype != v.dtype || k.ld_row != v.ld_row || k.ld_head != v.ld_head)
      throw NotPlain{};
    const tq_batch b = batch(p, k.rows, a[4], a[5], a[6], integer32(a[7]));
    void* const s = stream_of(p);
    return unlocked([&] { return tq_pages_append(p.c, &b, k.ptr, v.ptr, k.dtype, k.ld_row, k.ld_head, s); });
  });
}

// [rows][heads of the cache][n] places of pages, or None
int32_t* places(const Cache& p, PyObject* o, int64_t rows, int32_t* n) {
  *n = 0;
  if (o == Py_None) return nullptr;
  const at::Tensor& t = there(p, o, at::kInt, 3);
  if (t.size(0) != rows || t.size(1) != p.c->n_heads || t.size(2) < 1 || t.size(2) > INT32_MAX || !t.is_contiguous()) throw NotPlain{};
  *n = (int32_t)t.size(2);
  return static_cast<int32_t*>(t.data_ptr());
}

// p._scratch.call, p.k, q, table, lens, starts, max_new, scale, out, lse, window, chosen
PyObject* pages_attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 12, [&] {
    const Cache p = cache<Call>(a);
    const Vectors q = vectors(p, a[2]), out = vectors(p, a[8]);
    if (q.rows != out.rows || q.heads != out.heads || q.dtype != out.dtype || q.heads < 1 || q.heads % p.c->n_heads != 0 || q.rows < 1 ||
        (out.rows > 1 && out.ld_row == 0) || (out.heads > 1 && out.ld_head == 0) || !PyFloat_CheckExact(a[7]))
      throw NotPlain{};
    const float scale = (float)PyFloat_AS_DOUBLE(a[7]);
    float* lse = nullptr;
    if (a[9] != Py_None) {
      const at::Tensor& t = there(p, a[9], at::kFloat, 2);
      if (t.size(0) != q.rows || t.size(1) != q.heads || !t.is_contiguous()) throw NotPlain{};
      lse = static_cast<float*>(t.data_ptr());
    }
    const int32_t window = integer32(a[10]);
    int32_t n_chosen;
    const int32_t* const chosen = places(p, a[11], q.rows, &n_chosen);
    const tq_batch b = batch(p, q.rows, a[3], a[4], a[5], integer32(a[6]));
    void* const s = stream_of(p);
    scratch(p, tq_pages_attend_workspace_bytes(p.c, &b, (int32_t)q.heads, n_chosen, window), s);
    return unlocked([&] {
      return tq_pages_attend(p.c, &b, q.ptr, q.dtype, q.ld_row, q.ld_head, (int32_t)q.heads, scale, window, chosen, n_chosen, out.ptr, out.ld_row,
                             out.ld_head, lse, s);
    });
  });
}

// p._scratch.call, p.k, q, table, lens, starts, max_new, chosen, keep_first, keep_last
PyObject* pages_select(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 10, [&] {
    const Cache p = cache<Call>(a);
    const Vectors q = vectors(p, a[2]);
    if (q.heads < 1 || q.heads % p.c->n_heads != 0 || q.rows < 1 || a[7] == Py_None || p.c->bounds == nullptr) throw NotPlain{};
    int32_t n_chosen;
    int32_t* const chosen = places(p, a[7], q.rows, &n_chosen);
    const tq_batch b = batch(p, q.rows, a[3], a[4], a[5], integer32(a[6]));
    const int32_t first = integer32(a[8]), last = integer32(a[9]);
    void* const s = stream_of(p);
    scratch(p, tq_pages_select_workspace_bytes(p.c, &b), s);
    return unlocked([&] {
      return tq_pages_select(p.c, &b, q.ptr, q.dtype, q.ld_row, q.ld_head, (int32_t)q.heads, first, last, chosen, n_chosen, s);
    });
  });
}

void pool(const Cache& p, int64_t n, void* stream) {
  if (p.c->refs == nullptr) throw NotPlain{};
  scratch(p, tq_pages_pool_workspace_bytes(p.c, n), stream);
}
int32_t* one(const Cache& p, PyObject* o) { return o == Py_None ? nullptr : ints(p, o, 1); }

// p._scratch.call, p.k, table, lens, starts, max_new, missing
PyObject* pages_reserve(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 7, [&] {
    const Cache p = cache<Call>(a);
    void* const s = stream_of(p);
    pool(p, 0, s);
    const tq_batch b = batch(p, -1, a[2], a[3], a[4], integer32(a[5]));
    int32_t* const missing = one(p, a[6]);
    return unlocked([&] { return tq_pages_reserve(p.c, &b, missing, s); });
  });
}

// p._scratch.call, p.k, table, lens, parents, children, missing
PyObject* pages_fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 7, [&] {
    const Cache p = cache<Call>(a);
    void* const s = stream_of(p);
    const int64_t forks = there(p, a[4], at::kInt, 1).size(0);
    if (forks > INT32_MAX) throw NotPlain{};
    pool(p, forks, s);
    const int32_t *const parents = ints(p, a[4], forks), *const children = ints(p, a[5], forks);
    const tq_batch b = batch(p, -1, a[2], a[3], Py_None, 0);
    int32_t* const missing = one(p, a[6]);
    return unlocked([&] { return tq_pages_fork(p.c, &b, parents, children, (int32_t)forks, missing, s); });
  });
}

// p.c, p.k, table, lens, rows
PyObject* pages_free(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 5, [&] {
    const Cache p = cache(a);
    const int64_t many = there(p, a[4], at::kInt, 1).size(0);
    if (many > INT32_MAX || p.c->refs == nullptr) throw NotPlain{};
    const int32_t* const rows = ints(p, a[4], many);
    const tq_batch b = batch(p, -1, a[2], a[3], Py_None, 0);
    void* const s = stream_of(p);
    return unlocked([&] { return tq_pages_free(p.c, &b, rows, (int32_t)many, s); });
  });
}

// p._scratch.call, p.k, table, n_live
PyObject* pages_compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 4, [&] {
    const Cache p = cache<Call>(a);
    void* const s = stream_of(p);
    pool(p, 0, s);
    const tq_batch b = batch(p, -1, a[2], Py_None, Py_None, 0);
    int32_t* const live = one(p, a[3]);
    return unlocked([&] { return tq_pages_compact(p.c, &b, live, s); });
  });
}

// p.c, p.k, src, dst
PyObject* pages_copy(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 4, [&] {
    const Cache p = cache(a);
    const int64_t pairs = there(p, a[2], at::kInt, 1).size(0);
    const int32_t *const src = ints(p, a[2], pairs), *const dst = ints(p, a[3], pairs);
    void* const s = stream_of(p);
    return unlocked([&] { return tq_pages_copy(p.c, src, dst, pairs, s); });
  });
}

#define TQ_METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {TQ_METHOD(quantize_mse), TQ_METHOD(quantize_prod), TQ_METHOD(append), TQ_METHOD(dequantize),
                         TQ_METHOD(score), TQ_METHOD(attend), TQ_METHOD(pages_append), TQ_METHOD(pages_attend),
                         TQ_METHOD(pages_select), TQ_METHOD(pages_reserve), TQ_METHOD(pages_fork), TQ_METHOD(pages_free),
                         TQ_METHOD(pages_compact), TQ_METHOD(pages_copy), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tqcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tqcall(void) { return PyModule_Create(&module); }

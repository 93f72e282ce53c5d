// Python side of the entry points that a decode step calls around its linears: argument marshalling only, as the ctypes binding of the other calls, but
// compiled, because a decode step makes many of these calls on small tensors (a call through ctypes took 12 us on the host,
// of which the launch itself is 4).  Takes torch tensors, checks what the C ABI cannot see (types, shapes, strides,
// devices), and calls the library's functions at the addresses given to bind().
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "bitnet_b200.h"

namespace {

PyObject* g_error = nullptr;       // BitnetError
PyObject* g_status_error = nullptr;   // called with (status, name); raises
struct {
  decltype(&bitnet_kv_append) append;
  decltype(&bitnet_kv_reserve) reserve;
  decltype(&bitnet_kv_fork) fork;
  decltype(&bitnet_kv_free) free_;
  decltype(&bitnet_kv_trim) trim;
  decltype(&bitnet_kv_compact) compact;
  decltype(&bitnet_kv_copy_pages) copy_pages;
  decltype(&bitnet_attn_decode) decode;
  decltype(&bitnet_attn_prompt) prompt;
  decltype(&bitnet_attn_shared) shared;
  decltype(&bitnet_kv_append_rope) append_rope;
  decltype(&bitnet_add_rmsnorm_quant) norm;
  decltype(&bitnet_sample) sample;
} g_fn;

struct Refused {};                 // a Python exception is set

[[noreturn]] void refuse(const char* name, const char* what) {
  PyErr_Format(g_error, "%s: %s", name, what);
  throw Refused{};
}

thread_local int g_device;         // the current one, for this call

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(name, "expected a tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.is_cuda() && t.get_device() != g_device) refuse(name, "on another device than the current one");
  return t;
}
int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused{};
  return v;
}
double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused{};
  return v;
}
const bitnet_kv_cache_t* cache(PyObject* o) { return static_cast<const bitnet_kv_cache_t*>(PyLong_AsVoidPtr(o)); }

// An int32 array of the books: contiguous, on the GPU, `dim` dimensions, at least `rows` rows.
int32_t* book(PyObject* o, const char* name, int64_t dim, int64_t rows = 0) {
  const at::Tensor& t = tensor(o, name);
  if (!t.is_cuda() || t.scalar_type() != at::kInt || t.dim() != dim || !t.is_contiguous())
    refuse(name, dim == 1 ? "expected a contiguous 1-D CUDA tensor of int32" : "expected a contiguous 2-D CUDA tensor of int32");
  if (t.size(0) < rows) refuse(name, "too few entries");
  return t.data_ptr<int32_t>();
}
int32_t* book_or_none(PyObject* o, const char* name) { return o == Py_None ? nullptr : book(o, name, 1); }

int type_code(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kBFloat16: return BITNET_KV_BF16;
    case at::kHalf: return BITNET_KV_F16;
    case at::kFloat: return BITNET_KV_F32;
    default: return -1;
  }
}
// [tokens][heads][head_dim] rows.
const at::Tensor& rows(PyObject* o, const char* name, int64_t heads, int64_t dim) {
  const at::Tensor& t = tensor(o, name);
  if (!t.is_cuda() || t.dim() != 3 || type_code(t) < 0) refuse(name, "expected a CUDA tensor [tokens][heads][head_dim] of fp32, bf16 or fp16");
  if (t.size(2) != dim || (heads && t.size(1) != heads)) refuse(name, "heads or head_dim are not the cache's");
  if (t.stride(2) != 1 && dim > 1) refuse(name, "head_dim must be contiguous");
  return t;
}
// The stride of a dimension of one entry says nothing (torch may leave anything there).
int64_t step(const at::Tensor& t, int dim) { return t.size(dim) > 1 ? t.stride(dim) : 0; }
void* stream(PyObject* o, const at::Tensor& t) {
  if (o != Py_None) return PyLong_AsVoidPtr(o);
  return c10::cuda::getCurrentCUDAStream(t.get_device()).stream();
}
struct Space {
  void* p;
  size_t n;
};
Space space(PyObject* o) {
  if (o == Py_None) return {nullptr, 0};
  const at::Tensor& t = tensor(o, "workspace");
  if (!t.is_cuda() || !t.is_contiguous()) refuse("workspace", "expected a contiguous CUDA tensor");
  return {t.data_ptr(), t.nbytes()};
}
PyObject* done(int rc, const char* name) {
  if (rc) {
    PyObject* r = PyObject_CallFunction(g_status_error, "is", rc, name);
    Py_XDECREF(r);
    if (!PyErr_Occurred()) PyErr_SetString(g_error, name);
    return nullptr;
  }
  Py_RETURN_NONE;
}

// [rows][columns], columns contiguous, of fp32, bf16 or fp16.
const at::Tensor& matrix(PyObject* o, const char* name, int64_t rows = -1, int64_t columns = -1) {
  const at::Tensor& t = tensor(o, name);
  if (!t.is_cuda() || t.dim() != 2 || type_code(t) < 0 || (t.stride(1) != 1 && t.size(1) > 1))
    refuse(name, "expected a CUDA matrix of fp32, bf16 or fp16 with contiguous rows");
  if ((rows >= 0 && t.size(0) != rows) || (columns >= 0 && t.size(1) != columns)) refuse(name, "not of the expected shape");
  return t;
}
// The caller's contiguous tensor of that type and shape, or a new one.
at::Tensor made(PyObject* o, const char* name, at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like) {
  if (o == Py_None) return at::empty(shape, like.options().dtype(type));
  const at::Tensor& t = tensor(o, name);
  if (!t.is_cuda() || t.sizes() != shape || t.scalar_type() != type || !t.is_contiguous()) refuse(name, "expected a contiguous CUDA tensor of its shape and type");
  return t;
}
// A contiguous vector of n values of that type; null where it is None.
const void* vector(PyObject* o, const char* name, int64_t n, at::ScalarType type) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, name);
  if (!t.is_cuda() || t.dim() != 1 || t.size(0) != n || t.scalar_type() != type || !t.is_contiguous()) refuse(name, "expected a contiguous CUDA vector of its length and type");
  return t.data_ptr();
}

// Every entry: a fixed number of positional arguments (the Python functions supply the defaults).
template <int N, PyObject* (*F)(PyObject* const*)>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != N) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    c10::DeviceIndex current = -1;
    g_device = c10::cuda::GetDevice(&current) == cudaSuccess ? current : -1;
    return F(a);
  } catch (const Refused&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// cache, layer, k, v, table, kv_len, q_start, dev_status, stream
PyObject* append(PyObject* const* a) {
  const bitnet_kv_cache_t* c = cache(a[0]);
  const at::Tensor &k = rows(a[2], "k", c->kv_heads, c->head_dim), &v = rows(a[3], "v", c->kv_heads, c->head_dim);
  if (k.scalar_type() != v.scalar_type() || k.size(0) != v.size(0) || k.size(1) != v.size(1) || step(k, 0) != step(v, 0) || step(k, 1) != step(v, 1))
    refuse("bitnet_kv_append", "k and v must have one type, shape and strides");
  const int32_t* q_start = book_or_none(a[6], "q_start");
  const int64_t seqs = q_start ? tensor(a[6], "q_start").size(0) - 1 : tensor(a[4], "table").size(0);
  const int32_t* table = book(a[4], "table", 2, seqs);
  return done(g_fn.append(c, integer(a[1]), k.data_ptr(), v.data_ptr(), type_code(k), step(k, 0), step(k, 1), k.size(0), table,
                          tensor(a[4], "table").size(1), book(a[5], "kv_len", 1, seqs), q_start, seqs, book_or_none(a[7], "dev_status"),
                          stream(a[8], k)),
              "bitnet_kv_append");
}

// refs, table, from_len, to_len, page_size, dev_status, stream
PyObject* reserve(PyObject* const* a) {
  int32_t* refs = book(a[0], "refs", 1);
  int32_t* table = book(a[1], "table", 2);
  const at::Tensor& t = tensor(a[1], "table");
  const int64_t seqs = t.size(0);
  return done(g_fn.reserve(refs, tensor(a[0], "refs").size(0), table, seqs, t.size(1), book(a[2], "from_len", 1, seqs),
                           book(a[3], "to_len", 1, seqs), integer(a[4]), book_or_none(a[5], "dev_status"), stream(a[6], t)),
              "bitnet_kv_reserve");
}

// cache, refs, table, kv_len, parents, children, workspace, dev_status, stream
PyObject* fork(PyObject* const* a) {
  const bitnet_kv_cache_t* c = cache(a[0]);
  int32_t* refs = book(a[1], "refs", 1);
  int32_t* table = book(a[2], "table", 2);
  const at::Tensor& t = tensor(a[2], "table");
  const int32_t *parents = book(a[4], "parents", 1), *children = book(a[5], "children", 1);
  const int64_t n = tensor(a[4], "parents").size(0);
  if (tensor(a[1], "refs").size(0) != c->num_pages || tensor(a[5], "children").size(0) != n)
    refuse("bitnet_kv_fork", "refs must have one entry per page, parents and children one length");
  const Space ws = space(a[6]);
  return done(g_fn.fork(c, refs, table, t.size(0), t.size(1), book(a[3], "kv_len", 1, t.size(0)), parents, children, n, ws.p, ws.n,
                        book_or_none(a[7], "dev_status"), stream(a[8], t)),
              "bitnet_kv_fork");
}

// refs, table, kv_len, rows, dev_status, stream
PyObject* free_rows(PyObject* const* a) {
  int32_t* refs = book(a[0], "refs", 1);
  int32_t* table = book(a[1], "table", 2);
  const at::Tensor& t = tensor(a[1], "table");
  const int32_t* list = book(a[3], "rows", 1);
  return done(g_fn.free_(refs, tensor(a[0], "refs").size(0), table, t.size(0), t.size(1), book(a[2], "kv_len", 1, t.size(0)), list,
                         tensor(a[3], "rows").size(0), book_or_none(a[4], "dev_status"), stream(a[5], t)),
              "bitnet_kv_free");
}

// refs, table, kv_len, page_size, window, sinks, stream
PyObject* trim(PyObject* const* a) {
  int32_t* refs = book(a[0], "refs", 1);
  int32_t* table = book(a[1], "table", 2);
  const at::Tensor& t = tensor(a[1], "table");
  return done(g_fn.trim(refs, tensor(a[0], "refs").size(0), table, t.size(0), t.size(1), book(a[2], "kv_len", 1, t.size(0)), integer(a[3]),
                        integer(a[4]), integer(a[5]), stream(a[6], t)),
              "bitnet_kv_trim");
}

// cache, refs, table, live, workspace, stream
PyObject* compact(PyObject* const* a) {
  const bitnet_kv_cache_t* c = cache(a[0]);
  int32_t* refs = book(a[1], "refs", 1);
  if (tensor(a[1], "refs").size(0) != c->num_pages) refuse("bitnet_kv_compact", "refs must have one entry per page");
  int32_t* table = book(a[2], "table", 2);
  const at::Tensor& t = tensor(a[2], "table");
  const Space ws = space(a[4]);
  return done(g_fn.compact(c, refs, table, t.size(0), t.size(1), book_or_none(a[3], "live"), ws.p, ws.n, stream(a[5], t)),
              "bitnet_kv_compact");
}

// cache, src, dst, dev_status, stream
PyObject* copy_pages(PyObject* const* a) {
  const int32_t *src = book(a[1], "src", 1), *dst = book(a[2], "dst", 1);
  const at::Tensor& t = tensor(a[1], "src");
  if (t.size(0) != tensor(a[2], "dst").size(0)) refuse("bitnet_kv_copy_pages", "src and dst must have one length");
  return done(g_fn.copy_pages(cache(a[0]), src, dst, t.size(0), book_or_none(a[3], "dev_status"), stream(a[4], t)), "bitnet_kv_copy_pages");
}

// out: the caller's, or a new contiguous tensor of q's shape and type.
at::Tensor output(PyObject* o, const at::Tensor& q, const char* name) {
  if (o == Py_None) return at::empty(q.sizes(), q.options());
  const at::Tensor& t = tensor(o, "out");
  if (!t.is_cuda() || t.sizes() != q.sizes() || t.scalar_type() != q.scalar_type() || !t.is_contiguous())
    refuse(name, "out must be contiguous, with q's shape and type");
  return t;
}

// cache, layer, q, table, kv_len, scale, window, sinks, out, workspace, dev_status, stream
PyObject* decode(PyObject* const* a) {
  const bitnet_kv_cache_t* c = cache(a[0]);
  const at::Tensor& q = rows(a[2], "q", 0, c->head_dim);
  const int64_t n = q.size(0);
  const int32_t *table = book(a[3], "table", 2, n), *len = book(a[4], "kv_len", 1, n);
  const at::Tensor out = output(a[8], q, "bitnet_attn_decode");
  const Space ws = space(a[9]);
  const int rc = g_fn.decode(c, integer(a[1]), q.data_ptr(), type_code(q), q.size(1), step(q, 0), step(q, 1), table,
                             tensor(a[3], "table").size(1), len, n, (float)real(a[5]), integer(a[6]), integer(a[7]), out.data_ptr(), ws.p,
                             ws.n, book_or_none(a[10], "dev_status"), stream(a[11], q));
  return rc ? done(rc, "bitnet_attn_decode") : THPVariable_Wrap(out);
}

// cache, layer, q, table, kv_len, q_start, max_new, scale, window, sinks, out, workspace, dev_status, stream
PyObject* prompt(PyObject* const* a) {
  const bitnet_kv_cache_t* c = cache(a[0]);
  const at::Tensor& q = rows(a[2], "q", 0, c->head_dim);
  const int32_t* q_start = book(a[5], "q_start", 1);
  const int64_t seqs = tensor(a[5], "q_start").size(0) - 1;
  const int32_t *table = book(a[3], "table", 2, seqs), *len = book(a[4], "kv_len", 1, seqs);
  const at::Tensor out = output(a[10], q, "bitnet_attn_prompt");
  const Space ws = space(a[11]);
  const int rc = g_fn.prompt(c, integer(a[1]), q.data_ptr(), type_code(q), q.size(1), step(q, 0), step(q, 1), q.size(0), table,
                             tensor(a[3], "table").size(1), len, q_start, seqs, integer(a[6]), (float)real(a[7]), integer(a[8]),
                             integer(a[9]), out.data_ptr(), ws.p, ws.n, book_or_none(a[12], "dev_status"), stream(a[13], q));
  return rc ? done(rc, "bitnet_attn_prompt") : THPVariable_Wrap(out);
}

// cache, layer, q, table, kv_len, group_start, prefix_len, scale, window, sinks, out, workspace, dev_status, stream
PyObject* shared(PyObject* const* a) {
  const bitnet_kv_cache_t* c = cache(a[0]);
  const at::Tensor& q = rows(a[2], "q", 0, c->head_dim);
  const int64_t n = q.size(0);
  const int32_t *table = book(a[3], "table", 2, n), *len = book(a[4], "kv_len", 1, n);
  const int32_t* start = book(a[5], "group_start", 1);
  const int64_t groups = tensor(a[5], "group_start").size(0) - 1;
  const int32_t* prefix = book(a[6], "prefix_len", 1, groups);
  const at::Tensor out = output(a[10], q, "bitnet_attn_shared");
  const Space ws = space(a[11]);
  const int rc = g_fn.shared(c, integer(a[1]), q.data_ptr(), type_code(q), q.size(1), step(q, 0), step(q, 1), table, tensor(a[3], "table").size(1),
                             len, n, start, prefix, groups, (float)real(a[7]), integer(a[8]), integer(a[9]), out.data_ptr(), ws.p, ws.n,
                             book_or_none(a[12], "dev_status"), stream(a[13], q));
  return rc ? done(rc, "bitnet_attn_shared") : THPVariable_Wrap(out);
}

// cache, layer, rope, q, k, v, table, kv_len, q_start, q_out, q_type (a code; used without q_out), dev_status, stream
PyObject* append_rope(PyObject* const* a) {
  const bitnet_kv_cache_t* c = cache(a[0]);
  const at::Tensor &k = rows(a[4], "k", c->kv_heads, c->head_dim), &v = rows(a[5], "v", c->kv_heads, c->head_dim);
  if (k.scalar_type() != v.scalar_type() || k.size(0) != v.size(0) || step(k, 0) != step(v, 0) || step(k, 1) != step(v, 1))
    refuse("bitnet_kv_append_rope", "k and v must have one type, shape and strides");
  const bool with_q = a[3] != Py_None;
  const at::Tensor& q = with_q ? rows(a[3], "q", 0, c->head_dim) : k;
  if (with_q && (q.scalar_type() != k.scalar_type() || q.size(0) != k.size(0))) refuse("q", "must have k's type and number of tokens");
  const int32_t* q_start = book_or_none(a[8], "q_start");
  const int64_t seqs = q_start ? tensor(a[8], "q_start").size(0) - 1 : tensor(a[6], "table").size(0);
  const int32_t* table = book(a[6], "table", 2, seqs);
  at::Tensor out;
  if (with_q) {
    const int64_t code = integer(a[10]);
    const at::ScalarType type = a[9] != Py_None ? tensor(a[9], "q_out").scalar_type()
                                : code < 0      ? q.scalar_type()
                                : code == BITNET_KV_F32 ? at::kFloat : code == BITNET_KV_F16 ? at::kHalf : at::kBFloat16;
    out = made(a[9], "q_out", q.sizes(), type, q);
  }
  const int rc = g_fn.append_rope(c, integer(a[1]), static_cast<const bitnet_rope_t*>(PyLong_AsVoidPtr(a[2])), with_q ? q.data_ptr() : nullptr,
                                  with_q ? q.size(1) : 0, step(q, 0), step(q, 1), k.data_ptr(), v.data_ptr(), type_code(k), step(k, 0), step(k, 1),
                                  k.size(0), table, tensor(a[6], "table").size(1), book(a[7], "kv_len", 1, seqs), q_start, seqs,
                                  with_q ? out.data_ptr() : nullptr, with_q ? type_code(out) : 0, book_or_none(a[11], "dev_status"), stream(a[12], k));
  if (rc) return done(rc, "bitnet_kv_append_rope");
  if (!with_q) Py_RETURN_NONE;
  return THPVariable_Wrap(out);
}

// x, weight, eps, residual, residual_out, y, q, act_scale, act_sum, stream -> (q, act_scale)
PyObject* norm(PyObject* const* a) {
  const at::Tensor& x = matrix(a[0], "x");
  const int64_t T = x.size(0), K = x.size(1);
  const at::Tensor *res = nullptr, *res_out = nullptr, *w = nullptr, *y = nullptr;
  if (a[1] != Py_None) {
    w = &tensor(a[1], "weight");
    if (!w->is_cuda() || w->dim() != 1 || w->size(0) != K || type_code(*w) < 0 || !w->is_contiguous()) refuse("weight", "expected a contiguous CUDA vector of x's width");
  }
  if (a[3] != Py_None) {
    res = &matrix(a[3], "residual", T, K);
    res_out = &matrix(a[4], "residual_out", T, K);
    if (res->scalar_type() != res_out->scalar_type()) refuse("residual_out", "must have residual's type");
  } else if (a[4] != Py_None) {
    refuse("residual_out", "without a residual");
  }
  if (a[5] != Py_None) {
    y = &matrix(a[5], "y", T, K);
    if (!y->is_contiguous()) refuse("y", "must be contiguous");
  }
  const at::Tensor q = made(a[6], "q", {T, K}, at::kChar, x), scale = made(a[7], "act_scale", {T}, at::kFloat, x);
  const void* sum = vector(a[8], "act_sum", T, at::kInt);
  const int rc = g_fn.norm(x.data_ptr(), type_code(x), step(x, 0), res ? res->data_ptr() : nullptr, res ? type_code(*res) : 0, res ? step(*res, 0) : 0,
                           res ? res_out->data_ptr() : nullptr, res ? step(*res_out, 0) : 0, w ? w->data_ptr() : nullptr, w ? type_code(*w) : 0,
                           (float)real(a[2]), T, K, y ? y->data_ptr() : nullptr, y ? type_code(*y) : 0, q.data_ptr<int8_t>(),
                           scale.data_ptr<float>(), static_cast<int32_t*>(const_cast<void*>(sum)), stream(a[9], x));
  if (rc) return done(rc, "bitnet_add_rmsnorm_quant");
  return Py_BuildValue("(NN)", THPVariable_Wrap(q), THPVariable_Wrap(scale));
}

// logits, u, temperature, top_k, top_p, min_p, tokens, prob, stream -> (tokens, prob)
PyObject* sample(PyObject* const* a) {
  const at::Tensor& x = matrix(a[0], "logits");
  const int64_t n = x.size(0);
  if (a[1] == Py_None) refuse("u", "expected a random number per row");
  const at::Tensor tokens = made(a[6], "tokens", {n}, at::kInt, x), prob = made(a[7], "prob", {n}, at::kFloat, x);
  auto f = [&](int i, const char* name) { return static_cast<const float*>(vector(a[i], name, n, at::kFloat)); };
  const int rc = g_fn.sample(x.data_ptr(), type_code(x), step(x, 0), n, x.size(1), f(1, "u"), f(2, "temperature"),
                             static_cast<const int32_t*>(vector(a[3], "top_k", n, at::kInt)), f(4, "top_p"), f(5, "min_p"),
                             tokens.data_ptr<int32_t>(), prob.data_ptr<float>(), stream(a[8], x));
  if (rc) return done(rc, "bitnet_sample");
  return Py_BuildValue("(NN)", THPVariable_Wrap(tokens), THPVariable_Wrap(prob));
}

// BitnetError, the function that raises for a status, and the addresses of the library's functions in the order of g_fn.
PyObject* bind(PyObject*, PyObject* args) {
  PyObject *error, *status, *addresses;
  if (!PyArg_ParseTuple(args, "OOO!", &error, &status, &PyTuple_Type, &addresses)) return nullptr;
  constexpr Py_ssize_t N = sizeof(g_fn) / sizeof(void*);
  if (PyTuple_GET_SIZE(addresses) != N) {
    PyErr_SetString(PyExc_TypeError, "bind: one address per entry point");
    return nullptr;
  }
  void* fn[N];
  for (Py_ssize_t i = 0; i < N; ++i) {
    fn[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(addresses, i));
    if (!fn[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "bind: null address");
      return nullptr;
    }
  }
  memcpy(&g_fn, fn, sizeof g_fn);
  Py_INCREF(error);
  Py_INCREF(status);
  Py_XSETREF(g_error, error);
  Py_XSETREF(g_status_error, status);
  Py_RETURN_NONE;
}

#define ENTRY(name, n, f) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&entry<n, f>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, nullptr},
                         ENTRY("kv_append", 9, append),
                         ENTRY("kv_reserve", 7, reserve),
                         ENTRY("kv_fork", 9, fork),
                         ENTRY("kv_free", 6, free_rows),
                         ENTRY("kv_trim", 7, trim),
                         ENTRY("kv_compact", 6, compact),
                         ENTRY("kv_copy_pages", 5, copy_pages),
                         ENTRY("attn_decode", 12, decode),
                         ENTRY("attn_prompt", 14, prompt),
                         ENTRY("attn_shared", 14, shared),
                         ENTRY("kv_append_rope", 13, append_rope),
                         ENTRY("add_rmsnorm_quant", 10, norm),
                         ENTRY("sample", 9, sample),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&module); }

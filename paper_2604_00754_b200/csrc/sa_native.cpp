// Python entry of the calls a model makes per layer: takes torch tensors, allocates what the call
// returns and enqueues the C ABI call on the current stream.  A pass over a small problem is bound
// by host work, and through ctypes that work (struct and pointer objects, one Python call per
// allocation, the stream look-up) was several times the launches themselves: make_perm 36 us and
// the forward 18 us of host time, of which 12 and 3 us were launches.  The functions take their
// arguments by position; defaults and names live in the Python wrappers.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/EmptyTensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "sa.h"

namespace {

PyObject* g_error_class = nullptr;   // binding.SaError

struct Raised {};                    // a Python exception is set

[[noreturn]] void raise(PyObject* type, const char* text) {
  PyErr_SetString(type, text);
  throw Raised{};
}

void check(int status, const char* where) {
  if (status == SA_OK) return;
  PyObject* e = PyObject_CallFunction(g_error_class, "is", status, where);
  if (e) {
    PyErr_SetObject(g_error_class, e);
    Py_DECREF(e);
  }
  throw Raised{};
}

// The C call, with its arguments in hand, without the interpreter's lock: a launch waits for room
// where the device's queue is full, and other threads go on meanwhile.
template <typename... P, typename... A>
int unlocked(sa_status (*call)(P...), A... args) {
  PyThreadState* state = PyEval_SaveThread();
  const int status = call(static_cast<P>(args)...);
  PyEval_RestoreThread(state);
  return status;
}

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) raise(PyExc_TypeError, "expected a tensor");
  return THPVariable_Unpack(o);
}
const at::Tensor* tensor_or_null(PyObject* o) { return o == Py_None ? nullptr : &tensor(o); }
void* ptr(const at::Tensor& t) { return t.data_ptr(); }
void* ptr(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }

unsigned long long integer_mask(PyObject* o) {        // as int(o), modulo 2^64
  PyObject* i = PyLong_CheckExact(o) ? o : PyNumber_Long(o);
  if (!i) throw Raised{};
  const unsigned long long v = PyLong_AsUnsignedLongLongMask(i);
  if (i != o) Py_DECREF(i);
  return v;
}
long long integer(PyObject* o) { return (long long)integer_mask(o); }
int64_t size(PyObject* o) {                           // a tensor's extent: whole numbers only
  const Py_ssize_t v = PyNumber_AsSsize_t(o, PyExc_OverflowError);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  return v;
}
double real(PyObject* o) {                            // as float(o)
  PyObject* f = PyFloat_CheckExact(o) ? o : PyNumber_Float(o);
  if (!f) throw Raised{};
  const double v = PyFloat_AS_DOUBLE(f);
  if (f != o) Py_DECREF(f);
  return v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Raised{};
  return v != 0;
}

sa_stream_t stream() { return (sa_stream_t)c10::cuda::getCurrentCUDAStream().stream(); }

at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType type, c10::Device dev) {
  if (!dev.is_cuda()) return at::empty(sizes, at::TensorOptions().dtype(type).device(dev));
  return at::detail::empty_cuda(sizes, type, dev, std::nullopt);
}
void same_layout(const at::Tensor& ref, const at::Tensor* t) {
  if (t && (t->sizes() != ref.sizes() || t->strides() != ref.strides() ||
            t->scalar_type() != ref.scalar_type()))
    raise(PyExc_ValueError, "tensor does not share the layout of its reference tensor");
}

// A tensor with the shape, strides and type of `t`.  A slice of a larger tensor or an expanded one
// has strides that a fresh tensor cannot have: the kernels, which are told one set of strides for
// both, would write outside it.
at::Tensor fresh_like(const at::Tensor& t) {
  if (t.is_cuda() && t.is_non_overlapping_and_dense())
    return at::detail::empty_strided_cuda(t.sizes(), t.strides(), t.scalar_type(), t.device());
  const at::Tensor r = at::empty_like(t);
  same_layout(t, &r);
  return r;
}

sa_problem problem(const at::Tensor& q, const at::Tensor& k, PyObject* w, uint32_t flags,
                   PyObject* scale) {
  sa_problem p{};
  if (q.scalar_type() == at::kFloat) p.dtype = SA_F32;
  else if (q.scalar_type() == at::kBFloat16) p.dtype = SA_BF16;
  else raise(PyExc_TypeError, "q/k/v must be float32 or bfloat16");
  if (q.dim() != 4 || k.dim() != 4) raise(PyExc_ValueError, "q, k, v must be [B,H,n,d]");
  p.B = (int32_t)q.size(0);
  p.Hq = (int32_t)q.size(1);
  p.Hkv = (int32_t)k.size(1);
  p.n = (int32_t)q.size(2);
  p.d = (int32_t)q.size(3);
  p.w = (int32_t)integer(w);
  p.flags = flags;
  p.softmax_scale = (float)real(scale);
  if (q.stride(3) != 1 || k.stride(3) != 1)
    raise(PyExc_ValueError, "the head dimension must be contiguous");
  for (int i = 0; i < 3; ++i) {
    p.q_stride[i] = q.stride(i);
    p.kv_stride[i] = k.stride(i);
  }
  return p;
}

size_t ws_bytes(const sa_problem& p, int op) {
  const size_t n = sa_workspace_bytes(&p, op);
  if (n == (size_t)-1) check(SA_ERR_INVALID_ARG, "sa_workspace_bytes");
  return n;
}

// Scratch for the SA branch's key lists, from the allocator's pool of the current stream; undefined
// where the problem has no use for any, and, with a warning (the sums run in another order then), where there
// is no memory for it.
at::Tensor key_lists(const sa_problem& p, c10::Device dev) {
  const size_t n = sa_workspace_bytes(&p, SA_OP_KEY_LISTS);
  if (n == 0 || n == (size_t)-1) return at::Tensor();
  try {
    return fresh({(int64_t)n}, at::kByte, dev);
  } catch (const c10::OutOfMemoryError&) {
    if (PyErr_WarnEx(PyExc_RuntimeWarning, "no memory for the key lists: the call goes without them", 1) < 0)
      throw Raised{};
    return at::Tensor();
  }
}
void* ptr_or_null(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
size_t bytes_of(const at::Tensor& t) { return t.defined() ? (size_t)t.numel() : 0; }

PyObject* wrap(at::Tensor t) { return THPVariable_Wrap(std::move(t)); }
PyObject* pass(PyObject* o) {
  Py_INCREF(o);
  return o;
}

PyObject* tuple(std::initializer_list<PyObject*> items) {
  PyObject* r = PyTuple_New((Py_ssize_t)items.size());
  Py_ssize_t i = 0;
  for (PyObject* o : items) PyTuple_SET_ITEM(r, i++, o);
  return r;
}

// An output: the caller's tensor, or a fresh one (kept alive by `own`).
struct Out {
  at::Tensor own;
  PyObject* given = nullptr;
  const at::Tensor* t = nullptr;
  PyObject* result() { return given ? pass(given) : wrap(own); }
};
template <typename F>
Out output(PyObject* o, F&& make) {
  Out r;
  if (o != Py_None) {
    r.given = o;
    r.t = &tensor(o);
  } else {
    r.own = make();
  }
  return r;
}
void* ptr(const Out& o) { return o.t ? o.t->data_ptr() : o.own.data_ptr(); }

at::Tensor rows_f32(const at::Tensor& q) {
  return fresh({q.size(0), q.size(1), q.size(2)}, at::kFloat, q.device());
}

// make_perm(seed, layer, B, n, perm, inv, ws): perm or inv None: made on the current device
PyObject* make_perm(PyObject* const* a) {
  const int64_t B = size(a[2]), n = size(a[3]);
  const c10::Device dev = a[4] != Py_None ? tensor(a[4]).device()
                                          : c10::Device(c10::kCUDA, c10::cuda::current_device());
  auto make = [&] { return fresh({B, n}, at::kInt, dev); };
  sa_problem p{};
  p.B = (int32_t)B;
  p.n = (int32_t)n;
  const size_t need = ws_bytes(p, SA_OP_MAKE_PERM);
  Out perm = output(a[4], make), inv = output(a[5], make);
  at::Tensor own;
  const at::Tensor* ws = tensor_or_null(a[6]);
  if (!ws) ws = &(own = fresh({(int64_t)need}, at::kByte, dev));
  check(unlocked(sa_make_perm, integer_mask(a[0]), (uint32_t)integer(a[1]), p.B, p.n, (int32_t*)ptr(perm),
                     (int32_t*)ptr(inv), ptr(*ws), (size_t)ws->numel(), stream()),
        "sa_make_perm");
  return tuple({perm.result(), inv.result()});
}

// forward(q, k, v, perm, inv, w, flags, scale, y, want_lse, lse)
PyObject* forward(PyObject* const* a) {
  const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]), &v = tensor(a[2]);
  same_layout(k, &v);
  const sa_problem p = problem(q, k, a[5], (uint32_t)integer(a[6]), a[7]);
  Out y = output(a[8], [&] { return fresh_like(q); });
  same_layout(q, y.t);
  const bool has_lse = a[10] != Py_None || truth(a[9]);
  Out lse;
  if (has_lse) lse = output(a[10], [&] { return rows_f32(q); });
  at::Tensor lists = key_lists(p, q.device());
  check(unlocked(sa_forward_lists, &p, ptr(q), ptr(k), ptr(v), (const int32_t*)ptr(tensor(a[3])),
                   (const int32_t*)ptr(tensor(a[4])), ptr(y), has_lse ? (float*)ptr(lse) : nullptr,
                   ptr_or_null(lists), bytes_of(lists), stream()),
        "sa_forward");
  return has_lse ? tuple({y.result(), lse.result()}) : y.result();
}

// gated_forward(q, k, v, perm, inv, gate_logits, w, flags, scale, save_for_bwd,
//               y, y_sa, y_swa, lse_sa, lse_swa, ws)
PyObject* gated_forward(PyObject* const* a) {
  const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]), &v = tensor(a[2]);
  same_layout(k, &v);
  const bool save = truth(a[9]);
  const uint32_t flags = (uint32_t)integer(a[7]) | (save ? SA_SAVE_FOR_BWD : 0u);
  auto like_q = [&] { return fresh_like(q); };
  auto rows = [&] { return rows_f32(q); };
  Out y = output(a[10], like_q), branch[2], lse[2];
  same_layout(q, y.t);
  for (int x = 0; x < 2; ++x) {
    if (save || a[11 + x] != Py_None) branch[x] = output(a[11 + x], like_q);
    same_layout(q, branch[x].t);
    if (save || a[13 + x] != Py_None) lse[x] = output(a[13 + x], rows);
  }
  auto at_or_null = [](const Out& o) { return o.t || o.own.defined() ? ptr(o) : nullptr; };
  const sa_problem p = problem(q, k, a[6], flags, a[8]);
  const at::Tensor* ws = tensor_or_null(a[15]);
  if (ws && ((uintptr_t)ptr(ws) & 15u)) check(SA_ERR_INVALID_ARG, "sa_swa_gated_forward");
  at::Tensor lists = key_lists(p, q.device());
  check(unlocked(sa_swa_gated_forward_lists, &p, ptr(q), ptr(k), ptr(v), (const int32_t*)ptr(tensor(a[3])),
                             (const int32_t*)ptr(tensor(a[4])), (const float*)ptr(tensor(a[5])),
                             ptr(y), at_or_null(branch[0]), at_or_null(branch[1]),
                             (float*)at_or_null(lse[0]), (float*)at_or_null(lse[1]), ptr_or_null(lists),
                             bytes_of(lists), stream()),
        "sa_swa_gated_forward");
  if (!save) return y.result();
  return tuple({y.result(), branch[0].result(), branch[1].result(), lse[0].result(),
                lse[1].result()});
}

// backward(q, k, v, perm, inv, gate_logits, y_sa, y_swa, lse_sa, lse_swa, dy, w, flags, scale, ws,
//          dq, dk, dv, dgate)
PyObject* backward(PyObject* const* a) {
  const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]), &v = tensor(a[2]);
  same_layout(k, &v);
  const at::Tensor *gate = tensor_or_null(a[5]), *y_swa = tensor_or_null(a[7]),
                   *lse_swa = tensor_or_null(a[9]);
  const at::Tensor &y_sa = tensor(a[6]), &dy = tensor(a[10]);
  same_layout(q, &dy);
  same_layout(q, &y_sa);
  same_layout(q, y_swa);
  Out dq = output(a[15], [&] { return fresh_like(q); });
  Out dk = output(a[16], [&] { return fresh_like(k); });
  Out dv = output(a[17], [&] { return fresh_like(v); });
  same_layout(q, dq.t);
  same_layout(k, dk.t);
  same_layout(k, dv.t);
  Out dgate;
  if (gate) dgate = output(a[18], [&] { return fresh({2, q.size(1)}, at::kFloat, q.device()); });
  const sa_problem p = problem(q, k, a[11], (uint32_t)integer(a[12]), a[13]);
  at::Tensor own;
  const at::Tensor* ws = tensor_or_null(a[14]);
  if (!ws) ws = &(own = fresh({(int64_t)ws_bytes(p, SA_OP_BACKWARD)}, at::kByte, q.device()));
  check(unlocked(sa_backward, &p, ptr(q), ptr(k), ptr(v), (const int32_t*)ptr(tensor(a[3])),
                    (const int32_t*)ptr(tensor(a[4])), (const float*)ptr(gate), ptr(y_sa),
                    ptr(y_swa), (const float*)ptr(tensor(a[8])), (const float*)ptr(lse_swa),
                    ptr(dy), ptr(dq), ptr(dk), ptr(dv), gate ? (float*)ptr(dgate) : nullptr,
                    ptr(*ws), (size_t)ws->numel(), stream()),
        "sa_backward");
  return tuple({dq.result(), dk.result(), dv.result(), gate ? dgate.result() : pass(Py_None)});
}

// ---- 4-bit paged cache ----

// A number that the C call takes in 32 bits, signed or not: refused here where it would lose some.
long long small(PyObject* o) {
  PyObject* i = PyLong_CheckExact(o) ? o : PyNumber_Long(o);
  if (!i) throw Raised{};
  int over = 0;
  const long long v = PyLong_AsLongLongAndOverflow(i, &over);
  if (i != o) Py_DECREF(i);
  if (over || v < -(1ll << 31) || v >= (1ll << 32))
    raise(PyExc_ValueError, "layer, w, flags and page must be numbers of 32 bits");
  return v;
}
int32_t extent(const at::Tensor& t, int i) {
  if (t.size(i) > 0x7fffffff) raise(PyExc_ValueError, "a dimension of 2^31 or more");
  return (int32_t)t.size(i);
}

void ints(const at::Tensor* t, at::IntArrayRef sizes, const at::Tensor& like, const char* text) {
  if (t && (t->scalar_type() != at::kInt || t->sizes() != sizes || !t->is_contiguous() ||
            t->device() != like.device()))
    raise(PyExc_ValueError, text);
}
int32_t* int_ptr(const at::Tensor* t) { return t ? (int32_t*)t->data_ptr() : nullptr; }

// The cache that pool, table, lens and refs (nullable: not needed) describe.  Without a pool, the books
// alone, any head dimension is valid.
sa_cache cache(const at::Tensor* pool, const at::Tensor& table, const at::Tensor* lens,
               const at::Tensor* refs, int64_t page, int64_t d) {
  if (table.dim() != 2 || table.scalar_type() != at::kInt || !table.is_contiguous())
    raise(PyExc_ValueError, "table must be contiguous int32 [slots, row]");
  sa_cache c{};
  c.k_scale = c.v_scale = 1.f;
  c.layers = c.pages = c.Hkv = 1;
  c.d = (int32_t)d;
  c.page = (int32_t)page;
  c.slots = (int32_t)table.size(0);
  c.row = (int32_t)table.size(1);
  c.table = int_ptr(&table);
  ints(lens, {table.size(0)}, table, "lens must be contiguous int32 [slots] on the table's device");
  c.lens = int_ptr(lens);
  if (pool) {
    if (pool->scalar_type() != at::kByte || pool->dim() != 5 || pool->size(3) != 2 || !pool->is_contiguous() ||
        pool->device() != table.device())
      raise(PyExc_ValueError,
            "pool must be contiguous uint8 [layers, pages, Hkv, 2, page * (d/2 + d/16)] on the table's device");
    if (d % 16 || pool->size(4) != page * (d / 2 + d / 16))
      raise(PyExc_ValueError, "the pool's pages do not hold that many tokens of this head dimension");
    c.pool = (uint8_t*)pool->data_ptr();
    c.layers = (int32_t)pool->size(0);
    c.pages = (int32_t)pool->size(1);
    c.Hkv = (int32_t)pool->size(2);
  } else if (refs) {
    c.pages = (int32_t)refs->numel();
  }
  ints(refs, {c.pages}, table, "refs must be contiguous int32 [pages] on the table's device");
  c.refs = int_ptr(refs);
  return c;
}

// Tokens per page: what the caller says, else what the pool's bytes make of the tensors' head dimension.
int64_t page_of(const at::Tensor& pool, int64_t d, PyObject* page) {
  if (page != Py_None) return small(page);
  return pool.dim() == 5 && d ? pool.size(4) * 16 / (9 * d) : 0;
}

int rows_dtype(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return SA_F32;
  if (t.scalar_type() == at::kBFloat16) return SA_BF16;
  raise(PyExc_TypeError, "tensors must be float32 or bfloat16");
}

// Element strides of [B,H,T,d]; a dimension of one may have any, an output none of 0 otherwise.
struct Strides {
  int64_t s[3];
};
Strides row_strides(const at::Tensor& t, bool written) {
  if (t.stride(3) != 1) raise(PyExc_ValueError, "the head dimension must be contiguous");
  Strides r;
  for (int i = 0; i < 3; ++i) {
    r.s[i] = t.size(i) > 1 ? t.stride(i) : 0;
    if (written && t.size(i) > 1 && t.stride(i) == 0)
      raise(PyExc_ValueError, "an output shares memory between its rows");
  }
  return r;
}

void on_gpu(const at::Tensor& t) {
  if (!t.is_cuda()) raise(PyExc_ValueError, "the cache must be on a CUDA device");
}

at::Tensor scratch(PyObject* given, size_t need, const at::Tensor& like, const char* where, size_t* bytes,
                   void** at) {
  if (need == (size_t)-1) check(SA_ERR_INVALID_ARG, where);
  on_gpu(like);
  at::Tensor own;
  const at::Tensor* ws = tensor_or_null(given);
  if (!ws) ws = &(own = fresh({(int64_t)need}, at::kByte, like.device()));
  else if (ws->device() != like.device() || !ws->is_contiguous())
    raise(PyExc_ValueError, "ws must be contiguous on the cache's device");
  *bytes = ws->numel() * ws->element_size();
  *at = ws->data_ptr();
  return own;
}

// What append and read share: their checks, and the cache.
struct Rows {
  sa_cache c;
  Strides st;
  int32_t B, T, layer;
};
Rows rows(const at::Tensor& pool, const at::Tensor& table, const at::Tensor* lens, const at::Tensor& k,
          const at::Tensor& v, std::initializer_list<const at::Tensor*> lists, PyObject* k_scale,
          PyObject* v_scale, PyObject* page, PyObject* layer, bool written) {
  if (k.dim() != 4 || v.sizes() != k.sizes() || v.scalar_type() != k.scalar_type() ||
      k.device() != pool.device() || v.device() != pool.device())
    raise(PyExc_ValueError, "k and v must be [B,Hkv,T,d] of one type on the cache's device");
  Rows r;
  r.st = row_strides(k, written);
  const Strides sv = row_strides(v, written);
  for (int i = 0; i < 3; ++i)
    if (r.st.s[i] != sv.s[i]) raise(PyExc_ValueError, "k and v must share their strides");
  r.B = extent(k, 0);
  r.T = extent(k, 2);
  r.layer = (int32_t)small(layer);
  r.c = cache(&pool, table, lens, nullptr, page_of(pool, k.size(3), page), k.size(3));
  r.c.k_scale = (float)real(k_scale);
  r.c.v_scale = (float)real(v_scale);
  if (k.size(1) != r.c.Hkv) raise(PyExc_ValueError, "k and v must have the pool's heads");
  for (const at::Tensor* t : lists)
    ints(t, {k.size(0)}, table, "slots, starts and counts must be contiguous int32 [B] on the cache's device");
  return r;
}

// cache_append(pool, table, lens, k, v, layer, slots, counts, k_scale, v_scale, refs, page)
PyObject* cache_append(PyObject* const* a) {
  const at::Tensor &pool = tensor(a[0]), &k = tensor(a[3]), &v = tensor(a[4]);
  const at::Tensor *slots = tensor_or_null(a[6]), *counts = tensor_or_null(a[7]);
  Rows r = rows(pool, tensor(a[1]), &tensor(a[2]), k, v, {slots, counts}, a[8], a[9], a[11], a[5], false);
  const at::Tensor* refs = tensor_or_null(a[10]);
  ints(refs, {r.c.pages}, pool, "refs must be contiguous int32 [pages] on the cache's device");
  r.c.refs = int_ptr(refs);
  on_gpu(pool);
  const c10::cuda::CUDAGuard guard(pool.device());
  check(unlocked(sa_cache_append, &r.c, r.layer, r.B, r.T, ptr(k), ptr(v), rows_dtype(k), r.st.s,
                 int_ptr(slots), int_ptr(counts), stream()),
        "sa_cache_append");
  return pass(Py_None);
}

// cache_read(pool, table, k, v, layer, slots, starts, counts, k_scale, v_scale, page)
PyObject* cache_read(PyObject* const* a) {
  const at::Tensor &pool = tensor(a[0]), &k = tensor(a[2]), &v = tensor(a[3]);
  const at::Tensor *slots = tensor_or_null(a[5]), *starts = tensor_or_null(a[6]), *counts = tensor_or_null(a[7]);
  const Rows r = rows(pool, tensor(a[1]), nullptr, k, v, {slots, starts, counts}, a[8], a[9], a[10], a[4], true);
  on_gpu(pool);
  const c10::cuda::CUDAGuard guard(pool.device());
  check(unlocked(sa_cache_read, &r.c, r.layer, r.B, r.T, ptr(k), ptr(v), rows_dtype(k), r.st.s,
                 int_ptr(slots), int_ptr(starts), int_ptr(counts), stream()),
        "sa_cache_read");
  return tuple({pass(a[2]), pass(a[3])});
}

// cache_attend(pool, table, lens, q, layer, slots, counts, w, flags, scale, k_scale, v_scale, y, want_lse,
//              lse, ws, page)
PyObject* cache_attend(PyObject* const* a) {
  const at::Tensor &pool = tensor(a[0]), &table = tensor(a[1]), &q = tensor(a[3]);
  if (q.dim() != 4 || q.device() != pool.device())
    raise(PyExc_ValueError, "q must be [B,Hq,T,d] on the cache's device");
  sa_cache c = cache(&pool, table, &tensor(a[2]), nullptr, page_of(pool, q.size(3), a[16]), q.size(3));
  c.k_scale = (float)real(a[10]);
  c.v_scale = (float)real(a[11]);
  const int dtype = rows_dtype(q);
  const Strides qs = row_strides(q, false);
  const at::Tensor *slots = tensor_or_null(a[5]), *counts = tensor_or_null(a[6]);
  for (const at::Tensor* t : {slots, counts})
    ints(t, {q.size(0)}, table, "slots and counts must be contiguous int32 [B] on the cache's device");
  const int32_t B = extent(q, 0), Hq = extent(q, 1), T = extent(q, 2);
  const int32_t layer = (int32_t)small(a[4]), w = (int32_t)small(a[7]);
  const uint32_t flags = (uint32_t)small(a[8]);
  const at::Tensor *y_in = tensor_or_null(a[12]), *lse_in = tensor_or_null(a[14]);
  if (y_in && (y_in->sizes() != q.sizes() || y_in->scalar_type() != q.scalar_type() || y_in->device() != q.device()))
    raise(PyExc_ValueError, "y must have the shape and type of q");
  if (lse_in && (lse_in->sizes() != q.sizes().slice(0, 3) || lse_in->scalar_type() != at::kFloat ||
                 !lse_in->is_contiguous() || lse_in->device() != q.device()))
    raise(PyExc_ValueError, "lse must be contiguous float32 [B,Hq,T]");
  if (y_in) row_strides(*y_in, true);
  const bool has_lse = lse_in || truth(a[13]);
  const size_t need = sa_cache_attend_ws_bytes(&c, B, T, Hq, dtype);
  size_t bytes;
  void* ws;
  const c10::cuda::OptionalCUDAGuard guard(pool.is_cuda() ? std::optional<c10::Device>(pool.device()) : std::nullopt);
  const at::Tensor own = scratch(a[15], need, pool, "sa_cache_attend", &bytes, &ws);
  Out y = output(a[12], [&] { return fresh(q.sizes(), q.scalar_type(), q.device()); });
  const Strides ys = row_strides(y.t ? *y.t : y.own, true);
  Out lse;
  if (has_lse) lse = output(a[14], [&] { return rows_f32(q); });
  check(unlocked(sa_cache_attend, &c, layer, B, T, Hq, ptr(q), dtype, qs.s, int_ptr(slots), int_ptr(counts), w,
                 flags, (float)real(a[9]), ptr(y), ys.s, has_lse ? (float*)ptr(lse) : nullptr, ws, bytes, stream()),
        "sa_cache_attend");
  return has_lse ? tuple({y.result(), lse.result()}) : y.result();
}

const at::Tensor& list_of(PyObject* o, const at::Tensor& table) {
  const at::Tensor& t = tensor(o);
  ints(&t, {t.numel()}, table, "slot lists must be contiguous int32 [n] on the cache's device");
  return t;
}

// cache_free(table, lens, refs, slots)
PyObject* cache_free(PyObject* const* a) {
  const at::Tensor& table = tensor(a[0]);
  const sa_cache c = cache(nullptr, table, &tensor(a[1]), &tensor(a[2]), 16, 16);
  const at::Tensor& slots = list_of(a[3], table);
  on_gpu(table);
  const c10::cuda::CUDAGuard guard(table.device());
  check(unlocked(sa_cache_free, &c, (int32_t)slots.numel(), int_ptr(&slots), stream()), "sa_cache_free");
  return pass(Py_None);
}

// cache_fork(table, lens, refs, parents, children, page)
PyObject* cache_fork(PyObject* const* a) {
  const at::Tensor& table = tensor(a[0]);
  const sa_cache c = cache(nullptr, table, &tensor(a[1]), &tensor(a[2]), small(a[5]), 16);
  const at::Tensor &parents = list_of(a[3], table), &children = list_of(a[4], table);
  if (parents.numel() != children.numel())
    raise(PyExc_ValueError, "parents and children must have one length");
  on_gpu(table);
  const c10::cuda::CUDAGuard guard(table.device());
  check(unlocked(sa_cache_fork, &c, (int32_t)parents.numel(), int_ptr(&parents), int_ptr(&children), stream()),
        "sa_cache_fork");
  return pass(Py_None);
}

// The head dimension that a page of the pool has with this many tokens.
int64_t head_dim(const at::Tensor& pool, int64_t page) {
  return pool.dim() == 5 && page > 0 ? pool.size(4) * 16 / (9 * page) : 0;
}

// cache_reserve(pool, table, lens, refs, add, page, got, ws)
PyObject* cache_reserve(PyObject* const* a) {
  const at::Tensor &pool = tensor(a[0]), &table = tensor(a[1]), &add = tensor(a[4]);
  const int64_t page = small(a[5]);
  const sa_cache c = cache(&pool, table, &tensor(a[2]), &tensor(a[3]), page, head_dim(pool, page));
  ints(&add, {c.slots}, table, "add must be contiguous int32 [slots] on the cache's device");
  ints(tensor_or_null(a[6]), {c.slots}, table, "got must be contiguous int32 [slots] on the cache's device");
  size_t bytes;
  void* ws;
  const c10::cuda::OptionalCUDAGuard guard(pool.is_cuda() ? std::optional<c10::Device>(pool.device()) : std::nullopt);
  const at::Tensor own = scratch(a[7], sa_cache_ws_bytes(&c), pool, "sa_cache_ws_bytes", &bytes, &ws);
  Out got = output(a[6], [&] { return fresh({c.slots}, at::kInt, pool.device()); });
  check(unlocked(sa_cache_reserve, &c, int_ptr(&add), (int32_t*)ptr(got), ws, bytes, stream()), "sa_cache_reserve");
  return got.result();
}

// cache_compact(pool, table, refs, live, ws)
PyObject* cache_compact(PyObject* const* a) {
  const at::Tensor &pool = tensor(a[0]), &table = tensor(a[1]);
  // any page and head dimension with the pool's bytes describe the moves
  int64_t page = 128;
  if (pool.dim() != 5) raise(PyExc_ValueError, "pool must be [layers, pages, Hkv, 2, bytes]");
  while (page > 16 && (pool.size(4) % (9 * page) || head_dim(pool, page) < 16 || head_dim(pool, page) > 256)) page /= 2;
  const sa_cache c = cache(&pool, table, nullptr, &tensor(a[2]), page, head_dim(pool, page));
  ints(tensor_or_null(a[3]), {1}, table, "live must be int32 [1] on the cache's device");
  size_t bytes;
  void* ws;
  const c10::cuda::OptionalCUDAGuard guard(pool.is_cuda() ? std::optional<c10::Device>(pool.device()) : std::nullopt);
  const at::Tensor own = scratch(a[4], sa_cache_ws_bytes(&c), pool, "sa_cache_ws_bytes", &bytes, &ws);
  Out live = output(a[3], [&] { return fresh({1}, at::kInt, pool.device()); });
  check(unlocked(sa_cache_compact, &c, (int32_t*)ptr(live), ws, bytes, stream()), "sa_cache_compact");
  return live.result();
}

template <PyObject* (*F)(PyObject* const*), int kArgs>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != kArgs) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return F(args);
  } catch (const Raised&) {
  } catch (const c10::OutOfMemoryError& e) {
    PyObject* torch_module = PyImport_ImportModule("torch");
    PyObject* type = torch_module ? PyObject_GetAttrString(torch_module, "OutOfMemoryError") : nullptr;
    if (type) PyErr_SetString(type, e.what_without_backtrace());
    Py_XDECREF(type);
    Py_XDECREF(torch_module);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

PyObject* set_error_class(PyObject*, PyObject* cls) {
  Py_INCREF(cls);
  Py_XDECREF(g_error_class);
  g_error_class = cls;
  Py_RETURN_NONE;
}

#define SA_FAST(name, n) \
  {#name, (PyCFunction)(void (*)(void))entry<name, n>, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {
    SA_FAST(make_perm, 7),
    SA_FAST(forward, 11),
    SA_FAST(gated_forward, 16),
    SA_FAST(backward, 19),
    SA_FAST(cache_append, 12),
    SA_FAST(cache_read, 11),
    SA_FAST(cache_attend, 17),
    SA_FAST(cache_free, 4),
    SA_FAST(cache_fork, 6),
    SA_FAST(cache_reserve, 8),
    SA_FAST(cache_compact, 5),
    {"set_error_class", set_error_class, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, g_methods,
                        nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&g_module); }

// Entry points of the 4-bit cache: argument checks, then the launchers.
#include <cmath>

#include "sa_cache.cuh"

namespace sa {
namespace {

bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool ints(const void* p) { return p && aligned(p, 4); }
bool ints_or_null(const void* p) { return aligned(p, 4); }

bool power_of_two(float x) {
  int e;
  return x > 0.f && std::isfinite(x) && std::frexp(x, &e) == 0.5f && e >= -31 && e <= 33;
}

sa_status check_geometry(const sa_cache* c) {
  if (!c) return SA_ERR_INVALID_ARG;
  if (c->layers < 1 || c->pages < 1 || c->Hkv < 1 || c->d < 1 || c->slots < 1 || c->row < 1)
    return SA_ERR_INVALID_ARG;
  if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return SA_ERR_INVALID_ARG;
  if (c->d % 16 != 0 || c->d > 256 || c->Hkv > 32767) return SA_ERR_UNSUPPORTED;
  // positions and table entries are counted in 32 bits
  if ((int64_t)c->row * c->page > (1ll << 30) || (int64_t)c->slots * c->row > 0x7fffffff) return SA_ERR_UNSUPPORTED;
  return SA_OK;
}

// The books that a call reads or writes, by what it needs.
sa_status check_books(const sa_cache* c, bool pool, bool lens, bool refs) {
  const sa_status s = check_geometry(c);
  if (s != SA_OK) return s;
  if (!ints(c->table) || (lens && !ints(c->lens)) || (refs && !ints(c->refs)) ||
      (pool && (!c->pool || !aligned(c->pool, 16))))
    return SA_ERR_INVALID_ARG;
  return SA_OK;
}

// Strides of [B,H,T,d]: whole 16-byte pieces; a dimension of one has any stride.
bool good_strides(const int64_t* s, int d, int T) {
  if (!s) return false;
  for (int i = 0; i < 3; ++i)
    if (s[i] < 0 || s[i] % 8 != 0) return false;
  return T == 1 || s[2] >= d;
}

// Of an output: no two rows in one place.
bool rows_apart(const int64_t* s, int B, int H) { return (B == 1 || s[0] > 0) && (H == 1 || s[1] > 0); }

sa_status check_rows(const sa_cache* c, int32_t layer, int32_t B, int32_t T, int32_t dtype,
                     bool lens) {
  const sa_status s = check_books(c, true, lens, false);
  if (s != SA_OK) return s;
  if (!power_of_two(c->k_scale) || !power_of_two(c->v_scale)) return SA_ERR_INVALID_ARG;
  if (layer < 0 || layer >= c->layers || B < 1 || T < 1) return SA_ERR_INVALID_ARG;
  if (dtype != SA_F32 && dtype != SA_BF16) return SA_ERR_INVALID_ARG;
  if (B > 65535 || T > (1 << 28)) return SA_ERR_UNSUPPORTED;
  return SA_OK;
}

CacheView view(const sa_cache* c, int32_t layer, int* status) {
  CacheView v{};
  v.page_bytes = (int64_t)sa_cache_page_bytes(c);
  v.pool = c->pool + (int64_t)layer * c->pages * v.page_bytes;
  v.table = c->table;
  v.lens = c->lens;
  v.pages = c->pages;
  v.Hkv = c->Hkv;
  v.d = c->d;
  v.P = c->page;
  v.p_shift = c->page == 16 ? 4 : c->page == 32 ? 5 : c->page == 64 ? 6 : 7;
  v.slots = c->slots;
  v.row = c->row;
  v.side = c->page * (c->d / 2 + c->d / 16);
  v.k_scale = c->k_scale;
  v.v_scale = c->v_scale;
  v.status = status;
  return v;
}

sa_status rows(const sa_cache* c, bool read, int32_t layer, int32_t B, int32_t T, void* k, void* v,
               int32_t dtype, const int64_t* stride, const int32_t* slots, const int32_t* starts,
               const int32_t* counts, sa_stream_t stream) {
  const sa_status s = check_rows(c, layer, B, T, dtype, !read);
  if (s != SA_OK) return s;
  if (!k || !v || (read && k == v) || !aligned(k, 16) || !aligned(v, 16) || !good_strides(stride, c->d, T) ||
      (read && !rows_apart(stride, B, c->Hkv)) || !ints_or_null(slots) || !ints_or_null(starts) || !ints_or_null(counts) || (!read && !ints_or_null(c->refs)))
    return SA_ERR_INVALID_ARG;
  int* status = cache_status_ptr();
  if (!status) return SA_ERR_CUDA;
  return launch_cache_rows(view(c, layer, status), read, B, T, k, v, dtype, stride, slots, starts, counts,
                           read ? nullptr : c->refs, (cudaStream_t)stream) == cudaSuccess ? SA_OK : SA_ERR_CUDA;
}

bool good_heads(const sa_cache* c, int32_t Hq) { return Hq >= c->Hkv && Hq % c->Hkv == 0 && Hq <= 65535; }

// Row tiles of all sequences are counted in 32 bits.
bool attend_fits(const sa_cache* c, int32_t B, int32_t T, int32_t Hq) {
  const int64_t rows = (int64_t)Hq / c->Hkv * T;
  return rows < (1ll << 30) && (rows / 8 + 1) * B < (1ll << 30);
}

}  // namespace
}  // namespace sa

using namespace sa;

extern "C" {

size_t sa_cache_page_bytes(const sa_cache* c) {
  return check_geometry(c) == SA_OK ? (size_t)c->Hkv * 2 * c->page * (c->d / 2 + c->d / 16) : 0;
}

sa_status sa_cache_append(const sa_cache* c, int32_t layer, int32_t B, int32_t T, const void* k,
                          const void* v, int32_t dtype, const int64_t kv_stride[3],
                          const int32_t* slots, const int32_t* counts, sa_stream_t stream) {
  return rows(c, false, layer, B, T, const_cast<void*>(k), const_cast<void*>(v), dtype, kv_stride, slots,
              nullptr, counts, stream);
}

sa_status sa_cache_read(const sa_cache* c, int32_t layer, int32_t B, int32_t T, void* k, void* v,
                        int32_t dtype, const int64_t kv_stride[3], const int32_t* slots,
                        const int32_t* starts, const int32_t* counts, sa_stream_t stream) {
  return rows(c, true, layer, B, T, k, v, dtype, kv_stride, slots, starts, counts, stream);
}

size_t sa_cache_attend_ws_bytes(const sa_cache* c, int32_t B, int32_t T, int32_t Hq, int32_t dtype) {
  if (check_geometry(c) != SA_OK || B < 1 || T < 1 || !good_heads(c, Hq) || !attend_fits(c, B, T, Hq) ||
      (dtype != SA_F32 && dtype != SA_BF16))
    return (size_t)-1;
  return cache_attend_ws_bytes(B, T, Hq, c->Hkv, c->d, dtype);
}

sa_status sa_cache_attend(const sa_cache* c, int32_t layer, int32_t B, int32_t T, int32_t Hq,
                          const void* q, int32_t dtype, const int64_t q_stride[3],
                          const int32_t* slots, const int32_t* counts, int32_t w, uint32_t flags,
                          float softmax_scale, void* y, const int64_t y_stride[3], float* lse,
                          void* ws, size_t ws_bytes, sa_stream_t stream) {
  const sa_status s = check_rows(c, layer, B, T, dtype, true);
  if (s != SA_OK) return s;
  if (!good_heads(c, Hq) || w < 0 || (flags & ~(uint32_t)SA_CAUSAL) || !(softmax_scale >= 0.f) ||
      std::isinf(softmax_scale))
    return SA_ERR_INVALID_ARG;
  if (!attend_fits(c, B, T, Hq)) return SA_ERR_UNSUPPORTED;
  if (!q || !y || q == y || !ws || !aligned(q, 16) || !aligned(y, 16) || !aligned(ws, 16) || !ints_or_null(lse) ||
      !ints_or_null(slots) || !ints_or_null(counts) || !good_strides(q_stride, c->d, T) ||
      !good_strides(y_stride, c->d, T) || !rows_apart(y_stride, B, Hq))
    return SA_ERR_INVALID_ARG;
  if (ws_bytes < cache_attend_ws_bytes(B, T, Hq, c->Hkv, c->d, dtype)) return SA_ERR_WORKSPACE;
  int* status = cache_status_ptr();
  if (!status) return SA_ERR_CUDA;
  AttendArgs a{};
  a.c = view(c, layer, status);
  a.q = q;
  a.y = y;
  a.lse = lse;
  a.slots = slots;
  a.counts = counts;
  for (int i = 0; i < 3; ++i) {
    a.qs[i] = q_stride[i];
    a.ys[i] = y_stride[i];
  }
  a.B = B;
  a.T = T;
  a.Hq = Hq;
  a.w = w;
  a.causal = flags & SA_CAUSAL;
  a.scale = softmax_scale > 0.f ? softmax_scale : 1.0f / std::sqrt((float)c->d);
  a.ws = ws;
  return launch_cache_attend(a, dtype, (cudaStream_t)stream) == cudaSuccess ? SA_OK : SA_ERR_CUDA;
}

sa_status sa_cache_free(const sa_cache* c, int32_t n, const int32_t* slots, sa_stream_t stream) {
  const sa_status s = check_books(c, false, true, true);
  if (s != SA_OK) return s;
  if (n < 0 || (n && !ints(slots))) return SA_ERR_INVALID_ARG;
  if (n == 0) return SA_OK;
  int* status = cache_status_ptr();
  if (!status) return SA_ERR_CUDA;
  return launch_cache_free(*c, n, slots, status, (cudaStream_t)stream) == cudaSuccess ? SA_OK : SA_ERR_CUDA;
}

sa_status sa_cache_fork(const sa_cache* c, int32_t n, const int32_t* parents,
                        const int32_t* children, sa_stream_t stream) {
  const sa_status s = check_books(c, false, true, true);
  if (s != SA_OK) return s;
  if (n < 0 || (n && (!ints(parents) || !ints(children)))) return SA_ERR_INVALID_ARG;
  if (n == 0) return SA_OK;
  int* status = cache_status_ptr();
  if (!status) return SA_ERR_CUDA;
  return launch_cache_fork(*c, n, parents, children, status, (cudaStream_t)stream) == cudaSuccess
             ? SA_OK : SA_ERR_CUDA;
}

size_t sa_cache_ws_bytes(const sa_cache* c) {
  return check_geometry(c) == SA_OK ? cache_books_ws_bytes(*c) : (size_t)-1;
}

sa_status sa_cache_reserve(const sa_cache* c, const int32_t* add, int32_t* got, void* ws,
                           size_t ws_bytes, sa_stream_t stream) {
  const sa_status s = check_books(c, true, true, true);
  if (s != SA_OK) return s;
  // add is read after the first of got is written
  if (!ints(add) || !ints(got) || add == got || !ws || !aligned(ws, 16)) return SA_ERR_INVALID_ARG;
  if (ws_bytes < cache_books_ws_bytes(*c)) return SA_ERR_WORKSPACE;
  int* status = cache_status_ptr();
  if (!status) return SA_ERR_CUDA;
  return launch_cache_reserve(*c, add, got, ws, status, (cudaStream_t)stream) == cudaSuccess
             ? SA_OK : SA_ERR_CUDA;
}

sa_status sa_cache_compact(const sa_cache* c, int32_t* live, void* ws, size_t ws_bytes,
                           sa_stream_t stream) {
  const sa_status s = check_books(c, true, false, true);
  if (s != SA_OK) return s;
  if (!ints_or_null(live) || !ws || !aligned(ws, 16)) return SA_ERR_INVALID_ARG;
  if (ws_bytes < cache_books_ws_bytes(*c)) return SA_ERR_WORKSPACE;
  int* status = cache_status_ptr();
  if (!status) return SA_ERR_CUDA;
  return launch_cache_compact(*c, live, ws, status, (cudaStream_t)stream) == cudaSuccess
             ? SA_OK : SA_ERR_CUDA;
}

}  // extern "C"

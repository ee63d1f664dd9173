// The books of the 4-bit cache: who holds which pages, and the moves of pages that follow.
//
// Everything is decided on the device from the state before the call, in the order of slots, list
// entries and pages, so a captured call does the same as an eager one and no result depends on
// timing (counts are integers: the order of their atomics is free).
//
// The plans are chains of dependent accesses by one CTA (the order over all slots and pages needs one).  Calls with next
// to nothing to move, back to back: room for a token in 64 slots 7.3 us, in 1024 slots with 49152 pages 14.7, packing
// 8000 pages 8.2 (the plan alone from cold caches: 9.0, 19.2, 8.8).  The moves are copies: 3.5 GB in 550 us, 98 % of the
// copy bandwidth.
#include "sa_cache.cuh"

namespace sa {
namespace {

constexpr int kBook = 1024;        // threads of the single-CTA plans
constexpr int kMove = 256;         // threads of a copying CTA
constexpr int kPiece = 16 << 10;   // bytes a CTA copies at a time: 64 per thread

struct Books {
  uint8_t* pool;
  int32_t *table, *lens, *refs;
  int layers, pages, P, slots, row;
  int64_t page_bytes;
  int* status;
};

__device__ __forceinline__ void report(const Books& c) { atomicCAS(c.status, SA_OK, SA_ERR_BAD_CACHE); }

// Sum of v over the threads before this one, and over all of them.  All kBook threads call it.
__device__ __forceinline__ int before_me(int v, int* total) {
  __shared__ int sums[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int upto = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += u;
  }
  __syncthreads();   // the last call's readers are done
  if (lane == 31) sums[warp] = upto;
  __syncthreads();
  int s = sums[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += u;
  }
  *total = __shfl_sync(0xffffffffu, s, 31);
  const int base = __shfl_sync(0xffffffffu, s, max(warp - 1, 0));
  return upto - v + (warp ? base : 0);
}

// One CTA per listed slot.
__global__ void __launch_bounds__(128) free_kernel(const Books c, int n, const int32_t* list) {
  grid_dependency_wait();
  const int i = blockIdx.x, slot = list[i];
  bool bad = (unsigned)slot >= (unsigned)c.slots;
  for (int j = threadIdx.x; j < i; j += 128) bad |= list[j] == slot;   // the first mention counts
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) report(c);
    return;
  }
  int32_t* row = c.table + (int64_t)slot * c.row;
  for (int j = threadIdx.x; j < c.row; j += 128) {
    const int p = row[j];
    row[j] = -1;
    if (p == -1) continue;
    if ((unsigned)p >= (unsigned)c.pages) report(c);
    else if (atomicSub(&c.refs[p], 1) <= 0) {      // nobody held it: the books were wrong
      atomicAdd(&c.refs[p], 1);
      report(c);
    }
  }
  if (threadIdx.x == 0) c.lens[slot] = 0;
}

// One CTA per fork.  Refused (reported, child left as it is): a slot out of range, a child that is
// listed before, is a parent too or holds anything, a parent without the pages of its length.
__global__ void __launch_bounds__(128) fork_kernel(const Books c, int n, const int32_t* parents,
                                                   const int32_t* children) {
  grid_dependency_wait();
  const int i = blockIdx.x, from = parents[i], to = children[i];
  bool bad = (unsigned)from >= (unsigned)c.slots || (unsigned)to >= (unsigned)c.slots;
  for (int j = threadIdx.x; j < n; j += 128) bad |= (j < i && children[j] == to) || parents[j] == to;
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) report(c);
    return;
  }
  const int len = c.lens[from];
  const int held = len > 0 ? (len - 1) / c.P + 1 : 0;
  const int32_t* src = c.table + (int64_t)from * c.row;
  int32_t* dst = c.table + (int64_t)to * c.row;
  bad = len < 0 || held > c.row || c.lens[to] != 0;
  if (!bad) {
    for (int j = threadIdx.x; j < c.row; j += 128)
      bad |= dst[j] != -1 || (j < held && (unsigned)src[j] >= (unsigned)c.pages);
  }
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) report(c);
    return;
  }
  for (int j = threadIdx.x; j < held; j += 128) {
    const int p = src[j];
    dst[j] = p;
    atomicAdd(&c.refs[p], 1);
  }
  if (threadIdx.x == 0) c.lens[to] = len;
}

// Workspace of reserve: number of copies, [slots] wants, [slots] pages to copy, [pages] free pages.
struct Reserve {
  const int32_t* add;
  int32_t* got;
  int32_t* n_copy;
  int32_t* want;
  int2* copy;
  int32_t* free_list;
};

// Entries [lo, hi) of a slot's row that its next `add` tokens fall into; false: none asked for.
struct Span {
  int lo, hi, len;
  bool fits;
};
__device__ __forceinline__ Span span_of(const Books& c, const Reserve& r, int b) {
  Span s{0, 0, 0, true};
  const int add = r.add[b];
  s.len = c.lens[b];
  if (add == 0) return s;
  const int64_t most = (int64_t)c.row * c.P, upto = (int64_t)s.len + add;
  if (add < 0 || s.len < 0) {
    report(c);
    s.fits = false;
  } else if (upto > most) {
    s.fits = false;
  } else {
    s.lo = s.len / c.P;
    s.hi = (int)((upto + c.P - 1) / c.P);
  }
  return s;
}

// Every lane of a warp has a slot and a span of its entries (maybe empty).  Short spans are gone through by their
// lane, long ones (a prompt's) by the whole warp, one after the other.
constexpr int kShort = 4;

// f(entry, j) returns 1 to count the entry, -1 for a bad one; totals go to the span's own lane.
template <typename F>
__device__ __forceinline__ void entries_of(const Books& c, int b, const Span& s, F&& f, int* count, bool* bad) {
  const int lane = threadIdx.x & 31;
  int32_t* row = c.table + (int64_t)b * c.row;
  const bool is_long = s.hi - s.lo > kShort;
  if (!is_long)
    for (int j = s.lo; j < s.hi; ++j) {
      const int v = f(row + j, j);
      *count += v > 0;
      *bad |= v < 0;
    }
  for (uint32_t todo = __ballot_sync(0xffffffffu, is_long); todo; todo &= todo - 1) {
    const int of = __ffs(todo) - 1;
    const int lo = __shfl_sync(0xffffffffu, s.lo, of), hi = __shfl_sync(0xffffffffu, s.hi, of);
    int32_t* r = c.table + (int64_t)__shfl_sync(0xffffffffu, b, of) * c.row;
    for (int j0 = lo; j0 < hi; j0 += 32) {
      const int j = j0 + lane, v = j < hi ? f(r + j, j) : 0;
      const int n = __popc(__ballot_sync(0xffffffffu, v > 0));
      const bool any_bad = __any_sync(0xffffffffu, v < 0);
      if (lane == of) {
        *count += n;
        *bad |= any_bad;
      }
    }
  }
}

// take(entry, j, k, len) for the entries whose value passes, k = first, first + 1, ... in their order.
template <typename P, typename F>
__device__ __forceinline__ void ranked_entries_of(const Books& c, int b, const Span& s, int first, P&& passes, F&& take) {
  const int lane = threadIdx.x & 31;
  int32_t* row = c.table + (int64_t)b * c.row;
  const bool is_long = s.hi - s.lo > kShort;
  if (!is_long) {
    int k = first;
    for (int j = s.lo; j < s.hi; ++j)
      if (passes(row[j])) take(row + j, j, k++, s.len);
  }
  for (uint32_t todo = __ballot_sync(0xffffffffu, is_long); todo; todo &= todo - 1) {
    const int of = __ffs(todo) - 1;
    const int lo = __shfl_sync(0xffffffffu, s.lo, of), hi = __shfl_sync(0xffffffffu, s.hi, of);
    const int len = __shfl_sync(0xffffffffu, s.len, of);
    int k = __shfl_sync(0xffffffffu, first, of);
    int32_t* r = c.table + (int64_t)__shfl_sync(0xffffffffu, b, of) * c.row;
    for (int j0 = lo; j0 < hi; j0 += 32) {
      const int j = j0 + lane;
      const bool mine = j < hi && passes(r[j]);
      const uint32_t all = __ballot_sync(0xffffffffu, mine);
      if (mine) take(r + j, j, k + __popc(all & ((1u << lane) - 1u)), len);
      k += __popc(all);
    }
  }
}

// A warp's run of pages, 32 at a time and eight of those loads on the way: f(first page of the 32, this lane's count
// of holders, -1 behind the pool's end), called by all lanes.
struct Run {
  int p0, p1, pages;
  __device__ Run(int n) : pages(n) {
    const int chunks = (n + 31) / 32, per = (chunks + kBook / 32 - 1) / (kBook / 32), warp = threadIdx.x >> 5;
    p0 = min(warp * per, chunks) * 32;
    p1 = min((warp + 1) * per, chunks) * 32;
  }
  template <typename F>
  __device__ __forceinline__ void each(const int32_t* refs, F&& f) const {
    const int lane = threadIdx.x & 31;
    for (int q = p0; q < p1; q += 256) {
      int v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = q + 32 * k < p1 && q + 32 * k + lane < pages ? __ldcg(refs + q + 32 * k + lane) : -1;
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (q + 32 * k < p1) f(q + 32 * k, v[k]);
    }
  }
};
// Sum of the warps' n (alike in their lanes) before this warp, and over all.
__device__ __forceinline__ int before_warp(int n, int* total) {
  return __shfl_sync(0xffffffffu, before_me(threadIdx.x & 31 ? 0 : n, total), 0);
}

// One CTA: counts what every slot wants, gives the lowest free pages out in order, marks the moves.
__global__ void __launch_bounds__(kBook, 1) reserve_kernel(const Books c, const Reserve r) {
  __shared__ int copies;
  grid_dependency_wait();
  const int tid = threadIdx.x;
  if (tid == 0) copies = 0;
  const uint32_t below = (1u << (tid & 31)) - 1u;      // lanes before this one
  const Run run(c.pages);
  int free = 0, n_free, n_want;
  run.each(c.refs, [&](int, int refs) { free += __popc(__ballot_sync(0xffffffffu, refs == 0)); });
  // wants, in order of the slots; once one does not fit, none behind it does
  const int run_b = (c.slots + kBook - 1) / kBook;
  const int b0 = min(tid * run_b, c.slots), b1 = min(b0 + run_b, c.slots);
  int wants = 0;
  for (int i = 0; i < run_b; ++i) {
    const int b = b0 + i;
    const Span s = b < b1 ? span_of(c, r, b) : Span{0, 0, 0, true};
    int want = 0;
    bool bad = false;
    entries_of(c, b, s, [&](int32_t* e, int) {
      const int p = *e;
      if (p == -1) return 1;
      if ((unsigned)p >= (unsigned)c.pages) return -1;
      return c.refs[p] > 1 ? 1 : 0;
    }, &want, &bad);
    if (b < b1) {
      if (bad) report(c);
      r.want[b] = s.fits && !bad ? want : -1;
      wants += bad ? 0 : want;
    }
  }
  int at = before_warp(free, &n_free);
  const int at_want = before_me(wants, &n_want);      // all have looked at the counts as they were
  if (at < n_want)
    run.each(c.refs, [&](int q, int refs) {
      const uint32_t bits = __ballot_sync(0xffffffffu, refs == 0);
      if (refs == 0) r.free_list[at + __popc(bits & below)] = q + (tid & 31);
      at += __popc(bits);
    });
  at = at_want;
  for (int i = 0; i < run_b; ++i) {
    const int b = b0 + i, want = b < b1 ? r.want[b] : 0;
    const bool ok = want == 0 || (want > 0 && at + want <= n_free);
    if (b < b1) r.got[b] = ok;
    // entries that this slot alone holds keep their page; a shared one counted above is marked
    int none = 0;
    bool no = false;
    entries_of(c, b, ok && want ? span_of(c, r, b) : Span{0, 0, 0, true}, [&](int32_t* e, int) {
      const int p = *e;
      if (p >= 0 && c.refs[p] > 1) *e = -2 - p;
      return 0;
    }, &none, &no);
    at += max(want, 0);
  }
  __syncthreads();   // marks are set from the counts as they were; now the counts change
  at = at_want;
  for (int i = 0; i < run_b; ++i) {
    const int b = b0 + i, want = b < b1 ? r.want[b] : 0;
    const Span s = want > 0 && at + want <= n_free ? span_of(c, r, b) : Span{0, 0, 0, true};
    // the k-th entry that is missing or marked takes the k-th page of this slot's
    ranked_entries_of(c, b, s, at, [&](int p) { return p < 0; }, [&](int32_t* e, int j, int k, int len) {
      const int p = *e, page = r.free_list[k];
      *e = page;
      c.refs[page] = 1;
      if (p != -1) {
        atomicSub(&c.refs[-2 - p], 1);
        // only the page of the last token so far has anything in it: one copy a slot at most
        if ((int64_t)j * c.P < len) r.copy[atomicAdd(&copies, 1)] = make_int2(-2 - p, page);
      }
    });
    at += max(want, 0);
  }
  __syncthreads();
  if (tid == 0) *r.n_copy = copies;
}

// Copies pages in every layer: moves[k] = (from, to), k < n.  No page is both.
__device__ void copy_pages(const Books& c, const int2* moves, int n) {
  const int pieces = (int)((c.page_bytes + kPiece - 1) / kPiece);
  const int64_t items = (int64_t)n * c.layers * pieces;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int piece = (int)(it % pieces);
    const int64_t rest = it / pieces;
    const int layer = (int)(rest % c.layers);
    const int2 m = moves[rest / c.layers];
    uint8_t* base = c.pool + (int64_t)layer * c.pages * c.page_bytes;
    const uint4* src = reinterpret_cast<const uint4*>(base + m.x * c.page_bytes);
    uint4* dst = reinterpret_cast<uint4*>(base + m.y * c.page_bytes);
    const int lo = piece * (kPiece / 16), hi = min(lo + kPiece / 16, (int)(c.page_bytes / 16));
    uint4 v[kPiece / 16 / kMove];
#pragma unroll
    for (int i = 0; i < kPiece / 16 / kMove; ++i) {
      const int x = lo + threadIdx.x + i * kMove;
      if (x < hi) v[i] = src[x];
    }
#pragma unroll
    for (int i = 0; i < kPiece / 16 / kMove; ++i) {
      const int x = lo + threadIdx.x + i * kMove;
      if (x < hi) dst[x] = v[i];
    }
  }
}

__global__ void __launch_bounds__(kMove) reserve_copy_kernel(const Books c, const Reserve r) {
  grid_dependency_wait();
  copy_pages(c, r.copy, *r.n_copy);
}

// Workspace of compact: live pages and moves, [pages] moves, [pages] new places.
struct Compact {
  int32_t* head;    // live, moves
  int2* moves;      // (from, to)
  int32_t* to;      // by page, from the number of live ones on: where it moves, or -1
  int32_t* live;    // nullable: caller's
};

// One CTA: the i-th hole below the number of live pages takes the i-th live page above it.
__global__ void __launch_bounds__(kBook, 1) compact_kernel(const Books c, const Compact w) {
  grid_dependency_wait();
  const int tid = threadIdx.x;
  const uint32_t below = (1u << (tid & 31)) - 1u;      // lanes before this one
  const Run run(c.pages);
  int mine = 0, live, n;
  run.each(c.refs, [&](int q, int refs) {
    if (refs < 0 && q + (tid & 31) < c.pages) report(c);
    mine += __popc(__ballot_sync(0xffffffffu, refs > 0));
  });
  before_warp(mine, &live);
  auto is_hole = [&](int q, int refs) { return q + (tid & 31) < live && refs <= 0; };
  auto is_mover = [&](int q, int refs) { return q + (tid & 31) >= live && refs > 0; };
  int holes = 0, movers = 0;
  run.each(c.refs, [&](int q, int refs) {
    holes += __popc(__ballot_sync(0xffffffffu, is_hole(q, refs)));
    movers += __popc(__ballot_sync(0xffffffffu, is_mover(q, refs)));
  });
  int at_hole = before_warp(holes, &n), at_mover = before_warp(movers, &n);
  run.each(c.refs, [&](int q, int refs) {
    const uint32_t h = __ballot_sync(0xffffffffu, is_hole(q, refs)), m = __ballot_sync(0xffffffffu, is_mover(q, refs));
    if (is_hole(q, refs)) w.moves[at_hole + __popc(h & below)].y = q + (tid & 31);
    if (is_mover(q, refs)) w.moves[at_mover + __popc(m & below)].x = q + (tid & 31);
    at_hole += __popc(h);
    at_mover += __popc(m);
  });
  for (int p = live + tid; p < c.pages; p += kBook) w.to[p] = -1;
  __syncthreads();
  for (int k = tid; k < n; k += kBook) {
    const int2 m = w.moves[k];
    w.to[m.x] = m.y;
    c.refs[m.y] = c.refs[m.x];
    c.refs[m.x] = 0;
  }
  if (tid == 0) {
    w.head[0] = live;
    w.head[1] = n;
    if (w.live) *w.live = live;
  }
}

__global__ void __launch_bounds__(kMove) compact_move_kernel(const Books c, const Compact w) {
  grid_dependency_wait();
  const int live = w.head[0], n = w.head[1];
  const int64_t entries = (int64_t)c.slots * c.row;
  for (int64_t i = blockIdx.x * (int64_t)kMove + threadIdx.x; i < entries; i += (int64_t)gridDim.x * kMove) {
    const int p = c.table[i];
    if (p < live) continue;
    const int to = p < c.pages ? w.to[p] : -1;
    if (to >= 0) c.table[i] = to;
    else report(c);     // an entry that names no live page
  }
  copy_pages(c, w.moves, n);
}

Books books(const sa_cache& c, int* status) {
  return Books{c.pool, c.table, c.lens, c.refs, c.layers, c.pages, c.page, c.slots, c.row,
               (int64_t)sa_cache_page_bytes(&c), status};
}
size_t up16(size_t n) { return (n + 15) / 16 * 16; }
constexpr int kMoveCtas = 148 * 8;

}  // namespace

size_t cache_books_ws_bytes(const sa_cache& c) {
  const size_t reserve = 16 + up16(4 * (size_t)c.slots) + up16(8 * (size_t)c.slots) + up16(4 * (size_t)c.pages);
  const size_t compact = 16 + up16(8 * (size_t)c.pages) + up16(4 * (size_t)c.pages);
  return reserve > compact ? reserve : compact;
}

cudaError_t launch_cache_free(const sa_cache& c, int n, const int32_t* slots, int* status,
                              cudaStream_t st) {
  bump_launches();
  return launch_dependent(free_kernel, dim3(n), dim3(128), 0, st, books(c, status), n, slots);
}

cudaError_t launch_cache_fork(const sa_cache& c, int n, const int32_t* parents,
                              const int32_t* children, int* status, cudaStream_t st) {
  bump_launches();
  return launch_dependent(fork_kernel, dim3(n), dim3(128), 0, st, books(c, status), n, parents, children);
}

cudaError_t launch_cache_reserve(const sa_cache& c, const int32_t* add, int32_t* got, void* ws,
                                 int* status, cudaStream_t st) {
  const Books b = books(c, status);
  uint8_t* at = (uint8_t*)ws;
  Reserve r{add, got, (int32_t*)at, (int32_t*)(at + 16), nullptr, nullptr};
  at += 16 + up16(4 * (size_t)c.slots);
  r.copy = (int2*)at;
  r.free_list = (int32_t*)(at + up16(8 * (size_t)c.slots));
  bump_launches();
  const cudaError_t e = launch_dependent(reserve_kernel, dim3(1), dim3(kBook), 0, st, b, r);
  if (e != cudaSuccess) return e;
  bump_launches();
  return launch_dependent(reserve_copy_kernel, dim3(kMoveCtas), dim3(kMove), 0, st, b, r);
}

cudaError_t launch_cache_compact(const sa_cache& c, int32_t* live, void* ws, int* status,
                                 cudaStream_t st) {
  const Books b = books(c, status);
  uint8_t* at = (uint8_t*)ws;
  Compact w{(int32_t*)at, (int2*)(at + 16), nullptr, live};
  w.to = (int32_t*)(at + 16 + up16(8 * (size_t)c.pages));
  bump_launches();
  const cudaError_t e = launch_dependent(compact_kernel, dim3(1), dim3(kBook), 0, st, b, w);
  if (e != cudaSuccess) return e;
  bump_launches();
  return launch_dependent(compact_move_kernel, dim3(kMoveCtas), dim3(kMove), 0, st, b, w);
}

}  // namespace sa

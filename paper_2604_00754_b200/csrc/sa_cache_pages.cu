// The books of the 4-bit cache: who holds which pages, and the moves of pages that follow.
//
// Everything is decided on the device from the state before the call, in the order of slots, list
// entries and pages, so a captured call does the same as an eager one and no result depends on
// timing (counts are integers: the order of their atomics is free).
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

// A thread's run of pages, looked at 32 at a time: bit i of a look is test(refs[q + i]), and the looks of runs up to
// 32 pages are remembered.
struct Run {
  int p0, p1;
  __device__ Run(int pages) {
    const int run = (pages + kBook - 1) / kBook;
    p0 = min((int)threadIdx.x * run, pages);
    p1 = min(p0 + run, pages);
  }
  template <typename F>
  __device__ uint32_t look(const int32_t* refs, int q, F&& test) const {
    uint32_t bits = 0;
    for (int i = 0; i < 32 && q + i < p1; i += 8)
#pragma unroll
      for (int k = i; k < i + 8; ++k)
        if (q + k < p1 && test(__ldcg(refs + q + k))) bits |= 1u << k;
    return bits;
  }
  __device__ bool one_look() const { return p1 - p0 <= 32; }
};

// One CTA: counts what every slot wants, gives the lowest free pages out in order, marks the moves.
__global__ void __launch_bounds__(kBook, 1) reserve_kernel(const Books c, const Reserve r) {
  __shared__ int copies;
  grid_dependency_wait();
  const int tid = threadIdx.x;
  if (tid == 0) copies = 0;
  auto is_free = [](int refs) { return refs == 0; };
  const Run run(c.pages);
  const uint32_t first = run.look(c.refs, run.p0, is_free);
  int free = __popc(first), n_free, n_want;
  for (int q = run.p0 + 32; q < run.p1; q += 32) free += __popc(run.look(c.refs, q, is_free));
  // wants, in order of the slots; once one does not fit, none behind it does
  const int run_b = (c.slots + kBook - 1) / kBook;
  const int b0 = min(tid * run_b, c.slots), b1 = min(b0 + run_b, c.slots);
  int wants = 0;
  for (int b = b0; b < b1; ++b) {
    const Span s = span_of(c, r, b);
    const int32_t* row = c.table + (int64_t)b * c.row;
    int want = 0;
    bool bad = false;
    for (int j = s.lo; j < s.hi; ++j) {
      const int p = row[j];
      if (p == -1) ++want;
      else if ((unsigned)p >= (unsigned)c.pages) bad = true;
      else want += c.refs[p] > 1;
    }
    if (bad) report(c);
    r.want[b] = s.fits && !bad ? want : -1;
    wants += bad ? 0 : want;
  }
  int at = before_me(free, &n_free);
  const int at_want = before_me(wants, &n_want);      // all have looked at the counts as they were
  if (n_want > 0)
    for (int q = run.p0; q < run.p1; q += 32)
      for (uint32_t bits = run.one_look() ? first : run.look(c.refs, q, is_free); bits; bits &= bits - 1)
        r.free_list[at++] = q + __ffs(bits) - 1;
  at = at_want;
  for (int b = b0; b < b1; ++b) {
    const int want = r.want[b];
    const bool ok = want == 0 || (want > 0 && at + want <= n_free);
    r.got[b] = ok;
    if (ok && want) {
      const Span s = span_of(c, r, b);
      int32_t* row = c.table + (int64_t)b * c.row;
      // entries that this slot alone holds keep their page; a shared one counted above is marked
      for (int j = s.lo; j < s.hi; ++j) {
        const int p = row[j];
        if (p >= 0 && c.refs[p] > 1) row[j] = -2 - p;
      }
    }
    at += max(want, 0);
  }
  __syncthreads();   // marks are set from the counts as they were; now the counts change
  at = at_want;
  for (int b = b0; b < b1; ++b) {
    const int want = r.want[b];
    if (want > 0 && at + want <= n_free) {
      const Span s = span_of(c, r, b);
      int32_t* row = c.table + (int64_t)b * c.row;
      int k = at;
      for (int j = s.lo; j < s.hi; ++j) {
        const int p = row[j];
        if (p >= 0) continue;
        const int page = r.free_list[k++];
        row[j] = page;
        c.refs[page] = 1;
        if (p != -1) {
          atomicSub(&c.refs[-2 - p], 1);
          // only the page of the last token so far has anything in it: one copy a slot at most
          if ((int64_t)j * c.P < s.len) r.copy[atomicAdd(&copies, 1)] = make_int2(-2 - p, page);
        }
      }
    }
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
  auto is_held = [&](int refs) {
    if (refs < 0) report(c);
    return refs > 0;
  };
  const Run run(c.pages);
  const uint32_t first = run.look(c.refs, run.p0, is_held);
  int mine = __popc(first), live, n;
  for (int q = run.p0 + 32; q < run.p1; q += 32) mine += __popc(run.look(c.refs, q, is_held));
  before_me(mine, &live);
  // of pages q .. q + 31 of the run: those below `live`, those in the run
  auto upto = [](int count) { return count >= 32 ? ~0u : count <= 0 ? 0u : (1u << count) - 1u; };
  auto holes_of = [&](uint32_t held, int q) { return ~held & upto(run.p1 - q) & upto(live - q); };
  auto movers_of = [&](uint32_t held, int q) { return held & ~upto(live - q); };
  int holes = 0, movers = 0;
  for (int q = run.p0; q < run.p1; q += 32) {
    const uint32_t held = run.one_look() ? first : run.look(c.refs, q, is_held);
    holes += __popc(holes_of(held, q));
    movers += __popc(movers_of(held, q));
  }
  int at_hole = before_me(holes, &n), at_mover = before_me(movers, &n);
  for (int q = run.p0; q < run.p1; q += 32) {
    const uint32_t held = run.one_look() ? first : run.look(c.refs, q, is_held);
    for (uint32_t bits = holes_of(held, q); bits; bits &= bits - 1) w.moves[at_hole++].y = q + __ffs(bits) - 1;
    for (uint32_t bits = movers_of(held, q); bits; bits &= bits - 1) w.moves[at_mover++].x = q + __ffs(bits) - 1;
  }
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

// What the attention kernels over the 4-bit cache share: how the work is cut, and what a share leaves.
//
// The query rows of a KV head (its G query heads times the T new tokens) are cut into tiles of
// `rows`; an entry is a sequence and a row tile, a segment an entry and a KV head, a step 64 of its
// keys.  All steps stand in one line, segment after segment, each with kOpen more in front for what it costs
// to begin and to join one, and each CTA takes an equal share of the line, whatever the lengths are: the
// lengths are known to the device alone, and a batch of uneven ones fills the GPU as an even one does.  A segment that lies within one share is finished there; of one that
// does not, each share leaves maximum, sum and unnormalised rows in the workspace, and the second launch
// joins them in the order of the shares (so results do not depend on timing).
#pragma once

#include "sa_cache.cuh"

namespace sa {
namespace attend {

constexpr int kStep = 64;      // keys per step
constexpr int kUnit = 16;      // keys a warp takes of a step; pages hold a multiple of it
constexpr int kWarps = 4;
// Beginning and joining a segment, in steps.  64 sequences of 0 .. 8191 keys, 32/8 heads of 128: 106 us with 0, 96
// with 2, 92 with 3, 85 with 5, 84 with 8; one of 131072 keys, 32/4 heads: 31.5, 30.9, 31.4, 29.9, 34.4.
constexpr int kOpen = 5;

// A split segment: the share that begins it and how many have a part of it (0: none is split).  Filed by
// segment where the segments are no more than the shares, else by the share that begins it.
struct Split {
  int e, h, share, parts;
};

struct Params {
  AttendArgs a;
  int G, rows, tiles, entries;  // query heads per KV head, rows of a tile, tiles of a sequence, all entries
  int shares;                   // CTAs of the launch
  bool by_segment;              // how splits are filed
  bool few;                     // no line of steps that the table allows passes 31 bits
  float* part;                  // [shares][2][rows * (d + 2)]: a share's first and last segment
  Split* split;                 // [shares], or as many as there are segments
  float scale2;                 // scores times log2(e), K's power of two folded in
};

// Keys [lo, hi) that the rows of an entry may see, in steps [first, first + n); n = 0: no rows.
struct Entry {
  int b, slot, len, r0, rows, t0, t1, lo, hi, first, n;   // t0 .. t1: the rows' tokens
  __device__ int span() const { return n ? n + kOpen : 0; }   // of a segment in the line
};

__device__ inline Entry entry(const Params& p, int e) {
  const AttendArgs& a = p.a;
  Entry r{};
  r.b = p.tiles == 1 ? e : e / p.tiles;
  r.r0 = (e - r.b * p.tiles) * p.rows;
  const int count = cache_count(a.c, a.counts, r.b, a.T);
  if (count <= 0 || r.r0 >= p.G * count) return r;
  r.slot = cache_slot(a.c, a.slots, r.b);
  if (r.slot < 0) return r;
  r.len = a.c.lens[r.slot];
  const int64_t most = (int64_t)a.c.row * a.c.P;
  if (r.len < 0 || r.len > most) {
    report_cache(a.c);
    return r;
  }
  r.rows = min(p.rows, p.G * count - r.r0);
  r.t0 = a.T == 1 ? 0 : r.r0 / p.G;
  r.t1 = a.T == 1 ? 0 : (r.r0 + r.rows - 1) / p.G;
  int64_t hi = a.causal ? (int64_t)r.len + r.t1 + 1 : r.len;
  if (hi > most) {
    report_cache(a.c);
    hi = most;
  }
  r.hi = (int)hi;
  r.lo = a.w > 0 ? min((int)max((int64_t)r.len + r.t0 - a.w + 1, (int64_t)0), r.hi) : 0;
  r.first = r.lo / kStep;
  r.n = max((r.hi + kStep - 1) / kStep - r.first, 1);   // one step at least: empty rows are written too
  return r;
}

__device__ inline int64_t quotient(int64_t a, int64_t b) {   // of positive numbers, mostly small ones
  return (a | b) >> 31 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

// Where the line of steps is cut: every share takes `per` steps, the first `extra` one more.
struct Line {
  int64_t total, per;
  int shares, extra;
  __device__ int64_t begin(int i) const { return i * per + min(i, extra); }
  __device__ int of(int64_t s) const {      // the share that holds step s
    const int64_t longer = extra * (per + 1);
    return (int)(s < longer ? quotient(s, per + 1) : extra + quotient(s - longer, per));
  }
};

// The line, and the entry that holds the first step of share `blockIdx.x` with the steps before that
// entry (-1: no such share).  Each of 32 lanes, in every warp alike, or of all threads adds up a run of entries;
// one scan of the runs' sums.  All threads call it.
template <typename N, bool kWarp>
__device__ __forceinline__ Line find_in(const Params& p, int* e_out, int64_t* before_out) {
  __shared__ N sums[kWarps];
  __shared__ N found_before;
  __shared__ int found;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int id = kWarp ? lane : threadIdx.x, ids = kWarp ? 32 : 32 * kWarps;
  const int run = p.entries <= ids ? 1 : (p.entries + ids - 1) / ids;
  const int e0 = min(id * run, p.entries), e1 = min(e0 + run, p.entries);
  N mine = 0;
  for (int e = e0; e < e1; ++e) mine += entry(p, e).span();
  mine *= p.a.c.Hkv;
  N upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const N v = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += v;
  }
  Line line{};
  if (kWarp) {
    line.total = __shfl_sync(0xffffffffu, upto, 31);
  } else {
    if (lane == 31) sums[warp] = upto;
    if (threadIdx.x == 0) found = -1;
    __syncthreads();
    for (int i = 0; i < kWarps; ++i) {
      if (i < warp) upto += sums[i];
      line.total += sums[i];
    }
  }
  line.shares = (int)min((int64_t)p.shares, line.total);
  int e = -1;
  N at = upto - mine;
  if ((int)blockIdx.x < line.shares) {
    line.per = quotient(line.total, line.shares);
    line.extra = (int)(line.total - line.per * line.shares);
    const N s = (N)line.begin(blockIdx.x);
    if (s >= at && s < upto) {
      e = e0;
      while (run > 1) {
        const N n = (N)entry(p, e).span() * p.a.c.Hkv;
        if (s < at + n) break;
        at += n;
        ++e;
      }
    }
  }
  if (kWarp) {
    const int from = max(__ffs(__ballot_sync(0xffffffffu, e >= 0)) - 1, 0);
    *e_out = __shfl_sync(0xffffffffu, e, from);
    *before_out = __shfl_sync(0xffffffffu, at, from);
  } else {
    if (e >= 0) {
      found = e;
      found_before = at;
    }
    __syncthreads();
    *e_out = found;
    *before_out = found_before;
  }
  return line;
}
__device__ __forceinline__ Line find(const Params& p, int* e_out, int64_t* before_out) {
  if (p.few && p.entries <= 128) return find_in<int32_t, true>(p, e_out, before_out);   // no barrier
  return find_in<int64_t, false>(p, e_out, before_out);
}

// A share's way along the line: the portions of segments that it takes.
struct Walk {
  int64_t s, end, before, seg;   // next step, end of the share, steps before entry e, begin of the segment
  int e, h, k0, k1;              // entry, KV head, the segment's steps [k0, k1) that are this share's
  Entry en;
};
__device__ __forceinline__ bool start(const Params& p, const Line& line, int e, int64_t before, Walk* w) {
  if (e < 0) return false;
  w->s = line.begin(blockIdx.x);
  w->end = line.begin(blockIdx.x + 1);
  w->before = before;
  w->e = e;
  w->en = entry(p, e);
  return true;
}
// The next portion; false: none is left.
__device__ __forceinline__ bool next(const Params& p, Walk* w) {
  const int heads = p.a.c.Hkv;
  while (w->s < w->end) {
    while (w->en.n == 0 || w->s >= w->before + (int64_t)w->en.span() * heads) {
      w->before += (int64_t)w->en.span() * heads;
      w->en = entry(p, ++w->e);
    }
    const int span = w->en.span();
    w->h = (int)quotient(w->s - w->before, span);
    w->seg = w->before + (int64_t)w->h * span;
    const int x0 = (int)(w->s - w->seg), x1 = (int)min((int64_t)span, w->end - w->seg);
    w->k0 = max(x0 - kOpen, 0);
    w->k1 = max(x1 - kOpen, 0);
    w->s = w->seg + x1;
    if (w->k1 > w->k0) return true;
  }
  return false;
}

// One row of the result: o over its sum, and the log-sum-exp; m in log2 units, the sum relative to it.
__device__ __forceinline__ float row_lse(float m, float l) {
  return l > 0.f || l != l ? (m + log2f(l)) * kLn2 : -INFINITY;
}
__device__ __forceinline__ float row_scale(float l, float v_scale) {
  return l > 0.f || l != l ? __fdiv_rn(v_scale, l) : 0.f;
}

template <typename T>
__device__ __forceinline__ T* row_of(const Params& p, T* base, const int64_t (&s)[3], const Entry& en, int h, int r) {
  const int t = (en.r0 + r) / p.G, g = (en.r0 + r) - t * p.G;
  return base + en.b * s[0] + (int64_t)(h * p.G + g) * s[1] + (int64_t)t * s[2];
}
__device__ __forceinline__ float* lse_of(const Params& p, const Entry& en, int h, int r) {
  const int t = (en.r0 + r) / p.G, g = (en.r0 + r) - t * p.G;
  return p.a.lse + ((int64_t)en.b * p.a.Hq + h * p.G + g) * p.a.T + t;
}

// Files what became of the portion's segment, if this share begins it.  Without `by_segment` a share's last one
// counts: of the segments that it begins, only that can go on in the next.
__device__ __forceinline__ bool file_split(const Params& p, const Line& line, const Walk& w) {
  if (w.k0 != 0) return false;
  const int parts = w.k1 == w.en.n ? 0 : line.of(w.seg + w.en.span() - 1) - (int)blockIdx.x + 1;
  if (threadIdx.x == 0)
    p.split[p.by_segment ? w.e * p.a.c.Hkv + w.h : (int)blockIdx.x] = Split{w.e, w.h, (int)blockIdx.x, parts};
  return true;
}
__device__ __forceinline__ void file_nothing(const Params& p) {      // this share begins no segment
  if (!p.by_segment && threadIdx.x == 0) p.split[blockIdx.x] = Split{0, 0, 0, 0};
}

// Where a share's part of a segment goes: `last` where the share begins the segment.
__device__ __forceinline__ float* part_of(const Params& p, int share, bool last) {
  return p.part + ((int64_t)share * 2 + last) * p.rows * (p.a.c.d + 2);
}

// Bytes of the workspace, and its carving.
inline size_t ws_bytes(int shares, int rows, int d) {
  return (size_t)shares * (2 * (size_t)rows * (d + 2) * 4 + sizeof(Split));
}
inline Params params(const AttendArgs& a, int shares, int rows) {
  Params p{};
  p.a = a;
  p.G = a.Hq / a.c.Hkv;
  p.rows = rows;
  p.tiles = (p.G * a.T + rows - 1) / rows;
  p.entries = a.B * p.tiles;
  p.shares = shares;
  p.by_segment = (int64_t)p.entries * a.c.Hkv <= shares;
  p.few = (double)p.entries * a.c.Hkv * ((double)a.c.row * a.c.P / kStep + 2 + kOpen) < 2e9;
  p.split = (Split*)a.ws;
  p.part = (float*)(p.split + shares);
  p.scale2 = a.scale * kLog2e * a.c.k_scale;
  return p;
}

}  // namespace attend

// Shares and rows of a tile for a call; the launch that attends, and the second, which joins what the shares left.
void cache_attend_shape(int T, int G, int d, int dtype, int* shares, int* rows);
cudaError_t launch_cache_attend_tiles(const attend::Params& p, int dtype, cudaStream_t st);

}  // namespace sa

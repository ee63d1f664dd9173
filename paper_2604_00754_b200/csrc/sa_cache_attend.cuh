// What the attention kernels over the 4-bit cache share: how the work is cut, and what a share leaves.
//
// The query rows of a KV head (its G query heads times the T new tokens) are cut into tiles of
// `rows`; an entry is a sequence and a row tile, a segment an entry and a KV head, a step 64 of its
// keys.  All steps stand in one line, segment after segment, and each CTA takes an equal share of it,
// whatever the lengths are: the lengths are known to the device alone, and a batch of uneven ones fills
// the GPU as an even one does.  A segment that lies within one share is finished there; of one that
// does not, each share leaves maximum, sum and unnormalised rows in the workspace, and the second launch
// joins them in the order of the shares (so results do not depend on timing).
#pragma once

#include "sa_cache.cuh"

namespace sa {
namespace attend {

constexpr int kStep = 64;      // keys per step
constexpr int kUnit = 16;      // keys a warp takes of a step; pages hold a multiple of it
constexpr int kWarps = 4;

// A split segment, filed under the share that begins it.
struct Split {
  int e, h, parts, pad;
};

struct Params {
  AttendArgs a;
  int G, rows, tiles, entries;  // query heads per KV head, rows of a tile, tiles of a sequence, all entries
  int shares;                   // CTAs of the launch
  float* part;                  // [shares][2][rows * (d + 2)]: a share's first and last segment
  Split* split;                 // [shares]
  float scale2;                 // scores times log2(e), K's power of two folded in
};

// Keys [lo, hi) that the rows of an entry may see, in steps [first, first + n); n = 0: no rows.
struct Entry {
  int b, slot, len, r0, rows, lo, hi, first, n;
};

__device__ inline Entry entry(const Params& p, int e) {
  const AttendArgs& a = p.a;
  Entry r{};
  r.b = e / p.tiles;
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
  const int t0 = r.r0 / p.G, t1 = (r.r0 + r.rows - 1) / p.G;
  int64_t hi = a.causal ? (int64_t)r.len + t1 + 1 : r.len;
  if (hi > most) {
    report_cache(a.c);
    hi = most;
  }
  r.hi = (int)hi;
  r.lo = a.w > 0 ? min((int)max((int64_t)r.len + t0 - a.w + 1, (int64_t)0), r.hi) : 0;
  r.first = r.lo / kStep;
  r.n = max((r.hi + kStep - 1) / kStep - r.first, 1);   // one step at least: empty rows are written too
  return r;
}

// Where the line of steps is cut: share i takes [total * i / shares, total * (i + 1) / shares).
struct Line {
  int64_t total;
  int shares;
  __device__ int64_t begin(int i) const { return total * i / shares; }
  // the share that holds step s
  __device__ int of(int64_t s) const { return (int)(((s + 1) * shares - 1) / total); }
};

// The line, and the entry that holds the first step of share `blockIdx.x` with the steps before that
// entry.  Each thread adds up a run of entries; one scan of the runs' sums.  All threads call it.
__device__ inline Line find(const Params& p, int* e_out, int64_t* before_out) {
  __shared__ int64_t sums[kWarps];
  __shared__ int64_t found_before;
  __shared__ int found;
  const int tid = threadIdx.x, threads = 32 * kWarps;
  const int run = (p.entries + threads - 1) / threads;
  const int e0 = min(tid * run, p.entries), e1 = min(e0 + run, p.entries);
  int64_t mine = 0;
  for (int e = e0; e < e1; ++e) mine += entry(p, e).n;
  mine *= p.a.c.Hkv;
  int64_t upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t v = __shfl_up_sync(0xffffffffu, upto, o);
    if ((tid & 31) >= o) upto += v;
  }
  if ((tid & 31) == 31) sums[tid >> 5] = upto;
  if (tid == 0) found = -1;
  __syncthreads();
  Line line{0, 1};
  for (int i = 0; i < kWarps; ++i) {
    if (i < (tid >> 5)) upto += sums[i];
    line.total += sums[i];
  }
  line.shares = (int)min((int64_t)p.shares, line.total);
  if ((int)blockIdx.x < line.shares) {
    const int64_t s = line.begin(blockIdx.x);
    int64_t at = upto - mine;
    if (s >= at && s < upto)
      for (int e = e0; e < e1; ++e) {
        const int64_t n = (int64_t)entry(p, e).n * p.a.c.Hkv;
        if (s < at + n) {
          found = e;
          found_before = at;
          break;
        }
        at += n;
      }
  }
  __syncthreads();
  *e_out = found;
  *before_out = found_before;
  return line;
}

// One row of the result: o over its sum, and the log-sum-exp; m in log2 units, the sum relative to it.
__device__ __forceinline__ float row_lse(float m, float l) {
  return l > 0.f || l != l ? (m + log2f(l)) * kLn2 : -INFINITY;
}
__device__ __forceinline__ float row_scale(float l, float v_scale) {
  return l > 0.f || l != l ? v_scale / l : 0.f;
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
  p.split = (Split*)a.ws;
  p.part = (float*)(p.split + shares);
  p.scale2 = a.scale * kLog2e * a.c.k_scale;
  return p;
}

}  // namespace attend

// The second launch: joins what the shares left.
cudaError_t launch_cache_join(const attend::Params& p, int dtype, cudaStream_t st);
// The tensor-core kernels: whether they take the head dimension, their shape for a call, the call.
bool cache_attend_mma_takes(int d);
void cache_attend_mma_shape(int T, int G, int d, int dtype, int* shares, int* rows);
cudaError_t launch_cache_attend_mma(const attend::Params& p, int dtype, cudaStream_t st);

}  // namespace sa

// Attention of a sequence's newest tokens over its 4-bit cache.
//
// The query rows of a KV head (its G query heads times the T new tokens) are cut into tiles of kRows;
// an entry is a sequence and a row tile, a segment an entry and a KV head, a step 64 of its keys.
// All steps stand in one line, segment after segment, and each CTA takes an equal share of it,
// whatever the lengths are: the lengths are known to the device alone, and a batch of uneven ones fills
// the GPU as an even one does.  A segment that lies within one share is finished there; of one that
// does not, each share leaves maximum, sum and unnormalised rows in the workspace, and the second launch
// joins them in the order of the shares (so results do not depend on timing).
//
// This kernel takes any head dimension and computes on the CUDA cores in fp32.
#include <algorithm>

#include "sa_cache.cuh"

namespace sa {
namespace {

constexpr int kStep = 64;      // keys per step
constexpr int kUnit = 16;      // keys a warp takes of a step; pages hold a multiple of it
constexpr int kWarps = 4;
constexpr int kRows = 8;       // query rows of a tile
constexpr int kShares = 4 * 148;  // CTAs: four per SM

// A split segment, filed under the share that begins it.
struct Split {
  int e, h, parts, pad;
};

struct Params {
  AttendArgs a;
  int G, tiles, entries;  // query heads per KV head, row tiles of a sequence, all entries
  float* part;            // [kShares][2][kRows * (d + 2)]: a share's first and last segment
  Split* split;           // [kShares]
  float scale2;           // scores times log2(e), K's power of two folded in
};

// Keys [lo, hi) that the rows of an entry may see, in steps [first, first + n); n = 0: no rows.
struct Entry {
  int b, slot, len, r0, rows, lo, hi, first, n;
};

__device__ Entry entry(const Params& p, int e) {
  const AttendArgs& a = p.a;
  Entry r{};
  r.b = e / p.tiles;
  r.r0 = (e - r.b * p.tiles) * kRows;
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
  r.rows = min(kRows, p.G * count - r.r0);
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
__device__ Line find(const Params& p, int* e_out, int64_t* before_out) {
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
  line.shares = (int)min((int64_t)kShares, line.total);
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
__global__ void __launch_bounds__(32 * kWarps) attend_kernel(const Params p) {
  extern __shared__ float smem[];
  const AttendArgs& a = p.a;
  const CacheView& c = a.c;
  const int d = c.d, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  float* q_s = smem;                            // [kRows][d]
  float* p_s = q_s + kRows * d;                 // [kWarps][kUnit][kRows]
  float* o_s = p_s + kWarps * kUnit * kRows;    // [kWarps][kRows][d]
  float* ml_s = o_s + kWarps * kRows * d;       // [kWarps][2][kRows]
  grid_dependency_wait();
  grid_dependents_launch();
  int e;
  int64_t before;
  const Line line = find(p, &e, &before);
  if (e < 0) {
    if (tid == 0) p.split[blockIdx.x] = Split{0, 0, 0, 0};
    return;
  }
  int64_t s = line.begin(blockIdx.x);
  const int64_t end = line.begin(blockIdx.x + 1);
  Split mine{0, 0, 0, 0};
  bool first = true;
  Entry en = entry(p, e);
  while (s < end) {
    while (en.n == 0 || s >= before + (int64_t)en.n * c.Hkv) {
      before += (int64_t)en.n * c.Hkv;
      en = entry(p, ++e);
    }
    const int h = (int)((s - before) / en.n);
    const int64_t seg = before + (int64_t)h * en.n;
    const int k0 = (int)(s - seg), k1 = (int)min((int64_t)en.n, end - seg);
    __syncthreads();
    for (int i = tid; i < kRows * d; i += 32 * kWarps) {
      const int r = i / d, x = i - r * d;
      float v = 0.f;
      if (r < en.rows) {
        const int t = (en.r0 + r) / p.G, g = (en.r0 + r) - t * p.G;
        v = to_f32(reinterpret_cast<const T*>(a.q)[en.b * a.qs[0] + (int64_t)(h * p.G + g) * a.qs[1] +
                                                   (int64_t)t * a.qs[2] + x]);
      }
      q_s[i] = v;
    }
    __syncthreads();
    // lanes: key lane / 2, half lane % 2 of its dimensions for the scores; for the sums word lane % words of
    // a key's codes, of every apart-th key
    float m[kRows], l[kRows], o[8][kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      m[r] = -INFINITY;
      l[r] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i][r] = 0.f;
    }
    const int words = d / 8, apart = 32 / words, word = lane % words;
    const int key0 = lane < apart * words ? lane / words : kUnit;   // lanes left over have no key
    for (int k = k0; k < k1; ++k) {
      const int unit = (en.first + k) * kStep + warp * kUnit;
      if (unit >= en.hi || unit + kUnit <= en.lo) continue;
      const int page = cache_page(c, en.slot, unit);
      if (page < 0) continue;
      const int row = unit % c.P;
      const uint8_t* kb = cache_side(c, page, h, 0);
      const uint8_t* vb = cache_side(c, page, h, 1);
      const int j = unit + lane / 2;
      float x[kRows];
#pragma unroll
      for (int r = 0; r < kRows; ++r) x[r] = 0.f;
      const bool here = j >= en.lo && j < en.hi;
      if (here) {
        const uint8_t* codes = kb + (row + lane / 2) * (d / 2);
        const uint8_t* scales = kb + c.P * (d / 2) + (row + lane / 2) * (d / 16);
        for (int i = (lane & 1) * 8; i < d; i += 16) {
          const float f = scale_to_f32(scales[i / 16]);
          uint32_t hv[4];
          codes_to_half2(*reinterpret_cast<const uint32_t*>(codes + i / 2), hv);
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&hv[z]));
#pragma unroll
            for (int r = 0; r < kRows; ++r)
              x[r] += v.x * f * q_s[r * d + i + 2 * z] + v.y * f * q_s[r * d + i + 2 * z + 1];
          }
        }
      }
      float* ps = p_s + warp * kUnit * kRows;
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        x[r] += __shfl_xor_sync(0xffffffffu, x[r], 1);
        const int pos = en.len + (en.r0 + r) / p.G;
        const bool sees = here && r < en.rows && (!a.causal || j <= pos) &&
                          (a.w <= 0 || pos - j < a.w);
        x[r] = sees ? x[r] * p.scale2 : -INFINITY;
        float top = x[r];
#pragma unroll
        for (int z = 2; z < 32; z <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, z));
        const float to = fmaxf(m[r], top);
        const float ref = to == -INFINITY ? 0.f : to;
        const float keep = exp2f(m[r] - ref);
        m[r] = to;
        const float pr = sees ? exp2f(x[r] - ref) : 0.f;
        l[r] = l[r] * keep + ((lane & 1) ? 0.f : pr);
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i][r] *= keep;
        if (!(lane & 1)) ps[lane / 2 * kRows + r] = pr;
      }
      __syncwarp();
      for (int u = key0; u < kUnit; u += apart) {
        if (unit + u < en.lo || unit + u >= en.hi) continue;   // what no row sees is not touched
        const uint8_t* codes = vb + (row + u) * (d / 2);
        const float f = scale_to_f32(vb[c.P * (d / 2) + (row + u) * (d / 16) + word / 2]);
        uint32_t hv[4];
        codes_to_half2(reinterpret_cast<const uint32_t*>(codes)[word], hv);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
          const float pr = ps[u * kRows + r];
          if (pr == 0.f) continue;       // a NaN behind a mask stays there
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&hv[z]));
            o[2 * z][r] += pr * (v.x * f);
            o[2 * z + 1][r] += pr * (v.y * f);
          }
        }
      }
      __syncwarp();
    }
    // the warps' parts join, in their order
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const float sum = warp_sum(l[r]);
      if (lane == 0) {
        ml_s[warp * 2 * kRows + r] = m[r];
        ml_s[warp * 2 * kRows + kRows + r] = sum;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float v = o[i][r];
        for (int g = 1; g < apart; ++g) v += __shfl_sync(0xffffffffu, o[i][r], (lane + g * words) & 31);
        if (lane < words) o_s[(warp * kRows + r) * d + 8 * lane + i] = v;
      }
    }
    __syncthreads();
    const bool whole = k0 == 0 && k1 == en.n;
    float* part = p.part + ((int64_t)blockIdx.x * 2 + (first ? 0 : 1)) * kRows * (d + 2);
    if (!whole && k0 == 0) {
      // filed by the share that begins it; the others' parts are their first segments
      part = p.part + ((int64_t)blockIdx.x * 2 + 1) * kRows * (d + 2);
      mine = Split{e, h, line.of(seg + en.n - 1) - (int)blockIdx.x + 1, 0};
    }
    for (int i = tid; i < en.rows * d; i += 32 * kWarps) {
      const int r = i / d, x = i - r * d;
      float to = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) to = fmaxf(to, ml_s[w * 2 * kRows + r]);
      const float ref = to == -INFINITY ? 0.f : to;
      float sum = 0.f, v = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float keep = exp2f(ml_s[w * 2 * kRows + r] - ref);
        sum += keep * ml_s[w * 2 * kRows + kRows + r];
        v += keep * o_s[(w * kRows + r) * d + x];
      }
      if (whole) {
        const int t = (en.r0 + r) / p.G, g = (en.r0 + r) - t * p.G, hq = h * p.G + g;
        reinterpret_cast<T*>(a.y)[en.b * a.ys[0] + hq * a.ys[1] + (int64_t)t * a.ys[2] + x] =
            from_f32<T>(v * row_scale(sum, c.v_scale));
        if (x == 0 && a.lse) a.lse[((int64_t)en.b * a.Hq + hq) * a.T + t] = row_lse(to, sum);
      } else {
        part[r * d + x] = v;
        if (x == 0) {
          part[kRows * d + r] = to;
          part[kRows * (d + 1) + r] = sum;
        }
      }
    }
    s = seg + k1;
    first = false;
  }
  if (tid == 0) p.split[blockIdx.x] = mine;
}

// Joins the parts of the segment that share blockIdx.x began: one row per blockIdx.y.
template <typename T>
__global__ void __launch_bounds__(32 * kWarps) join_kernel(const Params p) {
  extern __shared__ float smem[];
  const AttendArgs& a = p.a;
  const int d = a.c.d, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = blockIdx.y;
  grid_dependency_wait();
  const Split sp = p.split[blockIdx.x];
  if (sp.parts == 0) return;
  const Entry en = entry(p, sp.e);
  if (r >= en.rows) return;
  const int stride = kRows * (d + 2);
  auto part = [&](int i) {
    return p.part + ((int64_t)(blockIdx.x + i) * 2 + (i == 0 ? 1 : 0)) * stride;
  };
  float to = -INFINITY;
  for (int i = tid; i < sp.parts; i += 32 * kWarps) to = fmaxf(to, part(i)[kRows * d + r]);
  __shared__ float tops[kWarps];
  to = warp_max(to);
  if (lane == 0) tops[warp] = to;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps; ++w) to = fmaxf(to, tops[w]);
  const float ref = to == -INFINITY ? 0.f : to;
  // warp w adds up parts w, w + 4, ...; then the warps' sums in their order
  float v[8] = {}, sum = 0.f;
  for (int i = warp; i < sp.parts; i += kWarps) {
    const float* f = part(i);
    const float keep = exp2f(f[kRows * d + r] - ref);
    sum += keep * f[kRows * (d + 1) + r];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (lane + 32 * j < d) v[j] += keep * f[r * d + lane + 32 * j];
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (lane + 32 * j < d) smem[warp * (d + 1) + lane + 32 * j] = v[j];
  if (lane == 0) smem[warp * (d + 1) + d] = sum;
  __syncthreads();
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) sum += smem[w * (d + 1) + d];
  const int t = (en.r0 + r) / p.G, g = (en.r0 + r) - t * p.G, hq = sp.h * p.G + g;
  for (int x = tid; x < d; x += 32 * kWarps) {
    float o = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) o += smem[w * (d + 1) + x];
    reinterpret_cast<T*>(a.y)[en.b * a.ys[0] + hq * a.ys[1] + (int64_t)t * a.ys[2] + x] =
        from_f32<T>(o * row_scale(sum, a.c.v_scale));
  }
  if (tid == 0 && a.lse) a.lse[((int64_t)en.b * a.Hq + hq) * a.T + t] = row_lse(to, sum);
}

template <typename T>
cudaError_t launch(const Params& p, cudaStream_t st) {
  const int d = p.a.c.d;
  const size_t smem = 4 * (size_t)(kRows * d + kWarps * kUnit * kRows + kWarps * kRows * d + kWarps * 2 * kRows);
  bump_launches();
  cudaError_t e = launch_dependent(attend_kernel<T>, dim3(kShares), dim3(32 * kWarps), smem, st, p);
  if (e != cudaSuccess) return e;
  bump_launches();
  return launch_dependent(join_kernel<T>, dim3(kShares, kRows), dim3(32 * kWarps),
                          4 * (size_t)kWarps * (d + 1), st, p);
}

}  // namespace

size_t cache_attend_ws_bytes(int B, int T, int Hq, int Hkv, int d, int dtype) {
  return (size_t)kShares * (2 * kRows * (d + 2) * 4 + sizeof(Split));
}

cudaError_t launch_cache_attend(const AttendArgs& a, int dtype, cudaStream_t st) {
  Params p{};
  p.a = a;
  p.G = a.Hq / a.c.Hkv;
  p.tiles = (p.G * a.T + kRows - 1) / kRows;
  p.entries = a.B * p.tiles;
  p.split = (Split*)a.ws;
  p.part = (float*)(p.split + kShares);
  p.scale2 = a.scale * kLog2e * a.c.k_scale;
  return dtype == SA_BF16 ? launch<__nv_bfloat16>(p, st) : launch<float>(p, st);
}

}  // namespace sa

// Attention of a sequence's newest tokens over its 4-bit cache: the kernel for any head dimension, on the
// CUDA cores in fp32, the launch that joins split segments, and the choice between the kernels.
// sa_cache_attend.cuh says how the work is cut.
#include "sa_cache_attend.cuh"

namespace sa {
using namespace attend;
namespace {

constexpr int kRows = 8;          // query rows of a tile of this kernel
constexpr int kShares = 2 * 148;  // its CTAs: two per SM (217 registers)

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
  Walk w;
  bool begins = false;
  if (!start(p, line, e, before, &w)) return file_nothing(p);
  while (next(p, &w)) {
    const Entry& en = w.en;
    const int h = w.h, k0 = w.k0, k1 = w.k1;
    __syncthreads();
    for (int i = tid; i < kRows * d; i += 32 * kWarps) {
      const int r = i / d, x = i - r * d;
      float v = 0.f;
      if (r < en.rows) v = to_f32(row_of(p, reinterpret_cast<const T*>(a.q), a.qs, en, h, r)[x]);
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
    float* part = part_of(p, blockIdx.x, k0 == 0);
    begins |= file_split(p, line, w);
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
        row_of(p, reinterpret_cast<T*>(a.y), a.ys, en, h, r)[x] = from_f32<T>(v * row_scale(sum, c.v_scale));
        if (x == 0 && a.lse) *lse_of(p, en, h, r) = row_lse(to, sum);
      } else {
        part[r * d + x] = v;
        if (x == 0) {
          part[kRows * d + r] = to;
          part[kRows * (d + 1) + r] = sum;
        }
      }
    }
  }
  if (!begins) file_nothing(p);
}

// Joins the parts of split segments.  A CTA has eight warps for rows / gridDim.y rows of one segment; the warps
// of a row take every so-many-th part, each with a maximum of its own, and join in their order.  A part
// is an L2 access away: four of them are on the way at once.
constexpr int kJoinWarps = 8, kAtOnce = 4;

template <typename T, int J>
__global__ void __launch_bounds__(32 * kJoinWarps) join_kernel(const Params p) {
  __shared__ float o_s[kJoinWarps][32 * J];
  __shared__ float ml_s[kJoinWarps][2];
  const AttendArgs& a = p.a;
  const int d = a.c.d, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rows = p.rows;
  grid_dependency_wait();
  const Split sp = p.split[blockIdx.x];                   // left over where nobody began the segment
  const Entry en = entry(p, p.by_segment ? blockIdx.x / a.c.Hkv : sp.e);
  if (en.n == 0 || sp.parts == 0) return;
  const int mine = rows / gridDim.y, per = kJoinWarps / mine;   // rows of this CTA, warps of a row
  const int r = blockIdx.y * mine + warp / per, sub = warp % per;
  float m = -INFINITY, l = 0.f, o[J] = {};
  if (r < en.rows) {
    for (int i0 = sub; i0 < sp.parts; i0 += per * kAtOnce) {
      float mi[kAtOnce], li[kAtOnce], v[kAtOnce][J];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const int i = i0 + k * per;
        const bool there = i < sp.parts;
        const float* f = part_of(p, sp.share + (there ? i : 0), !there || i == 0);
        mi[k] = there ? f[rows * d + r] : -INFINITY;
        li[k] = there ? f[rows * (d + 1) + r] : 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j) v[k][j] = there && lane + 32 * j < d ? f[r * d + lane + 32 * j] : 0.f;
      }
      float to = m;
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) to = fmaxf(to, mi[k]);
      const float ref = to == -INFINITY ? 0.f : to, keep = exp2f(m - ref);
      m = to;
      l *= keep;
#pragma unroll
      for (int j = 0; j < J; ++j) o[j] *= keep;
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const float w = exp2f(mi[k] - ref);
        l += w * li[k];
#pragma unroll
        for (int j = 0; j < J; ++j) o[j] += w * v[k][j];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < J; ++j) o_s[warp][lane + 32 * j] = o[j];
  if (lane == 0) {
    ml_s[warp][0] = m;
    ml_s[warp][1] = l;
  }
  __syncthreads();
  if (sub != 0 || r >= en.rows) return;
  for (int k = 1; k < per; ++k) m = fmaxf(m, ml_s[warp + k][0]);
  const float ref = m == -INFINITY ? 0.f : m;
  l = 0.f;
#pragma unroll
  for (int j = 0; j < J; ++j) o[j] = 0.f;
  for (int k = 0; k < per; ++k) {
    const float w = exp2f(ml_s[warp + k][0] - ref);
    l += w * ml_s[warp + k][1];
#pragma unroll
    for (int j = 0; j < J; ++j) o[j] += w * o_s[warp + k][lane + 32 * j];
  }
  T* y = row_of(p, reinterpret_cast<T*>(a.y), a.ys, en, sp.h, r);
  const float by = row_scale(l, a.c.v_scale);
#pragma unroll
  for (int j = 0; j < J; ++j)
    if (lane + 32 * j < d) y[lane + 32 * j] = from_f32<T>(o[j] * by);
  if (lane == 0 && a.lse) *lse_of(p, en, sp.h, r) = row_lse(m, l);
}

template <typename T>
cudaError_t join(const Params& p, cudaStream_t st) {
  const int64_t segments = (int64_t)p.entries * p.a.c.Hkv;
  // few segments have many parts each: a CTA per row, eight warps of which share the parts; many segments have
  // two or three: a warp per row
  const bool wide = segments * 8 < p.shares;
  const dim3 grid((unsigned)(p.by_segment ? segments : p.shares), wide ? p.rows : p.rows / kJoinWarps);
  const int d = p.a.c.d;
  return d <= 64    ? launch_dependent(join_kernel<T, 2>, grid, dim3(32 * kJoinWarps), 0, st, p)
         : d <= 128 ? launch_dependent(join_kernel<T, 4>, grid, dim3(32 * kJoinWarps), 0, st, p)
                    : launch_dependent(join_kernel<T, 8>, grid, dim3(32 * kJoinWarps), 0, st, p);
}

template <typename T>
cudaError_t launch(const Params& p, cudaStream_t st) {
  const int d = p.a.c.d;
  const size_t smem = 4 * (size_t)(kRows * d + kWarps * kUnit * kRows + kWarps * kRows * d + kWarps * 2 * kRows);
  return launch_dependent(attend_kernel<T>, dim3(p.shares), dim3(32 * kWarps), smem, st, p);
}

}  // namespace

cudaError_t launch_cache_join(const Params& p, int dtype, cudaStream_t st) {
  bump_launches();
  return dtype == SA_BF16 ? join<__nv_bfloat16>(p, st) : join<float>(p, st);
}

static void shape(int T, int G, int d, int dtype, int* shares, int* rows) {
  if (cache_attend_mma_takes(d)) return cache_attend_mma_shape(T, G, d, dtype, shares, rows);
  *shares = kShares;
  *rows = kRows;
}

size_t cache_attend_ws_bytes(int B, int T, int Hq, int Hkv, int d, int dtype) {
  int shares, rows;
  shape(T, Hq / Hkv, d, dtype, &shares, &rows);
  return attend::ws_bytes(shares, rows, d);
}

cudaError_t launch_cache_attend(const AttendArgs& a, int dtype, cudaStream_t st) {
  int shares, rows;
  shape(a.T, a.Hq / a.c.Hkv, a.c.d, dtype, &shares, &rows);
  const Params p = attend::params(a, shares, rows);
  bump_launches();
  const cudaError_t e = cache_attend_mma_takes(a.c.d) ? launch_cache_attend_mma(p, dtype, st)
                        : dtype == SA_BF16            ? launch<__nv_bfloat16>(p, st)
                                                      : launch<float>(p, st);
  return e == cudaSuccess ? launch_cache_join(p, dtype, st) : e;
}

}  // namespace sa

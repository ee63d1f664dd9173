// Attention of a sequence's newest tokens over its 4-bit cache: the launch that joins split segments, and the call.
// sa_cache_attend.cuh says how the work is cut, sa_cache_attend_mma.cuh has the attention itself.
#include "sa_cache_attend.cuh"

namespace sa {
using namespace attend;
namespace {

// Joins the parts of split segments.  A CTA has eight warps for rows / gridDim.y rows of one segment; the warps
// of a row take every so-many-th part, each with a maximum of its own, and join in their order.  A part
// is an L2 access away: eight of them are on the way at once (one of 131072 keys,
// 111 parts per head: 28.6 us in all, 30.2 with four; the join alone 8.8 with four, 19.4 one at a time).
constexpr int kJoinWarps = 8, kAtOnce = 8;

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

}  // namespace

size_t cache_attend_ws_bytes(int B, int T, int Hq, int Hkv, int d, int dtype) {
  int shares, rows;
  cache_attend_shape(T, Hq / Hkv, d, dtype, &shares, &rows);
  return attend::ws_bytes(shares, rows, d);
}

cudaError_t launch_cache_attend(const AttendArgs& a, int dtype, cudaStream_t st) {
  int shares, rows;
  cache_attend_shape(a.T, a.Hq / a.c.Hkv, a.c.d, dtype, &shares, &rows);
  const Params p = attend::params(a, shares, rows);
  const cudaError_t e = launch_cache_attend_tiles(p, dtype, st);
  if (e != cudaSuccess) return e;
  bump_launches();
  return dtype == SA_BF16 ? join<__nv_bfloat16>(p, st) : join<float>(p, st);
}

}  // namespace sa

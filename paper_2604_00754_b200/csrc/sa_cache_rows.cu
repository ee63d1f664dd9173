// Appending tokens to the 4-bit cache and reading them back.
//
// A thread takes 16 dimensions of a token, head and side at a time: one scale, two words of codes.  With
// x the values over the side's power of two t, s = e4m3(min(max|x| / 6, 448)) and each code is
// e2m1(x / s), both to the nearest with ties to even.  All of it is decided exactly, so the bytes
// are a function of the input's bits alone:
//   - a border between two scales is 6 m with m of at most 5 significant bits, one between two codes
//     b s with 3 + 4 bits, and a value that is not on a border is at least one unit of its last place away:
//     as a quotient of 24 bits, over half a unit (0.53) from b.  A quotient that is right to 2^-40 before its one
//     rounding therefore lands on b for values on the border and for no others.
//   - fp32, and the scale: with y a reciprocal within two units, q = x y is off by at most 5 units, r = x - q s
//     is exact in one multiply-add, and q + r y is right to 2^-42 before it is rounded.
//   - bf16 values have 8 bits, so x / s is a border or at least 2^-10 from it: there x y (off by less than
//     2^-18 for |x / s| < 10), rounded to a multiple of 2^-13, stands on the right side of every border or on it.
// Bound by HBM as long as few instructions stand between: a CTA takes one head and side, a thread keeps its
// place within the row and moves on by whole rows; t is folded into y and s; the tensors' 32 bytes of a thread (64
// in fp32) go in whole sectors by 32-byte accesses where they are aligned to that.  32768 tokens of 8 heads of 128 in
// bf16, 172 MB each way: append 32-33 us (81 % of the copy bandwidth; 33.1 where it looks at the pages' holders, a
// load that the tokens of a page share in L1), read 31 (86 %).
#include "sa_cache.cuh"

namespace sa {
namespace {

constexpr int kThreads = 256;

struct RowArgs {
  CacheView c;
  void *k, *v;
  int64_t s0, s1, s2;
  const int32_t *slots, *starts, *counts;
  const int32_t* refs;         // of an append, nullable: holders of the pages
  int T, groups, per, loops;   // 16-dimension groups of a row, tokens of a CTA at a time, how many times
  float over[2];               // 1 / t of K and V
};

// What a thread works on: blockIdx = (piece of the tokens, head and side, sequence).
struct Work {
  int g, t, end, first, slot;      // group of the row, its tokens t, t + per, ... < end, position of token 0
  int side, h;
};
template <bool kRead>
__device__ __forceinline__ bool work_of(const RowArgs& a, Work* w) {
  const CacheView& c = a.c;
  const int b = blockIdx.z, n = cache_count(c, a.counts, b, a.T);
  const int row = threadIdx.x / a.groups;
  w->g = threadIdx.x - row * a.groups;
  w->t = blockIdx.x * a.per * a.loops + row;
  w->end = min(n, (int)(blockIdx.x + 1) * a.per * a.loops);
  w->side = blockIdx.y & 1;
  w->h = blockIdx.y >> 1;
  if (w->t >= w->end) return false;
  w->slot = cache_slot(c, a.slots, b);
  if (w->slot < 0) return false;
  // without `starts` from lens (append) or from 0 (read)
  w->first = kRead ? (a.starts ? a.starts[b] : 0) : c.lens[w->slot];
  if (w->first < 0) report_cache(c);
  return w->first >= 0;
}

// Codes and scale byte of a token's group in the pool; false (recorded): it has no page, or an append would write
// into one that other sequences hold too.
struct Place {
  uint8_t *codes, *scale;
};
__device__ __forceinline__ bool place_of(const RowArgs& a, const Work& w, int t, Place* r) {
  const CacheView& c = a.c;
  const int64_t pos = (int64_t)w.first + t;
  const int page = cache_page(c, w.slot, pos);
  if (page < 0) return false;
  if (a.refs && a.refs[page] > 1) {
    report_cache(c);
    return false;
  }
  uint8_t* base = const_cast<uint8_t*>(cache_side(c, page, w.h, w.side));
  const int i = (int)pos & (c.P - 1);
  r->codes = base + i * (c.d / 2) + w.g * 8;
  r->scale = base + c.P * (c.d / 2) + i * a.groups + w.g;
  return true;
}

// 32 bytes of a tensor, aligned to that (kWide) or to 16.
template <bool kWide>
__device__ __forceinline__ void load32(const void* p, uint32_t (&w)[8]) {
  if (kWide) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p));
  } else {
    const uint4 a = reinterpret_cast<const uint4*>(p)[0], b = reinterpret_cast<const uint4*>(p)[1];
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
    w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
  }
}
template <bool kWide>
__device__ __forceinline__ void store32(void* p, const uint32_t (&w)[8]) {
  if (kWide) {
    asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(w[0]), "r"(w[1]), "r"(w[2]),
                 "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "l"(p)
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
    reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}

// 16 values as fp32, and the bits of the largest magnitude (7f800000 or more: not finite).
template <bool kWide>
__device__ __forceinline__ uint32_t load16(const __nv_bfloat16* p, float (&x)[16]) {
  uint32_t w[8];
  load32<kWide>(p, w);
  auto pair = [&](int i) { return __habs2(*reinterpret_cast<const __nv_bfloat162*>(&w[i])); };
  __nv_bfloat162 top = pair(0);
#pragma unroll
  for (int i = 1; i < 8; ++i) top = __hmax2_nan(top, pair(i));
  const uint32_t t = *reinterpret_cast<const uint32_t*>(&top);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
  return max(t << 16, t & 0xffff0000u);
}
template <bool kWide>
__device__ __forceinline__ uint32_t load16(const float* p, float (&x)[16]) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    uint32_t w[8];
    load32<kWide>(p + 8 * j, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[8 * j + i] = __uint_as_float(w[i]);
      top = max(top, w[i] & 0x7fffffffu);
    }
  }
  return top;
}

// x / s from y, 1 / s within two units: right to 2^-42 before its rounding.
__device__ __forceinline__ float quotient(float x, float s, float y) {
  const float q = __fmul_rn(x, y);
  return __fmaf_rn(__fmaf_rn(-q, s, x), y, q);
}

// The bytes of 16 values whose largest magnitude has the bits `top`.
template <typename T>
__device__ __forceinline__ void quantise(float (&x)[16], uint32_t top, float t, float over, const Place& r) {
  if (top >= 0x7f800000u) {       // an infinity or a NaN among them: all 16 read as NaN
    *r.scale = 0x7f;
    *reinterpret_cast<uint2*>(r.codes) = make_uint2(0, 0);
    return;
  }
  // 4096 saturates under every scale, and what exceeds it has the largest one
  const float most = fminf(__uint_as_float(top) * over, 4096.f);
  const uint8_t scale = f32_to_scale(quotient(most, 6.f, 1.f / 6.f));
  const float s = scale_to_f32(scale);
  const float y = s > 0.f ? __fdividef(1.f, s) * over : 0.f, st = s * t;          // no scale: all codes 0
  if (most == 4096.f) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = fminf(fmaxf(x[i], -4096.f * t), 4096.f * t);
  }
  uint32_t w[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v = x[8 * j + i];
      q[i] = sizeof(T) == 2 ? __fadd_rn(__fmaf_rn(v, y, 1536.f), -1536.f) : quotient(v, st, y);
    }
    w[j] = floats_to_codes(q);
  }
  *r.scale = scale;
  *reinterpret_cast<uint2*>(r.codes) = make_uint2(w[0], w[1]);
}

template <typename T, bool kWide>
__global__ void __launch_bounds__(kThreads) append_kernel(const RowArgs a) {
  grid_dependency_wait();
  Work w;
  if (!work_of<false>(a, &w)) return;
  const T* p = reinterpret_cast<const T*>(w.side ? a.v : a.k) + blockIdx.z * a.s0 + w.h * a.s1 + (int64_t)w.t * a.s2 + 16 * w.g;
  const float t = w.side ? a.c.v_scale : a.c.k_scale, over = a.over[w.side];
  for (; w.t < w.end; w.t += a.per, p += a.per * a.s2) {
    float x[16];
    const uint32_t top = load16<kWide>(p, x);
    Place r;
    if (place_of(a, w, w.t, &r)) quantise<T>(x, top, t, over, r);
  }
}

template <bool kWide>
__device__ __forceinline__ void store16(__nv_bfloat16* p, const float (&y)[16]) {
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(y[2 * i], y[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  store32<kWide>(p, w);
}
template <bool kWide>
__device__ __forceinline__ void store16(float* p, const float (&y)[16]) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(y[8 * j + i]);
    store32<kWide>(p + 8 * j, w);
  }
}

template <typename T, bool kWide>
__global__ void __launch_bounds__(kThreads) read_kernel(const RowArgs a) {
  grid_dependency_wait();
  Work w;
  if (!work_of<true>(a, &w)) return;
  T* p = reinterpret_cast<T*>(w.side ? a.v : a.k) + blockIdx.z * a.s0 + w.h * a.s1 + (int64_t)w.t * a.s2 + 16 * w.g;
  const float t = w.side ? a.c.v_scale : a.c.k_scale;
  for (; w.t < w.end; w.t += a.per, p += a.per * a.s2) {
    Place r;
    if (!place_of(a, w, w.t, &r)) continue;
    const uint2 codes = *reinterpret_cast<const uint2*>(r.codes);
    const float s = scale_to_f32(*r.scale) * t;
    float y[16];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      uint32_t h[4];
      codes_to_half2(j ? codes.y : codes.x, h);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[k]));
        y[8 * j + 2 * k] = f.x * s;
        y[8 * j + 2 * k + 1] = f.y * s;
      }
    }
    store16<kWide>(p, y);
  }
}

template <typename T, bool kWide>
cudaError_t launch(const RowArgs& a, bool read, dim3 grid, cudaStream_t st) {
  const dim3 block(a.groups * a.per);
  return read ? launch_dependent(read_kernel<T, kWide>, grid, block, 0, st, a)
              : launch_dependent(append_kernel<T, kWide>, grid, block, 0, st, a);
}

}  // namespace

cudaError_t launch_cache_rows(const CacheView& c, bool read, int B, int T, void* k, void* v,
                              int dtype, const int64_t stride[3], const int32_t* slots,
                              const int32_t* starts, const int32_t* counts, const int32_t* refs,
                              cudaStream_t st) {
  RowArgs a{c, k, v, stride[0], stride[1], stride[2], slots, starts, counts, refs, T};
  a.groups = c.d / 16;
  a.per = kThreads / a.groups < T ? kThreads / a.groups : T;
  a.over[0] = 1.f / c.k_scale;
  a.over[1] = 1.f / c.v_scale;
  // a thread goes round as often as leaves four full waves of CTAs, eight times at most
  const int64_t ctas = (int64_t)((T + a.per - 1) / a.per) * c.Hkv * 2 * B, waves = ctas / (148 * 8 * 4);
  a.loops = (int)(waves < 1 ? 1 : waves > 8 ? 8 : waves);
  const int span = a.per * a.loops;
  const dim3 grid((T + span - 1) / span, c.Hkv * 2, B);
  const int elt = dtype == SA_BF16 ? 2 : 4;
  const uintptr_t odd = (uintptr_t)k | (uintptr_t)v | (uintptr_t)((stride[0] | stride[1] | stride[2]) * elt);
  const bool wide = odd % 32 == 0;
  bump_launches();
  if (dtype == SA_BF16)
    return wide ? launch<__nv_bfloat16, true>(a, read, grid, st) : launch<__nv_bfloat16, false>(a, read, grid, st);
  return wide ? launch<float, true>(a, read, grid, st) : launch<float, false>(a, read, grid, st);
}

}  // namespace sa

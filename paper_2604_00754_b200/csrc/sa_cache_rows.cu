// Appending tokens to the 4-bit cache and reading them back.
//
// A thread takes 16 dimensions of one token, head and side: one scale, two words of codes.  With
// x the values over the side's power of two (exact), s = e4m3(min(max|x| / 6, 448)) and each code is
// e2m1(x / s), both to the nearest with ties to even.  All of it is decided exactly, so the bytes
// are a function of the input's bits alone:
//   - a border between two scales is 6 m with m of at most 5 significant bits, one between two codes
//     b s with 3 + 4 bits; the correctly rounded fp32 quotient of another value never lands on one
//     (the value is at least one unit of its last place away, the quotient then over half a unit);
//   - bf16 values have 8 bits, so x / s is a border or at least 2^-10 from it: there the product with
//     the rounded reciprocal (off by less than 2^-19 for |x / s| < 10), rounded to a multiple of 2^-13,
//     stands on the right side of every border or on it.
#include "sa_cache.cuh"

namespace sa {
namespace {

struct RowArgs {
  CacheView c;
  void *k, *v;
  int64_t s0, s1, s2;
  const int32_t *slots, *starts, *counts;
  int T;
};

// Where group `x` of sequence blockIdx.y lies: codes and scale byte in the pool, offset in the tensor.
// False: nothing there (past the sequence's tokens, or reported).  `starts` null: from lens (append)
// or from 0 (read).
struct RowPlace {
  uint8_t *codes, *scale;
  int64_t at;
  bool value;   // the V side
};
template <bool kRead>
__device__ __forceinline__ bool place(const RowArgs& a, unsigned x, RowPlace* r) {
  const CacheView& c = a.c;
  const unsigned groups = (unsigned)c.d / 16;
  const unsigned g = x % groups;
  x /= groups;
  const unsigned t = x % (unsigned)a.T;
  x /= (unsigned)a.T;
  const unsigned side = x & 1, h = x >> 1;
  if (h >= (unsigned)c.Hkv) return false;
  const int b = blockIdx.y;
  const int n = cache_count(c, a.counts, b, a.T);
  if ((int)t >= n) return false;
  const int slot = cache_slot(c, a.slots, b);
  if (slot < 0) return false;
  const int first = kRead ? (a.starts ? a.starts[b] : 0) : c.lens[slot];
  if (first < 0) {
    report_cache(c);
    return false;
  }
  const int64_t pos = (int64_t)first + t;
  const int page = cache_page(c, slot, pos);
  if (page < 0) return false;
  uint8_t* base = const_cast<uint8_t*>(cache_side(c, page, h, side));
  const int i = (int)(pos % c.P);
  r->codes = base + i * (c.d / 2) + g * 8;
  r->scale = base + c.P * (c.d / 2) + i * (int)groups + g;
  r->at = b * a.s0 + h * a.s1 + (int64_t)t * a.s2 + 16 * g;
  r->value = side;
  return true;
}

__device__ __forceinline__ void load16(const __nv_bfloat16* p, uint32_t (&x)[16]) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint4 w = reinterpret_cast<const uint4*>(p)[j];
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[8 * j + 2 * k] = v[k] << 16;
      x[8 * j + 2 * k + 1] = v[k] & 0xffff0000u;
    }
  }
}
__device__ __forceinline__ void load16(const float* p, uint32_t (&x)[16]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint4 w = reinterpret_cast<const uint4*>(p)[j];
    x[4 * j] = w.x;
    x[4 * j + 1] = w.y;
    x[4 * j + 2] = w.z;
    x[4 * j + 3] = w.w;
  }
}

template <typename T>
__global__ void __launch_bounds__(256) append_kernel(const RowArgs a) {
  grid_dependency_wait();
  RowPlace r;
  if (!place<false>(a, blockIdx.x * 256u + threadIdx.x, &r)) return;
  uint32_t x[16];
  load16(reinterpret_cast<const T*>(r.value ? a.v : a.k) + r.at, x);
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max(top, x[i] & 0x7fffffffu);
  if (top >= 0x7f800000u) {       // an infinity or a NaN among them: all 16 read as NaN
    *r.scale = 0x7f;
    *reinterpret_cast<uint2*>(r.codes) = make_uint2(0, 0);
    return;
  }
  const float over = __fdiv_rn(1.f, r.value ? a.c.v_scale : a.c.k_scale);   // a power of two
  // 4096 saturates under every scale, and what exceeds it has the largest one
  const uint8_t scale = f32_to_scale(__fdiv_rn(fminf(__uint_as_float(top) * over, 4096.f), 6.f));
  const float s = scale_to_f32(scale);
  const float inv = s > 0.f ? __fdiv_rn(1.f, s) : 0.f;
  uint32_t w[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v = fminf(fmaxf(__uint_as_float(x[8 * j + i]) * over, -4096.f), 4096.f);
      if (sizeof(T) == 2) y[i] = __fadd_rn(__fmaf_rn(v, inv, 1536.f), -1536.f);
      else y[i] = s > 0.f ? __fdiv_rn(v, s) : 0.f;
    }
    w[j] = floats_to_codes(y);
  }
  *r.scale = scale;
  *reinterpret_cast<uint2*>(r.codes) = make_uint2(w[0], w[1]);
}

__device__ __forceinline__ void store16(__nv_bfloat16* p, const float (&y)[16]) {
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(y[2 * i], y[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
  reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
}
__device__ __forceinline__ void store16(float* p, const float (&y)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    reinterpret_cast<float4*>(p)[i] = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
}

template <typename T>
__global__ void __launch_bounds__(256) read_kernel(const RowArgs a) {
  grid_dependency_wait();
  RowPlace r;
  if (!place<true>(a, blockIdx.x * 256u + threadIdx.x, &r)) return;
  const uint2 w = *reinterpret_cast<const uint2*>(r.codes);
  const float s = scale_to_f32(*r.scale) * (r.value ? a.c.v_scale : a.c.k_scale);
  float y[16];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    uint32_t h[4];
    codes_to_half2(j ? w.y : w.x, h);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
      y[8 * j + 2 * i] = f.x * s;
      y[8 * j + 2 * i + 1] = f.y * s;
    }
  }
  store16(reinterpret_cast<T*>(r.value ? a.v : a.k) + r.at, y);
}

}  // namespace

cudaError_t launch_cache_rows(const CacheView& c, bool read, int B, int T, void* k, void* v,
                              int dtype, const int64_t stride[3], const int32_t* slots,
                              const int32_t* starts, const int32_t* counts, cudaStream_t st) {
  const RowArgs a{c, k, v, stride[0], stride[1], stride[2], slots, starts, counts, T};
  const int64_t groups = (int64_t)T * c.Hkv * 2 * (c.d / 16);
  const dim3 grid((unsigned)((groups + 255) / 256), B);
  bump_launches();
  if (read)
    return dtype == SA_BF16 ? launch_dependent(read_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, a)
                            : launch_dependent(read_kernel<float>, grid, dim3(256), 0, st, a);
  return dtype == SA_BF16 ? launch_dependent(append_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, a)
                          : launch_dependent(append_kernel<float>, grid, dim3(256), 0, st, a);
}

}  // namespace sa

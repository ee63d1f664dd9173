// The 4-bit paged cache: geometry, checks of what only the device can see, conversions.
//
// A page holds P tokens of every KV head.  Per head and side (0 = K, 1 = V) it has P rows of d/2
// bytes of e2m1 codes (dimension 2i in the low half of byte i) and then P rows of d/16 e4m3 scales,
// one per 16 dimensions: 4.5 bits a value.  code * scale has at most 6 significant bits and lies in
// [2^-10, 2688], so fp16 and bf16 both hold it exactly: dequantising never rounds.
#pragma once

#include <cuda_fp16.h>

#include "sa_common.cuh"

namespace sa {

// What the kernels need of an sa_cache: `pool` is that of one layer.
struct CacheView {
  uint8_t* pool;
  const int32_t *table, *lens;
  int pages, Hkv, d, P, p_shift, slots, row;   // P = 1 << p_shift
  int side;               // bytes of one head and side of a page
  int64_t page_bytes;     // of one layer
  float k_scale, v_scale;
  int* status;
};

// The device status word of the cache's calls: apart from the attention calls' word, which makes
// later launches return early.
int* cache_status_ptr();

__device__ __forceinline__ void report_cache(const CacheView& c) {
  atomicCAS(c.status, SA_OK, SA_ERR_BAD_CACHE);
}

// Table row of sequence b, or -1 (reported) where the caller's list names none.
__device__ __forceinline__ int cache_slot(const CacheView& c, const int32_t* slots, int b) {
  const int s = slots ? slots[b] : b;
  if ((unsigned)s < (unsigned)c.slots) return s;
  report_cache(c);
  return -1;
}

// New tokens of sequence b: counts[b], or all T; -1 (reported) where that is no number of tokens.
__device__ __forceinline__ int cache_count(const CacheView& c, const int32_t* counts, int b, int T) {
  const int n = counts ? counts[b] : T;
  if (n >= 0 && n <= T) return n;
  report_cache(c);
  return -1;
}

// Page that holds token `pos` (not negative) of a slot, or -1 (reported) where the slot has none there.
__device__ __forceinline__ int cache_page(const CacheView& c, int slot, int64_t pos) {
  const int64_t i = pos >> c.p_shift;
  if (i < c.row) {
    const int p = c.table[(int64_t)slot * c.row + i];
    if ((unsigned)p < (unsigned)c.pages) return p;
  }
  report_cache(c);
  return -1;
}

__device__ __forceinline__ const uint8_t* cache_side(const CacheView& c, int page, int h, int side) {
  return c.pool + (int64_t)page * c.page_bytes + (int64_t)(2 * h + side) * c.side;
}

// Eight codes of a word as four pairs of fp16 (low half: even dimension).  Exact.
__device__ __forceinline__ void codes_to_half2(uint32_t w, uint32_t (&r)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
      : "r"(w));
}

// Eight floats to codes, to the nearest, ties to the even code, saturating at 6.
__device__ __forceinline__ uint32_t floats_to_codes(const float (&x)[8]) {
  uint32_t w;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(w)
      : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
  return w;
}

// Two scales (low byte first) as a pair of fp16.  Exact; 0x7f and 0xff are NaN.
__device__ __forceinline__ uint32_t scales_to_half2(uint32_t two) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)two));
  return r;
}
__device__ __forceinline__ float scale_to_f32(uint8_t s) {
  return __half2float(__ushort_as_half((uint16_t)scales_to_half2(s)));
}

// A positive float to its scale, to the nearest, ties to even, saturating at 448.
__device__ __forceinline__ uint8_t f32_to_scale(float x) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(x));
  return (uint8_t)r;
}

struct AttendArgs {
  CacheView c;
  const void* q;
  void* y;
  float* lse;                     // nullable
  const int32_t *slots, *counts;  // nullable
  int64_t qs[3], ys[3];
  int B, T, Hq, w;
  bool causal;
  float scale;
  void* ws;
};

cudaError_t launch_cache_rows(const CacheView& c, bool read, int B, int T, void* k, void* v,
                              int dtype, const int64_t stride[3], const int32_t* slots,
                              const int32_t* starts, const int32_t* counts, const int32_t* refs,
                              cudaStream_t st);
cudaError_t launch_cache_attend(const AttendArgs& a, int dtype, cudaStream_t st);
size_t cache_attend_ws_bytes(int B, int T, int Hq, int Hkv, int d, int dtype);

// The books: the caller's struct with its checks done.
cudaError_t launch_cache_free(const sa_cache& c, int n, const int32_t* slots, int* status,
                              cudaStream_t st);
cudaError_t launch_cache_fork(const sa_cache& c, int n, const int32_t* parents,
                              const int32_t* children, int* status, cudaStream_t st);
cudaError_t launch_cache_reserve(const sa_cache& c, const int32_t* add, int32_t* got, void* ws,
                                 int* status, cudaStream_t st);
cudaError_t launch_cache_compact(const sa_cache& c, int32_t* live, void* ws, int* status,
                                 cudaStream_t st);
size_t cache_books_ws_bytes(const sa_cache& c);

}  // namespace sa

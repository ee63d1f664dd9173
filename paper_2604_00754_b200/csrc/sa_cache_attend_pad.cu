// The tensor-core attention over the 4-bit cache for head dimensions between the tiles' 64, 128 and 256.
#include "sa_cache_attend_mma.cuh"

namespace sa {
namespace attend {
namespace {

template <typename T>
int ctas(int d, int nt) {
  return with_shape<true>(d, nt, [](auto D, auto NT) { return Shape<T, decltype(D)::value, decltype(NT)::value, true>::kCtas; });
}
template <typename T>
cudaError_t launch_rows(const Params& p, int nt, cudaStream_t st) {
  return with_shape<true>(p.a.c.d, nt, [&](auto D, auto NT) {
    return launch<T, decltype(D)::value, decltype(NT)::value, true>(p, st);
  });
}

}  // namespace

int padded_ctas(int d, int nt, int dtype) {
  return dtype == SA_BF16 ? ctas<__nv_bfloat16>(d, nt) : ctas<float>(d, nt);
}
cudaError_t launch_padded(const Params& p, int nt, int dtype, cudaStream_t st) {
  return dtype == SA_BF16 ? launch_rows<__nv_bfloat16>(p, nt, st) : launch_rows<float>(p, nt, st);
}

}  // namespace attend
}  // namespace sa

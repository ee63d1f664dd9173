// The tensor-core attention over the 4-bit cache for head dimensions 64, 128 and 256, and its shape for a call.
#include "sa_cache_attend_mma.cuh"

namespace sa {
using namespace attend;
namespace {

template <typename T>
int ctas(int d, int nt) {
  return with_shape<false>(d, nt, [](auto D, auto NT) { return Shape<T, decltype(D)::value, decltype(NT)::value, false>::kCtas; });
}
template <typename T>
cudaError_t launch_rows(const Params& p, int nt, cudaStream_t st) {
  return with_shape<false>(p.a.c.d, nt, [&](auto D, auto NT) {
    return launch<T, decltype(D)::value, decltype(NT)::value, false>(p, st);
  });
}

// Row tiles that a warp takes of a KV head's rows: K and V are dequantised once per so many, so as many as there are or
// fit, spread evenly (37 rows: two times three tiles, not four and one).
int row_tiles(int T, int G, int d) {
  const int most = most_tiles(tile_dim(d), tile_dim(d) != d);
  const int64_t all = ((int64_t)T * G + 7) / 8, times = (all + most - 1) / most;
  return (int)((all + times - 1) / times);
}

}  // namespace

void cache_attend_shape(int T, int G, int d, int dtype, int* shares, int* rows) {
  const int nt = row_tiles(T, G, d);
  *rows = 8 * nt;
  *shares = 148 * (tile_dim(d) != d   ? padded_ctas(d, nt, dtype)
                   : dtype == SA_BF16 ? ctas<__nv_bfloat16>(d, nt)
                                      : ctas<float>(d, nt));
}

cudaError_t launch_cache_attend_tiles(const Params& p, int dtype, cudaStream_t st) {
  const int d = p.a.c.d, nt = p.rows / 8;
  bump_launches();
  if (tile_dim(d) != d) return launch_padded(p, nt, dtype, st);
  return dtype == SA_BF16 ? launch_rows<__nv_bfloat16>(p, nt, st) : launch_rows<float>(p, nt, st);
}

}  // namespace sa

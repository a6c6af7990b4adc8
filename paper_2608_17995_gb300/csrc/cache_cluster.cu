// cache_cluster.cu — the cache attention of shorter sequences in one launch: a
// cluster of CTAs per unit.
#include "cache_cluster.cuh"

namespace avits {
namespace cache {

cudaError_t launch_cluster(CacheAttn& a, int D, int ncta, int warps, cudaStream_t s) {
  return by_rows(a, D, [&](auto rows) {
    using Rows = decltype(rows);
    CUtensorMap mk{}, mv{};
    map_cache<Rows>(a, &mk, &mv);
    if constexpr (Rows::kBf16 && Rows::kR <= 16)
      if (warps == 1)
        return launch_rows<Rows, 1, kAlone>(mk, mv, a, ncta, a.c.max_len, {}, s);
    if (warps <= 2) return launch_rows<Rows, 2, kAlone>(mk, mv, a, ncta, a.c.max_len, {}, s);
    return launch_rows<Rows, 4, kAlone>(mk, mv, a, ncta, a.c.max_len, {}, s);
  });
}

}  // namespace cache
}  // namespace avits

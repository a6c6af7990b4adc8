// cache_shared_own.cu — shared prefixes: the own tokens of short sequences, as parts beside the
// kernel over the prefixes, or with a short prefix in one launch.
#include "cache_cluster.cuh"

namespace avits {
namespace cache {

cudaError_t launch_own_parts(CacheAttn& a, int D, int warps, cudaStream_t s) {
  return by_rows(a, D, [&](auto rows) {
    using Rows = decltype(rows);
    CUtensorMap mk{}, mv{};
    map_cache<Rows>(a, &mk, &mv);
    const Beside<kParts> none{};
    if (warps == 2) return launch_rows<Rows, 2, kParts>(mk, mv, a, 1, 0, none, s);
    return launch_rows<Rows, 4, kParts>(mk, mv, a, 1, 0, none, s);
  });
}

cudaError_t launch_both(CacheAttn& a, const CacheAttn& p, int D, int ncta, cudaStream_t s) {
  return by_rows(a, D, [&](auto rows) {
    using Rows = decltype(rows);
    CUtensorMap mk{}, mv{};
    Beside<kBoth> x{};
    x.p = p;
    x.p.tile = a.tile;      // as the own tokens: pieces of a warp, not of the tensor cores
    map_cache<Rows>(a, &mk, &mv);
    map_cache<Rows>(x.p, &x.mk, &x.mv);
    if (a.box == 0 || x.p.box == 0) a.box = x.p.box = 0;      // one kind of copies for both
    return launch_rows<Rows, 4, kBoth>(mk, mv, a, ncta, 0, x, s);
  });
}

}  // namespace cache
}  // namespace avits

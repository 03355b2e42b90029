// Attention over shared prefixes on fp32 caches: the variants.
#include "paged_shared.cuh"

namespace dck {
namespace paged {
namespace {

template <int DP, int S>
cudaError_t own(const Args& g, cudaStream_t s) {
  using Z = Sizes<float, DP, warps_of(DP, false), S, 8>;
  if (g.p.rows == 1) return launch_own<Z, SimtTile<Z, 1>>(g, s);
  return g.p.rows <= 4 ? launch_own<Z, SimtTile<Z, 4>>(g, s) : launch_own<Z, SimtTile<Z, 8>>(g, s);
}

template <int DP, int S>
cudaError_t prefix(const Args& g, cudaStream_t s) {
  using Z = Sizes<float, DP, warps_of(DP, false), S, 8>;
  return launch_prefix<Z, SimtTile<Z, 8>>(g, s);  // (blocks of 8 queries: layout_of)
}

}  // namespace

cudaError_t launch_own_f32(const Args& g, cudaStream_t s) {
  return g.DP == 64 ? own<64, 4>(g, s) : g.DP == 128 ? own<128, 2>(g, s) : own<256, 2>(g, s);
}

cudaError_t launch_prefix_f32(const Args& g, cudaStream_t s) {
  return g.DP == 64 ? prefix<64, 4>(g, s) : g.DP == 128 ? prefix<128, 2>(g, s) : prefix<256, 2>(g, s);
}

}  // namespace paged
}  // namespace dck

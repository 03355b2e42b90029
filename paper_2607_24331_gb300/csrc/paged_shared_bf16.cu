// Attention over shared prefixes on bf16 caches: the variants.
#include "paged_shared.cuh"

namespace dck {
namespace paged {
namespace {

template <int DP, int S, bool PACK>
cudaError_t own(const Args& g, cudaStream_t s) {
  using Z = Sizes<__nv_bfloat16, DP, warps_of(DP, false), S, 16>;
  return launch_own<Z, TensorTile<Z, PACK>>(g, s);
}

template <int DP, int S, bool PACK>
cudaError_t prefix(const Args& g, cudaStream_t s) {
  using Z = Sizes<__nv_bfloat16, DP, warps_of(DP, false), S, 16>;
  return launch_prefix<Z, TensorTile<Z, PACK>>(g, s);
}

}  // namespace

cudaError_t launch_own_bf16(const Args& g, cudaStream_t s) {
  if (g.DP == 256) return own<256, 2, true>(g, s);
  if (g.DP == 128) return g.p.rows > 8 ? own<128, 2, false>(g, s) : own<128, 2, true>(g, s);
  return g.p.rows > 8 ? own<64, 4, false>(g, s) : own<64, 4, true>(g, s);
}

cudaError_t launch_prefix_bf16(const Args& g, cudaStream_t s) {
  if (g.DP == 256) return prefix<256, 2, true>(g, s);
  if (g.DP == 128) return g.x.rows > 8 ? prefix<128, 2, false>(g, s) : prefix<128, 2, true>(g, s);
  return g.x.rows > 8 ? prefix<64, 4, false>(g, s) : prefix<64, 4, true>(g, s);
}

}  // namespace paged
}  // namespace dck

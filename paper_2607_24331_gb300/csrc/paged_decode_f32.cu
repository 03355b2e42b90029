// dck_paged_decode_attention on fp32 caches: the CUDA-core variants.
#include "paged_decode.cuh"

namespace dck {
namespace paged {
namespace {

template <class Z>
cudaError_t by_rows(const Args& g, cudaStream_t s) {
  if (g.p.rows == 1) return launch_tile<Z, SimtTile<Z, 1>>(g, s);
  if (g.p.rows <= 4) return launch_tile<Z, SimtTile<Z, 4>>(g, s);
  return launch_tile<Z, SimtTile<Z, 8>>(g, s);
}

}  // namespace

cudaError_t launch_f32(const Args& g, cudaStream_t s) {
  if (g.DP == 64) return by_rows<Sizes<float, 64, 8, 4, 8>>(g, s);
  if (g.DP == 128) return by_rows<Sizes<float, 128, 8, 2, 8>>(g, s);
  return by_rows<Sizes<float, 256, 4, 2, 8>>(g, s);
}

}  // namespace paged
}  // namespace dck

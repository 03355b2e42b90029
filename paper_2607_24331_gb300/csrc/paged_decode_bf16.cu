// dck_paged_decode_attention on bf16 caches: the tensor-core variants.
#include "paged_decode.cuh"

namespace dck {
namespace paged {

cudaError_t launch_bf16(const Args& g, cudaStream_t s) {
  using bf16 = __nv_bfloat16;
  if (g.DP == 256) {
    using Z = Sizes<bf16, 256, 4, 3, 16>;
    return launch_tile<Z, TensorTile<Z, true>>(g, s);
  }
  if (g.DP == 128) {
    using Z = Sizes<bf16, 128, 8, 3, 16>;
    return g.p.rows > 8 ? launch_tile<Z, TensorTile<Z, false>>(g, s) : launch_tile<Z, TensorTile<Z, true>>(g, s);
  }
  using Z = Sizes<bf16, 64, 8, 6, 16>;
  return g.p.rows > 8 ? launch_tile<Z, TensorTile<Z, false>>(g, s) : launch_tile<Z, TensorTile<Z, true>>(g, s);
}

}  // namespace paged
}  // namespace dck

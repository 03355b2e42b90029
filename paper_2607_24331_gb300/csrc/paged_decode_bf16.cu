// dck_paged_decode_attention on bf16 caches: the tensor-core variants.
#include "paged_decode.cuh"

namespace dck {
namespace paged {
namespace {

template <int DP, int S, bool PACK>
cudaError_t launch_pack(const Args& g, cudaStream_t s) {
  if (g.p.warps == warps_of(DP, true)) {
    using Z = Sizes<__nv_bfloat16, DP, warps_of(DP, true), S, 16>;
    return launch_kernel<Z, TensorTile<Z, PACK>, true>(g, s);
  }
  using Z = Sizes<__nv_bfloat16, DP, warps_of(DP, false), S, 16>;
  return g.p.cluster ? launch_kernel<Z, TensorTile<Z, PACK>, true>(g, s) : launch_kernel<Z, TensorTile<Z, PACK>, false>(g, s);
}

}  // namespace

cudaError_t launch_bf16(const Args& g, cudaStream_t s) {
  if (g.DP == 256) return launch_pack<256, 3, true>(g, s);
  if (g.DP == 128) return g.p.rows > 8 ? launch_pack<128, 3, false>(g, s) : launch_pack<128, 3, true>(g, s);
  return g.p.rows > 8 ? launch_pack<64, 6, false>(g, s) : launch_pack<64, 6, true>(g, s);
}

}  // namespace paged
}  // namespace dck

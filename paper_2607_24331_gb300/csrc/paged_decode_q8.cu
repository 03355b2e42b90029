// dck_quant_decode_attention: the variants of attention over 8-bit caches.
#include "paged_decode_q8.cuh"

namespace dck {
namespace paged {
namespace {

template <typename T, int DP, int S, int S_ALONE, bool PACK>
cudaError_t launch_pack(const Args& g, cudaStream_t s) {
  if (g.p.warps == warps_of(DP, true)) {
    using Z = QuantSizes<T, DP, warps_of(DP, true), S_ALONE>;
    return launch_kernel<Z, QuantTile<Z, PACK>, true>(g, s);
  }
  using Z = QuantSizes<T, DP, warps_of(DP, false), S>;
  return g.p.cluster ? launch_kernel<Z, QuantTile<Z, PACK>, true>(g, s) : launch_kernel<Z, QuantTile<Z, PACK>, false>(g, s);
}

}  // namespace

cudaError_t launch_q8(const Args& g, int dtype, cudaStream_t s) {
  if (dtype == DCK_F32) {
    if (g.DP == 256) return launch_pack<float, 256, 2, 2, true>(g, s);
    return g.DP == 128 ? launch_pack<float, 128, 2, 2, true>(g, s) : launch_pack<float, 64, 4, 4, true>(g, s);
  }
  using T = __nv_bfloat16;
  if (g.DP == 256) return launch_pack<T, 256, 2, 2, true>(g, s);
  if (g.DP == 128) return g.p.rows > 8 ? launch_pack<T, 128, 2, 2, false>(g, s) : launch_pack<T, 128, 2, 3, true>(g, s);
  return g.p.rows > 8 ? launch_pack<T, 64, 4, 4, false>(g, s) : launch_pack<T, 64, 4, 4, true>(g, s);
}

}  // namespace paged
}  // namespace dck

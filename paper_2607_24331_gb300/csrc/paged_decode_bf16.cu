// dck_paged_decode_attention on bf16 caches: the tensor-core variants.
#include "paged_decode.cuh"

namespace dck {
namespace paged {
namespace {

// S: stages of a warp.  Two keep enough copies in flight with the two CTAs of an SM, and HBM
// gives more with no more than that under way (16 x 4096 tokens of 32 heads 150 us, three 154);
// a cluster's CTA, alone on its SM, has up to S_ALONE.
template <int DP, int S, int S_ALONE, bool PACK>
cudaError_t launch_pack(const Args& g, cudaStream_t s) {
  if (g.p.warps == warps_of(DP, true)) {
    using Z = Sizes<__nv_bfloat16, DP, warps_of(DP, true), S_ALONE, 16>;
    return launch_kernel<Z, TensorTile<Z, PACK>, true>(g, s);
  }
  using Z = Sizes<__nv_bfloat16, DP, warps_of(DP, false), S, 16>;
  return g.p.cluster ? launch_kernel<Z, TensorTile<Z, PACK>, true>(g, s) : launch_kernel<Z, TensorTile<Z, PACK>, false>(g, s);
}

}  // namespace

cudaError_t launch_bf16(const Args& g, cudaStream_t s) {
  if (g.DP == 256) return launch_pack<256, 2, 2, true>(g, s);
  if (g.DP == 128) return g.p.rows > 8 ? launch_pack<128, 2, 2, false>(g, s) : launch_pack<128, 2, 3, true>(g, s);
  return g.p.rows > 8 ? launch_pack<64, 4, 4, false>(g, s) : launch_pack<64, 4, 4, true>(g, s);
}

}  // namespace paged
}  // namespace dck

// dck_paged_decode_attention on fp32 caches: the CUDA-core variants.
#include "paged_decode.cuh"

namespace dck {
namespace paged {
namespace {

template <int DP, int S, int ROWS>
cudaError_t launch_rows(const Args& g, cudaStream_t s) {
  if (g.p.warps == warps_of(DP, true)) {
    using Z = Sizes<float, DP, warps_of(DP, true), S, 8>;
    return launch_kernel<Z, SimtTile<Z, ROWS>, true>(g, s);
  }
  using Z = Sizes<float, DP, warps_of(DP, false), S, 8>;
  return g.p.cluster ? launch_kernel<Z, SimtTile<Z, ROWS>, true>(g, s) : launch_kernel<Z, SimtTile<Z, ROWS>, false>(g, s);
}

template <int DP, int S>
cudaError_t by_rows(const Args& g, cudaStream_t s) {
  if (g.p.rows == 1) return launch_rows<DP, S, 1>(g, s);
  if (g.p.rows <= 4) return launch_rows<DP, S, 4>(g, s);
  return launch_rows<DP, S, 8>(g, s);
}

}  // namespace

cudaError_t launch_f32(const Args& g, cudaStream_t s) {
  if (g.DP == 64) return by_rows<64, 4>(g, s);
  if (g.DP == 128) return by_rows<128, 2>(g, s);
  return by_rows<256, 2>(g, s);
}

}  // namespace paged
}  // namespace dck

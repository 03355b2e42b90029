// Attention over shared prefixes on 8-bit caches: the variants.
#include "paged_decode_q8.cuh"
#include "paged_shared.cuh"

namespace dck {
namespace paged {
namespace {

template <typename T, int DP, int S, bool PACK>
cudaError_t own(const Args& g, cudaStream_t s) {
  using Z = QuantSizes<T, DP, warps_of(DP, false), S>;
  return launch_own<Z, QuantTile<Z, PACK>>(g, s);
}

template <typename T, int DP, int S>
cudaError_t prefix(const Args& g, cudaStream_t s) {
  using Z = QuantSizes<T, DP, warps_of(DP, false), S>;
  return launch_prefix<Z, QuantTile<Z, true>>(g, s);
}
template <int DP, int S>
cudaError_t prefix_16(const Args& g, cudaStream_t s) {
  using Z = QuantSizes<__nv_bfloat16, DP, warps_of(DP, false), S>;
  return launch_prefix<Z, QuantTile<Z, false, true>, 3>(g, s);
}

}  // namespace

cudaError_t launch_own_q8(const Args& g, int dtype, cudaStream_t s) {
  if (dtype == DCK_F32) {
    if (g.DP == 256) return own<float, 256, 2, true>(g, s);
    return g.DP == 128 ? own<float, 128, 2, true>(g, s) : own<float, 64, 4, true>(g, s);
  }
  using T = __nv_bfloat16;
  if (g.DP == 256) return own<T, 256, 2, true>(g, s);
  if (g.DP == 128) return g.p.rows > 8 ? own<T, 128, 2, false>(g, s) : own<T, 128, 2, true>(g, s);
  return g.p.rows > 8 ? own<T, 64, 4, false>(g, s) : own<T, 64, 4, true>(g, s);
}

cudaError_t launch_prefix_q8(const Args& g, int dtype, cudaStream_t s) {
  if (dtype == DCK_F32)
    return g.DP == 256 ? prefix<float, 256, 2>(g, s) : g.DP == 128 ? prefix<float, 128, 2>(g, s) : prefix<float, 64, 4>(g, s);
  using T = __nv_bfloat16;
  if (g.DP == 256) return prefix<T, 256, 2>(g, s);
  if (g.DP == 128) return g.x.rows > 8 ? prefix_16<128, 2>(g, s) : prefix<T, 128, 2>(g, s);
  return g.x.rows > 8 ? prefix_16<64, 3>(g, s) : prefix<T, 64, 4>(g, s);
}

}  // namespace paged
}  // namespace dck

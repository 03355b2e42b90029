// Rotary positions (dck_rope) and the rotated append to a paged cache
// (dck_paged_append).  A pair (x, y) of a head's elements at position t becomes
//   m (x cos a - y sin a, x sin a + y cos a),  a = t w_i  (sin negated: the transpose).
// Bound by memory: each element is read and written once.
#include "paged.cuh"
#include "rope.cuh"

namespace dck {
namespace {

constexpr int kThreads = 256;

// A block per token; a thread per pair of elements.
template <typename T>
__global__ void __launch_bounds__(kThreads) rope_rows_kernel(const RopeLaunch a) {
  const int64_t i = blockIdx.x;
  const uint32_t pos = a.rope.rot ? (uint32_t)a.positions[i] : 0u;
  int64_t page = 0, off = 0;
  bool cached = false;
  if (a.slots) {
    const int64_t slot = a.slots[i];
    page = slot / a.page;
    off = slot - page * a.page;
    cached = slot >= 0 && page < a.n_pages;
    if (!cached && slot != -1 && threadIdx.x == 0) atomicOr(a.err, kErrBadRow);
  }
  for (int r = 0; r < a.n_rows; ++r) {
    const RopeRows& rows = a.rows[r];
    if (rows.cached && !cached) continue;
    const T* src = static_cast<const T*>(rows.src) + i * rows.src_tok;
    T* dst = static_cast<T*>(rows.dst) + (rows.cached ? page * rows.dst_page + off * rows.dst_tok : i * rows.dst_tok);
    const int half = rows.rotate ? a.rope.rot / 2 : 0;
    const int per = half + (a.d - 2 * half);  // pairs, then single elements
    for (int e = threadIdx.x; e < rows.heads * per; e += kThreads) {
      const int h = e / per, j = e - h * per;
      const T* sp = src + h * rows.src_head;
      T* dp = dst + h * rows.dst_head;
      if (j < half) {
        const int i0 = a.rope.layout == DCK_ROPE_HALF ? j : 2 * j, i1 = a.rope.layout == DCK_ROPE_HALF ? j + half : 2 * j + 1;
        float sn, cs;
        rope_sincos(a.rope.f[j], pos, sn, cs);
        sn *= a.rope.sign * a.rope.magnitude;
        cs *= a.rope.magnitude;
        const float x = to_f32(sp[i0]), y = to_f32(sp[i1]);
        dp[i0] = from_f32<T>(x * cs - y * sn);
        dp[i1] = from_f32<T>(x * sn + y * cs);
      } else {
        dp[j + half] = sp[j + half];
      }
    }
  }
}

}  // namespace

cudaError_t launch_rope_rows(const RopeLaunch& a, int dtype, cudaStream_t s) {
  if (dtype == DCK_F32) rope_rows_kernel<float><<<a.n_tok, kThreads, 0, s>>>(a);
  else rope_rows_kernel<__nv_bfloat16><<<a.n_tok, kThreads, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace dck

// Attention of one new token per sequence over a paged key-value cache
// (dck_paged_decode_attention).
#include <math_constants.h>

#include "paged.cuh"

namespace dck {
namespace {

constexpr int kWarps = 8;

// A block per (sequence, query head); warp w takes tokens w, w + 8, ...: the
// score by a shuffle sum over the head's elements, an online softmax per warp,
// the warps' sums joined in shared memory.
template <typename T>
__global__ void __launch_bounds__(kWarps * 32) paged_decode_kernel(const PagedDecodeArgs a) {
  constexpr int E = kMaxPagedHeadDim / 32;
  const int b = blockIdx.y, j = blockIdx.x, h = j / a.v.qpg, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int d = a.v.d;
  int L = a.seq_len[b];
  bool bad = L < 0 || L > a.max_len || ((int64_t)L + a.v.page - 1) / a.v.page > a.table_stride;
  if (bad) L = 0;
  const int first = a.window > 0 && L > a.window ? L - a.window : 0;
  const T* q = static_cast<const T*>(a.q) + b * a.q_stride + (int64_t)j * d;
  const T* kc = static_cast<const T*>(a.kc) + h * a.v.k_head;
  const T* vc = static_cast<const T*>(a.vc) + h * a.v.v_head;
  float qr[E], o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int i = e * 32 + lane;
    qr[e] = i < d ? to_f32(q[i]) : 0.f;
    o[e] = 0.f;
  }
  float m = -CUDART_INF_F, l = 0.f;
  for (int t = first + warp; t < L; t += kWarps) {
    const uint32_t c = a.v.by_page.div(t);
    const int page = a.table[b * a.table_stride + c], off = t - c * a.v.page;
    if (page < 0 || page >= a.v.n_pages) {
      bad = true;
      continue;
    }
    const T* kp = kc + page * a.v.k_page + off * a.v.k_tok;
    const T* vp = vc + page * a.v.v_page + off * a.v.v_tok;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = e * 32 + lane;
      if (i < d) s = fmaf(qr[e], to_f32(kp[i]), s);
    }
#pragma unroll
    for (int x = 16; x; x >>= 1) s += __shfl_xor_sync(~0u, s, x);
    s *= a.scale;
    if (a.softcap > 0.f) s = a.softcap * tanhf(s / a.softcap);
    const float mn = fmaxf(m, s), w = mn == -CUDART_INF_F ? 0.f : expf(s - mn), c0 = m == -CUDART_INF_F ? 0.f : expf(m - mn);
    l = l * c0 + w;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = e * 32 + lane;
      if (i < d) o[e] = o[e] * c0 + w * to_f32(vp[i]);
    }
    m = mn;
  }
  __shared__ float sm[kWarps], sl[kWarps], so[kWarps][kMaxPagedHeadDim];
  __shared__ int sbad;
  if (threadIdx.x == 0) sbad = 0;
  __syncthreads();
  if (bad && lane == 0) sbad = 1;
  if (lane == 0) sm[warp] = m, sl[warp] = l;
#pragma unroll
  for (int e = 0; e < E; ++e) so[warp][e * 32 + lane] = o[e];
  __syncthreads();
  if (sbad && threadIdx.x == 0) atomicOr(a.err, kErrBadSeq);
  float M = -CUDART_INF_F, total = 0.f;
  for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sm[w]);
  for (int w = 0; w < kWarps; ++w) total += sm[w] == -CUDART_INF_F ? 0.f : sl[w] * expf(sm[w] - M);
  for (int i = threadIdx.x; i < d; i += kWarps * 32) {
    float r = 0.f;
    for (int w = 0; w < kWarps; ++w) r += sm[w] == -CUDART_INF_F ? 0.f : so[w][i] * expf(sm[w] - M);
    r = sbad || total == 0.f ? 0.f : r / total;
    static_cast<T*>(a.out)[((int64_t)b * a.v.Hq + j) * d + i] = from_f32<T>(r);
  }
  if (a.lse && threadIdx.x == 0) a.lse[(int64_t)b * a.v.Hq + j] = sbad || total == 0.f ? -CUDART_INF_F : M + logf(total);
}

}  // namespace

size_t paged_decode_workspace(const PagedView&, int, int, int, int) { return 0; }

cudaError_t launch_paged_decode(const PagedDecodeArgs& a, int dtype, int, cudaStream_t s) {
  const dim3 grid(a.v.Hq, a.B);
  if (dtype == DCK_F32) paged_decode_kernel<float><<<grid, kWarps * 32, 0, s>>>(a);
  else paged_decode_kernel<__nv_bfloat16><<<grid, kWarps * 32, 0, s>>>(a);
  return hook_launched(a.hook, s);
}

}  // namespace dck

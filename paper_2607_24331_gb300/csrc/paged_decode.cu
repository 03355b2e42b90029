// Attention of one new token per sequence over a paged key-value cache
// (dck_paged_decode_attention).
//
// Mathematics: with s_t = scale <q, k_t> log2(e) the output is
// sum_t 2^(s_t - m) v_t / sum_t 2^(s_t - m) for any m; m is the running maximum, and
// sums over disjoint sets of tokens join as sum_i 2^(m_i - M) (.)_i, M = max m_i.
// One pass reads every key and value once: 4 flops per key-value element and query of
// the group against 2 bytes (bf16), so HBM is the bound up to some 100 queries per KV
// head.
//
// Split: query heads of one KV head form rows of one tile (up to 8, or 16); 1 to 8
// heads ("a head group") by 8 to 1 runs of 16 tokens are the warps of a CTA, so that
// neighbouring heads of a token, which lie side by side in most caches, are read
// together.  Every (head group, sequence) is cut into tiles; the flattened list of
// tiles is dealt to one CTA per SM in equal contiguous ranges, whatever the lengths.
// A (head group, sequence) that one CTA has whole is written by it; of any other each
// CTA stores its partial sums, at most two per CTA (its range's first and last), and
// a second launch joins them.
//
// Each warp runs a ring of its own (asynchronous 16-byte copies, no block barrier in
// the loop): page numbers are read one tile ahead of the copies, copies run ahead of
// the arithmetic over the ends of sequences.
//
// Where the sequences are few and short, the list, the partial sums in memory and the
// second launch would take longer than the attention: there a cluster of CTAs takes each
// (KV head, sequence), all warps of a CTA on runs of its tokens, and joins the CTAs' sums
// through distributed shared memory.
#include "paged_decode.cuh"

namespace dck {
namespace paged {
namespace {

// Joins the partial sums of what several CTAs share: a block per (entry, row).  Weights
// first (a thread per partial), then 16-byte loads of the partials by kJoinWarps warps'
// groups of lanes, several in flight.
constexpr int kJoinThreads = 256;
constexpr int kJoinBatch = 8;

template <typename T>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ Args g) {
  __shared__ float weight[kJoinThreads];
  __shared__ float2 warp_ml[kJoinThreads / 32];
  __shared__ int any_bad;
  __shared__ float4 sums[kJoinThreads];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, per = g.p.wh * g.p.rows, d = g.a.v.d;
  const int quads = g.DP / 4, lanes = kJoinThreads / quads, quad = tid % quads, turn = tid / quads;
  pdl_launch_dependents();
  pdl_wait();
  const int n = g.header->n_entries;
  for (int64_t x = blockIdx.x; x < (int64_t)n * per; x += gridDim.x) {
    const Entry e = g.entries[x / per];
    const int hr = (int)(x % per), h = hr / g.p.rows, r = hr - h * g.p.rows;
    const int group = e.pair / g.a.B, b = e.pair - group * g.a.B;
    const Queries qs = queries_of(g, group, h);
    if (r >= qs.count) continue;
    const int64_t out_row = (int64_t)b * g.a.v.Hq + qs.first + r;
    const auto row = [&](int i) { return ((int64_t)(2 * (e.c0 + i) + (i == 0 ? e.second : 0)) * g.p.wh + h) * g.p.rows + r; };
    const int parts = e.c1 - e.c0 + 1;
    float M = -CUDART_INF_F, total = 0.f;
    bool bad = false;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = 0; i0 < parts; i0 += kJoinThreads) {  // twice at most: CTAs are two per SM
      const int count = min(kJoinThreads, parts - i0);
      // the loads of the first partials go out before the weights are known
      float4 v[kJoinBatch];
      const auto fetch = [&](int i) {
#pragma unroll
        for (int k = 0; k < kJoinBatch; ++k)
          if (i + k * lanes < count && 4 * quad < d)
            v[k] = *reinterpret_cast<const float4*>(g.part_u + row(i0 + i + k * lanes) * g.DP + 4 * quad);
      };
      fetch(turn);
      float2 ml = make_float2(-CUDART_INF_F, 0.f);
      if (tid < count) ml = *reinterpret_cast<const float2*>(g.part_ml + 2 * row(i0 + tid));
      if (tid == 0) any_bad = 0;
      float m = ml.x;
#pragma unroll
      for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
      if (lane == 0) warp_ml[warp].x = m;
      __syncthreads();
      if (ml.y < 0.f) any_bad = 1;
      float top = M;
#pragma unroll
      for (int w = 0; w < kJoinThreads / 32; ++w) top = fmaxf(top, warp_ml[w].x);
      const float base = top == -CUDART_INF_F ? 0.f : top, w = exp2_approx(ml.x - base), before = exp2_approx(M - base);
      weight[tid] = w;
      float l = ml.y * w;
#pragma unroll
      for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(~0u, l, o);
      if (lane == 0) warp_ml[warp].y = l;
      __syncthreads();
      bad |= any_bad != 0;
      total *= before;
#pragma unroll
      for (int k = 0; k < kJoinThreads / 32; ++k) total += warp_ml[k].y;
      sum.x *= before, sum.y *= before, sum.z *= before, sum.w *= before;
      M = top;
      for (int i = turn; i < count; i += kJoinBatch * lanes) {
        if (i != turn) fetch(i);
#pragma unroll
        for (int k = 0; k < kJoinBatch; ++k)
          if (i + k * lanes < count && 4 * quad < d && weight[i + k * lanes] != 0.f) {
            const float c = weight[i + k * lanes];
            sum.x += v[k].x * c, sum.y += v[k].y * c, sum.z += v[k].z * c, sum.w += v[k].w * c;
          }
      }
      __syncthreads();
    }
    sums[tid] = sum;
    __syncthreads();
    if (turn == 0 && 4 * quad < d) {
      for (int k = 1; k < lanes; ++k) {
        const float4 y = sums[k * quads + quad];
        sum.x += y.x, sum.y += y.y, sum.z += y.z, sum.w += y.w;
      }
      const float f = bad || total == 0.f ? 0.f : 1.f / total;
      put4(static_cast<T*>(g.a.out) + out_row * d + 4 * quad,
           f == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(sum.x * f, sum.y * f, sum.z * f, sum.w * f),
           (reinterpret_cast<uintptr_t>(g.a.out) & 3) == 0);
      if (g.a.lse && quad == 0)
        g.a.lse[out_row] = bad || total == 0.f ? -CUDART_INF_F : (M + log2f(total)) * 0.693147180559945f;
    }
    __syncthreads();
  }
}

Plan plan_of(const PagedView& v, int dtype, int B, int max_len, int window, int sms) {
  Plan p;
  const int DP = padded_dim(v.d);
  const int most = dtype == DCK_BF16 && DP <= 128 && v.qpg > 8 ? 16 : 8;
  p.chunks = (v.qpg + most - 1) / most;
  p.rows = (v.qpg + p.chunks - 1) / p.chunks;
  p.by_chunks = divider((uint32_t)p.chunks);
  const int heads = v.Hkv * p.chunks;
  const int64_t span = window > 0 ? std::min(window, max_len) : max_len;
  // Clusters: one (head, sequence) each, as many CTAs as have a tile and one SM each
  p.cluster = 0;
  const int of_cluster = warps_of(DP, true) * run_of(dtype);
  const int64_t pairs = (int64_t)heads * std::max(B, 1), tiles = (span + of_cluster - 1) / of_cluster;
  if (pairs <= sms) {
    int c = 1;
    while (2 * c <= kMaxCluster && 2 * c * pairs <= sms && c < tiles) c *= 2;
    if (tiles <= kClusterTiles * c) p.cluster = c;
  }
  const int NW = warps_of(DP, p.cluster != 0);
  p.wh = p.cluster ? 1 : NW;
  while (heads % p.wh) p.wh /= 2;
  p.wt = NW / p.wh;
  p.groups = heads / p.wh;
  p.tile = p.wt * run_of(dtype);
  p.n_items = (int)std::min<int64_t>(kPerSm * sms, (int64_t)p.groups * std::max(B, 1) * ((span + p.tile - 1) / p.tile));
  return p;
}

size_t bytes_u(const Plan& p, int DP) { return align_up((size_t)2 * p.n_items * p.wh * p.rows * DP * sizeof(float), 256); }
size_t bytes_ml(const Plan& p) { return align_up((size_t)2 * p.n_items * p.wh * p.rows * 2 * sizeof(float), 256); }

}  // namespace
}  // namespace paged

using namespace paged;

size_t paged_decode_workspace(const PagedView& v, int dtype, int B, int max_len, int sms) {
  // windows only make calls smaller: fewer CTAs, and clusters where the whole length has them
  const Plan p = plan_of(v, dtype, std::max(B, 1), max_len, 0, sms);
  if (p.cluster) return 0;
  return 256 + align_up(p.n_items * sizeof(Entry), 256) + bytes_ml(p) + bytes_u(p, padded_dim(v.d));
}

cudaError_t launch_paged_decode(const PagedDecodeArgs& a, int dtype, int sms, cudaStream_t s) {
  Args g;
  g.a = a;
  g.p = plan_of(a.v, dtype, a.B, a.max_len, a.window, sms);
  g.DP = padded_dim(a.v.d);
  char* ws = static_cast<char*>(a.ws);
  g.header = reinterpret_cast<Header*>(ws);
  g.entries = reinterpret_cast<Entry*>(ws + 256);
  ws += 256 + align_up(g.p.n_items * sizeof(Entry), 256);
  g.part_ml = reinterpret_cast<float*>(ws);
  g.part_u = reinterpret_cast<float*>(ws + bytes_ml(g.p));
  cudaError_t e = dtype == DCK_F32 ? launch_f32(g, s) : launch_bf16(g, s);
  if (e != cudaSuccess || g.p.cluster) return e;
  // one tile per (head group, sequence) at most: nothing is shared
  if ((a.window > 0 ? std::min(a.window, a.max_len) : a.max_len) <= g.p.tile) return cudaSuccess;
  const int64_t work = (int64_t)g.p.n_items * g.p.wh * g.p.rows;
  const int grid = (int)std::min<int64_t>(work, 4 * sms);
  e = dtype == DCK_F32 ? launch_pdl(join_kernel<float>, grid, kJoinThreads, 0, s, g)
                       : launch_pdl(join_kernel<__nv_bfloat16>, grid, kJoinThreads, 0, s, g);
  if (e != cudaSuccess) return e;
  return hook_launched(a.hook, s);
}

}  // namespace dck

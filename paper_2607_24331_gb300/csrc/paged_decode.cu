// Attention of one new token per sequence over a paged key-value cache
// (dck_paged_decode_attention): work plan, join and launch.
//
// Mathematics: with s_t = scale <q, k_t> log2(e) the output is
// sum_t 2^(s_t - m) v_t / sum_t 2^(s_t - m) for any m; a reference m near the running
// maximum keeps the powers in range, and sums over disjoint sets of tokens join as
// sum_i 2^(m_i - M) (.)_i, M = max m_i.  One pass reads every key and value once: 4 flops
// per key-value element and query of the group against 2 bytes (bf16), so HBM is the bound
// (16 x 4096 tokens of 32 heads of 128: 1.07 GB in 152 us, 7.0 TB/s, 88% of the DRAM's peak
// cycles; the tensor pipe is at 19%, instruction issue at 28%).
//
// Split: query heads of one KV head form the rows of one tile of queries (up to 8, or 16); a
// CTA's warps are heads side by side (neighbours in most caches, so that they are read
// together) by runs of 16 tokens (fp32: 8).  Each warp runs a ring of its own of asynchronous
// 16-byte copies, without a block barrier in the loop; page numbers are read two tiles ahead
// of the copies, and copies run ahead of the arithmetic over the ends of sequences.
//
// Three ways to deal the work (plan_of):
//  - Ranges: every (head group, sequence) is cut into tiles, and the flattened list of tiles is
//    dealt to two CTAs per SM in equal contiguous ranges, whatever the lengths.  A (head group,
//    sequence) that one CTA has whole is written by it; of any other each CTA stores its
//    partial sums, at most two per CTA (its range's first and last), and a second launch joins
//    them.
//  - Clusters, where sequences are few and short and partial sums in memory and a second launch
//    would take longer than the attention: up to eight CTAs take each (KV head, sequence) and
//    join their sums through distributed shared memory.
//  - Whole: many short sequences, a CTA for each of some heads.
#include <cmath>

#include "paged_decode.cuh"

namespace dck {
namespace paged {
namespace {

// Joins the partial sums of what several CTAs share: per (entry, row) weights first,
// then 16-byte loads of the partials, several in flight.  Few entries of many partials:
// blocks of 256 threads list the entries that are any and take their rows in turn.
constexpr int kJoinThreads = 256;

template <typename T>
__device__ __forceinline__ void put_joined(const Args& g, int64_t out_row, int e, float4 sum, float m, float l, bool bad) {
  const bool none = bad || l == 0.f;
  const float f = 1.f / l;
  put4(static_cast<T*>(g.a.out) + out_row * g.a.v.d + e,
       none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(sum.x * f, sum.y * f, sum.z * f, sum.w * f),
       (reinterpret_cast<uintptr_t>(g.a.out) & 3) == 0);
  if (g.a.lse && e == 0) g.a.lse[out_row] = none ? -CUDART_INF_F : (m + log2f(l)) * 0.693147180559945f;
}

template <typename T>
__global__ void __launch_bounds__(kJoinThreads, 2)
    join_kernel(const __grid_constant__ Args g, const Divider by_per, const Divider by_rows) {
  constexpr int THREADS = kJoinThreads, kBatch = 8;  // kBatch: loads in flight per thread
  __shared__ float2 warp_ml[THREADS / 32];
  __shared__ float weight[THREADS];
  __shared__ int any_bad;
  __shared__ float4 sums[THREADS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, d = g.a.v.d, per = g.p.wh * g.p.rows;
  const int quads = g.DP / 4, lanes = THREADS / quads, quad = tid % quads, turn = tid / quads, el = 4 * quad;
  pdl_launch_dependents();
  pdl_wait();
  // the entries that are any, in the order of CTAs
  __shared__ uint16_t shared_by[kMaxItems];
  __shared__ int counts[THREADS / 32];
  int n_entries = 0;
  for (int i0 = 0; i0 < g.p.n_items; i0 += THREADS) {
    const int c = i0 + tid;
    const uint32_t any = __ballot_sync(~0u, c < g.p.n_items && g.entries[c].last >= 0);
    if (lane == 0) counts[warp] = __popc(any);
    __syncthreads();
    int before = n_entries;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
      if (w < warp) before += counts[w];
      n_entries += counts[w];
    }
    if (any >> lane & 1) shared_by[before + __popc(any & ((1u << lane) - 1))] = (uint16_t)c;
    __syncthreads();
  }
  const int n_rows = n_entries * per;
  for (int x = blockIdx.x; x < n_rows; x += gridDim.x) {
    const int nth = by_per.div(x), c0 = shared_by[nth], hr = x - nth * per, h = by_rows.div(hr), r = hr - h * g.p.rows;
    const Entry e = g.entries[c0];
    const Queries qs = queries_of(g, e.group, h);
    if (r >= qs.count) continue;
    const int64_t out_row = (int64_t)e.b * g.a.v.Hq + qs.first + r;
    const int parts = e.last - c0 + 1, stride = 2 * g.p.wh * g.p.rows;  // partial rows from CTA to CTA
    const int row0 = (2 * c0 * g.p.wh + h) * g.p.rows + r;
    const auto row = [&](int i) { return (int64_t)(row0 + i * stride + (i == 0 && e.second ? stride / 2 : 0)); };
    float M = -CUDART_INF_F, total = 0.f;
    bool bad = false;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = 0; i0 < parts; i0 += THREADS) {
      const int count = min(THREADS, parts - i0);
      // the loads of the first partials go out before the weights are known
      float4 v[kBatch];
      const auto fetch = [&](int i) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
          if (i + k * lanes < count && el < d)
            v[k] = *reinterpret_cast<const float4*>(g.part_u + row(i0 + i + k * lanes) * g.DP + el);
      };
      float2 ml = make_float2(-CUDART_INF_F, 0.f);
      if (tid < count) ml = *reinterpret_cast<const float2*>(g.part_ml + 2 * row(i0 + tid));
      fetch(turn);
      if (tid == 0) any_bad = 0;
      float m = ml.x;
#pragma unroll
      for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
      if (lane == 0) warp_ml[warp].x = m;
      __syncthreads();
      if (ml.y < 0.f) any_bad = 1;
      float top = M;
#pragma unroll
      for (int w = 0; w < THREADS / 32; ++w) top = fmaxf(top, warp_ml[w].x);
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
      for (int k = 0; k < THREADS / 32; ++k) total += warp_ml[k].y;
      sum.x *= before, sum.y *= before, sum.z *= before, sum.w *= before;
      M = top;
      for (int i = turn; i < count; i += kBatch * lanes) {
        if (i != turn) fetch(i);
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
          if (i + k * lanes < count && el < d && weight[i + k * lanes] != 0.f) {
            const float c = weight[i + k * lanes];
            sum.x += v[k].x * c, sum.y += v[k].y * c, sum.z += v[k].z * c, sum.w += v[k].w * c;
          }
      }
      __syncthreads();
    }
    if (lanes > 1) {
      sums[tid] = sum;
      __syncthreads();
    }
    if (turn == 0 && el < d) {
      for (int k = 1; k < lanes; ++k) {
        const float4 y = sums[k * quads + quad];
        sum.x += y.x, sum.y += y.y, sum.z += y.z, sum.w += y.w;
      }
      put_joined<T>(g, out_row, el, sum, M, total, bad);
    }
    __syncthreads();
  }
}

// Many entries of few partials: a warp per CTA's entry and row, whether there is one or
// not, two warps a block, so that all are on the GPU at once.
constexpr int kFewThreads = 64;

template <typename T>
__global__ void __launch_bounds__(kFewThreads, 16)
    join_few_kernel(const __grid_constant__ Args g, const Divider by_per, const Divider by_rows) {
  constexpr int kBatch = 4;
  const int lane = threadIdx.x & 31, d = g.a.v.d, per = g.p.wh * g.p.rows;
  const int x = (blockIdx.x * kFewThreads + threadIdx.x) / 32;
  pdl_launch_dependents();
  pdl_wait();
  if (x >= g.p.n_items * per) return;
  const int c0 = by_per.div(x), hr = x - c0 * per, h = by_rows.div(hr), r = hr - h * g.p.rows;
  const Entry e = g.entries[c0];
  if (e.last < 0) return;
  const Queries qs = queries_of(g, e.group, h);
  if (r >= qs.count) return;
  const int64_t out_row = (int64_t)e.b * g.a.v.Hq + qs.first + r;
  const int parts = e.last - c0 + 1, stride = 2 * per, row0 = (2 * c0 * g.p.wh + h) * g.p.rows + r;
  const auto row = [&](int i) { return (int64_t)(row0 + i * stride + (i == 0 && e.second ? per : 0)); };
  const int quads = min(g.DP / 4, 32), lanes = 32 / quads, turn = lane / quads;
  for (int q0 = 0; q0 < g.DP / 4; q0 += quads) {  // once, but twice for heads above 128
    const int el = 4 * (q0 + lane % quads);
    float M = -CUDART_INF_F, total = 0.f;
    bool bad = false;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = 0; i0 < parts; i0 += 32) {
      const int count = min(32, parts - i0);
      float4 v[kBatch];
      const auto fetch = [&](int i) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
          if (i + k * lanes < count && el < d)
            v[k] = *reinterpret_cast<const float4*>(g.part_u + row(i0 + i + k * lanes) * g.DP + el);
      };
      float2 ml = make_float2(-CUDART_INF_F, 0.f);
      if (lane < count) ml = *reinterpret_cast<const float2*>(g.part_ml + 2 * row(i0 + lane));
      fetch(turn);
      float top = fmaxf(M, ml.x);
#pragma unroll
      for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
      const float base = top == -CUDART_INF_F ? 0.f : top, w = exp2_approx(ml.x - base), before = exp2_approx(M - base);
      float l = ml.y * w;
#pragma unroll
      for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(~0u, l, o);
      bad |= __any_sync(~0u, ml.y < 0.f) != 0;
      total = total * before + l;
      sum.x *= before, sum.y *= before, sum.z *= before, sum.w *= before;
      M = top;
      for (int i = 0; i < count; i += kBatch * lanes) {
        if (i) fetch(i + turn);
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
          const int p = i + turn + k * lanes;
          const float c = __shfl_sync(~0u, w, p & 31);
          if (p < count && el < d && c != 0.f)
            sum.x += v[k].x * c, sum.y += v[k].y * c, sum.z += v[k].z * c, sum.w += v[k].w * c;
        }
      }
    }
    for (int k = quads; k < 32; k <<= 1) {  // the lanes that share a quad of elements
      sum.x += __shfl_xor_sync(~0u, sum.x, k);
      sum.y += __shfl_xor_sync(~0u, sum.y, k);
      sum.z += __shfl_xor_sync(~0u, sum.z, k);
      sum.w += __shfl_xor_sync(~0u, sum.w, k);
    }
    if (turn == 0 && el < d) put_joined<T>(g, out_row, el, sum, M, total, bad);
  }
}

template <typename T>
cudaError_t launch_join(const Args& g, int sms, cudaStream_t s) {
  const int per = g.p.wh * g.p.rows, rows = g.p.n_items * per;
  // partials per entry, on average, where all sequences are alike: 16 or more
  cudaError_t e = (int64_t)g.p.groups * g.a.B * 16 <= g.p.n_items
                      ? launch_pdl(join_kernel<T>, std::min(rows, 4 * sms), kJoinThreads, 0, s, g, divider(per),
                                   divider(g.p.rows))
                      : launch_pdl(join_few_kernel<T>, (rows * 32 + kFewThreads - 1) / kFewThreads, kFewThreads, 0, s, g,
                                   divider(per), divider(g.p.rows));
  return e == cudaSuccess ? hook_launched(g.a.hook, s) : e;
}

// Which of the three ways a call takes: the one of the least time by a model in us, fitted
// to 650 measured calls (six head layouts, bf16 and fp32, 1 to 128 sequences of 16 to 4096
// tokens, half of them ragged 16-fold); its choice is 1.4% off the best of the three on
// average.  The host knows a bound on the lengths only, so a way is judged by the geometric
// mean of its times for sequences of that length and for ragged ones, 0.34 of it on average.
// On 8-bit caches the figures are fitted to 148 calls of their own (the choice 0.5% off the best on average).
// Measured, ranges / clusters / whole, 32 query heads on 8 KV heads of 128 in bf16:
//   1 x 128   6.9 /  4.6 /  4.4     16 x 512       13.6 /  8.4 / 10.5    64 x 256        21 / - / 15
//   1 x 1024  9.1 /  6.4 / 14.6     16 x 4096      49.8 / 46.3 / 56      64 x 2048       87 / - / 83
//   4 x 4096 18.6 / 17.4 / 58       16 x 128..2048 17.3 / 16.1 / 21      64 x 128..2048  37 / - / 44
// With `ranges` always by those.
Plan plan_of(const PagedView& v, DecodeKind kind, int B, int max_len, int window, int sms, bool ranges = false) {
  Plan p;
  const int DP = padded_dim(v.d), dtype = kind.dtype;
  const int most = dtype == DCK_BF16 && DP <= 128 && v.qpg > 8 ? 16 : 8;
  p.chunks = (v.qpg + most - 1) / most;
  p.rows = (v.qpg + p.chunks - 1) / p.chunks;
  p.by_chunks = divider((uint32_t)p.chunks);
  p.alike = v.k_page_b == v.v_page_b && v.k_tok_b == v.v_tok_b && v.k_head_b == v.v_head_b;
  const int el = kind.quant ? 1 : dtype == DCK_BF16 ? 2 : 4;  // bytes of a cached element
  const int heads = v.Hkv * p.chunks, few = warps_of(DP, false), many = warps_of(DP, true), run = run_of(kind);
  const int64_t span = window > 0 ? std::min(window, max_len) : max_len, pairs = (int64_t)heads * std::max(B, 1);
  const auto tiles_of = [&](int tokens) { return (span + tokens - 1) / tokens; };
  int wide = few;  // heads side by side in a CTA, at most
  while (heads % wide) wide /= 2;

  const int row = DP * el, slots = kPerSm * sms;
  const double step = kind.quant ? (DP == 64 ? 1.55 : DP == 128 ? 2.15 : 2.95)
                                 : row <= 128 ? 0.45 : row == 256 ? 0.65 : row == 512 ? 0.95 : 1.37;  // a warp's run of tokens
  const double bytes = 1.07 * 2. * B * span * v.Hkv * (v.d * el + (kind.quant ? 4 : 0)) / 6.8e6;
  // (product of the two times) of a way with a fixed part and the longest CTA's part
  const auto times = [&](double fixed, double longest) {
    return (fixed + std::max(longest, bytes)) * (fixed + std::max(longest, 0.34 * bytes));
  };
  const double fixed = (kind.quant ? 10.5 : dtype == DCK_BF16 ? 7.5 : 12.7) + 0.45 * std::max(0., (double)pairs / wide / slots - 1) -
                       (span <= few / wide * run ? 2.8 : 0);
  // (a CTA's tiles in ranges take longer than HBM does for 8-bit rows only; fewer of them where sequences are shorter)
  const double ranged = kind.quant ? 1.4 * step * std::ceil((double)(pairs / wide * tiles_of(few / wide * run)) / slots) : 0;
  double best = (fixed + std::max(ranged, bytes)) * (fixed + 0.34 * std::max(ranged, bytes));
  if (ranges) best = 0;
  p.cluster = 0;
  p.warps = few;
  p.wh = wide;
  // clusters of c (not all SMs take part in those of 8: 15 of them on 152)
  for (int c = 1; c <= kMaxCluster && c * pairs <= sms - (c > 1 ? 4 * c : 0); c *= 2) {
    const double t = times(c > 1 ? (kind.quant ? 4.7 : 5.4) : 4.3, tiles_of(many * run * c) * step);
    if (t < best) best = t, p.cluster = c, p.warps = many, p.wh = 1;
  }
  // a CTA of `few` warps for w heads of a sequence
  for (int w = 1; w <= wide; w *= 2) {
    const double waves = std::ceil((double)(pairs / w) / slots);
    const double t = times(4.1 * (1 + 0.43 * (waves - 1)), waves * tiles_of(few / w * run) * step * (kind.quant ? 1.03 : 0.89));
    if (t < best) best = t, p.cluster = 1, p.warps = few, p.wh = w;
  }
  p.wt = p.warps / p.wh;
  p.groups = heads / p.wh;
  p.tile = p.wt * run;
  p.by_tile = divider((uint32_t)p.tile);
  // CTAs of tiles dealt in ranges (whichever way this call takes: it sizes the workspace)
  p.n_items = (int)std::min<int64_t>(std::min(slots, kMaxItems), pairs / wide * tiles_of(few / wide * run));
  p.part_rows = wide * p.rows;
  return p;
}

size_t bytes_entries(const Plan& p) { return align_up(p.n_items * sizeof(Entry), 256); }
size_t bytes_ml(const Plan& p) { return align_up((size_t)2 * p.n_items * p.part_rows * 2 * sizeof(float), 256); }
size_t bytes_u(const Plan& p, int DP) { return align_up((size_t)2 * p.n_items * p.part_rows * DP * sizeof(float), 256); }

}  // namespace

Plan range_plan(const PagedView& v, DecodeKind kind, int B, int max_len, int sms) {
  return plan_of(v, kind, B, max_len, 0, sms, true);
}

}  // namespace paged

using namespace paged;

size_t paged_decode_workspace(const PagedView& v, DecodeKind kind, int B, int max_len, int sms) {
  const Plan p = plan_of(v, kind, std::max(B, 1), max_len, 0, sms);  // a window only takes CTAs away
  return bytes_entries(p) + bytes_ml(p) + bytes_u(p, padded_dim(v.d));
}

cudaError_t launch_paged_decode(const PagedDecodeArgs& a, DecodeKind kind, int sms, cudaStream_t s) {
  Args g;
  g.a = a;
  g.p = plan_of(a.v, kind, a.B, a.max_len, a.window, sms);
  g.DP = padded_dim(a.v.d);
  g.score.set(a.scale, a.softcap);
  const int dtype = kind.dtype, el = dtype == DCK_F32 ? 4 : 2;
  g.p.q_copied = reinterpret_cast<uintptr_t>(a.q) % 16 == 0 && a.q_stride * el % 16 == 0;
  char* ws = static_cast<char*>(a.ws);
  g.entries = reinterpret_cast<Entry*>(ws);
  ws += bytes_entries(g.p);
  g.part_ml = reinterpret_cast<float*>(ws);
  g.part_u = reinterpret_cast<float*>(ws + bytes_ml(g.p));
  cudaError_t e = kind.quant ? launch_q8(g, dtype, s) : dtype == DCK_F32 ? launch_f32(g, s) : launch_bf16(g, s);
  if (e != cudaSuccess || g.p.cluster) return e;
  // one tile per (head group, sequence) at most: nothing is shared
  if ((a.window > 0 ? std::min(a.window, a.max_len) : a.max_len) <= g.p.tile) return cudaSuccess;
  return dtype == DCK_F32 ? launch_join<float>(g, sms, s) : launch_join<__nv_bfloat16>(g, sms, s);
}

}  // namespace dck

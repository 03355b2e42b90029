// Attention of rows that share the beginnings of their sequences (dck_paged_shared_attention,
// dck_quant_shared_attention): plan, work split and launch.
//
// Mathematics: sums over disjoint sets of tokens join as sum_i 2^(m_i - M) (.)_i (paged_decode.cu), so a row's sums over
// the tokens that its group shares may be formed elsewhere than those over its own.  The shared tokens are
// attended to once per block of queries of the group's rows, whose queries on a KV head are the rows of one product;
// each row's own tokens by a CTA or cluster as in a call by single rows, which then adds what the first left.
//
// Which tokens: those that all the rows that take part see, so that the first part needs no mask (and what a row may not
// see cannot reach it, infinities and NaN included).  A group's rows take part if they see nearly as many of the
// shared tokens as the longest does, at most 256 and the number of rows fewer: a chunk's tokens all do,
// and attend one by one to those at its end, while a row far behind does by itself what it sees.
//
// Three launches: the plan (one block), the shared part, the own tokens.  The last starts while the second runs.
#include <cmath>

#include "paged_decode.cuh"

namespace dck {
namespace paged {
namespace {

constexpr int kPlanThreads = 512;

// A row's first visible token, those it sees of the shared ones (0: none, or a bad length), and its length.
struct RowView {
  int first, eff, len;
};
__device__ __forceinline__ RowView row_view(const PagedDecodeArgs& a, int b, int shared) {
  RowView r;
  bool bad;
  const int span = visible(a, b, r.first, bad);
  r.len = bad ? 0 : span + r.first;
  r.eff = min(r.len, shared);
  return r;
}

// A subgroup of LANES threads per group of rows at a time.
template <int LANES>
__device__ __forceinline__ void plan_group(const Args& g, int at, bool there) {
  const PagedDecodeArgs& a = g.a;
  const Prefix& x = g.x;
  const int lane = threadIdx.x % LANES;
  const int start = there ? a.group_start[at] : 0, end = there ? a.group_start[at + 1] : 0;
  const int said = there ? a.shared_len[at] : 0, shared = max(said, 0), rows = end - start;
  if (said < 0 && lane == 0) atomicOr(a.err, kErrBadSeq);
  // the longest row, the first of them
  int longest = 0, row = start;
  for (int b = start + lane; b < end; b += LANES) {
    const RowView r = row_view(a, b, shared);
    if (r.len > longest) longest = r.len, row = b;
    x.group_of[b] = at;
  }
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1) {
    const int n = __shfl_xor_sync(~0u, longest, o), b = __shfl_xor_sync(~0u, row, o);
    if (n > longest || (n == longest && b < row)) longest = n, row = b;
  }
  const int most = min(longest, shared), least = max(1, most - 256 - rows);
  int last = most, first = 0;
  for (int b = start + lane; b < end; b += LANES) {
    const RowView r = row_view(a, b, shared);
    if (r.eff >= least) last = min(last, r.eff), first = max(first, r.first);
  }
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1) {
    last = min(last, __shfl_xor_sync(~0u, last, o));
    first = max(first, __shfl_xor_sync(~0u, first, o));
  }
  if (rows < 2 || last <= first) last = first = 0;
  if (!there || lane) return;
  GroupPlan p;
  p.start = start;
  p.rows = rows;
  p.first = first;
  p.end = last;
  p.table = row;
  p.tiles = (last - first + x.tile - 1) / x.tile;
  p.blocks = (int)(((int64_t)rows * a.v.qpg + x.rows - 1) / x.rows);
  p.units = p.queries = p.bad = p.pad[0] = p.pad[1] = 0;
  x.groups[at] = p;
}

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const __grid_constant__ Args g) {
  const PagedDecodeArgs& a = g.a;
  const Prefix& x = g.x;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = x.n_groups;
  __shared__ int64_t sums[2][kPlanThreads / 32];
  pdl_launch_dependents();
  pdl_wait();
  int wrong = 0;
  for (int i = tid; i < n; i += kPlanThreads) {
    const int s = a.group_start[i], e = a.group_start[i + 1];
    wrong |= s < 0 || e < s || e > a.B || (i == 0 && s != 0) || (i == n - 1 && e != a.B);
  }
  wrong = __syncthreads_or(wrong);
  int64_t units = 0, queries = 0;
  if (!wrong) {
    if (n <= 2 * kPlanThreads / 32) {
      for (int i = warp; i < n; i += kPlanThreads / 32) plan_group<32>(g, i, true);
    } else {
      for (int i = 0; i < n; i += kPlanThreads / 8) plan_group<8>(g, i + tid / 8, i + tid / 8 < n);
    }
    __syncthreads();
    const int head_groups = a.v.Hkv / x.wh;
    for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
      const int i = i0 + tid;
      const int64_t mine = i < n ? (int64_t)x.groups[i].tiles * x.groups[i].blocks * head_groups : 0;
      const int64_t q = i < n ? (int64_t)x.groups[i].rows * a.v.qpg : 0;
      int64_t u = mine, v = q;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(~0u, u, o), z = __shfl_up_sync(~0u, v, o);
        if (lane >= o) u += y, v += z;
      }
      if (lane == 31) sums[0][warp] = u, sums[1][warp] = v;
      __syncthreads();
      int64_t before = units, ahead = queries;
      for (int w = 0; w < kPlanThreads / 32; ++w) {
        if (w < warp) before += sums[0][w], ahead += sums[1][w];
        units += sums[0][w], queries += sums[1][w];
      }
      if (i < n) {
        x.groups[i].units = (int)min(before + u - mine, (int64_t)kUnitLimit);
        x.groups[i].queries = (int)(ahead + v - q);
      }
      __syncthreads();
    }
    if (units > kUnitLimit) wrong = 1;
  }
  if (tid == 0) {
    if (wrong) atomicOr(a.err, kErrBadSeq);
    x.all->units = wrong ? 0 : (int)units;
    x.all->bad = wrong;
  }
}

// How the shared part of a call is laid out.
struct Layout {
  bool tc;  // on tcgen05
  int rows, wh, tile, n_items;
};
Layout layout_of(const PagedView& v, DecodeKind kind, int B, int n_groups, int sms) {
  Layout l;
  const int DP = padded_dim(v.d), warps = warps_of(DP, false);
  const int64_t queries = (int64_t)v.qpg * B / std::max(n_groups, 1);  // of a group, on average
  l.tc = kind.dtype == DCK_BF16 && !kind.quant && DP <= 128 && queries > 16;
  if (l.tc) {
    l.rows = 128;
    l.tile = 64;
    l.wh = 1;
    l.n_items = sms;
    return l;
  }
  l.rows = kind.dtype == DCK_BF16 && DP <= 128 && queries > 8 ? 16 : 8;
  l.wh = warps;
  while (v.Hkv % l.wh) l.wh /= 2;
  l.tile = warps / l.wh * run_of(kind);
  l.n_items = std::min(kPerSm * sms, kMaxItems);
  return l;
}

size_t bytes_all(int B) { return 256 + align_up((size_t)B * sizeof(GroupPlan), 256) + align_up((size_t)B * sizeof(int), 256); }
// (a CTA leaves 128 rows of an item, or each of two on an SM 16 for up to four heads)
int64_t partial_rows(const PagedView& v, int B, int sms) {
  return (int64_t)B * v.Hq + (int64_t)sms * 128;
}

}  // namespace
}  // namespace paged

using namespace paged;

size_t paged_shared_workspace(const PagedView& v, DecodeKind kind, int B, int max_len, int max_own, int sms) {
  const int64_t rows = partial_rows(v, std::max(B, 1), sms);
  return std::max(paged_decode_workspace(v, kind, B, max_len, sms),
                  bytes_all(std::max(B, 1)) + align_up((size_t)rows * 2 * sizeof(float), 256) +
                      align_up((size_t)rows * padded_dim(v.d) * sizeof(float), 256));
}

cudaError_t launch_paged_shared(const PagedDecodeArgs& a, DecodeKind kind, int sms, cudaStream_t s) {
  Args g = {};
  g.a = a;
  g.p = own_plan(a.v, kind, a.B, std::min(a.max_own, a.max_len), a.window, sms);
  g.DP = padded_dim(a.v.d);
  g.score.set(a.scale, a.softcap);
  const int el = kind.dtype == DCK_F32 ? 4 : 2;
  g.p.q_copied = reinterpret_cast<uintptr_t>(a.q) % 16 == 0 && a.q_stride * el % 16 == 0;
  const Layout l = layout_of(a.v, kind, a.B, a.n_groups, sms);
  char* ws = static_cast<char*>(a.ws);
  g.x.all = reinterpret_cast<Shared0*>(ws);
  g.x.groups = reinterpret_cast<GroupPlan*>(ws + 256);
  g.x.group_of = reinterpret_cast<int*>(ws + 256 + align_up((size_t)a.B * sizeof(GroupPlan), 256));
  ws += bytes_all(a.B);
  g.x.part_ml = reinterpret_cast<float*>(ws);
  g.x.part_u = reinterpret_cast<float*>(ws + align_up((size_t)partial_rows(a.v, a.B, sms) * 2 * sizeof(float), 256));
  g.x.n_groups = a.n_groups;
  g.x.n_items = l.n_items;
  g.x.rows = l.rows;
  g.x.wh = l.wh;
  g.x.tile = l.tile;
  g.x.by_qpg = divider((uint32_t)a.v.qpg);
  cudaError_t e = launch_pdl(plan_kernel, 1, kPlanThreads, 0, s, g);
  if (e == cudaSuccess) e = hook_launched(a.hook, s);
  // heads of the shared part are KV heads themselves
  Args h = g;
  h.p.chunks = 1;
  h.p.by_chunks = divider(1);
  h.p.wh = l.wh;
  if (e == cudaSuccess)
    e = l.tc ? launch_prefix_tc(h, s) : kind.quant ? launch_prefix_q8(h, kind.dtype, s) : kind.dtype == DCK_F32 ? launch_prefix_f32(h, s) : launch_prefix_bf16(h, s);
  if (e == cudaSuccess)
    e = kind.quant ? launch_own_q8(g, kind.dtype, s) : kind.dtype == DCK_F32 ? launch_own_f32(g, s) : launch_own_bf16(g, s);
  return e;
}

}  // namespace dck

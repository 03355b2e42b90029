// Attention of rows that share the beginnings of their sequences (dck_paged_shared_attention,
// dck_quant_shared_attention): plan, work split and launch.
//
// Mathematics: sums over disjoint sets of tokens join as sum_i 2^(m_i - M) (.)_i (paged_decode.cu), so a row's sums over
// the tokens that its group shares may be formed elsewhere than those over its own.  The shared tokens are
// attended to once per block of queries of the group's rows, whose queries on a KV head are the rows of one product;
// each row's own tokens by CTAs that tiles are dealt to in ranges, as in a call by single rows; a launch of its own joins what both
// left.
//
// Which tokens: those that all the rows that take part see, so that the first part needs no mask (and what a row may not
// see cannot reach it, infinities and NaN included).  A group's rows take part if they see nearly as many of the
// shared tokens as the longest does, at most 256 and the number of rows fewer: a chunk's tokens all do,
// and attend one by one to those at its end, while a row far behind does by itself what it sees.
//
// Four launches: the plan (one block), the shared part, the own tokens (which do not wait for that: they take SMs as its CTAs
// end), the join.
#include <cmath>

#include "paged_shared.cuh"

namespace dck {
namespace paged {
namespace {

constexpr int kPlanThreads = 512;
constexpr int kLeastPartLog2 = 5, kMostPartLog2 = 7;  // rows that are planned together, at most (by layout_of)

// What the plan works on: its records, in shared memory where they fit (kFew groups and rows), else where they go; tiles
// of all groups, and of all rows, before each.
constexpr int kFew = kPlanThreads;
struct PlanState {
  GroupPlan* groups;
  RowPlan* own;
  int *units, *tiles;  // [n_parts + 1], [B + 1]
};

// A row's first visible token, those it sees of the shared ones (0: none), and its length. A bad row, by its length or by
// more tokens of its own than the call says, has none at all: it may not decide for its group, by its length or by its table.
struct RowView {
  int first, eff, len;
  bool bad;
};
__device__ __forceinline__ RowView row_view(const PagedDecodeArgs& a, int len, int shared) {
  RowView r;
  const int span = visible_of(a, len, r.first, r.bad);
  r.len = span + r.first;
  r.eff = min(r.len, shared);
  r.bad |= r.len - max(r.eff, r.first) > a.max_own;
  if (r.bad) r.first = r.len = r.eff = 0;
  return r;
}

// Group `at` of the call, its first row, its rows and their parts; `wrong`: d_group_start is not as it must be (no rows).
struct GroupView {
  int start, rows, parts;
  bool wrong;
};
// Leaves a place empty that no part has, between this group's and the next one's (`speaks`: in one thread).
__device__ __forceinline__ GroupView group_view(const Args& g, const PlanState& s, int at, bool speaks) {
  const int start = g.a.group_start[at], end = g.a.group_start[at + 1];
  GroupView v;
  v.wrong = start < 0 || end < start || end > g.a.B || (at == 0 && start != 0) || (at == g.x.n_groups - 1 && end != g.a.B);
  v.start = start;
  v.rows = v.wrong ? 0 : end - start;
  const int log2 = g.x.most_rows_log2;
  v.parts = (v.rows + (1 << log2) - 1) >> log2;
  const int past = at + (start >> log2) + v.parts;
  if (speaks && !v.wrong && past < at + 1 + (end >> log2)) s.units[past] = s.groups[past].tiles = 0;
  return v;
}

// Part `part` of group `at` (where `there`), planned by LANES threads; all groups of them in a warp at once.
template <int LANES>
__device__ __forceinline__ void plan_part(const Args& g, const PlanState& s, int at, const GroupView& whole, int part, bool there) {
  const PagedDecodeArgs& a = g.a;
  const Prefix& x = g.x;
  const int lane = threadIdx.x % LANES;
  there = there && part < whole.parts;
  int start = 0, end = 0, said = 0;
  if (there) {
    start = whole.start, end = start + whole.rows;
    if (whole.parts > 1) {
      start = whole.start + part * whole.rows / whole.parts;
      end = whole.start + (part + 1) * whole.rows / whole.parts;
    }
    said = a.shared_len[at];
    if (said < 0 && lane == 0) atomicOr(a.err, kErrBadSeq);
  }
  const int rows = end - start, shared = rows > 1 ? max(said, 0) : 0;
  // all its rows' lengths at once, by a warp: a read takes longer than the rest of a row
  constexpr int kKept = LANES == 32 ? (1 << kMostPartLog2) / 32 : 1;
  int kept[kKept];
#pragma unroll
  for (int i = 0; i < kKept; ++i) kept[i] = start + lane + i * LANES < end ? a.seq_len[start + lane + i * LANES] : 0;
  const auto each_row = [&](auto f) {
    if (LANES == 32) {
#pragma unroll
      for (int i = 0; i < kKept; ++i)
        if (start + lane + i * LANES < end) f(start + lane + i * LANES, kept[i]);
    } else {
      for (int b = start + lane; b < end; b += LANES) f(b, b == start + lane ? kept[0] : a.seq_len[b]);
    }
  };
  // the longest row, the first of them
  int longest = 0, row = start;
  each_row([&](int b, int len) {
    const RowView r = row_view(a, len, shared);
    if (r.len > longest) longest = r.len, row = b;
  });
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1) {
    const int n = __shfl_xor_sync(~0u, longest, o), b = __shfl_xor_sync(~0u, row, o);
    if (n > longest || (n == longest && b < row)) longest = n, row = b;
  }
  const int most = min(longest, shared), least = max(1, most - 256 - rows);
  int last = most, first = 0;
  each_row([&](int, int len) {
    const RowView r = row_view(a, len, shared);
    if (r.eff >= least) last = min(last, r.eff), first = max(first, r.first);
  });
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1) {
    last = min(last, __shfl_xor_sync(~0u, last, o));
    first = max(first, __shfl_xor_sync(~0u, first, o));
  }
  if (rows < 2 || last <= first) last = first = 0;
  const int64_t blocks = ((int64_t)rows * a.v.qpg + x.rows - 1) / x.rows;
  const int slot = at + (whole.start >> x.most_rows_log2) + part;
  // what each row has of its own
  each_row([&](int b, int len) {
    const RowView r = row_view(a, len, shared);
    RowPlan own;
    const bool takes_part = last > first && r.eff >= last && r.first <= first;
    if (r.bad) atomicOr(a.err, kErrBadSeq);
    own.state = r.bad ? kEmpty : 0;
    own.group = takes_part ? slot : -1;
    own.skip_at = takes_part ? first : 0;
    own.skip = takes_part ? last - first : 0;
    own.first = r.first;
    own.end = r.len - own.skip;
    own.start = start;
    own.rows = rows;
    own.blocks = (int)blocks;
    s.own[b] = own;
    s.tiles[b] = max(1, (own.end - own.first + g.p.tile - 1) / g.p.tile);
  });
  if (!there || lane) return;
  GroupPlan p;
  p.start = start;
  p.rows = rows;
  p.first = first;
  p.end = last;
  p.table = row;
  p.tiles = (last - first + x.tile - 1) / x.tile;
  p.blocks = (int)blocks;
  p.bad = 0;
  s.groups[slot] = p;
  s.units[slot] = (int)min((int64_t)p.tiles * blocks * a.v.Hkv, (int64_t)kUnitLimit + 1);
}

// In place of units[0 .. n - 1] and tiles[0 .. m - 1] the sums of all before each, and of all in units[n] and tiles[m]:
// kUnitLimit + 1 at most.  Called by the whole block.
__device__ __forceinline__ void sum_before(const PlanState& s, int n, int m, int64_t (&scratch)[2][kPlanThreads / 32]) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int64_t base[2] = {0, 0};
  for (int i0 = 0; i0 < max(n, m); i0 += kPlanThreads) {
    const int i = i0 + tid;
    const int64_t mine[2] = {i < n ? s.units[i] : 0, i < m ? s.tiles[i] : 0};
    int64_t t[2] = {mine[0], mine[1]};
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int64_t y = __shfl_up_sync(~0u, t[k], o);
        if (lane >= o) t[k] += y;
      }
    if (lane == 31) scratch[0][warp] = t[0], scratch[1][warp] = t[1];
    __syncthreads();
    const int warps = min(kPlanThreads, max(n, m) - i0 + 31) / 32;
    int64_t before[2] = {base[0], base[1]};
    for (int w = 0; w < warps; ++w)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int64_t y = scratch[k][w];
        if (w < warp) before[k] += y;
        base[k] += y;
      }
    if (i < n) s.units[i] = (int)min(before[0] + t[0] - mine[0], (int64_t)kUnitLimit + 1);
    if (i < m) s.tiles[i] = (int)min(before[1] + t[1] - mine[1], (int64_t)kUnitLimit + 1);
    __syncthreads();
  }
  if (tid == 0) {
    s.units[n] = (int)min(base[0], (int64_t)kUnitLimit + 1);
    s.tiles[m] = (int)min(base[1], (int64_t)kUnitLimit + 1);
  }
  __syncthreads();
}
// The last i of 0 .. n - 1 with v[i] <= u.
__device__ __forceinline__ int last_of(const int* v, int n, int u) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (v[mid] <= u) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

size_t plan_bytes(int groups, int rows) {
  const bool few = groups <= kFew && rows <= kFew;
  return (few ? groups * sizeof(GroupPlan) + rows * sizeof(RowPlan) : 0) + sizeof(int) * (groups + 1 + rows + 1);
}

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const __grid_constant__ Args g) {
  const PagedDecodeArgs& a = g.a;
  const Prefix& x = g.x;
  const int tid = threadIdx.x, n = x.n_groups, parts = x.n_parts;
  extern __shared__ __align__(16) uint8_t plan_memory[];
  __shared__ int64_t scratch[2][kPlanThreads / 32];
  pdl_launch_dependents();
  pdl_wait();
  const bool few = parts <= kFew && a.B <= kFew;
  PlanState s;
  uint8_t* at = plan_memory;
  s.groups = few ? reinterpret_cast<GroupPlan*>(at) : x.groups;
  if (few) at += parts * sizeof(GroupPlan);
  s.own = few ? reinterpret_cast<RowPlan*>(at) : x.own;
  if (few) at += a.B * sizeof(RowPlan);
  s.units = reinterpret_cast<int*>(at);
  s.tiles = s.units + parts + 1;
  int wrong = 0;
  if (n < 16 && n << (x.most_rows_log2 + 1) <= a.B) {  // few groups of many parts: a warp per part
    for (int i = 0; i < n; ++i) {
      const GroupView v = group_view(g, s, i, tid == 0);
      wrong |= v.wrong;
      for (int k = tid / 32; k < v.parts; k += kPlanThreads / 32) plan_part<32>(g, s, i, v, k, true);
    }
  } else if (n <= 2 * kPlanThreads / 32) {  // a warp per group
    for (int i = tid / 32; i < n; i += kPlanThreads / 32) {
      const GroupView v = group_view(g, s, i, tid % 32 == 0);
      wrong |= v.wrong;
      for (int k = 0; k < v.parts; ++k) plan_part<32>(g, s, i, v, k, true);
    }
  } else {
    for (int i0 = 0; i0 < n; i0 += kPlanThreads / 8) {
      const int i = i0 + tid / 8;
      const GroupView v = i < n ? group_view(g, s, i, tid % 8 == 0) : GroupView{0, 0, 0, false};
      wrong |= v.wrong;
      const int most = __reduce_max_sync(~0u, v.parts);
      for (int k = 0; k < most; ++k) plan_part<8>(g, s, i, v, k, i < n);
    }
  }
  wrong = __syncthreads_or(wrong);
  if (!wrong) {
    sum_before(s, parts, a.B, scratch);
    wrong = s.units[parts] > kUnitLimit || (int64_t)s.tiles[a.B] * g.p.groups > kUnitLimit;
    __syncthreads();
  }
  if (wrong) {  // every row is empty, of one tile
    for (int b = tid; b <= a.B; b += kPlanThreads) {
      if (b < a.B) s.own[b] = {0, 0, 0, 0, -1, kEmpty, 0, 0, 0, 0, {0, 0}};
      s.tiles[b] = b;
    }
    for (int i = tid; i <= parts; i += kPlanThreads) s.units[i] = 0;
    if (tid == 0) atomicOr(a.err, kErrBadSeq);
  }
  __syncthreads();
  // where each CTA begins
  const int units = s.units[parts], own_tiles = s.tiles[a.B];
  int n_items = min(x.n_items, units);
  if (n == 1 && a.B <= 1 << x.most_rows_log2 && units) {
    // Items that are all alike: whole CTAs for each, if that leaves out less than an eighth of them, so that none has the end
    // of one and the beginning of another (3 us more where an end leaves 256 rows).  For one group that is planned whole:
    // items of several have as many tiles each as their group's tokens make.
    const int alike = units / s.groups[0].tiles, each = n_items / alike;
    if (8 * each * alike >= 7 * n_items) n_items = each * alike;
  }
  const Ranges items(units, n_items);
  for (int c = tid; c < x.n_items; c += kPlanThreads) {
    ItemStart r;
    r.n = 0;
    if (c < items.n) {
      const int u = items.begin(c);
      r.n = items.begin(c + 1) - u;
      r.g = last_of(s.units, parts, u);
      r.p = s.groups[r.g];
      const int inside = u - s.units[r.g], item = inside / r.p.tiles, tile = inside - item * r.p.tiles;
      r.head = item / r.p.blocks;
      r.block = item - r.head * r.p.blocks;
      r.token = r.p.first + tile * x.tile;
      r.left = r.p.tiles - tile;
    }
    x.item_start[c] = r;
  }
  const int own_units = own_tiles * g.p.groups;
  const Ranges rows(own_units, min(g.p.n_items, own_units));
  for (int c = kPlanThreads - 1 - tid; c < g.p.n_items; c += kPlanThreads) {
    OwnStart r;
    r.n = r.b = r.hg = 0;
    if (c < rows.n) {
      const int u = rows.begin(c);
      r.n = rows.begin(c + 1) - u;
      r.hg = u / own_tiles;
      const int inside = u - r.hg * own_tiles;
      r.b = last_of(s.tiles, a.B, inside);
      r.p = s.own[r.b];
      r.token = r.p.first + (inside - s.tiles[r.b]) * g.p.tile;
      r.left = s.tiles[r.b + 1] - inside;
    }
    x.own_start[c] = r;
  }
  // the records themselves
  for (int i = tid; i < parts; i += kPlanThreads) {
    GroupPlan r = s.groups[i];
    r.units = s.units[i];
    x.groups[i] = r;
  }
  for (int b = tid; b < a.B; b += kPlanThreads) {
    RowPlan r = s.own[b];
    r.tiles = s.tiles[b];
    x.own[b] = r;
  }
}

// Joins a row's partial sums, those of its own tokens and of what it shares: a warp per row and query head.
constexpr int kJoinThreads = 128;

template <typename T>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ Args g, const Divider by_heads,
                                                            const Divider by_rows, const int heads_log2) {
  constexpr int kBatch = 8;
  const PagedDecodeArgs& a = g.a;
  const Prefix& x = g.x;
  const int lane = threadIdx.x & 31, d = a.v.d, qpg = a.v.qpg;
  const int64_t nth = (int64_t)blockIdx.x * (kJoinThreads / 32) + threadIdx.x / 32;
  pdl_launch_dependents();
  if (nth >= (int64_t)a.B * a.v.Hq) return;
  // (the launch before begins once the plan is complete)
  const int b = by_heads.div((uint32_t)nth), j = (int)(nth - (int64_t)b * a.v.Hq);
  const RowPlan own = load_record(x.own + b);
  const int h = x.by_qpg.div(j), q = j - h * qpg, chunk = by_rows.div(q), r = q - chunk * g.p.rows, vh = h * g.p.chunks + chunk;
  const int group = vh >> heads_log2, w = vh & (g.p.wh - 1);
  const int row = (b - own.start) * qpg + q, block = x.by_rows.div(row);
  const bool shares = own.group >= 0;
  pdl_wait();
  bool bad = own.state == kEmpty;
  // the CTAs that have left sums of its own tokens, and of what its group shares
  const CtaRange mine = x.own_ctas[(int64_t)group * a.B + b];
  CtaRange theirs = {0, -1};
  if (shares) {
    theirs = x.item_ctas[x.item_id(own.start, own.blocks, a.v.Hq, h, block)];
    // (numbers that are none: a CTA gave up waiting)
    bad |= x.groups[own.group].bad != 0 || theirs.first < 0 || theirs.first > theirs.last || theirs.last >= x.n_items;
  }
  const int n_own = own.end > own.first ? mine.last - mine.first + 1 : 0, n = bad ? 0 : n_own + theirs.last - theirs.first + 1;
  const int64_t own0 = x.own_row(g.p, a.B, group, b, mine.first, w) + r, own_step = (int64_t)g.p.wh * g.p.rows;
  const int64_t part0 = x.row_of(own.start, own.rows * qpg, a.v.Hq, h, block, theirs.first, row - block * x.rows);
  const int64_t part_step = x.rows;
  const auto sums_of = [&](int i) {
    return i < n_own ? x.own_u + (own0 + i * own_step) * g.DP : x.part_u + (part0 + (i - n_own) * part_step) * g.DP;
  };
  const auto ml_of = [&](int i) {
    return *reinterpret_cast<const float2*>(i < n_own ? x.own_ml + 2 * (own0 + i * own_step)
                                                      : x.part_ml + 2 * (part0 + (i - n_own) * part_step));
  };
  T* out = static_cast<T*>(a.out);
  const int quads = min(g.DP / 4, 32), lanes = 32 / quads, turn = lane / quads;
  for (int q0 = 0; q0 < g.DP / 4; q0 += quads) {  // once, but twice for heads above 128
    const int el = 4 * (q0 + lane % quads);
    float M = -CUDART_INF_F, total = 0.f;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = 0; i0 < n; i0 += 32) {
      const int count = min(32, n - i0);
      float4 v[kBatch];
      const auto fetch = [&](int i) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
          if (i + k * lanes < count && el < d) v[k] = *reinterpret_cast<const float4*>(sums_of(i0 + i + k * lanes) + el);
      };
      float2 ml = make_float2(-CUDART_INF_F, 0.f);
      if (lane < count) ml = ml_of(i0 + lane);
      fetch(turn);
      float top = fmaxf(M, ml.x);
#pragma unroll
      for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
      const float base = top == -CUDART_INF_F ? 0.f : top, f = exp2_approx(ml.x - base), before = exp2_approx(M - base);
      float l = ml.y * f;
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
          const float c = __shfl_sync(~0u, f, p & 31);
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
    if (turn == 0 && el < d) {
      const bool none = bad || total == 0.f;
      const float f = 1.f / total;
      put4(out + nth * d + el, none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(sum.x * f, sum.y * f, sum.z * f, sum.w * f),
           (reinterpret_cast<uintptr_t>(out) & 3) == 0);
      if (a.lse && el == 0) a.lse[nth] = none ? -CUDART_INF_F : (M + log2f(total)) * 0.693147180559945f;
    }
  }
}

// A group of more than 2^most_rows_log2 rows is planned in parts, each as a group of its own: the tokens of a long chunk that all its rows
// see end where its first row does, and what its rows have of their own, by rows, grows as the square of its length. Parts of 256 queries, a
// whole block on tcgen05, read the shared tokens no more often.  Part k of group i has place i + (start >> most_rows_log2) + k, so that
// groups need not know of each other's parts.
// Measured, 1024 tokens after 16384, in one part and so: 32 query heads on 8 KV heads of 128 in bf16 558 and 291 us; on 32
// KV heads 1294 and 532; of 8 bits 1856 and 1517, and 3304 and 1734.

// How the shared part of a call is laid out.
struct Layout {
  bool tc;  // on tcgen05
  int rows, tile, n_items, most_rows_log2;
};
Layout layout_of(const PagedView& v, DecodeKind kind, int B, int n_groups, int sms) {
  Layout l;
  const int DP = padded_dim(v.d);
  const int64_t queries = (int64_t)v.qpg * B / std::max(n_groups, 1);  // of a group, on average
  l.tc = kind.dtype == DCK_BF16 && !kind.quant && DP <= 128 && queries > 16;
  if (l.tc) {
    l.rows = 256;
    l.tile = 64;
    l.most_rows_log2 = kLeastPartLog2;
    while (l.most_rows_log2 < kMostPartLog2 && v.qpg << (l.most_rows_log2 + 1) <= 256) ++l.most_rows_log2;
    l.n_items = std::max(1, sms - 1);  // the plan's block has the last SM while they get ready
    return l;
  }
  l.rows = kind.dtype == DCK_BF16 && DP <= 128 && queries > 8 ? 16 : 8;
  l.tile = warps_of(DP, false) * run_of(kind);
  l.most_rows_log2 = kLeastPartLog2;
  l.n_items = std::min(prefix_per_sm(kind, l.rows) * sms, kMaxItems);
  return l;
}

// The parts of the workspace.
struct Parts {
  size_t groups, own, item_start, own_start, item_ctas, own_ctas, part_ml, part_u, own_ml, own_u, all = 0;
  Parts(const PagedView& v, const Plan& p, int B, int sms) {
    // (a CTA leaves 256 rows of an item, or each of three on an SM 16)
    const size_t rows = (size_t)B * v.Hq + (size_t)sms * 256, DP = padded_dim(v.d);
    const size_t own_rows = ((size_t)p.groups * B + p.n_items) * p.wh * p.rows;
    const auto take = [&](size_t bytes) {
      const size_t at = all;
      all += align_up(bytes, 256);
      return at;
    };
    groups = take((size_t)(B + (B >> kLeastPartLog2)) * sizeof(GroupPlan));
    own = take((size_t)B * sizeof(RowPlan));
    item_start = take(kMaxItems * sizeof(ItemStart));
    own_start = take(kMaxItems * sizeof(OwnStart));
    item_ctas = take((size_t)B * v.Hq * sizeof(CtaRange));
    own_ctas = take((size_t)B * p.groups * sizeof(CtaRange));
    part_ml = take(rows * 2 * sizeof(float));
    part_u = take(rows * DP * sizeof(float));
    own_ml = take(own_rows * 2 * sizeof(float));
    own_u = take(own_rows * DP * sizeof(float));
  }
};

}  // namespace
}  // namespace paged

using namespace paged;

size_t paged_shared_workspace(const PagedView& v, DecodeKind kind, int B, int max_len, int max_own, int sms) {
  const Plan p = range_plan(v, kind, std::max(B, 1), std::min(max_own, max_len), sms);
  return std::max(paged_decode_workspace(v, kind, B, max_len, sms), Parts(v, p, std::max(B, 1), sms).all);
}

namespace paged {
namespace {

// Whether what groups share is attended to once, or every row by itself: the one of the less time by models in us of both, fitted
// to 142 measured calls of groups and rows that are alike. Rows by themselves read mostly from L2; the shared way is four
// launches. The host knows bounds only: rows are taken to be as long as they may, with half as many own tokens as they may
// have and the rest shared, and groups to be of one size. Over 500 other calls (six head layouts, three kinds of caches, 1 to
// 32 groups of 1 to 64 rows, chunks, windows, alike and ragged) the choice is 3% off the better one on average where max_own is
// what rows have at most, 10% where it is no bound (max_seq_len), and up to 4 times in a single call.
// Measured, by rows / shared, 32 query heads on 8 KV heads of 128 in bf16, one group:
//   4 rows on 512 tokens 6.1 / 16.5     16 on 2048 18.6 / 21.4     64 on 2048  56 / 25
//   8 on 2048  12.4 / 20.7               8 on 8192 33.7 / 24.0     64 on 32768 767 / 53
bool prefer_shared(const PagedDecodeArgs& a, DecodeKind kind) {
  if (a.n_groups == a.B) return false;  // rows of their own groups share nothing
  const PagedView& v = a.v;
  const int DP = padded_dim(v.d), el = kind.quant ? 1 : kind.dtype == DCK_F32 ? 4 : 2;
  const double row = 2. * v.Hkv * (v.d * el + (kind.quant ? 4 : 0));  // bytes of a token
  const double seen = a.window > 0 ? std::min(a.window, a.max_len) : a.max_len, own = std::min<double>(a.max_own, seen) / 2;
  const double shared = seen - own;
  // bytes per us that rows by themselves, and blocks of queries, get through
  const double rate = (kind.quant ? (DP == 256 ? 3.9 : 6.4) : kind.dtype == DCK_F32 || DP == 256 ? 9. : 11.) * 1e6;
  const double by_rows = 6 + a.B * seen * row / rate;
  const double queries = (double)v.qpg * a.B / a.n_groups;
  const bool tc = kind.dtype == DCK_BF16 && !kind.quant && DP <= 128;
  const double blocks = std::ceil(queries / (tc ? 256 : kind.dtype == DCK_BF16 && DP <= 128 ? 16 : 8));
  const double once = a.n_groups * shared * row, again = once * blocks / (tc ? 7e6 : 6e6);
  // (own tokens are the same work as rows by themselves, without what those find in L2)
  return 18 + std::max(once / 5.9e6, again) + a.B * own * row / std::min(6e6, rate) + 1.2e-3 * a.B * v.Hq < by_rows;
}

}  // namespace
}  // namespace paged

cudaError_t launch_paged_shared(const PagedDecodeArgs& a, DecodeKind kind, int sms, cudaStream_t s) {
  if (a.way == 1 || (a.way == 0 && !prefer_shared(a, kind))) return launch_paged_decode(a, kind, sms, s);
  Args g = {};
  g.a = a;
  g.p = range_plan(a.v, kind, a.B, std::min(a.max_own, a.max_len), sms);
  g.DP = padded_dim(a.v.d);
  g.score.set(a.scale, a.softcap);
  const int el = kind.dtype == DCK_F32 ? 4 : 2;
  g.p.q_copied = reinterpret_cast<uintptr_t>(a.q) % 16 == 0 && a.q_stride * el % 16 == 0;
  const Layout l = layout_of(a.v, kind, a.B, a.n_groups, sms);
  const Parts parts(a.v, g.p, a.B, sms);
  char* ws = static_cast<char*>(a.ws);
  g.x.item_ctas = reinterpret_cast<CtaRange*>(ws + parts.item_ctas);
  g.x.own_ctas = reinterpret_cast<CtaRange*>(ws + parts.own_ctas);
  g.x.groups = reinterpret_cast<GroupPlan*>(ws + parts.groups);
  g.x.own = reinterpret_cast<RowPlan*>(ws + parts.own);
  g.x.item_start = reinterpret_cast<ItemStart*>(ws + parts.item_start);
  g.x.own_start = reinterpret_cast<OwnStart*>(ws + parts.own_start);
  g.x.part_ml = reinterpret_cast<float*>(ws + parts.part_ml);
  g.x.part_u = reinterpret_cast<float*>(ws + parts.part_u);
  g.x.own_ml = reinterpret_cast<float*>(ws + parts.own_ml);
  g.x.own_u = reinterpret_cast<float*>(ws + parts.own_u);
  g.x.n_groups = a.n_groups;
  g.x.most_rows_log2 = l.most_rows_log2;
  g.x.n_parts = a.n_groups + (a.B >> l.most_rows_log2);
  g.x.n_items = l.n_items;
  g.x.rows = l.rows;
  g.x.tile = l.tile;
  g.x.by_qpg = divider((uint32_t)a.v.qpg);
  g.x.by_rows = divider((uint32_t)l.rows);
  static std::atomic<uint64_t> ready{0};
  cudaError_t e = allow_shared(plan_kernel, ready, plan_bytes(kFew, kFew));
  if (e == cudaSuccess) e = launch_pdl(plan_kernel, 1, kPlanThreads, plan_bytes(g.x.n_parts, a.B), s, g);
  if (e == cudaSuccess) e = hook_launched(a.hook, s);
  // heads of the shared part are KV heads themselves
  Args h = g;
  h.p.chunks = 1;
  h.p.by_chunks = divider(1);
  h.p.wh = 1;
  if (e == cudaSuccess)
    e = l.tc ? launch_prefix_tc(h, s) : kind.quant ? launch_prefix_q8(h, kind.dtype, s) : kind.dtype == DCK_F32 ? launch_prefix_f32(h, s) : launch_prefix_bf16(h, s);
  if (e == cudaSuccess)
    e = kind.quant ? launch_own_q8(g, kind.dtype, s) : kind.dtype == DCK_F32 ? launch_own_f32(g, s) : launch_own_bf16(g, s);
  if (e != cudaSuccess) return e;
  const int64_t warps = (int64_t)a.B * a.v.Hq, blocks = (warps * 32 + kJoinThreads - 1) / kJoinThreads;
  int heads_log2 = 0;
  while (1 << heads_log2 < g.p.wh) ++heads_log2;
  const auto join = kind.dtype == DCK_F32 ? join_kernel<float> : join_kernel<__nv_bfloat16>;
  e = launch_pdl(join, (unsigned)blocks, kJoinThreads, 0, s, g, divider((uint32_t)a.v.Hq), divider((uint32_t)g.p.rows), heads_log2);
  return e == cudaSuccess ? hook_launched(a.hook, s) : e;
}

}  // namespace dck

// Calls over shared prefixes: what the rows of a group see together, by per-warp rings as in
// paged_decode.cuh (a tile of up to 16 or 8 queries, of any rows of the group).
#pragma once

#include "paged_decode.cuh"

namespace dck {
namespace paged {

// A position in the list of the items' tiles.
struct ItemWalk {
  GroupPlan p;
  int g, head, block;
  int token, left;  // the tile's first token, and the tiles from it to the end of the item

  __device__ __forceinline__ void see(const Prefix& x, int at) {
    g = at;
    p = load_record(x.groups + at);
  }
  // Enters where CTA c begins; its number of tiles.
  __device__ __forceinline__ int enter(const Prefix& x, int c) {
    const ItemStart s = load_record(x.item_start + c);
    p = s.p;
    g = s.g, head = s.head, block = s.block, token = s.token, left = s.left;
    return s.n;
  }
  // The next item.
  __device__ __forceinline__ void leave(const Prefix& x, int heads) {
    if (++block == p.blocks) {
      block = 0;
      if (++head == heads) {
        head = 0;
        do see(x, g + 1);
        while (p.tiles == 0);
      }
    }
    token = p.first;
    left = p.tiles;
  }
  __device__ __forceinline__ int count(const Prefix& x, int qpg) const { return min(x.rows, p.rows * qpg - block * x.rows); }
  // Whether the tile is the item's first.
  __device__ __forceinline__ bool begins() const { return token == p.first; }
  // Notes that this CTA has a part of the item, its first or last.
  __device__ __forceinline__ void sign(const Prefix& x, int Hq, bool begun, bool ended) const {
    CtaRange* r = x.item_ctas + x.item_id(p.start, p.blocks, Hq, head, block);
    if (begun) r->first = blockIdx.x;
    if (ended) r->last = blockIdx.x;
  }
  // Where this CTA's sums of its query r go.
  __device__ __forceinline__ int64_t row_of(const Prefix& x, int Hq, int qpg, int r) const {
    return x.row_of(p.start, p.rows * qpg, Hq, head, block, blockIdx.x, r);
  }
};

// Stores the sums of a CTA's tiles of queries: `count` of them per head, from partial row row0 on (of this warp's head).
// A head's runs of tokens add up first: each warp leaves its sums in stage `used`, which it has just read.
// Sum -1: a page outside the pool.
template <class Z, class Tile, class Shm>
__device__ __forceinline__ void leave_sums(uint8_t* raw, Shm& sh, const Tile& tile, int warp, int lane, int n_heads, int n_runs,
                                           int used, int count, int d, bool bad, float* part_u, float* part_ml, int64_t row0) {
  const int wh = warp & (n_heads - 1), wt = warp / n_heads;
  if (n_runs == 1) {
#pragma unroll
    for (int y = 0; y < Tile::kMine; ++y) {
      const int r = Tile::row(y, lane);
      if (r >= count) continue;
      if (Tile::speaks(lane)) *reinterpret_cast<float2*>(part_ml + 2 * (row0 + r)) = make_float2(tile.m[y], bad ? -1.f : tile.l[y]);
      float* p = part_u + (row0 + r) * Z::DP;
      tile.each(y, lane, d, [&](int e, float u, float v) { *reinterpret_cast<float2*>(p + e) = make_float2(u, v); });
    }
    return;
  }
  float* left = reinterpret_cast<float*>(raw + (warp * Z::S + used) * Z::kStage);
#pragma unroll
  for (int y = 0; y < Tile::kMine; ++y) {
    const int r = Tile::row(y, lane);
    if (Tile::speaks(lane)) sh.ml[warp][r] = make_float2(tile.m[y], bad ? -1.f : tile.l[y]);
    tile.each(y, lane, d, [&](int e, float u, float v) {
      *reinterpret_cast<float2*>(left + r * Z::DP + (e ^ (r & 7) * 8)) = make_float2(u, v);
    });
  }
  __syncthreads();
  for (int i = wt * 32 + lane; i < count * (Z::DP / 4); i += n_runs * 32) {
    const int r = i / (Z::DP / 4), e = i % (Z::DP / 4) * 4;
    if (e >= d) continue;
    float w[Z::NW];
    const Joined j = join_rows<Z::NW>(n_runs, w, [&](int k) { return sh.ml[k * n_heads + wh][r]; });
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < Z::NW; ++k)
      if (k < n_runs && w[k] != 0.f) {
        const float* from = reinterpret_cast<const float*>(raw + ((k * n_heads + wh) * Z::S + used) * Z::kStage);
        const float4 v = *reinterpret_cast<const float4*>(from + r * Z::DP + (e ^ (r & 7) * 8));
        sum.x += v.x * w[k], sum.y += v.y * w[k], sum.z += v.z * w[k], sum.w += v.w * w[k];
      }
    *reinterpret_cast<float4*>(part_u + (row0 + r) * Z::DP + e) = sum;
    if (e == 0) *reinterpret_cast<float2*>(part_ml + 2 * (row0 + r)) = make_float2(j.m, j.bad ? -1.f : j.l);
  }
  __syncthreads();
}

template <class Z, class Tile>
struct PrefixShared {  // after the rings
  alignas(16) uint8_t q[Tile::kRows * Z::kQRow];  // the item's queries
  alignas(16) uint8_t operands[Tile::kOperands];   // the same as a tile reads them from here, if it does
  alignas(16) float mine[std::is_same<typename Z::T, float>::value && !Z::kQuant ? Z::NW * 8 * Tile::kRows : 4];  // fp32: a warp's weights
  alignas(16) float2 ml[Z::NW][Tile::kRows];
};

// The item's queries to `to` (rows past them, and rows' ends, as zeros), by the whole CTA.
template <class Z, int ROWS>
__device__ __forceinline__ void read_item_queries(const Args& g, const ItemWalk& at, int count, uint8_t* to) {
  using T = typename Z::T;
  constexpr int el = sizeof(T), per = 16 / el, kChunks = Z::kQRow / 16;
  const int qpg = g.a.v.qpg, d = g.a.v.d;
  for (int i = threadIdx.x; i < ROWS * kChunks; i += Z::NW * 32) {
    const int row = i / kChunks, c = i % kChunks, x = at.block * g.x.rows + row, b = g.x.by_qpg.div(x), j = at.head * qpg + x - b * qpg;
    const T* from = static_cast<const T*>(g.a.q) + (int64_t)(at.p.start + b) * g.a.q_stride + (int64_t)j * d + c * per;
    alignas(16) T v[per];
    if (row < count && c * per < d) {
      if (g.p.q_copied) {
        *reinterpret_cast<uint4*>(v) = *reinterpret_cast<const uint4*>(from);
      } else {
#pragma unroll
        for (int k = 0; k < per; ++k) v[k] = from[k];
      }
    } else {
#pragma unroll
      for (int k = 0; k < per; ++k) v[k] = from_f32<T>(0.f);
    }
    *reinterpret_cast<uint4*>(to + row * Z::kQRow + (c ^ (row & 7)) * 16) = *reinterpret_cast<const uint4*>(v);
  }
}

// An item's tiles: its warps are runs of tokens, all with the same queries.  PER_SM: CTAs on an SM.
template <class Z, class Tile, int PER_SM>
__global__ void __launch_bounds__(Z::NW * 32, PER_SM) prefix_kernel(const __grid_constant__ Args g) {
  extern __shared__ __align__(128) uint8_t raw[];
  using Shm = PrefixShared<Z, Tile>;
  Shm& sh = *reinterpret_cast<Shm*>(raw + Z::kRing);
  const PagedDecodeArgs& a = g.a;
  const Prefix& x = g.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, d = a.v.d, qpg = a.v.qpg, heads = a.v.Hkv;
  pdl_wait();
  pdl_launch_dependents();  // the plan, and with it all that the own tokens' launch reads, is there
  ItemWalk ahead;
  int to_compute = ahead.enter(x, blockIdx.x);
  if (to_compute == 0) return;
  const typename LoaderOf<Z, Tile::kRows, 1>::type load(g, raw, sh.q, warp, lane, 0, warp);
  load.clear(raw);
  ItemWalk at = ahead;
  int to_copy = to_compute, to_fetch = to_compute;

  // page numbers are read two tiles ahead of the copies
  Pages next = {0, -1, 0, -1}, next2 = {0, -1, 0, -1};
  const auto fetch_next = [&]() {
    Walk w;
    w.token = ahead.token;
    w.len = ahead.p.end;
    w.b = ahead.p.table;
    w.group = ahead.head;
    const Pages r = load.fetch(w, false);
    ahead.token += x.tile;
    if (--to_fetch > 0 && --ahead.left == 0) ahead.leave(x, heads);
    return r;
  };
  if (to_fetch > 0) next = fetch_next();
  if (to_fetch > 0) next2 = fetch_next();
  uint32_t outside = 0;
  int put = 0;
  const auto copy_next = [&]() {
    if (to_copy > 0) {
      --to_copy;
      const bool bad = load.issue(next, put);
      outside = (outside & ~(1u << put)) | (uint32_t)bad << put;
      next = next2;
      if (to_fetch > 0) next2 = fetch_next();
      put = put + 1 == Z::S ? 0 : put + 1;
    }
    cp_async_commit();
  };
  float* mine = sh.mine + warp * 8 * Tile::kRows;
  Tile tile;
#pragma unroll 1
  for (int i = 0; i < Z::S - 1; ++i) copy_next();
  int get = 0, count = 0;
  bool bad = false, fresh = true, begun = at.begins();
  while (true) {
    __syncwarp();  // the stage that is filled next has been read
    copy_next();
    if (fresh) {  // (the queries before are not in use any more: see leave_sums)
      count = at.count(x, qpg);
      read_item_queries<Z, Tile::kRows>(g, at, count, sh.q);
      __syncthreads();
      if (Tile::kOperands > 16) {
        Tile::lay_out(sh.q, sh.operands);
        __syncthreads();
        tile.begin((uint32_t)__cvta_generic_to_shared(sh.operands), lane);
      } else {
        tile.begin((uint32_t)__cvta_generic_to_shared(sh.q), lane);
      }
      fresh = false;
    }
    cp_async_wait<Z::S - 1>();
    __syncwarp();
    bad |= outside >> get & 1;
    tile.step(load.ring + get * Z::kStage, at.p.end - at.token - load.run, lane, g.score, mine);
    const int used = get;
    get = get + 1 == Z::S ? 0 : get + 1;
    at.token += x.tile;
    const bool last = --to_compute <= 0;
    if (--at.left > 0 && !last) continue;
    // the end of an item, or of this CTA's part of it
    if (bad && lane == 0) {
      atomicOr(a.err, kErrBadSeq);
      atomicOr(&x.groups[at.g].bad, 1);
    }
    tile.finish();
    leave_sums<Z>(raw, sh, tile, warp, lane, 1, Z::NW, used, count, d, false, x.part_u, x.part_ml, at.row_of(x, a.v.Hq, qpg, 0));
    if (threadIdx.x == 0) at.sign(x, a.v.Hq, begun, at.left == 0);
    begun = true;
    load.clear_stage(raw + (warp * Z::S + used) * Z::kStage);
    if (last) break;
    bad = false;
    fresh = true;
    at.leave(x, heads);
  }
  cp_async_wait<0>();
}

// A position in the list of the rows' own tiles (head groups outermost).
struct OwnWalk : Walk {
  RowPlan p, next;

  __device__ __forceinline__ void take(int tile) {
    token = p.first;
    len = p.end;
    skip_at = p.skip_at;
    skip = p.skip;
    left = max(1, (p.end - p.first + tile - 1) / tile);
  }
  // Enters where CTA c begins; its number of tiles.
  __device__ __forceinline__ int enter(const Args& g, int c) {
    const OwnStart s = load_record(g.x.own_start + c);
    p = s.p;
    b = s.b;
    group = s.hg;
    if (s.n == 0) return 0;
    next = load_record(g.x.own + (b + 1 < g.a.B ? b + 1 : 0));
    take(g.p.tile);
    token = s.token;
    left = s.left;
    return s.n;
  }
  // The next (head group, row); the plan of the one after it is read ahead.
  __device__ __forceinline__ void leave(const Args& g) {
    if (++b == g.a.B) b = 0, ++group;
    p = next;
    next = load_record(g.x.own + (b + 1 < g.a.B ? b + 1 : 0));
    take(g.p.tile);
  }
};

// What the rows have of their own: tiles dealt in ranges as in paged_decode_kernel, a partial sum left of each (head group,
// row) by each CTA that has tiles of it.
template <class Z, class Tile>
__global__ void __launch_bounds__(Z::NW * 32, 3) own_kernel(const __grid_constant__ Args g) {
  extern __shared__ __align__(128) uint8_t raw[];
  using Shm = Shared<Z, Tile, false>;
  Shm& sh = *reinterpret_cast<Shm*>(raw + Z::kRing);
  const PagedDecodeArgs& a = g.a;
  const Prefix& x = g.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n_heads = g.p.wh, n_runs = g.p.wt, wh = warp & (n_heads - 1), wt = warp / n_heads;
  const int d = a.v.d;
  pdl_launch_dependents();  // (the shared part let this launch begin: the plan and all before it are complete)
  __threadfence();          // what the L1 still has of earlier calls' tables and scales is not read
  OwnWalk ahead;
  int to_compute = ahead.enter(g, blockIdx.x);
  if (to_compute == 0) {
    pdl_wait();  // what waits for this launch waits for the shared part too
    return;
  }
  const typename LoaderOf<Z, Tile::kRows, Shm::kPlaces>::type load(g, raw, sh.q, warp, lane, wh, wt);
  load.clear(raw);
  OwnWalk at = ahead;
  int to_copy = to_compute, to_fetch = to_compute;
  Pages pages = {0, -1, 0, -1}, pages2 = {0, -1, 0, -1};
  bool first = true;
  const auto fetch_next = [&]() {
    const Pages p = load.template fetch<true>(ahead, first);
    first = false;
    ahead.token += g.p.tile;
    if (--to_fetch > 0 && --ahead.left == 0) {
      ahead.leave(g);
      first = true;
    }
    return p;
  };
  if (to_fetch > 0) pages = fetch_next();
  if (to_fetch > 0) pages2 = fetch_next();
  uint32_t outside = 0;
  int put = 0;
  const auto copy_next = [&]() {
    if (to_copy > 0) {
      --to_copy;
      const bool bad = load.issue(pages, put);
      outside = (outside & ~(1u << put)) | (uint32_t)bad << put;
      pages = pages2;
      if (to_fetch > 0) pages2 = fetch_next();
      put = put + 1 == Z::S ? 0 : put + 1;
    }
    cp_async_commit();
  };
  float* mine = sh.mine + warp * 8 * Tile::kRows;
  Tile tile;
  Queries qs;
#pragma unroll 1
  for (int i = 0; i < Z::S - 1; ++i) copy_next();
  int get = 0;
  bool bad = false, fresh = true, begun = at.token == at.p.first;
  while (true) {
    __syncwarp();  // the stage that is filled next has been read
    copy_next();
    cp_async_wait<Z::S - 1>();
    __syncwarp();
    if (fresh) {
      qs = queries_of(g, at.group, wh);
      if (!g.p.q_copied) load.read_queries(qs, at.b, sh.q, warp, get);
      tile.begin(load.places + get * load.kPlace, lane);
      fresh = false;
    }
    bad |= outside >> get & 1;
    tile.step(load.ring + get * Z::kStage, at.len - at.token - load.run, lane, g.score, mine);
    const int used = get;
    get = get + 1 == Z::S ? 0 : get + 1;
    at.token += g.p.tile;
    const bool last = --to_compute <= 0;
    if (--at.left > 0 && !last) continue;
    // the end of a (head group, row), or of this CTA's part of it
    if (bad && lane == 0) atomicOr(a.err, kErrBadSeq);
    tile.finish();
    leave_sums<Z>(raw, sh, tile, warp, lane, n_heads, n_runs, used, qs.count, d, bad, x.own_u, x.own_ml,
                  x.own_row(g.p, a.B, at.group, at.b, blockIdx.x, wh));
    if (threadIdx.x == 0) {
      CtaRange* r = x.own_ctas + (int64_t)at.group * a.B + at.b;
      if (begun) r->first = blockIdx.x;
      if (at.left == 0) r->last = blockIdx.x;
    }
    begun = true;
    if (last) break;
    if (n_runs > 1) load.clear_stage(raw + (warp * Z::S + used) * Z::kStage);
    bad = false;
    fresh = true;
    at.leave(g);
  }
  cp_async_wait<0>();
  pdl_wait();
}

// Lets `kernel` use `bytes` of shared memory, once per device.
template <class K>
cudaError_t allow_shared(K kernel, std::atomic<uint64_t>& ready, size_t bytes) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (dev < 64 && ready.load(std::memory_order_relaxed) >> dev & 1)) return e;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == cudaSuccess && dev < 64) ready.fetch_or(uint64_t(1) << dev, std::memory_order_relaxed);
  return e;
}
template <class K>
cudaError_t launch_part(K kernel, std::atomic<uint64_t>& ready, int grid, int threads, size_t smem, const Args& g, cudaStream_t s) {
  cudaError_t e = allow_shared(kernel, ready, smem);
  if (e == cudaSuccess) e = launch_pdl(kernel, grid, threads, smem, s, g);
  return e == cudaSuccess ? hook_launched(g.a.hook, s) : e;
}

template <class Z, class Tile>
cudaError_t launch_own(const Args& g, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};
  return launch_part(own_kernel<Z, Tile>, ready, g.p.n_items, Z::NW * 32, Z::kRing + sizeof(Shared<Z, Tile, false>), g, s);
}

template <class Z, class Tile, int PER_SM = kPerSm>
cudaError_t launch_prefix(const Args& g, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};
  constexpr size_t smem = Z::kRing + sizeof(PrefixShared<Z, Tile>);
  static_assert((smem + 1024) * PER_SM <= 233472, "an SM's shared memory");
  return launch_part(prefix_kernel<Z, Tile, PER_SM>, ready, g.x.n_items, Z::NW * 32, smem, g, s);
}

}  // namespace paged
}  // namespace dck

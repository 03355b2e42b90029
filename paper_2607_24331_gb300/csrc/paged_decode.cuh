// Shared by the translation units of dck_paged_decode_attention: the work plan and
// the device code that runs it.
#pragma once

#include <math_constants.h>

#include <algorithm>
#include <atomic>
#include <cfloat>
#include <cstddef>
#include <type_traits>

#include "paged.cuh"

namespace dck {
namespace paged {

constexpr int kMaxLen = 1 << 29;     // tokens of a sequence
constexpr int kUnitLimit = 1 << 30;  // tiles of one call, over all head groups
constexpr int kMaxCluster = 8;

// How a call is laid over warps and CTAs.
struct Plan {
  int chunks, rows;  // a KV head's queries: `chunks` tiles of up to `rows`
  int wh, wt;        // warps of a CTA: wh heads (a power of two) x wt runs of tokens
  int groups;        // head groups: Hkv * chunks / wh
  int tile;          // tokens of a CTA's tile
  int cluster;       // 0: tiles dealt in ranges; else CTAs per (head group, sequence), where more than 1 a cluster
  int warps;         // of a CTA
  int n_items;       // CTAs of tiles dealt in ranges
  int part_rows;     // rows of partial sums that each of them has twice
  int alike;         // keys and values have the same strides
  int q_copied;      // queries in whole aligned 16-byte chunks
  Divider by_chunks, by_tile;
};

// What CTA c of tiles dealt in ranges leaves to the second launch: the (head group,
// sequence) that it begins and that other CTAs, up to `last`, go on with.
struct Entry {
  int b, group, last;  // last < 0: none
  int second;          // the CTA's partial of it is its second one
};
constexpr int kMaxItems = 512;  // CTAs of tiles dealt in ranges

constexpr float kHeadroom = 8.f;  // log2 units that a score may lie above the running reference

// Scores in log2 units.
__device__ __forceinline__ float tanh_of(float x);
struct ScoreScale {
  float scale2, inv_cap, cap2;  // cap2 = 0: no cap
  // Factors that stay finite, so that a product of 0 stays 0.  c tanh(s / c) is s to fp32
  // rounding for |s| < 2^-12 c: a cap from 2^100 on is none.
  void set(float scale, float softcap) {
    const auto finite = [](float x) { return std::min(std::max(x, -FLT_MAX), FLT_MAX); };
    const bool capped = softcap > 0.f && softcap < 1.2676506e30f;
    scale2 = finite(scale * 1.44269504088896f);
    cap2 = capped ? softcap * 1.44269504088896f : 0.f;
    inv_cap = capped ? finite(scale / softcap) : 0.f;
  }
  template <int N>
  __device__ __forceinline__ void apply(float (&s)[N]) const {
    if (cap2 > 0.f) {
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] = cap2 * tanh_of(s[i] * inv_cap);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] *= scale2;
    }
  }
};

// Calls over shared prefixes (paged_shared.cu): what the rows of group g see together, tokens [first, end), is attended
// to for all of them at once (of a long group, for parts of it: each like a group), in items of a block of their queries on a KV head, each cut into tiles; the items'
// tiles form one list, dealt to CTAs in equal ranges.
struct alignas(16) GroupPlan {
  int start, rows;   // its rows
  int first, end;    // the tokens; none: end = first
  int table;         // the row whose block table they are read by
  int tiles, blocks; // of an item; items per KV head
  int units;         // tiles of all groups before
  int bad;           // a page outside the pool
  int pad[3];
};
// What a row attends to by itself: tokens [first, end), counted without `skip` of them from token skip_at on.
struct alignas(16) RowPlan {
  int first, end, skip_at, skip;
  int group;      // its group, -1 if the row takes no part in what that shares
  int state;      // 0, or kEmpty: zeros whatever the group has
  int tiles;      // of all rows before (a row has one at least)
  int start, rows, blocks;  // of its group
  int pad[2];
};
constexpr int kEmpty = 1;
// Where a CTA begins: its first item, or (head group, row), the tile's first token and the tiles from it to the end
// of that, and how many it has in all.
struct alignas(16) ItemStart {
  GroupPlan p;
  int g, head, block, token, left, n, pad[2];
};
struct alignas(16) OwnStart {
  RowPlan p;
  int b, hg, token, left, n, pad[3];
};
struct CtaRange {  // of those that have tiles of an item, or of a (head group, row)
  int first, last;
};
// (past the L1, where a launch that does not wait for all before it may find what another call left)
template <class S>
__device__ __forceinline__ S load_record(const S* from) {
  S r;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(S) / 16); ++i) reinterpret_cast<int4*>(&r)[i] = __ldcg(reinterpret_cast<const int4*>(from) + i);
  return r;
}
struct Prefix {
  GroupPlan* groups;
  RowPlan* own;    // [B]
  ItemStart* item_start;  // [n_items]
  OwnStart* own_start;    // [p.n_items]
  CtaRange* item_ctas;    // [B Hq] by item_id: who leaves sums
  CtaRange* own_ctas;     // [(head group, row)]
  float *part_u, *part_ml;  // partial sums, as in Args, of what groups share: rows by row_of
  float *own_u, *own_ml;    // and of rows' own tokens: rows by own_row
  int n_groups, n_items;  // groups; CTAs that tiles are dealt to
  int most_rows_log2, n_parts;  // of the rows of a group that is planned whole; places for groups and their parts
  int rows, tile;         // queries of a block, tokens of a tile
  Divider by_qpg, by_rows;

  __device__ __forceinline__ int64_t own_row(const Plan& p, int B, int group, int b, int c, int w) const;
  // A number below B Hq of an item: every block has a query.
  __device__ __forceinline__ int64_t item_id(int start, int blocks, int Hq, int head, int block) const {
    return (int64_t)start * Hq + (int64_t)head * blocks + block;
  }
  // Where query `r` of the block `block` of KV head `head` has the partial sum that CTA c leaves: items in order, CTAs that
  // share one behind one another.  The next item of a CTA or the next CTA of an item is further on by all the rows
  // that one of them can fill.  The group: rows from `start` on, `queries` on a KV head.
  __device__ __forceinline__ int64_t row_of(int start, int queries, int Hq, int head, int block, int c, int r) const {
    return (int64_t)start * Hq + (int64_t)head * queries + (int64_t)block * rows + (int64_t)c * rows + r;
  }
};

// Where CTA c leaves the sums of row b's own tokens, head w of head group `group`: as row_of, (head group, row) in order.
__device__ __forceinline__ int64_t Prefix::own_row(const Plan& p, int B, int group, int b, int c, int w) const {
  return ((int64_t)((int64_t)group * B + b + c) * p.wh + w) * p.rows;
}

struct Args {
  PagedDecodeArgs a;
  Plan p;
  ScoreScale score;
  Prefix x;  // calls over shared prefixes
  int DP;          // head dim, rounded up to the variant's
  float* part_u;   // [2 n_items][wh][rows][DP]
  float* part_ml;  // [2 n_items][wh][rows][2]: maximum (log2 units), sum (-1: a page outside the pool)
  Entry* entries;  // [n_items]
};

cudaError_t launch_bf16(const Args& g, cudaStream_t s);
cudaError_t launch_f32(const Args& g, cudaStream_t s);
cudaError_t launch_q8(const Args& g, int dtype, cudaStream_t s);
// Of calls over shared prefixes, what groups share (x) and what rows have of their own (p).
cudaError_t launch_prefix_bf16(const Args& g, cudaStream_t s);
cudaError_t launch_prefix_f32(const Args& g, cudaStream_t s);
cudaError_t launch_prefix_q8(const Args& g, int dtype, cudaStream_t s);
cudaError_t launch_prefix_tc(const Args& g, cudaStream_t s);  // bf16, head dims up to 128: blocks of up to 256 queries
cudaError_t launch_own_bf16(const Args& g, cudaStream_t s);
cudaError_t launch_own_f32(const Args& g, cudaStream_t s);
cudaError_t launch_own_q8(const Args& g, int dtype, cudaStream_t s);
Plan range_plan(const PagedView& v, DecodeKind kind, int B, int max_len, int sms);  // tiles dealt in ranges

inline int padded_dim(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }
// Warps of a CTA: two CTAs per SM fill its shared memory with rings, or one of twice the warps.
constexpr int warps_of(int DP, bool one_per_sm) { return (DP == 256 ? 2 : 4) * (one_per_sm ? 2 : 1); }
constexpr int kPerSm = 2;
// (paged_shared.cuh) CTAs per SM of what groups share: three where 8-bit rows meet 16 queries.
inline int prefix_per_sm(DecodeKind kind, int rows) { return kind.quant && rows > 8 ? 3 : kPerSm; }
inline int run_of(DecodeKind k) { return k.quant ? 32 : k.dtype == DCK_BF16 ? 16 : 8; }  // tokens of a warp's step

// Visible tokens of a sequence of length L and the first of them; 0 for invalid lengths.
__device__ __forceinline__ int visible_of(const PagedDecodeArgs& a, int L, int& first, bool& bad) {
  bad = L < 0 || L > a.max_len || L > kMaxLen || (L > 0 && (int64_t)a.v.by_page.div(L - 1) >= a.table_stride);
  first = a.window > 0 && L > a.window ? L - a.window : 0;
  return bad ? 0 : L - first;
}
// Of sequence b.
__device__ __forceinline__ int visible(const PagedDecodeArgs& a, int b, int& first, bool& bad) {
  return visible_of(a, a.seq_len[b], first, bad);
}

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Exclusive prefix sums of the sequences' tile counts in shared memory
// prefix[0..B], and their lengths (len may be null).  Called by the whole block.
template <int NW>
__device__ __forceinline__ int tile_prefix(const PagedDecodeArgs& a, const Divider& by_tile, int groups, int* prefix,
                                           int* len, bool report) {
  const int64_t limit = kUnitLimit / groups;
  __shared__ int64_t scratch[NW];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const auto tiles_of = [&](int b) -> uint32_t {  // at most 2^26
    if (b >= a.B) return 0;
    int first;
    bool bad;
    const int span = visible(a, b, first, bad);
    if (bad && report && (a.B > 32 || warp == 0)) atomicOr(a.err, kErrBadSeq);
    if (len && (a.B > 32 || warp == 0)) len[b] = span + first;
    return by_tile.div(span + by_tile.d - 1);
  };
  const auto scan = [&](auto v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const auto y = __shfl_up_sync(~0u, v, o);
      if (lane >= o) v += y;
    }
    return v;
  };
  if (a.B <= 32) {  // every warp by itself
    const uint32_t n = tiles_of(lane), v = scan(n), most = (uint32_t)limit;
    const uint32_t all = min(__shfl_sync(~0u, v, 31), most);
    if (warp == 0) {
      if (v > most && n > 0 && report) atomicOr(a.err, kErrBadSeq);
      if (lane < a.B) prefix[lane] = (int)min(v - n, most);
      if (lane == 0) prefix[a.B] = (int)all;
    }
    __syncthreads();
    return (int)all;
  }
  int64_t base = 0;
  for (int b0 = 0; b0 < a.B; b0 += NW * 32) {
    const int b = b0 + tid;
    const int64_t n = tiles_of(b), v = scan(n);
    if (lane == 31) scratch[warp] = v;
    __syncthreads();
    int64_t before = base;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const int64_t y = scratch[w];
      if (w < warp) before += y;
      base += y;
    }
    if (b < a.B) {
      if (before + v > limit && n > 0 && report) atomicOr(a.err, kErrBadSeq);
      prefix[b] = (int)min(before + v - n, limit);
    }
    base = min(base, limit);
    __syncthreads();
  }
  if (tid == 0) prefix[a.B] = (int)base;
  __syncthreads();
  return (int)base;
}

// CTA c of n has tiles [begin(c), begin(c + 1)) of `units`, begin(c) = floor(c units / n).
struct Ranges {
  int units, n, each, rest;
  __device__ __forceinline__ Ranges(int units, int n)
      : units(units), n(n), each(n ? units / n : 0), rest(units - each * n) {}
  __device__ __forceinline__ int begin(int c) const { return c * each + c * rest / n; }
  __device__ __forceinline__ int item_of(int u) const { return (int)(((int64_t)(u + 1) * n + units - 1) / units) - 1; }
};

// What the plan keeps of the sequences in shared memory.
struct Batch {
  int* prefix;  // [B + 1] exclusive prefix sums of the tile counts
  int* len;     // [B] lengths, of sequences that have tiles (null: more than kKeptLens sequences, lengths from memory)
};
constexpr int kKeptLens = 1024;

// A position in the flattened list of tiles (head groups outermost).
struct Walk {
  int token, left;  // the tile's first token, and the tiles from it to the end of its (head group, sequence)
  int b, group, len;
  // calls over shared prefixes: tokens are counted without `skip` of them from token skip_at on
  int skip_at, skip;

  // Sets len, and token to the first visible one.
  __device__ __forceinline__ void see(const PagedDecodeArgs& a, const Batch& q) {
    if (q.len) {
      len = q.len[b];
      token = a.window > 0 && len > a.window ? len - a.window : 0;
    } else {
      bool bad;
      const int span = visible(a, b, token, bad);  // (sets token)
      len = span + token;
    }
  }
  // Enters at tile u; true if that is the first of its (head group, sequence).
  __device__ __forceinline__ bool enter(const PagedDecodeArgs& a, const Batch& q, int n_tiles, int tile, int u) {
    group = u / n_tiles;
    const int x = u - group * n_tiles;
    b = seq_of_tile(q.prefix, a.B, x);
    see(a, q);
    token += (x - q.prefix[b]) * tile;
    left = q.prefix[b + 1] - x;
    return x == q.prefix[b];
  }
  // The next (head group, sequence) that has tiles.
  __device__ __forceinline__ void leave(const PagedDecodeArgs& a, const Batch& q) {
    do {
      if (++b == a.B) b = 0, ++group;
      left = q.prefix[b + 1] - q.prefix[b];
    } while (left == 0);
    see(a, q);
  }
};

// 16-byte asynchronous copy of `bytes` (16 or 0) bytes, the rest zero.
__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// Sizes of a variant: elements T, head dim up to DP, NW warps, S stages of TOK tokens.
template <typename T_, int DP_, int NW_, int S_, int TOK_>
struct Sizes {
  using T = T_;
  static constexpr int DP = DP_, NW = NW_, S = S_, TOK = TOK_;
  static constexpr bool kQuant = false;
  static constexpr int kRow = DP * sizeof(T);   // bytes of a head's row
  static constexpr int kChunks = kRow / 16;     // 16-byte chunks of it
  static constexpr int kQRow = kRow;            // bytes of a query
  static constexpr int kHalf = TOK * kRow;      // a stage's keys (values: the same)
  static constexpr int kStage = 2 * kHalf;
  static constexpr int kRing = NW * S * kStage;
};

// The queries of one head of a head group: `count` of them from query head `first` on.
struct Queries {
  int first, count;
};
__device__ __forceinline__ Queries queries_of(const Args& g, int group, int wh) {
  const int vh = group * g.p.wh + wh, h = g.p.by_chunks.div(vh), r0 = (vh - h * g.p.chunks) * g.p.rows;
  return {h * g.a.v.qpg + r0, min(g.p.rows, g.a.v.qpg - r0)};
}

// The page number and offset of a token of one warp's run of a tile: lane r holds token r.
struct Pages {
  int page, off;  // off < 0: no token
  int group;
  int b;          // the sequence whose queries come with this tile, or -1
};

// What copies have in common, whatever the caches' type.  ROWS: queries of a warp; they are
// copied along with the first tile of a (head group, sequence), QS places for them per warp.
template <class Z, int ROWS, int QS>
struct LoaderBase {
  static constexpr int el = sizeof(typename Z::T);
  static constexpr int kPlace = ROWS * Z::kQRow;
  static constexpr int kQChunks = Z::kQRow / 16;
  const Args& g;
  uint32_t ring, places;     // this warp's stages and places
  int lane, run, wh;      // run: the warp's first token of a tile

  __device__ __forceinline__ LoaderBase(const Args& g, const uint8_t* raw, const void* q, int warp, int lane, int wh, int wt)
      : g(g), lane(lane), run(wt * Z::TOK), wh(wh) {
    ring = (uint32_t)__cvta_generic_to_shared(raw) + warp * Z::S * Z::kStage;
    places = (uint32_t)__cvta_generic_to_shared(q) + warp * QS * kPlace;
  }

  // Heads shorter than the variant's: the rest of each row stays zero.
  __device__ __forceinline__ void clear(uint8_t* raw) const {
    if (g.a.v.d == Z::DP) return;
    for (int i = threadIdx.x; i < Z::kRing / 16; i += Z::NW * 32) reinterpret_cast<uint4*>(raw)[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
  }

  // The same for a stage of this warp that has held something else.
  __device__ __forceinline__ void clear_stage(uint8_t* stage) const {
    if (g.a.v.d == Z::DP) return;
    for (int i = lane; i < Z::kStage / 16; i += 32) reinterpret_cast<uint4*>(stage)[i] = make_uint4(0, 0, 0, 0);
  }

  template <bool SKIP = false>
  __device__ __forceinline__ Pages fetch(const Walk& w, bool first) const {
    Pages r;
    r.b = first ? w.b : -1;
    r.group = w.group;
    int t = w.token + run + lane;
    const bool have_it = lane < Z::TOK && t < w.len;
    if (SKIP && t >= w.skip_at) t += w.skip;
    const uint32_t col = g.a.v.by_page.div(have_it ? t : 0);
    r.off = have_it ? t - (int)col * g.a.v.page : -1;
    r.page = have_it ? g.a.table[w.b * g.a.table_stride + col] : 0;
    return r;
  }

  // Starts the copy of the queries to place `at`: rows past them, and rows' ends, as zeros.
  __device__ __forceinline__ void copy_queries(const Pages& r, int at) const {
    const Queries qs = queries_of(g, r.group, wh);
    const char* q = static_cast<const char*>(g.a.q) + ((int64_t)r.b * g.a.q_stride + (int64_t)qs.first * g.a.v.d) * el;
    const int row_bytes = g.a.v.d * el;
    const uint32_t to = places + at * kPlace;
#pragma unroll
    for (int i = 0; i < ROWS * kQChunks / 32 + (ROWS * kQChunks % 32 != 0); ++i) {
      const int x = i * 32 + lane, row = x / kQChunks, c = x % kQChunks;
      const bool have = row < qs.count && c * 16 < row_bytes;
      if (ROWS * kQChunks % 32 == 0 || row < ROWS)
        cp_async16_or_zero(to + row * Z::kQRow + (c ^ (row & 7)) * 16, q + (have ? row * row_bytes + c * 16 : 0),
                           have ? 16 : 0);
    }
  }
  // The same by single elements, for queries off 16-byte boundaries.
  __device__ __forceinline__ void read_queries(const Queries& qs, int b, uint8_t* q_all, int warp, int at) const {
    using T = typename Z::T;
    T* to = reinterpret_cast<T*>(q_all + (warp * QS + at) * kPlace);
    const T* q = static_cast<const T*>(g.a.q) + (int64_t)b * g.a.q_stride + (int64_t)qs.first * g.a.v.d;
    constexpr int per = 16 / el;
    for (int x = lane; x < ROWS * Z::DP; x += 32) {
      const int row = x / Z::DP, e = x % Z::DP;
      to[row * Z::DP + ((e / per) ^ (row & 7)) * per + e % per] =
          row < qs.count && e < g.a.v.d ? q[row * g.a.v.d + e] : from_f32<T>(0.f);
    }
    __syncwarp();
  }
};

// Copies of bf16 and fp32 rows.
template <class Z, int ROWS, int QS>
struct Loader : LoaderBase<Z, ROWS, QS> {
  using Base = LoaderBase<Z, ROWS, QS>;
  using Base::el, Base::g, Base::lane, Base::ring, Base::wh;
  const char *kc, *vc;    // with this lane's chunk
  uint32_t even, odd;        // where this lane's chunk of rows 4 i + sub lies in a stage, i even or odd
  int have;               // chunks of a row from this lane's first on

  __device__ __forceinline__ Loader(const Args& g, const uint8_t* raw, const void* q, int warp, int lane, int wh, int wt)
      : Base(g, raw, q, warp, lane, wh, wt) {
    const int sub = lane >> 3, c = lane & 7;
    kc = static_cast<const char*>(g.a.kc) + c * 16;
    vc = static_cast<const char*>(g.a.vc) + c * 16;
    even = sub * Z::kRow + (c ^ sub) * 16;
    odd = sub * Z::kRow + (c ^ (sub + 4)) * 16;
    have = g.a.v.d * el / 16 - c;
  }

  // Starts the copies of a stage; true if a page lies outside the pool (its tokens read as
  // zeros).  Eight lanes copy 128 bytes of a row, a warp four rows at a time.
  __device__ __forceinline__ bool issue(const Pages& r, int stage) const {
    const PagedView& v = g.a.v;
    if (QS > 1 && r.b >= 0 && g.p.q_copied) this->copy_queries(r, stage);
    const uint32_t head = g.p.by_chunks.div(r.group * g.p.wh + wh);
    const bool inside = (uint32_t)r.page < (uint32_t)v.n_pages, ok = inside && r.off >= 0;
    const uint32_t page = inside ? r.page : 0, off = max(r.off, 0);
    const int64_t ko = (int64_t)((uint64_t)page * v.k_page_b + (uint64_t)off * v.k_tok_b + (uint64_t)head * v.k_head_b);
    int64_t vo = ko;
    if (!g.p.alike)
      vo = (int64_t)((uint64_t)page * v.v_page_b + (uint64_t)off * v.v_tok_b + (uint64_t)head * v.v_head_b);
    const uint32_t mask = __ballot_sync(~0u, ok), at = ring + stage * Z::kStage;
    const int sub = lane >> 3;
#pragma unroll
    for (int i = 0; i < Z::TOK / 4; ++i) {
      const int row = i * 4 + sub;
      const int64_t kr = __shfl_sync(~0u, ko, row);
      const int64_t vr = g.p.alike ? kr : __shfl_sync(~0u, vo, row);
      const int bytes = mask >> row & 1 ? 16 : 0;
      const uint32_t dst = at + (i & 1 ? odd : even) + i * 4 * Z::kRow;
      const char *kp = kc + kr, *vp = vc + vr;
#pragma unroll
      for (int j = 0; j < Z::kChunks / 8; ++j)
        if (8 * j < have) {
          cp_async16_or_zero(dst + 128 * j, kp + 128 * j, bytes);
          cp_async16_or_zero(dst + 128 * j + Z::kHalf, vp + 128 * j, bytes);
        }
    }
    return __any_sync(~0u, !inside);
  }
};

// The loader of a variant.
template <class Z, int ROWS, int QS>
struct LoaderOf {
  using type = Loader<Z, ROWS, QS>;
};

// tanh to 3e-7 of its value: below 1/2 an odd polynomial (least squares in x^2 on
// tanh(x) / x, 6e-8), above it 1 - 2 / (e^2x + 1).
__device__ __forceinline__ float tanh_of(float x) {
  const float ax = fabsf(x), u = x * x;
  float p = -6.6395057e-3f;
  p = fmaf(p, u, 2.1292942e-2f);
  p = fmaf(p, u, -5.3898074e-2f);
  p = fmaf(p, u, 1.3332954e-1f);
  p = fmaf(p, u, -3.3333325e-1f);
  const float big = 1.f - __fdividef(2.f, exp2_approx(ax * 2.88539008f) + 1.f);
  return ax < 0.5f ? fmaf(x * u, p, x) : copysignf(ax > 20.f ? 1.f : big, x);
}

// ---------------------------------------------------------------------------
// bf16: tensor cores (mma.sync m16n8k16, queries as rows)
// ---------------------------------------------------------------------------

__device__ __forceinline__ void ldmatrix4_plain(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
// Matrices 16-byte chunks 2 k and 2 k + 1 of rows whose chunk 0 or 1 is at `at`: the swizzle
// flips bits 4 to 6 of the address, whole 128-byte lines add.
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t at, int k) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"((at ^ (k % 4 * 32)) + k / 4 * 128)
               : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t at, int k) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"((at ^ (k % 4 * 32)) + k / 4 * 128)
               : "memory");
}
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Two weights as bf16 pairs hi + lo.  Rounding weights to one bf16 would add 2^-9 to
// the output's own rounding; two of them leave 2^-16.  hi lies below the weight, so lo
// is positive too: an infinite value gives an infinity, never inf - inf or 0 inf.
__device__ __forceinline__ void split_weights(float p0, float p1, uint32_t& hi, uint32_t& lo) {
  const uint32_t h0 = __float_as_uint(p0 * 0.998f) & 0xffff0000u, h1 = __float_as_uint(p1 * 0.998f) & 0xffff0000u;
  hi = h0 >> 16 | h1;
  const __nv_bfloat162 l = __floats2bfloat162_rn(p0 - __uint_as_float(h0), p1 - __uint_as_float(h1));
  lo = *reinterpret_cast<const uint32_t*>(&l);
}

// One warp's tile of queries and its running sums, 16 tokens a step: keys and values are read
// from shared memory once, straight into MMA operands, whatever the number of queries; at 1.1
// to 1.4 us per step of an SM's eight warps HBM is the slower (0.65 us alone).  PACK: up to 8 queries, rows 0-7
// of the tile; the value product's rows 8-15 take the low halves of the weights, so
// that two-term weights cost no further MMA.  Otherwise up to 16 queries and two MMAs.
template <class Z, bool PACK>
struct TensorTile {
  static constexpr int kQ = PACK ? 1 : 2;  // query rows per lane
  static constexpr int kRows = PACK ? 8 : 16, kOperands = 16;
  static __device__ __forceinline__ void lay_out(const uint8_t*, uint8_t*) {}
  float o[Z::DP / 8][4], m[kQ], l[kQ];
  uint32_t q[Z::DP / 16][2 * kQ];

  // `place`: the queries in shared memory.
  __device__ __forceinline__ void begin(uint32_t place, int lane) {
    const int row = PACK ? lane & 7 : lane & 15, c = PACK ? lane >> 3 : lane >> 4;
#pragma unroll
    for (int k = 0; k < Z::DP / 16; k += PACK ? 2 : 1) {
      uint32_t r[4];
      ldmatrix4_plain(r, place + row * Z::kRow + ((2 * k + c) ^ (row & 7)) * 16);
      if (PACK) {
        q[k][0] = r[0], q[k][1] = r[1], q[k + 1][0] = r[2], q[k + 1][1] = r[3];
      } else {
#pragma unroll
        for (int y = 0; y < 4; ++y) q[k][y % (2 * kQ)] = r[y];
      }
    }
#pragma unroll
    for (int x = 0; x < kQ; ++x) {
      m[x] = -CUDART_INF_F;
      l[x] = 0.f;
    }
#pragma unroll
    for (int n = 0; n < Z::DP / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
  }

  // The 16 tokens of a stage, the first `live` of them present (0 or fewer: none).
  __device__ __forceinline__ void step(uint32_t keys, int live, int lane, const ScoreScale& scale, float*) {
    if (live <= 0) return;
    float s[2][4] = {};
    {
      const int row = (lane & 7) + (lane >> 4) * 8, c = lane >> 3 & 1;
      const uint32_t at = keys + row * Z::kRow + (c ^ (row & 7)) * 16;
      float s2[2][4] = {};  // every other k-step: chains of half the length
#pragma unroll
      for (int k = 0; k < Z::DP / 16; ++k) {
        uint32_t b[4];
        ldmatrix4(b, at, k);
        float(&t)[2][4] = k & 1 ? s2 : s;
        if (PACK) {
          mma16816(t[0], q[k][0], 0u, q[k][1], 0u, b[0], b[1]);
          mma16816(t[1], q[k][0], 0u, q[k][1], 0u, b[2], b[3]);
        } else {
          mma16816(t[0], q[k][0], q[k][1], q[k][2 % (2 * kQ)], q[k][3 % (2 * kQ)], b[0], b[1]);
          mma16816(t[1], q[k][0], q[k][1], q[k][2 % (2 * kQ)], q[k][3 % (2 * kQ)], b[2], b[3]);
        }
      }
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int y = 0; y < (PACK ? 2 : 4); ++y) s[n][y] += s2[n][y];
    }
    if (PACK) {  // rows 8-15 of the tile hold nothing
      float v[4] = {s[0][0], s[0][1], s[1][0], s[1][1]};
      scale.apply(v);
      s[0][0] = v[0], s[0][1] = v[1], s[1][0] = v[2], s[1][1] = v[3];
    } else {
      scale.apply(s[0]);
      scale.apply(s[1]);
    }
    if (live < 16) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int y = 0; y < 4; ++y)
          if (n * 8 + (lane & 3) * 2 + (y & 1) >= live) s[n][y] = -CUDART_INF_F;
    }
    uint32_t hi[kQ][2], lo[kQ][2];
    // m need not be the maximum, only near it: raised where a score is 2^8 above
    bool raise = false;
#pragma unroll
    for (int x = 0; x < kQ; ++x)
#pragma unroll
      for (int n = 0; n < 2; ++n) raise |= fmaxf(s[n][2 * x], s[n][2 * x + 1]) > m[x] + kHeadroom;
    if (__any_sync(~0u, raise)) {
#pragma unroll
      for (int x = 0; x < kQ; ++x) {
        float top = fmaxf(fmaxf(fmaxf(s[0][2 * x], s[0][2 * x + 1]), fmaxf(s[1][2 * x], s[1][2 * x + 1])), m[x]);
        top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
        top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
        const float c = m[x] == top ? 1.f : exp2_approx(m[x] - top);
        m[x] = top;
        l[x] *= c;
#pragma unroll
        for (int n = 0; n < Z::DP / 8; ++n) {
          o[n][2 * x] *= c, o[n][2 * x + 1] *= c;
          if (PACK) o[n][2] *= c, o[n][3] *= c;
        }
      }
    }
#pragma unroll
    for (int x = 0; x < kQ; ++x) {
      const float base = m[x] == -CUDART_INF_F ? 0.f : m[x];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const float p0 = exp2_approx(s[n][2 * x] - base), p1 = exp2_approx(s[n][2 * x + 1] - base);
        l[x] += p0 + p1;
        split_weights(p0, p1, hi[x][n], lo[x][n]);
      }
    }
    const uint32_t vals = keys + Z::kHalf;
    const int row = lane & 15, c = lane >> 4;
    const uint32_t at = vals + row * Z::kRow + (c ^ (row & 7)) * 16;
#pragma unroll
    for (int n = 0; n < Z::DP / 16; ++n) {
      uint32_t b[4];
      ldmatrix4_trans(b, at, n);
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        if (PACK) {
          mma16816(o[2 * n + y], hi[0][0], lo[0][0], hi[0][1], lo[0][1], b[2 * y], b[2 * y + 1]);
        } else {
          mma16816(o[2 * n + y], hi[0][0], hi[kQ - 1][0], hi[0][1], hi[kQ - 1][1], b[2 * y], b[2 * y + 1]);
          mma16816(o[2 * n + y], lo[0][0], lo[kQ - 1][0], lo[0][1], lo[kQ - 1][1], b[2 * y], b[2 * y + 1]);
        }
      }
    }
  }

  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int x = 0; x < kQ; ++x) {
      l[x] += __shfl_xor_sync(~0u, l[x], 1);
      l[x] += __shfl_xor_sync(~0u, l[x], 2);
    }
    if (PACK)
#pragma unroll
      for (int n = 0; n < Z::DP / 8; ++n) o[n][0] += o[n][2], o[n][1] += o[n][3];
  }
  // This lane's kMine rows, and f(element, value, next value) for its pairs of elements below d of row x.
  static constexpr int kMine = kQ;
  static __device__ __forceinline__ int row(int x, int lane) { return lane / 4 + 8 * x; }
  static __device__ __forceinline__ bool speaks(int lane) { return (lane & 3) == 0; }  // one lane per row
  template <class F>
  __device__ __forceinline__ void each(int x, int lane, int d, F f) const {
#pragma unroll
    for (int n = 0; n < Z::DP / 8; ++n)
      if (n * 8 < d) f(n * 8 + (lane & 3) * 2, o[n][2 * x], o[n][2 * x + 1]);
  }
};

// ---------------------------------------------------------------------------
// fp32: CUDA cores
// ---------------------------------------------------------------------------

// Up to ROWS queries, 8 tokens a stage (products on tensor cores would round to 10 bits).  A
// lane owns chunks of four elements, of the queries and the output in registers and of each key
// and value it reads once; a token's products with all queries are summed up over the lanes by
// exchanging halves (5 steps for all tokens and rows), so that lane 4 t + j ends with token t and
// the rows of row_of.  HBM bounds it up to four queries: 64 x 4096 tokens of 32 query heads on 8
// KV heads, 2.1 GB, 309 us.  With 16 queries on one KV head (268 MB there) 91 us, bound by the
// length of a step with eight warps on an SM; with queries in shared memory, read by eight lanes
// a token (no exchanges, but eight times the loads), 128.
template <class Z, int ROWS>
struct SimtTile {
  static constexpr int kRows = ROWS, kOperands = 16;
  static __device__ __forceinline__ void lay_out(const uint8_t*, uint8_t*) {}
  static constexpr int kOwn = Z::kChunks >= 32 ? Z::kChunks / 32 : 1;  // chunks per lane
  static constexpr int kSplit = Z::kChunks >= 32 ? 1 : 32 / Z::kChunks;  // lanes that share a chunk, by tokens
  static constexpr int kVals = ROWS > 4 ? ROWS / 4 : 1;                  // scores per lane
  static_assert(Z::TOK == 8 && kSplit <= 2 && (ROWS & (ROWS - 1)) == 0 && ROWS <= 8, "lanes by tokens and rows");
  float4 q[ROWS][kOwn], o[ROWS][kOwn];
  float near[kVals], sum[kVals];  // this lane's reference maxima and sums
  float m[ROWS], l[ROWS];         // all of them, after finish

  static __device__ __forceinline__ int row_of(int i, int lane) { return (lane & 3) * ROWS / 4 + i; }
  static __device__ __forceinline__ int chunk_of(int k, int lane) { return (kSplit > 1 ? lane % Z::kChunks : lane) + 32 * k; }
  static __device__ __forceinline__ float4 chunk(uint32_t at) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at));
    return v;
  }
  // x of row r from the lane that has it to all
  static __device__ __forceinline__ float of_row(const float (&x)[kVals], int r) {
    return __shfl_sync(~0u, x[r % kVals], r * 4 / ROWS);
  }

  // `place`: the queries in shared memory, as long as it lasts.
  __device__ __forceinline__ void begin(uint32_t place, int lane) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
      for (int k = 0; k < kOwn; ++k) {
        q[r][k] = chunk(place + r * Z::kRow + (chunk_of(k, lane) ^ (r & 7)) * 16);
        o[r][k] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
    for (int i = 0; i < kVals; ++i) near[i] = -CUDART_INF_F, sum[i] = 0.f;
  }

  // This lane's share of the products of a token with all queries.
  __device__ __forceinline__ void products(uint32_t keys, int tok, int lane, float (&s)[ROWS]) const {
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
      const float4 x = chunk(keys + tok * Z::kRow + (chunk_of(k, lane) ^ tok) * 16);
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const float4 y = q[r][k];
        const float rest = fmaf(x.y, y.y, fmaf(x.z, y.z, x.w * y.w));
        s[r] = k ? s[r] + fmaf(x.x, y.x, rest) : fmaf(x.x, y.x, rest);
      }
    }
  }
  // Sums over the lanes that differ in bit O, of the lower half of s where it is clear, else the upper.
  template <int N, int O>
  static __device__ __forceinline__ void halve(float (&s)[4 * ROWS], int lane) {
    const bool up = lane & O;
    if (N == 1) {
      s[0] += __shfl_xor_sync(~0u, s[0], O);
    } else {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const float give = up ? s[i] : s[i + N / 2], keep = up ? s[i + N / 2] : s[i];
        s[i] = keep + __shfl_xor_sync(~0u, give, O);
      }
    }
  }

  __device__ __forceinline__ void step(uint32_t keys, int live, int lane, const ScoreScale& scale, float* weights) {
    if (live <= 0) return;
    const int t = lane >> 2;
    float s[4 * ROWS];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float x[ROWS];
      if (kSplit > 1) {
        products(keys, i + (lane >> 4) * 4, lane, x);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) s[i * ROWS + r] = x[r];
      } else {
        float y[ROWS];
        products(keys, i, lane, x);
        products(keys, i + 4, lane, y);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
          const float give = lane & 16 ? x[r] : y[r], keep = lane & 16 ? y[r] : x[r];
          s[i * ROWS + r] = keep + __shfl_xor_sync(~0u, give, 16);
        }
      }
    }
    halve<4 * ROWS, 8>(s, lane);
    halve<2 * ROWS, 4>(s, lane);
    halve<ROWS, 2>(s, lane);
    halve<(ROWS > 1 ? ROWS / 2 : 1), 1>(s, lane);
    float v[kVals];
#pragma unroll
    for (int i = 0; i < kVals; ++i) v[i] = s[i];
    scale.apply(v);
    bool raise = false;  // as in TensorTile
#pragma unroll
    for (int i = 0; i < kVals; ++i) {
      if (t >= live) v[i] = -CUDART_INF_F;
      raise |= v[i] > near[i] + kHeadroom;
    }
    if (__any_sync(~0u, raise)) {
      float c[kVals];
#pragma unroll
      for (int i = 0; i < kVals; ++i) {
        float top = fmaxf(near[i], v[i]);
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, x));
        c[i] = near[i] == top ? 1.f : exp2_approx(near[i] - top);
        near[i] = top;
        sum[i] *= c[i];
      }
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const float cr = of_row(c, r);
#pragma unroll
        for (int k = 0; k < kOwn; ++k) o[r][k].x *= cr, o[r][k].y *= cr, o[r][k].z *= cr, o[r][k].w *= cr;
      }
    }
#pragma unroll
    for (int i = 0; i < kVals; ++i) {
      v[i] = exp2_approx(v[i] - (near[i] == -CUDART_INF_F ? 0.f : near[i]));
      sum[i] += v[i];
      weights[t * ROWS + row_of(i, lane)] = v[i];  // (the same from lanes that share a score)
    }
    __syncwarp();
    const uint32_t vals = keys + Z::kHalf;
#pragma unroll
    for (int i = 0; i < Z::TOK / kSplit; ++i) {
      const int tok = i * kSplit + (kSplit > 1 ? lane / Z::kChunks : 0);
      float p[ROWS];
      if (ROWS >= 4) {
#pragma unroll
        for (int r = 0; r < ROWS; r += 4) {
          const float4 w = *reinterpret_cast<const float4*>(weights + tok * ROWS + r);
          p[r] = w.x, p[(r + 1) % ROWS] = w.y, p[(r + 2) % ROWS] = w.z, p[(r + 3) % ROWS] = w.w;
        }
      } else {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) p[r] = weights[tok * ROWS + r];
      }
#pragma unroll
      for (int k = 0; k < kOwn; ++k) {
        const float4 x = chunk(vals + tok * Z::kRow + (chunk_of(k, lane) ^ (tok & 7)) * 16);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
          o[r][k].x = fmaf(p[r], x.x, o[r][k].x);
          o[r][k].y = fmaf(p[r], x.y, o[r][k].y);
          o[r][k].z = fmaf(p[r], x.z, o[r][k].z);
          o[r][k].w = fmaf(p[r], x.w, o[r][k].w);
        }
      }
    }
    __syncwarp();  // the weights are read
  }

  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int i = 0; i < kVals; ++i)
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) sum[i] += __shfl_xor_sync(~0u, sum[i], x);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      m[r] = of_row(near, r);
      l[r] = of_row(sum, r);
#pragma unroll
      for (int x = 32 / kSplit; x < 32; x <<= 1) {
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
          o[r][k].x += __shfl_xor_sync(~0u, o[r][k].x, x);
          o[r][k].y += __shfl_xor_sync(~0u, o[r][k].y, x);
          o[r][k].z += __shfl_xor_sync(~0u, o[r][k].z, x);
          o[r][k].w += __shfl_xor_sync(~0u, o[r][k].w, x);
        }
      }
    }
  }
  static constexpr int kMine = ROWS;
  static __device__ __forceinline__ int row(int x, int) { return x; }
  static __device__ __forceinline__ bool speaks(int lane) { return lane == 0; }
  template <class F>
  __device__ __forceinline__ void each(int x, int lane, int d, F f) const {
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
      const int e = 4 * chunk_of(k, lane);
      if (lane < 32 / kSplit && e < d) {
        f(e, o[x][k].x, o[x][k].y);
        f(e + 2, o[x][k].z, o[x][k].w);
      }
    }
  }
};

// ---------------------------------------------------------------------------
// the kernel
// ---------------------------------------------------------------------------

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// The address in CTA `rank`'s shared memory of what `p` is in this one's.
__device__ __forceinline__ uint32_t remote(const void* p, uint32_t rank) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ void store_remote(uint32_t at, float4 v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(at), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void store_remote(uint32_t at, float2 v) {
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1,%2};" ::"r"(at), "f"(v.x), "f"(v.y) : "memory");
}

// Two or four elements of an output row, 4-byte aligned for bf16 where `even`.
__device__ __forceinline__ void put2(float* p, float x, float y, bool) { p[0] = x, p[1] = y; }
__device__ __forceinline__ void put2(__nv_bfloat16* p, float x, float y, bool even) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(x, y);
  if (even) *reinterpret_cast<__nv_bfloat162*>(p) = a;
  else p[0] = a.x, p[1] = a.y;
}
__device__ __forceinline__ void put4(float* p, float4 v, bool) { p[0] = v.x, p[1] = v.y, p[2] = v.z, p[3] = v.w; }
__device__ __forceinline__ void put4(__nv_bfloat16* p, float4 v, bool even) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
  if (even) {
    reinterpret_cast<__nv_bfloat162*>(p)[0] = a;
    reinterpret_cast<__nv_bfloat162*>(p)[1] = b;
  } else {
    p[0] = a.x, p[1] = a.y, p[2] = b.x, p[3] = b.y;
  }
}

template <class Z, class Tile, bool CLUSTER>
struct Shared {  // after the rings
  // places for queries: as many segments as tiles are copied ahead
  static constexpr int kPlaces = CLUSTER ? 1 : Z::S;
  alignas(16) uint8_t q[Z::NW * kPlaces * Tile::kRows * Z::kQRow];
  float4 part[CLUSTER ? Tile::kRows * Z::DP / 4 : 1];  // of the cluster's CTAs, this one's share of the elements
  float2 cluster_ml[CLUSTER ? kMaxCluster : 1][Tile::kRows];
  alignas(16) float mine[std::is_same<typename Z::T, float>::value && !Z::kQuant ? Z::NW * 8 * Tile::kRows : 4];  // fp32: a warp's weights
  alignas(16) float2 ml[Z::NW][Tile::kRows];  // sum -1: a page outside the pool
};

template <class Z, class Tile, bool CLUSTER>
constexpr size_t shared_bytes(int B) {
  return Z::kRing + sizeof(Shared<Z, Tile, CLUSTER>) + (CLUSTER ? 0 : sizeof(int) * (B + 1 + (B <= kKeptLens ? B : 0)));
}

// The maximum and sum that `n` partial sums have together, and each one's weight.
struct Joined {
  float m, l;
  bool bad;
};
template <int MOST, class F>
__device__ __forceinline__ Joined join_rows(int n, float (&weight)[MOST], F ml_of) {
  Joined r = {-CUDART_INF_F, 0.f, false};
  float l[MOST];
#pragma unroll
  for (int k = 0; k < MOST; ++k) {
    weight[k] = -CUDART_INF_F;
    l[k] = 0.f;
    if (k < n) {
      const float2 v = ml_of(k);
      weight[k] = v.x, l[k] = v.y;
      r.bad |= v.y < 0.f;
      r.m = fmaxf(r.m, v.x);
    }
  }
  const float base = r.m == -CUDART_INF_F ? 0.f : r.m;
#pragma unroll
  for (int k = 0; k < MOST; ++k) {
    weight[k] = exp2_approx(weight[k] - base);
    r.l += l[k] * weight[k];
  }
  return r;
}

template <class Z, class Tile, bool CLUSTER>
__global__ void __launch_bounds__(Z::NW * 32, Z::NW == warps_of(Z::DP, true) ? 1 : kPerSm)
    paged_decode_kernel(const __grid_constant__ Args g) {
  using T = typename Z::T;
  extern __shared__ __align__(128) uint8_t raw[];
  using Shm = Shared<Z, Tile, CLUSTER>;
  Shm& sh = *reinterpret_cast<Shm*>(raw + Z::kRing);
  const PagedDecodeArgs& a = g.a;
  static_assert(Z::kRing % 16 == 0 && offsetof(Shm, mine) % 16 == 0 && sizeof(Shm) % 16 == 0, "16-byte accesses");
  static_assert(Z::kStage >= Tile::kRows * Z::DP * 4, "a warp's sums in a stage");
  Batch batch;
  batch.prefix = reinterpret_cast<int*>(raw + Z::kRing + sizeof(sh));
  batch.len = a.B <= kKeptLens ? batch.prefix + a.B + 1 : nullptr;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n_heads = g.p.wh, n_runs = g.p.wt, wh = warp & (n_heads - 1), wt = warp / n_heads;
  const int d = a.v.d;
  T* out = static_cast<T*>(a.out);
  const bool even = (reinterpret_cast<uintptr_t>(out) & 3) == 0;
  pdl_launch_dependents();
  pdl_wait();

  int n_tiles = 0;
  Ranges ranges(0, 0);
  int u0, u1;
  Walk ahead;
  bool begins = true;  // the first (head group, sequence) is this CTA's from its first tile on
  uint32_t rank = 0;
  const typename LoaderOf<Z, Tile::kRows, Shm::kPlaces>::type load(g, raw, sh.q, warp, lane, wh, wt);
  load.clear(raw);
  if (CLUSTER) {
    cluster_arrive();  // remote stores must find the other CTAs running: waited for before the first
    rank = cluster_rank();
    const int pair = blockIdx.x / g.p.cluster;
    ahead.group = pair / a.B;
    ahead.b = pair - ahead.group * a.B;
    bool bad;
    const int span = visible(a, ahead.b, ahead.token, bad), tiles = (span + g.p.tile - 1) / g.p.tile;
    if (bad && ahead.group == 0 && rank == 0 && threadIdx.x == 0) atomicOr(a.err, kErrBadSeq);
    ahead.len = span + ahead.token;
    u0 = (int)rank * tiles / g.p.cluster;
    u1 = ((int)rank + 1) * tiles / g.p.cluster;
    ahead.token += u0 * g.p.tile;
    ahead.left = u1 - u0;
  } else {
    n_tiles = tile_prefix<Z::NW>(a, g.p.by_tile, g.p.groups, batch.prefix, batch.len, blockIdx.x == 0);
    const int units = g.p.groups * n_tiles;
    ranges = Ranges(units, min(g.p.n_items, units));
    // empty sequences
    for (int b = blockIdx.x; b < a.B; b += gridDim.x)
      if (batch.prefix[b + 1] == batch.prefix[b]) {
        for (int e = threadIdx.x; e < a.v.Hq * d; e += Z::NW * 32) out[(int64_t)b * a.v.Hq * d + e] = from_f32<T>(0.f);
        if (a.lse)
          for (int j = threadIdx.x; j < a.v.Hq; j += Z::NW * 32) a.lse[(int64_t)b * a.v.Hq + j] = -CUDART_INF_F;
      }
    if ((int)blockIdx.x >= ranges.n) {
      if (threadIdx.x == 0) g.entries[blockIdx.x].last = -1;
      return;
    }
    u0 = ranges.begin(blockIdx.x);
    u1 = ranges.begin(blockIdx.x + 1);
    begins = ahead.enter(a, batch, n_tiles, g.p.tile, u0);
  }

  Walk at = ahead;
  int to_compute = u1 - u0, to_copy = to_compute, to_fetch = to_compute;
  // page numbers are read two tiles ahead of the copies: a read takes longer than a tile's arithmetic
  Pages pages = {0, -1, 0, -1}, pages2 = {0, -1, 0, -1};
  bool first = true;  // of its (head group, sequence), for this CTA
  const auto fetch_next = [&]() {
    const Pages p = load.fetch(ahead, first);
    first = false;
    ahead.token += g.p.tile;
    if (--to_fetch > 0 && --ahead.left == 0 && !CLUSTER) {
      ahead.leave(a, batch);
      first = true;
    }
    return p;
  };
  if (to_fetch > 0) pages = fetch_next();
  if (to_fetch > 0) pages2 = fetch_next();
  uint32_t outside = 0;  // bit s: stage s has a page outside the pool
  int put = 0;           // stage that the next copies go to
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
  if (CLUSTER) {  // the queries by themselves, before the copies
    qs = queries_of(g, at.group, wh);
    if (g.p.q_copied) load.copy_queries({0, 0, at.group, at.b}, 0);
    else load.read_queries(qs, at.b, sh.q, warp, 0);
    cp_async_commit();
  }
#pragma unroll 1
  for (int i = 0; i < Z::S - 1; ++i) copy_next();

  int get = 0, nth = 0;  // nth: this (head group, sequence) among the CTA's
  bool bad = false, fresh = !CLUSTER;
  if (CLUSTER) {
    cp_async_wait<Z::S - 1>();
    __syncwarp();
    tile.begin(load.places, lane);
  }
  while (true) {
    if (!CLUSTER || to_compute > 0) {
      __syncwarp();  // the stage that is filled next has been read
      copy_next();
      cp_async_wait<Z::S - 1>();
      __syncwarp();
      if (!CLUSTER && fresh) {
        qs = queries_of(g, at.group, wh);
        if (!g.p.q_copied) load.read_queries(qs, at.b, sh.q, warp, get);
        tile.begin(load.places + get * load.kPlace, lane);
        fresh = false;
      }
      bad |= outside >> get & 1;
      tile.step(load.ring + get * Z::kStage, at.len - at.token - load.run, lane, g.score, mine);
    }
    const int used = get;
    get = get + 1 == Z::S ? 0 : get + 1;
    at.token += g.p.tile;
    const bool ends = --at.left <= 0, last = --to_compute <= 0;
    if (!ends && !last) continue;
    // the end of a (head group, sequence), or of this CTA's part of it
    const bool whole = CLUSTER ? g.p.cluster == 1 : begins && ends;
    if (bad && lane == 0) atomicOr(a.err, kErrBadSeq);
    tile.finish();
    const int64_t out_row = (int64_t)at.b * a.v.Hq + qs.first;
    const int64_t part_row = CLUSTER ? 0 : (int64_t)((2 * blockIdx.x + (nth > 0)) * n_heads + wh) * g.p.rows;
    // the sum of row r (lse, or the partial's maximum and sum)
    const auto put_sum = [&](int r, const Joined& j) {
      if (!whole) *reinterpret_cast<float2*>(g.part_ml + 2 * (part_row + r)) = make_float2(j.m, j.bad ? -1.f : j.l);
      else if (a.lse) a.lse[out_row + r] = j.bad || j.l == 0.f ? -CUDART_INF_F : (j.m + log2f(j.l)) * 0.693147180559945f;
    };
    if (n_runs == 1) {
#pragma unroll
      for (int x = 0; x < Tile::kMine; ++x) {
        const int r = Tile::row(x, lane);
        if (r >= qs.count) continue;
        const bool none = bad || tile.l[x] == 0.f;
        if (Tile::speaks(lane)) put_sum(r, {tile.m[x], tile.l[x], bad});
        if (whole) {
          const float f = 1.f / tile.l[x];
          T* p = out + (out_row + r) * d;
          tile.each(x, lane, d, [&](int e, float y, float z) {
            put2(p + e, none ? 0.f : y * f, none ? 0.f : z * f, even);
          });
        } else {
          float* p = g.part_u + (part_row + r) * Z::DP;
          tile.each(x, lane, d, [&](int e, float y, float z) { *reinterpret_cast<float2*>(p + e) = make_float2(y, z); });
        }
      }
    } else {
      // The head's runs of tokens join: each warp leaves its sums in the stage that it has
      // just read (not filled again before the barrier behind), then all of them add up.
      float* left = reinterpret_cast<float*>(raw + (warp * Z::S + used) * Z::kStage);
#pragma unroll
      for (int x = 0; x < Tile::kMine; ++x) {
        const int r = Tile::row(x, lane);
        if (Tile::speaks(lane)) sh.ml[warp][r] = make_float2(tile.m[x], bad ? -1.f : tile.l[x]);
        tile.each(x, lane, d, [&](int e, float y, float z) {
          *reinterpret_cast<float2*>(left + r * Z::DP + (e ^ (r & 7) * 8)) = make_float2(y, z);
        });
      }
      __syncthreads();
      if (CLUSTER && g.p.cluster > 1) cluster_wait();
      for (int i = wt * 32 + lane; i < qs.count * (Z::DP / 4); i += n_runs * 32) {
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
        if (CLUSTER && g.p.cluster > 1) {
          const int at_rank = rank * (Tile::kRows * Z::DP / 4 / g.p.cluster);
          store_remote(remote(&sh.part[i / g.p.cluster + at_rank], i % g.p.cluster), sum);
          if (e == 0)
            for (int c = 0; c < g.p.cluster; ++c)
              store_remote(remote(&sh.cluster_ml[rank][r], c), make_float2(j.m, j.bad ? -1.f : j.l));
        } else if (whole) {
          const float f = j.bad || j.l == 0.f ? 0.f : 1.f / j.l;
          put4(out + (out_row + r) * d + e,
               f == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(sum.x * f, sum.y * f, sum.z * f, sum.w * f), even);
          if (e == 0) put_sum(r, j);
        } else {
          *reinterpret_cast<float4*>(g.part_u + (part_row + r) * Z::DP + e) = sum;
          if (e == 0) put_sum(r, j);
        }
      }
      if (!CLUSTER) {
        __syncthreads();
        load.clear_stage(reinterpret_cast<uint8_t*>(left));
      }
    }
    if (last) {
      if (!CLUSTER && threadIdx.x == 0)
        g.entries[blockIdx.x] = {at.b, at.group, begins && !ends ? ranges.item_of(u1 + at.left - 1) : -1, nth > 0};
      break;
    }
    bad = false;
    begins = fresh = true;
    ++nth;
    at.leave(a, batch);
  }
  cp_async_wait<0>();
  if (!CLUSTER) return;
  if (g.p.cluster == 1) {
    cluster_wait();
    return;
  }
  // Every CTA of the cluster has sent its sums: each joins its share of the elements.
  cluster_arrive();
  cluster_wait();
  const int per = Tile::kRows * Z::DP / 4 / g.p.cluster;
  for (int i = threadIdx.x * g.p.cluster + rank; i < qs.count * (Z::DP / 4); i += Z::NW * 32 * g.p.cluster) {
    const int r = i / (Z::DP / 4), e = i % (Z::DP / 4) * 4;
    if (e >= d) continue;
    float w[kMaxCluster];
    const Joined j = join_rows<kMaxCluster>(g.p.cluster, w, [&](int k) { return sh.cluster_ml[k][r]; });
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kMaxCluster; ++k)
      if (k < g.p.cluster && w[k] != 0.f) {
        const float4 v = sh.part[i / g.p.cluster + k * per];
        sum.x += v.x * w[k], sum.y += v.y * w[k], sum.z += v.z * w[k], sum.w += v.w * w[k];
      }
    const int64_t row = (int64_t)at.b * a.v.Hq + qs.first + r;
    const float f = j.bad || j.l == 0.f ? 0.f : 1.f / j.l;
    put4(out + row * d + e,
         f == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(sum.x * f, sum.y * f, sum.z * f, sum.w * f), even);
    if (e == 0 && a.lse) a.lse[row] = j.bad || j.l == 0.f ? -CUDART_INF_F : (j.m + log2f(j.l)) * 0.693147180559945f;
  }
}

// ---------------------------------------------------------------------------
// launch
// ---------------------------------------------------------------------------

template <class Z, class Tile, bool CLUSTER>
cudaError_t launch_kernel(const Args& g, cudaStream_t s) {
  const auto k = paged_decode_kernel<Z, Tile, CLUSTER>;
  static std::atomic<uint64_t> ready{0};  // devices on which the kernel may use its shared memory
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev > 63 || !(ready.load(std::memory_order_relaxed) >> dev & 1)) {
    const size_t most = std::max(shared_bytes<Z, Tile, CLUSTER>(kMaxBatch), shared_bytes<Z, Tile, CLUSTER>(kKeptLens));
    e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
    if (e != cudaSuccess) return e;
    if (dev < 64) ready.fetch_or(uint64_t(1) << dev, std::memory_order_relaxed);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = CLUSTER ? g.p.groups * g.a.B * g.p.cluster : g.p.n_items;
  cfg.blockDim = Z::NW * 32;
  cfg.dynamicSmemBytes = shared_bytes<Z, Tile, CLUSTER>(g.a.B);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = CLUSTER ? g.p.cluster : 1;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = CLUSTER ? 2 : 1;
  e = cudaLaunchKernelEx(&cfg, k, g);
  if (e != cudaSuccess) return e;
  return hook_launched(g.a.hook, s);
}

}  // namespace paged
}  // namespace dck

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
#include <math_constants.h>

#include <algorithm>
#include <type_traits>

#include "paged.cuh"

namespace dck {
namespace {

// How the heads of a call are laid over warps and CTAs.
struct PagedPlan {
  int chunks, rows;  // a KV head's queries: `chunks` tiles of up to `rows`
  int wh, wt;        // warps of a CTA: wh heads (a power of two) x wt runs of tokens
  int groups;        // head groups: Hkv * chunks / wh
  int tile;          // tokens of a CTA's tile
  int n_items;       // CTAs
  Divider by_chunks;
};

struct Entry {  // a (head group, sequence) shared by CTAs c0 .. c1
  int pair, c0, c1, second;  // second: the partial is c0's second one
};

struct Header {
  int n_entries;
};

struct PagedKernelArgs {
  PagedDecodeArgs a;
  PagedPlan p;
  float* part_u;   // [2 n_items][wh][rows][DP]
  float* part_ml;  // [2 n_items][wh][rows][2]: maximum (log2 units), sum (-1: a page outside the pool)
  Header* header;
  Entry* entries;  // [n_items]
};

constexpr int kMaxLen = 1 << 30;     // tokens of a sequence
constexpr int kTileLimit = 1 << 30;  // tiles of one call's sequences, per head group

// Visible tokens of sequence b and the first of them; 0 for invalid lengths.
__device__ __forceinline__ int visible(const PagedDecodeArgs& a, int b, int& first, bool& bad) {
  const int L = a.seq_len[b];
  bad = L < 0 || L > a.max_len || L > kMaxLen || (L > 0 && (int64_t)a.v.by_page.div(L - 1) >= a.table_stride);
  first = a.window > 0 && L > a.window ? L - a.window : 0;
  return bad ? 0 : L - first;
}

// Exclusive prefix sums of the sequences' tile counts in shared memory
// prefix[0..B].  Called by the whole block.
template <int NW>
__device__ __forceinline__ int tile_prefix(const PagedDecodeArgs& a, int tile, int* prefix, bool report) {
  __shared__ int64_t scratch[NW];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int64_t base = 0;
  for (int b0 = 0; b0 < a.B; b0 += NW * 32) {
    const int b = b0 + tid;
    int64_t n = 0;
    if (b < a.B) {
      int first;
      bool bad;
      const int span = visible(a, b, first, bad);
      if (bad && report) atomicOr(a.err, kErrBadSeq);
      n = (span + (int64_t)tile - 1) / tile;
    }
    int64_t v = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(~0u, v, o);
      if (lane >= o) v += y;
    }
    if (lane == 31) scratch[warp] = v;
    __syncthreads();
    int64_t before = base;
    for (int w = 0; w < NW; ++w) {
      const int64_t y = scratch[w];
      if (w < warp) before += y;
      base += y;
    }
    if (b < a.B) {
      if (before + v > kTileLimit && n > 0 && report) atomicOr(a.err, kErrBadSeq);
      prefix[b] = (int)min(before + v - n, (int64_t)kTileLimit);
    }
    base = min(base, (int64_t)kTileLimit);
    __syncthreads();
  }
  if (tid == 0) prefix[a.B] = (int)base;
  __syncthreads();
  return prefix[a.B];
}

__device__ __forceinline__ int64_t range_begin(int c, int64_t units, int n) { return (int64_t)c * units / n; }
__device__ __forceinline__ int item_of(int64_t u, int64_t units, int n) { return (int)(((u + 1) * n + units - 1) / units) - 1; }

// A position in the flattened list of tiles (head groups outermost).
struct Cursor {
  int64_t u, start, end;  // the tile, and the range of its (head group, sequence)
  int b, group, first, len;

  __device__ __forceinline__ void enter(const PagedDecodeArgs& a, const int* prefix, int n_tiles, int64_t at) {
    u = at;
    group = (int)(at / n_tiles);
    const int64_t base = (int64_t)group * n_tiles;
    b = seq_of_tile(prefix, a.B, (int)(at - base));
    start = base + prefix[b];
    end = base + prefix[b + 1];
    bool bad;
    len = visible(a, b, first, bad) + first;
  }
  __device__ __forceinline__ void next(const PagedDecodeArgs& a, const int* prefix, int n_tiles, int64_t stop) {
    if (++u < end || u >= stop) return;
    enter(a, prefix, n_tiles, u);
  }
  __device__ __forceinline__ int token(int tile) const { return first + (int)(u - start) * tile; }
};

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 16-byte asynchronous copy of `bytes` (16 or 0) bytes, the rest zero.
__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// Sizes of a variant: elements T, head dim up to DP, NW warps, S stages of TOK tokens.
template <typename T_, int DP_, int NW_, int S_, int TOK_>
struct Sizes {
  using T = T_;
  static constexpr int DP = DP_, NW = NW_, S = S_, TOK = TOK_;
  static constexpr int kRow = DP * sizeof(T);   // bytes of a head's row
  static constexpr int kChunks = kRow / 16;     // 16-byte chunks of it
  static constexpr int kHalf = TOK * kRow;      // a stage's keys (values: the same)
  static constexpr int kStage = 2 * kHalf;
  static constexpr int kRing = NW * S * kStage;
};

// The page numbers and offsets of one warp's run of a tile: lane r holds token r.
struct Pages {
  int page, off, head;
  bool valid;
};

template <class Z>
struct Loader {
  const PagedKernelArgs& g;
  uint32_t ring;  // this warp's stages
  int lane, wh, wt;

  __device__ __forceinline__ Pages fetch(const Cursor& c) const {
    Pages r;
    const int t = c.token(g.p.tile) + wt * Z::TOK + lane;
    r.valid = lane < Z::TOK && t < c.len;
    const uint32_t col = g.a.v.by_page.div(r.valid ? t : 0);
    r.off = t - col * g.a.v.page;
    r.page = r.valid ? g.a.table[(int64_t)c.b * g.a.table_stride + col] : 0;
    r.head = g.p.by_chunks.div(c.group * g.p.wh + wh);
    return r;
  }

  // Starts the copies of a stage; true if a page lies outside the pool (its tokens read as zeros).
  __device__ __forceinline__ bool issue(const Pages& r, int stage) const {
    const PagedView& v = g.a.v;
    const bool outside = r.valid && (r.page < 0 || r.page >= v.n_pages);
    const bool ok = r.valid && !outside;
    const int page = ok ? r.page : 0, off = ok ? r.off : 0;
    const int64_t ko = (int64_t)page * v.k_page + (int64_t)off * v.k_tok + (int64_t)r.head * v.k_head;
    const int64_t vo = (int64_t)page * v.v_page + (int64_t)off * v.v_tok + (int64_t)r.head * v.v_head;
    const uint32_t mask = __ballot_sync(~0u, ok);
    const uint32_t at = ring + stage * Z::kStage;
    constexpr int kPer = Z::kChunks < 32 ? 32 / Z::kChunks : 1;    // rows per instruction
    constexpr int kTurns = Z::kChunks > 32 ? Z::kChunks / 32 : 1;  // instructions per row
    const char* kc = static_cast<const char*>(g.a.kc);
    const char* vc = static_cast<const char*>(g.a.vc);
    const int have = v.d * (int)sizeof(typename Z::T) / 16;  // chunks of a row
#pragma unroll
    for (int i = 0; i < Z::TOK / kPer; ++i) {
      const int row = i * kPer + lane / (32 / kPer);
      const int64_t kr = __shfl_sync(~0u, ko, row), vr = __shfl_sync(~0u, vo, row);
#pragma unroll
      for (int j = 0; j < kTurns; ++j) {
        const int c = lane % (32 / kPer) + 32 * j;
        const int bytes = (mask >> row & 1) && c < have ? 16 : 0;
        const int64_t ce = bytes ? c * 16 : 0;
        const uint32_t dst = at + row * Z::kRow + ((c ^ (row & 7)) * 16);
        cp_async16_or_zero(dst, kc + kr * (int64_t)sizeof(typename Z::T) + ce, bytes);
        cp_async16_or_zero(dst + Z::kHalf, vc + vr * (int64_t)sizeof(typename Z::T) + ce, bytes);
      }
    }
    return __any_sync(~0u, outside);
  }
};

// The queries of one head of a head group: `count` of them from query head `first` on.
struct Queries {
  int first, count;
};
__device__ __forceinline__ Queries queries_of(const PagedKernelArgs& g, int group, int wh) {
  const int vh = group * g.p.wh + wh, h = g.p.by_chunks.div(vh), r0 = (vh - h * g.p.chunks) * g.p.rows;
  return {h * g.a.v.qpg + r0, min(g.p.rows, g.a.v.qpg - r0)};
}

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

// Scores in log2 units.
struct ScoreScale {
  float scale2, inv_cap, cap2;  // cap2 = 0: no cap
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

// ---------------------------------------------------------------------------
// bf16: tensor cores (mma.sync m16n8k16, queries as rows)
// ---------------------------------------------------------------------------

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
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

// One warp's tile of queries and its running sums.  PACK: up to 8 queries, rows 0-7
// of the tile; the value product's rows 8-15 take the low halves of the weights, so
// that two-term weights cost no further MMA.  Otherwise up to 16 queries and two MMAs.
template <class Z, bool PACK>
struct TensorTile {
  static constexpr int kQ = PACK ? 1 : 2;  // query rows per lane
  static constexpr int kRows = PACK ? 8 : 16;
  float o[Z::DP / 8][4], m[kQ], l[kQ];
  uint32_t q[Z::DP / 16][2 * kQ];

  __device__ __forceinline__ void begin(const PagedKernelArgs& g, int b, const Queries& qs, int lane, float*) {
    const int words = g.a.v.d / 8;  // runs of 8 elements in a row
#pragma unroll
    for (int x = 0; x < kQ; ++x) {
      const int r = lane / 4 + 8 * x;
      const uint16_t* src = static_cast<const uint16_t*>(g.a.q) + b * g.a.q_stride +
                            (int64_t)(qs.first + (r < qs.count ? r : 0)) * g.a.v.d + (lane & 3) * 2;
      const int have = r < qs.count ? words : 0;
      if ((reinterpret_cast<uintptr_t>(src) & 3) == 0) {
#pragma unroll
        for (int w = 0; w < Z::DP / 8; ++w)
          q[w / 2][w % 2 * kQ + x] = w < have ? *reinterpret_cast<const uint32_t*>(src + 8 * w) : 0u;
      } else {
#pragma unroll
        for (int w = 0; w < Z::DP / 8; ++w)
          q[w / 2][w % 2 * kQ + x] = w < have ? src[8 * w] | (uint32_t)src[8 * w + 1] << 16 : 0u;
      }
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
#pragma unroll
      for (int k = 0; k < Z::DP / 16; ++k) {
        uint32_t b[4];
        ldmatrix4(b, keys + row * Z::kRow + (((2 * k + c) ^ (row & 7)) * 16));
        if (PACK) {
          mma16816(s[0], q[k][0], 0u, q[k][1], 0u, b[0], b[1]);
          mma16816(s[1], q[k][0], 0u, q[k][1], 0u, b[2], b[3]);
        } else {
          mma16816(s[0], q[k][0], q[k][1], q[k][2 % (2 * kQ)], q[k][3 % (2 * kQ)], b[0], b[1]);
          mma16816(s[1], q[k][0], q[k][1], q[k][2 % (2 * kQ)], q[k][3 % (2 * kQ)], b[2], b[3]);
        }
      }
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
    bool raise = false;
    float top[kQ];
#pragma unroll
    for (int x = 0; x < kQ; ++x) {
      float mx = m[x];
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int y = 0; y < 2; ++y) mx = fmaxf(mx, s[n][2 * x + y]);
      mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 2));
      raise |= mx > m[x];
      top[x] = mx;
    }
    if (__any_sync(~0u, raise)) {
#pragma unroll
      for (int x = 0; x < kQ; ++x) {
        const float c = m[x] == top[x] ? 1.f : exp2_approx(m[x] - top[x]);
        m[x] = top[x];
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
#pragma unroll
    for (int n = 0; n < Z::DP / 16; ++n) {
      uint32_t b[4];
      ldmatrix4_trans(b, vals + row * Z::kRow + (((2 * n + c) ^ (row & 7)) * 16));
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
  // Rows and elements of this lane: f(x, row) for each of its rows, then
  // g(x, element, value, next value) for each pair of elements of row x.
  static constexpr int kMine = kQ;
  static __device__ __forceinline__ int row(int x, int lane) { return lane / 4 + 8 * x; }
  static __device__ __forceinline__ bool speaks(int lane) { return (lane & 3) == 0; }  // one lane per row
  template <class F>
  __device__ __forceinline__ void each(int x, int lane, int e0, int e1, F f) const {
#pragma unroll
    for (int n = 0; n < Z::DP / 8; ++n)
      if (n * 8 >= e0 && n * 8 < e1) f(n * 8 + (lane & 3) * 2, o[n][2 * x], o[n][2 * x + 1]);
  }
  __device__ __forceinline__ void times(int x, float c) {
#pragma unroll
    for (int n = 0; n < Z::DP / 8; ++n) o[n][2 * x] *= c, o[n][2 * x + 1] *= c;
  }
};

// ---------------------------------------------------------------------------
// fp32: CUDA cores
// ---------------------------------------------------------------------------

// Up to ROWS queries, 8 tokens a stage.  Scores: lane = (token, quarter of the
// chunks), the queries from shared memory; values: a lane owns chunks of the output.
template <class Z, int ROWS>
struct SimtTile {
  static constexpr int kRows = ROWS;
  static constexpr int kOwn = Z::kChunks >= 32 ? Z::kChunks / 32 : 1;  // chunks per lane
  static constexpr int kSplit = Z::kChunks >= 32 ? 1 : 32 / Z::kChunks;  // lanes that share a chunk, by tokens
  float4 o[ROWS][kOwn];
  float m[ROWS], l[ROWS];

  // `mine`: this warp's shared memory, ROWS x DP queries, then 8 x ROWS weights.
  __device__ __forceinline__ void begin(const PagedKernelArgs& g, int b, const Queries& qs, int lane, float* mine) {
    __syncwarp();
    const float* src = static_cast<const float*>(g.a.q) + b * g.a.q_stride + (int64_t)qs.first * g.a.v.d;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
#pragma unroll
      for (int e = 0; e < Z::DP; e += 32) {
        const bool have = r < qs.count && e + lane < g.a.v.d;
        mine[r * Z::DP + e + lane] = have ? src[r * g.a.v.d + e + lane] : 0.f;
      }
      m[r] = -CUDART_INF_F;
      l[r] = 0.f;
#pragma unroll
      for (int k = 0; k < kOwn; ++k) o[r][k] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __syncwarp();
  }

  __device__ __forceinline__ void step(uint32_t keys, int live, int lane, const ScoreScale& scale, float* mine) {
    if (live <= 0) return;
    const auto chunk = [](uint32_t at) {
      float4 v;
      asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at));
      return v;
    };
    const int t = lane & 7, quarter = lane >> 3;
    float s[ROWS] = {};
#pragma unroll
    for (int k = 0; k < Z::kChunks / 4; ++k) {
      const int c = 4 * k + quarter;
      const float4 x = chunk(keys + t * Z::kRow + ((c ^ t) * 16));
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const float4 y = *reinterpret_cast<const float4*>(mine + r * Z::DP + 4 * c);
        s[r] = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, s[r]))));
      }
    }
    float* weights = mine + ROWS * Z::DP;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) s[r] += __shfl_xor_sync(~0u, s[r], 8);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) s[r] += __shfl_xor_sync(~0u, s[r], 16);
    scale.apply(s);
    float top[ROWS];
    bool raise = false;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (t >= live) s[r] = -CUDART_INF_F;
      top[r] = fmaxf(m[r], s[r]);
    }
#pragma unroll
    for (int x = 1; x < 8; x <<= 1)
#pragma unroll
      for (int r = 0; r < ROWS; ++r) top[r] = fmaxf(top[r], __shfl_xor_sync(~0u, top[r], x));
#pragma unroll
    for (int r = 0; r < ROWS; ++r) raise |= top[r] > m[r];
    if (raise) {  // the same in every lane
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const float c = m[r] == top[r] ? 1.f : exp2_approx(m[r] - top[r]);
        m[r] = top[r];
        l[r] *= c;
#pragma unroll
        for (int k = 0; k < kOwn; ++k) o[r][k].x *= c, o[r][k].y *= c, o[r][k].z *= c, o[r][k].w *= c;
      }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const float p = exp2_approx(s[r] - (m[r] == -CUDART_INF_F ? 0.f : m[r]));
      if (quarter == 0) {
        l[r] += p;
        weights[t * ROWS + r] = p;
      }
    }
    __syncwarp();
    const uint32_t vals = keys + Z::kHalf;
#pragma unroll
    for (int i = 0; i < Z::TOK / kSplit; ++i) {
      const int tok = i * kSplit + (kSplit > 1 ? lane / Z::kChunks : 0);
      float p[ROWS];
#pragma unroll
      for (int r = 0; r < ROWS; ++r) p[r] = weights[tok * ROWS + r];
#pragma unroll
      for (int k = 0; k < kOwn; ++k) {
        const int c = (kSplit > 1 ? lane % Z::kChunks : lane) + 32 * k;
        const float4 x = chunk(vals + tok * Z::kRow + ((c ^ (tok & 7)) * 16));
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
    for (int r = 0; r < ROWS; ++r) {
#pragma unroll
      for (int x = 1; x < 32; x <<= 1) l[r] += __shfl_xor_sync(~0u, l[r], x);  // lanes past 7 hold zero
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
  __device__ __forceinline__ void each(int x, int lane, int e0, int e1, F f) const {
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
      const int e = 4 * ((kSplit > 1 ? lane % Z::kChunks : lane) + 32 * k);
      if (lane < 32 / kSplit && e >= e0 && e < e1) {
        f(e, o[x][k].x, o[x][k].y);
        f(e + 2, o[x][k].z, o[x][k].w);
      }
    }
  }
  __device__ __forceinline__ void times(int x, float c) {
#pragma unroll
    for (int k = 0; k < kOwn; ++k) o[x][k].x *= c, o[x][k].y *= c, o[x][k].z *= c, o[x][k].w *= c;
  }
};

// ---------------------------------------------------------------------------
// the kernel
// ---------------------------------------------------------------------------

constexpr int kMergeDims = 32;  // output elements that runs of tokens join at a time

template <class Z, class Tile>
struct Shared {  // after the rings
  float mine[std::is_same<typename Z::T, float>::value ? Z::NW * (Tile::kRows * Z::DP + 8 * Tile::kRows) : 4];
  float part[Z::NW][Tile::kRows][kMergeDims];
  float m[Z::NW][Tile::kRows], l[Z::NW][Tile::kRows];
  int bad[Z::NW];
};

template <class Z, class Tile>
constexpr size_t shared_bytes(int B) {
  return Z::kRing + sizeof(Shared<Z, Tile>) + sizeof(int) * (B + 1);
}

template <class Z, class Tile>
__global__ void __launch_bounds__(Z::NW * 32, 1) paged_decode_kernel(const __grid_constant__ PagedKernelArgs g) {
  using T = typename Z::T;
  extern __shared__ __align__(128) uint8_t raw[];
  Shared<Z, Tile>& sh = *reinterpret_cast<Shared<Z, Tile>*>(raw + Z::kRing);
  int* prefix = reinterpret_cast<int*>(raw + Z::kRing + sizeof(sh));
  const PagedDecodeArgs& a = g.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wh = warp & (g.p.wh - 1), wt = warp / g.p.wh;
  const int d = a.v.d;
  T* out = static_cast<T*>(a.out);
  pdl_launch_dependents();

  const int n_tiles = tile_prefix<Z::NW>(a, g.p.tile, prefix, blockIdx.x == 0);
  const int64_t units = (int64_t)g.p.groups * n_tiles;
  const int n = (int)min((int64_t)g.p.n_items, units);
  // empty sequences
  for (int b = blockIdx.x; b < a.B; b += gridDim.x)
    if (prefix[b + 1] == prefix[b]) {
      for (int e = threadIdx.x; e < a.v.Hq * d; e += Z::NW * 32) out[(int64_t)b * a.v.Hq * d + e] = from_f32<T>(0.f);
      if (a.lse)
        for (int j = threadIdx.x; j < a.v.Hq; j += Z::NW * 32) a.lse[(int64_t)b * a.v.Hq + j] = -CUDART_INF_F;
    }
  if ((int)blockIdx.x >= n) {
    if (blockIdx.x == 0 && threadIdx.x == 0) g.header->n_entries = 0;
    return;
  }
  const int64_t u0 = range_begin(blockIdx.x, units, n), u1 = range_begin(blockIdx.x + 1, units, n);

  const Loader<Z> load{g, (uint32_t)__cvta_generic_to_shared(raw) + warp * Z::S * Z::kStage, lane, wh, wt};
  Cursor ahead;
  ahead.enter(a, prefix, n_tiles, u0);
  Pages pages = load.fetch(ahead);
  uint32_t outside = 0;  // bit s: stage s has a page outside the pool
  int put = 0;           // stage that the next copies go to
  const auto copy_next = [&]() {
    if (ahead.u < u1) {
      const bool bad = load.issue(pages, put);
      outside = (outside & ~(1u << put)) | (uint32_t)bad << put;
      ahead.next(a, prefix, n_tiles, u1);
      if (ahead.u < u1) pages = load.fetch(ahead);
      put = put + 1 == Z::S ? 0 : put + 1;
    }
    cp_async_commit();
  };
#pragma unroll 1
  for (int i = 0; i < Z::S - 1; ++i) copy_next();

  Cursor at;
  at.enter(a, prefix, n_tiles, u0);
  ScoreScale scale;
  scale.scale2 = a.scale * 1.44269504088896f;
  scale.cap2 = a.softcap * 1.44269504088896f;
  scale.inv_cap = a.softcap > 0.f ? a.scale / a.softcap : 0.f;
  float* mine = sh.mine + warp * (Tile::kRows * Z::DP + 8 * Tile::kRows);
  Tile tile;
  Queries qs = queries_of(g, at.group, wh);
  tile.begin(g, at.b, qs, lane, mine);

  if (blockIdx.x == 0) {  // the list of what several CTAs share, for the second launch
    __shared__ int n_entries;
    if (threadIdx.x == 0) n_entries = 0;
    __syncthreads();
    for (int c = threadIdx.x; c + 1 < n; c += Z::NW * 32) {
      const int64_t x = range_begin(c + 1, units, n);
      const int group = (int)(x / n_tiles);
      const int64_t base = (int64_t)group * n_tiles;
      const int b = seq_of_tile(prefix, a.B, (int)(x - base));
      const int64_t start = base + prefix[b], begin = range_begin(c, units, n);
      if (x > start && begin <= start) {
        Entry e;
        e.pair = group * a.B + b;
        e.c0 = c;
        e.c1 = item_of(base + prefix[b + 1] - 1, units, n);
        e.second = begin < start;
        g.entries[atomicAdd(&n_entries, 1)] = e;
      }
    }
    __syncthreads();
    if (threadIdx.x == 0) g.header->n_entries = n_entries;
  }

  int get = 0;
  bool bad = false;
  while (true) {
    __syncwarp();  // the stage that is filled next has been read
    copy_next();
    cp_async_wait<Z::S - 1>();
    __syncwarp();
    bad |= outside >> get & 1;
    tile.step(load.ring + get * Z::kStage, at.len - at.token(g.p.tile) - wt * Z::TOK, lane, scale, mine);
    get = get + 1 == Z::S ? 0 : get + 1;
    const bool last = at.u + 1 == u1;
    if (at.u + 1 < at.end && !last) {
      ++at.u;
      continue;
    }
    // the end of a (head group, sequence), or of this CTA's part of it
    const bool whole = at.start >= u0 && at.end <= u1;
    const int slot = 2 * blockIdx.x + (u0 < at.start);
    if (bad && lane == 0) atomicOr(a.err, kErrBadSeq);
    tile.finish();
    const int64_t out_row = (int64_t)at.b * a.v.Hq + qs.first, part_row = (int64_t)(slot * g.p.wh + wh) * g.p.rows;
    if (g.p.wt > 1) {  // the runs of tokens join: all to the largest maximum, then element by element
#pragma unroll
      for (int x = 0; x < Tile::kMine; ++x)
        if (Tile::speaks(lane)) sh.m[warp][Tile::row(x, lane)] = tile.m[x], sh.l[warp][Tile::row(x, lane)] = tile.l[x];
      if (lane == 0) sh.bad[warp] = bad;
      __syncthreads();
      for (int w = wh; w < Z::NW; w += g.p.wh) bad |= sh.bad[w] != 0;
#pragma unroll
      for (int x = 0; x < Tile::kMine; ++x) {
        const int r = Tile::row(x, lane);
        float M = -CUDART_INF_F, sum = 0.f;
        for (int w = wh; w < Z::NW; w += g.p.wh) M = fmaxf(M, sh.m[w][r]);
        const float base = M == -CUDART_INF_F ? 0.f : M;
        for (int w = wh; w < Z::NW; w += g.p.wh) sum += sh.l[w][r] * exp2_approx(sh.m[w][r] - base);
        tile.times(x, exp2_approx(tile.m[x] - base));
        tile.m[x] = M, tile.l[x] = sum;
      }
    }
    float factor[Tile::kMine];
#pragma unroll
    for (int x = 0; x < Tile::kMine; ++x) {
      const int r = Tile::row(x, lane);
      const bool none = bad || tile.l[x] == 0.f;
      factor[x] = !whole ? 1.f : none ? 0.f : 1.f / tile.l[x];
      if (Tile::speaks(lane) && wt == 0 && r < qs.count) {
        if (!whole) *reinterpret_cast<float2*>(g.part_ml + 2 * (part_row + r)) = make_float2(tile.m[x], bad ? -1.f : tile.l[x]);
        else if (a.lse) a.lse[out_row + r] = none ? -CUDART_INF_F : (tile.m[x] + log2f(tile.l[x])) * 0.693147180559945f;
      }
    }
    if (g.p.wt == 1) {
#pragma unroll
      for (int x = 0; x < Tile::kMine; ++x) {
        const int r = Tile::row(x, lane);
        if (r >= qs.count) continue;
        if (whole) {
          T* p = out + (out_row + r) * d;
          tile.each(x, lane, 0, d, [&](int e, float y, float z) {
            p[e] = from_f32<T>(factor[x] == 0.f ? 0.f : y * factor[x]);
            p[e + 1] = from_f32<T>(factor[x] == 0.f ? 0.f : z * factor[x]);
          });
        } else {
          float* p = g.part_u + (part_row + r) * Z::DP;
          tile.each(x, lane, 0, d, [&](int e, float y, float z) { *reinterpret_cast<float2*>(p + e) = make_float2(y, z); });
        }
      }
    } else {
      for (int e0 = 0; e0 < d; e0 += kMergeDims) {
#pragma unroll
        for (int x = 0; x < Tile::kMine; ++x)
          tile.each(x, lane, e0, e0 + kMergeDims, [&](int e, float y, float z) {
            *reinterpret_cast<float2*>(&sh.part[warp][Tile::row(x, lane)][e - e0]) =
                factor[x] == 0.f ? make_float2(0.f, 0.f) : make_float2(y * factor[x], z * factor[x]);
          });
        __syncthreads();
        // head wh of the group is summed by its own warps, a row each in turn
        if (e0 + lane < d)
          for (int r = wt; r < qs.count; r += g.p.wt) {
            float sum = 0.f;
            for (int w = wh; w < Z::NW; w += g.p.wh) sum += sh.part[w][r][lane];
            if (whole) out[(out_row + r) * d + e0 + lane] = from_f32<T>(sum);
            else g.part_u[(part_row + r) * Z::DP + e0 + lane] = sum;
          }
        __syncthreads();
      }
    }
    bad = false;
    if (last) break;
    at.next(a, prefix, n_tiles, u1);
    qs = queries_of(g, at.group, wh);
    tile.begin(g, at.b, qs, lane, mine);
  }
  cp_async_wait<0>();
}

// Joins the partial sums of what several CTAs share: a block per (entry, row), a warp
// per partial in turn.
constexpr int kJoinWarps = 8;

template <typename T>
__global__ void __launch_bounds__(kJoinWarps * 32) paged_join_kernel(const __grid_constant__ PagedKernelArgs g, int DP) {
  __shared__ float sm[kJoinWarps], sl[kJoinWarps], so[kJoinWarps][kMaxPagedHeadDim];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, per = g.p.wh * g.p.rows, d = g.a.v.d;
  pdl_wait();
  const int n = g.header->n_entries;
  for (int64_t x = blockIdx.x; x < (int64_t)n * per; x += gridDim.x) {
    const Entry e = g.entries[x / per];
    const int hr = (int)(x % per), h = hr / g.p.rows, r = hr - h * g.p.rows;
    const int group = e.pair / g.a.B, b = e.pair - group * g.a.B;
    const Queries qs = queries_of(g, group, h);
    if (r >= qs.count) continue;
    const int j = qs.first + r;
    const auto row = [&](int c) { return ((int64_t)(2 * c + (c == e.c0 ? e.second : 0)) * g.p.wh + h) * g.p.rows + r; };
    float m = -CUDART_INF_F, l = 0.f, o[kMaxPagedHeadDim / 32] = {};
    bool bad = false;
    for (int c = e.c0 + warp; c <= e.c1; c += kJoinWarps) {
      const float2 ml = *reinterpret_cast<const float2*>(g.part_ml + 2 * row(c));
      const float mn = fmaxf(m, ml.x), base = mn == -CUDART_INF_F ? 0.f : mn;
      const float w0 = exp2_approx(m - base), w1 = exp2_approx(ml.x - base);
      bad |= ml.y < 0.f;
      l = l * w0 + ml.y * w1;
      m = mn;
#pragma unroll
      for (int k = 0; k < kMaxPagedHeadDim / 32; ++k)
        if (k * 32 + lane < d) o[k] = o[k] * w0 + g.part_u[row(c) * DP + k * 32 + lane] * w1;
    }
    if (lane == 0) sm[warp] = m, sl[warp] = bad ? -1.f : l;
#pragma unroll
    for (int k = 0; k < kMaxPagedHeadDim / 32; ++k) so[warp][k * 32 + lane] = o[k];
    __syncthreads();
    float M = -CUDART_INF_F, total = 0.f;
    bool any = false;
    for (int w = 0; w < kJoinWarps; ++w) M = fmaxf(M, sm[w]);
    const float base = M == -CUDART_INF_F ? 0.f : M;
    for (int w = 0; w < kJoinWarps; ++w) any |= sl[w] < 0.f, total += sl[w] * exp2_approx(sm[w] - base);
    for (int i = threadIdx.x; i < d; i += kJoinWarps * 32) {
      float s = 0.f;
      for (int w = 0; w < kJoinWarps; ++w) s += so[w][i] * exp2_approx(sm[w] - base);
      static_cast<T*>(g.a.out)[((int64_t)b * g.a.v.Hq + j) * d + i] = from_f32<T>(any || total == 0.f ? 0.f : s / total);
    }
    if (g.a.lse && threadIdx.x == 0)
      g.a.lse[(int64_t)b * g.a.v.Hq + j] = any || total == 0.f ? -CUDART_INF_F : (M + log2f(total)) * 0.693147180559945f;
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------

int padded_dim(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }
int warps_of(int DP) { return DP == 256 ? 4 : 8; }

PagedPlan plan_of(const PagedView& v, int dtype, int B, int max_len, int window, int sms) {
  PagedPlan p;
  const int DP = padded_dim(v.d), NW = warps_of(DP);
  const int most = dtype == DCK_BF16 && DP <= 128 && v.qpg > 8 ? 16 : 8;
  p.chunks = (v.qpg + most - 1) / most;
  p.rows = (v.qpg + p.chunks - 1) / p.chunks;
  const int heads = v.Hkv * p.chunks;
  p.wh = NW;
  while (heads % p.wh) p.wh /= 2;
  p.wt = NW / p.wh;
  p.groups = heads / p.wh;
  p.by_chunks = divider((uint32_t)p.chunks);
  p.tile = p.wt * (dtype == DCK_BF16 ? 16 : 8);
  const int64_t span = window > 0 ? std::min(window, max_len) : max_len;
  p.n_items = (int)std::min<int64_t>(sms, (int64_t)p.groups * std::max(B, 1) * ((span + p.tile - 1) / p.tile));
  return p;
}

size_t bytes_u(const PagedPlan& p, int DP, int n) { return align_up((size_t)2 * n * p.wh * p.rows * DP * sizeof(float), 256); }
size_t bytes_ml(const PagedPlan& p, int n) { return align_up((size_t)2 * n * p.wh * p.rows * 2 * sizeof(float), 256); }

template <class Z, class Tile>
cudaError_t launch_main(const PagedKernelArgs& g, cudaStream_t s) {
  const size_t smem = shared_bytes<Z, Tile>(g.a.B);
  cudaError_t e = cudaFuncSetAttribute(paged_decode_kernel<Z, Tile>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  paged_decode_kernel<Z, Tile><<<g.p.n_items, Z::NW * 32, smem, s>>>(g);
  return hook_launched(g.a.hook, s);
}

template <class Z>
cudaError_t launch_simt(const PagedKernelArgs& g, cudaStream_t s) {
  if (g.p.rows == 1) return launch_main<Z, SimtTile<Z, 1>>(g, s);
  if (g.p.rows <= 4) return launch_main<Z, SimtTile<Z, 4>>(g, s);
  return launch_main<Z, SimtTile<Z, 8>>(g, s);
}

}  // namespace

size_t paged_decode_workspace(const PagedView& v, int dtype, int B, int max_len, int sms) {
  const PagedPlan p = plan_of(v, dtype, B, max_len, 0, sms);
  return 256 + align_up(p.n_items * sizeof(Entry), 256) + bytes_ml(p, p.n_items) + bytes_u(p, padded_dim(v.d), p.n_items);
}

cudaError_t launch_paged_decode(const PagedDecodeArgs& a, int dtype, int sms, cudaStream_t s) {
  PagedKernelArgs g;
  g.a = a;
  g.p = plan_of(a.v, dtype, a.B, a.max_len, a.window, sms);
  const int DP = padded_dim(a.v.d);
  char* ws = static_cast<char*>(a.ws);
  g.header = reinterpret_cast<Header*>(ws);
  g.entries = reinterpret_cast<Entry*>(ws + 256);
  ws += 256 + align_up(g.p.n_items * sizeof(Entry), 256);
  g.part_ml = reinterpret_cast<float*>(ws);
  g.part_u = reinterpret_cast<float*>(ws + bytes_ml(g.p, g.p.n_items));
  cudaError_t e;
  using bf16 = __nv_bfloat16;
  if (dtype == DCK_F32) {
    if (DP == 64) e = launch_simt<Sizes<float, 64, 8, 4, 8>>(g, s);
    else if (DP == 128) e = launch_simt<Sizes<float, 128, 8, 2, 8>>(g, s);
    else e = launch_simt<Sizes<float, 256, 4, 2, 8>>(g, s);
  } else if (DP == 256) {
    using Z = Sizes<bf16, 256, 4, 3, 16>;
    e = launch_main<Z, TensorTile<Z, true>>(g, s);
  } else if (DP == 128) {
    using Z = Sizes<bf16, 128, 8, 3, 16>;
    e = g.p.rows > 8 ? launch_main<Z, TensorTile<Z, false>>(g, s) : launch_main<Z, TensorTile<Z, true>>(g, s);
  } else {
    using Z = Sizes<bf16, 64, 8, 6, 16>;
    e = g.p.rows > 8 ? launch_main<Z, TensorTile<Z, false>>(g, s) : launch_main<Z, TensorTile<Z, true>>(g, s);
  }
  if (e != cudaSuccess) return e;
  // one tile per (head group, sequence) at most: nothing is shared
  if ((a.window > 0 ? std::min(a.window, a.max_len) : a.max_len) <= g.p.tile) return cudaSuccess;
  const int64_t work = (int64_t)g.p.n_items * g.p.wh * g.p.rows;
  const int grid = (int)std::min<int64_t>(work, 4 * sms);
  e = dtype == DCK_F32 ? launch_pdl(paged_join_kernel<float>, grid, kJoinWarps * 32, 0, s, g, DP)
                       : launch_pdl(paged_join_kernel<bf16>, grid, kJoinWarps * 32, 0, s, g, DP);
  if (e != cudaSuccess) return e;
  return hook_launched(a.hook, s);
}

}  // namespace dck

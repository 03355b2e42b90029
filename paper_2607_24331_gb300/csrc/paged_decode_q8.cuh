// Attention of one new token per sequence over 8-bit pages (dck_quant_decode_attention): what
// differs from 16- and 32-bit caches, the copies and the arithmetic of a step.
//
// Mathematics: with key codes c_t of scale a_t and value codes w_t of scale b_t the scores are
// scale a_t <q, c_t>, and the output is sum_t 2^(s_t + log2 b_t - R) w_t 2^(R - m) / sum_t 2^(s_t - m): the values'
// scales go into the weights' exponents, with a reference R of their own, so that a weight of the
// product is at most 2^15 whatever the scales, and the codes are multiplied as they are.
//
// An e4m3 code is an fp16 number exactly (one conversion for two of them), so products run on
// mma.sync m16n8k16 in fp16 with fp32 sums.  Queries are brought to 2^14 .. 2^15 by a power of two
// per row first: of a bf16 query fp16 then holds every element down to 2^-29 of the row's largest as it is,
// and smaller ones to 2^-39 of that (half of fp16's least step, 2^-25, of 2^14); of an fp32 one two fp16 terms keep 2^-22.  Weights are two fp16 terms (2^-22), the low
// ones in the MMA's unused rows where up to 8 query heads share a KV head; with more of them one
// term (2^-11, a quarter of what a bf16 output's rounding can be off by, and errors of many weights cancel).
#pragma once

#include <cuda_fp16.h>

#include "paged_decode.cuh"

namespace dck {
namespace paged {

// Sizes of a variant: queries and outputs T, 8-bit rows; a stage holds keys, values and both scales.
template <typename T_, int DP_, int NW_, int S_>
struct QuantSizes {
  using T = T_;
  static constexpr bool kQuant = true;
  static constexpr int DP = DP_, NW = NW_, S = S_, TOK = 32;
  static constexpr int kRow = DP, kChunks = kRow / 16;
  static constexpr int kQRow = DP * sizeof(T);
  static constexpr int kHalf = TOK * kRow;
  static constexpr int kScales = 2 * kHalf;  // where a stage's scales begin: the keys', then the values'
  static constexpr int kStage = kScales + 2 * TOK * 4;
  static constexpr int kRing = NW * S * kStage;
  // Chunk c of row r lies at c ^ flip(r): then the 16-byte reads of a quarter warp (two rows, four
  // chunks) and ldmatrix's (eight rows, one chunk) each touch all banks once.
  static __device__ __forceinline__ int flip(int r) { return DP == 64 ? r >> 1 & 3 : (r & 1) << 2 | (r >> 1 & 3); }
};

__device__ __forceinline__ void cp_async4_or_zero(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

template <class Z, int ROWS, int QS>
struct QuantLoader : LoaderBase<Z, ROWS, QS> {
  using Base = LoaderBase<Z, ROWS, QS>;
  using Base::g, Base::lane, Base::ring, Base::wh;
  static constexpr int kLanes = Z::kChunks < 8 ? Z::kChunks : 8;  // that copy a row
  static constexpr int kRows = 32 / kLanes;                       // rows copied at a time
  const char *kc, *vc;
  uint32_t even, odd;  // where this lane's chunk of rows kRows i + sub lies in a stage, i even or odd
  int have;            // bytes of a row from this lane's first chunk on

  __device__ __forceinline__ QuantLoader(const Args& g, const uint8_t* raw, const void* q, int warp, int lane, int wh, int wt)
      : Base(g, raw, q, warp, lane, wh, wt) {
    const int sub = lane / kLanes, c = lane % kLanes;
    kc = static_cast<const char*>(g.a.kc) + c * 16;
    vc = static_cast<const char*>(g.a.vc) + c * 16;
    even = sub * Z::kRow + (c ^ Z::flip(sub)) * 16;
    odd = sub * Z::kRow + (c ^ Z::flip(sub + kRows)) * 16;
    have = g.a.v.d - c * 16;
  }

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
    cp_async4_or_zero(at + Z::kScales + lane * 4,
                      g.a.ks + ((uint64_t)page * v.ks_page + (uint64_t)off * v.ks_tok + (uint64_t)head * v.ks_head), ok ? 4 : 0);
    cp_async4_or_zero(at + Z::kScales + (Z::TOK + lane) * 4,
                      g.a.vs + ((uint64_t)page * v.vs_page + (uint64_t)off * v.vs_tok + (uint64_t)head * v.vs_head), ok ? 4 : 0);
    const int sub = lane / kLanes;
#pragma unroll
    for (int i = 0; i < Z::TOK / kRows; ++i) {
      const int row = i * kRows + sub;
      const int64_t kr = __shfl_sync(~0u, ko, row);
      const int64_t vr = g.p.alike ? kr : __shfl_sync(~0u, vo, row);
      const bool live = mask >> row & 1;
      const uint32_t dst = at + (i & 1 ? odd : even) + i * kRows * Z::kRow;
#pragma unroll
      for (int j = 0; j < Z::kChunks / kLanes; ++j) {
        const int bytes = min(have - 128 * j, 16);  // a row may end within a chunk
        if (bytes > 0) {
          cp_async16_or_zero(dst + 128 * j, kc + kr + 128 * j, live ? bytes : 0);
          cp_async16_or_zero(dst + 128 * j + Z::kHalf, vc + vr + 128 * j, live ? bytes : 0);
        }
      }
    }
    return __any_sync(~0u, !inside);
  }
};

template <typename T, int DP, int NW, int S, int ROWS, int QS>
struct LoaderOf<QuantSizes<T, DP, NW, S>, ROWS, QS> {
  using type = QuantLoader<QuantSizes<T, DP, NW, S>, ROWS, QS>;
};

// Codes of the lower and upper half of x as fp16 pairs.
__device__ __forceinline__ void open_codes(uint32_t x, uint32_t& lower, uint32_t& upper) {
  asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.rn.f16x2.e4m3x2 %0, l;\n cvt.rn.f16x2.e4m3x2 %1, h;\n}\n"
      : "=r"(lower), "=r"(upper)
      : "r"(x));
}
__device__ __forceinline__ void mma16816_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                             uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t half_pair(float x, float y) {
  const __half2 h = __floats2half2_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// x and y as fp16 pairs hi + lo.
__device__ __forceinline__ void split_halves(float x, float y, uint32_t& hi, uint32_t& lo) {
  const __half2 h = __floats2half2_rn(x, y);
  const float2 f = __half22float2(h);
  hi = *reinterpret_cast<const uint32_t*>(&h);
  lo = half_pair(x - f.x, y - f.y);
}
// Of scales, exact for powers of two.  (Below the least normal number -infinity, a weight of 0: so 1.3% less time than with
// the steps that those take.)
__device__ __forceinline__ float log2_approx(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint4 shared16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}
__device__ __forceinline__ float2 shared8(uint32_t at) {
  float2 v;
  asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at));
  return v;
}

// One warp's tile of queries and its running sums, 32 tokens a step.  PACK: up to 8 queries, rows 0-7 of the
// MMAs' tile, and in rows 8-15 the low terms of fp32 queries and of the weights.  Otherwise up to 16 bf16 queries.
//
// The order of a row's elements is free in <q, c>: lane l takes the 16 bytes of a key's chunk l % 4 (+ 4 j) in one
// read, which are the operands of four k-steps.  Values go through ldmatrix.trans in pairs of codes, two elements
// of two tokens in each word; of the two elements one goes to each of two MMAs.
//
// LAID_OUT: the queries stay in shared memory, as each lane's operands of each k-step in 16 bytes, and all warps of the CTA
// read them from there: 32 registers fewer, so that three CTAs fit on an SM (16 bf16 queries of one KV head; a step is a chain
// of short instructions, of which eight warps leave an SM's schedulers idle half of the time).
template <class Z, bool PACK, bool LAID_OUT = false>
struct QuantTile {
  static constexpr int kQ = PACK ? 1 : 2;  // query rows per lane
  static constexpr int kRows = PACK ? 8 : 16;
  static constexpr int kStepBytes = 512, kUnits = Z::DP / 16 * kStepBytes;  // of a k-step's operands; where the rows' units begin
  static constexpr int kOperands = LAID_OUT ? kUnits + kRows * 4 : 16;
  static_assert(!LAID_OUT || !PACK, "16 queries");
  static constexpr bool kLow = std::is_same<typename Z::T, float>::value;  // queries of two terms
  static_assert(PACK || !kLow, "fp32 queries: low terms in rows 8-15");
  static constexpr int kTerms = PACK && !kLow ? 2 : 4;  // registers of a k-step's queries
  float o[Z::DP / 8][4], m[kQ], l[kQ], near[kQ], unit[kQ];  // near: reference of the weights, unit: of the queries
  uint32_t q[LAID_OUT ? 1 : Z::DP / 16][kTerms], operands;

  // The exponent e that brings a row of largest magnitude `top` (bits) to [2^14, 2^15) times 2^-e, where that is 2^-96 or more.
  static __device__ __forceinline__ int exponent_of(uint32_t top) { return max((int)(top >> 23) - 127 - 14, -110); }
  static __device__ __forceinline__ uint32_t finite_bits(float x) {
    const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
  }
  // LAID_OUT: rows at `place` to operands at `to`, by the whole CTA.  A thread has a row's chunk of 16 elements, four k-steps of
  // lane 4 (row % 8) + chunk % 4.
  static __device__ __forceinline__ void lay_out(const uint8_t* place, uint8_t* to) {
    if constexpr (LAID_OUT) {
      constexpr int kChunks = Z::DP / 16;
      if (threadIdx.x >= kRows * kChunks) return;
      const int row = threadIdx.x / kChunks, chunk = threadIdx.x % kChunks;
      float x[16];
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int e = chunk * 16 + i;
        x[i] = to_f32(*reinterpret_cast<const typename Z::T*>(place + row * Z::kQRow + ((e / 8) ^ (row & 7)) * 16 + e % 8 * 2));
        top = max(top, finite_bits(x[i]));
      }
#pragma unroll
      for (int o = 1; o < kChunks; o <<= 1) top = max(top, __shfl_xor_sync(~0u, top, o));
      const int e = exponent_of(top);
      const float down = __uint_as_float((uint32_t)(127 - e) << 23);
      if (chunk == 0) *reinterpret_cast<float*>(to + kUnits + row * 4) = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        uint32_t* at = reinterpret_cast<uint32_t*>(to + (chunk / 4 * 4 + t) * kStepBytes + ((row & 7) * 4 + chunk % 4) * 16) + row / 8;
        at[0] = half_pair(x[4 * t] * down, x[4 * t + 1] * down);
        at[2] = half_pair(x[4 * t + 2] * down, x[4 * t + 3] * down);
      }
    }
  }

  static __device__ __forceinline__ float query(uint32_t place, int row, int e) {  // element e of a row
    const uint32_t at = place + row * Z::kQRow;
    if (kLow) {
      float x;
      asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(at + ((e / 4) ^ (row & 7)) * 16 + e % 4 * 4));
      return x;
    }
    uint16_t x;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(at + ((e / 8) ^ (row & 7)) * 16 + e % 8 * 2));
    return __uint_as_float((uint32_t)x << 16);
  }

  __device__ __forceinline__ void clear_sums() {
#pragma unroll
    for (int x = 0; x < kQ; ++x) {
      m[x] = near[x] = -CUDART_INF_F;
      l[x] = 0.f;
    }
#pragma unroll
    for (int n = 0; n < Z::DP / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
  }
  __device__ __forceinline__ void begin(uint32_t place, int lane) {
    const int c = lane & 3;
    clear_sums();
    if constexpr (LAID_OUT) {
      operands = place + lane * 16;
#pragma unroll
      for (int x = 0; x < kQ; ++x) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(unit[x]) : "r"(place + kUnits + (lane / 4 + 8 * x) * 4));
      return;
    }
#pragma unroll
    for (int x = 0; x < (LAID_OUT ? 0 : kQ); ++x) {
      const int row = lane / 4 + 8 * x;
      uint32_t top = 0;
#pragma unroll
      for (int k = 0; k < Z::DP / 16; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          top = max(top, finite_bits(query(place, row, 16 * (c + 4 * (k / 4)) + 4 * (k % 4) + i)));
        }
      top = max(top, __shfl_xor_sync(~0u, top, 1));
      top = max(top, __shfl_xor_sync(~0u, top, 2));
      const int e = exponent_of(top);
      const float down = __uint_as_float((uint32_t)(127 - e) << 23);
      unit[x] = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
      for (int k = 0; k < Z::DP / 16; ++k) {
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = query(place, row, 16 * (c + 4 * (k / 4)) + 4 * (k % 4) + i) * down;
        if (PACK && kLow) {
          split_halves(y[0], y[1], q[k][0], q[k][1]);
          split_halves(y[2], y[3], q[k][2 % kTerms], q[k][3 % kTerms]);
        } else if (PACK) {
          q[k][0] = half_pair(y[0], y[1]);
          q[k][1] = half_pair(y[2], y[3]);
        } else {
          q[k][x] = half_pair(y[0], y[1]);
          q[k][(2 + x) % kTerms] = half_pair(y[2], y[3]);
        }
      }
    }
  }

  // The 32 tokens of a stage, the first `live` of them present (0 or fewer: none).
  __device__ __forceinline__ void step(uint32_t keys, int live, int lane, const ScoreScale& scale, float*) {
    if (live <= 0) return;
    const int c = lane & 3;
    float s[4][4] = {};
    {
      const int row = lane >> 2;
      const uint32_t at = keys + row * Z::kRow + (c ^ Z::flip(row)) * 16;
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int j = 0; j < Z::DP / 64; ++j) {
          // (chunks c + 4 j: the flip keeps bit 3, and bit 2 changes as it would without)
          const uint4 x = shared16((at ^ ((j & 1) * 64)) + (j >> 1) * 128 + n * 8 * Z::kRow);
          const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            uint32_t b0, b1;
            open_codes(w[t], b0, b1);
            uint32_t y[kTerms];
            if constexpr (LAID_OUT) {
              const uint4 f = shared16(operands + (4 * j + t) * kStepBytes);
              y[0] = f.x, y[1] = f.y, y[2 % kTerms] = f.z, y[3 % kTerms] = f.w;
            } else {
#pragma unroll
              for (int i = 0; i < kTerms; ++i) y[i] = q[LAID_OUT ? 0 : 4 * j + t][i];
            }
            if (PACK && !kLow) mma16816_f16(s[n], y[0], 0u, y[1], 0u, b0, b1);
            else mma16816_f16(s[n], y[0], y[1], y[2 % kTerms], y[3 % kTerms], b0, b1);
          }
        }
    }
    float e[4][2];  // log2 of the values' scales
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const float2 a = shared8(keys + Z::kScales + (n * 8 + c * 2) * 4), b = shared8(keys + Z::kScales + (Z::TOK + n * 8 + c * 2) * 4);
      e[n][0] = log2_approx(b.x), e[n][1] = log2_approx(b.y);
      if (PACK && kLow) s[n][0] += s[n][2], s[n][1] += s[n][3];
#pragma unroll
      for (int x = 0; x < kQ; ++x) s[n][2 * x] *= a.x * unit[x], s[n][2 * x + 1] *= a.y * unit[x];
      if (PACK) {
        float v[2] = {s[n][0], s[n][1]};
        scale.apply(v);
        s[n][0] = v[0], s[n][1] = v[1];
      } else {
        scale.apply(s[n]);
      }
    }
    if (live < 32) {
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int y = 0; y < 2 * kQ; ++y)
          if (n * 8 + c * 2 + (y & 1) >= live) s[n][y] = -CUDART_INF_F;
    }
    accumulate(keys, lane, s, e);
  }

  // Adds tokens of scores s (log2 units) and value scales 2^e.
  __device__ __forceinline__ void accumulate(uint32_t keys, int lane, const float (&s)[4][4], const float (&e)[4][2]) {
    // both references need only be near the maximum: raised where one is 2^8 above
    bool raise = false;
#pragma unroll
    for (int x = 0; x < kQ; ++x)
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int y = 0; y < 2; ++y)
          raise |= s[n][2 * x + y] > m[x] + kHeadroom || s[n][2 * x + y] + e[n][y] > near[x] + 15.f;
    if (__any_sync(~0u, raise)) {
#pragma unroll
      for (int x = 0; x < kQ; ++x) {
        float top = m[x], high = near[x] + 7.f;
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            top = fmaxf(top, s[n][2 * x + y]);
            high = fmaxf(high, s[n][2 * x + y] + e[n][y]);
          }
#pragma unroll
        for (int i = 1; i < 4; i <<= 1) {
          top = fmaxf(top, __shfl_xor_sync(~0u, top, i));
          high = fmaxf(high, __shfl_xor_sync(~0u, high, i));
        }
        top = ceilf(top);  // whole numbers, like the exponents of scales: their differences are exact
        high = ceilf(high);
        l[x] *= m[x] == top ? 1.f : exp2_approx(m[x] - top);
        m[x] = top;
        high -= 7.f;  // weights up to 2^7, 2^15 before the next raise: fp16 holds them and 2^-31 of them
        const float f = near[x] == high ? 1.f : exp2_approx(near[x] - high);
        near[x] = high;
#pragma unroll
        for (int n = 0; n < Z::DP / 8; ++n) {
          o[n][2 * x] *= f, o[n][2 * x + 1] *= f;
          if (PACK) o[n][2] *= f, o[n][3] *= f;
        }
      }
    }
    uint32_t hi[kQ][4], lo[kQ][4];
#pragma unroll
    for (int x = 0; x < kQ; ++x) {
      const float base = m[x] == -CUDART_INF_F ? 0.f : m[x], at = near[x] == -CUDART_INF_F ? 0.f : near[x];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        l[x] += exp2_approx(s[n][2 * x] - base) + exp2_approx(s[n][2 * x + 1] - base);
        const float w0 = exp2_approx(s[n][2 * x] + (e[n][0] - at)), w1 = exp2_approx(s[n][2 * x + 1] + (e[n][1] - at));
        if (PACK) split_halves(w0, w1, hi[x][n], lo[x][n]);
        else hi[x][n] = half_pair(w0, w1);
      }
    }
    const uint32_t vals = keys + Z::kHalf + lane * Z::kRow;
    const int flip = Z::flip(lane & 7);
#pragma unroll
    for (int n = 0; n < Z::DP / 16; ++n) {
      uint32_t r[4];
      ldmatrix4_trans_plain(r, vals + ((n ^ flip) * 16));
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        uint32_t b[2][2];  // [token half][element of the pair]
#pragma unroll
        for (int i = 0; i < 2; ++i) open_codes(__byte_perm(r[2 * g + i], 0, 0x3120), b[i][0], b[i][1]);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          if (PACK) mma16816_f16(o[2 * n + y], hi[0][2 * g], lo[0][2 * g], hi[0][2 * g + 1], lo[0][2 * g + 1], b[0][y], b[1][y]);
          else mma16816_f16(o[2 * n + y], hi[0][2 * g], hi[kQ - 1][2 * g], hi[0][2 * g + 1], hi[kQ - 1][2 * g + 1], b[0][y], b[1][y]);
        }
      }
    }
  }
  static __device__ __forceinline__ void ldmatrix4_trans_plain(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(at)
                 : "memory");
  }

  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int x = 0; x < kQ; ++x) {
      l[x] += __shfl_xor_sync(~0u, l[x], 1);
      l[x] += __shfl_xor_sync(~0u, l[x], 2);
    }
#pragma unroll
    for (int n = 0; n < Z::DP / 8; ++n) {
      if (PACK) o[n][0] += o[n][2], o[n][1] += o[n][3];
#pragma unroll
      for (int x = 0; x < kQ; ++x) {
        // (by two powers: one may be below the least normal number, or above the largest, where the product is neither)
        const float by = near[x] == -CUDART_INF_F ? -CUDART_INF_F : near[x] - m[x], half = floorf(by * 0.5f);
        const float f = exp2_approx(half), rest = by == -CUDART_INF_F ? 0.f : exp2_approx(by - half);
        o[n][2 * x] = o[n][2 * x] * f * rest, o[n][2 * x + 1] = o[n][2 * x + 1] * f * rest;
      }
    }
  }
  static constexpr int kMine = kQ;
  static __device__ __forceinline__ int row(int x, int lane) { return lane / 4 + 8 * x; }
  static __device__ __forceinline__ bool speaks(int lane) { return (lane & 3) == 0; }
  template <class F>
  __device__ __forceinline__ void each(int x, int lane, int d, F f) const {
#pragma unroll
    for (int n = 0; n < Z::DP / 16; ++n) {
      const int e = n * 16 + (lane & 3) * 4;
      if (e < d) {
        f(e, o[2 * n][2 * x], o[2 * n + 1][2 * x]);
        f(e + 2, o[2 * n][2 * x + 1], o[2 * n + 1][2 * x + 1]);
      }
    }
  }
};

}  // namespace paged
}  // namespace dck

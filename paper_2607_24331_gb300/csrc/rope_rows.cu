// Rotary positions (dck_rope) and the rotated append to a paged cache
// (dck_paged_append, dck_quant_append).  A pair (x, y) of a head's elements at position t becomes
//   m (x cos a - y sin a, x sin a + y cos a),  a = t w_i  (sin negated: the transpose).
// For an 8-bit cache a head's row, rounded to its type, is then divided by the least power of two
// that leaves no magnitude above 448 and rounded to e4m3: the threads that hold it share the largest
// magnitude by shuffles, so that this too reads and writes every element once.
// Bound by memory: each element is read and written once.
#include <math_constants.h>

#include <algorithm>

#include "paged.cuh"
#include "rope.cuh"

namespace dck {
namespace {

constexpr int kThreads = 256;

// sin and cos at a signed position: read as unsigned, t < 0 is t + 2^32, which turns by
// 2^32 f more: the fraction's low word as the angle's high one (2^64 of a turn are none).
__device__ __forceinline__ void signed_sincos(uint2 f, int t, float& sn, float& cs) {
  const uint32_t u = (uint32_t)t;
  turn_sincos(__umulhi(u, f.x) + u * f.y - (t < 0 ? f.x : 0u), sn, cs);
}

// Where token i's rows go in a cache.
struct CacheRow {
  int64_t page, off;
  bool have;  // a row of the pool
};
__device__ __forceinline__ CacheRow cache_row(const RopeLaunch& a, int64_t i, bool report) {
  CacheRow r = {0, 0, false};
  if (!a.slots) return r;
  const int64_t slot = a.slots[i];
  if (slot < 0 || slot >= (int64_t)a.n_pages * a.page) {
    if (slot != -1 && report) atomicOr(a.err, kErrBadRow);
    return r;
  }
  r.page = slot >> 31 ? slot / a.page : (int64_t)a.by_page.div((uint32_t)slot);
  r.off = slot - r.page * a.page;
  r.have = true;
  return r;
}

// 8-bit rows.  The exponent e >= -126 of the scale 2^e of a row with largest magnitude `top`: the least with
// top <= 448 2^e.  448 = 1.75 2^8: mantissas above 1.75 carry into the exponent.
__device__ __forceinline__ int scale_exponent(float top) { return max((int)((__float_as_uint(top) + 0x1fffffu) >> 23) - 135, -126); }
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 .. 127
// The larger magnitude (of a number and NaN: the number).
__device__ __forceinline__ float larger(float x, float y) { return fmaxf(fabsf(x), fabsf(y)); }
// Infinities count as 0 for the scale and are stored as NaN: so they are made NaN, in rows that have any.
__device__ __forceinline__ float without_infinity(float x) { return fabsf(x) < CUDART_INF_F ? x : CUDART_NAN_F; }
// Two codes (x the lower).
__device__ __forceinline__ uint32_t codes2(float x, float y) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(y), "f"(x));
  return r;
}

template <typename T>
__device__ __forceinline__ float rounded(float x) { return to_f32(from_f32<T>(x)); }

// Any rotary dimension, stride and alignment: a block per token, a thread per pair of
// elements (or single element past the rotary dimension), a warp per head of an 8-bit cache.
template <typename T>
__global__ void __launch_bounds__(kThreads) rope_any_kernel(const __grid_constant__ RopeLaunch a) {
  pdl_launch_dependents();
  pdl_wait();
  const int64_t i = blockIdx.x;
  const int pos = a.rope.rot ? a.positions[i] : 0;
  const CacheRow to = cache_row(a, i, threadIdx.x == 0);
  for (int r = 0; r < a.n_rows; ++r) {
    const RopeRows& rows = a.rows[r];
    if (rows.cached && !to.have) continue;
    if (rows.scale) {
      constexpr int kMost = kMaxPagedHeadDim / 32;  // elements per lane
      const int lane = threadIdx.x & 31, half = rows.rotate ? a.rope.rot / 2 : 0;
      const bool halves = a.rope.layout == DCK_ROPE_HALF;
      for (int h = threadIdx.x >> 5; h < rows.heads; h += kThreads / 32) {
        const T* sp = static_cast<const T*>(rows.src) + i * rows.src_tok + h * rows.src_head;
        float x[kMost];
        float top = 0.f;
#pragma unroll
        for (int k = 0; k < kMost; ++k) {
          const int e = lane + 32 * k;
          x[k] = 0.f;
          if (e < 2 * half) {  // one of pair j's elements
            const int j = halves ? (e < half ? e : e - half) : e / 2;
            const bool second = halves ? e >= half : e & 1;
            float sn, cs;
            signed_sincos(a.rope.f[j], pos, sn, cs);
            sn *= a.rope.sign * a.rope.magnitude;
            cs *= a.rope.magnitude;
            const float u = to_f32(sp[halves ? j : 2 * j]), w = to_f32(sp[halves ? j + half : 2 * j + 1]);
            x[k] = rounded<T>(second ? u * sn + w * cs : u * cs - w * sn);
          } else if (e < a.d) {
            x[k] = to_f32(sp[e]);
          }
          x[k] = without_infinity(x[k]);
          top = larger(top, x[k]);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
        const int s = scale_exponent(top);
        const float inverse = power_of_two(-s);
        uint8_t* dp = static_cast<uint8_t*>(rows.dst) + to.page * rows.dst_page + to.off * rows.dst_tok + h * rows.dst_head;
#pragma unroll
        for (int k = 0; k < kMost; ++k)
          if (lane + 32 * k < a.d) dp[lane + 32 * k] = (uint8_t)codes2(x[k] * inverse, 0.f);
        if (lane == 0)
          rows.scale[to.page * rows.scale_page + to.off * rows.scale_tok + h * rows.scale_head] = power_of_two(s);
      }
      continue;
    }
    const T* src = static_cast<const T*>(rows.src) + i * rows.src_tok;
    T* dst = static_cast<T*>(rows.dst) + (rows.cached ? to.page * rows.dst_page + to.off * rows.dst_tok : i * rows.dst_tok);
    const int half = rows.rotate ? a.rope.rot / 2 : 0;
    const int per = half + (a.d - 2 * half);  // pairs, then single elements
    for (int64_t e = threadIdx.x; e < (int64_t)rows.heads * per; e += kThreads) {
      const int h = (int)(e / per), j = (int)(e - (int64_t)h * per);
      const T* sp = src + h * rows.src_head;
      T* dp = dst + h * rows.dst_head;
      if (j < half) {
        const int i0 = a.rope.layout == DCK_ROPE_HALF ? j : 2 * j, i1 = a.rope.layout == DCK_ROPE_HALF ? j + half : 2 * j + 1;
        float sn, cs;
        signed_sincos(a.rope.f[j], pos, sn, cs);
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

template <typename T>
struct Vec;  // 16 bytes of elements
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void open(const uint4& v, float* x) {
    x[0] = __uint_as_float(v.x), x[1] = __uint_as_float(v.y), x[2] = __uint_as_float(v.z), x[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 close(const float* x) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void open(const uint4& v, float* x) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
  static __device__ __forceinline__ uint4 close(const float* x) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// Rows of whole 16-byte vectors, a rotary dimension of whole pairs of vectors.  A
// thread's unit is two vectors of a head: those of N pairs, or of elements past the
// rotary dimension.  Threads are laid out (head, unit) over the heads of all the block's
// tokens, and each visits its unit of every across-th head.  The first loads are under way
// while the block computes its tokens' sines and cosines (once per token, for all heads)
// into shared memory.  One unit in flight per thread and six blocks per SM: with two or
// four units in flight and as many blocks as their registers leave, 16384 x 32 heads of 128
// took 42.8 and 49.5 us for 42.3 (268 MB, 93% of the copy bandwidth); with eight blocks 42.0,
// but small fp32 calls 15% more.
struct VecLaunch {
  int turned;   // units of pairs per head
  int units;    // units per head
  int lanes;    // threads per head: as many, or for 8-bit caches the next power of two
  int across;   // heads that a block's threads cover at a time
  int tokens;   // tokens per block
  int heads;    // heads of all row sets
  Divider by_lanes, by_heads, by_turned;
};
constexpr int kRounds = 2;  // units per thread that a block's tokens are chosen for (1, 4 or 8: 43, 44, 48 us there)

template <typename T, bool HALF, bool QUANT>
__global__ void __launch_bounds__(kThreads, 6) rope_vec_kernel(const __grid_constant__ RopeLaunch a,
                                                               const __grid_constant__ VecLaunch v) {
  constexpr int N = Vec<T>::N;
  // [tokens][N][turned] (cos, sin) of pair j N + k at k turned + j; then the tokens' cache rows
  extern __shared__ float2 turn[];
  const int pairs = a.rope.rot / 2;
  CacheRow* rows_to = reinterpret_cast<CacheRow*>(turn + v.tokens * pairs);
  const int tid = threadIdx.x, h0 = v.by_lanes.div(tid), j = tid - h0 * v.lanes;
  const int64_t first = (int64_t)blockIdx.x * v.tokens;
  const int n_here = (int)min((int64_t)v.tokens, a.n_tok - first), n_heads = n_here * v.heads;
  // the unit's two vectors: pairs (x, y) side by side or half the rotary dimension apart
  const int past = 2 * v.turned + 2 * (j - v.turned);
  const int va = (j >= v.turned ? past : HALF ? j : 2 * j) * N, vb = (j >= v.turned ? past + 1 : HALF ? j + v.turned : 2 * j + 1) * N;
  const bool one = !QUANT || va < a.d, two = vb < a.d;
  const uint32_t sharers = QUANT ? (v.lanes < 32 ? ((1u << v.lanes) - 1) << (tid & 31 & -v.lanes) : ~0u) : 0;

  int next = h0 < v.across ? h0 : n_heads, t, head, set;
  uint4 x, y;
  const auto load = [&]() {
    if (next >= n_heads) return;
    t = v.by_heads.div(next);
    head = next - t * v.heads;
    set = 0;
    while (set + 1 < a.n_rows && head >= a.rows[set].heads) head -= a.rows[set++].heads;
    const T* src = static_cast<const T*>(a.rows[set].src) + (first + t) * a.rows[set].src_tok + head * a.rows[set].src_head;
    if (one) x = *reinterpret_cast<const uint4*>(src + va);
    if (two) y = *reinterpret_cast<const uint4*>(src + vb);
  };
  pdl_launch_dependents();
  pdl_wait();
  load();
  for (int z = tid; z < n_here * pairs; z += kThreads) {
    const int q = v.by_turned.div(z), jj = z - q * v.turned, tok = q / N, k = q - tok * N;
    float sn, cs;
    signed_sincos(a.rope.f[jj * N + k], a.positions[first + tok], sn, cs);
    turn[z] = make_float2(cs * a.rope.magnitude, sn * (a.rope.sign * a.rope.magnitude));
  }
  if (a.slots)
    for (int i = tid; i < n_here; i += kThreads) rows_to[i] = cache_row(a, first + i, true);
  __syncthreads();
  for (; next < n_heads; next += v.across, load()) {
    const RopeRows& rows = a.rows[set];
    int64_t at = (first + t) * rows.dst_tok;
    if (rows.cached) {
      const CacheRow to = rows_to[t];
      if (!to.have) continue;
      at = to.page * rows.dst_page + to.off * rows.dst_tok;
    }
    float p[N], q[N];
    if (rows.rotate && j < v.turned) {
      const float2* cs = turn + t * pairs + j;
      Vec<T>::open(x, p);
      Vec<T>::open(y, q);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float2 z = cs[k * v.turned];
        float& e0 = HALF ? p[k] : k < N / 2 ? p[2 * k % N] : q[2 * k % N];
        float& e1 = HALF ? q[k] : k < N / 2 ? p[(2 * k + 1) % N] : q[(2 * k + 1) % N];
        const float w = e0 * z.x - e1 * z.y;
        e1 = e0 * z.y + e1 * z.x;
        e0 = w;
      }
      x = Vec<T>::close(p);
      y = Vec<T>::close(q);
    }
    if (QUANT && rows.scale) {
      Vec<T>::open(one ? x : make_uint4(0, 0, 0, 0), p);  // what was rounded to T
      Vec<T>::open(two ? y : make_uint4(0, 0, 0, 0), q);
      const auto largest = [&]() {
        float top = 0.f;
#pragma unroll
        for (int k = 0; k < N; ++k) top = larger(top, p[k]), top = larger(top, q[k]);
        for (int o = v.lanes / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(sharers, top, o));
        return top;
      };
      float top = largest();
      if (top == CUDART_INF_F) {  // (alike in all threads of the row)
#pragma unroll
        for (int k = 0; k < N; ++k) p[k] = without_infinity(p[k]), q[k] = without_infinity(q[k]);
        top = largest();
      }
      const int e = scale_exponent(top);
      const float inverse = power_of_two(-e);
      uint8_t* dst = static_cast<uint8_t*>(rows.dst) + at + head * rows.dst_head;
      uint32_t c[N / 2];
#pragma unroll
      for (int k = 0; k < N / 4; ++k) {
        c[k] = codes2(p[4 * k] * inverse, p[4 * k + 1] * inverse) | codes2(p[4 * k + 2] * inverse, p[4 * k + 3] * inverse) << 16;
        c[N / 4 + k] = codes2(q[4 * k] * inverse, q[4 * k + 1] * inverse) | codes2(q[4 * k + 2] * inverse, q[4 * k + 3] * inverse) << 16;
      }
      if (N == 8) {
        if (one) *reinterpret_cast<uint2*>(dst + va) = make_uint2(c[0], c[1]);
        if (two) *reinterpret_cast<uint2*>(dst + vb) = make_uint2(c[N / 4], c[N / 4 + 1 < N / 2 ? N / 4 + 1 : 0]);
      } else {
        if (one) *reinterpret_cast<uint32_t*>(dst + va) = c[0];
        if (two) *reinterpret_cast<uint32_t*>(dst + vb) = c[N / 4];
      }
      if (j == 0) {
        const CacheRow to = rows_to[t];
        rows.scale[to.page * rows.scale_page + to.off * rows.scale_tok + head * rows.scale_head] = power_of_two(e);
      }
      continue;
    }
    T* dst = static_cast<T*>(rows.dst) + at + head * rows.dst_head;
    if (!one) continue;
    *reinterpret_cast<uint4*>(dst + va) = x;
    if (two) *reinterpret_cast<uint4*>(dst + vb) = y;
  }
}

template <typename T>
bool vec_plan(const RopeLaunch& a, int sms, VecLaunch* v) {
  constexpr int N = Vec<T>::N;
  if (a.d % N || a.rope.rot % (2 * N)) return false;
  v->heads = 0;
  bool quant = false;
  for (int r = 0; r < a.n_rows; ++r) {
    const RopeRows& w = a.rows[r];
    if (reinterpret_cast<uintptr_t>(w.src) % 16 || reinterpret_cast<uintptr_t>(w.dst) % 16) return false;
    for (int64_t st : {w.src_tok, w.src_head, w.dst_tok, w.dst_head, w.dst_page})  // (8-bit caches: multiples of 16)
      if (st % N) return false;
    quant |= w.scale != nullptr;
    v->heads += w.heads;
  }
  v->turned = a.rope.rot / (2 * N);
  v->units = v->turned + ((a.d - a.rope.rot) / N + 1) / 2;
  if (v->units > (quant ? 32 : kThreads)) return false;
  v->lanes = v->units;
  if (quant)
    for (v->lanes = 1; v->lanes < v->units;) v->lanes *= 2;
  v->across = kThreads / v->lanes;
  // as many tokens as give every thread a few units, if eight blocks per SM remain
  const int64_t full = (kRounds * v->across + v->heads - 1) / v->heads, one = (v->across + v->heads - 1) / v->heads;
  v->tokens = (int)std::min<int64_t>(std::max<int64_t>(std::min(full, (int64_t)a.n_tok / (8 * sms)), one), a.n_tok);
  v->by_lanes = divider(v->lanes);
  v->by_heads = divider(v->heads);
  v->by_turned = divider(std::max(1, v->turned));
  return true;
}

template <typename T>
cudaError_t launch(const RopeLaunch& a, int sms, cudaStream_t s) {
  VecLaunch v;
  if (!vec_plan<T>(a, sms, &v)) {
    return launch_pdl(rope_any_kernel<T>, a.n_tok, kThreads, 0, s, a);
  }
  const int64_t grid = ((int64_t)a.n_tok + v.tokens - 1) / v.tokens;
  const size_t smem = (size_t)v.tokens * (a.rope.rot / 2 * sizeof(float2) + sizeof(CacheRow));
  const bool half = a.rope.layout == DCK_ROPE_HALF;
  const auto k = a.rows[0].scale ? (half ? rope_vec_kernel<T, true, true> : rope_vec_kernel<T, false, true>)
                                 : (half ? rope_vec_kernel<T, true, false> : rope_vec_kernel<T, false, false>);
  return launch_pdl(k, (unsigned)grid, kThreads, smem, s, a, v);
}

}  // namespace

cudaError_t launch_rope_rows(const RopeLaunch& a, int dtype, int sms, cudaStream_t s) {
  return dtype == DCK_F32 ? launch<float>(a, sms, s) : launch<__nv_bfloat16>(a, sms, s);
}

}  // namespace dck

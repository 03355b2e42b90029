// Rotary positions (dck_rope) and the rotated append to a paged cache
// (dck_paged_append).  A pair (x, y) of a head's elements at position t becomes
//   m (x cos a - y sin a, x sin a + y cos a),  a = t w_i  (sin negated: the transpose).
// Bound by memory: each element is read and written once.
#include <algorithm>

#include "paged.cuh"
#include "rope.cuh"

namespace dck {
namespace {

constexpr int kThreads = 256;

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

// Any rotary dimension, stride and alignment: a block per token, a thread per pair of
// elements (or single element past the rotary dimension).
template <typename T>
__global__ void __launch_bounds__(kThreads) rope_any_kernel(const __grid_constant__ RopeLaunch a) {
  const int64_t i = blockIdx.x;
  const uint32_t pos = a.rope.rot ? (uint32_t)a.positions[i] : 0u;
  const CacheRow to = cache_row(a, i, threadIdx.x == 0);
  for (int r = 0; r < a.n_rows; ++r) {
    const RopeRows& rows = a.rows[r];
    if (rows.cached && !to.have) continue;
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
        rope_sincos(a.rope.f[j], pos, sn, cs);
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
// rotary dimension.  Threads are laid out (token, head, unit); each visits its unit of
// further heads and tokens, with the loads of kUnroll of them in flight, the first of
// them while the block computes its tokens' sines and cosines (once per token, for all
// heads) into shared memory.
struct VecLaunch {
  int turned;   // units of pairs per head
  int units;    // units per head
  int across;   // heads that a token's threads cover at a time
  int abreast;  // tokens that a block's threads cover at a time
  int tokens;   // tokens per block
  int heads;    // heads of all row sets
  Divider by_token, by_head;  // threads per token, units per head
  Divider by_turned;
};
constexpr int kUnroll = 4;

template <typename T, bool HALF>
__global__ void __launch_bounds__(kThreads, 3) rope_vec_kernel(const __grid_constant__ RopeLaunch a,
                                                               const __grid_constant__ VecLaunch v) {
  constexpr int N = Vec<T>::N;
  // [tokens][N][turned] (cos, sin) of pair j N + k at k turned + j; then the tokens' cache rows
  extern __shared__ float2 turn[];
  const int pairs = a.rope.rot / 2;
  CacheRow* rows_to = reinterpret_cast<CacheRow*>(turn + v.tokens * pairs);
  const int tid = threadIdx.x;
  const int tok = v.by_token.div(tid), in_tok = tid - tok * v.by_token.d;
  const int h0 = v.by_head.div(in_tok), j = in_tok - h0 * v.units;
  const int64_t first = (int64_t)blockIdx.x * v.tokens;
  const int n_here = (int)min((int64_t)v.tokens, a.n_tok - first);
  // the unit's two vectors: pairs (x, y) side by side or half the rotary dimension apart
  const int past = 2 * v.turned + 2 * (j - v.turned);
  const int va = j >= v.turned ? past : HALF ? j : 2 * j, vb = j >= v.turned ? past + 1 : HALF ? j + v.turned : 2 * j + 1;
  const bool two = vb * N < a.d;

  struct Unit {
    int t, set, head;  // t < 0: none
  };
  int t_next = tok < v.abreast ? tok : n_here, h_next = h0;
  Unit unit[kUnroll];
  uint4 x[kUnroll], y[kUnroll];
  const auto load = [&]() {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      unit[u].t = -1;
      if (t_next >= n_here) continue;
      int hh = h_next, r = 0;
      while (r + 1 < a.n_rows && hh >= a.rows[r].heads) hh -= a.rows[r++].heads;
      unit[u] = {t_next, r, hh};
      const T* src = static_cast<const T*>(a.rows[r].src) + (first + t_next) * a.rows[r].src_tok + hh * a.rows[r].src_head;
      x[u] = *reinterpret_cast<const uint4*>(src + va * N);
      if (two) y[u] = *reinterpret_cast<const uint4*>(src + vb * N);
      h_next += v.across;
      if (h_next >= v.heads) h_next = h0, t_next += v.abreast;
    }
  };
  load();
  for (int z = tid; z < n_here * pairs; z += kThreads) {
    const int q = v.by_turned.div(z), jj = z - q * v.turned, t = q / N, k = q - t * N;
    float sn, cs;
    rope_sincos(a.rope.f[jj * N + k], (uint32_t)a.positions[first + t], sn, cs);
    turn[z] = make_float2(cs * a.rope.magnitude, sn * (a.rope.sign * a.rope.magnitude));
  }
  if (a.slots)
    for (int t = tid; t < n_here; t += kThreads) rows_to[t] = cache_row(a, first + t, true);
  __syncthreads();
  while (unit[0].t >= 0) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (unit[u].t < 0) continue;
      const RopeRows& rows = a.rows[unit[u].set];
      int64_t at = (first + unit[u].t) * rows.dst_tok;
      if (rows.cached) {
        const CacheRow to = rows_to[unit[u].t];
        if (!to.have) continue;
        at = to.page * rows.dst_page + to.off * rows.dst_tok;
      }
      T* dst = static_cast<T*>(rows.dst) + at + unit[u].head * rows.dst_head;
      if (rows.rotate && j < v.turned) {
        const float2* cs = turn + unit[u].t * pairs + j;
        float p[N], q[N];
        Vec<T>::open(x[u], p);
        Vec<T>::open(y[u], q);
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const float2 z = cs[k * v.turned];
          float& e0 = HALF ? p[k] : k < N / 2 ? p[2 * k % N] : q[2 * k % N];
          float& e1 = HALF ? q[k] : k < N / 2 ? p[(2 * k + 1) % N] : q[(2 * k + 1) % N];
          const float w = e0 * z.x - e1 * z.y;
          e1 = e0 * z.y + e1 * z.x;
          e0 = w;
        }
        x[u] = Vec<T>::close(p);
        y[u] = Vec<T>::close(q);
      }
      *reinterpret_cast<uint4*>(dst + va * N) = x[u];
      if (two) *reinterpret_cast<uint4*>(dst + vb * N) = y[u];
    }
    load();
  }
}

template <typename T>
bool vec_plan(const RopeLaunch& a, int sms, VecLaunch* v) {
  constexpr int N = Vec<T>::N;
  if (a.d % N || a.rope.rot % (2 * N)) return false;
  v->heads = 0;
  for (int r = 0; r < a.n_rows; ++r) {
    const RopeRows& w = a.rows[r];
    if (reinterpret_cast<uintptr_t>(w.src) % 16 || reinterpret_cast<uintptr_t>(w.dst) % 16) return false;
    for (int64_t st : {w.src_tok, w.src_head, w.dst_tok, w.dst_head, w.dst_page})
      if (st % N) return false;
    v->heads += w.heads;
  }
  v->turned = a.rope.rot / (2 * N);
  v->units = v->turned + ((a.d - a.rope.rot) / N + 1) / 2;
  if (v->units > kThreads) return false;
  v->across = std::min(v->heads, kThreads / v->units);
  v->abreast = (int)std::min<int64_t>(kThreads / (v->across * v->units), a.n_tok);
  // enough tokens for a few rounds of loads per thread, as long as four blocks per SM remain
  const int rounds = (v->heads + v->across - 1) / v->across;
  const int64_t spread = a.n_tok / ((int64_t)v->abreast * 4 * sms);
  v->tokens = v->abreast * (int)std::max<int64_t>(1, std::min<int64_t>(spread, (2 * kUnroll + rounds - 1) / rounds));
  v->by_token = divider(v->across * v->units);
  v->by_head = divider(v->units);
  v->by_turned = divider(std::max(1, v->turned));
  return true;
}

template <typename T>
cudaError_t launch(const RopeLaunch& a, int sms, cudaStream_t s) {
  VecLaunch v;
  if (!vec_plan<T>(a, sms, &v)) {
    rope_any_kernel<T><<<a.n_tok, kThreads, 0, s>>>(a);
    return cudaGetLastError();
  }
  const int grid = (a.n_tok + v.tokens - 1) / v.tokens;
  const size_t smem = (size_t)v.tokens * (a.rope.rot / 2 * sizeof(float2) + sizeof(CacheRow));
  if (a.rope.layout == DCK_ROPE_HALF) rope_vec_kernel<T, true><<<grid, kThreads, smem, s>>>(a, v);
  else rope_vec_kernel<T, false><<<grid, kThreads, smem, s>>>(a, v);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_rope_rows(const RopeLaunch& a, int dtype, int sms, cudaStream_t s) {
  return dtype == DCK_F32 ? launch<float>(a, sms, s) : launch<__nv_bfloat16>(a, sms, s);
}

}  // namespace dck

// Rows of an 8-bit cache in full width (dck_quant_read): code times scale, rounded once.
// Bound by memory: (d + 4) bytes read and 2 or 4 d written per head's row.  A thread's unit is 16 bytes
// of output (8 or 4 codes), kInFlight units of a block under way at a time.
#include <cuda_fp16.h>

#include <algorithm>

#include "paged.cuh"

namespace dck {
namespace {

constexpr int kThreads = 256, kInFlight = 4;

struct Units {
  uint32_t per_token, per_head;  // units of both caches; of a head's row
  Divider by_token, by_head;
  int64_t n;
};

__device__ __forceinline__ float2 two_values(uint32_t codes, float scale) {
  uint32_t h;
  asm("{\n .reg .b16 l, u;\n mov.b32 {l, u}, %1;\n cvt.rn.f16x2.e4m3x2 %0, l;\n}\n" : "=r"(h) : "r"(codes));
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
  return make_float2(f.x * scale, f.y * scale);
}

template <typename T>
struct Out;
template <>
struct Out<__nv_bfloat16> {
  static constexpr int N = 8;
  using Codes = uint2;
  static __device__ __forceinline__ uint4 open(uint2 c, float s) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = two_values((i < 2 ? c.x : c.y) >> (i & 1) * 16, s);
      const __nv_bfloat162 b = __floats2bfloat162_rn(f.x, f.y);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <>
struct Out<float> {
  static constexpr int N = 4;
  using Codes = uint32_t;
  static __device__ __forceinline__ uint4 open(uint32_t c, float s) {
    const float2 a = two_values(c, s), b = two_values(c >> 16, s);
    return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
  }
};

// WIDE: outputs in 16-byte stores.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(kThreads) quant_read_kernel(const __grid_constant__ QuantReadArgs a,
                                                              const __grid_constant__ Units u) {
  constexpr int N = Out<T>::N;
  pdl_launch_dependents();
  pdl_wait();
  const PagedView& v = a.v;
  for (int64_t base = (int64_t)blockIdx.x * kThreads * kInFlight; base < u.n; base += (int64_t)gridDim.x * kThreads * kInFlight) {
    typename Out<T>::Codes codes[kInFlight];
    float scale[kInFlight];
    T* to[kInFlight];
#pragma unroll
    for (int k = 0; k < kInFlight; ++k) {
      const int64_t at = base + k * kThreads + threadIdx.x;
      to[k] = nullptr;
      if (at >= u.n) continue;
      const int64_t tok = at >> 31 ? at / u.per_token : (int64_t)u.by_token.div((uint32_t)at);
      const uint32_t x = (uint32_t)(at - tok * u.per_token), row = u.by_head.div(x), e = (x - row * u.per_head) * N;
      const bool value = row >= (uint32_t)v.Hkv;
      const uint32_t head = value ? row - v.Hkv : row;
      to[k] = static_cast<T*>(value ? a.v_out : a.k) + tok * (value ? a.v_stride : a.k_stride) + head * v.d + e;
      const int64_t slot = a.slots[tok];
      codes[k] = {};
      scale[k] = 0.f;
      if (slot < 0 || slot >= (int64_t)v.n_pages * v.page) {
        if (slot != -1 && x == 0) atomicOr(a.err, kErrBadRow);
        continue;
      }
      const uint64_t page = slot >> 31 ? slot / v.page : (int64_t)v.by_page.div((uint32_t)slot), off = slot - page * v.page;
      const char* p = static_cast<const char*>(value ? a.vc : a.kc);
      codes[k] = *reinterpret_cast<const typename Out<T>::Codes*>(
          p + (value ? page * v.v_page_b + off * v.v_tok_b + (uint64_t)head * v.v_head_b
                     : page * v.k_page_b + off * v.k_tok_b + (uint64_t)head * v.k_head_b) + e);
      scale[k] = value ? a.vs[page * v.vs_page + off * v.vs_tok + (uint64_t)head * v.vs_head]
                       : a.ks[page * v.ks_page + off * v.ks_tok + (uint64_t)head * v.ks_head];
    }
#pragma unroll
    for (int k = 0; k < kInFlight; ++k) {
      if (!to[k]) continue;
      const uint4 w = Out<T>::open(codes[k], scale[k]);
      if (WIDE) {
        *reinterpret_cast<uint4*>(to[k]) = w;
      } else {
        const T* from = reinterpret_cast<const T*>(&w);
#pragma unroll
        for (int i = 0; i < N; ++i) to[k][i] = from[i];
      }
    }
  }
}

template <typename T>
cudaError_t launch(const QuantReadArgs& a, int sms, cudaStream_t s) {
  constexpr int N = Out<T>::N;
  Units u;
  u.per_head = a.v.d / N;
  u.per_token = 2 * a.v.Hkv * u.per_head;
  u.by_token = divider(u.per_token);
  u.by_head = divider(u.per_head);
  u.n = (int64_t)a.n_tok * u.per_token;
  const bool wide = reinterpret_cast<uintptr_t>(a.k) % 16 == 0 && reinterpret_cast<uintptr_t>(a.v_out) % 16 == 0 &&
                    a.k_stride % N == 0 && a.v_stride % N == 0;
  const int64_t blocks = (u.n + kThreads * kInFlight - 1) / (kThreads * kInFlight);
  const auto k = wide ? quant_read_kernel<T, true> : quant_read_kernel<T, false>;
  return launch_pdl(k, (unsigned)std::min<int64_t>(blocks, int64_t(1) << 30), kThreads, 0, s, a, u);
}

}  // namespace

cudaError_t launch_quant_read(const QuantReadArgs& a, int dtype, int sms, cudaStream_t s) {
  return dtype == DCK_F32 ? launch<float>(a, sms, s) : launch<__nv_bfloat16>(a, sms, s);
}

}  // namespace dck

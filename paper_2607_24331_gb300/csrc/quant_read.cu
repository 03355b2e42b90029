// Rows of an 8-bit cache in full width (dck_quant_read): code times scale, rounded once.
// Bound by memory: (d + 4) bytes read and 2 or 4 d written per head's row.  A thread's unit is 16 codes (8 where the head
// dim is no multiple of 16), read at once and written in 32-byte stores, whole sectors, where the output lies so; kInFlight
// units are under way at a time.  (Units of 8 codes, 16-byte stores: 65536 x 8 heads of 128 in bf16, 407 MB, 90 us, bound by
// instructions: most of a unit's are for its addresses; 65 us so.)
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

__device__ __forceinline__ float2 two_values(uint32_t codes, float scale) {  // of the lower 16 bits
  uint32_t h;
  asm("{\n .reg .b16 l, u;\n mov.b32 {l, u}, %1;\n cvt.rn.f16x2.e4m3x2 %0, l;\n}\n" : "=r"(h) : "r"(codes));
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
  return make_float2(f.x * scale, f.y * scale);
}
// Four codes as elements in 32-bit words.
__device__ __forceinline__ void open4(uint32_t c, float s, uint32_t* w, float) {
  const float2 a = two_values(c, s), b = two_values(c >> 16, s);
  w[0] = __float_as_uint(a.x), w[1] = __float_as_uint(a.y), w[2] = __float_as_uint(b.x), w[3] = __float_as_uint(b.y);
}
__device__ __forceinline__ void open4(uint32_t c, float s, uint32_t* w, __nv_bfloat16) {
  const float2 a = two_values(c, s), b = two_values(c >> 16, s);
  const __nv_bfloat162 x = __floats2bfloat162_rn(a.x, a.y), y = __floats2bfloat162_rn(b.x, b.y);
  w[0] = *reinterpret_cast<const uint32_t*>(&x), w[1] = *reinterpret_cast<const uint32_t*>(&y);
}
__device__ __forceinline__ void store32(void* p, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
               "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

// N: codes of a unit; ALIGN: bytes that the outputs' units are aligned to (32, 16 or an element).
template <typename T, int N, int ALIGN>
__global__ void __launch_bounds__(kThreads) quant_read_kernel(const __grid_constant__ QuantReadArgs a,
                                                              const __grid_constant__ Units u) {
  constexpr int kWords = N * sizeof(T) / 4;
  pdl_launch_dependents();
  pdl_wait();
  const PagedView& v = a.v;
  const int64_t base = (int64_t)blockIdx.x * (kThreads * kInFlight) + threadIdx.x;
  uint32_t codes[kInFlight][N / 4];
  float scale[kInFlight];
  T* to[kInFlight];
#pragma unroll
  for (int k = 0; k < kInFlight; ++k) {
    const int64_t at = base + k * kThreads;
    to[k] = nullptr;
    if (at >= u.n) continue;
    const int64_t tok = at >> 31 ? at / u.per_token : (int64_t)u.by_token.div((uint32_t)at);
    const uint32_t x = (uint32_t)(at - tok * u.per_token), row = u.by_head.div(x), e = (x - row * u.per_head) * N;
    const bool value = row >= (uint32_t)v.Hkv;
    const uint32_t head = value ? row - v.Hkv : row;
    to[k] = static_cast<T*>(value ? a.v_out : a.k) + tok * (value ? a.v_stride : a.k_stride) + head * v.d + e;
    const int64_t slot = a.slots[tok];
#pragma unroll
    for (int i = 0; i < N / 4; ++i) codes[k][i] = 0;
    scale[k] = 0.f;
    if (slot < 0 || slot >= (int64_t)v.n_pages * v.page) {
      if (slot != -1 && x == 0) atomicOr(a.err, kErrBadRow);
      continue;
    }
    const uint64_t page = slot >> 31 ? slot / v.page : (int64_t)v.by_page.div((uint32_t)slot);
    const uint32_t off = (uint32_t)(slot - page * v.page);
    const char* p = static_cast<const char*>(value ? a.vc : a.kc) + e + page * (value ? v.v_page_b : v.k_page_b) +
                    (uint64_t)off * (value ? v.v_tok_b : v.k_tok_b) + (uint64_t)head * (value ? v.v_head_b : v.k_head_b);
    if (N == 16) {
      const uint4 c = *reinterpret_cast<const uint4*>(p);
      codes[k][0] = c.x, codes[k][1] = c.y, codes[k][2 % (N / 4)] = c.z, codes[k][3 % (N / 4)] = c.w;
    } else {
      const uint2 c = *reinterpret_cast<const uint2*>(p);
      codes[k][0] = c.x, codes[k][1] = c.y;
    }
    scale[k] = (value ? a.vs : a.ks)[page * (value ? v.vs_page : v.ks_page) + (uint64_t)off * (value ? v.vs_tok : v.ks_tok) +
                                     (uint64_t)head * (value ? v.vs_head : v.ks_head)];
  }
#pragma unroll
  for (int k = 0; k < kInFlight; ++k) {
    if (!to[k]) continue;
    uint32_t w[kWords];
#pragma unroll
    for (int i = 0; i < N / 4; ++i) open4(codes[k][i], scale[k], w + i * (kWords * 4 / N), T());
    if (ALIGN == 32) {
#pragma unroll
      for (int i = 0; i < kWords; i += 8) store32(reinterpret_cast<uint32_t*>(to[k]) + i, w + i % kWords);
    } else if (ALIGN == 16) {
#pragma unroll
      for (int i = 0; i < kWords; i += 4)
        reinterpret_cast<uint4*>(to[k])[i / 4] = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
    } else {
      const T* from = reinterpret_cast<const T*>(w);
#pragma unroll
      for (int i = 0; i < N; ++i) to[k][i] = from[i];
    }
  }
}

template <typename T, int N>
cudaError_t launch(const QuantReadArgs& a, cudaStream_t s) {
  Units u;
  u.per_head = a.v.d / N;
  u.per_token = 2 * a.v.Hkv * u.per_head;
  u.by_token = divider(u.per_token);
  u.by_head = divider(u.per_head);
  u.n = (int64_t)a.n_tok * u.per_token;
  const auto aligned = [&](uintptr_t bytes) {
    return reinterpret_cast<uintptr_t>(a.k) % bytes == 0 && reinterpret_cast<uintptr_t>(a.v_out) % bytes == 0 &&
           a.k_stride * sizeof(T) % bytes == 0 && a.v_stride * sizeof(T) % bytes == 0;
  };
  const int64_t blocks = (u.n + kThreads * kInFlight - 1) / (kThreads * kInFlight);  // (2^31 of them would write 2^45 bytes)
  const auto k = aligned(32) && N * sizeof(T) >= 32 ? quant_read_kernel<T, N, N * sizeof(T) >= 32 ? 32 : 16>
                 : aligned(16)                       ? quant_read_kernel<T, N, 16>
                                                     : quant_read_kernel<T, N, sizeof(T)>;
  return launch_pdl(k, (unsigned)blocks, kThreads, 0, s, a, u);
}

}  // namespace

cudaError_t launch_quant_read(const QuantReadArgs& a, int dtype, cudaStream_t s) {
  if (a.v.d % 16 == 0) return dtype == DCK_F32 ? launch<float, 16>(a, s) : launch<__nv_bfloat16, 16>(a, s);
  return dtype == DCK_F32 ? launch<float, 8>(a, s) : launch<__nv_bfloat16, 8>(a, s);
}

}  // namespace dck

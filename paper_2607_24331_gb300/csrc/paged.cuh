// Internal declarations of the paged key-value cache's kernels (page
// bookkeeping, rotary positions and cache writes, decode attention).
#pragma once

#include "common.cuh"

namespace dck {

constexpr int kMaxPagedHeadDim = 256;
constexpr int kMaxPageSize = 65536;

// Exact n / d for 0 <= n < 2^31, 1 <= d <= 2^31, without a division: with
// 2^(s-1) < d <= 2^s and m = floor(2^32 (2^s - d) / d) + 1 the quotient is
// (hi32(n m) + n) >> s (Granlund and Montgomery 1994).
struct Divider {
  uint32_t m, s, d;
  __device__ __forceinline__ uint32_t div(uint32_t n) const { return (__umulhi(n, m) + n) >> s; }
};
inline Divider divider(uint32_t d) {
  Divider v;
  v.d = d;
  v.s = 0;
  while ((uint64_t(1) << v.s) < d) ++v.s;
  v.m = (uint32_t)((((uint64_t(1) << v.s) - d) << 32) / d + 1);
  return v;
}

// One layer's paged caches, by value.
struct PagedView {
  int32_t Hq, Hkv, d, qpg, page, n_pages;
  uint32_t k_page_b, k_tok_b, k_head_b, v_page_b, v_tok_b, v_head_b;  // strides, in bytes
  Divider by_page;
};

// The rotation, by value (dck_rope_table).
struct RopeArgs {
  int32_t layout, rot;  // rot = 0: no rotation
  float magnitude, sign;  // sign -1: the transpose
  uint2 f[128];           // {low, high} words of the turns
};

struct PageUpdateArgs {
  int32_t B, page, n_pages;
  const int32_t* old_len;
  const int32_t* new_len;
  int32_t* seq_len;
  int32_t* table;
  int64_t table_stride;
  int32_t* free_pages;
  const int32_t* free_in;
  int32_t* free_out;
  int64_t n_tok;
  int64_t* slots;
  int32_t* positions;
  int32_t* cu_new;
  int* err;
};
cudaError_t launch_page_update(const PageUpdateArgs& a, cudaStream_t s);

// A set of rows to rotate (or copy) by token: element (i, h, e) from
// src + i src_tok + h src_head + e to dst + row(i) + h dst_head + e, where
// row(i) is i dst_tok, or, with slots, the cache row of slots[i].
struct RopeRows {
  const void* src;
  void* dst;
  int64_t src_tok, src_head, dst_tok, dst_head;
  int32_t heads;
  int32_t rotate;  // 0: copy
  int32_t cached;  // dst is a cache: rows by slot (dst_tok between a page's tokens, dst_page between pages)
  int64_t dst_page;
};
struct RopeLaunch {
  RopeRows rows[3];
  int32_t n_rows, n_tok, d;
  const int32_t* positions;
  const int64_t* slots;
  int32_t page, n_pages;
  Divider by_page;
  int* err;
  RopeArgs rope;
};
cudaError_t launch_rope_rows(const RopeLaunch& a, int dtype, int sms, cudaStream_t s);

struct PagedDecodeArgs {
  PagedView v;
  const void* q;
  int64_t q_stride;
  const void* kc;
  const void* vc;
  const int32_t* table;
  int64_t table_stride;
  const int32_t* seq_len;
  int32_t B, max_len, window;
  float scale, softcap;
  void* out;
  float* lse;  // may be null
  void* ws;
  int* err;
  LaunchHook* hook;
};
size_t paged_decode_workspace(const PagedView& v, int dtype, int B, int max_len, int sms);
cudaError_t launch_paged_decode(const PagedDecodeArgs& a, int dtype, int sms, cudaStream_t s);

}  // namespace dck

// Page bookkeeping of one step (dck_page_update): prefix sums over the requests
// of pages given back, pages asked for and new tokens, then every page and every
// token finds its request by binary search in them.
//
// No page goes through memory on its way from the free list to a table entry and
// on to a slot: page number a of those taken is a function of the prefix sums and
// of entries that the call does not write (free_pages below the old count, table
// columns that a request had before).  So one launch suffices, and a token's slot
// does not wait for the table entry that it equals.  The pages that would be taken are all
// looked at before the first is written: a number outside the pool ends the list there.
#include <algorithm>

#include "paged.cuh"

namespace dck {
namespace {

constexpr int kThreads = 512;
constexpr int kNone = 0x7fffffff;

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// What CTA `rank` of the cluster holds where `p` is in this one's shared memory.
__device__ __forceinline__ int read_remote(const int* p, int rank) {
  uint32_t at;
  int v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}

struct Sums {
  int64_t rel, grow, tok;
};

// The request whose range [prefix[b], prefix[b+1]) holds x (x < prefix[B]).
__device__ __forceinline__ int request_of(const int64_t* prefix, int B, int64_t x) {
  int lo = 0, hi = B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (prefix[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// `share` of `shares`: the CTAs of the cluster each sum up all requests and take their part of
// the pages and tokens.
__global__ void __launch_bounds__(kThreads) page_update_kernel(const PageUpdateArgs a) {
  extern __shared__ int64_t sh[];
  int64_t* rel = sh;                     // [B+1] exclusive prefix sums
  int64_t* grow = rel + a.B + 1;
  int64_t* tok = grow + a.B + 1;
  int32_t* olen = reinterpret_cast<int32_t*>(tok + a.B + 1);  // [B] lengths (-1 - old: the request is refused outright)
  int32_t* nlen = olen + a.B;
  __shared__ Sums part[kThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, shares = gridDim.x, share = blockIdx.x;
  pdl_launch_dependents();
  pdl_wait();
  int64_t f = a.free_in[0];
  if (f < 0 || f > a.n_pages) {
    if (tid == 0) atomicOr(a.err, kErrBadSeq);  // (every share finds the same)
    f = 0;
  }
  Sums base = {0, 0, 0};
  for (int b0 = 0; b0 < a.B; b0 += kThreads) {
    const int b = b0 + tid;
    Sums v = {0, 0, 0};
    if (b < a.B) {
      int o = a.old_len[b], n = a.new_len[b];
      if (o >= 0 && n > o) v.tok = (int64_t)n - o;
      const int64_t po = ((int64_t)o + a.page - 1) / a.page, pn = ((int64_t)n + a.page - 1) / a.page;
      const bool old_ok = o >= 0 && po <= a.table_stride;
      if (!old_ok || n < 0 || pn > a.table_stride) {
        atomicOr(a.err, kErrBadSeq);
        o = -1 - (old_ok ? o : 0);
      } else {
        // the page that a request goes on filling: a table entry that it has already
        const int last = n > o && po * a.page > o ? a.table[(int64_t)b * a.table_stride + po - 1] : 0;
        if (last < 0 || last >= a.n_pages) {
          atomicOr(a.err, kErrBadRow);
          o = -1 - o;
        } else {
          v.rel = po > pn ? po - pn : 0;
          v.grow = pn > po ? pn - po : 0;
        }
      }
      olen[b] = o;
      nlen[b] = n;
    }
    Sums s = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t r = __shfl_up_sync(~0u, s.rel, d), g = __shfl_up_sync(~0u, s.grow, d), t = __shfl_up_sync(~0u, s.tok, d);
      if (lane >= d) s.rel += r, s.grow += g, s.tok += t;
    }
    if (lane == 31) part[warp] = s;
    __syncthreads();
    Sums before = base;
    for (int w = 0; w < kThreads / 32; ++w) {
      const Sums p = part[w];
      if (w < warp) before.rel += p.rel, before.grow += p.grow, before.tok += p.tok;
      base.rel += p.rel, base.grow += p.grow, base.tok += p.tok;
    }
    if (b < a.B) {
      rel[b] = before.rel + s.rel - v.rel;
      grow[b] = before.grow + s.grow - v.grow;
      tok[b] = before.tok + s.tok - v.tok;
    }
    __syncthreads();
  }
  if (tid == 0) rel[a.B] = base.rel, grow[a.B] = base.grow, tok[a.B] = base.tok;
  __shared__ int refused_s, first_outside;
  if (tid == 0) refused_s = 0, first_outside = kNone;
  __syncthreads();

  int64_t have = f + base.rel;  // free pages and those given back
  if (have > a.n_pages) {
    if (tid == 0) atomicOr(a.err, kErrBadSeq);
    have = a.n_pages;
  }
  const auto pages_of = [&](int len) { return ((int64_t)len + a.page - 1) / a.page; };
  // page j of the free list with the pages given back behind it
  const auto page_at = [&](int64_t j) -> int {
    if (j < f) return a.free_pages[j];
    const int b = request_of(rel, a.B, j - f);
    return a.table[(int64_t)b * a.table_stride + pages_of(nlen[b]) + (j - f - rel[b])];
  };
  const auto taken = [&](int64_t x) { return page_at(have - 1 - x); };  // the x-th page that is taken
  const int me = share * kThreads + tid, all = shares * kThreads;
  // Requests are granted pages up to the first whose own go beyond what there is, and tokens
  // up to the first whose own go beyond the slots: of those that grow, the ones before both,
  // so a prefix sum is what they take.
  const auto pages_within = [&](int64_t most) { return base.grow <= most ? base.grow : grow[request_of(grow, a.B, most)]; };
  int64_t used = pages_within(have);
  if (base.tok > a.n_tok) {
    if (tid == 0) atomicOr(a.err, kErrBadSeq);
    used = min(used, grow[request_of(tok, a.B, a.n_tok)]);
  }
  int page0 = 0;  // this thread's first page of those taken
  for (int64_t x = me; x < used; x += all) {
    const int p = taken(x);
    if (x == me) page0 = p;
    if (p < 0 || p >= a.n_pages) atomicMin(&first_outside, (int)x);
  }
  __syncthreads();
  int outside = first_outside;
  if (shares > 1) {
    // Every CTA has read the lengths, the free count and the pages: they may be written after the wait.
    cluster_arrive();
    cluster_wait();
    outside = __reduce_min_sync(~0u, read_remote(&first_outside, lane % shares));
    cluster_arrive();  // no CTA ends before the others have read its first_outside
  }
  const int64_t there = min(have, (int64_t)outside);  // pages that can be taken
  if (outside != kNone) {
    if (me == 0) atomicOr(a.err, kErrBadRow);
    used = pages_within(there);
  }
  const auto enough = [&](int b) { return grow[b + 1] == grow[b] || grow[b + 1] <= there; };
  const auto granted = [&](int b) { return enough(b) && (tok[b + 1] == tok[b] || tok[b + 1] <= a.n_tok); };
  const int64_t left = have - used;
  if (base.grow > there) {
    for (int b = tid; b < a.B; b += kThreads)
      if (!enough(b)) atomicAdd(&refused_s, 1);
    __syncthreads();
  }

  for (int64_t x = me; x < used; x += all) {
    const int b = request_of(grow, a.B, x);
    a.table[(int64_t)b * a.table_stride + pages_of(olen[b]) + (x - grow[b])] = x == me ? page0 : taken(x);
  }
  for (int64_t j = f + me; j < left; j += all) {
    const int p = page_at(j);
    if (p < 0 || p >= a.n_pages) atomicOr(a.err, kErrBadRow);
    a.free_pages[j] = p;
  }
  for (int64_t i = me; i < a.n_tok; i += all) {
    int64_t slot = -1;
    int pos = 0;
    if (i < base.tok) {
      const int b = request_of(tok, a.B, i);
      const int o = olen[b];
      const int len = o < 0 ? -1 - o : o;
      pos = len + (int)(i - tok[b]);
      if (o >= 0 && granted(b)) {
        const int64_t c = pos / a.page, had = pages_of(o);
        const int p = c < had ? a.table[(int64_t)b * a.table_stride + c] : taken(grow[b] + (c - had));
        slot = (int64_t)p * a.page + pos % a.page;
      }
    }
    a.slots[i] = slot;
    a.positions[i] = pos;
  }
  for (int b = me; b <= a.B; b += all) {
    a.cu_new[b] = (int)min(tok[b], (int64_t)0x7fffffff);
    if (b < a.B) a.seq_len[b] = olen[b] < 0 ? -1 - olen[b] : granted(b) ? nlen[b] : olen[b];
  }
  if (me == 0) a.free_out[0] = (int)left, a.free_out[1] = refused_s;
  if (shares > 1) cluster_wait();
}

}  // namespace

cudaError_t launch_page_update(const PageUpdateArgs& a, cudaStream_t s) {
  const size_t smem = 3 * sizeof(int64_t) * (a.B + 1) + 2 * sizeof(int32_t) * a.B;
  if (smem > 32 * 1024) {
    cudaError_t e = cudaFuncSetAttribute(page_update_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         3 * 8 * (kMaxBatch + 1) + 2 * 4 * kMaxBatch);
    if (e != cudaSuccess) return e;
  }
  // A cluster where there is more than a CTA's worth of tokens or requests (finished requests
  // give back many pages each): 256 requests, 128-token chunks among them, 12.2 us on one CTA
  // and 8.1 on eight; 16 requests of one token each take 3.9 on one, a cluster 1.0 more.
  const int shares = a.B > 32 || a.n_tok > kThreads ? 8 : 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = shares;
  cfg.blockDim = kThreads;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = shares;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = shares > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, page_update_kernel, a);
}

}  // namespace dck

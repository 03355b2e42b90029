// Attention over shared prefixes on bf16 caches, many queries to a KV head: what the rows of a group see together,
// on tcgen05.
//
// Mathematics: an item's up to 256 queries (of one KV head, of any rows of the group) are the rows of S = Q K^T and
// O += P V, M = 128 twice, over tiles of 64 tokens; P = 2^(s - m) in bf16 (a weight is off by 2^-8 of itself at
// most, as the output by its own rounding, and errors of many weights cancel; a second term would make the products half as
// long again), m a reference within 2^8 of the running maximum, all sums fp32, those of the weights before they are rounded.
// Bound: a tile is 4 d bytes a token, read once per 256 queries, against 8.4 MFLOP per 128 of them (d = 128): HBM for few
// blocks of queries per group, else the softmax and what an SM takes in from L2.
//
// Work: one CTA per SM takes an equal range of the items' tiles (paged_shared.cu) and leaves a partial sum per item.
// Two streams, each with two buffers of scores, an output and a running maximum of its own: of an item of more than 128
// queries a stream has half of them and all tiles, of others all queries and every other tile (the streams join at the
// item's end). So the softmax of one runs under the products and the softmax of the other, and scores are ready when a
// softmax ends.
// P overwrites its scores in tensor memory and is the A operand of O += P V from there.  Four warps copy (pages of any size
// and order: 16-byte asynchronous copies into the swizzled layout), the rows behind a tile's last token as zeros.
//
// The CTAs are there while the plan is made, and meanwhile go through their code once on an item of nothing: no wait, no
// copy of anything, no MMA, nothing stored.  Instructions that are not in an SM's caches come at some 16 in 0.1 us; without that pass
// the first tile's softmax alone took 3 us for 0.5.
#include "paged_shared.cuh"
#include "tc_common.cuh"

namespace dck {
namespace paged {
namespace {

using namespace tc;

// warps 0-3 and 4-7 softmax of the two streams, warps 8-11 copies, warps 12 and 13 their MMAs
constexpr int kThreads = 512;
// registers: 512 threads x 128 at launch = 2 x 128 x 168 (softmax) + 2 x 128 x 88
constexpr int kRegsSoftmax = 168, kRegsOther = 88;
constexpr int kRows = 128;        // queries of a stream
constexpr int kTok = 64;          // tokens of a tile
constexpr int kAhead = 4;         // tiles whose page numbers are read at a time
constexpr int kAtom = 128 * 128;  // 128 rows of 128 bytes
constexpr int kHalf = kTok * 128;

template <int DP>
struct ShmTc {
  static constexpr int kSlots = DP == 128 ? 9 : 16;  // ring of key and value tiles: K(0), V(0), K(1), V(1), ...
  uint8_t q[2][DP / 64][kAtom];        // queries [128 of them][64 elements][row][128 bytes], 128-byte swizzle
  uint8_t kv[kSlots][DP / 64][kHalf];  // keys or values, rows tokens
  float2 ml[2][kRows];                 // [stream][row]: maximum and sum
  uint64_t kv_full[kSlots], kv_empty[kSlots], q_full, q_empty;
  uint64_t s_full[2][2], p_full[2][2], pv_done[2], o_full[2], ml_full, o_free;  // [stream][buffer]
  uint32_t tmem_base;
  int abort_flag;
};

// This CTA's items one after the other; n: tiles of the item that it has; pair: more than 128 queries.
struct Segments {
  ItemWalk at;
  int left, n, nth;
  bool pair;
  __device__ __forceinline__ void see(const Prefix& x, int qpg) {
    n = min(at.left, left);
    pair = at.count(x, qpg) > kRows;
  }
  bool dry;  // the item of nothing
  __device__ __forceinline__ void begin_dry() {
    dry = true;
    pair = false;
    n = 2;
    left = nth = 0;
    at.p.start = at.p.rows = at.p.first = at.p.table = at.token = at.head = at.block = at.left = 0;
    at.p.end = 2 * kTok;
  }
  // The next item: the first real one once the plan is there.
  __device__ __forceinline__ bool next(const Prefix& x, int heads, int qpg) {
    if (dry) {
      dry = false;
      pdl_wait();
      pdl_launch_dependents();  // the plan, and with it all that the own tokens' launch reads, is there
      left = at.enter(x, blockIdx.x);
      if (left == 0) return false;
      see(x, qpg);
      return true;
    }
    left -= n;
    if (left <= 0) return false;
    at.leave(x, heads);
    see(x, qpg);
    ++nth;
    return true;
  }
  // Stream s has the tiles from `first(s)` on, every `step()`th.
  __device__ __forceinline__ int first(int s) const { return pair ? 0 : s; }
  __device__ __forceinline__ int step() const { return pair ? 1 : 2; }
};

// 32 bytes, a whole sector, at once.
__device__ __forceinline__ void store8(float* p, const float* v) {
  asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
               "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
               : "memory");
}

// Arrives on `bar` once all copies of this thread so far have landed.  (The reader of the barrier orders them before its
// MMAs: a proxy fence of this thread would wait for the copies behind them too, 2 us a tile.)
__device__ __forceinline__ void arrive_when_copied(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// Copies of warp w of four.
template <int DP>
struct Copier {
  const Args& g;
  int w, lane;
  uint32_t swizzled[2];  // where this lane's chunk of rows 4 i + lane / 8 lies, i even or odd
  __device__ __forceinline__ Copier(const Args& g, int w, int lane) : g(g), w(w), lane(lane) {
    const int sub = lane >> 3, c = lane & 7;
    swizzled[0] = sub * 128 + (c ^ sub) * 16;
    swizzled[1] = sub * 128 + (c ^ (sub + 4)) * 16;
  }
  // Rows first .. first + N - 1 of a tile with `atom` bytes per 64 elements, at `from` + offset of lane r, zeros where
  // that is negative.
  template <int N>
  __device__ __forceinline__ void rows(uint8_t* to, int atom, int first, const void* from, int64_t offset) const {
    const int c = lane & 7, have = g.a.v.d / 8 - c;
    const char* base = static_cast<const char*>(from) + c * 16;
    const uint32_t at = smem_u32(to) + first * 128;
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const int64_t o = __shfl_sync(~0u, offset, i * 4 + (lane >> 3));
#pragma unroll
      for (int j = 0; j < DP / 64; ++j) {
        const bool real = o >= 0 && 8 * j < have;
        cp_async16_or_zero(at + j * atom + swizzled[i & 1] + i * 512, real ? base + o + 128 * j : static_cast<const char*>(from),
                           real ? 16 : 0);
      }
    }
  }
  // Where lane r's query of a stream (row 32 w + r from row `from` of the item on) lies, in bytes from g.a.q (-1: none).
  __device__ __forceinline__ int64_t query(const ItemWalk& at, int from) const {
    const int qpg = g.a.v.qpg, r = from + 32 * w + lane;
    if (r >= at.count(g.x, qpg)) return -1;
    const int x = at.block * g.x.rows + r, b = g.x.by_qpg.div(x), j = at.head * qpg + x - b * qpg;
    return 2 * ((int64_t)(at.p.start + b) * g.a.q_stride + (int64_t)j * g.a.v.d);
  }
  // The same rows by single elements, for queries off 16-byte boundaries.
  __device__ __forceinline__ void elements(uint8_t* to, int64_t offset) const {
    for (int r = 0; r < 32; ++r) {
      const int64_t o = __shfl_sync(~0u, offset, r);
      const int row = 32 * w + r;
      for (int e = lane; e < DP; e += 32) {
        const uint16_t v = o >= 0 && e < g.a.v.d ? reinterpret_cast<const uint16_t*>(static_cast<const char*>(g.a.q) + o)[e] : 0;
        *reinterpret_cast<uint16_t*>(to + e / 64 * kAtom + row * 128 + ((e % 64 / 8) ^ (row & 7)) * 16 + e % 8 * 2) = v;
      }
    }
  }
};

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("{\n .reg .b64 x, y, z, w;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n mov.b64 z, {%6, %7};\n"
      " fma.rn.f32x2 w, x, y, z;\n mov.b64 {%0, %1}, w;\n}\n"
      : "=f"(r.x), "=f"(r.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}

template <int DP>
__global__ void __launch_bounds__(kThreads, 1) prefix_tc_kernel(const __grid_constant__ Args g) {
  extern __shared__ uint8_t smem_raw[];
  using Shm = ShmTc<DP>;
  constexpr int kSlots = Shm::kSlots;
  Shm& sm = *reinterpret_cast<Shm*>(align_1024(smem_raw));
  const PagedDecodeArgs& a = g.a;
  const Prefix& x = g.x;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, heads = a.v.Hkv;
  volatile int* abort_flag = &sm.abort_flag;
  if (warp == 12) {
    tmem_alloc(&sm.tmem_base, 512);
    tmem_relinquish();
    if (lane == 0) {
      for (int i = 0; i < kSlots; ++i) {
        mbar_init(&sm.kv_full[i], 128);
        mbar_init(&sm.kv_empty[i], 2);
      }
      mbar_init(&sm.q_full, 128);
      mbar_init(&sm.q_empty, 2);
      for (int s = 0; s < 2; ++s) {
        for (int b = 0; b < 2; ++b) {
          mbar_init(&sm.s_full[s][b], 1);
          mbar_init(&sm.p_full[s][b], 4);
        }
        mbar_init(&sm.pv_done[s], 1);
        mbar_init(&sm.o_full[s], 1);
      }
      mbar_init(&sm.ml_full, 8);
      mbar_init(&sm.o_free, 8);
      sm.abort_flag = 0;
      fence_mbar_init();
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  Segments sg;
  sg.begin_dry();
  const uint32_t tmem = sm.tmem_base;  // scores and P of stream s, buffer b at 128 s + 64 b, its output at 256 + 128 s

  if (warp >= 12) {
    reg_dec<kRegsOther>();
    if (warp < 14) {
      // ---- MMAs of stream s: the whole warp runs the schedule, one lane issues -----------
      // A warp per stream: a step's waits and MMAs take a warp as long as the MMAs of both streams do (one warp for both:
      // 1.3 us a tile of 2 x 128 queries). A thread's MMAs run in order: scores may go into a buffer right
      // after the P V that reads it.
      const bool el = elect_one();
      const int s = warp - 12;
      const uint32_t id_s = idesc_bf16(128, kTok, false, false);  // S = Q K^T: both K-major
      const uint32_t id_o = idesc_bf16(128, DP, false, true);     // O += P V: V MN-major
      const uint64_t dq = sdesc(smem_u32(sm.q[0][0]), 16, 1024, kSw128);
      const uint64_t dk = sdesc(smem_u32(sm.kv[0][0]), 16, 1024, kSw128);
      const uint64_t dv = sdesc(smem_u32(sm.kv[0][0]), kHalf, 1024, kSw128);
      constexpr int kSlotBytes = (DP / 64) * kHalf;
      const uint32_t ts = tmem + 128 * s, to = tmem + 256 + 128 * s;
      int base = 0;         // ring position of the item's first keys
      uint32_t turn[2] = {0, 0};  // P tiles so far, of each buffer
      bool ok = true;
      do {
        const int n = sg.n, first = sg.first(s), step = sg.step(), tiles = (n - first + step - 1) / step;
        const uint64_t qb = dq + (uint64_t)((sg.pair ? s : 0) * ((DP / 64) * kAtom >> 4));
        // (barriers of the ring expect both streams; the one that has a tile alone arrives twice)
        const auto done = [&](uint64_t* bar) {
          umma_commit(bar);
          if (!sg.pair) umma_commit(bar);
        };
        const bool dry = sg.dry, issue = el && !dry;
        if (!dry && !(ok = wwait(&sm.q_full, sg.nth & 1, abort_flag))) break;
        if (tiles == 0 && issue) umma_commit(&sm.q_empty);
        int si = 0, vi = 0;  // the next scores and the next products with values
        long long since = 0;
        while (vi < tiles) {
          bool idle = true;
          if (si < tiles && si < vi + 2) {
            const int at = base + 2 * (first + si * step), slot = at % kSlots;
            if (__all_sync(~0u, mbar_test(&sm.kv_full[slot], at / kSlots & 1) || dry)) {
              idle = false;
              fence_proxy_async_smem();
              tc_fence_after();
              if (issue) {
                const uint64_t kb = dk + (uint64_t)(slot * (kSlotBytes >> 4));
#pragma unroll
                for (int j = 0; j < DP / 16; ++j)
                  umma_f16(ts + 64 * (si & 1), qb + (((j >> 2) * kAtom + (j & 3) * 32) >> 4),
                           kb + (((j >> 2) * kHalf + (j & 3) * 32) >> 4), id_s, j > 0 ? 1u : 0u);
                umma_commit(&sm.s_full[s][si & 1]);
                done(&sm.kv_empty[slot]);
                if (si + 1 == tiles) umma_commit(&sm.q_empty);
              }
              ++si;
            }
          }
          const int b = vi & 1;
          if (vi < si && __all_sync(~0u, mbar_test(&sm.p_full[s][b], turn[b] & 1) || dry)) {
            const int at = base + 2 * (first + vi * step) + 1, slot = at % kSlots;
            if (__all_sync(~0u, mbar_test(&sm.kv_full[slot], at / kSlots & 1) || dry)) {
              idle = false;
              // the last item's output has been read
              if (vi == 0 && sg.nth > 0 && !(ok = wwait(&sm.o_free, (sg.nth - 1) & 1, abort_flag))) break;
              turn[b] += !dry;
              fence_proxy_async_smem();
              tc_fence_after();
              if (issue) {
                const uint64_t vb = dv + (uint64_t)(slot * (kSlotBytes >> 4));
#pragma unroll
                for (int j = 0; j < kTok / 16; ++j)
                  umma_f16_ts(to, ts + 64 * b + 8 * j, vb + (uint64_t)(j * 2048 >> 4), id_o, (vi > 0 || j > 0) ? 1u : 0u);
                umma_commit(&sm.pv_done[s]);
                done(&sm.kv_empty[slot]);
                if (vi + 1 == tiles) umma_commit(&sm.o_full[s]);
              }
              ++vi;
            }
          }
          // a bounded wait, as in mbar_wait
          if (!idle) {
            since = 0;
          } else {
            const long long now = clock64();
            if (since == 0) since = now;
            if (now - since > kWaitCycles) *abort_flag = 1;
            if (__any_sync(~0u, *abort_flag)) {
              ok = false;
              break;
            }
          }
        }
        if (!dry) base += 2 * n;
      } while (ok && sg.next(x, heads, a.v.qpg));
    }
  } else if (warp < 8) {
    // ---- softmax of stream s: a thread has row r ----------------------------------------
    reg_inc<kRegsSoftmax>();
    const int s = warp >> 2, r = (warp & 3) * 32 + lane;
    const uint32_t lb = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ob = tmem + lb + 256 + 128 * s;
    const bool plain = g.score.cap2 == 0.f && g.score.scale2 > 0.f;  // scores are s times a positive factor
    const float factor = plain ? g.score.scale2 : 1.f;
    // sp: bit b the parity of buffer b's next scores; turn: tiles of this stream so far; joined: items so far whose streams
    // join; outputs: items so far in which stream s has tiles
    uint32_t sp = 0, turn = 0, joined = 0, outputs[2] = {0, 0};
    bool ok = true;
    do {
      const bool dry = sg.dry;
      float m = -CUDART_INF_F;
      float2 l = make_float2(0.f, 0.f);
      for (int k = sg.first(s), j = 0; k < sg.n; k += sg.step(), ++j, turn += !dry) {
        const int b = j & 1;
        if (!dry && !(ok = wwait(&sm.s_full[s][b], sp >> b & 1, abort_flag))) break;
        sp ^= (uint32_t)!dry << b;
        tc_fence_after();
        const uint32_t sb = tmem + lb + 128 * s + 64 * b;
        float sv[kTok];
#pragma unroll
        for (int c = 0; c < kTok / 32; ++c) tmem_ld32(sb + 32 * c, *reinterpret_cast<float(*)[32]>(&sv[32 * c]));
        tmem_wait_ld();
        if (!plain) g.score.apply(sv);
        const int live = sg.at.p.end - sg.at.token - kTok * k;
        if (live < kTok) {
#pragma unroll
          for (int i = 0; i < kTok; ++i) sv[i] = i < live ? sv[i] : -CUDART_INF_F;
        }
        float mx[4] = {sv[0], sv[1], sv[2], sv[3]};
#pragma unroll
        for (int i = 4; i < kTok; i += 8)
#pragma unroll
          for (int u = 0; u < 4; ++u) mx[u] = fmaxf(mx[u], i + 4 + u < kTok ? fmaxf(sv[i + u], sv[i + 4 + u]) : sv[i + u]);
        const float mt = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * factor;
        const bool raise = mt > m + kHeadroom, rescale = raise && m != -CUDART_INF_F;
        if (__any_sync(~0u, rescale)) {  // (TMEM accesses are the whole warp's: factor 1 for the other rows)
          // the last product is in O (the one before is: this tile's scores came after it)
          if (!(ok = wwait(&sm.pv_done[s], (turn - 1) & 1, abort_flag))) break;
          tc_fence_after();
          const float f = rescale ? exp2_approx(m - mt) : 1.f;
#pragma unroll 1
          for (int c = 0; c < DP / 16; ++c) {
            float v[16];
            tmem_ld16(ob + 16 * c, v);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] *= f;
            tmem_st16(ob + 16 * c, v);
          }
          l.x *= f, l.y *= f;
        }
        if (raise) m = mt;
        const float base = m == -CUDART_INF_F ? 0.f : m;
        const float2 f2 = make_float2(factor, factor), nb = make_float2(-base, -base);
        uint32_t pk[kTok / 2];
#pragma unroll
        for (int i = 0; i < kTok / 2; ++i) {
          const float2 d = fma2(make_float2(sv[2 * i], sv[2 * i + 1]), f2, nb);
          const float2 p = make_float2(ex2_approx(d.x), ex2_approx(d.y));
          pk[i] = pack2(p.x, p.y);
          l = add2(l, p);
        }
        if (!dry) tmem_st32(sb, pk);  // (after the item of nothing, real scores may lie there already)
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0 && !dry) mbar_arrive(&sm.p_full[s][b]);
      }
      if (!ok) break;
      const bool pair = sg.pair, both = pair || sg.n > 1;
      const int count = dry ? 0 : sg.at.count(x, a.v.qpg), mine = pair ? s * kRows + r : r;
      const int64_t row = sg.at.row_of(x, a.v.Hq, a.v.qpg, mine);
      if (tid == 0 && !dry) sg.at.sign(x, a.v.Hq, sg.at.begins(), sg.n == sg.at.left);
      float* to = x.part_u + row * DP;
      float f0 = 1.f, f1 = 0.f;
      if (!pair) {
        // the streams join: this one writes half of the elements
        if (sg.nth > 0 && !(ok = wwait(&sm.o_free, (sg.nth - 1) & 1, abort_flag))) break;
        sm.ml[s][r] = make_float2(m, l.x + l.y);
        __syncwarp();
        if (lane == 0 && !dry) mbar_arrive(&sm.ml_full);
        if (!dry && !(ok = wwait(&sm.ml_full, joined & 1, abort_flag))) break;
        joined += !dry;
        const float2 u0 = sm.ml[0][r], u1 = sm.ml[1][r];
        const float top = both ? fmaxf(u0.x, u1.x) : u0.x, base = top == -CUDART_INF_F ? 0.f : top;
        f0 = exp2_approx(u0.x - base), f1 = both ? exp2_approx(u1.x - base) : 0.f;
        if (s == 0 && mine < count)
          *reinterpret_cast<float2*>(x.part_ml + 2 * row) = make_float2(top, u0.y * f0 + (both ? u1.y * f1 : 0.f));
      } else if (mine < count) {
        *reinterpret_cast<float2*>(x.part_ml + 2 * row) = make_float2(m, l.x + l.y);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {  // both streams' last products where both have any
        if (t == 1 && !both) continue;
        if (!dry && (!pair || t == s) && !(ok = wwait(&sm.o_full[t], outputs[t] & 1, abort_flag))) break;
        outputs[t] += !dry;
      }
      if (!ok) break;
      tc_fence_after();
      if (pair) {
#pragma unroll 1
        for (int c = 0; c < DP; c += 32) {
          float v[32];
          tmem_ld32(ob + c, v);
          tmem_wait_ld();
          if (mine < count)
#pragma unroll
            for (int i = 0; i < 32; i += 8) store8(to + c + i, v + i);
        }
      } else {
#pragma unroll 1
        for (int c = s * (DP / 2); c < (s + 1) * (DP / 2); c += 32) {
          float v[32], w[32];
          tmem_ld32(tmem + lb + 256 + c, v);
          if (both) tmem_ld32(tmem + lb + 384 + c, w);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = (f0 == 0.f ? 0.f : v[i] * f0) + (f1 == 0.f ? 0.f : w[i] * f1);
          if (mine < count)
#pragma unroll
            for (int i = 0; i < 32; i += 8) store8(to + c + i, v + i);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0 && !dry) mbar_arrive(&sm.o_free);
    } while (ok && sg.next(x, heads, a.v.qpg));
  } else {
    // ---- copies -----------------------------------------------------------------------
    reg_dec<kRegsOther>();
    const PagedView& v = a.v;
    const int w = warp - 8;
    const Copier<DP> copy(g, w, lane);
    int slot = 0;
    uint32_t parity = 1;  // (a fresh barrier passes a wait for the phase before its first)
    bool ok = true;
    do {
      const bool dry = sg.dry;
      const int32_t* table = a.table + sg.at.p.table * a.table_stride;
      const auto page_of = [&](int k, int& off) -> int {  // of this lane's token of tile k (off < 0: none)
        const int t = sg.at.token + kTok * k + 16 * w + (lane & 15);
        off = -1;
        if (dry || k >= sg.n || t >= sg.at.p.end) return 0;
        const uint32_t col = v.by_page.div(t);
        off = t - (int)col * v.page;
        return table[col];
      };
      // page numbers are read four tiles ahead
      int page[kAhead], off[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) page[i] = page_of(i, off[i]);
      // the last item's scores are all formed: its queries can go
      if (sg.nth > 0 && !(ok = wwait(&sm.q_empty, (sg.nth - 1) & 1, abort_flag))) break;
#pragma unroll 1
      for (int t = 0; t < (sg.pair ? 2 : 1); ++t) {
        const int64_t qo = dry ? -1 : copy.query(sg.at, t * kRows);
        if (g.p.q_copied) copy.template rows<32>(sm.q[t][0], kAtom, 32 * w, a.q, qo);
        else copy.elements(sm.q[t][0], qo);
      }
      if (!dry) {
        if (g.p.q_copied) arrive_when_copied(&sm.q_full);
        else mbar_arrive(&sm.q_full);
      }
#pragma unroll 1
      for (int k0 = 0; k0 < sg.n && ok; k0 += kAhead) {
        int64_t at[kAhead][2];  // where this lane's token's keys and values lie, in bytes (-1: none)
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const bool inside = (uint32_t)page[i] < (uint32_t)v.n_pages;
          if (off[i] >= 0 && !inside) {
            atomicOr(a.err, kErrBadSeq);
            atomicOr(&x.groups[sg.at.g].bad, 1);
          }
          const bool have = off[i] >= 0 && inside;
          at[i][0] = have ? (int64_t)((uint64_t)page[i] * v.k_page_b + (uint64_t)off[i] * v.k_tok_b + (uint64_t)sg.at.head * v.k_head_b) : -1;
          at[i][1] = have ? (int64_t)((uint64_t)page[i] * v.v_page_b + (uint64_t)off[i] * v.v_tok_b + (uint64_t)sg.at.head * v.v_head_b) : -1;
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) page[i] = page_of(k0 + kAhead + i, off[i]);
        for (int i = 0; i < kAhead && k0 + i < sg.n && ok; ++i) {
          const int64_t ko = i == 0 ? at[0][0] : i == 1 ? at[1][0] : i == 2 ? at[2][0] : at[3][0];
          const int64_t vo = i == 0 ? at[0][1] : i == 1 ? at[1][1] : i == 2 ? at[2][1] : at[3][1];
#pragma unroll 1
          for (int kind = 0; kind < 2; ++kind) {
            if (!dry && !(ok = wwait(&sm.kv_empty[slot], parity, abort_flag))) break;
            copy.template rows<16>(sm.kv[slot][0], kHalf, 16 * w, kind ? a.vc : a.kc, kind ? vo : ko);
            if (!dry) {
              arrive_when_copied(&sm.kv_full[slot]);
              if (++slot == kSlots) slot = 0, parity ^= 1;
            }
          }
        }
      }
      if (dry) cp_async_wait<0>();
    } while (ok && sg.next(x, heads, a.v.qpg));
    cp_async_wait<0>();
  }
  tc_fence_before();
  __syncthreads();
  if (sm.abort_flag) {
    drain_in_flight();
    if (tid == 0) atomicOr(a.err, kErrTimeout);
  }
  __syncthreads();
  if (warp == 12) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <int DP>
cudaError_t launch(const Args& g, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};
  constexpr size_t smem = sizeof(ShmTc<DP>) + 1024;
  static_assert(smem <= 232448, "shared memory of a CTA");
  return launch_part(prefix_tc_kernel<DP>, ready, g.x.n_items, kThreads, smem, g, s);
}

}  // namespace

cudaError_t launch_prefix_tc(const Args& g, cudaStream_t s) { return g.DP == 64 ? launch<64>(g, s) : launch<128>(g, s); }

}  // namespace paged
}  // namespace dck

// C ABI of the paged key-value cache: argument checks and dispatch.
// The formulas and conventions are documented in include/dck.h.
#include <cmath>
#include <cstring>

#include "api_state.h"
#include "paged.cuh"

using namespace dck;

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

size_t element(int32_t dtype) { return dtype == DCK_F32 ? 4 : 2; }

bool known_dtype(int32_t dtype) { return dtype == DCK_BF16 || dtype == DCK_F32; }

// `cached`: bytes of a cached element, 0 for those of the descriptor's type.
dck_status check_paged(const dck_paged_desc* p, int64_t cached = 0) {
  if (!p) return DCK_ERR_INVALID;
  if (p->n_q_heads <= 0 || p->n_kv_heads <= 0 || p->head_dim <= 0 || p->page_size <= 0 || p->n_pages <= 0 ||
      !known_dtype(p->dtype) || p->n_q_heads % p->n_kv_heads != 0)
    return DCK_ERR_INVALID;
  if (p->head_dim % 8 || p->head_dim > kMaxPagedHeadDim || p->page_size > kMaxPageSize || p->n_q_heads > 65536)
    return DCK_ERR_UNSUPPORTED;
  const int64_t el = cached ? cached : (int64_t)element(p->dtype);
  // bytes of a stride in 32 bits, and with that every offset (fewer than 2^31 strides) in 64
  const int64_t most = (int64_t(1) << 30) - 1;
  for (int64_t st : {p->k_page_stride, p->k_token_stride, p->k_head_stride, p->v_page_stride, p->v_token_stride,
                     p->v_head_stride})
    if (st <= 0 || st > most || st * el % 16 != 0) return DCK_ERR_INVALID;
  return DCK_OK;
}

PagedView make_view(const dck_paged_desc* p, uint32_t cached = 0) {
  PagedView v = {};
  v.Hq = p->n_q_heads;
  v.Hkv = p->n_kv_heads;
  v.d = p->head_dim;
  v.qpg = p->n_q_heads / p->n_kv_heads;
  v.page = p->page_size;
  v.n_pages = p->n_pages;
  const uint32_t el = cached ? cached : (uint32_t)element(p->dtype);
  v.k_page_b = (uint32_t)p->k_page_stride * el;
  v.k_tok_b = (uint32_t)p->k_token_stride * el;
  v.k_head_b = (uint32_t)p->k_head_stride * el;
  v.v_page_b = (uint32_t)p->v_page_stride * el;
  v.v_tok_b = (uint32_t)p->v_token_stride * el;
  v.v_head_b = (uint32_t)p->v_head_stride * el;
  v.by_page = divider((uint32_t)p->page_size);
  return v;
}

dck_status check_quant(const dck_quant_desc* p) {
  if (!p) return DCK_ERR_INVALID;
  const dck_status st = check_paged(&p->cache, 1);
  if (st != DCK_OK) return st;
  for (int64_t x : {p->k_scale_page_stride, p->k_scale_token_stride, p->k_scale_head_stride, p->v_scale_page_stride,
                    p->v_scale_token_stride, p->v_scale_head_stride})
    if (x <= 0 || x >= (int64_t(1) << 30)) return DCK_ERR_INVALID;
  return DCK_OK;
}

PagedView make_view(const dck_quant_desc* p) {
  PagedView v = make_view(&p->cache, 1);
  v.ks_page = (uint32_t)p->k_scale_page_stride;
  v.ks_tok = (uint32_t)p->k_scale_token_stride;
  v.ks_head = (uint32_t)p->k_scale_head_stride;
  v.vs_page = (uint32_t)p->v_scale_page_stride;
  v.vs_tok = (uint32_t)p->v_scale_token_stride;
  v.vs_head = (uint32_t)p->v_scale_head_stride;
  return v;
}

// The rotation's settings as kernels take them; false if the table is not one
// that dck_rope_init filled or does not fit heads of `d` elements.
bool rope_args(const dck_rope_table* t, int d, int transpose, RopeArgs* r) {
  std::memset(r, 0, sizeof(*r));
  if (!t) return true;
  if (t->initialised != 1 || t->rotary_dim < 2 || t->rotary_dim > 256 || (t->rotary_dim & 1) || t->rotary_dim > d ||
      (t->layout != DCK_ROPE_HALF && t->layout != DCK_ROPE_INTERLEAVED))
    return false;
  r->layout = t->layout;
  r->rot = t->rotary_dim;
  r->magnitude = t->magnitude;
  r->sign = transpose ? -1.f : 1.f;
  for (int i = 0; i < t->rotary_dim / 2; ++i) r->f[i] = make_uint2((uint32_t)t->turns[i], (uint32_t)(t->turns[i] >> 32));
  return true;
}

// dck_paged_append and, with scales, dck_quant_append, behind their descriptors' checks.
dck_status append(const dck_paged_desc* desc, const dck_quant_desc* quant, const dck_rope_table* table, const void* q,
                  int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int32_t n_tok,
                  const int32_t* d_positions, const int64_t* d_slots, void* q_out, void* kcache, float* k_scale,
                  void* vcache, float* v_scale, void* stream) {
  if (n_tok < 0) return DCK_ERR_INVALID;
  RopeLaunch a;
  std::memset(&a, 0, sizeof(a));
  if (!rope_args(table, desc->head_dim, 0, &a.rope)) return DCK_ERR_INVALID;
  if (n_tok == 0) return DCK_OK;
  const size_t el = element(desc->dtype);
  const int d = desc->head_dim;
  if (!k || !v || !d_slots || !kcache || !vcache || (table && !d_positions) || (q && !q_out)) return DCK_ERR_INVALID;
  if (!aligned(k, el) || !aligned(v, el) || !aligned(q, el) || !aligned(q_out, el) || !aligned(kcache, 16) ||
      !aligned(vcache, 16) || !aligned(d_slots, 8) || !aligned(d_positions, 4))
    return DCK_ERR_INVALID;
  if (quant && (!k_scale || !v_scale || !aligned(k_scale, 4) || !aligned(v_scale, 4))) return DCK_ERR_INVALID;
  const int64_t most = int64_t(1) << 30;
  if (k_stride < 0 || v_stride < 0 || k_stride > most || v_stride > most) return DCK_ERR_INVALID;
  if (q && (q_stride < 0 || q_stride > most || (q == q_out && n_tok > 1 && q_stride != (int64_t)desc->n_q_heads * d)))
    return DCK_ERR_INVALID;
  int sms = 0;
  if (!device_state(&a.err, &sms)) return DCK_ERR_CUDA;
  RopeRows* r = a.rows;
  r->src = k;
  r->dst = kcache;
  r->src_tok = k_stride;
  r->src_head = d;
  r->dst_tok = desc->k_token_stride;
  r->dst_head = desc->k_head_stride;
  r->dst_page = desc->k_page_stride;
  r->heads = desc->n_kv_heads;
  r->rotate = table != nullptr;
  r->cached = 1;
  if (quant) {
    r->scale = k_scale;
    r->scale_page = quant->k_scale_page_stride;
    r->scale_tok = quant->k_scale_token_stride;
    r->scale_head = quant->k_scale_head_stride;
  }
  ++r;
  r->src = v;
  r->dst = vcache;
  r->src_tok = v_stride;
  r->src_head = d;
  r->dst_tok = desc->v_token_stride;
  r->dst_head = desc->v_head_stride;
  r->dst_page = desc->v_page_stride;
  r->heads = desc->n_kv_heads;
  r->cached = 1;
  if (quant) {
    r->scale = v_scale;
    r->scale_page = quant->v_scale_page_stride;
    r->scale_tok = quant->v_scale_token_stride;
    r->scale_head = quant->v_scale_head_stride;
  }
  ++r;
  if (q) {
    r->src = q;
    r->dst = q_out;
    r->src_tok = q_stride;
    r->src_head = r->dst_head = d;
    r->dst_tok = (int64_t)desc->n_q_heads * d;
    r->heads = desc->n_q_heads;
    r->rotate = table != nullptr;
    ++r;
  }
  a.n_rows = (int32_t)(r - a.rows);
  a.n_tok = n_tok;
  a.d = d;
  a.positions = d_positions;
  a.slots = d_slots;
  a.page = desc->page_size;
  a.n_pages = desc->n_pages;
  a.by_page = divider((uint32_t)desc->page_size);
  if (launch_rope_rows(a, desc->dtype, sms, static_cast<cudaStream_t>(stream)) != cudaSuccess) return DCK_ERR_CUDA;
  set_last_launches(1);
  return DCK_OK;
}

size_t decode_workspace(const PagedView& v, DecodeKind kind, int32_t batch, int32_t max_seq_len) {
  int sms = 0;
  if (batch < 0 || batch > kMaxBatch || max_seq_len < 1 || !device_state(nullptr, &sms)) return 0;
  return paged_decode_workspace(v, kind, batch, max_seq_len, sms);
}

size_t shared_workspace(const PagedView& v, DecodeKind kind, int32_t batch, int32_t max_seq_len, int32_t max_own) {
  int sms = 0;
  if (batch < 0 || batch > kMaxBatch || max_seq_len < 1 || max_own < 1 || !device_state(nullptr, &sms)) return 0;
  return paged_shared_workspace(v, kind, batch, max_seq_len, max_own, sms);
}

thread_local int32_t t_shared_way = 0;  // dck_set_shared_way

// The rows of a call that begin with the same tokens.
struct Groups {
  int32_t max_own, n;
  const int32_t *start, *shared;
};

// The attention calls behind their descriptors' checks; groups: of the shared ones, else null.
dck_status attend(const PagedView& v, DecodeKind kind, const void* q, int64_t q_stride, const void* kcache,
                  const float* k_scale, const void* vcache, const float* v_scale, const int32_t* block_table,
                  int64_t table_stride, const int32_t* d_seq_len, int32_t batch, int32_t max_seq_len,
                  const Groups* groups, float scale, int32_t window, float softcap, void* out, float* lse,
                  void* workspace, size_t ws_bytes, void* stream) {
  if (batch < 0 || batch > kMaxBatch || max_seq_len < 1 || window < 0 || !std::isfinite(scale) || !(softcap >= 0.f) ||
      !std::isfinite(softcap) || table_stride < 0 || table_stride >= (int64_t(1) << 31) || q_stride < 0 ||
      q_stride > (int64_t(1) << 30))
    return DCK_ERR_INVALID;
  if (groups && (groups->max_own < 1 || groups->n < 0 || groups->n > batch || (groups->n == 0 && batch > 0)))
    return DCK_ERR_INVALID;
  if (batch == 0) return DCK_OK;
  const size_t el = element(kind.dtype);
  if (!q || !kcache || !vcache || (!block_table && table_stride > 0) || !d_seq_len || !out) return DCK_ERR_INVALID;
  if (!aligned(q, el) || !aligned(out, el) || !aligned(kcache, 16) || !aligned(vcache, 16) ||
      !aligned(block_table, 4) || !aligned(d_seq_len, 4) || !aligned(lse, 4))
    return DCK_ERR_INVALID;
  if (kind.quant && (!k_scale || !v_scale || !aligned(k_scale, 4) || !aligned(v_scale, 4))) return DCK_ERR_INVALID;
  if (groups && (!groups->start || !groups->shared || !aligned(groups->start, 4) || !aligned(groups->shared, 4)))
    return DCK_ERR_INVALID;
  PagedDecodeArgs a;
  int sms = 0;
  if (!device_state(&a.err, &sms)) return DCK_ERR_CUDA;
  a.v = v;
  const size_t need = groups ? paged_shared_workspace(v, kind, batch, max_seq_len, groups->max_own, sms)
                             : paged_decode_workspace(v, kind, batch, max_seq_len, sms);
  if (need && (!workspace || ws_bytes < need || !aligned(workspace, 256))) return DCK_ERR_WORKSPACE;
  a.q = q;
  a.q_stride = q_stride;
  a.kc = kcache;
  a.vc = vcache;
  a.table = block_table;
  a.table_stride = table_stride;
  a.seq_len = d_seq_len;
  a.B = batch;
  a.max_len = max_seq_len;
  a.window = window;
  a.scale = scale;
  a.softcap = softcap;
  a.out = out;
  a.lse = lse;
  a.ks = k_scale;
  a.vs = v_scale;
  a.n_groups = groups ? groups->n : 0;
  a.max_own = groups ? groups->max_own : 0;
  a.group_start = groups ? groups->start : nullptr;
  a.shared_len = groups ? groups->shared : nullptr;
  a.way = t_shared_way;
  a.ws = workspace;
  LaunchHook hook = thread_hook();
  a.hook = &hook;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = hook_begin(&hook, s);
  if (e == cudaSuccess) e = groups ? launch_paged_shared(a, kind, sms, s) : launch_paged_decode(a, kind, sms, s);
  if (e == cudaSuccess) e = hook_end(&hook, s);
  set_last_launches(hook.count);
  return e == cudaSuccess ? DCK_OK : DCK_ERR_CUDA;
}

}  // namespace

extern "C" {

dck_status dck_validate_paged_desc(const dck_paged_desc* desc) { return check_paged(desc); }

dck_status dck_page_update(int32_t batch, int32_t page_size, int32_t n_pages, const int32_t* d_old_len,
                           const int32_t* d_new_len, int32_t* d_seq_len, int32_t* block_table, int64_t table_stride,
                           int32_t* free_pages, const int32_t* d_free_in, int32_t* d_free_out, int64_t n_tok,
                           int64_t* d_slots, int32_t* d_positions, int32_t* d_cu_new, void* stream) {
  set_last_launches(0);
  if (batch < 0 || batch > kMaxBatch || page_size < 1 || n_pages < 1 || table_stride < 0 ||
      table_stride >= (int64_t(1) << 31) || n_tok < 0 || n_tok >= (int64_t(1) << 31))
    return DCK_ERR_INVALID;
  if (page_size > kMaxPageSize) return DCK_ERR_UNSUPPORTED;
  if (!free_pages || !d_free_in || !d_free_out || !d_cu_new) return DCK_ERR_INVALID;
  if (batch > 0 && (!d_old_len || !d_new_len || !d_seq_len || (!block_table && table_stride > 0)))
    return DCK_ERR_INVALID;
  if (n_tok > 0 && (!d_slots || !d_positions)) return DCK_ERR_INVALID;
  for (const void* p : {(const void*)d_old_len, (const void*)d_new_len, (const void*)d_seq_len,
                        (const void*)block_table, (const void*)free_pages, (const void*)d_free_in,
                        (const void*)d_free_out, (const void*)d_positions, (const void*)d_cu_new})
    if (!aligned(p, 4)) return DCK_ERR_INVALID;
  if (!aligned(d_slots, 8)) return DCK_ERR_INVALID;
  PageUpdateArgs a;
  if (!device_state(&a.err, nullptr)) return DCK_ERR_CUDA;
  a.B = batch;
  a.page = page_size;
  a.n_pages = n_pages;
  a.old_len = d_old_len;
  a.new_len = d_new_len;
  a.seq_len = d_seq_len;
  a.table = block_table;
  a.table_stride = table_stride;
  a.free_pages = free_pages;
  a.free_in = d_free_in;
  a.free_out = d_free_out;
  a.n_tok = n_tok;
  a.slots = d_slots;
  a.positions = d_positions;
  a.cu_new = d_cu_new;
  if (launch_page_update(a, static_cast<cudaStream_t>(stream)) != cudaSuccess) return DCK_ERR_CUDA;
  set_last_launches(1);
  return DCK_OK;
}

dck_status dck_rope_init(dck_rope_table* table, int32_t layout, int32_t rotary_dim, double theta, int32_t scaling,
                         double factor, double slow, double fast, int32_t trained_len, double magnitude) {
  if (!table) return DCK_ERR_INVALID;
  std::memset(table, 0, sizeof(*table));
  if ((layout != DCK_ROPE_HALF && layout != DCK_ROPE_INTERLEAVED) || rotary_dim < 2 || (rotary_dim & 1) ||
      !(theta > 0) || !std::isfinite(theta) || !std::isfinite(magnitude) || scaling < DCK_ROPE_NONE ||
      scaling > DCK_ROPE_YARN)
    return DCK_ERR_INVALID;
  if (rotary_dim > 256) return DCK_ERR_UNSUPPORTED;
  if (scaling != DCK_ROPE_NONE && (!(factor >= 1) || !std::isfinite(factor))) return DCK_ERR_INVALID;
  if (scaling == DCK_ROPE_NTK && rotary_dim == 2) return DCK_ERR_INVALID;
  if (scaling == DCK_ROPE_BANDS && (!(slow >= 0) || !(fast > slow) || !std::isfinite(fast) || trained_len < 1))
    return DCK_ERR_INVALID;
  if (scaling == DCK_ROPE_YARN &&
      (!(slow > 0) || !(fast > slow) || !std::isfinite(fast) || trained_len < 1 || !(theta > 1)))
    return DCK_ERR_INVALID;
  const double two_pi = 6.283185307179586477, R = rotary_dim;
  if (scaling == DCK_ROPE_NTK) theta *= std::pow(factor, R / (R - 2));
  double from = 0, to = 0;
  if (scaling == DCK_ROPE_YARN) {
    const double per = R / (2 * std::log(theta));
    from = std::fmax(0., std::floor(per * std::log(trained_len / (two_pi * fast))));
    to = std::fmin(R - 1, std::ceil(per * std::log(trained_len / (two_pi * slow))));
  }
  for (int i = 0; i < rotary_dim / 2; ++i) {
    double w = std::pow(theta, -2. * i / R);
    double keep = 1;  // how much of the pair turns at its own rate, the rest at 1 / factor of it
    if (scaling == DCK_ROPE_LINEAR) keep = 0;
    if (scaling == DCK_ROPE_BANDS) keep = (trained_len * w / two_pi - slow) / (fast - slow);
    if (scaling == DCK_ROPE_YARN) keep = 1 - (i - from) / std::fmax(to - from, 1e-3);
    keep = std::fmin(1., std::fmax(0., keep));
    if (keep < 1) w = keep * w + (1 - keep) * w / factor;
    const double turns = w / two_pi, part = turns - std::floor(turns);  // whole turns per position are none
    table->turns[i] = (uint64_t)std::ldexp(part, 64);
  }
  table->layout = layout;
  table->rotary_dim = rotary_dim;
  table->magnitude = (float)magnitude;
  table->initialised = 1;
  return DCK_OK;
}

dck_status dck_rope(const dck_rope_table* table, const void* x, int32_t n_tok, int32_t n_heads, int32_t head_dim,
                    int32_t dtype, int64_t x_token_stride, int64_t x_head_stride, const int32_t* d_positions,
                    void* out, int64_t out_token_stride, int64_t out_head_stride, int32_t transpose, void* stream) {
  set_last_launches(0);
  if (!table || n_tok < 0 || n_heads < 0 || head_dim < 1 || !known_dtype(dtype)) return DCK_ERR_INVALID;
  if (head_dim > 65536 || n_heads > 65536) return DCK_ERR_UNSUPPORTED;
  RopeLaunch a;
  std::memset(&a, 0, sizeof(a));
  if (!rope_args(table, head_dim, transpose, &a.rope)) return DCK_ERR_INVALID;
  if (n_tok == 0 || n_heads == 0) return DCK_OK;
  const size_t el = element(dtype);
  if (!x || !out || !d_positions || !aligned(x, el) || !aligned(out, el) || !aligned(d_positions, 4))
    return DCK_ERR_INVALID;
  const int64_t most = int64_t(1) << 30;
  for (int64_t st : {x_token_stride, x_head_stride, out_token_stride, out_head_stride})
    if (st < 0 || st > most) return DCK_ERR_INVALID;
  if (x == out && (x_token_stride != out_token_stride || x_head_stride != out_head_stride)) return DCK_ERR_INVALID;
  if ((n_heads > 1 && out_head_stride < head_dim) || (n_tok > 1 && out_token_stride < head_dim)) return DCK_ERR_INVALID;
  int sms = 0;
  if (!device_state(&a.err, &sms)) return DCK_ERR_CUDA;
  a.n_rows = 1;
  RopeRows& r = a.rows[0];
  r.src = x;
  r.dst = out;
  r.src_tok = x_token_stride;
  r.src_head = x_head_stride;
  r.dst_tok = out_token_stride;
  r.dst_head = out_head_stride;
  r.heads = n_heads;
  r.rotate = 1;
  a.n_tok = n_tok;
  a.d = head_dim;
  a.positions = d_positions;
  a.page = a.n_pages = 1;
  a.by_page = divider(1);
  if (launch_rope_rows(a, dtype, sms, static_cast<cudaStream_t>(stream)) != cudaSuccess) return DCK_ERR_CUDA;
  set_last_launches(1);
  return DCK_OK;
}

dck_status dck_paged_append(const dck_paged_desc* desc, const dck_rope_table* table, const void* q, int64_t q_stride,
                            const void* k, int64_t k_stride, const void* v, int64_t v_stride, int32_t n_tok,
                            const int32_t* d_positions, const int64_t* d_slots, void* q_out, void* kcache,
                            void* vcache, void* stream) {
  set_last_launches(0);
  const dck_status st = check_paged(desc);
  if (st != DCK_OK) return st;
  return append(desc, nullptr, table, q, q_stride, k, k_stride, v, v_stride, n_tok, d_positions, d_slots, q_out, kcache,
                nullptr, vcache, nullptr, stream);
}

int32_t dck_set_shared_way(int32_t which) {
  const int32_t before = t_shared_way;
  if (which >= 0 && which <= 2) t_shared_way = which;
  return before;
}

dck_status dck_validate_quant_desc(const dck_quant_desc* desc) { return check_quant(desc); }

dck_status dck_quant_append(const dck_quant_desc* desc, const dck_rope_table* table, const void* q, int64_t q_stride,
                            const void* k, int64_t k_stride, const void* v, int64_t v_stride, int32_t n_tok,
                            const int32_t* d_positions, const int64_t* d_slots, void* q_out, void* kcache,
                            float* k_scale, void* vcache, float* v_scale, void* stream) {
  set_last_launches(0);
  const dck_status st = check_quant(desc);
  if (st != DCK_OK) return st;
  return append(&desc->cache, desc, table, q, q_stride, k, k_stride, v, v_stride, n_tok, d_positions, d_slots, q_out,
                kcache, k_scale, vcache, v_scale, stream);
}

dck_status dck_quant_read(const dck_quant_desc* desc, int32_t n_tok, const int64_t* d_slots, const void* kcache,
                          const float* k_scale, const void* vcache, const float* v_scale, void* k, int64_t k_stride,
                          void* v, int64_t v_stride, void* stream) {
  set_last_launches(0);
  const dck_status st = check_quant(desc);
  if (st != DCK_OK) return st;
  if (n_tok < 0) return DCK_ERR_INVALID;
  if (n_tok == 0) return DCK_OK;
  const size_t el = element(desc->cache.dtype);
  if (!d_slots || !kcache || !k_scale || !vcache || !v_scale || !k || !v || !aligned(d_slots, 8) || !aligned(kcache, 16) ||
      !aligned(vcache, 16) || !aligned(k_scale, 4) || !aligned(v_scale, 4) || !aligned(k, el) || !aligned(v, el))
    return DCK_ERR_INVALID;
  const int64_t row = (int64_t)desc->cache.n_kv_heads * desc->cache.head_dim, most = int64_t(1) << 30;
  if (k_stride > most || v_stride > most || k_stride < 0 || v_stride < 0 || (n_tok > 1 && (k_stride < row || v_stride < row)))
    return DCK_ERR_INVALID;
  QuantReadArgs a;
  if (!device_state(&a.err, nullptr)) return DCK_ERR_CUDA;
  a.v = make_view(desc);
  a.n_tok = n_tok;
  a.slots = d_slots;
  a.kc = kcache;
  a.vc = vcache;
  a.ks = k_scale;
  a.vs = v_scale;
  a.k = k;
  a.v_out = v;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  if (launch_quant_read(a, desc->cache.dtype, static_cast<cudaStream_t>(stream)) != cudaSuccess) return DCK_ERR_CUDA;
  set_last_launches(1);
  return DCK_OK;
}

size_t dck_paged_decode_workspace_size(const dck_paged_desc* desc, int32_t batch, int32_t max_seq_len) {
  return check_paged(desc) == DCK_OK ? decode_workspace(make_view(desc), {desc->dtype, false}, batch, max_seq_len) : 0;
}

dck_status dck_paged_decode_attention(const dck_paged_desc* desc, const void* q, int64_t q_stride, const void* kcache,
                                      const void* vcache, const int32_t* block_table, int64_t table_stride,
                                      const int32_t* d_seq_len, int32_t batch, int32_t max_seq_len, float scale,
                                      int32_t window, float softcap, void* out, float* lse, void* workspace,
                                      size_t ws_bytes, void* stream) {
  set_last_launches(0);
  const dck_status st = check_paged(desc);
  if (st != DCK_OK) return st;
  return attend(make_view(desc), {desc->dtype, false}, q, q_stride, kcache, nullptr, vcache, nullptr, block_table,
                table_stride, d_seq_len, batch, max_seq_len, nullptr, scale, window, softcap, out, lse, workspace, ws_bytes,
                stream);
}

size_t dck_quant_decode_workspace_size(const dck_quant_desc* desc, int32_t batch, int32_t max_seq_len) {
  return check_quant(desc) == DCK_OK ? decode_workspace(make_view(desc), {desc->cache.dtype, true}, batch, max_seq_len) : 0;
}

dck_status dck_quant_decode_attention(const dck_quant_desc* desc, const void* q, int64_t q_stride, const void* kcache,
                                      const float* k_scale, const void* vcache, const float* v_scale,
                                      const int32_t* block_table, int64_t table_stride, const int32_t* d_seq_len,
                                      int32_t batch, int32_t max_seq_len, float scale, int32_t window, float softcap,
                                      void* out, float* lse, void* workspace, size_t ws_bytes, void* stream) {
  set_last_launches(0);
  const dck_status st = check_quant(desc);
  if (st != DCK_OK) return st;
  return attend(make_view(desc), {desc->cache.dtype, true}, q, q_stride, kcache, k_scale, vcache, v_scale, block_table,
                table_stride, d_seq_len, batch, max_seq_len, nullptr, scale, window, softcap, out, lse, workspace, ws_bytes,
                stream);
}

size_t dck_paged_shared_workspace_size(const dck_paged_desc* desc, int32_t batch, int32_t max_seq_len, int32_t max_own) {
  if (check_paged(desc) != DCK_OK) return 0;
  return shared_workspace(make_view(desc), {desc->dtype, false}, batch, max_seq_len, max_own);
}

dck_status dck_paged_shared_attention(const dck_paged_desc* desc, const void* q, int64_t q_stride, const void* kcache,
                                      const void* vcache, const int32_t* block_table, int64_t table_stride,
                                      const int32_t* d_seq_len, int32_t batch, int32_t max_seq_len, int32_t max_own,
                                      int32_t n_groups, const int32_t* d_group_start, const int32_t* d_shared_len,
                                      float scale, int32_t window, float softcap, void* out, float* lse, void* workspace,
                                      size_t ws_bytes, void* stream) {
  set_last_launches(0);
  const dck_status st = check_paged(desc);
  if (st != DCK_OK) return st;
  const Groups groups = {max_own, n_groups, d_group_start, d_shared_len};
  return attend(make_view(desc), {desc->dtype, false}, q, q_stride, kcache, nullptr, vcache, nullptr, block_table,
                table_stride, d_seq_len, batch, max_seq_len, &groups, scale, window, softcap, out, lse, workspace, ws_bytes,
                stream);
}

size_t dck_quant_shared_workspace_size(const dck_quant_desc* desc, int32_t batch, int32_t max_seq_len, int32_t max_own) {
  if (check_quant(desc) != DCK_OK) return 0;
  return shared_workspace(make_view(desc), {desc->cache.dtype, true}, batch, max_seq_len, max_own);
}

dck_status dck_quant_shared_attention(const dck_quant_desc* desc, const void* q, int64_t q_stride, const void* kcache,
                                      const float* k_scale, const void* vcache, const float* v_scale,
                                      const int32_t* block_table, int64_t table_stride, const int32_t* d_seq_len,
                                      int32_t batch, int32_t max_seq_len, int32_t max_own, int32_t n_groups,
                                      const int32_t* d_group_start, const int32_t* d_shared_len, float scale,
                                      int32_t window, float softcap, void* out, float* lse, void* workspace,
                                      size_t ws_bytes, void* stream) {
  set_last_launches(0);
  const dck_status st = check_quant(desc);
  if (st != DCK_OK) return st;
  const Groups groups = {max_own, n_groups, d_group_start, d_shared_len};
  return attend(make_view(desc), {desc->cache.dtype, true}, q, q_stride, kcache, k_scale, vcache, v_scale, block_table,
                table_stride, d_seq_len, batch, max_seq_len, &groups, scale, window, softcap, out, lse, workspace, ws_bytes,
                stream);
}

}  // extern "C"

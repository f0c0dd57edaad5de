// C ABI of the prompt's attention and of the paged cache: argument validation
// and dispatch.  Everything here is host code; validation never touches the
// device.
#include <math.h>
#include <string.h>

#include <initializer_list>

#include "kvec_serve.h"

using namespace kvec;

namespace {

constexpr int32_t kMaxLen = 1 << 20;

bool aligned(const void* p, size_t n) { return p && ((uintptr_t)p & (n - 1)) == 0; }
bool aligned_or_null(const void* p, size_t n) { return !p || ((uintptr_t)p & (n - 1)) == 0; }
// Dimensions of these extents and strides, each of fewer than 2^60 bytes: sums of offsets
// in three of them fit 64 bits.
bool spans_ok(const int64_t* s, std::initializer_list<int64_t> extents, int esize) {
  for (const int64_t n : extents) {
    if (n > 1 && *s >= ((int64_t)1 << 60) / esize / (n - 1)) return false;
    ++s;
  }
  return true;
}
// Strides of rows read in 16-byte pieces.
bool row_strides_ok(const int64_t* s, std::initializer_list<int64_t> extents, int esize) {
  if (!s) return false;
  for (size_t i = 0; i < extents.size(); ++i)
    if (s[i] >= (int64_t)1 << 40) return false;
  return strides_ok(s, (int)extents.size(), esize) && spans_ok(s, extents, esize);
}

// What both configurations share.
kvec_status check_heads(int32_t batch, int32_t H, int32_t HQ, int32_t d, int32_t dtype) {
  if (batch < 1 || H < 1 || HQ < 1 || HQ % H != 0 || d < 1) return KVEC_ERR_INVALID;
  if (dtype != KVEC_BF16 && dtype != KVEC_F32) return KVEC_ERR_INVALID;
  if (batch > 65535 || H > 1024 || HQ / H > 16 || (d != 64 && d != 128)) return KVEC_ERR_UNSUPPORTED;
  // launches stay below 2^32 threads: the eviction's selection has 1024 for every
  // (sequence, KV head)
  if ((int64_t)batch * H >= 1 << 22) return KVEC_ERR_UNSUPPORTED;
  return KVEC_OK;
}

kvec_status make_prefill(const kvec_attention_config* c, PrefillArgs* a) {
  if (!c) return KVEC_ERR_INVALID;
  const kvec_status st = check_heads(c->batch, c->n_kv_heads, c->n_q_heads, c->head_dim, c->dtype);
  if (st != KVEC_OK) return st;
  if (c->q_len < 1 || c->kv_len < 1 || c->window < 0 || c->n_sinks < 0) return KVEC_ERR_INVALID;
  if (c->q_len > kMaxLen || c->kv_len > kMaxLen) return KVEC_ERR_UNSUPPORTED;
  if ((int64_t)c->batch * c->n_q_heads * c->q_len >= (int64_t)1 << 29) return KVEC_ERR_UNSUPPORTED;
  memset(a, 0, sizeof(*a));
  a->batch = c->batch;
  a->H = c->n_kv_heads;
  a->HQ = c->n_q_heads;
  a->G = c->n_q_heads / c->n_kv_heads;
  a->D = c->head_dim;
  a->q_len = c->q_len;
  a->kv_len = c->kv_len;
  // a window of every key is none
  a->window = c->window >= c->kv_len ? 0 : c->window;
  a->sinks = a->window == 0 ? 0 : c->n_sinks < c->kv_len ? c->n_sinks : c->kv_len;
  a->esize = c->dtype == KVEC_BF16 ? 2 : 4;
  return KVEC_OK;
}

kvec_status make_paged(const kvec_paged_config* c, PagedView* v) {
  if (!c) return KVEC_ERR_INVALID;
  const kvec_status st = check_heads(c->batch, c->n_kv_heads, c->n_q_heads, c->head_dim, c->dtype);
  if (st != KVEC_OK) return st;
  if (c->page_size < 1 || c->n_pages < 1 || c->max_pages < 1) return KVEC_ERR_INVALID;
  if (c->page_size % 16 != 0 || (int64_t)c->max_pages * c->page_size > kMaxLen) return KVEC_ERR_UNSUPPORTED;
  memset(v, 0, sizeof(*v));
  v->batch = c->batch;
  v->H = c->n_kv_heads;
  v->HQ = c->n_q_heads;
  v->G = c->n_q_heads / c->n_kv_heads;
  v->D = c->head_dim;
  v->esize = c->dtype == KVEC_BF16 ? 2 : 4;
  v->ps = c->page_size;
  v->n_pages = c->n_pages;
  v->max_pages = c->max_pages;
  v->gdiv = group_div(c->page_size / 16);
  return KVEC_OK;
}

// Pools and their strides; the rows of a group of 16 are addressed with 31-bit
// offsets.
kvec_status set_pools(PagedView* v, const void* k_pool, const void* v_pool, const int64_t strides[3]) {
  if (!aligned16(k_pool) || !aligned16(v_pool) || !row_strides_ok(strides, {v->n_pages, v->H, v->ps}, v->esize)) return KVEC_ERR_INVALID;
  if (strides[2] * v->esize >= (int64_t)1 << 26) return KVEC_ERR_UNSUPPORTED;
  v->k = static_cast<char*>(const_cast<void*>(k_pool));
  v->v = static_cast<char*>(const_cast<void*>(v_pool));
  v->sp = strides[0];
  v->sh = strides[1];
  v->sr = strides[2];
  return KVEC_OK;
}

kvec_status set_lens(PagedView* v, const int32_t* table, const int32_t* lens, int32_t max_len) {
  if (!aligned(table, 4) || !aligned(lens, 4)) return KVEC_ERR_INVALID;
  if (max_len < 1 || max_len > v->max_pages * v->ps) return KVEC_ERR_INVALID;
  v->table = table;
  v->lens = lens;
  v->max_len = max_len;
  return KVEC_OK;
}

// A prompt's launch stays below 2^32 threads.  Up to eight a row, and 512 for every
// (sequence, KV head), can pass that from 2^28 rows on.
kvec_status check_plan(const PrefillShape& a, const PfPlan& p) {
  return pf_work_groups(a, p) * pf_threads(p.kernel) >= (int64_t)1 << 32 ? KVEC_ERR_UNSUPPORTED : KVEC_OK;
}

kvec_status check_size(size_t need, const void* ws, size_t ws_bytes) {
  if (ws_bytes < need) return KVEC_ERR_WORKSPACE;
  if (need > 0 && !aligned16(ws)) return KVEC_ERR_INVALID;
  return KVEC_OK;
}

}  // namespace

extern "C" {

kvec_status kvec_prefill_workspace_size(const kvec_attention_config* cfg, size_t* bytes) {
  PrefillArgs a;
  kvec_status st = make_prefill(cfg, &a);
  if (st != KVEC_OK) return st;
  if (!bytes) return KVEC_ERR_INVALID;
  const PfPlan plan = pf_plan(a);
  if ((st = check_plan(a, plan)) != KVEC_OK) return st;
  *bytes = plan.bytes;
  return KVEC_OK;
}

kvec_status kvec_prefill_attention(const kvec_attention_config* cfg, const void* q, const int64_t q_strides[3],
                                   const void* k, const int64_t k_strides[3], const void* v,
                                   const int64_t v_strides[3], const int32_t* q_lens, const int32_t* kv_lens,
                                   void* out, const int64_t out_strides[3], float* lse,
                                   const int64_t lse_strides[2], void* ws, size_t ws_bytes,
                                   hipStream_t stream) {
  PrefillArgs a;
  kvec_status st = make_prefill(cfg, &a);
  if (st != KVEC_OK) return st;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) ||
      !row_strides_ok(q_strides, {a.batch, a.HQ, a.q_len}, a.esize) ||
      !row_strides_ok(k_strides, {a.batch, a.H, a.kv_len}, a.esize) ||
      !row_strides_ok(v_strides, {a.batch, a.H, a.kv_len}, a.esize) ||
      !row_strides_ok(out_strides, {a.batch, a.HQ, a.q_len}, a.esize) ||
      !aligned_or_null(q_lens, 4) || !aligned_or_null(kv_lens, 4))
    return KVEC_ERR_INVALID;
  if (lse && !(lse_ok(lse, lse_strides, 2) && spans_ok(lse_strides, {a.batch, a.HQ}, 4))) return KVEC_ERR_INVALID;
  const int64_t span = k_strides[2] > v_strides[2] ? k_strides[2] : v_strides[2];
  if ((int64_t)a.kv_len * (span > a.D ? span : a.D) * a.esize >= (int64_t)1 << 31) return KVEC_ERR_UNSUPPORTED;
  const PfPlan plan = pf_plan(a);
  if ((st = check_plan(a, plan)) != KVEC_OK) return st;
  if ((st = check_size(plan.bytes, ws, ws_bytes)) != KVEC_OK) return st;
  a.q = static_cast<const char*>(q);
  a.k = static_cast<const char*>(k);
  a.v = static_cast<const char*>(v);
  for (int i = 0; i < 3; ++i) {
    a.qs[i] = q_strides[i];
    a.ks[i] = k_strides[i];
    a.vs[i] = v_strides[i];
    a.os[i] = out_strides[i];
  }
  a.q_lens = q_lens;
  a.kv_lens = kv_lens;
  a.out = static_cast<char*>(out);
  a.lse = lse;
  if (lse) {
    a.ls[0] = lse_strides[0];
    a.ls[1] = lse_strides[1];
  }
  return dev(run_prefill(a, plan, static_cast<char*>(ws), stream));
}

kvec_status kvec_paged_append(const kvec_paged_config* cfg, int32_t n_tokens, const void* q,
                              const int64_t q_strides[2], const void* k, const int64_t k_strides[2],
                              const void* v, const int64_t v_strides[2], const void* q_weight,
                              const void* k_weight, float eps, const int32_t* positions,
                              const double* inv_freq, int32_t rot_dim, const int64_t* slots, void* q_out,
                              const int64_t q_out_strides[2], void* k_pool, void* v_pool,
                              const int64_t pool_strides[3], float* acc, int32_t* pos, hipStream_t stream) {
  PagedView c;
  kvec_status st = make_paged(cfg, &c);
  if (st != KVEC_OK) return st;
  if (n_tokens < 0 || !(eps >= 0.f) || !isfinite(eps) || rot_dim < 0 || rot_dim > c.D) return KVEC_ERR_INVALID;
  if (n_tokens > 1 << 24 || rot_dim % 16 != 0) return KVEC_ERR_UNSUPPORTED;
  if (!row_strides_ok(q_strides, {n_tokens, c.HQ}, c.esize) || !row_strides_ok(k_strides, {n_tokens, c.H}, c.esize) ||
      !row_strides_ok(v_strides, {n_tokens, c.H}, c.esize) || !row_strides_ok(q_out_strides, {n_tokens, c.HQ}, c.esize))
    return KVEC_ERR_INVALID;
  if ((st = set_pools(&c, k_pool, v_pool, pool_strides)) != KVEC_OK) return st;
  if (n_tokens == 0) return KVEC_OK;  // the token tensors may be empty, without an address
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned_or_null(q_weight, 16) ||
      !aligned_or_null(k_weight, 16) || !aligned(positions, 4) || !aligned(slots, 8) ||
      (rot_dim > 0 && !aligned(inv_freq, 8)) || !aligned_or_null(acc, 4) || !aligned_or_null(pos, 4))
    return KVEC_ERR_INVALID;
  AppendArgs a;
  memset(&a, 0, sizeof(a));
  a.n = n_tokens;
  a.q = static_cast<const char*>(q);
  a.k = static_cast<const char*>(k);
  a.v = static_cast<const char*>(v);
  a.q_t = q_strides[0];
  a.q_h = q_strides[1];
  a.k_t = k_strides[0];
  a.k_h = k_strides[1];
  a.v_t = v_strides[0];
  a.v_h = v_strides[1];
  a.o_t = q_out_strides[0];
  a.o_h = q_out_strides[1];
  a.wq = static_cast<const char*>(q_weight);
  a.wk = static_cast<const char*>(k_weight);
  a.eps = eps;
  a.positions = positions;
  a.inv_freq = inv_freq;
  a.rot = rot_dim;
  a.slots = slots;
  a.q_out = static_cast<char*>(q_out);
  a.acc = acc;
  a.pos = pos;
  return dev(run_append(c, a, stream));
}

kvec_status kvec_paged_decode_workspace_size(const kvec_paged_config* cfg, int32_t max_len, int32_t with_acc,
                                             size_t* bytes) {
  PagedView c;
  const kvec_status st = make_paged(cfg, &c);
  if (st != KVEC_OK) return st;
  if (!bytes || max_len < 1 || max_len > c.max_pages * c.ps) return KVEC_ERR_INVALID;
  c.max_len = max_len;
  // a window splits its slots no finer than the whole sequence
  *bytes = paged_decode_plan(c, 0, 0, with_acc != 0).total();
  return KVEC_OK;
}

kvec_status kvec_paged_decode(const kvec_paged_config* cfg, const void* q, const int64_t q_strides[2],
                              const void* k_pool, const void* v_pool, const int64_t pool_strides[3],
                              const int32_t* page_table, const int32_t* lens, int32_t max_len, int32_t window,
                              int32_t n_sinks, float* out, float* lse, float* acc, void* ws, size_t ws_bytes,
                              hipStream_t stream) {
  PagedView c;
  kvec_status st = make_paged(cfg, &c);
  if (st != KVEC_OK) return st;
  if ((st = set_pools(&c, k_pool, v_pool, pool_strides)) != KVEC_OK) return st;
  if ((st = set_lens(&c, page_table, lens, max_len)) != KVEC_OK) return st;
  if (window < 0 || n_sinks < 0 || !aligned16(q) || !row_strides_ok(q_strides, {c.batch, c.HQ}, c.esize) || !aligned(out, 4) ||
      !aligned_or_null(lse, 4) || !aligned_or_null(acc, 4))
    return KVEC_ERR_INVALID;
  const int w = window >= max_len ? 0 : window;
  const int sinks = w == 0 ? 0 : n_sinks < max_len ? n_sinks : max_len;
  if ((st = check_size(paged_decode_plan(c, 0, 0, acc != nullptr).total(), ws, ws_bytes)) != KVEC_OK) return st;
  return dev(run_paged_decode(c, q, q_strides, w, sinks, out, lse, acc, static_cast<char*>(ws), stream));
}

kvec_status kvec_paged_evict_workspace_size(const kvec_paged_config* cfg, int32_t max_len, int32_t budget,
                                            size_t* bytes) {
  PagedView c;
  const kvec_status st = make_paged(cfg, &c);
  if (st != KVEC_OK) return st;
  if (!bytes || budget < 1 || max_len < 1 || max_len > c.max_pages * c.ps) return KVEC_ERR_INVALID;
  if (budget > kMaxLen) return KVEC_ERR_UNSUPPORTED;
  c.max_len = max_len;
  *bytes = paged_evict_ws(c, budget);
  return KVEC_OK;
}

kvec_status kvec_paged_evict(const kvec_paged_config* cfg, int32_t budget, int32_t window, int32_t n_sinks,
                             void* k_pool, void* v_pool, const int64_t pool_strides[3],
                             const int32_t* page_table, const int32_t* lens, const int32_t* n_seen,
                             int32_t max_len, float* acc, int32_t* pos, int32_t* kept, int32_t* lens_out,
                             void* ws, size_t ws_bytes, hipStream_t stream) {
  PagedView c;
  kvec_status st = make_paged(cfg, &c);
  if (st != KVEC_OK) return st;
  if ((st = set_pools(&c, k_pool, v_pool, pool_strides)) != KVEC_OK) return st;
  if ((st = set_lens(&c, page_table, lens, max_len)) != KVEC_OK) return st;
  if (budget < 1 || window < 0 || n_sinks < 0 || (int64_t)window + n_sinks > budget || !aligned(n_seen, 4) ||
      !aligned(acc, 4) || !aligned(pos, 4) || !aligned_or_null(kept, 4) || !aligned(lens_out, 4))
    return KVEC_ERR_INVALID;
  if (budget > kMaxLen) return KVEC_ERR_UNSUPPORTED;
  if ((st = check_size(paged_evict_ws(c, budget), ws, ws_bytes)) != KVEC_OK) return st;
  return dev(run_paged_evict(c, budget, window, n_sinks, n_seen, acc, pos, kept, lens_out,
                             static_cast<char*>(ws), stream));
}

}  // extern "C"

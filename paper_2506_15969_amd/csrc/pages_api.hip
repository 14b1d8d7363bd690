// Host side of the calls that need no context: rows around a decode step and a cache in pages (include/lazyev.h).
// Checks of arguments and launches; nothing is kept.
#include "lazyev.h"

#include <cmath>
#include <cstring>

#include "pages_api.h"

namespace {

bool dtype_ok(int32_t dtype, int32_t head_dim) {
  return (dtype == LAZYEV_DTYPE_FP32 || dtype == LAZYEV_DTYPE_BF16) && (head_dim == 64 || head_dim == 128);
}

// Pointers start at a whole element (any: there are rows at all); strides beyond any memory are refused, so that no product with a
// number of tokens or heads that are there overflows.
bool rows_ok(const lazyev_heads &h, bool has_to, bool any, size_t elem) {
  if (h.n_heads < 1) return false;
  if (!any) return true;
  if (!h.rows || reinterpret_cast<uintptr_t>(h.rows) % elem || reinterpret_cast<uintptr_t>(h.weight) % elem) return false;
  if (has_to && (!h.to || reinterpret_cast<uintptr_t>(h.to) % elem)) return false;
  const int64_t strides[6] = {h.seq_stride, h.token_stride, h.head_stride, has_to ? h.to_seq_stride : 0, has_to ? h.to_token_stride : 0,
                              has_to ? h.to_head_stride : 0};
  for (int64_t s : strides)
    if (s > (1ll << 40) || s < -(1ll << 40)) return false;
  return true;
}

bool rotation_ok(const lazyev_rotation *r, int32_t head_dim, bool normed) {
  if (!r) return false;
  if (normed && !(r->eps >= 0.f && std::isfinite(r->eps))) return false;
  if (r->layout == LAZYEV_ROPE_NONE) return true;
  if (r->layout != LAZYEV_ROPE_HALVES && r->layout != LAZYEV_ROPE_PAIRS) return false;
  return r->dims >= 16 && r->dims % 16 == 0 && r->dims <= head_dim && r->inv_freq && reinterpret_cast<uintptr_t>(r->inv_freq) % 4 == 0;
}

lazyev::RopeRows rope_rows(const lazyev_heads &h, bool turn) {
  lazyev::RopeRows r;
  std::memset(&r, 0, sizeof(r));
  r.in = h.rows; r.out = h.to; r.weight = h.weight;
  r.in_seq = h.seq_stride; r.in_token = h.token_stride; r.in_head = h.head_stride;
  r.out_seq = h.to_seq_stride; r.out_token = h.to_token_stride; r.out_head = h.to_head_stride;
  r.heads = h.n_heads;
  r.turn = turn ? 1 : 0;
  return r;
}

void set_rotation(lazyev::RopeArgs &a, const lazyev_rotation &r) {
  a.layout = r.layout;
  a.half = r.layout == LAZYEV_ROPE_NONE ? 0 : r.dims / 2;
  a.eps = r.eps;
  a.inv_freq = r.inv_freq;
}

bool pages_ok(const lazyev_pages *p) {
  if (!p || !dtype_ok(p->dtype, p->head_dim)) return false;
  if (p->n_kv_heads < 1 || p->n_kv_heads > 65535 || p->n_pages < 1 || p->page_size < 1 || p->page_size > (1 << 20)) return false;
  if (p->n_seqs < 1 || p->table_stride < 1) return false;
  // (a pool's rows have 32-bit numbers; the product of the two is below 2^36)
  if (p->n_pages > (1ll << 32) / (static_cast<long long>(p->n_kv_heads) * p->page_size)) return false;
  if (!p->k_pages || !p->v_pages || !p->table) return false;
  return reinterpret_cast<uintptr_t>(p->k_pages) % 16 == 0 && reinterpret_cast<uintptr_t>(p->v_pages) % 16 == 0 &&
         reinterpret_cast<uintptr_t>(p->table) % 4 == 0;
}

lazyev::PageTable page_table(const lazyev_pages &p) {
  lazyev::PageTable t;
  t.table = p.table; t.stride = p.table_stride; t.n_pages = p.n_pages; t.page_size = p.page_size;
  lazyev::page_div(t);
  return t;
}

}  // namespace

namespace lazyev {

int page_of_entry(int page_size, int entry) {
  PageTable t;
  t.page_size = page_size;
  page_div(t);
  return page_of(t, entry);
}

bool attend_args(const lazyev_pages *p, int32_t length, int32_t n_tokens, int32_t n_q_heads, AttendArgs *out) {
  if (!pages_ok(p) || length < 0 || n_tokens < 0 || n_q_heads < 1 || n_q_heads % p->n_kv_heads != 0) return false;
  if (n_q_heads / p->n_kv_heads > 64 || static_cast<long long>(length) > static_cast<long long>(p->table_stride) * p->page_size) return false;
  // (rows and a table row's entries have 32-bit numbers; those of a table row and KV head are cut into at most 65535 blocks)
  if (static_cast<long long>(n_tokens) * (n_q_heads / p->n_kv_heads) > 65535 * 32) return false;
  // (a launch has 2^32 threads at most from one end to the other: 512 for each of the two)
  if (length > (1 << 30) || static_cast<long long>(p->n_seqs) * p->n_kv_heads > (1 << 22)) return false;
  if (n_tokens > 0 && static_cast<long long>(p->n_seqs) * n_tokens > (1ll << 30) / n_q_heads) return false;
  AttendArgs a;
  std::memset(&a, 0, sizeof(a));
  a.n_seqs = p->n_seqs; a.n_tokens = n_tokens; a.n_q_heads = n_q_heads; a.n_kv_heads = p->n_kv_heads; a.group = n_q_heads / p->n_kv_heads;
  a.head_dim = p->head_dim; a.dtype = p->dtype; a.length = length;
  a.k_pages = p->k_pages; a.v_pages = p->v_pages;
  a.pages = page_table(*p);
  *out = a;
  return true;
}

}  // namespace lazyev

extern "C" {

int lazyev_norm_rope(int32_t n_seqs, int32_t n_tokens, int32_t head_dim, int32_t dtype, const lazyev_heads *q, const lazyev_heads *k,
                     const lazyev_rotation *rotation, const int32_t *positions, int32_t start, void *stream) {
  if (n_seqs < 0 || n_tokens < 0 || !dtype_ok(dtype, head_dim) || (!q && !k)) return LAZYEV_EINVAL;
  if (static_cast<long long>(n_seqs) * n_tokens > (1ll << 30) || reinterpret_cast<uintptr_t>(positions) % 4) return LAZYEV_EINVAL;
  const size_t elem = dtype == LAZYEV_DTYPE_FP32 ? 4 : 2;
  bool normed = false;
  long long heads = 0;
  for (const lazyev_heads *h : {q, k}) {
    if (!h) continue;
    if (!rows_ok(*h, true, n_seqs > 0 && n_tokens > 0, elem)) return LAZYEV_EINVAL;
    normed = normed || h->weight;
    heads += h->n_heads;
  }
  if (heads > 65535 || !rotation_ok(rotation, head_dim, normed)) return LAZYEV_EINVAL;
  if (n_seqs == 0 || n_tokens == 0) return LAZYEV_OK;
  lazyev::RopeArgs a;
  std::memset(&a, 0, sizeof(a));
  const bool turn = rotation->layout != LAZYEV_ROPE_NONE;
  a.rows[0] = rope_rows(q ? *q : *k, turn);
  if (q && k) a.rows[1] = rope_rows(*k, turn);
  a.n_seqs = n_seqs; a.n_tokens = n_tokens;
  set_rotation(a, *rotation);
  a.positions = positions; a.start = start;
  return lazyev::launch_rope(a, dtype, head_dim, static_cast<hipStream_t>(stream)) == hipSuccess ? LAZYEV_OK : LAZYEV_EHIP;
}

int lazyev_pages_append(const lazyev_pages *pages, int32_t start, int32_t n_tokens, const lazyev_heads *k, const lazyev_heads *v,
                        const lazyev_rotation *rotation, int32_t position0, void *stream) {
  if (!pages_ok(pages) || start < 0 || n_tokens < 0 || !k || !v) return LAZYEV_EINVAL;
  const size_t elem = pages->dtype == LAZYEV_DTYPE_FP32 ? 4 : 2;
  if (!rows_ok(*k, false, n_tokens > 0, elem) || !rows_ok(*v, false, n_tokens > 0, elem) || v->weight) return LAZYEV_EINVAL;
  if (k->n_heads != pages->n_kv_heads || v->n_heads != pages->n_kv_heads || 2 * pages->n_kv_heads > 65535) return LAZYEV_EINVAL;
  if (!rotation_ok(rotation, pages->head_dim, k->weight != nullptr)) return LAZYEV_EINVAL;
  const long long end = static_cast<long long>(start) + n_tokens;
  if (end > (1 << 30) || end > static_cast<long long>(pages->table_stride) * pages->page_size) return LAZYEV_EINVAL;
  if (static_cast<long long>(pages->n_seqs) * n_tokens > (1ll << 30)) return LAZYEV_EINVAL;
  if (n_tokens == 0) return LAZYEV_OK;
  lazyev::RopeArgs a;
  std::memset(&a, 0, sizeof(a));
  a.rows[0] = rope_rows(*k, rotation->layout != LAZYEV_ROPE_NONE);
  a.rows[0].out = pages->k_pages;
  a.rows[1] = rope_rows(*v, false);
  a.rows[1].out = pages->v_pages;
  a.n_seqs = pages->n_seqs; a.n_tokens = n_tokens;
  set_rotation(a, *rotation);
  a.start = position0;
  a.pages = page_table(*pages);
  a.first_entry = start;
  return lazyev::launch_rope(a, pages->dtype, pages->head_dim, static_cast<hipStream_t>(stream)) == hipSuccess ? LAZYEV_OK : LAZYEV_EHIP;
}

size_t lazyev_pages_attend_workspace(const lazyev_pages *pages, int32_t length, int32_t n_tokens, int32_t n_q_heads) {
  lazyev::AttendArgs a;
  return lazyev::attend_args(pages, length, n_tokens, n_q_heads, &a) && n_tokens > 0 ? lazyev::attend_workspace(a) : 0;
}

int lazyev_pages_attend(const lazyev_pages *pages, int32_t length, int32_t n_tokens, int32_t n_q_heads, const int32_t *visible,
                        const void *q, const void *joined_out, const float *joined_lse, void *out, float *lse, float scale,
                        void *workspace, size_t workspace_bytes, void *stream) {
  lazyev::AttendArgs a;
  if (!lazyev::attend_args(pages, length, n_tokens, n_q_heads, &a) || !(scale >= 0.f) || !std::isfinite(scale)) return LAZYEV_EINVAL;
  if (n_tokens == 0) return LAZYEV_OK;
  if (!q || !out || q == out || !joined_out != !joined_lse) return LAZYEV_EINVAL;
  const size_t elem = pages->dtype == LAZYEV_DTYPE_FP32 ? 4 : 2;
  for (const void *x : {q, joined_out, static_cast<const void *>(out)})
    if (reinterpret_cast<uintptr_t>(x) % elem) return LAZYEV_EINVAL;
  for (const void *x : {static_cast<const void *>(visible), static_cast<const void *>(joined_lse), static_cast<const void *>(lse)})
    if (reinterpret_cast<uintptr_t>(x) % 4) return LAZYEV_EINVAL;
  const size_t need = lazyev::attend_workspace(a);
  if (need > 0 && (!workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(workspace) % 256 != 0)) return LAZYEV_EWORKSPACE;
  a.visible = visible;
  a.scale = scale > 0.f ? scale : 1.f / std::sqrt(static_cast<float>(pages->head_dim));
  a.q = q; a.joined_out = joined_out; a.joined_lse = joined_lse; a.out = out; a.lse = lse;
  a.workspace = workspace;
  return lazyev::launch_attend(a, static_cast<hipStream_t>(stream)) == hipSuccess ? LAZYEV_OK : LAZYEV_EHIP;
}

}  // extern "C"

// Host side of the calls around a long cache in pages: bounds and choice of blocks, attention over them, weights and eviction (include/lazyev.h).
// Checks of arguments and launches; nothing is kept.
#include <cmath>
#include <cstring>

#include "pages_api.h"

namespace {

bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
size_t elem(int32_t dtype) { return dtype == LAZYEV_DTYPE_FP32 ? 4 : 2; }
bool block_ok(int32_t block) { return block == 16 || block == 32 || block == 64 || block == 128; }
float scale_of(float scale, int32_t head_dim) { return scale > 0.f ? scale : 1.f / std::sqrt(static_cast<float>(head_dim)); }

bool blocks_ok(const lazyev_blocks *b) {
  if (!b || !lazyev::dtype_ok(b->dtype, b->head_dim) || !block_ok(b->block)) return false;
  if (b->n_kv_heads < 1 || b->n_kv_heads > 65535 || b->n_seqs < 1 || b->n_blocks < 1) return false;
  if (static_cast<long long>(b->n_seqs) * b->n_kv_heads > (1 << 22)) return false;
  return b->bounds && aligned(b->bounds, 16);
}

// A call's heads and tokens, as lazyev_pages_attend has them.
bool heads_ok(int32_t n_seqs, int32_t n_kv_heads, int32_t n_tokens, int32_t n_q_heads) {
  if (n_tokens < 0 || n_q_heads < 1 || n_q_heads % n_kv_heads != 0 || n_q_heads / n_kv_heads > 64) return false;
  if (static_cast<long long>(n_tokens) * (n_q_heads / n_kv_heads) > 65535 * 32 || static_cast<long long>(n_seqs) * n_kv_heads > (1 << 22)) return false;
  return n_tokens == 0 || static_cast<long long>(n_seqs) * n_tokens <= (1ll << 30) / n_q_heads;
}

bool length_ok(const lazyev_pages &p, int32_t length) {
  return length >= 0 && length <= (1 << 30) && length <= static_cast<long long>(p.table_stride) * p.page_size;
}

bool workspace_ok(const void *workspace, size_t bytes, size_t need) {
  return need == 0 || (workspace && bytes >= need && aligned(workspace, 256));
}

bool choose_args(const lazyev_blocks *b, int32_t length, int32_t n_tokens, int32_t n_q_heads, int32_t n_last, int32_t n_chosen,
                 lazyev::ChooseArgs *out) {
  if (!blocks_ok(b) || !heads_ok(b->n_seqs, b->n_kv_heads, n_tokens, n_q_heads)) return false;
  if (length < 0 || length > (1 << 30) || length > static_cast<long long>(b->n_blocks) * b->block) return false;
  if (n_last < 1 || n_chosen < n_last || n_chosen > (1 << 20)) return false;
  lazyev::ChooseArgs a;
  std::memset(&a, 0, sizeof(a));
  a.n_seqs = b->n_seqs; a.n_tokens = n_tokens; a.n_q_heads = n_q_heads; a.n_kv_heads = b->n_kv_heads; a.group = n_q_heads / b->n_kv_heads;
  a.head_dim = b->head_dim; a.dtype = b->dtype;
  a.length = length; a.block = b->block; a.n_blocks = b->n_blocks;
  a.n_last = n_last; a.n_chosen = n_chosen;
  const int32_t most = (length + b->block - 1) / b->block;
  a.scored = most > n_chosen ? most - n_last : 0;
  if (static_cast<long long>(b->n_seqs) * b->n_kv_heads * (length / b->block / 128 + 1) > (1 << 22)) return false;
  a.bounds = b->bounds;
  *out = a;
  return true;
}

bool list_args(const lazyev_pages *p, int32_t length, int32_t block, int32_t n_chosen, int32_t n_tokens, int32_t n_q_heads,
               lazyev::AttendArgs *out) {
  lazyev::AttendArgs a;
  // (checks of the pages, of lengths, heads and tokens; then every token is a sequence of its own)
  if (!lazyev::attend_args(p, length, n_tokens, n_q_heads, &a) || !block_ok(block)) return false;
  if (n_chosen < 1 || static_cast<long long>(n_chosen) * block > (1 << 30)) return false;
  if (static_cast<long long>(p->n_seqs) * n_tokens * p->n_kv_heads > (1 << 22)) return false;
  if (static_cast<long long>(p->n_pages) * p->n_kv_heads * p->page_size >= (1ll << 32)) return false;
  a.list.entries = length;
  a.list.n_listed = n_chosen;
  while ((1 << a.list.block_shift) < block) ++a.list.block_shift;
  // (a stage of the kernel has whole runs: 64 entries at most)
  while (a.list.run_shift < a.list.block_shift && a.list.run_shift < 6 && p->page_size % (2 << a.list.run_shift) == 0) ++a.list.run_shift;
  a.list.tokens = n_tokens;
  a.length = n_chosen * block;
  a.n_seqs = p->n_seqs * n_tokens;
  a.n_tokens = 1;
  *out = a;
  return true;
}

bool weigh_args(const lazyev_pages *p, int32_t length, int32_t n_tokens, int32_t n_q_heads, lazyev::WeighArgs *out) {
  if (!lazyev::pages_ok(p) || !heads_ok(p->n_seqs, p->n_kv_heads, n_tokens, n_q_heads) || !length_ok(*p, length)) return false;
  if (static_cast<long long>(p->n_seqs) * p->n_kv_heads * (length / 128 + 1) >= (1ll << 24)) return false;
  lazyev::WeighArgs a;
  std::memset(&a, 0, sizeof(a));
  a.n_seqs = p->n_seqs; a.n_tokens = n_tokens; a.n_q_heads = n_q_heads; a.n_kv_heads = p->n_kv_heads; a.group = n_q_heads / p->n_kv_heads;
  a.head_dim = p->head_dim; a.dtype = p->dtype; a.length = length;
  a.k_pages = p->k_pages;
  a.pages = lazyev::page_table(*p);
  *out = a;
  return true;
}

int done(hipError_t e) { return e == hipSuccess ? LAZYEV_OK : LAZYEV_EHIP; }

}  // namespace

extern "C" {

int lazyev_blocks_bound(const lazyev_pages *pages, const lazyev_blocks *blocks, int32_t start, int32_t n_tokens, void *stream) {
  if (!lazyev::pages_ok(pages) || !blocks_ok(blocks) || start < 0 || n_tokens < 0) return LAZYEV_EINVAL;
  if (pages->n_kv_heads != blocks->n_kv_heads || pages->head_dim != blocks->head_dim || pages->dtype != blocks->dtype ||
      pages->n_seqs != blocks->n_seqs)
    return LAZYEV_EINVAL;
  const long long end = static_cast<long long>(start) + n_tokens;
  if (end > (1 << 30) || end > static_cast<long long>(pages->table_stride) * pages->page_size ||
      end > static_cast<long long>(blocks->n_blocks) * blocks->block)
    return LAZYEV_EINVAL;
  if (n_tokens == 0) return LAZYEV_OK;
  lazyev::BoundArgs a;
  std::memset(&a, 0, sizeof(a));
  a.units = pages->n_seqs * pages->n_kv_heads; a.n_kv_heads = pages->n_kv_heads; a.head_dim = pages->head_dim; a.dtype = pages->dtype;
  a.start = start; a.end = static_cast<int32_t>(end);
  a.block = blocks->block; a.first_block = start / a.block; a.touched = (a.end + a.block - 1) / a.block - a.first_block;
  a.n_blocks = blocks->n_blocks;
  if ((static_cast<long long>(a.units) * a.touched + 3) / 4 > (1 << 23)) return LAZYEV_EINVAL;
  a.k_pages = pages->k_pages;
  a.pages = lazyev::page_table(*pages);
  a.bounds = blocks->bounds;
  return done(lazyev::launch_bound(a, static_cast<hipStream_t>(stream)));
}

size_t lazyev_blocks_choose_workspace(const lazyev_blocks *blocks, int32_t length, int32_t n_tokens, int32_t n_q_heads, int32_t n_last,
                                      int32_t n_chosen) {
  lazyev::ChooseArgs a;
  return choose_args(blocks, length, n_tokens, n_q_heads, n_last, n_chosen, &a) && n_tokens > 0 ? lazyev::choose_workspace(a) : 0;
}

int lazyev_blocks_choose(const lazyev_blocks *blocks, int32_t length, int32_t n_tokens, int32_t n_q_heads, const int32_t *visible,
                         const void *q, int32_t n_first, int32_t n_last, int32_t n_chosen, int32_t *chosen, void *workspace,
                         size_t workspace_bytes, void *stream) {
  lazyev::ChooseArgs a;
  if (!choose_args(blocks, length, n_tokens, n_q_heads, n_last, n_chosen, &a) || n_first < 0 || n_first > n_chosen - n_last) return LAZYEV_EINVAL;
  if (n_tokens == 0) return LAZYEV_OK;
  if (!q || !chosen || !aligned(q, elem(blocks->dtype)) || !aligned(visible, 4) || !aligned(chosen, 4)) return LAZYEV_EINVAL;
  if (!workspace_ok(workspace, workspace_bytes, lazyev::choose_workspace(a))) return LAZYEV_EWORKSPACE;
  a.n_first = n_first;
  a.visible = visible; a.q = q; a.chosen = chosen; a.workspace = workspace;
  return done(lazyev::launch_choose(a, static_cast<hipStream_t>(stream)));
}

size_t lazyev_blocks_attend_workspace(const lazyev_pages *pages, int32_t length, int32_t block, int32_t n_chosen, int32_t n_tokens,
                                      int32_t n_q_heads) {
  lazyev::AttendArgs a;
  return list_args(pages, length, block, n_chosen, n_tokens, n_q_heads, &a) && n_tokens > 0 ? lazyev::attend_list_workspace(a) : 0;
}

int lazyev_blocks_attend(const lazyev_pages *pages, int32_t length, int32_t block, int32_t n_chosen, const int32_t *chosen,
                         int32_t n_tokens, int32_t n_q_heads, const int32_t *visible, const void *q, const void *joined_out,
                         const float *joined_lse, void *out, float *lse, float scale, void *workspace, size_t workspace_bytes,
                         void *stream) {
  lazyev::AttendArgs a;
  if (!list_args(pages, length, block, n_chosen, n_tokens, n_q_heads, &a) || !(scale >= 0.f) || !std::isfinite(scale)) return LAZYEV_EINVAL;
  if (n_tokens == 0) return LAZYEV_OK;
  if (!q || !out || !chosen || q == out || !joined_out != !joined_lse) return LAZYEV_EINVAL;
  for (const void *x : {q, joined_out, static_cast<const void *>(out)})
    if (!aligned(x, elem(pages->dtype))) return LAZYEV_EINVAL;
  for (const void *x : {static_cast<const void *>(visible), static_cast<const void *>(joined_lse), static_cast<const void *>(lse),
                        static_cast<const void *>(chosen)})
    if (!aligned(x, 4)) return LAZYEV_EINVAL;
  if (!workspace_ok(workspace, workspace_bytes, lazyev::attend_list_workspace(a))) return LAZYEV_EWORKSPACE;
  a.list.list = chosen;
  a.visible = visible;
  a.scale = scale_of(scale, pages->head_dim);
  a.q = q; a.joined_out = joined_out; a.joined_lse = joined_lse; a.out = out; a.lse = lse;
  a.workspace = workspace;
  return done(lazyev::launch_attend_list(a, static_cast<hipStream_t>(stream)));
}

size_t lazyev_pages_weigh_workspace(const lazyev_pages *pages, int32_t length, int32_t n_tokens, int32_t n_q_heads) {
  lazyev::WeighArgs a;
  return weigh_args(pages, length, n_tokens, n_q_heads, &a) && n_tokens > 0 && length > 0 ? lazyev::weigh_workspace(a) : 0;
}

int lazyev_pages_weigh(const lazyev_pages *pages, int32_t length, int32_t n_tokens, int32_t n_q_heads, const int32_t *visible,
                       const void *q, const float *lse, float scale, const float *old, int32_t known, float decay, float *weights,
                       int64_t stride, void *workspace, size_t workspace_bytes, void *stream) {
  lazyev::WeighArgs a;
  if (!weigh_args(pages, length, n_tokens, n_q_heads, &a) || !(scale >= 0.f) || !std::isfinite(scale) || !std::isfinite(decay)) return LAZYEV_EINVAL;
  if (known < 0 || known > length || stride < length || stride > (1ll << 40)) return LAZYEV_EINVAL;
  if (length == 0) return LAZYEV_OK;
  if (!weights || (known > 0 && !old) || !aligned(weights, 4) || !aligned(old, 4)) return LAZYEV_EINVAL;
  if (n_tokens > 0 && (!q || !lse || !aligned(q, elem(pages->dtype)) || !aligned(lse, 4) || !aligned(visible, 4))) return LAZYEV_EINVAL;
  if (!workspace_ok(workspace, workspace_bytes, n_tokens > 0 ? lazyev::weigh_workspace(a) : 0)) return LAZYEV_EWORKSPACE;
  a.known = decay == 0.f ? 0 : known;
  a.decay = decay;
  a.scale = scale_of(scale, pages->head_dim);
  a.visible = visible; a.q = q; a.lse = lse; a.old = old; a.weights = weights; a.stride = stride;
  a.workspace = workspace;
  return done(lazyev::launch_weigh(a, static_cast<hipStream_t>(stream)));
}

size_t lazyev_pages_evict_workspace(const lazyev_pages *pages, int32_t keep) {
  if (!lazyev::pages_ok(pages) || keep < 1) return 0;
  lazyev::WeightEvictArgs a;
  std::memset(&a, 0, sizeof(a));
  a.n_seqs = pages->n_seqs; a.n_kv_heads = pages->n_kv_heads; a.keep = keep;
  return lazyev::weight_evict_workspace(a);
}

int lazyev_pages_evict(const lazyev_pages *pages, int32_t length, const int32_t *lengths, int32_t keep, int32_t n_recent, int32_t n_first,
                       const float *weights, const int32_t *positions, int64_t stride, int32_t *sources, float *weights_to,
                       int32_t *positions_to, int64_t to_stride, void *workspace, size_t workspace_bytes, void *stream) {
  if (!lazyev::pages_ok(pages) || !length_ok(*pages, length)) return LAZYEV_EINVAL;
  if (keep < 1 || n_recent < 0 || n_first < 0 || n_recent > keep || n_first > keep - n_recent) return LAZYEV_EINVAL;
  const long long units = static_cast<long long>(pages->n_seqs) * pages->n_kv_heads;
  if (units >= (1 << 22) || units * (keep / 64 + 1) >= (1ll << 24)) return LAZYEV_EINVAL;
  if (stride < length || stride > (1ll << 40) || ((weights_to || positions_to) && (to_stride < keep || to_stride > (1ll << 40)))) return LAZYEV_EINVAL;
  if ((!weights && length > 0) || !sources) return LAZYEV_EINVAL;
  for (const void *x : {static_cast<const void *>(lengths), static_cast<const void *>(weights), static_cast<const void *>(positions),
                        static_cast<const void *>(sources), static_cast<const void *>(weights_to), static_cast<const void *>(positions_to)})
    if (!aligned(x, 4)) return LAZYEV_EINVAL;
  lazyev::WeightEvictArgs a;
  std::memset(&a, 0, sizeof(a));
  a.n_seqs = pages->n_seqs; a.n_kv_heads = pages->n_kv_heads; a.head_dim = pages->head_dim; a.dtype = pages->dtype;
  a.length = length; a.keep = keep; a.n_recent = n_recent; a.n_first = n_first;
  if (!workspace_ok(workspace, workspace_bytes, lazyev::weight_evict_workspace(a))) return LAZYEV_EWORKSPACE;
  a.lengths = lengths; a.weights = weights; a.positions = positions; a.stride = stride; a.to_stride = to_stride;
  a.sources = sources; a.weights_to = weights_to; a.positions_to = positions_to;
  a.k_pages = pages->k_pages; a.v_pages = pages->v_pages;
  a.pages = lazyev::page_table(*pages);
  a.free_places = static_cast<int32_t *>(workspace);
  return done(lazyev::launch_weight_evict(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"

// extern "C" entry points of the attention operators: argument validation and
// dispatch.
#include <cmath>
#include <initializer_list>

#include "cache.h"

using namespace sparoa;

namespace {

constexpr int64_t kMax31 = INT32_MAX;

bool below_2g(int64_t a, int64_t b, int64_t c = 1) {
  int64_t p;
  return !__builtin_mul_overflow(a, b, &p) && !__builtin_mul_overflow(p, c, &p) && p <= kMax31;
}

sparoa_status check_ptrs16(std::initializer_list<const void *> ps) {
  for (const void *p : ps)
    if (p && !aligned16(p)) return fail(SPAROA_ERR_UNSUPPORTED, "pointer not 16-byte aligned");
  return SPAROA_OK;
}

sparoa_status check_kv(const sparoa_kv_desc *d) {
  if (!d) return fail(SPAROA_ERR_INVALID_ARG, "null kv descriptor");
  if (d->dtype != SPAROA_F32 && d->dtype != SPAROA_F16 && d->dtype != SPAROA_BF16)
    return fail(SPAROA_ERR_INVALID_ARG, "unknown dtype");
  for (int64_t v : {d->tokens, d->requests, d->heads, d->kv_heads, d->head_dim, d->pages,
                    d->page_size, d->table_pages, d->max_queries, d->max_keys})
    if (v <= 0) return fail(SPAROA_ERR_INVALID_ARG, "kv: sizes must be > 0");
  if (d->heads % d->kv_heads)
    return fail(SPAROA_ERR_INVALID_ARG, "kv: heads must be a multiple of kv_heads");
  if (d->head_dim > 256 || d->head_dim % 8)
    return fail(SPAROA_ERR_UNSUPPORTED, "kv: head_dim above 256 or no multiple of 8");
  // (a row tile's and a key tile's last index stay below 2^31, too)
  if (d->tokens > kMax31 - 1024 || !below_2g(d->tokens + 1024, d->heads) ||
      !below_2g(d->requests, d->table_pages) || d->requests >= kMax31 ||
      !below_2g(d->pages, d->kv_heads, d->page_size) || d->max_keys > kMax31 - 1024 ||
      d->page_size > kMax31)
    return fail(SPAROA_ERR_UNSUPPORTED, "kv: 2^31 or more rows, keys or table entries");
  int64_t held;
  if (!__builtin_mul_overflow(d->table_pages, d->page_size, &held) && d->max_keys > held)
    return fail(SPAROA_ERR_INVALID_ARG, "kv: max_keys above table_pages * page_size");
  return SPAROA_OK;
}

KvArgs kv_args(const sparoa_kv_desc &d, const int32_t *q_start, const int32_t *kv_len,
               const int32_t *table) {
  KvArgs a{};
  a.q_start = q_start, a.kv_len = kv_len, a.table = table;
  a.tokens = (int)d.tokens, a.requests = (int)d.requests, a.heads = (int)d.heads;
  a.kv_heads = (int)d.kv_heads, a.group = (int)(d.heads / d.kv_heads), a.dim = (int)d.head_dim;
  a.pages = (int)d.pages, a.page_size = (int)d.page_size, a.table_pages = (int)d.table_pages;
  a.max_queries = (int)(d.max_queries < d.tokens ? d.max_queries : d.tokens);
  a.max_keys = (int)d.max_keys;
  a.by_page = kv_div(d.page_size), a.by_group = kv_div(a.group);
  return a;
}

sparoa_status check_opts(const sparoa_attention_opts *o) {
  if (!o) return fail(SPAROA_ERR_INVALID_ARG, "null attention options");
  // (the kernel divides by both, and one by the other)
  constexpr float least = 0x1p-60f, most = 0x1p60f;
  if (!(o->scale >= least && o->scale <= most))
    return fail(SPAROA_ERR_INVALID_ARG, "attention: the scale must be in [2^-60, 2^60]");
  if (!(o->cap == 0.f || (o->cap >= least && o->cap <= most)) || o->window < 0)
    return fail(SPAROA_ERR_INVALID_ARG,
                "attention: cap must be 0 or in [2^-60, 2^60], window >= 0");
  return SPAROA_OK;
}

sparoa_status attend(const sparoa_kv_desc *d, const sparoa_attention_opts *o, AttnArgs a,
                     void *workspace, size_t ws_bytes, hipStream_t stream) {
  sparoa_status st = check_ptrs16({a.q, a.k, a.v, a.kv.q_start, a.kv.kv_len, a.kv.table, a.prefix,
                                   a.first, a.slopes, a.mask, a.positions, a.out, workspace});
  if (st != SPAROA_OK) return st;
  if (!workspace || ws_bytes < attention_workspace(*d))
    return fail(SPAROA_ERR_WORKSPACE, "attention: workspace too small");
  a.scale = o->scale, a.cap = o->cap;
  // (longer than any distance there is: none; a tree's positions may be any)
  a.window = (int)(o->window < (a.mask ? kMax31 : d->max_keys) ? o->window : 0);
  a.causal = o->causal != 0;
  return launch_attention(a, *d, workspace, stream);
}

}  // namespace

extern "C" {

sparoa_status sparoa_kv_append(const sparoa_kv_desc *d, int64_t rot_dim, int interleaved,
                               const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                               const void *v, int64_t v_stride, const double *freqs,
                               const int32_t *positions, const int32_t *q_start,
                               const int32_t *kv_len, const int32_t *page_table, void *q_out,
                               void *k_cache, void *v_cache, hipStream_t stream) {
  clear_error();
  sparoa_status st = check_kv(d);
  if (st != SPAROA_OK) return st;
  if (!k || !v || !q_start || !kv_len || !page_table || !k_cache || !v_cache)
    return fail(SPAROA_ERR_INVALID_ARG, "kv_append: null k, v, lengths, pages or cache");
  if ((q != nullptr) != (q_out != nullptr))
    return fail(SPAROA_ERR_INVALID_ARG, "kv_append: q and q_out go together");
  if (rot_dim < 0 || rot_dim > d->head_dim || rot_dim % 2)
    return fail(SPAROA_ERR_INVALID_ARG, "kv_append: rot_dim must be even and within the head");
  if ((rot_dim != 0) != (freqs != nullptr))
    return fail(SPAROA_ERR_INVALID_ARG, "kv_append: freqs must match rot_dim");
  const int64_t wide = d->heads * d->head_dim, narrow = d->kv_heads * d->head_dim;
  if ((q && q_stride < wide) || k_stride < narrow || v_stride < narrow)
    return fail(SPAROA_ERR_INVALID_ARG, "kv_append: a stride below a row");
  if (q == q_out && q && q_stride != wide)
    return fail(SPAROA_ERR_INVALID_ARG, "kv_append: q_out may be q only where its rows are dense");
  int64_t end;
  for (int64_t s : {q ? q_stride : 0, k_stride, v_stride})
    if (__builtin_mul_overflow(d->tokens, s, &end) || end > INT64_MAX / 8)
      return fail(SPAROA_ERR_INVALID_ARG, "kv_append: strides too large");
  st = check_ptrs16({q, k, v, freqs, positions, q_start, kv_len, page_table, q_out, k_cache,
                     v_cache});
  if (st != SPAROA_OK) return st;
  const AppendArgs a{kv_args(*d, q_start, kv_len, page_table), q, k, v, q_stride, k_stride,
                     v_stride, freqs, positions, q_out, k_cache, v_cache, (int)rot_dim,
                     interleaved != 0};
  return launch_kv_append(a, d->dtype, stream);
}

sparoa_status sparoa_attention_workspace_size(const sparoa_kv_desc *d, size_t *bytes) {
  clear_error();
  if (!bytes) return fail(SPAROA_ERR_INVALID_ARG, "null result pointer");
  sparoa_status st = check_kv(d);
  if (st != SPAROA_OK) return st;
  *bytes = attention_workspace(*d);
  return SPAROA_OK;
}

sparoa_status sparoa_paged_attention(const sparoa_kv_desc *d, const sparoa_attention_opts *opts,
                                     const void *q, const void *k_cache, const void *v_cache,
                                     const int32_t *q_start, const int32_t *kv_len,
                                     const int32_t *page_table, const int32_t *prefix_len,
                                     const int32_t *first_key, const float *slopes, void *out,
                                     void *workspace, size_t ws_bytes, hipStream_t stream) {
  clear_error();
  sparoa_status st = check_kv(d);
  if (st != SPAROA_OK) return st;
  st = check_opts(opts);
  if (st != SPAROA_OK) return st;
  if (!q || !k_cache || !v_cache || !q_start || !kv_len || !page_table || !out)
    return fail(SPAROA_ERR_INVALID_ARG, "paged_attention: null q, cache, lengths, pages or out");
  AttnArgs a{};
  a.kv = kv_args(*d, q_start, kv_len, page_table);
  a.q = q, a.k = k_cache, a.v = v_cache, a.out = out;
  a.prefix = prefix_len, a.first = first_key, a.slopes = slopes;
  return attend(d, opts, a, workspace, ws_bytes, stream);
}

sparoa_status sparoa_tree_attention(const sparoa_kv_desc *d, const sparoa_attention_opts *opts,
                                    const void *q, const void *k_cache, const void *v_cache,
                                    const int32_t *q_start, const int32_t *kv_len,
                                    const int32_t *page_table, const uint64_t *tree_mask,
                                    const int32_t *positions, const float *slopes, void *out,
                                    void *workspace, size_t ws_bytes, hipStream_t stream) {
  clear_error();
  sparoa_status st = check_kv(d);
  if (st != SPAROA_OK) return st;
  st = check_opts(opts);
  if (st != SPAROA_OK) return st;
  if (!q || !k_cache || !v_cache || !q_start || !kv_len || !page_table || !tree_mask || !out)
    return fail(SPAROA_ERR_INVALID_ARG,
                "tree_attention: null q, cache, lengths, pages, tree_mask or out");
  if ((slopes || opts->window) && !positions)
    return fail(SPAROA_ERR_INVALID_ARG, "tree_attention: slopes and a window want positions");
  if (d->max_queries > 256)
    return fail(SPAROA_ERR_UNSUPPORTED, "tree_attention: more than 256 nodes");
  AttnArgs a{};
  a.kv = kv_args(*d, q_start, kv_len, page_table);
  a.q = q, a.k = k_cache, a.v = v_cache, a.out = out;
  a.positions = positions, a.slopes = slopes;
  a.mask = tree_mask, a.mask_words = (int)cdiv(d->max_queries, 64);
  return attend(d, opts, a, workspace, ws_bytes, stream);
}

sparoa_status sparoa_kv_keep(const sparoa_kv_desc *d, int64_t layers, const int32_t *q_start,
                             const int32_t *kv_len, const int32_t *page_table,
                             const int32_t *keep, int64_t most, const int32_t *kept,
                             void *k_cache, void *v_cache, hipStream_t stream) {
  clear_error();
  sparoa_status st = check_kv(d);
  if (st != SPAROA_OK) return st;
  if (layers <= 0 || most <= 0)
    return fail(SPAROA_ERR_INVALID_ARG, "kv_keep: layers and most must be > 0");
  if (!q_start || !kv_len || !page_table || !keep || !kept || !k_cache || !v_cache)
    return fail(SPAROA_ERR_INVALID_ARG, "kv_keep: null lengths, pages, keep, kept or cache");
  if (most > 256 || layers > 65535)
    return fail(SPAROA_ERR_UNSUPPORTED, "kv_keep: more than 256 drafts or 65535 layers");
  st = check_ptrs16({q_start, kv_len, page_table, keep, kept, k_cache, v_cache});
  if (st != SPAROA_OK) return st;
  const int64_t rows = d->pages * d->kv_heads * d->page_size;
  const KeepArgs a{kv_args(*d, q_start, kv_len, page_table), keep, kept, (int)most,
                   rows * d->head_dim * elem_size(d->dtype), k_cache, v_cache};
  return launch_kv_keep(a, layers, d->dtype, stream);
}

}  // extern "C"

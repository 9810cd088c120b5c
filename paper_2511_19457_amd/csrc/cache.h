// Internal declarations of the attention operators: the paged cache's geometry,
// appends, attention, accepted drafts.
#pragma once

#include "block.h"

namespace sparoa {

// Division of a number below 2^31 by a constant d in [1, 2^31):
// n / d = n mul >> (31 + s), s = ceil(log2 d), mul = floor(2^(31 + s) / d) + 1
// (its error n (mul d - 2^(31 + s)) <= n d < 2^(31 + s) does not reach a quotient).
struct KvDiv {
  uint32_t mul;
  int shift;
};
inline KvDiv kv_div(int64_t d) {
  int s = 0;
  while (((int64_t)1 << s) < d) ++s;
  return KvDiv{(uint32_t)((((__int128)1 << (31 + s)) / d) + 1), 31 + s};
}

// The batch and its cache (the lengths and pages lie on the device).
struct KvArgs {
  const int32_t *q_start, *kv_len, *table;
  int tokens, requests, heads, kv_heads, group, dim;
  int pages, page_size, table_pages, max_queries, max_keys;
  KvDiv by_page, by_group;
};

#ifdef __HIPCC__
__device__ __forceinline__ int kv_quotient(int n, KvDiv d) {
  return (int)(((uint64_t)(uint32_t)n * d.mul) >> d.shift);
}

struct KvRequest {
  int start, n, len;   // first row, rows, keys; n 0: left out
};
__device__ __forceinline__ KvRequest kv_request(const KvArgs &a, int r) {
  const int s = a.q_start[r], e = a.q_start[r + 1], len = a.kv_len[r];
  const bool ok = s >= 0 && e <= a.tokens && e > s && e - s <= a.max_queries && len >= e - s &&
                  len <= a.max_keys;
  return KvRequest{s, ok ? e - s : 0, len};
}

// Cache row of a request's key at position p for kv head h, -1 where there is no page.
__device__ __forceinline__ int kv_row(const KvArgs &a, int r, int h, int p) {
  const int in = kv_quotient(p, a.by_page), page = a.table[(int64_t)r * a.table_pages + in];
  return (uint32_t)page < (uint32_t)a.pages
             ? (page * a.kv_heads + h) * a.page_size + (p - in * a.page_size)
             : -1;
}
#endif

struct AppendArgs {
  KvArgs kv;
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;
  const double *freqs;
  const int32_t *positions;
  void *q_out, *k_cache, *v_cache;
  int rot, interleaved;
};
sparoa_status launch_kv_append(const AppendArgs &a, sparoa_dtype dt, hipStream_t stream);

struct KeepArgs {
  KvArgs kv;
  const int32_t *keep, *kept;
  int most;
  int64_t layer_bytes;
  void *k_cache, *v_cache;
};
sparoa_status launch_kv_keep(const KeepArgs &a, int64_t layers, sparoa_dtype dt,
                             hipStream_t stream);

struct AttnArgs {
  KvArgs kv;
  const void *q, *k, *v;
  void *out;
  const int32_t *prefix, *first, *positions;
  const float *slopes;
  const uint64_t *mask;    // a tree's bits, or null
  int mask_words;
  float scale, cap;
  int window, causal;
  // how the work is split (attention_split)
  int target, slots, slot_waves;
  int elem;                // bytes of an element
  int tile_rows;           // rows of a tile at most
  int32_t *plan;           // workspace: the split of many requests, or null
  void *ml, *part;         // workspace: (maximum, sum) of rows, unscaled outputs
};
size_t attention_workspace(const sparoa_kv_desc &d);
sparoa_status launch_attention(AttnArgs a, const sparoa_kv_desc &d, void *workspace,
                               hipStream_t stream);

}  // namespace sparoa

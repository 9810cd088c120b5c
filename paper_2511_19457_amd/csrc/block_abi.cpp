// extern "C" entry points of the transformer-block operators: argument
// validation and dispatch.
#include <cmath>

#include "block.h"

using namespace sparoa;

namespace {

bool dtype_ok(int d) { return d == SPAROA_F32 || d == SPAROA_F16 || d == SPAROA_BF16; }

bool norm_ok(int n) {
  return n == SPAROA_NORM_NONE || n == SPAROA_NORM_RMS || n == SPAROA_NORM_LAYER;
}

sparoa_status check_ptrs16(std::initializer_list<const void *> ps) {
  for (const void *p : ps)
    if (p && !aligned16(p)) return fail(SPAROA_ERR_UNSUPPORTED, "pointer not 16-byte aligned");
  return SPAROA_OK;
}

// a * b * c fits 62 bits (every size positive).
bool product_ok(int64_t a, int64_t b, int64_t c = 1) {
  int64_t p;
  return !__builtin_mul_overflow(a, b, &p) && !__builtin_mul_overflow(p, c, &p) &&
         p <= INT64_MAX / 8;
}

sparoa_status check_plan(int64_t tokens, int64_t top_k, int64_t experts) {
  if (tokens <= 0 || top_k <= 0 || experts <= 0)
    return fail(SPAROA_ERR_INVALID_ARG, "experts: sizes must be > 0");
  if (experts > 512 || top_k > 32 || tokens > (1 << 30) / top_k)
    return fail(SPAROA_ERR_UNSUPPORTED,
                "experts: more than 512 experts, 32 choices or 2^30 slots");
  return SPAROA_OK;
}

sparoa_status check_route(const sparoa_expert_route_desc *d) {
  if (!d) return fail(SPAROA_ERR_INVALID_ARG, "null expert_route descriptor");
  if (!dtype_ok(d->dtype)) return fail(SPAROA_ERR_INVALID_ARG, "unknown dtype");
  if (d->score != SPAROA_SCORE_SOFTMAX && d->score != SPAROA_SCORE_SIGMOID)
    return fail(SPAROA_ERR_INVALID_ARG, "expert_route: unknown score");
  if (d->tokens <= 0 || d->top_k <= 0 || d->experts <= 0)
    return fail(SPAROA_ERR_INVALID_ARG, "expert_route: sizes must be > 0");
  if (d->groups <= 0 || d->experts % d->groups || d->top_groups < 1 ||
      d->top_groups > d->groups || (d->group_best != 1 && d->group_best != 2))
    return fail(SPAROA_ERR_INVALID_ARG, "expert_route: bad groups");
  if (d->top_k > d->experts / d->groups * d->top_groups)
    return fail(SPAROA_ERR_INVALID_ARG, "expert_route: more choices than experts to choose from");
  if (!std::isfinite(d->scale))
    return fail(SPAROA_ERR_INVALID_ARG, "expert_route: the scale must be finite");
  if (d->groups > 64) return fail(SPAROA_ERR_UNSUPPORTED, "expert_route: more than 64 groups");
  return check_plan(d->tokens, d->top_k, d->experts);
}

int64_t round4(int64_t n) { return (n + 3) / 4 * 4; }
// Words before the plan's order, and before its place.
int64_t plan_order(int64_t experts) { return round4(2 * experts + 2); }
int64_t plan_place(int64_t experts, int64_t slots) { return plan_order(experts) + round4(slots); }

void set_plan(RouteArgs &a, int32_t *plan) {
  a.plan = plan;
  a.order = plan ? plan + plan_order(a.experts) : nullptr;
  a.place = plan ? plan + plan_place(a.experts, a.tokens * a.top_k) : nullptr;
}

bool act_ok(int a, int last) { return a >= SPAROA_ACT_NONE && a <= last; }

// Bytes of an operand the kernels address with 31 bits.
bool below_2gib(int64_t rows, int64_t cols, int64_t size) {
  return product_ok(rows, cols, size) && rows * cols * size < (int64_t)1 << 31;
}

int64_t round8(int64_t n) { return (n + 7) / 8 * 8; }
size_t section(int64_t bytes) { return (size_t)((bytes + 255) / 256 * 256); }

sparoa_status check_ffn(const sparoa_expert_ffn_desc *d) {
  if (!d) return fail(SPAROA_ERR_INVALID_ARG, "null expert_ffn descriptor");
  if (!dtype_ok(d->dtype)) return fail(SPAROA_ERR_INVALID_ARG, "unknown dtype");
  sparoa_status st = check_plan(d->tokens, d->top_k, d->experts);
  if (st != SPAROA_OK) return st;
  if (d->hidden <= 0 || d->inner <= 0)
    return fail(SPAROA_ERR_INVALID_ARG, "expert_ffn: sizes must be > 0");
  const int64_t size = elem_size(d->dtype);
  // (a tile's rows of u and of the fp32 down products are addressed with 31 bits)
  if (!below_2gib(256, d->inner, 4) || !below_2gib(256, d->hidden, 4) ||
      !below_2gib(d->tokens, d->hidden, size) ||
      !below_2gib(d->inner * (d->gated ? 2 : 1), d->hidden, size))
    return fail(SPAROA_ERR_UNSUPPORTED,
                "expert_ffn: x or an expert's matrix of 2 GiB or more, or rows too long");
  if (!product_ok(d->tokens * d->top_k, round8(d->inner) + round8(d->hidden), 4) ||
      !product_ok(d->experts, 2 * d->inner * size, d->hidden))
    return fail(SPAROA_ERR_INVALID_ARG, "expert_ffn: sizes too large");
  return SPAROA_OK;
}
// Rows of x and of a matrix that start off 16 bytes are copied to rows that
// start on them (with zeros behind) where many rows share a matrix, so that the
// tile kernels serve them; the stream kernel reads them as they are.  A pass in us,
// copied against streamed: fp16 21 experts of 278 x 1928 gated, 11 rows each
// 56 / 53, 43 rows 62 / 98, 1000 rows 205 / 872; bf16 64 of 1021 x 512 gated, 32
// rows 123 / 120, 188 rows 166 / 338; fp32 16 of 1022 x 1024, 64 rows 123 / 110,
// 128 rows 168 / 183.
bool pads_ffn(const sparoa_expert_ffn_desc &d) {
  const int64_t size = elem_size(d.dtype), v = 16 / size, slots = d.tokens * d.top_k;
  return (d.hidden % v || d.inner % v) &&
         slots / (d.experts < slots ? d.experts : slots) > (size == 4 ? 96 : 32) &&
         below_2gib(d.tokens, round8(d.hidden), size) &&
         below_2gib(d.inner * (d.gated ? 2 : 1), round8(d.hidden), size) &&
         below_2gib(d.hidden, round8(d.inner), size);
}
struct FfnPads {   // bytes of the copies, 0: none
  size_t x = 0, up = 0, down = 0;
};
FfnPads ffn_pads(const sparoa_expert_ffn_desc &d) {
  FfnPads p;
  if (!pads_ffn(d)) return p;
  const int64_t size = elem_size(d.dtype), v = 16 / size;
  if (d.hidden % v) {
    p.x = section(d.tokens * round8(d.hidden) * size);
    p.up = section(d.experts * d.inner * (d.gated ? 2 : 1) * round8(d.hidden) * size);
  }
  if (d.inner % v) p.down = section(d.experts * d.hidden * round8(d.inner) * size);
  return p;
}
// Workspace: u, then the down products, then the copies.
size_t ffn_u_bytes(const sparoa_expert_ffn_desc &d) {
  return section(d.tokens * d.top_k * round8(d.inner) * elem_size(d.dtype));
}
size_t ffn_z_bytes(const sparoa_expert_ffn_desc &d) {
  return section(d.tokens * d.top_k * round8(d.hidden) * 4);
}
size_t ffn_bytes(const sparoa_expert_ffn_desc &d) {
  const FfnPads p = ffn_pads(d);
  return ffn_u_bytes(d) + ffn_z_bytes(d) + p.x + p.up + p.down;
}

sparoa_status check_adapted(const sparoa_fc_adapted_desc *d) {
  if (!d) return fail(SPAROA_ERR_INVALID_ARG, "null fc_adapted descriptor");
  if (!dtype_ok(d->dtype)) return fail(SPAROA_ERR_INVALID_ARG, "unknown dtype");
  if (d->m <= 0 || d->k <= 0 || d->n <= 0 || d->adapters <= 0 || d->rank <= 0)
    return fail(SPAROA_ERR_INVALID_ARG, "fc_adapted: sizes must be > 0");
  const int64_t size = elem_size(d->dtype);
  if (d->rank > 512) return fail(SPAROA_ERR_UNSUPPORTED, "fc_adapted: rank above 512");
  if (d->adapters > INT32_MAX || !below_2gib(256, d->k, size) || !below_2gib(256, d->n, size) ||
      !below_2gib(d->n, d->k, size) || !below_2gib(d->rank, d->k, size) ||
      !below_2gib(d->n, d->rank, size))
    return fail(SPAROA_ERR_UNSUPPORTED, "fc_adapted: rows of x or a matrix of 2 GiB or more");
  if (!product_ok(d->m, d->k, size) || !product_ok(d->m, d->n, size) ||
      !product_ok(d->m, round8(d->rank), 4) ||
      !product_ok(d->adapters, d->rank * size, d->k > d->n ? d->k : d->n))
    return fail(SPAROA_ERR_INVALID_ARG, "fc_adapted: sizes too large");
  return SPAROA_OK;
}
// As for the experts, but not where the adapters' matrices are most of the copy.
// bf16 6143 x 2048, 64 rows 42 us against 67, 4001 x 4096, 128 rows 54 / 47, 1000
// rows 102 / 312; fp16 1001 x 1001, 64 rows 19 / 19.
bool pads_adapted(const sparoa_fc_adapted_desc &d) {
  const int64_t v = 16 / elem_size(d.dtype);
  return d.k % v && d.m > 64 && d.adapters * d.rank <= 2 * (d.m + d.n) &&
         below_2gib(256, round8(d.k), elem_size(d.dtype)) &&
         below_2gib(d.n, round8(d.k), elem_size(d.dtype));
}
size_t adapted_h_bytes(const sparoa_fc_adapted_desc &d) {
  return section(d.m * round8(d.rank) * 4);   // h, fp32 or dtype
}
size_t adapted_bytes(const sparoa_fc_adapted_desc &d) {
  const int64_t row = round8(d.k) * elem_size(d.dtype);
  return adapted_h_bytes(d) + (pads_adapted(d) ? section(d.m * row) + section(d.n * row) +
                                                     section(d.adapters * d.rank * row) : 0);
}

}  // namespace

extern "C" {

// ---------------------------------------------------------- expert routing

sparoa_status sparoa_expert_plan_words(int64_t tokens, int64_t top_k, int64_t experts,
                                       int64_t *words) {
  clear_error();
  if (!words) return fail(SPAROA_ERR_INVALID_ARG, "null result pointer");
  sparoa_status st = check_plan(tokens, top_k, experts);
  if (st != SPAROA_OK) return st;
  *words = plan_place(experts, tokens * top_k) + round4(tokens * top_k);
  return SPAROA_OK;
}

sparoa_status sparoa_expert_route_workspace_size(const sparoa_expert_route_desc *d,
                                                 size_t *bytes) {
  clear_error();
  if (!bytes) return fail(SPAROA_ERR_INVALID_ARG, "null result pointer");
  sparoa_status st = check_route(d);
  if (st != SPAROA_OK) return st;
  *bytes = expert_plan_workspace(d->tokens, d->experts);
  return SPAROA_OK;
}

sparoa_status sparoa_expert_plan_workspace_size(int64_t tokens, int64_t top_k, int64_t experts,
                                                size_t *bytes) {
  clear_error();
  if (!bytes) return fail(SPAROA_ERR_INVALID_ARG, "null result pointer");
  sparoa_status st = check_plan(tokens, top_k, experts);
  if (st != SPAROA_OK) return st;
  *bytes = expert_plan_workspace(tokens, experts);
  return SPAROA_OK;
}

sparoa_status sparoa_expert_route(const sparoa_expert_route_desc *d, const void *logits,
                                  const float *bias, const uint8_t *token_mask, int32_t *idx,
                                  float *weights, int32_t *plan, void *workspace, size_t ws_bytes,
                                  hipStream_t stream) {
  clear_error();
  sparoa_status st = check_route(d);
  if (st != SPAROA_OK) return st;
  if (!logits || !idx || !weights)
    return fail(SPAROA_ERR_INVALID_ARG, "expert_route: null logits, idx or weights");
  st = check_ptrs16({logits, bias, token_mask, idx, weights, plan, workspace});
  if (st != SPAROA_OK) return st;
  if (plan && (!workspace || ws_bytes < expert_plan_workspace(d->tokens, d->experts)))
    return fail(SPAROA_ERR_WORKSPACE, "expert_route: workspace too small");
  RouteArgs a{};
  a.logits = logits, a.bias = bias, a.token_mask = token_mask, a.idx = idx, a.weights = weights;
  a.tokens = d->tokens, a.experts = (int)d->experts, a.top_k = (int)d->top_k;
  a.groups = (int)d->groups, a.top_groups = (int)d->top_groups;
  a.group_best = (int)d->group_best, a.score = d->score, a.renormalise = d->renormalise != 0;
  a.by_score = bias || (d->groups > 1 && d->group_best == 2);
  a.scale = d->scale;
  a.counts = reinterpret_cast<uint32_t *>(workspace);
  set_plan(a, plan);
  return launch_expert_route(a, d->dtype, stream);
}

sparoa_status sparoa_expert_plan(int64_t tokens, int64_t top_k, int64_t experts,
                                 const int32_t *idx, int32_t *plan, void *workspace,
                                 size_t ws_bytes, hipStream_t stream) {
  clear_error();
  sparoa_status st = check_plan(tokens, top_k, experts);
  if (st != SPAROA_OK) return st;
  if (!idx || !plan) return fail(SPAROA_ERR_INVALID_ARG, "expert_plan: null idx or plan");
  st = check_ptrs16({idx, plan, workspace});
  if (st != SPAROA_OK) return st;
  if (!workspace || ws_bytes < expert_plan_workspace(tokens, experts))
    return fail(SPAROA_ERR_WORKSPACE, "expert_plan: workspace too small");
  RouteArgs a{};
  a.idx = const_cast<int32_t *>(idx);   // (only read)
  a.tokens = tokens, a.experts = (int)experts, a.top_k = (int)top_k;
  a.counts = reinterpret_cast<uint32_t *>(workspace);
  set_plan(a, plan);
  return launch_expert_plan(a, stream);
}

// -------------------------------------------------------- experts' products

sparoa_status sparoa_expert_ffn_workspace_size(const sparoa_expert_ffn_desc *d, size_t *bytes) {
  clear_error();
  if (!bytes) return fail(SPAROA_ERR_INVALID_ARG, "null result pointer");
  sparoa_status st = check_ffn(d);
  if (st != SPAROA_OK) return st;
  *bytes = ffn_bytes(*d);
  return SPAROA_OK;
}

sparoa_status sparoa_expert_ffn(const sparoa_expert_ffn_desc *d, sparoa_act act, const void *x,
                                const void *w_up, const void *b_up, const void *w_down,
                                const void *b_down, const float *weights, const int32_t *plan,
                                const void *residual, void *y, void *workspace, size_t ws_bytes,
                                hipStream_t stream) {
  clear_error();
  sparoa_status st = check_ffn(d);
  if (st != SPAROA_OK) return st;
  if (!act_ok(act, SPAROA_ACT_GELU)) return fail(SPAROA_ERR_INVALID_ARG, "unknown activation");
  if (!x || !w_up || !w_down || !weights || !plan || !y)
    return fail(SPAROA_ERR_INVALID_ARG, "expert_ffn: null x, weights, plan or y");
  if ((d->has_bias != 0) != (b_up != nullptr) || (d->has_bias != 0) != (b_down != nullptr))
    return fail(SPAROA_ERR_INVALID_ARG, "expert_ffn: has_bias does not match the biases");
  st = check_ptrs16({x, w_up, b_up, w_down, b_down, weights, plan, residual, y, workspace});
  if (st != SPAROA_OK) return st;
  if (!workspace || ws_bytes < ffn_bytes(*d))
    return fail(SPAROA_ERR_WORKSPACE, "expert_ffn: workspace too small");
  const int64_t slots = d->tokens * d->top_k, size = elem_size(d->dtype);
  const int64_t ldu = round8(d->inner), ldz = round8(d->hidden);
  const int up_rows = (int)d->inner * (d->gated ? 2 : 1);
  char *ws = reinterpret_cast<char *>(workspace);
  void *u = ws, *z = ws + ffn_u_bytes(*d);
  RowsArgs a{};
  a.rows = slots;
  a.plan = plan;
  a.experts = (int)d->experts, a.top_k = (int)d->top_k;
  a.x = x, a.w = w_up, a.bias = b_up, a.y = u;
  a.order = plan + plan_order(d->experts);
  const FfnPads pads = ffn_pads(*d);
  char *const px = ws + ffn_u_bytes(*d) + ffn_z_bytes(*d), *const pu = px + pads.x;
  char *const pd = pu + pads.up;
  int64_t k = d->hidden;
  if (pads.x) {
    k = round8(d->hidden);
    st = launch_pad_rows(x, px, d->tokens, (int)d->hidden, (int)k, d->dtype, stream);
    if (st != SPAROA_OK) return st;
    st = launch_pad_rows(w_up, pu, d->experts * up_rows, (int)d->hidden, (int)k, d->dtype, stream);
    if (st != SPAROA_OK) return st;
    a.x = px, a.w = pu;
  }
  a.x_bytes = d->tokens * k * size;
  a.ldx = k, a.ldy = ldu;
  a.n = (int)d->inner, a.k = (int)k;
  a.w_rows = up_rows, a.w_stride = up_rows * k;
  a.act = act;
  st = launch_rows(d->gated ? kRowsUpGated : kRowsUp, a, d->dtype, stream);
  if (st != SPAROA_OK) return st;
  a.x = u, a.w = w_down, a.bias = b_down, a.y = z;
  a.order = nullptr;
  a.ldx = ldu, a.ldy = ldz;
  k = d->inner;
  if (pads.down) {   // (u's rows end in zeros)
    k = ldu;
    st = launch_pad_rows(w_down, pd, d->experts * d->hidden, (int)d->inner, (int)k, d->dtype,
                         stream);
    if (st != SPAROA_OK) return st;
    a.w = pd;
  }
  a.n = (int)d->hidden, a.k = (int)k;
  a.w_rows = (int)d->hidden, a.w_stride = d->hidden * k;
  // The down products of bf16 experts with many rows go to the weighted sum as 8
  // fp16 numbers that share an exponent (pack_scaled8), which halves their way
  // through memory: 4096 tokens, 64 experts, top 8, 2048 x 1024: the down product
  // 213 -> 179 us (least times), the weighted sum 55 -> 27.  9 bits behind the
  // point, for channels down to 2^-28 of their largest neighbour, add a fiftieth to
  // the error that u's rounding gives (root mean square, and no bias); more where a
  // single product is rounded again for y, and beside fp16's own 10 bits.
  const bool scaled = d->dtype == SPAROA_BF16 && d->top_k > 1 &&
                      rows_tile_for(kRowsDown, a, d->dtype) >= kTile64x64;
  st = launch_rows(scaled ? kRowsDownScaled : kRowsDown, a, d->dtype, stream);
  if (st != SPAROA_OK) return st;
  const CombineArgs c{z, scaled, residual, weights,
                      plan + plan_place(d->experts, slots), y, d->tokens, d->hidden, ldz,
                      (int)d->top_k};
  return launch_combine(c, d->dtype, stream);
}

// -------------------------------------------------------------- adapted FC

sparoa_status sparoa_fc_adapted_workspace_size(const sparoa_fc_adapted_desc *d, size_t *bytes) {
  clear_error();
  if (!bytes) return fail(SPAROA_ERR_INVALID_ARG, "null result pointer");
  sparoa_status st = check_adapted(d);
  if (st != SPAROA_OK) return st;
  *bytes = adapted_bytes(*d);
  return SPAROA_OK;
}

sparoa_status sparoa_fc_adapted(const sparoa_fc_adapted_desc *d, sparoa_act act, const void *x,
                                const void *w_nk, const void *bias, const void *lora_a,
                                const void *lora_b, const float *scale,
                                const int32_t *adapter_ids, const void *residual, void *y,
                                void *workspace, size_t ws_bytes, hipStream_t stream) {
  clear_error();
  sparoa_status st = check_adapted(d);
  if (st != SPAROA_OK) return st;
  if (!act_ok(act, SPAROA_ACT_RELU6)) return fail(SPAROA_ERR_INVALID_ARG, "unknown activation");
  if (!x || !w_nk || !lora_a || !lora_b || !scale || !adapter_ids || !y)
    return fail(SPAROA_ERR_INVALID_ARG, "fc_adapted: null x, w, adapters, ids or y");
  if ((d->has_bias != 0) != (bias != nullptr))
    return fail(SPAROA_ERR_INVALID_ARG, "fc_adapted: has_bias does not match bias");
  st = check_ptrs16({x, w_nk, bias, lora_a, lora_b, scale, adapter_ids, residual, y, workspace});
  if (st != SPAROA_OK) return st;
  if (!workspace || ws_bytes < adapted_bytes(*d))
    return fail(SPAROA_ERR_WORKSPACE, "fc_adapted: workspace too small");
  RowsArgs a{};
  a.rows = d->m;
  a.ids = adapter_ids;
  a.scale = scale;
  a.adapters = (int)d->adapters, a.rank = (int)d->rank, a.ldh = (int)round8(d->rank);
  const void *la = lora_a;
  int64_t k = d->k;
  a.x = x, a.w = w_nk;
  if (pads_adapted(*d)) {
    k = round8(d->k);
    const int64_t row = k * elem_size(d->dtype);
    char *const px = reinterpret_cast<char *>(workspace) + adapted_h_bytes(*d);
    char *const pw = px + section(d->m * row), *const pa = pw + section(d->n * row);
    st = launch_pad_rows(x, px, d->m, (int)d->k, (int)k, d->dtype, stream);
    if (st != SPAROA_OK) return st;
    st = launch_pad_rows(w_nk, pw, d->n, (int)d->k, (int)k, d->dtype, stream);
    if (st != SPAROA_OK) return st;
    st = launch_pad_rows(lora_a, pa, d->adapters * d->rank, (int)d->k, (int)k, d->dtype, stream);
    if (st != SPAROA_OK) return st;
    a.x = px, a.w = pw, la = pa;
  }
  a.ldx = k, a.ldy = d->n;
  a.n = (int)d->n, a.k = (int)k;
  // h is an operand of MFMA, but for the stream kernel, which adds it in fp32
  a.h_f32 = rows_tile_for(kRowsFc, a, d->dtype) == kRowsStream;
  // adapters of up to 64 bytes of rank lie 2, 4 or 8 to a chunk (all of b
  // below 2 GiB)
  const int64_t size = elem_size(d->dtype), rank_bytes = d->rank * size;
  a.pack = 1;
  if (product_ok(d->adapters, d->n, rank_bytes) && d->adapters * d->n * rank_bytes < INT32_MAX)
    while (a.pack < 8 && rank_bytes * 2 * a.pack <= 128) a.pack *= 2;
  RowsArgs s = a;
  s.w = la, s.y = workspace;
  s.ldy = a.ldh;
  s.n = s.w_rows = (int)d->rank;
  s.w_stride = d->rank * k;
  st = launch_rows(kRowsShrink, s, d->dtype, stream);
  if (st != SPAROA_OK) return st;
  a.bias = bias, a.residual = residual, a.y = y;
  a.h = workspace, a.b = lora_b;
  a.w_rows = (int)d->n;
  a.act = act;
  return launch_rows(kRowsFc, a, d->dtype, stream);
}

// ------------------------------------------------------------- block norm

sparoa_status sparoa_block_norm(const sparoa_block_norm_desc *d, const void *y,
                                const void *post_w, const void *post_b, const void *gate,
                                const void *r, const void *pre_w, const void *pre_b, void *r_out,
                                void *n_out, hipStream_t stream) {
  clear_error();
  if (!d) return fail(SPAROA_ERR_INVALID_ARG, "null block_norm descriptor");
  if (!dtype_ok(d->dtype)) return fail(SPAROA_ERR_INVALID_ARG, "unknown dtype");
  if (d->rows <= 0 || d->cols <= 0 || d->gate_rows <= 0 || !product_ok(d->rows, d->cols))
    return fail(SPAROA_ERR_INVALID_ARG, "block_norm: sizes must be > 0");
  if (!norm_ok(d->post) || !norm_ok(d->pre))
    return fail(SPAROA_ERR_INVALID_ARG, "block_norm: unknown norm");
  if (!(d->eps >= 0.f) || !std::isfinite(d->eps) || !std::isfinite(d->residual_scale))
    return fail(SPAROA_ERR_INVALID_ARG, "block_norm: eps must be finite and >= 0, the scale finite");
  if (!y && !r) return fail(SPAROA_ERR_INVALID_ARG, "block_norm: y and r both null");
  const bool norms = d->pre != SPAROA_NORM_NONE;
  if (norms ? !n_out : !r_out)
    return fail(SPAROA_ERR_INVALID_ARG, norms ? "block_norm: null n_out"
                                              : "block_norm: null r_out and no norm to write");
  if (d->cols > INT32_MAX)
    return fail(SPAROA_ERR_UNSUPPORTED, "block_norm: more than 2^31 - 1 columns");
  sparoa_status st = check_ptrs16({y, post_w, post_b, gate, r, pre_w, pre_b, r_out, n_out});
  if (st != SPAROA_OK) return st;
  NormArgs a{y, post_w, post_b, gate, r, pre_w, pre_b, r_out, n_out, d->rows, d->cols,
             d->gate_rows, d->post, d->pre, d->eps, d->residual_scale};
  return launch_block_norm(a, d->dtype, stream);
}

}  // extern "C"

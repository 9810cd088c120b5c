// Internal declarations of the transformer-block operators (expert routing,
// experts' products, adapted FCs, the norm between blocks).
#pragma once

#include "common.h"

namespace sparoa {

struct NormArgs {
  const void *y, *post_w, *post_b, *gate, *r, *pre_w, *pre_b;
  void *r_out, *n_out;
  int64_t rows, cols, gate_rows;
  int post, pre;
  float eps, scale;
};
sparoa_status launch_block_norm(const NormArgs &a, sparoa_dtype dt, hipStream_t stream);

// Routing and plan (expert_route.hip).  top_k <= 32, experts <= 512, groups <= 64.
constexpr int kMaxExperts = 512;
constexpr int kPlanBlocks = 256;       // blocks of tokens that leave their counts
constexpr int kPlaceGroups = 128;      // work-groups that place slots by them
constexpr int kOneGroupSlots = 4096;   // given choices that one work-group plans
struct RouteArgs {
  const void *logits;
  const float *bias;
  const uint8_t *token_mask;
  int32_t *idx;
  float *weights;
  int32_t *plan, *order, *place;   // the plan's parts; plan null: none is made
  uint32_t *counts;                // workspace: [blocks][count_stride]
  int64_t tokens;
  int experts, top_k, groups, top_groups, group_best, score, renormalise;
  int by_score;                    // keys are scores, not logits
  float scale;
  int64_t tokens_per_block;        // (set by the launchers)
  int blocks, blocks_per_group, bits;
  int count_stride;                // words of a block's counts
  int group_lanes;                 // lanes of a group that has lanes of its own, or 0
};
sparoa_status launch_expert_route(RouteArgs a, sparoa_dtype dt, hipStream_t stream);
sparoa_status launch_expert_plan(RouteArgs a, hipStream_t stream);
size_t expert_plan_workspace(int64_t tokens, int64_t experts);

// Products of gathered or consecutive rows with the weights of their segment
// (rows*.hip): y[p] = epilogue(W_s x[p]), rows p of segment s.
//   experts: segments are the plan's experts, weights w + s * w_stride;
//            up: x rows gathered through order; down: consecutive.
//   fc:      one segment of `rows` consecutive rows, low-rank adapters.
struct RowsArgs {
  const void *x, *w, *bias, *residual;
  void *y;
  int64_t rows;                // slots (experts) or rows (fc)
  int64_t x_bytes;             // gathered x: bytes of the whole of it (< 2^31)
  int64_t ldx, ldy;            // elements per row of x and y
  int n, k;                    // output columns, depth
  int64_t w_stride;            // elements between segments' weights
  int w_rows;                  // weight rows of a segment (2 n: gate rows, then up rows)
  int act;
  // experts
  const int32_t *plan, *order; // order: gather through it (null: consecutive)
  int experts, top_k;
  // adapters: y += h[row] b[ids[row]]^T before bias and activation
  const int32_t *ids;          // [rows]; outside [0, adapters): none
  const void *h, *b;           // h [rows][ldh], b [adapters][n][rank]
  const float *scale;          // (shrink: h = scale_a A_a x)
  int adapters, rank, ldh;
  int pack;                    // adapters side by side in a chunk of 128 bytes
  int h_f32;                   // h is fp32 whatever the dtype
  int col_groups;              // (set by the tile launcher)
};
enum RowsMode { kRowsUp, kRowsUpGated, kRowsDownScaled, kRowsDown, kRowsFc, kRowsShrink };
// Kernel and tile (rows x weight rows) of a product (rows.hip).
enum RowsTile {
  kRowsStream,       // rows of x or w that start off 16 bytes (rows_stream.hip)
  kTile16x64, kTile32x32, kTile32x32x8,        // 4 waves split K, or 8 (rows_split.hip)
  kTile64x64, kTile64x128, kTile128x256        // waves share the tile (rows_tile.hip)
};
RowsTile rows_tile_for(RowsMode mode, const RowsArgs &a, sparoa_dtype dt);
sparoa_status launch_rows(RowsMode mode, const RowsArgs &a, sparoa_dtype dt, hipStream_t stream);
sparoa_status launch_rows_stream(RowsMode mode, const RowsArgs &a, sparoa_dtype dt,
                                 hipStream_t stream);
sparoa_status launch_rows_split(RowsMode mode, RowsTile tile, const RowsArgs &a, sparoa_dtype dt,
                                hipStream_t stream);
sparoa_status launch_rows_tile(RowsMode mode, RowsTile tile, const RowsArgs &a, sparoa_dtype dt,
                               hipStream_t stream);

// Rows of k elements -> rows of pitch elements (a multiple of 8), zeros behind k.
sparoa_status launch_pad_rows(const void *from, void *to, int64_t rows, int k, int pitch,
                              sparoa_dtype dt, hipStream_t stream);

// y[t] = residual[t] + sum_j weights[t][j] z[place[t][j]]
struct CombineArgs {
  const void *z;               // the down products, fp32 or scaled (kRowsDownScaled)
  int z_scaled;
  const void *residual;
  const float *weights;
  const int32_t *place;
  void *y;
  int64_t tokens, hidden, ldz;
  int top_k;
};
sparoa_status launch_combine(const CombineArgs &a, sparoa_dtype dt, hipStream_t stream);

}  // namespace sparoa

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
constexpr int kPlanBlocks = 256;       // blocks of tokens that leave their counts
constexpr int kPlaceGroups = 64;       // work-groups that place slots by them
constexpr int kOneGroupSlots = 4096;   // given choices that one work-group plans
struct RouteArgs {
  const void *logits;
  const float *bias;
  const uint8_t *token_mask;
  int32_t *idx;
  float *weights;
  int32_t *plan, *order, *place;   // the plan's parts; plan null: none is made
  uint32_t *counts;                // workspace: [blocks][experts + 1]
  int64_t tokens;
  int experts, top_k, groups, top_groups, group_best, score, renormalise;
  int by_score;                    // keys are scores, not logits
  float scale;
  int64_t tokens_per_block;        // (set by the launchers)
  int blocks, blocks_per_group, bits;
};
sparoa_status launch_expert_route(RouteArgs a, sparoa_dtype dt, hipStream_t stream);
sparoa_status launch_expert_plan(RouteArgs a, hipStream_t stream);
size_t expert_plan_workspace(int64_t tokens, int64_t experts);

}  // namespace sparoa

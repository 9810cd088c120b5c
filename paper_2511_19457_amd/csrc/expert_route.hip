// Routing to experts and the dispatch plan.
//
// route: a wave per token, lane l holding the EPL experts l EPL .. l EPL +
// EPL - 1.  The k choices are k rounds of a wave-wide maximum; the lowest
// lane that holds it, and in it the lowest expert, wins a tie.  Keys are
// compared as the formula gives them (softmax or sigmoid, plus bias); where
// only their order matters (no bias, no sum over a group) the logits are
// compared, which have the same order and never meet in a rounding.
//
// Bound by instruction issue: 16384 tokens over 256 experts in 8 groups, top 8,
// 27 us (twice the waves of half the tokens: 29); one token 5.3 us, plan and
// launch included.
//
// plan: a stable counting sort of the (token, choice) slots by expert.  Every
// place follows from counts alone, never from the order in which atomics
// land, so the plan of equal choices is equal.
//   one work-group (few slots): counts, offsets and places in LDS;
//   else two launches: each block of tokens leaves its counts (the route
//   kernel itself where it has just chosen), then every work-group adds up
//   the counts before its own blocks and places its slots (131072 slots: 7 us).
#include <algorithm>

#include "block.h"
#include "dtype.h"

namespace sparoa {
namespace {

constexpr int kMaxWaves = 16;   // waves of a work-group (4 for up to 4 tokens)
constexpr float kLow = -__builtin_inff();

// Maximum over the wave, in every lane (no NaN among the values).
__device__ __forceinline__ float wave_max(float v) {
#define SPAROA_DPP_MAX(ctrl)                                                                  \
  v = __builtin_fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(               \
                             (int)0xFF800000, __builtin_bit_cast(int, v), ctrl, 0xF, 0xF, false)))
  SPAROA_DPP_MAX(0x111);   // row_shr 1, 2, 4, 8: lane 15 of each row of 16
  SPAROA_DPP_MAX(0x112);
  SPAROA_DPP_MAX(0x114);
  SPAROA_DPP_MAX(0x118);
  SPAROA_DPP_MAX(0x142);   // row_bcast 15, then 31: lane 63
  SPAROA_DPP_MAX(0x143);
#undef SPAROA_DPP_MAX
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// Sum over the wave, in every lane.
__device__ __forceinline__ float wave_add(float v) {
#define SPAROA_DPP_ADD(ctrl, rows)                                                         \
  v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), \
                                                             ctrl, rows, 0xF, false))
  SPAROA_DPP_ADD(0x111, 0xF);
  SPAROA_DPP_ADD(0x112, 0xF);
  SPAROA_DPP_ADD(0x114, 0xF);
  SPAROA_DPP_ADD(0x118, 0xF);
  SPAROA_DPP_ADD(0x142, 0xA);
  SPAROA_DPP_ADD(0x143, 0xC);
#undef SPAROA_DPP_ADD
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// The value of the lane that ctrl pairs with this one.
template <int CTRL>
__device__ __forceinline__ float paired(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF,
                                                            0xF, true));
}
// The two best of the pair's four.
template <int CTRL>
__device__ __forceinline__ void merge_best(float &b1, float &b2) {
  const float o1 = paired<CTRL>(b1), o2 = paired<CTRL>(b2);
  b2 = __builtin_fmaxf(__builtin_fminf(b1, o1), __builtin_fmaxf(b2, o2));
  b1 = __builtin_fmaxf(b1, o1);
}

// Orders LDS accesses of the lanes of one wave for the compiler (the hardware
// keeps a wave's LDS operations in order).
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Lanes of the wave with the same e (0 <= e < 2^bits).
__device__ __forceinline__ uint64_t same_lanes(int e, int bits) {
  uint64_t m = ~0ull;
  for (int b = 0; b < bits; ++b) {
    const bool one = (e >> b) & 1;
    const uint64_t bal = __ballot(one);
    m &= one ? bal : ~bal;
  }
  return m;
}

// The work-group places slots [s0, s1).  first[e]: the place of the first of
// them that goes to expert e (e = experts: no expert, places behind all
// others, which hold -1).  cnt: W x (experts + 1) words of LDS, W the waves.
template <int W, class ExpertOf>
__device__ __forceinline__ void place_slots(int64_t s0, int64_t s1, int experts, int bits,
                                            const uint32_t *first, uint32_t *cnt,
                                            int32_t *order, int32_t *place, ExpertOf expert_of) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, nb = experts + 1;
  // wave w has the w-th run of whole 64s
  const int64_t per = ((s1 - s0 + 63) / 64 + W - 1) / W * 64;
  const int64_t b = s0 + wave * per, e_ = b + per < s1 ? b + per : s1;
  for (int i = tid; i < W * nb; i += 64 * W) cnt[i] = 0;
  __syncthreads();
  for (int64_t s = b + lane; s < e_; s += 64) atomicAdd(&cnt[wave * nb + expert_of(s)], 1u);
  __syncthreads();
  for (int e = tid; e < nb; e += 64 * W) {
    uint32_t at = first[e];
    for (int w = 0; w < W; ++w) {
      const uint32_t c = cnt[w * nb + e];
      cnt[w * nb + e] = at;
      at += c;
    }
  }
  __syncthreads();
  for (int64_t s = b; s < e_; s += 64) {   // (the whole wave takes part in the ballots)
    const bool in = s + lane < e_;
    const int e = in ? expert_of(s + lane) : 0;
    const uint64_t mates = same_lanes(e, bits) & __ballot(in);
    if (in) {
      const uint32_t rank = __popcll(mates & ((1ull << lane) - 1ull));
      const uint32_t at = cnt[wave * nb + e] + rank;
      order[at] = e < experts ? (int32_t)(s + lane) : -1;
      place[s + lane] = e < experts ? (int32_t)at : -1;
      // (a wave's LDS operations are in order: every lane has read its start)
      if (rank == 0) cnt[wave * nb + e] = at + (uint32_t)__popcll(mates);
    }
    wave_fence();
  }
}

// total[0 .. nb) of LDS -> its exclusive prefix sums in first (wave 0).
__device__ __forceinline__ void scan_counts(const uint32_t *total, uint32_t *first, int nb) {
  if (threadIdx.x >= 64) return;
  const int lane = threadIdx.x, per = (nb + 63) / 64;
  uint32_t sum = 0;
  for (int i = 0; i < per; ++i) {
    const int e = lane * per + i;
    if (e < nb) sum += total[e];
  }
  uint32_t run = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(run, d);
    if (lane >= d) run += o;
  }
  run -= sum;
  for (int i = 0; i < per; ++i) {
    const int e = lane * per + i;
    if (e < nb) {
      first[e] = run;
      run += total[e];
    }
  }
}

// The plan's head: offsets [experts + 1] (first: their prefix sums) and the
// experts with a slot, ascending, behind their number (wave 0).
__device__ __forceinline__ void write_head(const uint32_t *total, const uint32_t *first,
                                           int experts, int32_t *plan) {
  if (threadIdx.x >= 64) return;
  const int lane = threadIdx.x;
  int32_t *active = plan + experts + 1;
  int n = 0;
  for (int b = 0; b <= experts; b += 64) {
    const int e = b + lane;
    if (e <= experts) plan[e] = (int32_t)first[e];
    const bool has = e < experts && total[e] != 0;
    const uint64_t bal = __ballot(has);
    if (has) active[1 + n + __popcll(bal & ((1ull << lane) - 1ull))] = e;
    n += __popcll(bal);
  }
  if (lane == 0) active[0] = n;
  // (entries past the last active expert are not read)
}

template <int DT, int EPL>
struct Router {
  using E = Elem<DT>;
  using raw = typename E::raw;
  const RouteArgs &a;
  const int lane;
  float bias[EPL];
  int group_lane[EPL];   // first lane of the lanes that score this expert's group
  int lpg;               // lanes per group (a power of two)

  __device__ Router(const RouteArgs &args) : a(args), lane(threadIdx.x & 63) {
    // whole lanes to a group where its experts are a power of two of lanes
    lpg = a.group_lanes;
    if (!lpg) {
      lpg = 64;
      while (lpg * a.groups > 64) lpg >>= 1;
    }
    const int per = a.experts / a.groups;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const int e = lane * EPL + i;
      bias[i] = a.bias && e < a.experts ? a.bias[e] : 0.f;
      group_lane[i] = min(e, a.experts - 1) / per * lpg;
    }
  }

  // This lane's logits of token t; an expert that takes no part holds -inf.
  __device__ __forceinline__ void request(int64_t t, raw (&l)[EPL], bool &live) const {
    const raw *row = reinterpret_cast<const raw *>(a.logits) + t * a.experts;
    live = !a.token_mask || a.token_mask[t] != 0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) l[i] = row[min(lane * EPL + i, a.experts - 1)];
  }

  // Routes token t (the whole wave); scratch: LDS words for the keys of one
  // wave (groups that share lanes).  Afterwards lane j < top_k holds choice j
  // (-1: none) and its weight.
  __device__ __forceinline__ void token(int64_t t, const raw (&lr)[EPL], bool live,
                                        float *scratch, int &choice, float &weight) {
    float l[EPL], key[EPL];
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      l[i] = live && lane * EPL + i < a.experts ? E::to_f32(lr[i]) : kLow;
      l[i] = l[i] > kLow ? l[i] : kLow;   // a NaN takes no part either
    }
    const bool softmax = a.score == SPAROA_SCORE_SOFTMAX;
    float top = 0.f, sum = 1.f;
    // a logit of +inf shares the whole weight with its equals
    auto exp_from = [&](float v, float m) { return v == m ? (v > kLow ? 1.f : 0.f) : expf(v - m); };
    if (softmax && (a.by_score || !a.renormalise)) {
      float m = l[0];
#pragma unroll
      for (int i = 1; i < EPL; ++i) m = __builtin_fmaxf(m, l[i]);
      top = wave_max(m);
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < EPL; ++i) s += l[i] > kLow ? exp_from(l[i], top) : 0.f;
      sum = wave_add(s);
    }
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      float k = l[i];
      if (a.by_score) {
        k = softmax ? exp_from(l[i], top) / sum : 1.f / (1.f + expf(-l[i]));
        k = a.bias ? k + bias[i] : k;
        k = l[i] > kLow && k > kLow ? k : kLow;
      }
      key[i] = k;
    }
    if (a.groups > 1 && !a.group_lanes) {   // scores from LDS, then the keys one by one
#pragma unroll
      for (int i = 0; i < EPL; ++i)
        if (lane * EPL + i < a.experts) scratch[lane * EPL + i] = key[i];
      wave_fence();
      const int per = a.experts / a.groups, g = lane / lpg;
      float b1 = kLow, b2 = kLow;
      if (g < a.groups)
        for (int j = lane & (lpg - 1); j < per; j += lpg) {
          const float v = scratch[g * per + j];
          b2 = __builtin_fmaxf(b2, __builtin_fminf(b1, v));
          b1 = __builtin_fmaxf(b1, v);
        }
      for (int d = 1; d < lpg; d <<= 1) {
        const float o1 = __shfl_xor(b1, d), o2 = __shfl_xor(b2, d);
        b2 = __builtin_fmaxf(__builtin_fminf(b1, o1), __builtin_fmaxf(b2, o2));
        b1 = __builtin_fmaxf(b1, o1);
      }
      const uint64_t keep = kept_groups(b1, b2);
#pragma unroll
      for (int i = 0; i < EPL; ++i) key[i] = keep >> group_lane[i] & 1 ? key[i] : kLow;
      wave_fence();
    }
    // this lane's keys in descending order (equal ones stay in the experts'),
    // their places in bits 3 i of `order`
    int at[EPL];
#pragma unroll
    for (int i = 0; i < EPL; ++i) at[i] = i;
#pragma unroll
    for (int r = 0; r < EPL; ++r)
#pragma unroll
      for (int i = r & 1; i + 1 < EPL; i += 2) {
        const bool swap = key[i + 1] > key[i];
        const float k = swap ? key[i + 1] : key[i], o = swap ? key[i] : key[i + 1];
        const int p = swap ? at[i + 1] : at[i], q = swap ? at[i] : at[i + 1];
        key[i] = k, key[i + 1] = o, at[i] = p, at[i + 1] = q;
      }
    int order = 0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) order |= at[i] << (3 * i);
    if (a.group_lanes) {   // a lane's two best are its first two; its keys stay or go together
      float b1 = key[0], b2 = kLow;
      if constexpr (EPL > 1) b2 = key[1];
      if (lpg > 1) merge_best<0xB1>(b1, b2);    // quad_perm 1 0 3 2
      if (lpg > 2) merge_best<0x4E>(b1, b2);    // quad_perm 2 3 0 1
      if (lpg > 4) merge_best<0x141>(b1, b2);   // row_half_mirror
      if (lpg > 8) merge_best<0x140>(b1, b2);   // row_mirror
      const uint64_t keep = kept_groups(b1, b2);
      const bool stays = keep >> (lane & ~(lpg - 1)) & 1;
#pragma unroll
      for (int i = 0; i < EPL; ++i) key[i] = stays ? key[i] : kLow;
    }
    choice = -1;
    for (int j = 0; j < a.top_k; ++j) {
      const float m = wave_max(key[0]);
      if (!(m > kLow)) break;
      const int w = __ffsll((unsigned long long)__ballot(key[0] == m)) - 1;
      const int e = w * EPL + (__builtin_amdgcn_readlane(order, w) & 7);
      choice = lane == j ? e : choice;
      const bool won = lane == w;   // the next of its keys comes up
#pragma unroll
      for (int i = 0; i + 1 < EPL; ++i) key[i] = won ? key[i + 1] : key[i];
      key[EPL - 1] = won ? kLow : key[EPL - 1];
      order = won ? order >> 3 : order;
    }
    // weights: of the choices alone where they are renormalised (the softmax's
    // own sum cancels, and choices far below the row's largest logit keep
    // their ratios)
    const raw *row = reinterpret_cast<const raw *>(a.logits) + t * a.experts;
    const float chosen = choice >= 0 ? E::to_f32(row[choice]) : kLow;
    float s = 0.f;
    if (softmax) {
      if (a.renormalise) top = wave_max(chosen);
      s = choice >= 0 ? exp_from(chosen, top) : 0.f;
      if (!a.renormalise) s /= sum;
    } else if (choice >= 0) {
      s = 1.f / (1.f + expf(-chosen));
    }
    if (a.renormalise) {
      const float total = wave_add(s);
      s = total > 0.f ? s / total : 0.f;
    }
    weight = choice >= 0 ? s * a.scale : 0.f;
  }

  // Bit g lpg: group g is among the best; b1, b2: the two best keys of the
  // group of this lane's lpg lanes.
  __device__ __forceinline__ uint64_t kept_groups(float b1, float b2) const {
    const int g = lane / lpg;
    const float score = a.group_best == 2 && b2 > kLow ? b1 + b2 : b1;
    int rank = 0;
    for (int o = 0; o < a.groups; ++o) {
      const float s = __builtin_bit_cast(
          float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, score), o * lpg));
      rank += s > score || (s == score && o < g) ? 1 : 0;
    }
    return __ballot(g < a.groups && rank < a.top_groups && score > kLow);
  }
};

__device__ __forceinline__ int slot_expert(const int32_t *idx, int64_t s, int experts) {
  const int e = idx[s];
  return (uint32_t)e < (uint32_t)experts ? e : experts;
}

// Routes a block of tokens_per_block tokens a work-group of W waves, a wave's
// next token sent for before it chooses for one.  ONE: the only work-group,
// which also makes the plan (choices kept in LDS).
template <int DT, int EPL, bool ONE, int W>
__global__ __launch_bounds__(64 * W) void route_kernel(RouteArgs a) {
  extern __shared__ uint32_t lds[];
  const int nb = a.experts + 1, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  // [counts nb][first nb][keys of each wave, or the waves' counts][ONE: choices]
  uint32_t *total = lds, *first = lds + nb, *scratch = first + nb;
  int32_t *mine = reinterpret_cast<int32_t *>(scratch + W * nb);
  const int64_t t0 = (int64_t)blockIdx.x * a.tokens_per_block;
  const int64_t t1 = t0 + a.tokens_per_block < a.tokens ? t0 + a.tokens_per_block : a.tokens;
  Router<DT, EPL> r(a);
  typename Elem<DT>::raw l[EPL], nl[EPL];
  bool live = false, next_live = false;
  if (t0 + wave < t1) r.request(t0 + wave, l, live);
  for (int i = threadIdx.x; i < nb; i += 64 * W) total[i] = 0;
  __syncthreads();
  for (int64_t t = t0 + wave; t < t1; t += W) {
    if (t + W < t1) r.request(t + W, nl, next_live);
    int choice;
    float weight;
    r.token(t, l, live, reinterpret_cast<float *>(scratch + wave * nb), choice, weight);
    if (lane < a.top_k) {
      a.idx[t * a.top_k + lane] = choice;
      a.weights[t * a.top_k + lane] = weight;
      if (a.plan) {
        const int e = choice >= 0 ? choice : a.experts;
        atomicAdd(&total[e], 1u);
        if (ONE) mine[t * a.top_k + lane] = e;
      }
    }
#pragma unroll
    for (int i = 0; i < EPL; ++i) l[i] = nl[i];
    live = next_live;
  }
  if (!a.plan) return;
  __syncthreads();
  if (ONE) {
    scan_counts(total, first, nb);
    __syncthreads();
    write_head(total, first, a.experts, a.plan);
    place_slots<W>(0, a.tokens * a.top_k, a.experts, a.bits, first, scratch, a.order, a.place,
                   [&](int64_t s) { return mine[s]; });
  } else {
    for (int i = threadIdx.x; i < nb; i += 64 * W)
      a.counts[(int64_t)blockIdx.x * a.count_stride + i] = total[i];
  }
}

// Counts of given choices, a block of slots a work-group.  ONE: the only
// work-group, which also makes the plan.
template <bool ONE, int W>
__global__ __launch_bounds__(64 * W) void count_kernel(RouteArgs a) {
  extern __shared__ uint32_t lds[];
  const int nb = a.experts + 1;
  uint32_t *total = lds, *first = lds + nb, *scratch = first + nb;
  for (int i = threadIdx.x; i < nb; i += 64 * W) total[i] = 0;
  __syncthreads();
  const int64_t slots = a.tokens * a.top_k, per = a.tokens_per_block * a.top_k;
  const int64_t s0 = blockIdx.x * per, s1 = s0 + per < slots ? s0 + per : slots;
  for (int64_t s = s0 + threadIdx.x; s < s1; s += 64 * W)
    atomicAdd(&total[slot_expert(a.idx, s, a.experts)], 1u);
  __syncthreads();
  if (ONE) {
    scan_counts(total, first, nb);
    __syncthreads();
    write_head(total, first, a.experts, a.plan);
    place_slots<W>(0, slots, a.experts, a.bits, first, scratch, a.order, a.place,
                [&](int64_t s) { return slot_expert(a.idx, s, a.experts); });
  } else {
    for (int i = threadIdx.x; i < nb; i += 64 * W)
      a.counts[(int64_t)blockIdx.x * a.count_stride + i] = total[i];
  }
}

// Places the slots of blocks_per_group blocks a work-group.
__global__ __launch_bounds__(64 * kMaxWaves) void place_kernel(RouteArgs a) {
  constexpr int W = kMaxWaves, NT = 64 * W;
  extern __shared__ uint32_t lds[];
  const int nb = a.experts + 1, vecs = a.count_stride / 4;
  uint32_t *total = lds, *first = lds + nb, *scratch = first + nb;
  uint32_t *before = scratch;   // until place_slots takes the scratch
  for (int i = threadIdx.x; i < nb; i += NT) total[i] = before[i] = 0;
  __syncthreads();
  // the threads as rows of blocks' counts, four experts each: every rows-th
  // block's, 8 in flight
  const int rows = NT / vecs, v = threadIdx.x % vecs, b0 = blockIdx.x * a.blocks_per_group;
  if ((int)threadIdx.x < rows * vecs) {
    uint32_t all[4] = {}, mine[4] = {};
#pragma unroll 8
    for (int b = threadIdx.x / vecs; b < a.blocks; b += rows) {
      const uint4 c =
          *reinterpret_cast<const uint4 *>(a.counts + (int64_t)b * a.count_stride + 4 * v);
      all[0] += c.x, all[1] += c.y, all[2] += c.z, all[3] += c.w;
      if (b < b0) mine[0] += c.x, mine[1] += c.y, mine[2] += c.z, mine[3] += c.w;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (4 * v + i < nb) {   // (a row's padding holds anything)
        atomicAdd(&total[4 * v + i], all[i]);
        atomicAdd(&before[4 * v + i], mine[i]);
      }
  }
  __syncthreads();
  scan_counts(total, first, nb);
  __syncthreads();
  if (blockIdx.x == 0) write_head(total, first, a.experts, a.plan);
  __syncthreads();
  for (int i = threadIdx.x; i < nb; i += NT) first[i] += before[i];
  __syncthreads();
  const int64_t slots = a.tokens * a.top_k;
  const int64_t per = a.tokens_per_block * a.top_k * a.blocks_per_group;
  const int64_t s0 = blockIdx.x * per, s1 = s0 + per < slots ? s0 + per : slots;
  place_slots<W>(s0, s1, a.experts, a.bits, first, scratch, a.order, a.place,
                 [&](int64_t s) { return slot_expert(a.idx, s, a.experts); });
}

unsigned lds_bytes(const RouteArgs &a, int waves, int64_t kept) {
  return (unsigned)(4 * ((2 + waves) * (a.experts + 1) + kept));
}

template <int DT, int EPL>
void launch_route(RouteArgs a, bool one, int waves, hipStream_t stream) {
  const int per = a.experts / a.groups, lanes = per / EPL;
  a.group_lanes = a.groups > 1 && per % EPL == 0 && lanes <= 16 && (lanes & (lanes - 1)) == 0 ? lanes : 0;
  if (one && a.tokens <= 4)
    route_kernel<DT, EPL, true, 4><<<1, 256, lds_bytes(a, 4, a.tokens * a.top_k), stream>>>(a);
  else if (one)
    route_kernel<DT, EPL, true, kMaxWaves>
        <<<1, 64 * kMaxWaves, lds_bytes(a, kMaxWaves, a.tokens * a.top_k), stream>>>(a);
  else if (waves == 4)
    route_kernel<DT, EPL, false, 4>
        <<<(unsigned)a.blocks, 256, lds_bytes(a, 4, 0), stream>>>(a);
  else
    route_kernel<DT, EPL, false, kMaxWaves>
        <<<(unsigned)a.blocks, 64 * kMaxWaves, lds_bytes(a, kMaxWaves, 0), stream>>>(a);
}
template <int DT>
void launch_route(const RouteArgs &a, bool one, int waves, hipStream_t stream) {
  if (a.experts <= 64) launch_route<DT, 1>(a, one, waves, stream);
  else if (a.experts <= 128) launch_route<DT, 2>(a, one, waves, stream);
  else if (a.experts <= 256) launch_route<DT, 4>(a, one, waves, stream);
  else launch_route<DT, 8>(a, one, waves, stream);
}

// Blocks of tokens, a token or more to every wave, at most kPlanBlocks.
void split_tokens(RouteArgs &a, int waves) {
  a.tokens_per_block = waves * cdiv(a.tokens, (int64_t)waves * kPlanBlocks);
  a.blocks = (int)cdiv(a.tokens, a.tokens_per_block);
  a.blocks_per_group = (int)cdiv(a.blocks, kPlaceGroups);
  a.count_stride = (a.experts + 1 + 3) / 4 * 4;
  a.bits = 1;
  while ((1 << a.bits) < a.experts + 1) ++a.bits;
}

}  // namespace

sparoa_status launch_expert_route(RouteArgs a, sparoa_dtype dt, hipStream_t stream) {
  // Work-groups of 4 waves where that spreads a lane's long work over the CUs (64
  // tokens over 400 experts, top 8: 21.4 us with 16 waves, 16.1 so; over 64
  // experts 10.3 / 9.6, 1003 over 60 9.9 / 10.6).
  const int waves = a.tokens <= (a.experts > 64 ? 4 : 1) * kPlanBlocks ? 4 : kMaxWaves;
  split_tokens(a, waves);
  // One work-group up to half a token, one or two a wave (us, one launch against
  // two): 8 tokens over 400 experts 13.1 / 15.0, 16 17.8 / 15.4; 16 over 256 10.0
  // / 11.1, 32 13.9 / 11.4; 32 over 64 10.2 / 9.6 (top 2: 7.5 / 9.7), 64 15.3 / 9.6.
  const bool one = a.tokens <= (a.experts > 256 ? 8 : a.experts > 64 ? 16 : 32);
  if (one) {
    a.blocks = 1;
    a.tokens_per_block = a.tokens;
  }
  switch (dt) {
    case SPAROA_F32: launch_route<SPAROA_F32>(a, one, waves, stream); break;
    case SPAROA_F16: launch_route<SPAROA_F16>(a, one, waves, stream); break;
    default: launch_route<SPAROA_BF16>(a, one, waves, stream); break;
  }
  SPAROA_LAUNCH_CHECK("expert_route");
  if (one || !a.plan) return SPAROA_OK;
  place_kernel<<<(unsigned)cdiv(a.blocks, a.blocks_per_group), 64 * kMaxWaves,
                 lds_bytes(a, kMaxWaves, 0), stream>>>(a);
  SPAROA_LAUNCH_CHECK("expert_route: plan");
  return SPAROA_OK;
}

sparoa_status launch_expert_plan(RouteArgs a, hipStream_t stream) {
  split_tokens(a, kMaxWaves);
  const int64_t slots = a.tokens * a.top_k;
  if (slots <= kOneGroupSlots) {
    a.tokens_per_block = a.tokens;
    if (slots <= 256)
      count_kernel<true, 4><<<1, 256, lds_bytes(a, 4, 0), stream>>>(a);
    else
      count_kernel<true, kMaxWaves>
          <<<1, 64 * kMaxWaves, lds_bytes(a, kMaxWaves, 0), stream>>>(a);
    SPAROA_LAUNCH_CHECK("expert_plan");
    return SPAROA_OK;
  }
  count_kernel<false, kMaxWaves>
      <<<(unsigned)a.blocks, 64 * kMaxWaves, lds_bytes(a, kMaxWaves, 0), stream>>>(a);
  SPAROA_LAUNCH_CHECK("expert_plan: counts");
  place_kernel<<<(unsigned)cdiv(a.blocks, a.blocks_per_group), 64 * kMaxWaves,
                 lds_bytes(a, kMaxWaves, 0), stream>>>(a);
  SPAROA_LAUNCH_CHECK("expert_plan");
  return SPAROA_OK;
}

size_t expert_plan_workspace(int64_t tokens, int64_t experts) {
  RouteArgs a{};
  a.tokens = tokens;
  a.experts = (int)experts;
  split_tokens(a, 4);   // (16 waves give as many blocks, or fewer)
  return (size_t)a.blocks * (size_t)a.count_stride * 4;
}

}  // namespace sparoa

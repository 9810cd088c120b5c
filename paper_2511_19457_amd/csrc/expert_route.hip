// Routing to experts and the dispatch plan.
//
// route: a wave per token, lane l holding the EPL experts l EPL .. l EPL +
// EPL - 1.  The k choices are k rounds of a wave-wide maximum; the lowest
// lane that holds it, and in it the lowest expert, wins a tie.  Keys are
// compared as the formula gives them (softmax or sigmoid, plus bias); where
// only their order matters (no bias, no sum over a group) the logits are
// compared, which have the same order and never meet in a rounding.
//
// plan: a stable counting sort of the (token, choice) slots by expert.  Every
// place follows from counts alone, never from the order in which atomics
// land, so the plan of equal choices is equal.
//   one work-group (few slots): counts, offsets and places in LDS;
//   else two launches: each block of tokens leaves its counts (the route
//   kernel itself where it has just chosen), then every work-group adds up
//   the counts before its own blocks and places its slots.
#include <algorithm>

#include "block.h"
#include "dtype.h"

namespace sparoa {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
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

__device__ __forceinline__ float wave_add(float v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
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
// others, which hold -1).  cnt: kWaves x (experts + 1) words of LDS.
template <class ExpertOf>
__device__ __forceinline__ void place_slots(int64_t s0, int64_t s1, int experts, int bits,
                                            const uint32_t *first, uint32_t *cnt,
                                            int32_t *order, int32_t *place, ExpertOf expert_of) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, nb = experts + 1;
  // wave w has the w-th run of whole 64s
  const int64_t per = ((s1 - s0 + 63) / 64 + kWaves - 1) / kWaves * 64;
  const int64_t b = s0 + wave * per, e_ = b + per < s1 ? b + per : s1;
  for (int i = tid; i < kWaves * nb; i += kThreads) cnt[i] = 0;
  __syncthreads();
  for (int64_t s = b + lane; s < e_; s += 64) atomicAdd(&cnt[wave * nb + expert_of(s)], 1u);
  __syncthreads();
  for (int e = tid; e < nb; e += kThreads) {
    uint32_t at = first[e];
    for (int w = 0; w < kWaves; ++w) {
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
    lpg = 64;
    while (lpg * a.groups > 64) lpg >>= 1;
    const int per = a.experts / a.groups;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const int e = lane * EPL + i;
      bias[i] = a.bias && e < a.experts ? a.bias[e] : 0.f;
      group_lane[i] = min(e, a.experts - 1) / per * lpg;
    }
  }

  // Routes token t (the whole wave); chosen: LDS words for the keys of one
  // wave, used where there are groups.  Afterwards lane j < top_k holds choice
  // j (-1: none) and its weight.
  __device__ void token(int64_t t, float *scratch, int &choice, float &weight) {
    const raw *row = reinterpret_cast<const raw *>(a.logits) + t * a.experts;
    const bool live = !a.token_mask || a.token_mask[t] != 0;
    float l[EPL], key[EPL];
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const int e = lane * EPL + i;
      l[i] = live && e < a.experts ? E::to_f32(row[e]) : kLow;
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
    if (a.groups > 1) {
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
      const float score = a.group_best == 2 && b2 > kLow ? b1 + b2 : b1;
      int rank = 0;
      for (int o = 0; o < a.groups; ++o) {
        const float s = __builtin_bit_cast(
            float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, score), o * lpg));
        rank += s > score || (s == score && o < g) ? 1 : 0;
      }
      const uint64_t keep = __ballot(g < a.groups && rank < a.top_groups && score > kLow);
#pragma unroll
      for (int i = 0; i < EPL; ++i) key[i] = keep >> group_lane[i] & 1 ? key[i] : kLow;
      wave_fence();
    }
    choice = -1;
    float chosen = kLow;   // lane j: the logit of choice j
    for (int j = 0; j < a.top_k; ++j) {
      float best = key[0], bl = l[0];
      int bi = 0;
#pragma unroll
      for (int i = 1; i < EPL; ++i)
        if (key[i] > best) best = key[i], bl = l[i], bi = i;
      const float m = wave_max(best);
      if (!(m > kLow)) break;
      const int w = __ffsll((unsigned long long)__ballot(best == m)) - 1;
      const int e = w * EPL + __builtin_amdgcn_readlane(bi, w);
      const float el = __builtin_bit_cast(
          float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, bl), w));
      if (lane == j) choice = e, chosen = el;
#pragma unroll
      for (int i = 0; i < EPL; ++i)
        if (lane * EPL + i == e) key[i] = kLow;
    }
    // weights: of the choices alone where they are renormalised (the softmax's
    // own sum cancels, and choices far below the row's largest logit keep
    // their ratios)
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
};

__device__ __forceinline__ int slot_expert(const int32_t *idx, int64_t s, int experts) {
  const int e = idx[s];
  return (uint32_t)e < (uint32_t)experts ? e : experts;
}

// Routes a block of tokens_per_block tokens a work-group.  ONE: the only
// work-group, which also makes the plan (choices kept in LDS).
template <int DT, int EPL, bool ONE>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a) {
  extern __shared__ uint32_t lds[];
  const int nb = a.experts + 1, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  // [counts nb][first nb][keys of each wave, or the waves' counts][ONE: choices]
  uint32_t *total = lds, *first = lds + nb, *scratch = first + nb;
  int32_t *mine = reinterpret_cast<int32_t *>(scratch + kWaves * nb);
  for (int i = threadIdx.x; i < nb; i += kThreads) total[i] = 0;
  __syncthreads();
  Router<DT, EPL> r(a);
  const int64_t t0 = (int64_t)blockIdx.x * a.tokens_per_block;
  const int64_t t1 = t0 + a.tokens_per_block < a.tokens ? t0 + a.tokens_per_block : a.tokens;
  for (int64_t t = t0 + wave; t < t1; t += kWaves) {
    int choice;
    float weight;
    r.token(t, reinterpret_cast<float *>(scratch + wave * nb), choice, weight);
    if (lane < a.top_k) {
      a.idx[t * a.top_k + lane] = choice;
      a.weights[t * a.top_k + lane] = weight;
      if (a.plan) {
        const int e = choice >= 0 ? choice : a.experts;
        atomicAdd(&total[e], 1u);
        if (ONE) mine[t * a.top_k + lane] = e;
      }
    }
  }
  if (!a.plan) return;
  __syncthreads();
  if (ONE) {
    scan_counts(total, first, nb);
    __syncthreads();
    write_head(total, first, a.experts, a.plan);
    place_slots(0, a.tokens * a.top_k, a.experts, a.bits, first, scratch, a.order, a.place,
                [&](int64_t s) { return mine[s]; });
  } else {
    for (int i = threadIdx.x; i < nb; i += kThreads)
      a.counts[(int64_t)blockIdx.x * nb + i] = total[i];
  }
}

// Counts of given choices, a block of slots a work-group.  ONE: the only
// work-group, which also makes the plan.
template <bool ONE>
__global__ __launch_bounds__(kThreads) void count_kernel(RouteArgs a) {
  extern __shared__ uint32_t lds[];
  const int nb = a.experts + 1;
  uint32_t *total = lds, *first = lds + nb, *scratch = first + nb;
  for (int i = threadIdx.x; i < nb; i += kThreads) total[i] = 0;
  __syncthreads();
  const int64_t slots = a.tokens * a.top_k, per = a.tokens_per_block * a.top_k;
  const int64_t s0 = blockIdx.x * per, s1 = s0 + per < slots ? s0 + per : slots;
  for (int64_t s = s0 + threadIdx.x; s < s1; s += kThreads)
    atomicAdd(&total[slot_expert(a.idx, s, a.experts)], 1u);
  __syncthreads();
  if (ONE) {
    scan_counts(total, first, nb);
    __syncthreads();
    write_head(total, first, a.experts, a.plan);
    place_slots(0, slots, a.experts, a.bits, first, scratch, a.order, a.place,
                [&](int64_t s) { return slot_expert(a.idx, s, a.experts); });
  } else {
    for (int i = threadIdx.x; i < nb; i += kThreads)
      a.counts[(int64_t)blockIdx.x * nb + i] = total[i];
  }
}

// Places the slots of blocks_per_group blocks a work-group.
__global__ __launch_bounds__(kThreads) void place_kernel(RouteArgs a) {
  extern __shared__ uint32_t lds[];
  const int nb = a.experts + 1;
  uint32_t *total = lds, *first = lds + nb, *scratch = first + nb;
  uint32_t *before = scratch;   // until place_slots takes the scratch
  for (int i = threadIdx.x; i < nb; i += kThreads) total[i] = before[i] = 0;
  __syncthreads();
  // 1024 threads as rows x experts: each adds up every rows-th block's counts
  const int width = 1 << a.bits, rows = kThreads / width;
  const int e = threadIdx.x & (width - 1), b0 = blockIdx.x * a.blocks_per_group;
  if (e < nb) {
    uint32_t all = 0, mine = 0;
#pragma unroll 8
    for (int b = threadIdx.x >> a.bits; b < a.blocks; b += rows) {
      const uint32_t c = a.counts[(int64_t)b * nb + e];
      all += c;
      mine += b < b0 ? c : 0;
    }
    atomicAdd(&total[e], all);
    atomicAdd(&before[e], mine);
  }
  __syncthreads();
  scan_counts(total, first, nb);
  __syncthreads();
  if (blockIdx.x == 0) write_head(total, first, a.experts, a.plan);
  __syncthreads();
  for (int i = threadIdx.x; i < nb; i += kThreads) first[i] += before[i];
  __syncthreads();
  const int64_t slots = a.tokens * a.top_k;
  const int64_t per = a.tokens_per_block * a.top_k * a.blocks_per_group;
  const int64_t s0 = blockIdx.x * per, s1 = s0 + per < slots ? s0 + per : slots;
  place_slots(s0, s1, a.experts, a.bits, first, scratch, a.order, a.place,
              [&](int64_t s) { return slot_expert(a.idx, s, a.experts); });
}

template <int DT, int EPL>
void launch_route(const RouteArgs &a, bool one, unsigned lds, hipStream_t stream) {
  if (one)
    route_kernel<DT, EPL, true><<<1, kThreads, lds, stream>>>(a);
  else
    route_kernel<DT, EPL, false><<<(unsigned)a.blocks, kThreads, lds, stream>>>(a);
}
template <int DT>
void launch_route(const RouteArgs &a, bool one, unsigned lds, hipStream_t stream) {
  if (a.experts <= 64) launch_route<DT, 1>(a, one, lds, stream);
  else if (a.experts <= 128) launch_route<DT, 2>(a, one, lds, stream);
  else if (a.experts <= 256) launch_route<DT, 4>(a, one, lds, stream);
  else launch_route<DT, 8>(a, one, lds, stream);
}

unsigned lds_bytes(const RouteArgs &a, int64_t kept) {
  return (unsigned)(4 * ((2 + kWaves) * (a.experts + 1) + kept));
}

// Blocks of tokens, a token or more to every wave, at most kPlanBlocks.
void split_tokens(RouteArgs &a) {
  a.tokens_per_block = kWaves * cdiv(a.tokens, (int64_t)kWaves * kPlanBlocks);
  a.blocks = (int)cdiv(a.tokens, a.tokens_per_block);
  a.blocks_per_group = (int)cdiv(a.blocks, kPlaceGroups);
  a.bits = 1;
  while ((1 << a.bits) < a.experts + 1) ++a.bits;
}

}  // namespace

sparoa_status launch_expert_route(RouteArgs a, sparoa_dtype dt, hipStream_t stream) {
  split_tokens(a);
  // one work-group up to four tokens a wave
  const bool one = a.tokens <= 4 * kWaves;
  if (one) {
    a.blocks = 1;
    a.tokens_per_block = a.tokens;
  }
  const unsigned lds = lds_bytes(a, one ? a.tokens * a.top_k : 0);
  switch (dt) {
    case SPAROA_F32: launch_route<SPAROA_F32>(a, one, lds, stream); break;
    case SPAROA_F16: launch_route<SPAROA_F16>(a, one, lds, stream); break;
    default: launch_route<SPAROA_BF16>(a, one, lds, stream); break;
  }
  SPAROA_LAUNCH_CHECK("expert_route");
  if (one || !a.plan) return SPAROA_OK;
  place_kernel<<<(unsigned)cdiv(a.blocks, a.blocks_per_group), kThreads, lds_bytes(a, 0),
                 stream>>>(a);
  SPAROA_LAUNCH_CHECK("expert_route: plan");
  return SPAROA_OK;
}

sparoa_status launch_expert_plan(RouteArgs a, hipStream_t stream) {
  split_tokens(a);
  if (a.tokens * a.top_k <= kOneGroupSlots) {
    a.tokens_per_block = a.tokens;
    count_kernel<true><<<1, kThreads, lds_bytes(a, 0), stream>>>(a);
    SPAROA_LAUNCH_CHECK("expert_plan");
    return SPAROA_OK;
  }
  count_kernel<false><<<(unsigned)a.blocks, kThreads, lds_bytes(a, 0), stream>>>(a);
  SPAROA_LAUNCH_CHECK("expert_plan: counts");
  place_kernel<<<(unsigned)cdiv(a.blocks, a.blocks_per_group), kThreads, lds_bytes(a, 0),
                 stream>>>(a);
  SPAROA_LAUNCH_CHECK("expert_plan");
  return SPAROA_OK;
}

size_t expert_plan_workspace(int64_t tokens, int64_t experts) {
  RouteArgs a{};
  a.tokens = tokens;
  a.experts = (int)experts;
  split_tokens(a);
  return (size_t)a.blocks * (size_t)(experts + 1) * 4;
}

}  // namespace sparoa

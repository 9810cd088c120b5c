// Attention of rows over a paged cache.
//
// For the rows (token, head of the group) of one request and one kv head:
//   S^T = K Q^T by MFMA, a lane holding 16 of every 32 keys' scores of one row;
//   p = 2^(c s - m), m the row's maximum so far, l its sum, both in the lane;
//   O^T += V^T P^T by MFMA: the lane's own p are this product's operand, since a
//   product over keys asks for no order of them, and V^T comes out of LDS by the
//   transposing read.  So no score leaves its lane and a row's factors meet its
//   outputs there.
// Keys and values go from memory to a ring of two stages in LDS by the loads
// themselves.  Work is cut into items (row tile, range of keys) of like size from the
// lengths on the device, by every wave for itself or, above 64 requests, by a kernel in
// front; the ranges of a row tile that has several are joined by a kernel behind.
#include <algorithm>

#include "cache.h"
#include "rows_ring.h"

namespace sparoa {
namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr int kWaveRows = 32, kTileRows = kWaves * kWaveRows;
constexpr int kMaxRanges = 64;     // of a row: a step of the join
// Items that the work is cut into.  Few rows: small ranges even the load out and cost
// little; many: a range's outputs pass through memory, so a row tile is cut only where
// it is longer than what 320 of the 512 resident work-groups would have each, in fp32,
// whose products take longer, 448 (64 decoding requests: 512 237 us, 768 217, 1024 222,
// 2048 223; 12 chunks of prompts: 320 56, 448 56, 512 90; 32 trees: 320 150, 448 170;
// 5 fp32 prompts: 320 35, 448 31, 640 31).
constexpr int kTargetFew = 1024, kTargetMany = 320, kTargetF32 = 448;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 8.f;      // a maximum may lag by 2^8 before sums are scaled

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

// Bytes of zeros: what lanes past the head's last dimension read.
__device__ const uint4 kZeros[1] = {};

// Pieces of a head: D (head_dim padded to 64, 96, 128, 192 or 256) in rows of 128 bytes'
// multiples, key tiles of KT rows.
template <int DT, int D>
struct Shape {
  static constexpr int size = Elem<DT>::size, row = (D * size + 127) / 128 * 128;
  static constexpr int vectors = row / 16;
  static constexpr int pitch = D <= 64 ? 64 : D <= 128 ? 128 : 256;   // of a range's outputs
  static constexpr int keys = row <= 256 ? 64 : 32;
  static constexpr int tile = keys * row, stage = 2 * tile, lds = 2 * stage;
  static constexpr int loads = keys * vectors / (64 * kWaves);   // a wave's, of K or V
  // Vector v of a tile's row r lies at vector v ^ (swizzle of r): LDS has 64 banks of 4
  // bytes, and the lanes that are served together (16 of 16 bytes: 16 rows of K; 32 of
  // 8: 4 rows of 64 bytes of V; 64 of 4: 2 rows of 128) shall meet all of them.
  __device__ static constexpr int swizzle_k(int r) { return vectors % 16 ? r >> 1 & 7 : r & 15; }
  __device__ static constexpr int swizzle_v(int r) {
    if (size == 4) return vectors % 16 ? 0 : 8 * (r >> 2 & 1);
    return vectors % 16 ? 4 * (r >> 1 & 1) : 4 * (r & 3);
  }
  static constexpr int groups = lds <= 64 * 1024 && D <= 128 ? 2 : 1;   // a CU's
};
inline int padded_dim(int64_t dim) {
  return dim <= 64 ? 64 : dim <= 96 ? 96 : dim <= 128 ? 128 : dim <= 192 ? 192 : 256;
}
inline int output_pitch(int64_t dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }
inline int tile_keys(int64_t dim, sparoa_dtype dt) {
  return (padded_dim(dim) * elem_size(dt) + 127) / 128 * 128 <= 256 ? 64 : 32;
}

// 16 elements of K (8 a lane) of a 32 x 32 block.
template <int DT>
struct Piece;
template <>
struct Piece<SPAROA_F32> {
  u32x4 v[2];
};
template <>
struct Piece<SPAROA_F16> {
  u32x4 v[1];
};
template <>
struct Piece<SPAROA_BF16> {
  u32x4 v[1];
};
template <int DT>
__device__ __forceinline__ f32x16 mma32(const Piece<DT> &a, const Piece<DT> &b, f32x16 acc) {
  if constexpr (DT == SPAROA_BF16) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a.v[0]),
                                                   __builtin_bit_cast(bf16x8, b.v[0]), acc, 0, 0, 0);
  } else if constexpr (DT == SPAROA_F16) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a.v[0]),
                                                  __builtin_bit_cast(f16x8, b.v[0]), acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.v[i / 4][i % 4]),
                                                 __uint_as_float(b.v[i / 4][i % 4]), acc, 0, 0, 0);
    return acc;
  }
}

// A 16-byte load whose data goes to LDS (lane l's to lds + 16 l, lds uniform); in
// assembly so that the compiler waits where the ring does (see ring_load).
__device__ __forceinline__ void cache_load(const void *p, uint32_t lds) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %1, off" : : "{m0}"(lds), "v"(p) : "memory");
}

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32); }

// ------------------------------------------------------------ split of the work

struct Item {
  int r, start, n, len;   // request (n 0: no item), its first row, rows, keys
  int row0;               // first row (token, group head) of the tile
  int slot, chunk, chunks;   // number `chunk` of the row tile's ranges of keys
};

// Row tiles of a request, key tiles that one of them reaches at most, and its work: half
// keys that its row tiles reach (on average, as far as lengths tell; not below half of the
// most).  Whole numbers: the kernels that find the split each for themselves add them in
// any order to the same sum.
struct Load {
  int tiles, spans;
  int64_t work;
};
__device__ __forceinline__ Load load_of(const AttnArgs &a, const KvRequest &q, int keys) {
  Load l{0, 0, 0};
  if (!q.n) return l;
  l.tiles = (q.n * a.kv.group + kTileRows - 1) / kTileRows;
  int reach = q.len;
  uint32_t mean2 = 2 * (uint32_t)q.len;
  if (a.causal && !a.mask) {
    if (a.window) reach = min(q.len, a.window + kTileRows / a.kv.group + 1);
    mean2 = min(mean2 - (uint32_t)q.n, 2 * (uint32_t)reach);
  }
  // (a window begins within a tile; no more than there are)
  l.spans = min((reach - 1) / keys + 2, (q.len - 1) / keys + 1);
  l.work = (int64_t)l.tiles * max(mean2, (uint32_t)(l.spans * keys));
  return l;
}

// The sum of all lanes' work (at most 2^51 of a lane's: there every row tile is one range),
// by moves between lanes; where one passes 26 bits, those and the rest by themselves.
__device__ __forceinline__ int64_t wave_work(int64_t work) {
  const uint32_t low =
      __builtin_amdgcn_readlane(wave_prefix((int)(work & ((1 << 26) - 1))), 63);
  if (!__any(work >> 26)) return low;
  const int high = wave_prefix((int)(min(work, (int64_t)1 << 51) >> 26));
  return ((int64_t)(uint32_t)__builtin_amdgcn_readlane(high, 63) << 26) + low;
}
// Key tiles of an item: the whole work over the wanted items.
__device__ __forceinline__ int chunk_of(const AttnArgs &a, int64_t work, int keys) {
  const float each = (float)work * (float)a.kv.kv_heads / (2.f * (float)keys * (float)a.target);
  return each < 1e9f ? max(1, (int)ceilf(each)) : 1 << 30;
}

// Ranges of a request's row tiles.  A range's outputs pass through memory twice (4
// bytes each), which shall not be more than twice what its keys and values do.
__device__ __forceinline__ int ranges_of(const AttnArgs &a, const KvRequest &q, const Load &l,
                                         int chunk, int keys) {
  const int rows = min(q.n * a.kv.group, kTileRows);
  const int least = (rows * 2 + keys * a.elem - 1) / (keys * a.elem);
  const int size = max(max(chunk, least), (l.spans + kMaxRanges - 1) / kMaxRanges);
  return (l.spans + size - 1) / size;
}

// A request's share of the work: its items (row tiles times ranges), those whose outputs
// are joined, and the row tiles that are.
struct Share {
  int items, slots, splits;
};
__device__ __forceinline__ Share share_of(const Load &l, int chunks) {
  const int items = l.tiles * chunks;
  return Share{items, chunks > 1 ? items : 0, chunks > 1 ? l.tiles : 0};
}

// Up to 64 requests every wave works the split out by itself, a lane a request.  More
// are planned by a kernel in front: plan[0] is the chunk, then, for every request and
// behind the last, the items, slots and split row tiles before it (arrays of
// requests + 1).
constexpr int kLaneRequests = 64;
constexpr int kPlanThreads = 1024;
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(AttnArgs a, int keys) {
  __shared__ int64_t work_of[kPlanThreads / 64];
  __shared__ int before[kPlanThreads / 64][3];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.kv.requests;
  int64_t work = 0;
  for (int r = tid; r < n; r += kPlanThreads)
    work = min(work + load_of(a, kv_request(a.kv, r), keys).work, (int64_t)1 << 51);
  work = wave_work(work);
  if (lane == 0) work_of[wave] = work;
  __syncthreads();
  work = 0;
  for (int w = 0; w < kPlanThreads / 64; ++w) work += work_of[w];
  const int chunk = chunk_of(a, work, keys);
  int32_t *const items = a.plan + 1, *const slots = items + n + 1, *const splits = slots + n + 1;
  int sum[3] = {0, 0, 0};
  for (int r0 = 0; r0 < n; r0 += kPlanThreads) {
    const int r = r0 + tid;
    KvRequest q = kv_request(a.kv, min(r, n - 1));
    if (r >= n) q.n = 0;
    const Load l = load_of(a, q, keys);
    const Share s = share_of(l, ranges_of(a, q, l, chunk, keys));
    const int mine[3] = {s.items, s.slots, s.splits};
    int upto[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      upto[i] = wave_prefix(mine[i]);
      if (lane == 63) before[wave][i] = upto[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      int at = sum[i] + upto[i] - mine[i];
      for (int w = 0; w < kPlanThreads / 64; ++w) {
        if (w < wave) at += before[w][i];
        sum[i] += before[w][i];
      }
      if (r < n) (i == 0 ? items : i == 1 ? slots : splits)[r] = at;
    }
    __syncthreads();
  }
  if (tid == 0) a.plan[0] = chunk, items[n] = sum[0], slots[n] = sum[1], splits[n] = sum[2];
}

// The split as a wave sees it: items (or with TILES row tiles that are split) of a kv
// head by their number.
template <bool TILES>
struct Split {
  const AttnArgs &a;
  const int keys;
  // up to 64 requests: the lane's, and the sums up to the lane's place in the order
  KvRequest q;
  Load l;
  int chunks, rank, counted, upto, slots, slots_upto;

  __device__ __forceinline__ Split(const AttnArgs &args, int tile_keys)
      : a(args), keys(tile_keys) {
    if (a.plan) return;
    const int lane = threadIdx.x & 63;
    q = kv_request(a.kv, min(lane, a.kv.requests - 1));
    if (lane >= a.kv.requests) q.n = 0;
    l = load_of(a, q, keys);
    chunks = ranges_of(a, q, l, chunk_of(a, wave_work(l.work), keys), keys);
    // The requests of the longest ranges first where rows are many: 12 chunks of prompts 63
    // -> 55 us, 32 trees the same.  (Single rows are a stream, whose last ranges have the
    // memory to themselves: 64 requests 224 us in their order, 238 by length.)
    rank = lane;
    if (a.tile_rows > kWaveRows && a.kv.requests > 1) {
      const int size = chunks ? (l.spans + chunks - 1) / chunks : 0;
      rank = 0;
      for (int o = 0; o < a.kv.requests; ++o) {
        const int other = __builtin_amdgcn_readlane(size, o);
        rank += other > size || (other == size && o < lane);
      }
      if (lane >= a.kv.requests) rank = lane;
    }
    const Share s = share_of(l, chunks);
    counted = TILES ? s.splits : s.items, slots = s.slots;
    if (a.tile_rows > kWaveRows) {
      counted = __builtin_amdgcn_ds_permute(4 * rank, counted);
      slots = __builtin_amdgcn_ds_permute(4 * rank, slots);
    }
    upto = wave_prefix(counted), slots_upto = wave_prefix(slots);
  }

  __device__ __forceinline__ Item find(int id) const {   // (the whole wave)
    const int lane = threadIdx.x & 63;
    Item it{};
    int local, slot0, tiles;
    if (!a.plan) {
      const uint64_t past = __ballot(upto > id);
      if (!past) return it;
      const int w = __builtin_ctzll(past);   // its rank
      it.r = __builtin_ctzll(__ballot(rank == w));
      auto at = [&](int v) { return __builtin_amdgcn_readlane(v, it.r); };
      it.start = at(q.start), it.n = at(q.n), it.len = at(q.len);
      it.chunks = at(chunks), tiles = at(l.tiles);
      local = id - __builtin_amdgcn_readlane(upto - counted, w);
      slot0 = __builtin_amdgcn_readlane(slots_upto - slots, w);
    } else {
      const int n = a.kv.requests;
      const int32_t *const items = a.plan + 1, *const slots_of = items + n + 1;
      const int32_t *const before = TILES ? slots_of + n + 1 : items;
      if (id >= before[n]) return it;
      // the last request that begins at id or before (64 ways a step)
      int at = 0, left = n;
      while (left > 1) {
        const int step = (left + 63) / 64, probe = at + lane * step;
        const uint64_t below = __ballot(lane * step < left && before[min(probe, n)] <= id);
        const int last = below ? 63 - __builtin_clzll(below) : 0;
        at += last * step;
        left = min(step, left - last * step);
      }
      it.r = __builtin_amdgcn_readfirstlane(at);
      const KvRequest mine = kv_request(a.kv, it.r);
      if (!mine.n) return it;
      const Load load = load_of(a, mine, keys);
      it.start = mine.start, it.n = mine.n, it.len = mine.len;
      it.chunks = ranges_of(a, mine, load, a.plan[0], keys);
      tiles = load.tiles, local = id - before[it.r], slot0 = slots_of[it.r];
    }
    // (sums that passed 2^31: requests that claim each other's rows)
    if ((uint32_t)local >= (uint32_t)(TILES ? tiles : tiles * it.chunks)) return Item{};
    // (row tiles innermost, the last rows, which see most, first)
    it.chunk = TILES ? 0 : local / tiles;
    const int tile = local - it.chunk * tiles;
    it.row0 = (tiles - 1 - tile) * kTileRows;
    it.slot = slot0 + tile + it.chunk * tiles;   // (TILES: range c has slot + c tiles)
    return it;
  }
};

// The least (or greatest) of all lanes' numbers, by moves between lanes within the
// vector unit (through LDS the same takes six of its latencies).
template <bool LEAST>
__device__ __forceinline__ int wave_limit(int v) {
#define SPAROA_DPP_LIMIT(ctrl, rows)                                             \
  {                                                                              \
    const int o = __builtin_amdgcn_update_dpp(v, v, ctrl, rows, 0xF, false);     \
    v = LEAST ? min(v, o) : max(v, o);                                           \
  }
  SPAROA_DPP_LIMIT(0x111, 0xF)
  SPAROA_DPP_LIMIT(0x112, 0xF)
  SPAROA_DPP_LIMIT(0x114, 0xF)
  SPAROA_DPP_LIMIT(0x118, 0xF)
  SPAROA_DPP_LIMIT(0x142, 0xA)
  SPAROA_DPP_LIMIT(0x143, 0xC)
#undef SPAROA_DPP_LIMIT
  return __builtin_amdgcn_readlane(v, 63);
}

// What row (token, group head) number `row` of a request sees, and where it lies.
struct Row {
  bool live;
  int token, head, pos, lo, hi;
  uint64_t bits;   // a tree's first 64
};
__device__ __forceinline__ Row row_of(const AttnArgs &a, const Item &it, int kv_head, int row) {
  Row o;
  o.live = row < it.n * a.kv.group;
  const int j = kv_quotient(o.live ? row : 0, a.kv.by_group);
  o.token = it.start + j;
  o.head = kv_head * a.kv.group + (o.live ? row : 0) - j * a.kv.group;
  o.pos = it.len - it.n + j;
  o.lo = 0, o.hi = it.len;
  o.bits = 0;
  if (a.mask) {
    o.bits = a.mask[(int64_t)o.token * a.mask_words];
    if (a.positions) o.pos = a.positions[o.token];
  } else if (a.causal) {
    o.hi = min(it.len, max(o.pos + 1, a.prefix ? a.prefix[it.r] : 0));
  }
  if (a.window) o.lo = max(0, o.pos - a.window + 1);
  if (a.mask) o.lo = min(o.lo, it.len - it.n);   // (bounds the context; nodes go by bits)
  if (a.first) o.lo = max(o.lo, a.first[o.token]);
  return o;
}

// Which of the 64 keys from k0 on a row sees, a bit a key.
__device__ __forceinline__ uint64_t low_bits(int n) {   // the n lowest, n of any size
  return n <= 0 ? 0 : n >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << n) - 1;
}
__device__ __forceinline__ uint64_t seen_keys(const AttnArgs &a, const Item &it, const Row &row,
                                              int k0) {
  if (!a.mask) return low_bits(row.hi - k0) & ~low_bits(row.lo - k0);
  const int context = it.len - it.n, first = k0 - context;   // the node at k0, or below 0
  uint64_t seen = low_bits(context - k0) & ~low_bits(row.lo - k0);
  if (first + 64 <= 0) return seen;
  const uint64_t *words = a.mask + (int64_t)row.token * a.mask_words;
  const int w = first >> 6, shift = first & 63;   // (w may be -1)
  uint64_t nodes = 0;
  // (the first word lies in registers: a load here waits for the tiles sent for before)
  if (w >= 0 && w < a.mask_words) nodes = (w ? words[w] : row.bits) >> shift;
  if (shift && w + 1 < a.mask_words) nodes |= (w + 1 ? words[w + 1] : row.bits) << (64 - shift);
  nodes &= low_bits(it.n - first) & ~low_bits(-first);
  if (a.window)   // nodes that lie too far back
#pragma nounroll
    for (int i = max(0, -first); i < min(64, it.n - first); ++i)
      if (row.pos - a.positions[it.start + first + i] >= a.window) nodes &= ~((uint64_t)1 << i);
  return seen | nodes;
}

// How far a row is from key k (a tree's nodes: by their positions).
__device__ __forceinline__ float distance(const AttnArgs &a, const Item &it, const Row &row,
                                          int k) {
  int at = k;
  if (a.mask) {
    const int node = k - (it.len - it.n);
    const int there = a.positions[it.start + min(max(node, 0), it.n - 1)];
    at = node < 0 ? k : there;
  }
  return fabsf((float)(row.pos - at));
}

// cap tanh(x), x = by s.  16-bit types: 1 - 2 / (1 + e^2x), off by about 2^-23 of the cap.
// That is less than 2^-14 in a score for caps up to kFewCap; above it, the series
// x - x^3 / 3 + 2 x^5 / 15 where |x| < 1/8 (off by 17 x^7 / 315, less than 2^-22 of x), so that
// the error is one of 2^-20 of the score, whatever the cap.
// (The series for every cap: 75 us against 60 for the capped chunks of prompts.)
constexpr float kFewCap = 256.f;

template <int DT, bool LARGE>
__device__ __forceinline__ float capped(float s, float cap, float by) {
  if constexpr (DT == SPAROA_F32) return cap * tanhf(s * by);
  const float far = cap - 2.f * cap * __builtin_amdgcn_rcpf(
                                    1.f + __builtin_amdgcn_exp2f(2.f * kLog2e * by * s));
  if (!LARGE) return far;
  const float x = by * s, x2 = x * x;
  const float near = cap * fmaf(x * x2, fmaf(x2, 2.f / 15.f, -1.f / 3.f), x);
  return fabsf(x) < 0.125f ? near : far;
}

// Outputs of one row tile's wave: lane l has row l & 31; register 16 b + r has
// dimension 32 b + 8 (r / 4) + 4 (l >> 5) + r % 4.
template <int DT, int D>
__device__ __forceinline__ void store_rows(const AttnArgs &a, const Row &row, int b,
                                           const f32x16 &o, float by) {
  const int half = (threadIdx.x & 63) >> 5;
  const int64_t at = ((int64_t)row.token * a.kv.heads + row.head) * a.kv.dim;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int d = 32 * b + 8 * g + 4 * half;
    if (!row.live || d >= a.kv.dim) continue;
    const float v[4] = {o[4 * g] * by, o[4 * g + 1] * by, o[4 * g + 2] * by, o[4 * g + 3] * by};
    store_elems<DT, 4>(a.out, at + d, v);
  }
}

// Whether a tile in LDS holds an infinity or NaN (an exponent of ones); the whole wave.
template <int DT>
__device__ __forceinline__ bool holds_bad(const char *tile, int bytes) {
  constexpr uint32_t kExp = DT == SPAROA_F32 ? 0x7F800000u : DT == SPAROA_F16 ? 0x7C007C00u
                                                                             : 0x7F807F80u;
  constexpr uint32_t kOne = DT == SPAROA_F32 ? 0x00800000u : DT == SPAROA_F16 ? 0x04000400u
                                                                             : 0x00800080u;
  uint32_t top = 0;   // (ones plus one carry to the sign's place)
#pragma unroll 4
  for (int i = 16 * (threadIdx.x & 63); i < bytes; i += 1024) {
    const u32x4 w = *reinterpret_cast<const u32x4 *>(tile + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) top |= (w[e] & kExp) + kOne;
  }
  return __any((top & (DT == SPAROA_F32 ? 0x80000000u : 0x80008000u)) != 0);
}

// Weights are 2^(c s - c m + up) as one fma of s, c and the rounded c m - up: a row's
// weights all have the same error, its sum of them too.  Behind 2^22 that rounding could
// pass the largest exponent there is: m is taken off first there.
// up: fp16 has 10 bits down to 2^-14 and none below 2^-25.  2^7 above the largest weight's
// size a long flat tail keeps its part of the sum (2^-32 of the largest weight a key is
// lost, half a step of an output for 2^20 keys), and a weight in front of a maximum that
// lags by 2^8 stays a number: 2^(7 + 8 + 1/2) at most, the half for what c m and its
// comparison are rounded by up to 2^22.
template <int DT>
struct Base {
  static constexpr float up = DT == SPAROA_F16 ? 7.f : 0.f;
  float shift, by;   // 2^(c (s - shift) - by)
  __device__ Base(float m, float c) {
    const float at = m == -__builtin_inff() ? 0.f : m * c;
    const bool large = fabsf(at) > 0x1p22f;
    shift = large ? m : 0.f, by = large ? -up : at - up;
  }
};
// What a row's weights, 2^(c (s - m) + left), have beside the maximum: `up`, and what the
// rounding of c m left out.
// Sums of weights by different maxima meet without it, or keys of like scores would weigh
// by the tile or range that they lie in (near 2^23 by up to half as much again).
template <int DT>
__device__ __forceinline__ float left_out(float m, float c) {
  const Base<DT> base(m, c);
  return m == -__builtin_inff() ? 0.f : base.shift != 0.f ? Base<DT>::up : fmaf(m, c, -base.by);
}
// Scores to log2: 2^(c s), s the product, or cap tanh(scale product / cap).
__device__ __forceinline__ float score_unit(const AttnArgs &a) {
  return a.cap > 0.f ? kLog2e : a.scale * kLog2e;
}

// The keys from .. to that each row sees, one by one, added to its sums (a weight by one
// score in both): m, l and acc, which are of weights 2^(c (s - m)) here.
template <int DT, int D>
__device__ __forceinline__ void add_seen(const AttnArgs &a, const Item &it, const Row &row,
                                         int kv_head, int from, int to, float c, float cap_by,
                                         float slope, float &m, float &l, f32x16 (&acc)[D / 32]) {
  const int half = (threadIdx.x & 63) >> 5;
  const int64_t q0 = ((int64_t)row.token * a.kv.heads + row.head) * a.kv.dim;
#pragma nounroll
  for (int k = from; k < min(to, it.len); ++k) {
    const int at = kv_row(a.kv, it.r, kv_head, k);
    if (at < 0 || !(row.live && (seen_keys(a, it, row, k) & 1))) continue;
    float x = 0.f;
    const int64_t k0 = (int64_t)at * a.kv.dim;
#pragma nounroll
    for (int d = 0; d < a.kv.dim; d += 4) {
      float qv[4], kv[4];
      load_elems<DT, 4>(a.q, q0 + d, qv);
      load_elems<DT, 4>(a.k, k0 + d, kv);
#pragma unroll
      for (int e = 0; e < 4; ++e) x = fmaf(qv[e], kv[e], x);
    }
    if (a.cap > 0.f) x = capped<DT, true>(x, a.cap, cap_by);
    if (a.slopes) x = fmaf(-slope, distance(a, it, row, k), x);
    const float top = fmaxf(m, x);   // (m, where x is NaN)
    if (top > m) {
      const float by = __builtin_amdgcn_exp2f((m - top) * c);
      m = top;
      l *= by;
#pragma unroll
      for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[b][i] *= by;
    }
    const float p = __builtin_amdgcn_exp2f((x - (m == -__builtin_inff() ? 0.f : m)) * c);
    if (half == 0) l += p;   // (l: the lane's own)
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int d = 32 * b + 8 * g + 4 * half;
        if (d >= a.kv.dim) continue;
        float v[4];
        load_elems<DT, 4>(a.v, k0 + d, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[b][4 * g + e] = fmaf(p, v[e], acc[b][4 * g + e]);
      }
  }
}

// A row tile's range of keys: 4 waves of 32 rows share every tile of keys and values.
// Many rows are bound by matrix and vector instructions alike (a tile of 64 keys takes a
// wave 1024 cycles of the one and some 1100 of the other, 2400 together): two work-groups
// a CU, one's products beside the other's weights.  2 x 4096 causal rows, 32 heads of 128,
// 8 kv heads, bf16: 305-335 us, 0.82-0.90 PFLOP/s; 64 single rows over 200 to 8000 keys:
// 218 us, the kernel 5.1 TB/s (256 of them, planned in front: 820 us, 5.3).  Built and dropped: the next tile's scores beside this
// one's weights (313 us against 305 then; fp32 42 against 35), 8 waves with rings of 4
// stages (325), a kernel for up to 32 rows with a ring a wave and no barrier (decoding
// 216 us against 221 then, one token 15.4 against 13.8).
template <int DT, int D>
__global__ __launch_bounds__(kThreads, (Shape<DT, D>::groups)) void attention_kernel(AttnArgs a,
                                                                                int id0) {
  using S = Shape<DT, D>;
  using E = Elem<DT>;
  constexpr int KT = S::keys, NB = KT / 32, DB = D / 32, NV = S::vectors;
  __shared__ __attribute__((aligned(1024))) char smem[S::lds];
  __shared__ int reach[kWaves][2];

  const int lane = threadIdx.x & 63, rl = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kv_head = blockIdx.x % a.kv.kv_heads, id = id0 + blockIdx.x / a.kv.kv_heads;
  const Item it = Split<false>(a, KT).find(id);
  if (!it.n) return;
  const int64_t slot = (int64_t)it.slot * a.kv.kv_heads + kv_head;

  const Row row = row_of(a, it, kv_head, it.row0 + wave * kWaveRows + rl);
  // the wave's range of keys, and the part that all its rows see
  const bool some = row.live && row.lo < row.hi;
  const int lo = wave_limit<true>(some ? row.lo : INT32_MAX);
  const int hi = wave_limit<false>(some ? row.hi : 0);
  const int all_lo = wave_limit<false>(row.live ? row.lo : 0);
  const int all_hi =
      wave_limit<true>(!row.live ? INT32_MAX : a.mask ? it.len - it.n : row.hi);
  if (lane == 0) reach[wave][0] = lo, reach[wave][1] = hi;
  __syncthreads();
  int tile_lo = INT32_MAX, tile_hi = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w)
    tile_lo = min(tile_lo, reach[w][0]), tile_hi = max(tile_hi, reach[w][1]);
  // this range of the key tiles that the rows reach
  const int begin = tile_lo / KT, reached = max(0, (tile_hi + KT - 1) / KT - begin);
  const int per = (reached + it.chunks - 1) / it.chunks;
  const int t0 = __builtin_amdgcn_readfirstlane(begin + min(it.chunk * per, reached));
  const int t1 = __builtin_amdgcn_readfirstlane(begin + min((it.chunk + 1) * per, reached));

  // ---- the ring: lane i of a wave knows the cache row of a tile's key i
  const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
  const int vectors = a.kv.dim * S::size / 16;
  const uint32_t row_bytes = (uint32_t)a.kv.dim * S::size;
  // (the page's number is only asked for; made use of a tile later, since its wait
  // would be one for the tile that was sent for before it, too)
  auto key_of = [&](int t) __attribute__((always_inline)) {
    return min(t * KT + (lane & (KT - 1)), it.len - 1);
  };
  const int32_t *const pages = a.kv.table + (int64_t)it.r * a.kv.table_pages;
  auto ask = [&](int t) __attribute__((always_inline)) {
    return pages[kv_quotient(key_of(t), a.kv.by_page)];
  };
  auto place = [&](int t, int page) __attribute__((always_inline)) {   // -1: no page
    const int k = key_of(t), in = kv_quotient(k, a.kv.by_page);
    const uint32_t at = ((uint32_t)page * a.kv.kv_heads + kv_head) * a.kv.page_size +
                        (k - in * a.kv.page_size);
    return (uint32_t)page < (uint32_t)a.kv.pages ? (int)at : -1;
  };
  auto load_rows = [&](const void *cache, int swizzle(int), const int (&at)[S::loads], uint32_t to)
                       __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < S::loads; ++u) {
      const int s = (u * kWaves + wave) * 64 + lane, r = s / NV, v = (s % NV) ^ swizzle(r);
      const char *const first = v < vectors ? reinterpret_cast<const char *>(cache) + 16 * v
                                            : reinterpret_cast<const char *>(kZeros);
      cache_load(first + (uint64_t)(uint32_t)at[u] * (v < vectors ? row_bytes : 0),
                 to + (u * kWaves + wave) * 1024);
    }
  };
  auto load_tile = [&](int at, int stage) __attribute__((always_inline)) {
    int row[S::loads];
#pragma unroll
    for (int u = 0; u < S::loads; ++u)
      row[u] = __builtin_amdgcn_ds_bpermute(4 * (((u * kWaves + wave) * 64 + lane) / NV), max(at, 0));
    load_rows(a.k, [](int r) { return S::swizzle_k(r); }, row, ring + stage * S::stage);
    load_rows(a.v, [](int r) { return S::swizzle_v(r); }, row, ring + stage * S::stage + S::tile);
  };

  // ---- the rows' queries, 16 dimensions a step
  constexpr int STEPS = D / 16, PV = S::size / 2;   // vectors of a lane's piece
  Piece<DT> q[STEPS];
  {
    const char *from = reinterpret_cast<const char *>(a.q) +
                       ((int64_t)row.token * a.kv.heads + row.head) * row_bytes;
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
      for (int e = 0; e < PV; ++e) {
        const int v = (2 * s + half) * PV + e;
        q[s].v[e] = v < vectors ? reinterpret_cast<const u32x4 *>(from)[v] : u32x4{0, 0, 0, 0};
      }
  }
  // (the bias by distance in units of 1 / c)
  const float c = score_unit(a);
  const float cap_by = a.cap > 0.f ? a.scale / a.cap : 0.f;
  const float slope = a.slopes ? a.slopes[row.head] / (a.cap > 0.f ? 1.f : a.scale) : 0.f;

  f32x16 acc[DB];
#pragma unroll
  for (int b = 0; b < DB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[b][i] = 0.f;
  float m = -__builtin_inff(), l = 0.f;   // (l: the lane's own keys)
  bool far = false;   // a row of the wave has a maximum behind 2^22
  // Tiles that hold an infinity or NaN beside keys that some row does not see (a weight of
  // 0 times it is NaN) are left to the end (behind the 64th with all that follow) and added
  // key by key: weight and value, since a score that is summed in another order is another
  // (by whole units behind 2^24).
  uint64_t put_off = 0;
  int put_off_from = INT32_MAX;

  int here = 0, page = 0;
  if (t0 < t1) {
    here = place(t0, ask(t0));
    load_tile(here, 0);
    page = ask(min(t0 + 1, t1 - 1));
  }
  for (int t = t0; t < t1; ++t) {
    const int stage = (t - t0) & 1;
    __builtin_amdgcn_s_waitcnt(vm_outstanding(0));
    __syncthreads();   // the tile is there, and the other stage is read
    const uint64_t pageless = __ballot(here < 0);
    if (t + 1 < t1) {
      here = place(t + 1, page);
      load_tile(here, stage ^ 1);
      page = ask(min(t + 2, t1 - 1));
    }
    const int k0 = t * KT;
    if (k0 >= hi || k0 + KT <= lo) continue;   // none of this wave's rows

    const char *keys = smem + stage * S::stage, *values = keys + S::tile;
    const bool hidden = k0 < all_lo || k0 + KT > all_hi || pageless;   // from some row
    if (t >= put_off_from || (hidden && holds_bad<DT>(values, S::tile))) {
      if (t - t0 < 64)
        put_off |= (uint64_t)1 << (t - t0);
      else
        put_off_from = min(put_off_from, t);
      continue;
    }
    constexpr int KA = 2, VA = 2;   // pieces that are read before their product
    f32x16 s[NB];
    {
      Piece<DT> k[KA + 1];
#pragma unroll
      for (int i = 0; i < NB * STEPS + KA; ++i) {   // (NB sums in turn: no product waits for one)
        if (i < NB * STEPS) {
          const int n = i % NB, st = i / NB;
#pragma unroll
          for (int e = 0; e < PV; ++e)
            k[i % (KA + 1)].v[e] = *reinterpret_cast<const u32x4 *>(
                keys + (32 * n + rl) * S::row +
                16 * (((2 * st + half) * PV + e) ^ S::swizzle_k(rl)));
        }
        if (i < KA) continue;
        const int n = (i - KA) % NB, st = (i - KA) / NB;
        if (st == 0)
#pragma unroll
          for (int e = 0; e < 16; ++e) s[n][e] = 0.f;
        s[n] = mma32<DT>(k[(i - KA) % (KA + 1)], q[st], s[n]);
      }
    }
    if (a.cap > kFewCap) {
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n][i] = capped<DT, true>(s[n][i], a.cap, cap_by);
    } else if (a.cap > 0.f) {
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n][i] = capped<DT, false>(s[n][i], a.cap, cap_by);
    }
    if (a.slopes) {   // (scores are in units of 1 / c here)
      if (!a.mask || k0 + KT <= it.len - it.n) {
        const int from = row.pos - k0 - 4 * half;
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            s[n][i] = fmaf(-slope, fabsf((float)(from - (32 * n + 8 * (i / 4) + i % 4))), s[n][i]);
      } else {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            s[n][i] = fmaf(-slope,
                           distance(a, it, row, k0 + 32 * n + 8 * (i / 4) + 4 * half + i % 4),
                           s[n][i]);
      }
    }
    if (hidden) {
      const uint64_t seen = (seen_keys(a, it, row, k0) & ~pageless) >> (4 * half);
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const int bits = (int)(uint32_t)(seen >> (32 * n));
#pragma unroll
        for (int i = 0; i < 16; ++i) {   // the bit as a mask: the score, or -infinity
          const int b = 8 * (i / 4) + i % 4, keep = (int)((uint32_t)bits << (31 - b)) >> 31;
          s[n][i] = __int_as_float((__float_as_int(s[n][i]) & keep) | (~keep & (int)0xFF800000));
        }
      }
    }
    float top = s[0][0];
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[n][i]);
    top = fmaxf(top, other_half(top));
    // (far: the two products can be alike where the scores are not; the first: its product
    // can be -infinity)
    if (__any(top * c > m * c + kSlack || ((far || m == -__builtin_inff()) && top > m))) {
      const float to = fmaxf(m, top);
      const float by = to == m ? 1.f : __builtin_amdgcn_exp2f(
          fmaf(m - to, c, left_out<DT>(to, c) - left_out<DT>(m, c)));
      m = to;
      far = __any(Base<DT>(m, c).shift != 0.f);
      l *= by;
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[b][i] *= by;
    }
    float base = (m == -__builtin_inff() ? 0.f : m * c) - Base<DT>::up;
    if (far) {
      const Base<DT> large(m, c);
      base = large.by;
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n][i] -= large.shift;
    }
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[n][i] = __builtin_amdgcn_exp2f(fmaf(s[n][i], c, -base));
        l += s[n][i];
      }
    Piece<DT> v[VA + 1], p;
#pragma unroll
    for (int i = 0; i < 2 * NB * DB + VA; ++i) {   // 16 keys of 32 dimensions
      if (i < 2 * NB * DB) {
        const int k0 = 16 * (i / DB), b = i % DB;
        if constexpr (DT == SPAROA_F32) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int r = k0 + 8 * (e / 4) + 4 * half + e % 4;
            v[i % (VA + 1)].v[e / 4][e % 4] = *reinterpret_cast<const uint32_t *>(
                values + r * S::row + 16 * ((8 * b + rl / 4) ^ S::swizzle_v(r)) + 4 * (rl & 3));
          }
        } else {
          // 16 lanes read 4 keys of 16 dimensions; lane i of them receives dimension i
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int r = k0 + 8 * x + 4 * half + ((lane & 15) >> 2);
            const int vec = (4 * b + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ S::swizzle_v(r);
            const char *from = values + r * S::row + 16 * vec + 8 * (lane & 1);
            const uint2 w = __builtin_bit_cast(
                uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                           (__attribute__((address_space(3))) i16x4 *)from));
            v[i % (VA + 1)].v[0][2 * x] = w.x, v[i % (VA + 1)].v[0][2 * x + 1] = w.y;
          }
        }
      }
      if (i < VA) continue;
      const int j = i - VA, u = j / DB, b = j % DB;
      // The lane's weights of these keys.  16-bit types round them once, as an operand
      // has to be: half a step each, without bias, which puts an output 1.4 times as far
      // from 64 bits as its own rounding does; their sum l is of the unrounded ones.
      if (b == 0) {
        if constexpr (DT == SPAROA_F32) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            p.v[e / 4][e % 4] = __float_as_uint(s[u / 2][8 * (u & 1) + e]);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            p.v[0][e] = E::pack2(s[u / 2][8 * (u & 1) + 2 * e], s[u / 2][8 * (u & 1) + 2 * e + 1]);
        }
      }
      acc[b] = mma32<DT>(v[j % (VA + 1)], p, acc[b]);
    }
  }

  float whole = __builtin_amdgcn_exp2f(-left_out<DT>(m, c));   // (to weights 2^(c (s - m)))
  if (put_off || put_off_from < t1) {
    l *= whole;
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[b][i] *= whole;
    whole = 1.f;
    for (int t = t0; t < t1; ++t)
      if (t >= put_off_from || (t - t0 < 64 && put_off >> (t - t0) & 1))
        add_seen<DT, D>(a, it, row, kv_head, t * KT, t * KT + KT, c, cap_by, slope, m, l, acc);
  }

  l += other_half(l);
  if (it.chunks == 1) {
    const float by = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int b = 0; b < DB; ++b) store_rows<DT, D>(a, row, b, acc[b], by);
    return;
  }
  if (slot < 0 || slot >= a.slots || !row.live || wave >= a.slot_waves) return;
  const int64_t part = (slot * a.slot_waves + wave) * kWaveRows + rl;
  if (half == 0) reinterpret_cast<float2 *>(a.ml)[part] = make_float2(m, l * whole);
  float *const o = reinterpret_cast<float *>(a.part) + part * S::pitch + 4 * half;
#pragma unroll
  for (int b = 0; b < DB; ++b)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<f32x4 *>(o + 32 * b + 8 * g) =
          f32x4{acc[b][4 * g] * whole, acc[b][4 * g + 1] * whole, acc[b][4 * g + 2] * whole,
                acc[b][4 * g + 3] * whole};
}

// Joins the ranges of a row tile: out = sum_r 2^(c (m_r - m)) o_r / sum_r 2^(c (m_r - m)) l_r.
// D / 4 lanes have a row; where a row has many ranges several such groups share them
// and meet in LDS, since the chain of loads is all that such a call takes.
template <int DT, int D>
__global__ __launch_bounds__(kThreads) void join_kernel(AttnArgs a, int step) {
  constexpr int KT = Shape<DT, D>::keys, LANES = Shape<DT, D>::pitch / 4;
  constexpr int GROUPS = kThreads / LANES;
  constexpr int AHEAD = 8;
  __shared__ f32x4 sums[GROUPS][LANES];
  __shared__ float2 stats[GROUPS];
  const int tid = threadIdx.x, group = tid / LANES, lane = tid % LANES;
  const Split<true> split(a, KT);
  const float c = score_unit(a);
  const int row_groups = (a.tile_rows + step - 1) / step;
  const int per = a.kv.kv_heads * row_groups;
  for (int u = blockIdx.x;; u += gridDim.x) {
    const int in = u % per, kv_head = in % a.kv.kv_heads, g = in / a.kv.kv_heads;
    const Item it = split.find(u / per);
    if (!it.n) return;
    const int rows = it.n * a.kv.group, tiles = (rows + kTileRows - 1) / kTileRows;
    if (it.row0 + g * step >= rows) continue;
    int share = 1;   // groups that share a row's ranges
    while (share * step < GROUPS && 2 * share <= it.chunks) share *= 2;
    const int part = group % share;
    for (int r0 = 0; r0 < step; r0 += GROUPS / share) {
      const int r = r0 + group / share, row = it.row0 + g * step + r;
      const bool live = r < step && row < rows;
      float m = -__builtin_inff(), l = 0.f;
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
      if (live)
        for (int c0 = part; c0 < it.chunks; c0 += AHEAD * share) {
          float2 ml[AHEAD];
          f32x4 o[AHEAD];
          bool has[AHEAD];
#pragma unroll
          for (int i = 0; i < AHEAD; ++i) {
            const int ch = c0 + i * share;
            const int64_t slot =
                ((int64_t)it.slot + (int64_t)min(ch, it.chunks - 1) * tiles) * a.kv.kv_heads +
                kv_head;
            has[i] = ch < it.chunks && slot >= 0 && slot < a.slots;
            const int64_t at = (has[i] ? slot : 0) * a.slot_waves * kWaveRows + g * step + r;
            ml[i] = reinterpret_cast<const float2 *>(a.ml)[at];
            o[i] = reinterpret_cast<const f32x4 *>(a.part)[at * LANES + lane];
          }
#pragma unroll
          for (int i = 0; i < AHEAD; ++i) {
            if (!has[i] || ml[i].y == 0.f) continue;   // (the range held nothing for this row)
            const float to = fmaxf(m, ml[i].x);
            const float old = m == to ? 1.f : __builtin_amdgcn_exp2f((m - to) * c);
            const float by = ml[i].x == to ? 1.f : __builtin_amdgcn_exp2f((ml[i].x - to) * c);
            m = to;
            l = fmaf(by, ml[i].y, l * old);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = fmaf(by, o[i][e], acc[e] * old);
          }
        }
      if (share > 1) {
        sums[group][lane] = acc;
        if (lane == 0) stats[group] = make_float2(m, l);
        __syncthreads();
        if (part == 0)
          for (int p = 1; p < share; ++p) {
            const float2 v = stats[group + p];
            const f32x4 x = sums[group + p][lane];
            if (v.y == 0.f) continue;
            const float to = fmaxf(m, v.x);
            const float old = m == to ? 1.f : __builtin_amdgcn_exp2f((m - to) * c);
            const float by = v.x == to ? 1.f : __builtin_amdgcn_exp2f((v.x - to) * c);
            m = to;
            l = fmaf(by, v.y, l * old);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = fmaf(by, x[e], acc[e] * old);
          }
        __syncthreads();
      }
      const int d = 4 * lane;
      if (!live || part || d >= a.kv.dim) continue;
      const int j = kv_quotient(row, a.kv.by_group);
      const int64_t to = ((int64_t)(it.start + j) * a.kv.heads + kv_head * a.kv.group +
                          (row - j * a.kv.group)) * a.kv.dim + d;
      const float by = l == 0.f ? 0.f : 1.f / l;
      const float v[4] = {acc[0] * by, acc[1] * by, acc[2] * by, acc[3] * by};
      store_elems<DT, 4>(a.out, to, v);
    }
  }
}

// Row tiles that the descriptor allows (a request that has some has a token).
int64_t most_tiles(const sparoa_kv_desc &d) {
  const int64_t group = d.heads / d.kv_heads;
  const int64_t queries = std::min(d.max_queries, d.tokens);
  const int64_t requests = std::min(d.requests, d.tokens);
  return std::min(requests * cdiv(queries * group, kTileRows),
                  d.tokens * group / kTileRows + requests);
}

struct Parts {
  int target, slots, slot_waves;
};
Parts attention_split(const sparoa_kv_desc &d) {
  const int64_t group = d.heads / d.kv_heads;
  Parts s;
  s.slot_waves = (int)std::min<int64_t>(
      kWaves, cdiv(std::min(d.max_queries, d.tokens) * group, kWaveRows));
  s.target = s.slot_waves == 1         ? kTargetFew
             : d.dtype == SPAROA_F32 ? kTargetF32
                                     : kTargetMany;
  // A request's row tiles that are split have ceil(spans / chunk) < 2 spans / chunk
  // ranges each, spans are at most twice their mean, and all means at most `target`
  // chunks.  (+ kv_heads: their quotient is rounded.)
  const int64_t chunks = cdiv(d.max_keys, tile_keys(d.head_dim, d.dtype));
  const int64_t most = most_tiles(d);
  const int64_t cap = 4 * s.target + 4 * d.kv_heads;
  s.slots = (int)(chunks <= 1 ? 0
                  : chunks < cap && most < cap && most * chunks < cap / d.kv_heads
                      ? most * chunks * d.kv_heads : cap);
  return s;
}
size_t ml_bytes(const Parts &s) {
  return (size_t)((int64_t)s.slots * s.slot_waves * kWaveRows * 8 + 255) / 256 * 256;
}

size_t plan_bytes(const sparoa_kv_desc &d) {
  return d.requests <= kLaneRequests ? 0 : (size_t)(12 * (d.requests + 1) + 4 + 255) / 256 * 256;
}

template <int DT, int D>
sparoa_status launch(const AttnArgs &a, int64_t tiles, hipStream_t stream) {
  // (by the work that they share, or by the ranges that a row tile can have)
  const int64_t ranges = std::min<int64_t>(kMaxRanges, cdiv(a.kv.max_keys, Shape<DT, D>::keys) + 1);
  const int64_t items = std::min(tiles + cdiv(2 * a.target, a.kv.kv_heads) + 2, tiles * ranges);
  if (items > INT32_MAX)
    return fail(SPAROA_ERR_UNSUPPORTED, "attention: 2^31 or more row tiles and ranges");
  if (a.plan) {
    plan_kernel<<<1, kPlanThreads, 0, stream>>>(a, Shape<DT, D>::keys);
    SPAROA_LAUNCH_CHECK("attention: plan");
  }
  // (2^31 threads a launch: a request of its own for every token makes an item of each)
  const int64_t most = (1 << 23) / a.kv.kv_heads;
  for (int64_t id0 = 0; id0 < items; id0 += most) {
    const unsigned grid = (unsigned)(std::min(items - id0, most) * a.kv.kv_heads);
    attention_kernel<DT, D><<<grid, kThreads, 0, stream>>>(a, (int)id0);
    SPAROA_LAUNCH_CHECK("attention");
  }
  if (a.slots) {
    // (a work-group a row where they are few altogether; else the lookups are made for
    // several: 64 requests of 4 rows a kv head 221 us with 1 each, 217 with 4)
    const int step = a.slot_waves == 1 ? (tiles * a.kv.kv_heads > 64 ? 4 : 1)
                                            : a.slot_waves == 2 ? 4 : 8;
    const unsigned grid = (unsigned)std::min<int64_t>(
        std::min<int64_t>(tiles, a.slots) * a.kv.kv_heads * cdiv(a.tile_rows, step),
        2048);
    join_kernel<DT, D><<<grid, kThreads, 0, stream>>>(a, step);
    SPAROA_LAUNCH_CHECK("attention: join");
  }
  return SPAROA_OK;
}
template <int DT>
sparoa_status launch_dim(const AttnArgs &a, int64_t tiles, hipStream_t stream) {
  switch (padded_dim(a.kv.dim)) {
    case 64: return launch<DT, 64>(a, tiles, stream);
    case 96: return launch<DT, 96>(a, tiles, stream);
    case 128: return launch<DT, 128>(a, tiles, stream);
    case 192: return launch<DT, 192>(a, tiles, stream);
    default: return launch<DT, 256>(a, tiles, stream);
  }
}

}  // namespace

size_t attention_workspace(const sparoa_kv_desc &d) {
  const Parts s = attention_split(d);
  return plan_bytes(d) + ml_bytes(s) + (size_t)((int64_t)s.slots * s.slot_waves * kWaveRows *
                                output_pitch(d.head_dim) * 4) + 256;
}

sparoa_status launch_attention(AttnArgs a, const sparoa_kv_desc &d, void *workspace,
                               hipStream_t stream) {
  const Parts s = attention_split(d);
  a.target = s.target, a.slots = s.slots, a.slot_waves = s.slot_waves;
  a.elem = (int)elem_size(d.dtype);
  a.tile_rows = (int)std::min<int64_t>(kTileRows, (int64_t)a.kv.max_queries * a.kv.group);
  char *const ws = reinterpret_cast<char *>(workspace);
  a.plan = d.requests <= kLaneRequests ? nullptr : reinterpret_cast<int32_t *>(ws);
  a.ml = ws + plan_bytes(d);
  a.part = ws + plan_bytes(d) + ml_bytes(s);
  const int64_t tiles = most_tiles(d);
  switch (d.dtype) {
    case SPAROA_F32: return launch_dim<SPAROA_F32>(a, tiles, stream);
    case SPAROA_F16: return launch_dim<SPAROA_F16>(a, tiles, stream);
    default: return launch_dim<SPAROA_BF16>(a, tiles, stream);
  }
}

}  // namespace sparoa

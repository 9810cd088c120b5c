// Products of many rows: MFMA tiles through LDS.
//
// A work-group has BM rows of one segment (an expert's gathered or consecutive
// rows, or an FC's) and BN rows of its weights; K runs in chunks of 128 bytes
// through a ring of S stages in LDS, sent there by the loads themselves.  One
// barrier a chunk; a wave reads the next chunk's operands and sends the loads
// that refill the stage the barrier freed between the MFMAs of the current
// chunk.  The MFMA's rows are weight rows, so a lane ends with 8 consecutive
// output channels of a row per block pair and the epilogue works from
// registers.  Gated: the pairs alternate between gate and up rows of the same
// channels, so the product gate * up is a lane's own.
// Low-rank adapters are chunks behind K's: for every adapter among the tile's
// rows, its rows of h (the others' read as zeros) against its matrix b.
// Bound by the matrix pipe and what feeds it: FC of 4096^3 bf16 128 us at least
// (1.07 PFLOP/s; 100 us with K's loads left out, 64 us at the pipe's rate), 143-157
// us in the median of 30 passes (the first ones are the fastest), the MFMAs busy
// half of the cycles; 4096 tokens over 64 experts (2048 x 1024 gated, top 8) at
// least 303 us up and 182 down, in the median 331 and 200.
// Work-groups are dealt round-robin to the 8 XCDs: XCD i takes the i-th run of
// tiles, column tiles innermost, so the tiles of one expert share an L2.
#include <algorithm>

#include "rows_ring.h"

namespace sparoa {
namespace {

// The lane's number, anew: what is derived from it is not kept in registers
// through the K loop.
__device__ __forceinline__ int fresh_lane(int lane) {
  asm volatile("" : "+v"(lane));
  return lane;
}

template <int DT, RowsMode MODE, int WGM, int WGN, int WTM, int WTN, int S>
__global__ __launch_bounds__(64 * WGM * WGN, 2) void rows_tile_kernel(RowsArgs a) {
  using E = Elem<DT>;
  using raw = typename E::raw;
  constexpr bool GATED = MODE == kRowsUpGated, FC = MODE == kRowsFc;
  constexpr int NW = WGM * WGN, BM = 16 * WGM * WTM, BN = 16 * WGN * WTN;
  constexpr int OC = GATED ? BN / 2 : BN;            // output columns
  constexpr int AV = BM / 8 / NW, BV = BN / 8 / NW;  // a wave's load covers 8 chunk rows
  static_assert(AV >= 1 && BV >= 1 && BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "tile too small");
  static_assert(WTN % 4 == 0 && NW % 2 == 0, "a lane's channels; weight row swizzle");
  constexpr int L = AV + BV;       // loads per wave and chunk
  constexpr int NG = WTN / 4;      // groups of 64 weight rows of a wave
  // the stages of x, then those of the weights (offsets that fit an LDS read)
  constexpr int XS = BM * kRow, WS = BN * kRow, W0 = S * XS;
  __shared__ __attribute__((aligned(1024))) char smem[S * (XS + WS) + (FC ? NW * 1024 : 0)];
  __shared__ int32_t list[FC ? BM : 1];
  __shared__ int list_len;
  __shared__ int32_t cum[MODE <= kRowsDown ? kMaxExperts : 1];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WGN, wn = wave % WGN;
  TileWalk<MODE, BM> walk{a, cum};
  if constexpr (walk.kExperts) {
    if (wave == 0) walk.fill(a, cum);
    __syncthreads();
  }
  walk.start((a.n + OC - 1) / OC);
  Tile tl = walk.next();
  if (tl.end == 0) return;
  const int kbytes = a.k * E::size;
  const int n = (kbytes + kRow - 1) / kRow;

  // ---- this lane's share of the loads: slot lane & 7 of chunk row lane >> 3.
  // Rows hold their 16-byte vectors swizzled, slot = vector ^ f(row), so that
  // the operand reads of 8 consecutive lanes meet distinct banks: rows of x f =
  // row & 7; weight rows, read in the order that leaves a lane 8 consecutive
  // channels (MFMA row 4 q + t of block b is tile row 32 (b / 2) + 8 q + 4 (b %
  // 2) + t), f = (row >> 3 & 1) * 4 + (row & 3).
  auto vector_a = [&](int l) { return (l & 7) ^ (l >> 3); };
  auto vector_b = [&](int l) { return (l & 7) ^ (((wave & 1) << 2) | (l >> 3 & 3)); };
  constexpr bool gather = MODE <= kRowsUpGated;
  // bits that put a lane's piece of the last chunk out of range, past K
  const int tail = kbytes - (n - 1) * kRow;

  // What a tile's rows are known by: their slots (gathered) or adapters.
  int place[AV], member[FC ? (BM + 63) / 64 : 1];
  auto fetch = [&](const Tile &t) __attribute__((always_inline)) {
    const int rows = (int)std::min<int64_t>(t.end - t.row0, BM);
    const int lane = fresh_lane(threadIdx.x & 63), lrow = lane >> 3;
    if constexpr (gather || FC) {
      if (!gather && !a.ids) return;
#pragma unroll
      for (int u = 0; u < AV; ++u) {
        const int64_t r = t.row0 + min(8 * (u * NW + wave) + lrow, rows - 1);
        place[u] = gather ? a.order[r] : a.ids[r];
      }
      if constexpr (FC) {
#pragma unroll
        for (int b = 0; b < (BM + 63) / 64; ++b) {
          const int m = a.ids[t.row0 + min(64 * b + lane, rows - 1)];
          member[b] = 64 * b + lane < rows ? m : -1;
        }
      }
    }
  };
  // The loads' descriptors and offsets of a tile, and the adapters among its
  // rows (chunks behind K's) in the list, which a barrier follows.
  u32x4 xr, wr;
  uint32_t a_off[AV], b_off[BV];
  int row_id[FC ? AV : 1];   // adapters of this lane's rows
  int rows = 0, n0 = 0;
  int64_t row0 = 0;
  auto make = [&](const Tile &t) __attribute__((always_inline)) {
    const int lane = fresh_lane(threadIdx.x & 63), lrow = lane >> 3;
    const int cgA = vector_a(lane), cgB = vector_b(lane);
    n0 = t.col * OC, row0 = t.row0;
    rows = (int)std::min<int64_t>(t.end - row0, BM);
    xr = gather ? descriptor(a.x, a.x_bytes)
                : descriptor(reinterpret_cast<const char *>(a.x) + row0 * a.ldx * E::size,
                             rows * a.ldx * E::size);
    wr = descriptor(reinterpret_cast<const char *>(a.w) + t.seg * a.w_stride * E::size,
                    (int64_t)a.w_rows * kbytes);
#pragma unroll
    for (int u = 0; u < AV; ++u) {
      const int r = 8 * (u * NW + wave) + lrow;
      const uint32_t row = gather ? (uint32_t)place[u] / (uint32_t)a.top_k : (uint32_t)r;
      a_off[u] = r < rows ? row * (uint32_t)(a.ldx * E::size) + cgA * 16 : kOut;
      if constexpr (FC) row_id[u] = a.ids && r < rows ? place[u] : -1;
    }
#pragma unroll
    for (int u = 0; u < BV; ++u) {
      const int tr = 8 * (u * NW + wave) + lrow;
      const int ch = n0 + (GATED ? (tr >> 6) * 32 + (tr & 31) : tr);
      const int row = GATED && (tr & 32) ? a.n + ch : ch;
      b_off[u] = ch < a.n ? (uint32_t)row * (uint32_t)kbytes + cgB * 16 : kOut;
    }
    if constexpr (FC) {
      if (a.ids && wave == 0) {
        const int f = distinct_values<(BM + 63) / 64>(member, a.adapters, list);
        if ((threadIdx.x & 63) == 0) list_len = f;
      }
    }
  };
  int chunks = n;
  AdapterChunks adapters;

  const uint32_t ring =
      (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem + wave * 1024;
  // What keeps a chunk's loads out of range: nothing, pieces past K in K's last
  // chunk, all of a chunk behind the last (loads that only keep the count).
  uint32_t past_a, past_b;
  {
    const int l = threadIdx.x & 63;
    past_a = vector_a(l) * 16 < tail ? 0u : kOut;
    past_b = vector_b(l) * 16 < tail ? 0u : kOut;
  }
  auto outside = [&](int i, uint32_t past) __attribute__((always_inline)) {
    return i < n - 1 ? 0u : i == n - 1 ? past : kOut;
  };
  // load u of K's chunk i into stage `slot` (behind K: zeros; in an adapter's
  // chunk the loads only keep the count, to a place apart)
  auto load_part = [&](int i, int slot, int u, uint32_t oa, uint32_t ob)
                       __attribute__((always_inline)) {
    const bool apart = FC && i >= n && i < chunks;
    const uint32_t to = apart ? ring + S * (XS + WS)
                        : u < AV ? ring + slot * XS + u * (NW * 1024)
                                 : ring + W0 + slot * WS + (u - AV) * (NW * 1024);
    if (u < AV) ring_load(xr, to, a_off[u] | oa, i * kRow);
    else ring_load(wr, to, b_off[u - AV] | ob, i * kRow);
  };
  // the loads of adapters' chunk i
  auto load_adapter = [&](int i, int slot) __attribute__((always_inline)) {
    const int lane = fresh_lane(threadIdx.x & 63), lrow = lane >> 3;
    const int cgA = vector_a(lane), cgB = vector_b(lane);
    const uint32_t xd = ring + slot * XS, wd = ring + W0 + slot * WS;
    const int hbytes = a.ldh * E::size;   // (columns past the rank hold zeros)
    const u32x4 hr = descriptor(reinterpret_cast<const char *>(a.h) + row0 * hbytes,
                                (int64_t)rows * hbytes);
    int which, at;
    adapters.place(a, i - n, cgA, which, at);
    const int ida = which < adapters.found ? list[which] : -1;
#pragma unroll
    for (int u = 0; u < AV; ++u) {
      const int row = 8 * (u * NW + wave) + lrow;
      const bool in = ida >= 0 && row_id[FC ? u : 0] == ida && at < hbytes;
      ring_load(hr, xd + u * (NW * 1024), in ? (uint32_t)(row * hbytes + at) : kOut, 0);
    }
    adapters.place(a, i - n, cgB, which, at);
    const int idb = which < adapters.found ? list[which] : -1;
    if (a.rank * E::size % 16 == 0) {
#pragma unroll
      for (int u = 0; u < BV; ++u)
        rank_vector<DT>(a, idb, n0 + 8 * (u * NW + wave) + lrow, at, wd + u * (NW * 1024));
    } else {
#pragma nounroll
      for (int u = 0; u < BV; ++u)
        rank_elements<DT>(a, idb, n0 + 8 * (u * NW + wave) + lrow, at,
                          smem + W0 + slot * WS + (wave + u * NW) * 1024);
    }
  };

  f32x4 acc[WTM][WTN];
  const int fB = [&](int rl) { return (((rl >> 2) & 1) << 2) | (rl & 3); }(threadIdx.x & 15);
  int offA[2], offB[2];   // this lane's operand offsets of a chunk's two halves
  {
    const int g = (threadIdx.x & 63) >> 4, rl = threadIdx.x & 15;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      offA[ks] = (wm * WTM * 16 + rl) * kRow + 16 * ((4 * ks + g) ^ (rl & 7));
      offB[ks] = W0 + (wn * WTN * 16 + 8 * (rl >> 2) + (rl & 3)) * kRow + 16 * ((4 * ks + g) ^ fB);
    }
  }
  // Everything a tile needs before its K loop: list, then the first chunks.
  auto begin = [&](const Tile &t) __attribute__((always_inline)) {
    make(t);
    __builtin_amdgcn_s_waitcnt(kLdsDone);
    asm volatile("s_barrier" ::: "memory");   // (and every wave has read its last stage)
    if constexpr (FC) {
      if (a.ids) {
        adapters.set<DT>(a, __builtin_amdgcn_readfirstlane(list_len));
        chunks = n + adapters.number;
      }
    }
#pragma nounroll
    for (int s = 0; s < S; ++s) {
      if (FC && s >= n && s < chunks) load_adapter(s, s);
      const uint32_t oa = outside(s, past_a), ob = outside(s, past_b);
#pragma unroll
      for (int u = 0; u < L; ++u) load_part(s, s, u, oa, ob);
    }
  };
  // The K loop.  A chunk's operands are read from LDS, and the loads that refill
  // the stage freed by the barrier are sent, between the MFMAs of the chunk
  // before, so they have a chunk's time to land.  No branch but the turn of two
  // chunks: loads behind the last chunk fall out of range, and so an odd last
  // chunk is followed by one of zeros.  A wave whose rows all lie past the
  // segment only loads.
  auto run = [&](auto busy) __attribute__((always_inline)) {
    constexpr bool BUSY = decltype(busy)::value;
    constexpr int MF = 2 * WTM * WTN, R = 2 * (WTM + WTN), RSPAN = MF * 3 / 4;
    struct Operands {
      u32x4 x[2][WTM], w[2][WTN];
    } p, q;
    auto read = [&](Operands &o, int slot, int v) __attribute__((always_inline)) {
      const int ks = v / (WTM + WTN), b = v % (WTM + WTN);
      if (b < WTN)
        o.w[ks][b] = *reinterpret_cast<const u32x4 *>(smem + offB[ks] + slot * WS +
                                                      (32 * (b >> 1) + 4 * (b & 1)) * kRow);
      else
        o.x[ks][b - WTN] = *reinterpret_cast<const u32x4 *>(smem + offA[ks] + slot * XS +
                                                            (b - WTN) * 16 * kRow);
    };
    int slot = 0;
    auto step = [&](int i, const Operands &cur, Operands &nxt) __attribute__((always_inline)) {
      if (i >= S - 1) wait_ring<S - 2, L>(S - 2);   // (the first S have landed)
      __builtin_amdgcn_s_waitcnt(kLdsDone);         // this wave has read its stage
      asm volatile("s_barrier" ::: "memory");
      if (FC && i + S >= n && i + S < chunks) load_adapter(i + S, slot);
      const int next = slot == S - 1 ? 0 : slot + 1;
      const uint32_t oa = outside(i + S, past_a), ob = outside(i + S, past_b);
#pragma unroll
      for (int m = 0; m < MF; ++m) {
        const int ks = m / (WTM * WTN), tm = m / WTN % WTM, b = m % WTN;
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (BUSY) {
          acc[tm][b] = mma16<DT>(cur.w[ks][b], cur.x[ks][tm], acc[tm][b]);
#pragma unroll
          for (int v = m * R / RSPAN; v < (m + 1) * R / RSPAN && v < R; ++v) read(nxt, next, v);
        }
#pragma unroll
        for (int u = m * L / MF; u < (m + 1) * L / MF; ++u) load_part(i + S, slot, u, oa, ob);
      }
      __builtin_amdgcn_sched_barrier(0);
      slot = next;
    };
    if constexpr (BUSY) {
#pragma unroll
      for (int v = 0; v < R; ++v) read(p, 0, v);
    }
    for (int i = 0; i < chunks; i += 2) {
      step(i, p, q);
      step(i + 1, q, p);
    }
  };
  // The epilogue, from registers: 8 consecutive channels of a row at a time, a
  // block of 16 rows an iteration, the next block's accumulators moved down
  // (unrolled, the kernel's code is 75 KB, longer than the instruction cache: FC of
  // 4096^3 132.8 us against 128.3, experts of 777 tokens 39 us against 36).
  // WHOLE vectors are stored unconditionally, those of no row or column at an
  // offset past the range, so the next tile's first wait knows their number.
  constexpr bool SCALED = MODE == kRowsDownScaled;
  constexpr int OS = MODE == kRowsDown ? 4 : E::size;
  constexpr int H = GATED ? 1 : 2;                      // runs of 8 channels of a group
  constexpr int kStores = WTM * NG * H * (OS / 2);
  // (u and z have rows of whole vectors, u's ends in zeros: it may be K's end)
  const bool whole = MODE <= kRowsDown || (a.n % 8 == 0 && a.ldy % 8 == 0);
  auto finish = [&](auto vectors, int seg, int n0, int64_t row0, int rows)
                    __attribute__((always_inline)) {
    constexpr bool WHOLE = decltype(vectors)::value;
    const int lane = fresh_lane(threadIdx.x & 63), g = lane >> 4;
    const int mw = wm * WTM * 16 + (lane & 15);
    const int64_t y0 = row0 * a.ldy;
    const __amdgpu_buffer_rsrc_t yr = __builtin_amdgcn_make_buffer_rsrc(
        reinterpret_cast<char *>(a.y) + y0 * OS, (short)0, (int)(rows * a.ldy * OS), kBufDword3);
    const raw *res = FC && a.residual ? reinterpret_cast<const raw *>(a.residual) + y0 : nullptr;
    const __amdgpu_buffer_rsrc_t rr = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<raw *>(res), (short)0, res ? (int)(rows * a.ldy * E::size) : 0, kBufDword3);
    // a run's first channel
    const int col0 = n0 + 8 * g + wn * WTN * (GATED ? 8 : 16);
    auto column = [&](int q, int h) { return col0 + (GATED ? 32 * q : 64 * q + 32 * h); };
    float bv[NG][H][8] = {}, bu[GATED ? NG : 1][8] = {};
    if (a.bias) {
      const raw *bias = reinterpret_cast<const raw *>(a.bias) + (int64_t)seg * a.w_rows;
#pragma unroll
      for (int q = 0; q < NG; ++q)
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int c = min(column(q, h) + e, a.n - 1);
            bv[q][h][e] = E::to_f32(bias[c]);
            if constexpr (GATED) bu[q][e] = E::to_f32(bias[a.n + c]);
          }
    }
#pragma nounroll
    for (int tm = 0; tm < WTM; ++tm) {
      const int r = mw + 16 * tm;
      float o[NG][H][8];
#pragma unroll
      for (int q = 0; q < NG; ++q)
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            o[q][h][e] = acc[0][4 * q + 2 * h + (e >> 2)][e & 3] + bv[q][h][e];
      if (FC && res) {
        constexpr int RV = E::size / 2;   // 16-byte vectors of 8 elements
#pragma unroll
        for (int q = 0; q < NG; ++q)
#pragma unroll
          for (int h = 0; h < H; ++h) {
            const int col = column(q, h);
            const bool in = r < rows && col < a.n;
            const uint32_t at = r * (uint32_t)a.ldy + col;
            u32x4 t[RV] = {};
            if constexpr (WHOLE) {
#pragma unroll
              for (int v = 0; v < RV; ++v)
                t[v] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                     rr, in ? at * E::size + 16 * v : kOut, 0, 0));
            }
            raw e8[8];
            __builtin_memcpy(e8, t, sizeof e8);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              if constexpr (!WHOLE) e8[e] = in && col + e < a.n ? res[at + e] : (raw)0;
              o[q][h][e] += E::to_f32(e8[e]);
            }
          }
      }
      if constexpr (FC) {
        if (a.act != SPAROA_ACT_NONE)
#pragma unroll
          for (int i = 0; i < NG * H * 8; ++i)
            o[i / (8 * H)][i / 8 % H][i % 8] = row_act(o[i / (8 * H)][i / 8 % H][i % 8], a.act);
      } else if constexpr (MODE <= kRowsUpGated) {
        // (a branch for all of the values, not one for each)
        auto all = [&](auto act) __attribute__((always_inline)) {
#pragma unroll
          for (int i = 0; i < NG * H * 8; ++i)
            o[i / (8 * H)][i / 8 % H][i % 8] =
                block_act<DT>(o[i / (8 * H)][i / 8 % H][i % 8], decltype(act)::value);
        };
        switch (a.act) {
          case SPAROA_ACT_SILU: all(std::integral_constant<int, SPAROA_ACT_SILU>{}); break;
          case SPAROA_ACT_GELU: all(std::integral_constant<int, SPAROA_ACT_GELU>{}); break;
          case SPAROA_ACT_RELU: all(std::integral_constant<int, SPAROA_ACT_RELU>{}); break;
          case SPAROA_ACT_RELU6: all(std::integral_constant<int, SPAROA_ACT_RELU6>{}); break;
          default: break;
        }
      }
#pragma unroll
      for (int q = 0; q < NG; ++q)
#pragma unroll
        for (int h = 0; h < H; ++h) {
          const int col = column(q, h);
          const bool in = r < rows && col < a.n;
          const uint32_t at = r * (uint32_t)a.ldy + col;   // (below 2^31 bytes)
          float (&v)[8] = o[q][h];
          if constexpr (GATED) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              v[e] *= acc[0][4 * q + 2 + (e >> 2)][e & 3] + bu[q][e];
          }
          if constexpr (MODE <= kRowsDown) {
            if (a.n % 8)
#pragma unroll
              for (int e = 0; e < 8; ++e) v[e] = col + e < a.n ? v[e] : 0.f;
          }
          if constexpr (OS == 4 && WHOLE) {
#pragma unroll
            for (int p = 0; p < 2; ++p) {
              const f32x4 f = {v[4 * p], v[4 * p + 1], v[4 * p + 2], v[4 * p + 3]};
              __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f), yr,
                                                     in ? at * 4 + 16 * p : kOut, 0, 0);
            }
          } else if constexpr (WHOLE) {
            __builtin_amdgcn_raw_buffer_store_b128(SCALED ? pack_scaled8(v) : pack8<DT>(v), yr,
                                                   in ? at * 2 : kOut, 0, 0);
          } else {
            raw *y = reinterpret_cast<raw *>(a.y) + y0;
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (in && col + e < a.n) y[at + e] = E::from_f32(v[e]);
          }
        }
#pragma unroll
      for (int j = 0; j + 1 < WTM; ++j)
#pragma unroll
        for (int b = 0; b < WTN; ++b) acc[j][b] = acc[j + 1][b];
    }
  };

  // Outputs that are NaN where the tile has adapters, worked out by themselves:
  // one accumulator after the other takes the first one's place.
  auto mend = [&](int n0, int64_t row0, int rows) __attribute__((always_inline)) {
    f32x4 sums = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < WTM * WTN; ++i) sums += acc[i / WTN][i % WTN];
    const float sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    if (!__ballot(sum != sum)) return;
    const int lane = threadIdx.x & 63, r0 = wm * WTM * 16 + (lane & 15);
    const int c0 = n0 + wn * WTN * 16 + 8 * (lane >> 4);
#pragma nounroll
    for (int i = 0; i < WTM * WTN; ++i) {
      const int b = i % WTN, r = r0 + i / WTN * 16;
      const int c = c0 + 64 * (b >> 2) + 32 * (b >> 1 & 1) + 4 * (b & 1);
      f32x4 v = acc[0][0];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (v[e] != v[e] && r < rows && c + e < a.n) v[e] = own_output<DT>(a, row0 + r, c + e);
#pragma unroll
      for (int j = 0; j + 1 < WTM * WTN; ++j)
        acc[j / WTN][j % WTN] = acc[(j + 1) / WTN][(j + 1) % WTN];
      acc[WTM - 1][WTN - 1] = v;
    }
  };

  // ---- tile by tile.  The next tile's first chunks are sent for before the
  // epilogue, and the rows of the tile behind it before the stores, which are
  // then the newest operations: K starts when the chunks have landed, under
  // the stores.
  fetch(tl);
  begin(tl);
  Tile nt = walk.next();
  if (nt.end) fetch(nt);
  bool stored = false;
  for (;;) {
    const bool busy = wm * WTM * 16 < rows;
    static_assert(kStores < 64, "vmcnt range");
    if (stored) __builtin_amdgcn_s_waitcnt(vm_outstanding(kStores));
    else __builtin_amdgcn_s_waitcnt(vm_outstanding(0));
    __builtin_amdgcn_s_waitcnt(kLdsDone);   // (pieces that passed through registers)
    asm volatile("s_barrier" ::: "memory");
#pragma unroll
    for (int i = 0; i < WTM; ++i)
#pragma unroll
      for (int j = 0; j < WTN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (busy) run(std::true_type{});
    else run(std::false_type{});
    const int seg = tl.seg, n0_ = n0, rows_ = rows;
    const int64_t row0_ = row0;
    const int found = adapters.found;
    const bool more = nt.end != 0;
    if (more) {
      tl = nt;
      begin(tl);
      nt = walk.next();
      if (nt.end) fetch(nt);
    }
    if (busy) {
      if constexpr (FC)
        if (found) mend(n0_, row0_, rows_);
      if (whole) finish(std::true_type{}, seg, n0_, row0_, rows_);
      else if constexpr (FC) finish(std::false_type{}, seg, n0_, row0_, rows_);
    }
    stored = busy && whole;
    if (!more) return;
  }
}

template <int DT, RowsMode MODE, int WGM, int WGN, int WTM, int WTN, int S>
sparoa_status launch_one(RowsArgs a, hipStream_t stream) {
  constexpr int BM = 16 * WGM * WTM, BN = 16 * WGN * WTN;
  const int64_t cols = cdiv(a.n, MODE == kRowsUpGated ? BN / 2 : BN);
  const int64_t row_tiles = MODE <= kRowsDown
                                ? a.rows / BM + std::min<int64_t>(a.experts, a.rows)
                                : cdiv(a.rows, BM);
  a.col_groups = cols >= 8 ? 2 : 1;
  const void *fn = reinterpret_cast<const void *>(
      &rows_tile_kernel<DT, MODE, WGM, WGN, WTM, WTN, S>);
  int resident = 0;
  const sparoa_status st = resident_blocks(fn, 64 * WGM * WGN, 0, &resident);
  if (st != SPAROA_OK) return st;
  const unsigned grid =
      (unsigned)(8 * cdiv(std::min<int64_t>(row_tiles * cols, resident), 8));
  rows_tile_kernel<DT, MODE, WGM, WGN, WTM, WTN, S><<<grid, 64 * WGM * WGN, 0, stream>>>(a);
  return SPAROA_OK;
}

template <int DT, RowsMode MODE>
sparoa_status launch_mode(RowsTile tile, const RowsArgs &a, hipStream_t stream) {
  if constexpr (DT != SPAROA_F32)
    if (tile == kTile128x256) return launch_one<DT, MODE, 2, 4, 4, 4, 3>(a, stream);   // 144 KB
  if (tile == kTile64x128) return launch_one<DT, MODE, 2, 2, 2, 4, 3>(a, stream);      // 72 KB
  return launch_one<DT, MODE, 4, 1, 1, 4, 4>(a, stream);                               // 64 KB
}

template <int DT>
sparoa_status launch_dt(RowsMode mode, RowsTile tile, const RowsArgs &a, hipStream_t stream) {
  switch (mode) {
    case kRowsUp: return launch_mode<DT, kRowsUp>(tile, a, stream);
    case kRowsUpGated: return launch_mode<DT, kRowsUpGated>(tile, a, stream);
    case kRowsDownScaled:
      if constexpr (DT == SPAROA_BF16) return launch_mode<DT, kRowsDownScaled>(tile, a, stream);
      return fail(SPAROA_ERR_UNSUPPORTED, "row products: scaled outputs are for bf16");
    case kRowsDown: return launch_mode<DT, kRowsDown>(tile, a, stream);
    default: return launch_mode<DT, kRowsFc>(tile, a, stream);
  }
}

}  // namespace

sparoa_status launch_rows_tile(RowsMode mode, RowsTile tile, const RowsArgs &a, sparoa_dtype dt,
                               hipStream_t stream) {
  const sparoa_status st = dt == SPAROA_F32   ? launch_dt<SPAROA_F32>(mode, tile, a, stream)
                           : dt == SPAROA_F16 ? launch_dt<SPAROA_F16>(mode, tile, a, stream)
                                              : launch_dt<SPAROA_BF16>(mode, tile, a, stream);
  if (st != SPAROA_OK) return st;
  SPAROA_LAUNCH_CHECK("row product tiles");
  return SPAROA_OK;
}

}  // namespace sparoa

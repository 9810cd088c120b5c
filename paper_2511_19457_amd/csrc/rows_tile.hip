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
// Work-groups are dealt round-robin to the 8 XCDs: XCD i takes the i-th run of
// tiles, column tiles innermost, so the tiles of one expert share an L2.
#include <algorithm>

#include "rows_ring.h"

namespace sparoa {
namespace {

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
  constexpr int STAGE = (BM + BN) * kRow;
  __shared__ __attribute__((aligned(1024))) char smem[S * STAGE];
  __shared__ int32_t list[FC ? BM : 1];
  __shared__ int list_len;

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WGN, wn = wave % WGN;
  const Tile tl = find_tile<MODE, BM>(a, (a.n + OC - 1) / OC);
  if (tl.end == 0) return;
  const int n0 = tl.col * OC;
  const int64_t row0 = tl.row0;
  const int rows = (int)std::min<int64_t>(tl.end - row0, BM);
  const int kbytes = a.k * E::size;
  const int n = (kbytes + kRow - 1) / kRow;

  // ---- this lane's share of the loads: slot lane & 7 of chunk row lane >> 3.
  // Rows hold their 16-byte vectors swizzled, slot = vector ^ f(row), so that
  // the operand reads of 8 consecutive lanes meet distinct banks: rows of x f =
  // row & 7; weight rows, read in the order that leaves a lane 8 consecutive
  // channels (MFMA row 4 q + t of block b is tile row 32 (b / 2) + 8 q + 4 (b %
  // 2) + t), f = (row >> 3 & 1) * 4 + (row & 3).
  const int lrow = lane >> 3;
  const int cgA = (lane & 7) ^ lrow;
  const int cgB = (lane & 7) ^ (((wave & 1) << 2) | (lrow & 3));
  const bool gather = MODE <= kRowsUpGated;
  const u32x4 xr = gather ? descriptor(a.x, a.x_bytes)
                          : descriptor(reinterpret_cast<const char *>(a.x) +
                                           row0 * a.ldx * E::size,
                                       rows * a.ldx * E::size);
  const u32x4 wr = descriptor(reinterpret_cast<const char *>(a.w) +
                                  tl.seg * a.w_stride * E::size,
                              (int64_t)a.w_rows * kbytes);
  uint32_t a_off[AV], b_off[BV];
  int a_id[AV];   // (FC) the row's adapter
#pragma unroll
  for (int u = 0; u < AV; ++u) {
    const int r = 8 * (u * NW + wave) + lrow;
    uint32_t row = r;
    if (gather && r < rows) row = (uint32_t)a.order[row0 + r] / (uint32_t)a.top_k;
    a_off[u] = r < rows ? row * (uint32_t)(a.ldx * E::size) + cgA * 16 : kOut;
    a_id[u] = FC && a.ids && r < rows ? a.ids[row0 + r] : -1;
  }
#pragma unroll
  for (int u = 0; u < BV; ++u) {
    const int tr = 8 * (u * NW + wave) + lrow;
    const int ch = n0 + (GATED ? (tr >> 6) * 32 + (tr & 31) : tr);
    const int row = GATED && (tr & 32) ? a.n + ch : ch;
    b_off[u] = ch < a.n ? (uint32_t)row * (uint32_t)kbytes + cgB * 16 : kOut;
  }
  // bits that put a lane's piece of the last chunk out of range, past K
  const int tail = kbytes - (n - 1) * kRow;
  const uint32_t pastA = cgA * 16 < tail ? 0u : kOut, pastB = cgB * 16 < tail ? 0u : kOut;

  // ---- chunks behind K's: the adapters among the rows
  int extra = 0, rank_chunks = 1;
  if constexpr (FC) {
    if (a.ids) {
      if (wave == 0) {
        const int f = distinct_ids<(BM + 63) / 64>(a.ids + row0, rows, a.adapters, list);
        if (lane == 0) list_len = f;
      }
      __syncthreads();
      rank_chunks = (a.rank * E::size + kRow - 1) / kRow;
      extra = __builtin_amdgcn_readfirstlane(list_len) * rank_chunks;
    }
  }
  const int chunks = n + extra;

  const uint32_t ring =
      (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem + wave * 1024;
  // load u of K's chunk i (any but the last) into the stage at dst
  auto load_plain = [&](int i, uint32_t dst, int u) __attribute__((always_inline)) {
    if (u < AV) ring_load(xr, dst + u * (NW * 1024), a_off[u], i * kRow);
    else ring_load(wr, dst + BM * kRow + (u - AV) * (NW * 1024), b_off[u - AV], i * kRow);
  };
  // the loads of any chunk
  auto load_any = [&](int i, uint32_t dst) __attribute__((always_inline)) {
    if (i < n) {
      const uint32_t last = i == n - 1 ? kOut : 0u;
#pragma unroll
      for (int u = 0; u < AV; ++u)
        ring_load(xr, dst + u * (NW * 1024), a_off[u] | (pastA & last), i * kRow);
#pragma unroll
      for (int u = 0; u < BV; ++u)
        ring_load(wr, dst + BM * kRow + u * (NW * 1024), b_off[u] | (pastB & last), i * kRow);
      return;
    }
    if constexpr (FC) {
      const int c = i - n, d = c / rank_chunks, r = (c - d * rank_chunks) * kRow;
      const int id = __builtin_amdgcn_readfirstlane(list[d]);
      const int hbytes = a.ldh * E::size;   // (columns past the rank hold zeros)
      const u32x4 hr = descriptor(reinterpret_cast<const char *>(a.h) + row0 * hbytes,
                                  (int64_t)rows * hbytes);
#pragma unroll
      for (int u = 0; u < AV; ++u) {
        const int row = 8 * (u * NW + wave) + lrow;
        const bool in = a_id[u] == id && r + cgA * 16 < hbytes;
        ring_load(hr, dst + u * (NW * 1024),
                  in ? (uint32_t)(row * hbytes + r + cgA * 16) : kOut, 0);
      }
#pragma unroll
      for (int u = 0; u < BV; ++u)
        rank_piece<DT>(a, id, n0 + 8 * (u * NW + wave) + lrow, r + cgB * 16,
                       dst + BM * kRow + u * (NW * 1024),
                       smem + (dst - ring) + wave * 1024 + BM * kRow + u * (NW * 1024));
    }
  };

  f32x4 acc[WTM][WTN];
#pragma unroll
  for (int i = 0; i < WTM; ++i)
#pragma unroll
    for (int j = 0; j < WTN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int g = lane >> 4, rl = lane & 15;
  const int fB = (((rl >> 2) & 1) << 2) | (rl & 3);
  int offA[2], offB[2];   // this lane's operand offsets of the chunk's two halves
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    offA[ks] = (wm * WTM * 16 + rl) * kRow + 16 * ((4 * ks + g) ^ (rl & 7));
    offB[ks] = (BM + wn * WTN * 16 + 8 * (rl >> 2) + (rl & 3)) * kRow + 16 * ((4 * ks + g) ^ fB);
  }
  struct Operands {
    u32x4 x[2][WTM], w[2][WTN];
  };
  constexpr int R = 2 * (WTM + WTN), MF = 2 * WTM * WTN, RSPAN = MF * 3 / 4;
  auto read_part = [&](Operands &o, int slot, int q) __attribute__((always_inline)) {
    const int ks = q / (WTM + WTN), v = q % (WTM + WTN);
    const char *st = smem + slot * STAGE;
    if (v < WTN)
      o.w[ks][v] = *reinterpret_cast<const u32x4 *>(st + offB[ks] +
                                                    (32 * (v >> 1) + 4 * (v & 1)) * kRow);
    else
      o.x[ks][v - WTN] = *reinterpret_cast<const u32x4 *>(st + offA[ks] + (v - WTN) * 16 * kRow);
  };
  // One step per chunk: on entry its operands are in registers or on their
  // way.  Steady steps (a next chunk, and a refill that is not K's last) have
  // no branch and constant stages.
  // A wave whose rows all lie past the segment only loads.
  const bool busy_wave = wm * WTM * 16 < rows;
  auto step = [&](auto steady, auto busy, Operands &cur, Operands &nxt, int slot, int i)
                  __attribute__((always_inline)) {
    constexpr bool STEADY = decltype(steady)::value, BUSY = decltype(busy)::value;
    const bool more = STEADY || i + 1 < chunks, refill = STEADY || i + S < chunks;
    const uint32_t dst = ring + slot * STAGE;
    if (more) {
      if constexpr (STEADY) wait_ring<S - 2, L>(S - 2);
      else wait_ring<S - 2, L>(min(S - 2, chunks - 2 - i));
      __builtin_amdgcn_s_waitcnt(kLdsDone);   // this wave has read its stage
      asm volatile("s_barrier" ::: "memory");
    }
    const int nslot = slot == S - 1 ? 0 : slot + 1;
    if (!STEADY && refill) load_any(i + S, dst);
#pragma unroll
    for (int m = 0; m < MF; ++m) {
      const int ks = m / (WTM * WTN), tm = m / WTN % WTM, b = m % WTN;
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (BUSY) acc[tm][b] = mma16<DT>(cur.w[ks][b], cur.x[ks][tm], acc[tm][b]);
      if (BUSY && more) {
#pragma unroll
        for (int q = m * R / RSPAN; q < (m + 1) * R / RSPAN && q < R; ++q) read_part(nxt, nslot, q);
      }
      if constexpr (STEADY) {
#pragma unroll
        for (int u = m * L / MF; u < (m + 1) * L / MF; ++u) load_plain(i + S, dst, u);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
#pragma unroll
  for (int s = 0; s < S; ++s)
    if (s < chunks) load_any(s, ring + s * STAGE);
  wait_ring<S - 1, L>(min(S - 1, chunks - 1));
  __builtin_amdgcn_s_waitcnt(kLdsDone);   // (pieces that passed through registers)
  asm volatile("s_barrier" ::: "memory");
  auto run = [&](auto busy) __attribute__((always_inline)) {
    Operands p, q;
    if constexpr (decltype(busy)::value) {
#pragma unroll
      for (int r = 0; r < R; ++r) read_part(p, 0, r);
    }
    constexpr int U = S % 2 ? 2 * S : S;   // a turn of the ring and of (p, q)
    int i = 0;
    for (; i + U + S < n; i += U) {
#pragma unroll
      for (int d = 0; d < U; ++d)
        step(std::true_type{}, busy, d % 2 ? q : p, d % 2 ? p : q, d % S, i + d);
    }
    for (; i < chunks; i += U) {
#pragma unroll
      for (int d = 0; d < U; ++d)
        if (i + d < chunks)
          step(std::false_type{}, busy, d % 2 ? q : p, d % 2 ? p : q, d % S, i + d);
    }
  };
  if (!busy_wave) return run(std::false_type{});
  run(std::true_type{});

  // ---- epilogue, from registers: 8 consecutive channels of a row at a time
  const int mw = wm * WTM * 16 + rl;
  const bool whole = a.n % 8 == 0 && a.ldy % 8 == 0;
  const raw *bias = reinterpret_cast<const raw *>(a.bias) + (a.bias ? (int64_t)tl.seg * a.w_rows : 0);
  auto get8 = [&](const raw *p, int c, float (&v)[8]) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = E::to_f32(p[min(c + e, a.n - 1)]);
  };
#pragma unroll
  for (int q = 0; q < NG; ++q)
#pragma unroll
    for (int h = 0; h < (GATED ? 1 : 2); ++h) {
      const int col = n0 + 8 * g + (GATED ? wn * WTN * 8 + 32 * q : wn * WTN * 16 + 64 * q + 32 * h);
      if (col >= a.n) continue;
      float bv[8], bu[8];
      if (a.bias) {
        get8(bias, col, bv);
        if constexpr (GATED) get8(bias + a.n, col, bu);
      }
#pragma unroll
      for (int tm = 0; tm < WTM; ++tm) {
        const int r = mw + 16 * tm;
        if (r >= rows) continue;
        const int64_t at = (row0 + r) * a.ldy + col;
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          o[e] = acc[tm][4 * q + 2 * h + (e >> 2)][e & 3];
          if (a.bias) o[e] += bv[e];
          if constexpr (GATED) {
            float up = acc[tm][4 * q + 2 + (e >> 2)][e & 3];
            if (a.bias) up += bu[e];
            o[e] = block_act(o[e], a.act) * up;
          }
        }
        if constexpr (MODE == kRowsDown) {
          float *z = reinterpret_cast<float *>(a.y) + at;   // (rows padded to 8 channels)
          *reinterpret_cast<f32x4 *>(z) = f32x4{o[0], o[1], o[2], o[3]};
          *reinterpret_cast<f32x4 *>(z + 4) = f32x4{o[4], o[5], o[6], o[7]};
          continue;
        }
        raw *y = reinterpret_cast<raw *>(a.y) + at;
        if (FC && a.residual) {
          const raw *res = reinterpret_cast<const raw *>(a.residual) + at;
          float rv[8];
          if (whole) {
            raw t[8];
            __builtin_memcpy(t, __builtin_assume_aligned(res, 16), sizeof t);
#pragma unroll
            for (int e = 0; e < 8; ++e) rv[e] = E::to_f32(t[e]);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) rv[e] = col + e < a.n ? E::to_f32(res[e]) : 0.f;
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] += rv[e];
        }
        if constexpr (!GATED) {
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = FC ? apply_act(o[e], a.act) : block_act(o[e], a.act);
        }
        if (whole) {
          raw t[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) t[e] = E::from_f32(o[e]);
          __builtin_memcpy(__builtin_assume_aligned(y, 16), t, sizeof t);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (col + e < a.n) y[e] = E::from_f32(o[e]);
        }
      }
    }
}

template <int DT, RowsMode MODE, int WGM, int WGN, int WTM, int WTN, int S>
void launch_one(RowsArgs a, hipStream_t stream) {
  constexpr int BM = 16 * WGM * WTM, BN = 16 * WGN * WTN;
  const int64_t cols = cdiv(a.n, MODE == kRowsUpGated ? BN / 2 : BN);
  const int64_t row_tiles = MODE <= kRowsDown
                                ? a.rows / BM + std::min<int64_t>(a.experts, a.rows)
                                : cdiv(a.rows, BM);
  a.col_groups = cols >= 8 ? 2 : 1;
  const unsigned grid = (unsigned)(8 * cdiv(row_tiles * cols, 8));
  rows_tile_kernel<DT, MODE, WGM, WGN, WTM, WTN, S><<<grid, 64 * WGM * WGN, 0, stream>>>(a);
}

template <int DT, RowsMode MODE>
void launch_mode(RowsTile tile, const RowsArgs &a, hipStream_t stream) {
  if (tile == kTile128x256) {
    if constexpr (DT != SPAROA_F32) launch_one<DT, MODE, 2, 4, 4, 4, 3>(a, stream);   // 144 KB
  } else if (tile == kTile64x128) {
    launch_one<DT, MODE, 2, 2, 2, 4, 3>(a, stream);                                   // 72 KB
  } else {
    launch_one<DT, MODE, 4, 1, 1, 4, 4>(a, stream);                                   // 64 KB
  }
}

template <int DT>
void launch_dt(RowsMode mode, RowsTile tile, const RowsArgs &a, hipStream_t stream) {
  switch (mode) {
    case kRowsUp: return launch_mode<DT, kRowsUp>(tile, a, stream);
    case kRowsUpGated: return launch_mode<DT, kRowsUpGated>(tile, a, stream);
    case kRowsDown: return launch_mode<DT, kRowsDown>(tile, a, stream);
    default: return launch_mode<DT, kRowsFc>(tile, a, stream);
  }
}

}  // namespace

sparoa_status launch_rows_tile(RowsMode mode, RowsTile tile, const RowsArgs &a, sparoa_dtype dt,
                               hipStream_t stream) {
  switch (dt) {
    case SPAROA_F32: launch_dt<SPAROA_F32>(mode, tile, a, stream); break;
    case SPAROA_F16: launch_dt<SPAROA_F16>(mode, tile, a, stream); break;
    default: launch_dt<SPAROA_BF16>(mode, tile, a, stream); break;
  }
  SPAROA_LAUNCH_CHECK("row product tiles");
  return SPAROA_OK;
}

}  // namespace sparoa

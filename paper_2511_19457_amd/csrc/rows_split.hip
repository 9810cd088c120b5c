// Products of few tiles: the waves of a work-group split K.
//
// A work-group has a tile of 16 TM rows and 16 TN weight rows, small enough to
// give every CU one or two; wave w takes K's chunks (128 bytes) w, w + NW, ...
// through a ring of its own of S stages in LDS, sent there by the loads, so
// the K loop has no barrier and S chunks a wave are in flight.  The waves'
// partial tiles meet in LDS, added in wave order.  Low-rank adapters are
// chunks behind K's, as in the tile kernel; their first product (shrink: h =
// scale_a A_a x) is a tile of its own for every adapter among the rows.
// Bound by the latency of a chain of chunks (few rows in all), or by the
// weights' stream (experts that serve few rows each).  bf16, 64 experts gated,
// 2048 x 1024, top 8: 64 tokens 97 + 51 us for 805 MB of weights (5.4 TB/s),
// one token 13.4 + 7.4 us for 100 MB; FC of 32 x 4096 x 4096 11.4 us.
#include <algorithm>

#include "rows_ring.h"

namespace sparoa {
namespace {

template <int DT, RowsMode MODE, int TM, int TN, int NW, int S>
__global__ __launch_bounds__(64 * NW, 2) void rows_split_kernel(RowsArgs a) {
  using E = Elem<DT>;
  using raw = typename E::raw;
  constexpr bool GATED = MODE == kRowsUpGated, FC = MODE == kRowsFc;
  constexpr bool SHRINK = MODE == kRowsShrink, UP = MODE <= kRowsUpGated;
  constexpr int BM = 16 * TM, BN = 16 * TN, OC = GATED ? BN / 2 : BN;
  constexpr int NB = GATED ? TN / 2 : TN;      // blocks of 16 output columns
  constexpr int AV = 2 * TM, BV = 2 * TN, L = AV + BV;   // loads of 8 rows
  constexpr int STAGE = (BM + BN) * kRow;
  static_assert(!GATED || TN % 2 == 0, "gate and up blocks in pairs");
  __shared__ __attribute__((aligned(1024))) char smem[NW * S * STAGE];
  __shared__ int32_t list[FC || SHRINK ? BM : 1];
  __shared__ int list_len;

  const int lane = threadIdx.x & 63, lrow = lane >> 3, q = lane >> 4, rl = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Tile tl = find_tile<MODE, BM>(a, (a.n + OC - 1) / OC);
  if (tl.end == 0) return;
  const int n0 = tl.col * OC;
  const int64_t row0 = tl.row0;
  const int rows = (int)std::min<int64_t>(tl.end - row0, BM);
  const int kbytes = a.k * E::size;
  const int n = (kbytes + kRow - 1) / kRow;

  // ---- this lane's share of the loads: slot lane & 7 of row lane >> 3 of 8,
  // which holds the row's vector (lane & 7) ^ (row & 7)
  const int cg = (lane & 7) ^ lrow;
  static_assert(BM <= 64, "a lane per row");
  int member[1] = {-1};   // (adapters) row `lane`'s
  if ((FC || SHRINK) && a.ids && lane < rows) member[0] = a.ids[row0 + lane];
  const bool gather = MODE <= kRowsUpGated;
  int slot[AV], id[AV];   // (sent for first: loads land in order)
#pragma unroll
  for (int u = 0; u < AV; ++u) {
    const int r = min(8 * u + lrow, rows - 1);
    slot[u] = gather ? a.order[row0 + r] : r;
    id[u] = (FC || SHRINK) && a.ids ? a.ids[row0 + r] : -1;
  }
  uint32_t a_off[AV], b_off[BV];
#pragma unroll
  for (int u = 0; u < BV; ++u) {
    const int tr = 8 * u + lrow;
    const int ch = n0 + (GATED ? (tr >> 5) * 16 + (tr & 15) : tr);
    const int row = GATED && (tr & 16) ? a.n + ch : ch;
    b_off[u] = ch < a.n ? (uint32_t)row * (uint32_t)kbytes + cg * 16 : kOut;
  }
  const uint32_t past = cg * 16 < kbytes - (n - 1) * kRow ? 0u : kOut;   // past K, last chunk

  // The adapters among the rows: (FC) chunks behind K's, (shrink) a tile each.
  int items = 1;
  AdapterChunks adapters;
  auto find_adapters = [&]() __attribute__((always_inline)) {
    if ((FC || SHRINK) && a.ids) {
      if (wave == 0) {
        const int f = distinct_values<1>(member, a.adapters, list);
        if (lane == 0) list_len = f;
      }
      __syncthreads();
      const int f = __builtin_amdgcn_readfirstlane(list_len);
      if constexpr (FC) adapters.set<DT>(a, f);
      else items = f;
    }
  };
  // (FC: the first chunks, all of K, are sent for before that)
  const bool early = FC && n >= S * NW;
  if (!early) find_adapters();

  const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem +
                        wave * (S * STAGE);
  char *const ring_at = smem + wave * (S * STAGE);
  const u32x4 xr = gather ? descriptor(a.x, a.x_bytes)
                          : descriptor(reinterpret_cast<const char *>(a.x) +
                                           row0 * a.ldx * E::size,
                                       rows * a.ldx * E::size);
  for (int item = 0; item < items; ++item) {   // (shrink: every adapter among the rows)
    if (item) __syncthreads();   // the last item's partial sums have been read
    const int seg = SHRINK ? __builtin_amdgcn_readfirstlane(list[item]) : tl.seg;
    const u32x4 wr = descriptor(reinterpret_cast<const char *>(a.w) + seg * a.w_stride * E::size,
                                (int64_t)a.w_rows * kbytes);
    // (at the start the weights are sent for before the rows' places are known)
    auto load_w = [&](int c, uint32_t dst) __attribute__((always_inline)) {
      if (!FC || c < n) {
        const uint32_t out = c == n - 1 ? past : 0u;
#pragma unroll
        for (int u = 0; u < BV; ++u)
          ring_load(wr, dst + BM * kRow + u * 1024, b_off[u] | out, c * kRow);
      } else {
        int which, from;
        adapters.place(a, c - n, cg, which, from);
        const int adapter = which < adapters.found ? list[which] : -1;
        if (a.rank * E::size % 16 == 0) {
#pragma unroll
          for (int u = 0; u < BV; ++u)
            rank_vector<DT>(a, adapter, n0 + 8 * u + lrow, from, dst + BM * kRow + u * 1024);
        } else {
#pragma nounroll
          for (int u = 0; u < BV; ++u)
            rank_elements<DT>(a, adapter, n0 + 8 * u + lrow, from,
                              ring_at + (dst - ring) + BM * kRow + u * 1024);
        }
      }
    };
    auto load_x = [&](int c, uint32_t dst) __attribute__((always_inline)) {
      if (!FC || c < n) {
        const uint32_t out = c == n - 1 ? past : 0u;
#pragma unroll
        for (int u = 0; u < AV; ++u) ring_load(xr, dst + u * 1024, a_off[u] | out, c * kRow);
      } else {   // the rows of this adapter; the others' read as zeros
        int which, from;
        adapters.place(a, c - n, cg, which, from);
        const int hbytes = a.ldh * E::size, adapter = which < adapters.found ? list[which] : -1;
        const u32x4 hr = descriptor(reinterpret_cast<const char *>(a.h) + row0 * hbytes,
                                    (int64_t)rows * hbytes);
#pragma unroll
        for (int u = 0; u < AV; ++u) {
          const int row = 8 * u + lrow;
          const bool in = row < rows && adapter >= 0 && id[u] == adapter && from < hbytes;
          ring_load(hr, dst + u * 1024, in ? (uint32_t)(row * hbytes + from) : kOut, 0);
        }
      }
    };
    int chunks = n + adapters.number;
    int mine = chunks > wave ? (chunks - wave + NW - 1) / NW : 0;   // this wave's chunks
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (s < mine) load_w(wave + s * NW, ring + s * STAGE);
#pragma unroll
    for (int u = 0; u < AV; ++u) {
      const uint32_t row = gather ? (uint32_t)slot[u] / (uint32_t)a.top_k : (uint32_t)slot[u];
      const bool in = 8 * u + lrow < rows && (!SHRINK || id[u] == seg);
      a_off[u] = in ? row * (uint32_t)(a.ldx * E::size) + cg * 16 : kOut;
    }
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (s < mine) load_x(wave + s * NW, ring + s * STAGE);
    if (early) {
      find_adapters();
      chunks = n + adapters.number;
      mine = (chunks - wave + NW - 1) / NW;
    }

    f32x4 acc[TN][TM];
#pragma unroll
    for (int b = 0; b < TN; ++b)
#pragma unroll
      for (int t = 0; t < TM; ++t) acc[b][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    int at[2];   // this lane's operand offsets of a chunk's two halves
#pragma unroll
    for (int h = 0; h < 2; ++h) at[h] = rl * kRow + 16 * ((4 * h + q) ^ (rl & 7));
    int stage = 0;
    for (int j = 0; j < mine; ++j) {
      // newer than this chunk's loads are those of the refills sent so far (the
      // first S chunks), else of the next S - 1 chunks
      wait_ring<S - 1, L>(j < S ? min(j, max(mine - S, 0)) : min(S - 1, mine - 1 - j));
      const char *st = ring_at + stage * STAGE;
      u32x4 x[2][TM], w[2][TN];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int t = 0; t < TM; ++t)
          x[h][t] = *reinterpret_cast<const u32x4 *>(st + at[h] + t * 16 * kRow);
#pragma unroll
        for (int b = 0; b < TN; ++b)
          w[h][b] = *reinterpret_cast<const u32x4 *>(st + at[h] + (BM + b * 16) * kRow);
      }
      __builtin_amdgcn_s_waitcnt(kLdsDone);   // the stage is read
      if (j + S < mine) {
        load_w(wave + (j + S) * NW, ring + stage * STAGE);
        load_x(wave + (j + S) * NW, ring + stage * STAGE);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int b = 0; b < TN; ++b)
#pragma unroll
          for (int t = 0; t < TM; ++t) acc[b][t] = mma16<DT>(w[h][b], x[h][t], acc[b][t]);
      stage = stage == S - 1 ? 0 : stage + 1;
    }

    __syncthreads();   // every wave has read its ring
    f32x4 *const part = reinterpret_cast<f32x4 *>(smem);   // [NW][TN][TM][64]
    static_assert(TM * TN <= 2 * S * (TM + TN), "the rings' place");
#pragma unroll
    for (int b = 0; b < TN; ++b)
#pragma unroll
      for (int t = 0; t < TM; ++t) part[((wave * TN + b) * TM + t) * 64 + lane] = acc[b][t];
    __syncthreads();

    // item: 4 consecutive channels of one row
    for (int i = wave; i < NB * TM; i += NW) {
      const int b = i / TM, t = i % TM;
      f32x4 v = {0.f, 0.f, 0.f, 0.f}, u = v;
#pragma unroll
      for (int o = 0; o < NW; ++o) {
        v += part[((o * TN + (GATED ? 2 * b : b)) * TM + t) * 64 + lane];
        if constexpr (GATED) u += part[((o * TN + 2 * b + 1) * TM + t) * 64 + lane];
      }
      const int r = 16 * t + rl, ch = n0 + 16 * b + 4 * q;
      // (u's rows end in zeros, to ldy)
      if (r >= rows || ch >= (SHRINK || UP ? a.ldy : a.n)) continue;
      if constexpr (FC) {
        const float sum = (v[0] + v[1]) + (v[2] + v[3]);
        if (adapters.found && sum != sum)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (v[e] != v[e] && ch + e < a.n) v[e] = own_output<DT>(a, row0 + r, ch + e);
      }
      const int64_t to = (row0 + r) * a.ldy + ch;
      if constexpr (SHRINK) {   // (columns past the rank, to ldy, are written as zeros)
        if (a.ids[row0 + r] != seg) continue;
        const float scale = a.scale[seg];
        float h[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = ch + e < a.n ? v[e] * scale : 0.f;
        store_elems<DT, 4>(a.y, to, h);
        continue;
      }
      const bool whole = UP || (a.n % 4 == 0 && a.ldy % 4 == 0);
      float g[4], m[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        g[e] = v[e], m[e] = u[e];
        const int c = min(ch + e, a.n - 1);
        if (a.bias) {
          const raw *bias = reinterpret_cast<const raw *>(a.bias) + (int64_t)seg * a.w_rows;
          g[e] += E::to_f32(bias[c]);
          if constexpr (GATED) m[e] += E::to_f32(bias[a.n + c]);
        }
        if (FC && a.residual && ch + e < a.n)
          g[e] += E::to_f32(reinterpret_cast<const raw *>(a.residual)[to + e]);
      }
      if constexpr (MODE == kRowsDown) {   // fp32; past n lies the row's padding
        *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(a.y) + to) =
            f32x4{g[0], g[1], g[2], g[3]};
        continue;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        g[e] = FC ? row_act(g[e], a.act) : block_act<DT>(g[e], a.act);
        if constexpr (GATED) g[e] *= m[e];
        if constexpr (UP) g[e] = ch + e < a.n ? g[e] : 0.f;
      }
      if (whole) {
        store_elems<DT, 4>(a.y, to, g);
      } else {
        for (int e = 0; e < 4 && ch + e < a.n; ++e)
          reinterpret_cast<raw *>(a.y)[to + e] = E::from_f32(g[e]);
      }
    }
  }
}

template <int DT, RowsMode MODE, int TM, int TN, int NW, int S>
void launch_one(RowsArgs a, hipStream_t stream) {
  constexpr int BM = 16 * TM, BN = 16 * TN;
  const int64_t cols = cdiv(a.n, MODE == kRowsUpGated ? BN / 2 : BN);
  const int64_t row_tiles = MODE <= kRowsDown
                                ? a.rows / BM + std::min<int64_t>(a.experts, a.rows)
                                : cdiv(a.rows, BM);
  const unsigned grid = (unsigned)(8 * cdiv(row_tiles * cols, 8));
  rows_split_kernel<DT, MODE, TM, TN, NW, S><<<grid, 64 * NW, 0, stream>>>(a);
}

// Experts that serve few rows each, an FC of few rows: the tiles measured best
// (rows_tile_for).
template <int DT, RowsMode MODE>
void launch_mode(RowsTile tile, const RowsArgs &a, hipStream_t stream) {
  if constexpr (MODE != kRowsFc) launch_one<DT, MODE, 1, 4, 4, 2>(a, stream);   // 80 KB
  else if (tile == kTile32x32) launch_one<DT, MODE, 2, 2, 4, 2>(a, stream);     // 64 KB
  else launch_one<DT, MODE, 2, 2, 8, 2>(a, stream);                             // 128 KB
}

template <int DT>
void launch_shrink(const RowsArgs &a, hipStream_t stream) {
  if (a.n <= 16) launch_one<DT, kRowsShrink, 1, 1, 8, 4>(a, stream);
  else if (a.n <= 32) launch_one<DT, kRowsShrink, 1, 2, 8, 3>(a, stream);
  else launch_one<DT, kRowsShrink, 1, 4, 4, 3>(a, stream);
}

template <int DT>
void launch_dt(RowsMode mode, RowsTile tile, const RowsArgs &a, hipStream_t stream) {
  switch (mode) {
    case kRowsUp: return launch_mode<DT, kRowsUp>(tile, a, stream);
    case kRowsUpGated: return launch_mode<DT, kRowsUpGated>(tile, a, stream);
    case kRowsDownScaled: return;   // (tile kernel only)
    case kRowsDown: return launch_mode<DT, kRowsDown>(tile, a, stream);
    case kRowsFc: return launch_mode<DT, kRowsFc>(tile, a, stream);
    case kRowsShrink: return launch_shrink<DT>(a, stream);
  }
}

}  // namespace

sparoa_status launch_rows_split(RowsMode mode, RowsTile tile, const RowsArgs &a, sparoa_dtype dt,
                                hipStream_t stream) {
  switch (dt) {
    case SPAROA_F32: launch_dt<SPAROA_F32>(mode, tile, a, stream); break;
    case SPAROA_F16: launch_dt<SPAROA_F16>(mode, tile, a, stream); break;
    default: launch_dt<SPAROA_BF16>(mode, tile, a, stream); break;
  }
  SPAROA_LAUNCH_CHECK("row products, K split");
  return SPAROA_OK;
}

}  // namespace sparoa

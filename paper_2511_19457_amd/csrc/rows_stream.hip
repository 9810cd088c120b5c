// Products of few rows: the weights are streamed.
//
// A work-group has a panel of 16 NB output columns of one segment (an
// expert, or the one matrix of an FC) and 16 MT rows; its waves split K.  A
// wave's step is 128 bytes of K: lane l loads 32 bytes of weight row l & 15 of
// each 16-row block and of x row l & 15, straight into the MFMA's operands --
// each weight byte is read once and used for every row of the tile, so
// nothing is staged.  PF steps are in flight a wave.  The waves' partial
// tiles meet in LDS, added in wave order.
// Loads go through buffer descriptors: rows past the segment, columns past n
// and pieces past K have offsets past their range and read zero without a
// memory access.
// Bound by the weights' stream (16-bit decode: 2 bytes a weight, at most
// 16 MT products of it).
#include <algorithm>

#include "rows.h"

namespace sparoa {
namespace {

constexpr int kNW = 8, kNT = 64 * kNW;   // waves, threads
constexpr uint32_t kOut = 0x80000000u;   // past every descriptor's range

template <int DT, bool VEC>
struct Operand {
  using raw = typename Elem<DT>::raw;
  __amdgpu_buffer_rsrc_t rsrc;
  const raw *base;
  __device__ Operand(const void *p, int64_t bytes) {
    base = reinterpret_cast<const raw *>(p);
    if constexpr (VEC)
      rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), (short)0, (int)bytes,
                                               kBufDword3);
  }
  // 16 bytes of K from byte kb of the row at byte offset `row` (kOut: none).
  __device__ __forceinline__ u32x4 piece(uint32_t row, int kb, int kbytes) const {
    if constexpr (VEC) {
      return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                           rsrc, kb < kbytes ? row + kb : kOut, 0, 0));
    } else {   // rows that start anywhere: element by element
      constexpr int S = Elem<DT>::size;
      raw v[16 / S];
#pragma unroll
      for (int e = 0; e < 16 / S; ++e)
        v[e] = !(row & kOut) && kb + e * S < kbytes ? base[(row + kb) / S + e] : (raw)0;
      u32x4 r;
      __builtin_memcpy(&r, v, 16);
      return r;
    }
  }
};

template <int DT, bool VEC, RowsMode MODE, int MT, int NB>
__global__ __launch_bounds__(kNT) void rows_stream_kernel(RowsArgs a) {
  using E = Elem<DT>;
  constexpr bool GATED = MODE == kRowsUpGated, EXPERTS = MODE <= kRowsDown;
  constexpr int WB = GATED ? 2 * NB : NB;      // weight blocks of 16 rows
  constexpr int PF = VEC ? (WB + MT <= 3 ? 4 : 2) : 1;   // steps in flight
  __shared__ f32x4 part[kNW][WB * MT][64];
  __shared__ int32_t list[16 * MT];
  __shared__ int list_len;

  const int tid = threadIdx.x, lane = tid & 63, rl = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * 16 * NB;
  const int kbytes = a.k * E::size, steps = (kbytes + 127) / 128;

  uint32_t woff[WB];
#pragma unroll
  for (int b = 0; b < WB; ++b) {
    const int ch = n0 + 16 * (GATED ? b >> 1 : b) + rl;
    const int row = GATED && (b & 1) ? a.n + ch : ch;
    woff[b] = ch < a.n ? (uint32_t)row * (uint32_t)kbytes : kOut;
  }

  // experts: the blockIdx.y-th that has rows, its rows tile by tile; else
  // tiles of rows, every gridDim.y-th
  const int64_t groups = EXPERTS ? a.plan[a.experts + 1] : (a.rows + 16 * MT - 1) / (16 * MT);
  for (int64_t group = blockIdx.y; group < groups; group += gridDim.y) {
    int64_t s0, s1;
    int seg = 0, items = 1;
    if constexpr (EXPERTS) {
      seg = a.plan[a.experts + 2 + group];
      s0 = a.plan[seg], s1 = a.plan[seg + 1];
    } else {
      s0 = group * 16 * MT;
      s1 = s0 + 16 * MT < a.rows ? s0 + 16 * MT : a.rows;
    }
    if constexpr (MODE == kRowsShrink) {   // once for every adapter among the rows
      __syncthreads();                     // (the last tile's list has been read)
      if (wave == 0) {
        const int n =
            distinct_ids<(16 * MT + 63) / 64>(a.ids + s0, (int)(s1 - s0), a.adapters, list);
        if (lane == 0) list_len = n;
      }
      __syncthreads();
      items = list_len;
    }

    for (int item = 0; item < items; ++item)
      for (int64_t r0 = s0; r0 < s1; r0 += 16 * MT) {
        if constexpr (MODE == kRowsShrink) seg = list[item];
        const Operand<DT, VEC> w(reinterpret_cast<const char *>(a.w) + (int64_t)seg * a.w_stride * E::size,
                                 (int64_t)a.w_rows * kbytes);
        const bool gather = EXPERTS && a.order;
        const Operand<DT, VEC> x(
            gather ? a.x : reinterpret_cast<const char *>(a.x) + r0 * a.ldx * E::size,
            gather ? a.x_bytes : std::min<int64_t>(s1 - r0, 16 * MT) * a.ldx * E::size);
        uint32_t xoff[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          const int64_t p = r0 + 16 * t + rl;
          bool in = p < s1;
          uint32_t row = 16 * t + rl;
          if (gather && in) row = (uint32_t)a.order[p] / (uint32_t)a.top_k;
          if (MODE == kRowsShrink && in) in = a.ids[p] == seg;
          xoff[t] = in ? row * (uint32_t)(a.ldx * E::size) : kOut;
        }

        f32x4 acc[WB][MT];
#pragma unroll
        for (int b = 0; b < WB; ++b)
#pragma unroll
          for (int t = 0; t < MT; ++t) acc[b][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        u32x4 wq[PF][WB][2], xq[PF][MT][2];
        auto load = [&](int i, int step) __attribute__((always_inline)) {
          const int kb = step * 128 + q * 32;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int b = 0; b < WB; ++b)
              wq[i][b][h] = w.piece(woff[b], kb + 16 * h, kbytes);
#pragma unroll
            for (int t = 0; t < MT; ++t)
              xq[i][t][h] = x.piece(xoff[t], kb + 16 * h, kbytes);
          }
        };
#pragma unroll
        for (int i = 0; i < PF; ++i) load(i, wave + i * kNW);
        for (int s = wave; s < steps; s += PF * kNW) {
#pragma unroll
          for (int i = 0; i < PF; ++i) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int b = 0; b < WB; ++b)
#pragma unroll
                for (int t = 0; t < MT; ++t)
                  acc[b][t] = mma16<DT>(wq[i][b][h], xq[i][t][h], acc[b][t]);
            load(i, s + (i + PF) * kNW);
          }
        }
        __syncthreads();   // the last tile's partial sums have been read
#pragma unroll
        for (int b = 0; b < WB; ++b)
#pragma unroll
          for (int t = 0; t < MT; ++t) part[wave][b * MT + t][lane] = acc[b][t];
        __syncthreads();

        // item: 4 consecutive channels of one row
        for (int i = wave; i < NB * MT; i += kNW) {
          const int b = i / MT, t = i % MT;
          f32x4 v = {0.f, 0.f, 0.f, 0.f}, u = v;
#pragma unroll
          for (int o = 0; o < kNW; ++o) v += part[o][(GATED ? 2 * b : b) * MT + t][lane];
          if constexpr (GATED)
#pragma unroll
            for (int o = 0; o < kNW; ++o) u += part[o][(2 * b + 1) * MT + t][lane];
          const int64_t p = r0 + 16 * t + rl;
          const int ch = n0 + 16 * b + 4 * q;
          if (p >= s1 || ch >= a.n) continue;
          if constexpr (MODE == kRowsShrink) {
            if (a.ids[p] != seg) continue;
            v *= a.scale[seg];
            for (int e = 0; e < 4 && ch + e < a.n; ++e) {
              if (a.h_f32) reinterpret_cast<float *>(a.y)[p * a.ldy + ch + e] = v[e];
              else reinterpret_cast<typename E::raw *>(a.y)[p * a.ldy + ch + e] = E::from_f32(v[e]);
            }
            continue;
          }
          if constexpr (MODE == kRowsDown) {   // fp32: what the weighted sum adds up
            if (a.bias)
              for (int e = 0; e < 4 && ch + e < a.n; ++e)
                v[e] += E::to_f32(reinterpret_cast<const typename E::raw *>(
                    a.bias)[(int64_t)seg * a.n + ch + e]);
            // (ldy % 4 == 0; past n lies the row's padding)
            *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(a.y) + p * a.ldy + ch) = v;
            continue;
          }
          float o[4];
          const int adapter = MODE == kRowsFc && a.ids ? a.ids[p] : -1;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float g = v[e], up = u[e];
            const int c = ch + e < a.n ? ch + e : a.n - 1;
            if (a.bias) {
              const typename E::raw *bias =
                  reinterpret_cast<const typename E::raw *>(a.bias) + (int64_t)seg * a.w_rows;
              g += E::to_f32(bias[c]);
              if (GATED) up += E::to_f32(bias[a.n + c]);
            }
            if (MODE == kRowsFc && (uint32_t)adapter < (uint32_t)a.adapters) {
              const float *h = reinterpret_cast<const float *>(a.h) + p * a.ldh;
              const int64_t at = ((int64_t)adapter * a.n + c) * a.rank;
              float d = 0.f;
              if (a.rank % 8 == 0) {   // (rows of b start on 16 bytes)
                for (int r = 0; r < a.rank; r += 8) {
                  float bv[8];
                  if constexpr (E::size == 2) {
                    load_elems<DT, 8>(a.b, at + r, bv);
                  } else {
                    float lo[4], hi[4];
                    load_elems<DT, 4>(a.b, at + r, lo);
                    load_elems<DT, 4>(a.b, at + r + 4, hi);
#pragma unroll
                    for (int z = 0; z < 4; ++z) bv[z] = lo[z], bv[4 + z] = hi[z];
                  }
#pragma unroll
                  for (int z = 0; z < 8; ++z) d = fmaf(h[r + z], bv[z], d);
                }
              } else {
                for (int r = 0; r < a.rank; ++r)
                  d = fmaf(h[r], E::to_f32(reinterpret_cast<const typename E::raw *>(a.b)[at + r]), d);
              }
              g += d;
            }
            if (MODE == kRowsFc && a.residual)
              g += E::to_f32(reinterpret_cast<const typename E::raw *>(a.residual)[p * a.ldy + c]);
            o[e] = block_act(g, a.act);
            if (GATED) o[e] *= up;
          }
          if (a.ldy % 4 == 0 && ch + 4 <= a.n) {
            store_elems<DT, 4>(a.y, p * a.ldy + ch, o);
          } else {
            for (int e = 0; e < 4 && ch + e < a.n; ++e)
              reinterpret_cast<typename E::raw *>(a.y)[p * a.ldy + ch + e] = E::from_f32(o[e]);
          }
        }
      }
  }
}

template <int DT, bool VEC, RowsMode MODE, int MT, int NB>
void launch_one(const RowsArgs &a, hipStream_t stream) {
  const int64_t groups = MODE <= kRowsDown ? std::min<int64_t>(a.experts, a.rows)
                                           : cdiv(a.rows, 16 * MT);
  const dim3 grid((unsigned)cdiv(a.n, 16 * NB), (unsigned)std::min<int64_t>(groups, 32768));
  rows_stream_kernel<DT, VEC, MODE, MT, NB><<<grid, kNT, 0, stream>>>(a);
}

// Rows a tile: as few 16-row blocks as hold an average segment.
template <int DT, bool VEC, RowsMode MODE>
void launch_mode(const RowsArgs &a, hipStream_t stream) {
  const int64_t per = MODE <= kRowsDown ? cdiv(a.rows, std::min<int64_t>(a.experts, a.rows))
                                        : a.rows;
  if constexpr (MODE == kRowsShrink) {
    launch_one<DT, VEC, MODE, 1, 1>(a, stream);
  } else if constexpr (!VEC) {
    launch_one<DT, VEC, MODE, 4, 1>(a, stream);
  } else {
    constexpr int NB = MODE == kRowsUpGated ? 1 : 2;
    if (per <= 16) launch_one<DT, VEC, MODE, 1, NB>(a, stream);
    else if (per <= 32) launch_one<DT, VEC, MODE, 2, NB>(a, stream);
    else launch_one<DT, VEC, MODE, 4, NB>(a, stream);
  }
}

template <int DT>
void launch_dt(RowsMode mode, const RowsArgs &a, bool vec, hipStream_t stream) {
#define SPAROA_ROWS(M)                                     \
  case M:                                                  \
    if (vec) launch_mode<DT, true, M>(a, stream);          \
    else launch_mode<DT, false, M>(a, stream);             \
    break
  switch (mode) {
    SPAROA_ROWS(kRowsUp);
    SPAROA_ROWS(kRowsUpGated);
    SPAROA_ROWS(kRowsDown);
    SPAROA_ROWS(kRowsFc);
    SPAROA_ROWS(kRowsShrink);
  }
#undef SPAROA_ROWS
}

template <int DT, int V>
__global__ __launch_bounds__(256) void combine_kernel(CombineArgs a) {
  const int64_t per = a.hidden / V, total = a.tokens * per;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
    const int64_t t = i / per, c = i % per * V;
    float s[V];
#pragma unroll
    for (int e = 0; e < V; ++e) s[e] = 0.f;
    for (int j = 0; j < a.top_k; ++j) {
      const int p = a.place[t * a.top_k + j];
      if (p < 0) continue;   // no expert: its weight is not looked at
      const float w = a.weights[t * a.top_k + j];
      const float *z = a.z + p * a.ldz + c;
      if constexpr (V % 4 == 0) {
#pragma unroll
        for (int e = 0; e < V; e += 4) {
          const f32x4 q = *reinterpret_cast<const f32x4 *>(z + e);
#pragma unroll
          for (int i = 0; i < 4; ++i) s[e + i] = fmaf(w, q[i], s[e + i]);
        }
      } else {
        s[0] = fmaf(w, z[0], s[0]);
      }
    }
    if (a.residual) {
      float r[V];
      load_elems<DT, V>(a.residual, t * a.hidden + c, r);
#pragma unroll
      for (int e = 0; e < V; ++e) s[e] += r[e];
    }
    store_elems<DT, V>(a.y, t * a.hidden + c, s);
  }
}

template <int DT>
void launch_combine_dt(const CombineArgs &a, hipStream_t stream) {
  constexpr int V = 16 / Elem<DT>::size;
  const bool vec = a.hidden % V == 0;
  const int64_t items = a.tokens * (vec ? a.hidden / V : a.hidden);
  const unsigned grid = (unsigned)std::min<int64_t>(cdiv(items, 256), 1 << 20);
  if (vec) combine_kernel<DT, V><<<grid, 256, 0, stream>>>(a);
  else combine_kernel<DT, 1><<<grid, 256, 0, stream>>>(a);
}

}  // namespace

bool rows_tiled(RowsMode mode, const RowsArgs &a, sparoa_dtype dt) {
  const int v = 16 / (int)elem_size(dt);
  if (mode == kRowsShrink || a.k % v || a.ldx % v) return false;
  if (mode == kRowsFc)
    return a.rank % v == 0 && a.rows > 256 && cdiv(a.rows, 128) * cdiv(a.n, 256) >= 128;
  return a.rows / std::min<int64_t>(a.experts, a.rows) > 64;
}

sparoa_status launch_rows(RowsMode mode, const RowsArgs &a, sparoa_dtype dt, hipStream_t stream) {
  if (rows_tiled(mode, a, dt)) return launch_rows_tile(mode, a, dt, stream);
  const int v = 16 / (int)elem_size(dt);
  const bool vec = a.k % v == 0 && a.ldx % v == 0;   // rows of x and w start on 16 bytes
  switch (dt) {
    case SPAROA_F32: launch_dt<SPAROA_F32>(mode, a, vec, stream); break;
    case SPAROA_F16: launch_dt<SPAROA_F16>(mode, a, vec, stream); break;
    default: launch_dt<SPAROA_BF16>(mode, a, vec, stream); break;
  }
  SPAROA_LAUNCH_CHECK("row products");
  return SPAROA_OK;
}

sparoa_status launch_combine(const CombineArgs &a, sparoa_dtype dt, hipStream_t stream) {
  switch (dt) {
    case SPAROA_F32: launch_combine_dt<SPAROA_F32>(a, stream); break;
    case SPAROA_F16: launch_combine_dt<SPAROA_F16>(a, stream); break;
    default: launch_combine_dt<SPAROA_BF16>(a, stream); break;
  }
  SPAROA_LAUNCH_CHECK("expert_ffn: combine");
  return SPAROA_OK;
}

}  // namespace sparoa

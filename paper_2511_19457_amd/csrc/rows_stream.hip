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

// A word every lane wants alike, by the scalar unit: memory that no kernel of
// this launch writes.
__device__ __forceinline__ int uniform_word(const int32_t *p) {
  return *reinterpret_cast<const __attribute__((address_space(4))) int32_t *>(
      reinterpret_cast<uintptr_t>(p));
}

// One operand matrix.  VEC: 16-byte pieces by buffer loads; else element by
// element (rows that start anywhere).
template <int DT, bool VEC>
struct Operand {
  using raw = typename Elem<DT>::raw;
  const void *base;
  int bytes;
  __device__ Operand(const void *p, int64_t n) : base(p), bytes((int)n) {}
  // 16 bytes of K from byte kb + at of the row at byte offset `row` (kOut:
  // none); kb alike in every lane, at < 128.  VEC: the whole 16 bytes lie
  // before kbytes, or kb does not and they read zero.
  __device__ __forceinline__ u32x4 piece(uint32_t row, int kb, int at, int kbytes) const {
    if constexpr (VEC) {
      const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<void *>(base), (short)0, kb < kbytes ? bytes : 0, kBufDword3);
      return __builtin_bit_cast(u32x4,
                                __builtin_amdgcn_raw_buffer_load_b128(rsrc, row + at, kb, 0));
    } else {
      constexpr int S = Elem<DT>::size;
      raw v[16 / S];
#pragma unroll
      for (int e = 0; e < 16 / S; ++e)
        v[e] = !(row & kOut) && kb + at + e * S < kbytes
                   ? reinterpret_cast<const raw *>(base)[(row + kb + at) / S + e]
                   : (raw)0;
      u32x4 r;
      __builtin_memcpy(&r, v, 16);
      return r;
    }
  }
};

// sum over the rank of h[row] b[adapter of row][ch].
template <int DT>
__device__ __forceinline__ float adapter_share(const RowsArgs &a, int64_t row, int ch) {
  using E = Elem<DT>;
  const int id = a.ids[row];
  if ((uint32_t)id >= (uint32_t)a.adapters) return 0.f;
  const float *h = reinterpret_cast<const float *>(a.h) + row * a.ldh;
  const int64_t at = ((int64_t)id * a.n + ch) * a.rank;
  float d = 0.f;
  constexpr int V = 16 / E::size;
  if (a.rank % V == 0) {   // (rows of b start on 16 bytes)
#pragma unroll 2
    for (int r = 0; r < a.rank; r += V) {
      float bv[V];
      load_elems<DT, V>(a.b, at + r, bv);
#pragma unroll
      for (int e = 0; e < V; e += 4) {
        const f32x4 hv = *reinterpret_cast<const f32x4 *>(h + r + e);
#pragma unroll
        for (int z = 0; z < 4; ++z) d = fmaf(hv[z], bv[e + z], d);
      }
    }
  } else {
    for (int r = 0; r < a.rank; ++r)
      d = fmaf(h[r], E::to_f32(reinterpret_cast<const typename E::raw *>(a.b)[at + r]), d);
  }
  return d;
}

// h[row][r] = scale_a a_a[r] x[row]: a wave per row and r (few rows, where
// their adapters differ).
template <int DT, bool VEC>
__global__ __launch_bounds__(256) void shrink_rows_kernel(RowsArgs a) {
  using E = Elem<DT>;
  using raw = typename E::raw;
  const int64_t row = blockIdx.y;
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int id = a.ids[row];
  if (r >= a.n || (uint32_t)id >= (uint32_t)a.adapters) return;   // (whole waves)
  const raw *x = reinterpret_cast<const raw *>(a.x) + row * a.ldx;
  const raw *w = reinterpret_cast<const raw *>(a.w) + id * a.w_stride + (int64_t)r * a.k;
  constexpr int V = VEC ? 16 / E::size : 1;
  float s = 0.f;
#pragma unroll 4
  for (int k = lane * V; k < a.k; k += 64 * V) {
    float xv[V], wv[V];
    load_elems<DT, V>(x, k, xv);
    load_elems<DT, V>(w, k, wv);
#pragma unroll
    for (int e = 0; e < V; ++e) s = fmaf(xv[e], wv[e], s);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  if (lane == 0) reinterpret_cast<float *>(a.y)[row * a.ldy + r] = s * a.scale[id];
}

// (VEC, up to 32 rows: two work-groups a CU, one's start and end under the
// other's stream)
template <int DT, bool VEC, RowsMode MODE, int MT, int NB>
__global__ __launch_bounds__(kNT, VEC && MODE != kRowsFc && MT <= 2 && NB <= 2 ? 4 : 2) void rows_stream_kernel(RowsArgs a) {
  using E = Elem<DT>;
  constexpr bool GATED = MODE == kRowsUpGated, EXPERTS = MODE <= kRowsDown;
  constexpr int WB = GATED ? 2 * NB : NB;      // weight blocks of 16 rows
  constexpr bool FC = MODE == kRowsFc;
  constexpr int PF = VEC ? std::max(2, (FC ? 12 : 8) / (WB + MT)) : 1;   // steps in flight
  __shared__ f32x4 part[kNW][WB * MT][64];
  __shared__ float tail[FC ? 16 * MT : 1][FC ? 16 * NB + 1 : 1];   // the adapters' share
  __shared__ int32_t list[MODE == kRowsShrink ? 16 * MT : 1];
  __shared__ int list_len;

  const int tid = threadIdx.x, lane = tid & 63, rl = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * 16 * NB;
  const int kbytes = a.k * E::size;
  // whole steps; VEC: what is left of K is a step of its own, behind them
  const int steps = VEC ? kbytes / 128 : (kbytes + 127) / 128;

  uint32_t woff[WB];
#pragma unroll
  for (int b = 0; b < WB; ++b) {
    const int ch = n0 + 16 * (GATED ? b >> 1 : b) + rl;
    const int row = GATED && (b & 1) ? a.n + ch : ch;
    woff[b] = ch < a.n ? (uint32_t)row * (uint32_t)kbytes : kOut;
  }

  // experts: the blockIdx.y-th that has rows, its rows tile by tile; else
  // tiles of rows, every gridDim.y-th
  const int64_t groups = EXPERTS ? uniform_word(a.plan + a.experts + 1) : (a.rows + 16 * MT - 1) / (16 * MT);
  for (int64_t group = blockIdx.y; group < groups; group += gridDim.y) {
    int64_t s0, s1;
    int seg = 0, items = 1;
    if constexpr (EXPERTS) {
      seg = uniform_word(a.plan + a.experts + 2 + group);
      s0 = uniform_word(a.plan + seg), s1 = uniform_word(a.plan + seg + 1);
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
        int slot[MT];   // (sent for first: loads land in order)
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          const int64_t p = r0 + 16 * t + rl < s1 ? r0 + 16 * t + rl : s1 - 1;
          slot[t] = gather ? a.order[p] : MODE == kRowsShrink ? a.ids[p] : 0;
        }

        f32x4 acc[WB][MT];
#pragma unroll
        for (int b = 0; b < WB; ++b)
#pragma unroll
          for (int t = 0; t < MT; ++t) acc[b][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        u32x4 wq[PF][WB][2], xq[PF][MT][2];
        uint32_t xoff[MT];
        auto load_w = [&](int i, int kb, int end) __attribute__((always_inline)) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int b = 0; b < WB; ++b) wq[i][b][h] = w.piece(woff[b], kb, q * 32 + 16 * h, end);
        };
        auto load_x = [&](int i, int kb, int end) __attribute__((always_inline)) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int t = 0; t < MT; ++t) xq[i][t][h] = x.piece(xoff[t], kb, q * 32 + 16 * h, end);
        };
        auto multiply = [&](int i) __attribute__((always_inline)) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int b = 0; b < WB; ++b)
#pragma unroll
              for (int t = 0; t < MT; ++t)
                acc[b][t] = mma16<DT>(wq[i][b][h], xq[i][t][h], acc[b][t]);
        };
        const int kend = VEC ? steps * 128 : kbytes;
        // (the weights are sent for before the rows' places are known)
#pragma unroll
        for (int i = 0; i < PF; ++i) load_w(i, (wave + i * kNW) * 128, kend);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          uint32_t row = 16 * t + rl;
          const bool in = r0 + row < s1 && (MODE != kRowsShrink || slot[t] == seg);
          if (gather) row = (uint32_t)slot[t] / (uint32_t)a.top_k;
          xoff[t] = in ? row * (uint32_t)(a.ldx * E::size) : kOut;
        }
#pragma unroll
        for (int i = 0; i < PF; ++i) load_x(i, (wave + i * kNW) * 128, kend);
        for (int s = wave; s < steps; s += PF * kNW) {
#pragma unroll
          for (int i = 0; i < PF; ++i) {
            multiply(i);
            load_w(i, (s + (i + PF) * kNW) * 128, kend);
            load_x(i, (s + (i + PF) * kNW) * 128, kend);
          }
        }
        if (VEC && kend < kbytes && wave == steps % kNW) {   // pieces past K read zero
          const uint32_t past0 = kend + q * 32 < kbytes ? 0u : kOut;
          const uint32_t past1 = kend + q * 32 + 16 < kbytes ? 0u : kOut;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int b = 0; b < WB; ++b)
              wq[0][b][h] = w.piece(woff[b] | (h ? past1 : past0), kend, q * 32 + 16 * h, kbytes);
#pragma unroll
            for (int t = 0; t < MT; ++t)
              xq[0][t][h] = x.piece(xoff[t] | (h ? past1 : past0), kend, q * 32 + 16 * h, kbytes);
          }
          multiply(0);
        }
        __syncthreads();   // the last tile's partial sums have been read
        // the adapters' share of an output is one thread's sum over the rank
        if constexpr (FC) {
          if (a.ids)
            for (int i = tid; i < 256 * MT * NB; i += kNT) {
              const int r = i / (16 * NB), c = i % (16 * NB);
              tail[r][c] = r0 + r < s1 && n0 + c < a.n ? adapter_share<DT>(a, r0 + r, n0 + c) : 0.f;
            }
        }
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
          float o[4], mul[4];
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
            if (FC && a.ids) g += tail[16 * t + rl][16 * b + 4 * q + e];
            if (FC && a.residual)
              g += E::to_f32(reinterpret_cast<const typename E::raw *>(a.residual)[p * a.ldy + c]);
            o[e] = g, mul[e] = up;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            o[e] = FC ? apply_act(o[e], a.act) : block_act(o[e], a.act);
            if (GATED) o[e] *= mul[e];
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
    // a wave per row and rank where all that these read is little (they share
    // nothing but the L2), else tiles of 16 rows that read x once
    if (a.h_f32 && a.rows <= 32768 &&
        a.rows * a.n * a.k * Elem<DT>::size <= (int64_t)32 << 20) {
      const dim3 grid((unsigned)cdiv(a.n, 4), (unsigned)a.rows);
      shrink_rows_kernel<DT, VEC><<<grid, 256, 0, stream>>>(a);
    } else if (a.n <= 16 || !VEC) {
      launch_one<DT, VEC, MODE, 1, 1>(a, stream);
    } else if (a.n <= 32) {
      launch_one<DT, VEC, MODE, 1, 2>(a, stream);
    } else {
      launch_one<DT, VEC, MODE, 1, 4>(a, stream);
    }
  } else if constexpr (!VEC) {
    launch_one<DT, VEC, MODE, 4, 1>(a, stream);
  } else {
    constexpr int NB = MODE == kRowsUpGated ? 1 : 2;
    if (MODE == kRowsFc && cdiv(a.n, 32) * cdiv(a.rows, per <= 16 ? 16 : per <= 32 ? 32 : 64) < 160) {
      // panels of 16 columns where those of 32 leave too many CUs without one
      if (per <= 16) launch_one<DT, VEC, MODE, 1, 1>(a, stream);
      else if (per <= 32) launch_one<DT, VEC, MODE, 2, 1>(a, stream);
      else launch_one<DT, VEC, MODE, 4, 1>(a, stream);
      return;
    }
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
    for (int j0 = 0; j0 < a.top_k; j0 += 8) {   // eight rows in flight
      int p[8];
      float w[8], z[8][V];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int64_t slot = t * a.top_k + (j0 + j < a.top_k ? j0 + j : 0);
        p[j] = j0 + j < a.top_k ? a.place[slot] : -1;
        w[j] = a.weights[slot];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float *from = a.z + (p[j] < 0 ? 0 : p[j]) * a.ldz + c;
        if constexpr (V % 4 == 0) {
#pragma unroll
          for (int e = 0; e < V; e += 4) {
            const f32x4 q = *reinterpret_cast<const f32x4 *>(from + e);
#pragma unroll
            for (int i = 0; i < 4; ++i) z[j][e + i] = q[i];
          }
        } else {
          z[j][0] = from[0];
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)   // no expert: neither weight nor row is looked at
#pragma unroll
        for (int e = 0; e < V; ++e) s[e] = p[j] < 0 ? s[e] : fmaf(w[j], z[j][e], s[e]);
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

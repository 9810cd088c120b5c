// Row products whose rows start off 16 bytes (k no multiple of a 16-byte
// vector) and are few: any size and alignment (many rows are copied to aligned
// ones first).  Bound by the loads' latency and the shifting: FC of 16 x 6143 x
// 2048 bf16 38 us with its adapters' product, 21 experts of 278 x 1928 with 11
// fp16 rows each 53 us.
//
// A work-group has a panel of 16 NB output columns of one segment (an
// expert, or the one matrix of an FC) and 16 MT rows; its waves split K.  A
// wave's step is 128 bytes of K: lane l loads 32 bytes of weight row l & 15 of
// each 16-row block and of x row l & 15, straight into the MFMA's operands.  A
// 16-byte piece of 16-bit elements may start between two words: five words
// are loaded and shifted into place.  The waves' partial tiles meet in LDS,
// added in wave order.  The adapters' share of an output is a thread's sum over
// the rank in fp32.
// Loads go through buffer descriptors: rows past the segment and columns past
// n have offsets past their range and read zero without a memory access;
// elements past K are masked.
#include <algorithm>

#include "rows.h"

namespace sparoa {
namespace {

constexpr int kNW = 8, kNT = 64 * kNW;   // waves, threads

// One operand matrix: 16-byte pieces of rows at any element.
template <int DT>
struct Operand {
  static constexpr int S = Elem<DT>::size;
  __amdgpu_buffer_rsrc_t rsrc;
  uint32_t lead;   // bytes from the descriptor's word-aligned base to the matrix
  struct Piece {
    u32x4 q;
    uint32_t tail;   // (16-bit) the word behind q
  };
  __device__ Operand(const void *p, int64_t n) {
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    lead = S == 2 ? (uint32_t)at & 2u : 0u;
    // (to the end of the last element's word: a word past the range reads zero)
    rsrc = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(at - lead), (short)0,
                                             (int)((n + lead + 3) & ~3ll), kBufDword3);
  }
  // The words that hold bytes [kb, kb + 16) of the row at byte offset `row`
  // (kOut: none).
  __device__ __forceinline__ Piece request(uint32_t row, int kb, int kbytes) const {
    const uint32_t at = kb < kbytes ? (row + lead + kb) & ~3u : kOut;
    Piece p;
    p.q = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, 0, 0));
    p.tail = S == 2 ? __builtin_amdgcn_raw_buffer_load_b32(rsrc, at + 16, 0, 0) : 0u;
    return p;
  }
  // The piece itself, zeros past K.
  __device__ __forceinline__ u32x4 value(const Piece &p, uint32_t row, int kb, int kbytes) const {
    u32x4 v = p.q;
    if constexpr (S == 2) {
      const uint32_t by = (row + lead + kb) & 2u;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        v[i] = __builtin_amdgcn_alignbyte(i < 3 ? p.q[i + 1] : p.tail, p.q[i], by);
    }
    const int left = (kbytes - kb) / S;   // elements of the piece before K's end
    if (left < 16 / S) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (S == 4) v[i] = i < left ? v[i] : 0u;
        else v[i] &= 2 * i + 1 < left ? ~0u : 2 * i < left ? 0xFFFFu : 0u;
      }
    }
    return v;
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

template <int DT, RowsMode MODE, int MT, int NB>
__global__ __launch_bounds__(kNT, 2) void rows_stream_kernel(RowsArgs a) {
  using E = Elem<DT>;
  constexpr bool GATED = MODE == kRowsUpGated, EXPERTS = MODE <= kRowsDown;
  constexpr int WB = GATED ? 2 * NB : NB;      // weight blocks of 16 rows
  constexpr bool FC = MODE == kRowsFc;
  constexpr int PF = 2;   // steps in flight
  __shared__ f32x4 part[kNW][WB * MT][64];
  __shared__ float tail[FC ? 16 * MT : 1][FC ? 16 * NB + 1 : 1];   // the adapters' share
  __shared__ int32_t list[MODE == kRowsShrink ? 16 * MT : 1];
  __shared__ int list_len;

  const int tid = threadIdx.x, lane = tid & 63, rl = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * 16 * NB;
  const int kbytes = a.k * E::size;
  const int steps = (kbytes + 127) / 128;

  uint32_t woff[WB];
#pragma unroll
  for (int b = 0; b < WB; ++b) {
    const int ch = n0 + 16 * (GATED ? b >> 1 : b) + rl;
    const int row = GATED && (b & 1) ? a.n + ch : ch;
    woff[b] = ch < a.n ? (uint32_t)row * (uint32_t)kbytes : kOut;
  }

  // experts: the blockIdx.y-th that has rows, its rows tile by tile; else
  // tiles of rows, every gridDim.y-th
  const int64_t groups = EXPERTS ? uniform_word(a.plan + a.experts + 1)
                                 : (a.rows + 16 * MT - 1) / (16 * MT);
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
        const Operand<DT> w(reinterpret_cast<const char *>(a.w) + (int64_t)seg * a.w_stride * E::size,
                                 (int64_t)a.w_rows * kbytes);
        const bool gather = EXPERTS && a.order;
        const Operand<DT> x(
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
        typename Operand<DT>::Piece wq[PF][WB][2], xq[PF][MT][2];
        uint32_t xoff[MT];
        auto load_w = [&](int i, int kb) __attribute__((always_inline)) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int b = 0; b < WB; ++b)
              wq[i][b][h] = w.request(woff[b], kb + q * 32 + 16 * h, kbytes);
        };
        auto load_x = [&](int i, int kb) __attribute__((always_inline)) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int t = 0; t < MT; ++t)
              xq[i][t][h] = x.request(xoff[t], kb + q * 32 + 16 * h, kbytes);
        };
        auto multiply = [&](int i, int kb) __attribute__((always_inline)) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            u32x4 wv[WB];
#pragma unroll
            for (int b = 0; b < WB; ++b)
              wv[b] = w.value(wq[i][b][h], woff[b], kb + q * 32 + 16 * h, kbytes);
#pragma unroll
            for (int t = 0; t < MT; ++t) {
              const u32x4 xv = x.value(xq[i][t][h], xoff[t], kb + q * 32 + 16 * h, kbytes);
#pragma unroll
              for (int b = 0; b < WB; ++b) acc[b][t] = mma16<DT>(wv[b], xv, acc[b][t]);
            }
          }
        };
        // (the weights are sent for before the rows' places are known)
#pragma unroll
        for (int i = 0; i < PF; ++i) load_w(i, (wave + i * kNW) * 128);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          uint32_t row = 16 * t + rl;
          const bool in = r0 + row < s1 && (MODE != kRowsShrink || slot[t] == seg);
          if (gather) row = (uint32_t)slot[t] / (uint32_t)a.top_k;
          xoff[t] = in ? row * (uint32_t)(a.ldx * E::size) : kOut;
        }
#pragma unroll
        for (int i = 0; i < PF; ++i) load_x(i, (wave + i * kNW) * 128);
        for (int s = wave; s < steps; s += PF * kNW) {
#pragma unroll
          for (int i = 0; i < PF; ++i) {
            multiply(i, (s + i * kNW) * 128);
            load_w(i, (s + (i + PF) * kNW) * 128);
            load_x(i, (s + (i + PF) * kNW) * 128);
          }
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
            for (int e = 0; e < 4 && ch + e < a.n; ++e)   // (h is fp32 here)
              reinterpret_cast<float *>(a.y)[p * a.ldy + ch + e] = v[e];
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
            o[e] = FC ? row_act(o[e], a.act) : block_act<DT>(o[e], a.act);
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

template <int DT, RowsMode MODE, int MT, int NB>
void launch_one(const RowsArgs &a, hipStream_t stream) {
  const int64_t groups = MODE <= kRowsDown ? std::min<int64_t>(a.experts, a.rows)
                                           : cdiv(a.rows, 16 * MT);
  const dim3 grid((unsigned)cdiv(MODE == kRowsShrink ? a.ldy : a.n, 16 * NB),
                  (unsigned)std::min<int64_t>(groups, 32768));
  rows_stream_kernel<DT, MODE, MT, NB><<<grid, kNT, 0, stream>>>(a);
}

// Rows a tile: one block of 16 where that holds an average segment.
template <int DT, RowsMode MODE>
void launch_mode(const RowsArgs &a, hipStream_t stream) {
  constexpr int NB = MODE == kRowsUpGated ? 1 : 2;
  const int64_t per = MODE <= kRowsDown ? cdiv(a.rows, std::min<int64_t>(a.experts, a.rows))
                                        : a.rows;
  if (MODE == kRowsShrink || per <= 16) launch_one<DT, MODE, 1, NB>(a, stream);
  else if constexpr (MODE != kRowsShrink) launch_one<DT, MODE, 4, NB>(a, stream);
}

template <int DT>
void launch_dt(RowsMode mode, const RowsArgs &a, hipStream_t stream) {
  switch (mode) {
    case kRowsUp: return launch_mode<DT, kRowsUp>(a, stream);
    case kRowsUpGated: return launch_mode<DT, kRowsUpGated>(a, stream);
    case kRowsDownScaled: return;   // (tile kernel only)
    case kRowsDown: return launch_mode<DT, kRowsDown>(a, stream);
    case kRowsFc: return launch_mode<DT, kRowsFc>(a, stream);
    case kRowsShrink: return launch_mode<DT, kRowsShrink>(a, stream);
  }
}

}  // namespace

sparoa_status launch_rows_stream(RowsMode mode, const RowsArgs &a, sparoa_dtype dt,
                                 hipStream_t stream) {
  switch (dt) {
    case SPAROA_F32: launch_dt<SPAROA_F32>(mode, a, stream); break;
    case SPAROA_F16: launch_dt<SPAROA_F16>(mode, a, stream); break;
    default: launch_dt<SPAROA_BF16>(mode, a, stream); break;
  }
  SPAROA_LAUNCH_CHECK("row products");
  return SPAROA_OK;
}

}  // namespace sparoa

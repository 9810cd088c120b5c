// Rings of K chunks in LDS, and the walk over tiles, of the row-product
// kernels.
#pragma once

#include "rows.h"

namespace sparoa {

constexpr int kRow = 128;                // bytes of a chunk row

// s_waitcnt immediates: at most n vector-memory operations outstanding; LDS
// operations done.
constexpr int vm_outstanding(int n) { return (n & 15) | (7 << 4) | (15 << 8) | ((n >> 4) << 14); }
constexpr int kLdsDone = 15 | (7 << 4) | (3 << 14);

// Waits until all but this wave's newest `chunks` <= C chunks' loads (L per
// chunk) have landed.
template <int C, int L>
__device__ __forceinline__ void wait_ring(int chunks) {
  static_assert(C * L < 64, "vmcnt range");
  if constexpr (C > 0) {
    if (chunks < C) return wait_ring<C - 1, L>(chunks);
  }
  __builtin_amdgcn_s_waitcnt(vm_outstanding(C * L));
}

// A 16-byte-per-lane buffer load whose data goes to LDS (lane l's to lds + 16
// l, lds uniform), zeros where the offset is past the range.  In assembly: by
// the builtin the compiler cannot tell the ring's stages apart and waits for
// every load in flight before each LDS read; the waits are at the barriers
// instead (wait_ring).  It writes no register.  The wait states: a scalar
// register that a vector instruction wrote (a descriptor from
// v_readfirstlane, a reloaded one) may be read by a memory instruction five
// states later, and the compiler does not look into the statement.
__device__ __forceinline__ void ring_load(u32x4 rsrc, uint32_t lds, uint32_t voffset,
                                          uint32_t soffset) {
  asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :
               : "{m0}"(lds), "v"(voffset), "s"(rsrc), "s"(soffset)
               : "memory");
}
__device__ __forceinline__ u32x4 descriptor(const void *p, int64_t bytes) {
  const uint64_t b = reinterpret_cast<uint64_t>(p);
  return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)b),
               (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(b >> 32) & 0xFFFF),
               (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)bytes),
               (uint32_t)kBufDword3};
}

// The chunks of the low-rank adapters among a tile's rows, behind K's: a chunk
// holds a.pack adapters side by side (a power of two; their ranks padded to
// 8 / pack vectors), or one adapter takes `per` chunks.
struct AdapterChunks {
  int number, found, per;
  __device__ AdapterChunks() : number(0), found(0), per(1) {}
  template <int DT>
  __device__ __forceinline__ void set(const RowsArgs &a, int distinct) {
    found = distinct;
    per = a.pack > 1 ? 1 : (a.rank * Elem<DT>::size + kRow - 1) / kRow;
    number = (found + a.pack - 1) / a.pack * per;
  }
  // Vector v of chunk c: which of the tile's adapters, and the byte of its rank.
  __device__ __forceinline__ void place(const RowsArgs &a, int c, int v, int &which,
                                        int &at) const {
    const int wide = 8 / a.pack;
    which = c / per * a.pack + v / wide;
    at = c % per * kRow + v % wide * 16;
  }
};

// Bytes [at, at + 16) of row ch of an adapter's second matrix b [n][rank], zeros
// past the rank and past n, to LDS; adapter -1: zeros.  Where b's rows start on
// 16 bytes they go there by themselves (pack > 1: all of b below 2 GiB), to
// lds + 16 lane.
template <int DT>
__device__ __forceinline__ void rank_vector(const RowsArgs &a, int adapter, int ch, int at,
                                            uint32_t lds) {
  const int bytes = a.rank * Elem<DT>::size;
  const bool in = adapter >= 0 && ch < a.n && at < bytes;
  if (a.pack > 1) {
    const u32x4 br = descriptor(a.b, (int64_t)a.adapters * a.n * bytes);
    ring_load(br, lds, in ? (uint32_t)(adapter * a.n + ch) * (uint32_t)bytes + at : kOut, 0);
  } else {   // (the adapter is alike in every lane)
    const int id = __builtin_amdgcn_readfirstlane(adapter < 0 ? 0 : adapter);
    const u32x4 br = descriptor(reinterpret_cast<const char *>(a.b) + (int64_t)id * a.n * bytes,
                                (int64_t)a.n * bytes);
    ring_load(br, lds, in ? (uint32_t)ch * (uint32_t)bytes + at : kOut, 0);
  }
}
// Others pass through registers, element by element: their own waits then
// cover every load before them, and nothing but adapters' chunks comes behind.
template <int DT>
__device__ __forceinline__ void rank_elements(const RowsArgs &a, int adapter, int ch, int at,
                                              char *to) {
  using raw = typename Elem<DT>::raw;
  constexpr int S = Elem<DT>::size;
  const int bytes = a.rank * S;
  const bool in = adapter >= 0 && ch < a.n && at < bytes;
  const raw *row = reinterpret_cast<const raw *>(a.b) + ((int64_t)adapter * a.n + ch) * a.rank;
  raw v[16 / S];
#pragma unroll
  for (int e = 0; e < 16 / S; ++e) v[e] = in && at + e * S < bytes ? row[at / S + e] : (raw)0;
  __builtin_memcpy(__builtin_assume_aligned(to + 16 * (threadIdx.x & 63), 16), v, 16);
}

// Output (row, ch) of an adapted FC before bias and activation, by itself.  In an
// adapter's chunk the rows of other adapters meet its matrix with zeros, and
// zero times an infinity or NaN in that matrix is NaN: a NaN in a tile with
// adapters is worked out again from what the row itself names.
template <int DT>
__device__ __forceinline__ float own_output(const RowsArgs &a, int64_t row, int ch) {
  using E = Elem<DT>;
  using raw = typename E::raw;
  constexpr int V = 16 / E::size;
  float s = 0.f;
  const int id = a.ids[row];
  if ((uint32_t)id < (uint32_t)a.adapters) {
    const raw *h = reinterpret_cast<const raw *>(a.h) + row * a.ldh;
    const raw *b = reinterpret_cast<const raw *>(a.b) + ((int64_t)id * a.n + ch) * a.rank;
#pragma nounroll
    for (int r = 0; r < a.rank; ++r) s = fmaf(E::to_f32(h[r]), E::to_f32(b[r]), s);
  }
  const raw *x = reinterpret_cast<const raw *>(a.x) + row * a.ldx;
  const raw *w = reinterpret_cast<const raw *>(a.w) + (int64_t)ch * a.k;
#pragma nounroll
  for (int k = 0; k < a.k && s == s; k += V) {   // (k % V == 0; a NaN stays)
    float xv[V], wv[V];
    load_elems<DT, V>(x, k, xv);
    load_elems<DT, V>(w, k, wv);
#pragma unroll
    for (int e = 0; e < V; ++e) s = fmaf(xv[e], wv[e], s);
  }
  return s;
}

// Inclusive prefix sum over the wave.
__device__ __forceinline__ int wave_prefix(int v) {
#define SPAROA_DPP_ADD(ctrl, rows) \
  v += __builtin_amdgcn_update_dpp(0, v, ctrl, rows, 0xF, false)
  SPAROA_DPP_ADD(0x111, 0xF);
  SPAROA_DPP_ADD(0x112, 0xF);
  SPAROA_DPP_ADD(0x114, 0xF);
  SPAROA_DPP_ADD(0x118, 0xF);
  SPAROA_DPP_ADD(0x142, 0xA);
  SPAROA_DPP_ADD(0x143, 0xC);
#undef SPAROA_DPP_ADD
  return v;
}

struct Tile {
  int seg, col;       // segment; column tile
  int64_t row0, end;  // rows [row0, min(row0 + BM, end)); end 0: no tile
};

// The tile of work-group b where every work-group has one: XCD b % 8 has the
// b % 8-th run of the tiles that there are (their number follows from the
// plan), column tiles innermost.  Each wave finds it by itself.
template <RowsMode MODE, int BM>
__device__ __forceinline__ Tile find_tile(const RowsArgs &a, int cols) {
  const int lane = threadIdx.x & 63, b = blockIdx.x;
  Tile t{0, 0, 0, 0};
  int total = 0;
  if constexpr (MODE <= kRowsDown) {
    for (int e0 = 0; e0 < a.experts; e0 += 64) {
      const int e = min(e0 + lane, a.experts - 1);
      const int n = e0 + lane < a.experts ? a.plan[e + 1] - a.plan[e] : 0;
      total += __builtin_amdgcn_readlane(wave_prefix((n + BM - 1) / BM), 63);
    }
  } else {
    total = (int)((a.rows + BM - 1) / BM);
  }
  const int64_t tiles = (int64_t)total * cols, per = (tiles + 7) / 8;
  const int64_t id = (b & 7) * per + (b >> 3);
  if ((b >> 3) >= per || id >= tiles) return t;
  int rt = (int)(id / cols);
  t.col = (int)(id - (int64_t)rt * cols);
  if constexpr (MODE <= kRowsDown) {
    for (int e0 = 0; e0 < a.experts; e0 += 64) {
      const int e = min(e0 + lane, a.experts - 1);
      const int at = a.plan[e], end = a.plan[e + 1];
      const int n = e0 + lane < a.experts ? (end - at + BM - 1) / BM : 0;
      const int upto = wave_prefix(n);
      const uint64_t past = __ballot(upto > rt);
      if (past) {
        const int l = __builtin_ctzll(past);
        t.seg = e0 + l;
        const int first = __builtin_amdgcn_readlane(upto - n, l);
        t.row0 = __builtin_amdgcn_readlane(at, l) + (int64_t)(rt - first) * BM;
        t.end = __builtin_amdgcn_readlane(end, l);
        return t;
      }
      rt -= __builtin_amdgcn_readlane(upto, 63);
    }
  } else {
    t.row0 = (int64_t)rt * BM;
    t.end = a.rows;
  }
  return t;
}

// The walk of work-groups that take several tiles: the same runs, of which an
// XCD's work-groups take every gridDim.x / 8-th tile.
template <RowsMode MODE, int BM>
struct TileWalk {
  static constexpr bool kExperts = MODE <= kRowsDown;
  const RowsArgs &a;
  const int32_t *cum;   // LDS: row tiles of the experts up to each
  int cols, total;
  int64_t at, end;      // this work-group's next tile, and its XCD's end

  // One wave fills the table; a barrier, then start().
  static __device__ __forceinline__ void fill(const RowsArgs &a, int32_t *cum) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int e0 = 0; e0 < a.experts; e0 += 64) {
      const int e = e0 + lane;
      const int n = e < a.experts ? a.plan[e + 1] - a.plan[e] : 0;
      const int upto = before + wave_prefix((n + BM - 1) / BM);
      if (e < a.experts) cum[e] = upto;
      before = __builtin_amdgcn_readlane(upto, 63);
    }
  }
  __device__ __forceinline__ void start(int column_tiles) {
    cols = column_tiles;
    total = kExperts ? __builtin_amdgcn_readfirstlane(cum[a.experts - 1])
                     : (int)((a.rows + BM - 1) / BM);
    const int64_t tiles = (int64_t)total * cols, per = (tiles + 7) / 8;
    const int xcd = blockIdx.x & 7;
    at = xcd * per + (blockIdx.x >> 3);
    end = std::min<int64_t>((xcd + 1) * per, tiles);
  }
  __device__ __forceinline__ Tile next() {
    Tile t{0, 0, 0, 0};
    if (at >= end) return t;
    const int64_t id = at;
    at += gridDim.x >> 3;
    if constexpr (kExperts) {
      const int rt = (int)(id / cols), lane = threadIdx.x & 63;
      t.col = (int)(id - (int64_t)rt * cols);
      for (int e0 = 0; e0 < a.experts; e0 += 64) {
        const int upto = cum[min(e0 + lane, a.experts - 1)];
        const uint64_t past = __ballot(upto > rt);
        if (!past) continue;
        t.seg = e0 + __builtin_ctzll(past);
        const int first = t.seg ? __builtin_amdgcn_readfirstlane(cum[t.seg - 1]) : 0;
        t.row0 = uniform_word(a.plan + t.seg) + (int64_t)(rt - first) * BM;
        t.end = uniform_word(a.plan + t.seg + 1);
        break;
      }
    } else {
      // column groups outermost: an XCD keeps to a part of the weights
      const int per_group = (cols + a.col_groups - 1) / a.col_groups;
      const int group = (int)(id / ((int64_t)total * per_group));
      const int64_t in = id - (int64_t)group * total * per_group;
      const int wide = min(per_group, cols - group * per_group);
      t.row0 = in / wide * BM;
      t.col = group * per_group + (int)(in % wide);
      t.end = a.rows;
    }
    return t;
  }
};

}  // namespace sparoa

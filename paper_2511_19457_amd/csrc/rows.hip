// Row products: the kernel and tile of a product, the adapters' first product
// of few rows, and the weighted sum of the experts' outputs.
#include <algorithm>

#include "rows.h"

namespace sparoa {
namespace {

// h[row][r] = scale_a a_a[r] x[row]: a wave per row and r (few rows, where
// their adapters differ).
template <int DT, bool VEC>
__global__ __launch_bounds__(256) void shrink_rows_kernel(RowsArgs a) {
  using E = Elem<DT>;
  using raw = typename E::raw;
  const int64_t row = blockIdx.y;
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int id = a.ids[row];
  // (whole waves; columns past the rank, to ldy, are written as zeros)
  if (r >= a.ldy || (uint32_t)id >= (uint32_t)a.adapters) return;
  const raw *x = reinterpret_cast<const raw *>(a.x) + row * a.ldx;
  const raw *w = reinterpret_cast<const raw *>(a.w) + id * a.w_stride + (int64_t)r * a.k;
  constexpr int V = VEC ? 16 / E::size : 1, U = VEC ? 8 : 4;   // pieces in flight
  float s = 0.f;
  for (int k0 = lane * V; k0 < (r < a.n ? a.k : 0); k0 += 64 * V * U) {
    float xv[U][V], wv[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u) {   // (past K: the row's first piece, not added)
      const int k = k0 + 64 * V * u < a.k ? k0 + 64 * V * u : 0;
      load_elems<DT, V>(x, k, xv[u]);
      load_elems<DT, V>(w, k, wv[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (k0 + 64 * V * u < a.k)
#pragma unroll
        for (int e = 0; e < V; ++e) s = fmaf(xv[u][e], wv[u][e], s);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  if (lane) return;
  s *= a.scale[id];
  if (a.h_f32) reinterpret_cast<float *>(a.y)[row * a.ldy + r] = s;
  else reinterpret_cast<raw *>(a.y)[row * a.ldy + r] = E::from_f32(s);
}

// The weighted sum of a token's slots: a lane has V channels of a token.  Bound
// by HBM: 32768 slots of 2048 in fp32 57 us (302 MB, 5.3 TB/s).
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
        const int64_t from = (p[j] < 0 ? 0 : p[j]) * a.ldz + c;
        if constexpr (V == 8) {
          f32x4 q[2];
#pragma unroll
          for (int h = 0; h < 2; ++h)
            q[h] = *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(a.z) + from +
                                                    4 * h);
#pragma unroll
          for (int e = 0; e < V; ++e) z[j][e] = q[e / 4][e % 4];
        } else {
          load_elems<SPAROA_F32, V>(a.z, from, z[j]);
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

// The same of scaled products: a lane has 8 channels, the last of a row fewer.  28
// us (168 MB, 6.0 TB/s).
template <int DT>
__global__ __launch_bounds__(256) void combine_scaled_kernel(CombineArgs a) {
  using E = Elem<DT>;
  using raw = typename E::raw;
  const int64_t per = a.ldz / 8, total = a.tokens * per;
  const u32x4 *zs = reinterpret_cast<const u32x4 *>(a.z);
  const bool whole = a.hidden % 8 == 0;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
    const int64_t t = i / per, v = i - t * per;
    float s[8] = {};
    for (int j0 = 0; j0 < a.top_k; j0 += 8) {   // eight rows in flight
      int p[8];
      float w[8];
      u32x4 z[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int64_t slot = t * a.top_k + (j0 + j < a.top_k ? j0 + j : 0);
        p[j] = j0 + j < a.top_k ? a.place[slot] : -1;
        w[j] = a.weights[slot];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] = zs[(p[j] < 0 ? 0 : p[j]) * per + v];
#pragma unroll
      for (int j = 0; j < 8; ++j) {   // no expert: neither weight nor row is looked at
        float x[8];
        unpack_scaled8(z[j], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = p[j] < 0 ? s[e] : fmaf(w[j], x[e], s[e]);
      }
    }
    const int64_t at = t * a.hidden + 8 * v;
    if (whole) {
      if (a.residual) {
        float r[8];
        load_elems<DT, 8>(a.residual, at, r);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += r[e];
      }
      store_elems<DT, 8>(a.y, at, s);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (8 * v + e < a.hidden) {
          if (a.residual) s[e] += E::to_f32(reinterpret_cast<const raw *>(a.residual)[at + e]);
          reinterpret_cast<raw *>(a.y)[at + e] = E::from_f32(s[e]);
        }
    }
  }
}

template <int DT>
void launch_combine_dt(const CombineArgs &a, hipStream_t stream) {
  constexpr int V = 16 / Elem<DT>::size;
  const bool vec = a.hidden % V == 0;
  const int64_t items = a.tokens * (vec ? a.hidden / V : a.hidden);
  const unsigned grid = (unsigned)std::min<int64_t>(cdiv(items, 256), 1 << 20);
  if constexpr (DT == SPAROA_BF16)
    if (a.z_scaled) {
      const unsigned groups =
          (unsigned)std::min<int64_t>(cdiv(a.tokens * (a.ldz / 8), 256), 1 << 20);
      return combine_scaled_kernel<DT><<<groups, 256, 0, stream>>>(a);
    }
  if (vec) combine_kernel<DT, V><<<grid, 256, 0, stream>>>(a);
  else combine_kernel<DT, 1><<<grid, 256, 0, stream>>>(a);
}

// A work-group has `per_group` rows, a thread 8 elements of a row at a time.
template <int DT>
__global__ __launch_bounds__(256) void pad_rows_kernel(const void *from, void *to, int64_t rows,
                                                       int k, int pitch, int per_group) {
  using raw = typename Elem<DT>::raw;
  const int64_t row0 = (int64_t)blockIdx.x * per_group;
  const uint32_t vecs = pitch / 8;
  const uint32_t items = (uint32_t)(rows - row0 < per_group ? rows - row0 : per_group) * vecs;
  const raw *src = reinterpret_cast<const raw *>(from) + row0 * k;
  raw *dst = reinterpret_cast<raw *>(to) + row0 * pitch;
  for (uint32_t i = threadIdx.x; i < items; i += 256) {
    const uint32_t row = i / vecs, c = (i - row * vecs) * 8;
    raw v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      v[e] = c + e < (uint32_t)k ? src[(int64_t)row * k + c + e] : (raw)0;
    __builtin_memcpy(__builtin_assume_aligned(dst + (int64_t)row * pitch + c, 16), v, sizeof v);
  }
}

template <int DT>
void launch_shrink_rows(const RowsArgs &a, hipStream_t stream) {
  constexpr int V = 16 / Elem<DT>::size;
  const dim3 grid((unsigned)cdiv(a.ldy, 4), (unsigned)a.rows);
  if (a.k % V == 0) shrink_rows_kernel<DT, true><<<grid, 256, 0, stream>>>(a);
  else shrink_rows_kernel<DT, false><<<grid, 256, 0, stream>>>(a);
}

}  // namespace

// 128 x 256 or 64 x 128 tiles (16-bit), by their rounds over the CUs in 10 ns: one
// large tile a CU takes 0.82 us a chunk of K and `besides` us more, up to two
// small ones 0.35 each and 3.
static RowsTile large_or_small(int64_t large, int64_t small, int64_t chunks, int besides) {
  return cdiv(large, 256) * (82 * chunks + 100 * besides) <=
                 cdiv(small, 256) * 35 * chunks + cdiv(small, 512) * 300
             ? kTile128x256 : kTile64x128;
}

RowsTile rows_tile_for(RowsMode mode, const RowsArgs &a, sparoa_dtype dt) {
  const int v = 16 / (int)elem_size(dt);
  const bool f32 = dt == SPAROA_F32;
  if (a.k % v || a.ldx % v) return kRowsStream;
  const int64_t chunks = cdiv(a.k * elem_size(dt), 128);
  const int64_t wide = (int64_t)a.n * (mode == kRowsUpGated ? 2 : 1);
  if (mode == kRowsFc) {
    // Few tiles: the waves split K, 8 of them (128 KB of rings) where every CU has
    // one tile, 4 where it has more.  bf16 (us): 96 x 4096 x 6144 (t32 576) 28.8
    // with 4 waves, 32.8 with 8, 22.6 in 64 x 64 tiles; 500 x 4096 x 1024 (512)
    // 20.1 / 26.5 / 22.1; 32 x 4096 x 4096 (128) 12.0 / 11.4 / 21.0.  fp32, whose MFMAs take 16
    // times as long: 1125 x 2208 x 424 (504) 27.9 / 31.4 / 49.6, 600 x 2048 x 2048
    // (1216) 63.1 / 70.0 / 73.3, 2048 x 1024 x 1024 (2048) 57.8 / 68.9 / 43.5.
    const int64_t t32 = cdiv(a.rows, 32) * cdiv(wide, 32), t64 = cdiv(a.rows, 64) * cdiv(wide, 64);
    if (t32 <= 256) return kTile32x32x8;
    if (t32 <= (f32 ? 1280 : 512)) return kTile32x32;
    // one 64 x 64 tile a CU: 1000 x 4096 x 1024 23.4 us against 28.9 in 64 x 128
    // (300 x 4096 x 4096, 320 tiles: 34.0 / 29.4); fp32 two (2048 x 1024 x 1024
    // 43.5 / 45.9, 4096 x 1024 x 1024 81.8 / 76.0)
    if (t64 <= (f32 ? 512 : 256)) return kTile64x64;
    if (f32) return kTile64x128;
    // 4068 x 3208 x 2248: 107.6 us in 128 x 256 against 115.1 in 64 x 128, 3000 x
    // 5000 x 1504 79.2 / 109.3, 2048^3 33.5 / 26.9, 600 x 4096 x 4096 51.2 / 37.8.
    return large_or_small(cdiv(a.rows, 128) * cdiv(wide, 256), cdiv(a.rows, 64) * cdiv(wide, 128),
                          chunks, 4);
  }
  // Experts, by their average rows: what the host knows.  (Slots without an expert
  // count as rows, and a popular expert takes the others' tile; the figures are of
  // even loads.)  In us, 16-bit unless it says fp32.  Few: bound
  // by the weights' stream (64 experts of 2048 x 1024 gated, 4 rows each: 142
  // against 156 in 64 x 64 tiles, 20 rows 204 / 177); fp32 products are slow
  // enough for 64 rows (16 experts of 1024 x 1024, 50 rows: 68 / 85, 125 rows
  // 128 / 124).  Then tiles that grow with the rows (64 experts, 50 rows: 209 in
  // 64 x 64 / 203 in 64 x 128; 80 rows 230 in 64 x 128 / 213 in 128 x 256; 16
  // experts of 1024 x 2048, 80 rows: 46 / 59; 81 of 264 x 384 gated, 225 rows,
  // short K: 55 / 61).
  const int64_t used = std::min<int64_t>(a.experts, a.rows), per = a.rows / used;
  if (per <= (f32 ? 64 : 12)) return kTile16x64;
  if (f32) return used * cdiv(per, 64) * cdiv(wide, 128) >= 1024 ? kTile64x128 : kTile64x64;
  if (per < 48) return kTile64x64;
  return large_or_small(used * cdiv(per, 128) * cdiv(wide, 256),
                        used * cdiv(per, 64) * cdiv(wide, 128), chunks, 10);
}

sparoa_status launch_rows(RowsMode mode, const RowsArgs &a, sparoa_dtype dt, hipStream_t stream) {
  if (mode == kRowsShrink) {
    // a wave per row and rank where all that these read is little (they share
    // nothing but the L2), else tiles of 16 rows that read x once
    if (a.rows <= 32768 && a.rows * a.n * a.k * elem_size(dt) <= (int64_t)32 << 20) {
      switch (dt) {
        case SPAROA_F32: launch_shrink_rows<SPAROA_F32>(a, stream); break;
        case SPAROA_F16: launch_shrink_rows<SPAROA_F16>(a, stream); break;
        default: launch_shrink_rows<SPAROA_BF16>(a, stream); break;
      }
      SPAROA_LAUNCH_CHECK("fc_adapted: first product of few rows");
      return SPAROA_OK;
    }
    if (a.h_f32) return launch_rows_stream(mode, a, dt, stream);
    // (a launch has fewer than 2^32 threads: rows in parts of whole tiles, up to 2^31
    // threads each)
    constexpr int64_t kPart = 1 << 24;
    for (int64_t r0 = 0; r0 < a.rows; r0 += kPart) {
      RowsArgs p = a;
      p.rows = std::min(a.rows - r0, kPart);
      p.x = reinterpret_cast<const char *>(a.x) + r0 * a.ldx * elem_size(dt);
      p.ids = a.ids + r0;
      p.y = reinterpret_cast<char *>(a.y) + r0 * a.ldy * elem_size(dt);
      const sparoa_status st = launch_rows_split(mode, kTile16x64, p, dt, stream);
      if (st != SPAROA_OK) return st;
    }
    return SPAROA_OK;
  }
  const RowsTile tile = rows_tile_for(mode, a, dt);
  if (mode == kRowsDownScaled && tile < kTile64x64)
    return fail(SPAROA_ERR_UNSUPPORTED, "row products: scaled outputs of few rows");
  if (tile == kRowsStream) return launch_rows_stream(mode, a, dt, stream);
  return tile >= kTile64x64 ? launch_rows_tile(mode, tile, a, dt, stream)
                            : launch_rows_split(mode, tile, a, dt, stream);
}

sparoa_status launch_pad_rows(const void *from, void *to, int64_t rows, int k, int pitch,
                              sparoa_dtype dt, hipStream_t stream) {
  // (some 256 pieces a work-group, a row at least, and fewer than 2^32 threads)
  const int64_t per = std::max<int64_t>(std::max<int64_t>(1, 256 / (pitch / 8)),
                                        cdiv(rows, 1 << 23));
  const unsigned grid = (unsigned)cdiv(rows, per);
  switch (elem_size(dt)) {
    case 4:
      pad_rows_kernel<SPAROA_F32><<<grid, 256, 0, stream>>>(from, to, rows, k, pitch, (int)per);
      break;
    default:   // (bits, whichever 16-bit type)
      pad_rows_kernel<SPAROA_F16><<<grid, 256, 0, stream>>>(from, to, rows, k, pitch, (int)per);
      break;
  }
  SPAROA_LAUNCH_CHECK("row products: padded rows");
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

// The paged cache's writers: rows appended with the rotation by position on the
// way, and accepted drafts moved into place.  Both move bytes once; calls of few
// rows are bound by their chain of dependent loads (lengths, page, row).
#include <algorithm>

#include "cache.h"
#include "rows_ring.h"

namespace sparoa {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxHalf = 128;   // pairs of a head
constexpr int kLeftOver = 128;

// The request of row t.  n 0: none.
struct RowOf {
  int r;
  KvRequest q;
};

// Of up to 64 requests, by the whole wave: one round trip to memory.
__device__ __forceinline__ RowOf request_of_few(const KvArgs &a, int t) {
  const int lane = threadIdx.x & 63, l = min(lane, a.requests - 1);
  RowOf f{0, {0, 0, 0}};
  const KvRequest mine = kv_request(a, l);
  const uint64_t has = __ballot(lane < a.requests && mine.n && mine.start <= t &&
                                t - mine.start < mine.n);
  if (!has) return f;
  f.r = __builtin_ctzll(has);
  f.q = KvRequest{__builtin_amdgcn_readlane(mine.start, f.r),
                  __builtin_amdgcn_readlane(mine.n, f.r),
                  __builtin_amdgcn_readlane(mine.len, f.r)};
  return f;
}

// Of more, by the whole wave: the last request that starts at t or before (64 ways a step,
// two round trips for 4096 requests).  Starts that decrease, which entries that break
// their bounds bring about, may lead it past the row's.
__device__ __forceinline__ RowOf request_of_many(const KvArgs &a, int t) {
  const int lane = threadIdx.x & 63;
  RowOf f{0, {0, 0, 0}};
  int at = 0, left = a.requests;
  while (left > 1) {
    const int step = (left + 63) / 64, probe = at + lane * step;
    const uint64_t below = __ballot(lane * step < left && a.q_start[min(probe, a.requests)] <= t);
    const int last = below ? 63 - __builtin_clzll(below) : 0;
    at += last * step;
    left = min(step, left - last * step);
  }
  f.r = __builtin_amdgcn_readfirstlane(at);
  f.q = kv_request(a, f.r);
  if (t < f.q.start || t - f.q.start >= f.q.n) f.q.n = 0;
  return f;
}

// Of any number, whatever the others' entries, by the whole work-group: the first that
// holds t.
__device__ __forceinline__ RowOf request_of_all(const KvArgs &a, int t) {
  __shared__ int first;
  if (threadIdx.x == 0) first = a.requests;
  __syncthreads();
  for (int r = threadIdx.x; r < a.requests; r += kThreads)
    if (a.q_start[r] <= t && t < a.q_start[r + 1] && kv_request(a, r).n) atomicMin(&first, r);
  __syncthreads();
  RowOf f{first, {0, 0, 0}};
  __syncthreads();   // (read, before another row's)
  if (f.r < a.requests) f.q = kv_request(a, f.r);
  return f;
}
// Whether no start decreases: what request_of_many does not find is not there.
__device__ __forceinline__ bool starts_rise(const KvArgs &a) {
  bool falls = false;
#pragma unroll 8
  for (int r = threadIdx.x; r < a.requests; r += kThreads)
    falls |= a.q_start[r + 1] < a.q_start[r];
  return !__syncthreads_or(falls);
}

template <int DT, int V, bool ALIGNED>
__device__ __forceinline__ void read(const void *p, int64_t at, float (&v)[V]) {
  if constexpr (ALIGNED) {
    load_elems<DT, V>(p, at, v);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      v[e] = Elem<DT>::to_f32(reinterpret_cast<const typename Elem<DT>::raw *>(p)[at + e]);
  }
}
template <int DT, int V, bool ALIGNED>
__device__ __forceinline__ void write(void *p, int64_t at, const float (&v)[V]) {
  if constexpr (ALIGNED) {
    store_elems<DT, V>(p, at, v);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      reinterpret_cast<typename Elem<DT>::raw *>(p)[at + e] = Elem<DT>::from_f32(v[e]);
  }
}

// A work-group a row (token): its heads' pieces of V elements.  Rotated pieces come in
// pairs half a rotation apart (PAIRS), or hold their pairs side by side.  Bound by memory:
// 7660 rows of 32 + 2 x 8 heads of 128, bf16, 44 us (4.3 TB/s); one row 3 us.
// With MANY (above 64 requests) kLeftOver work-groups in front look whether a start
// decreases, and only then for the rows that the search missed: 300 rows of 300 requests
// take 4.8 us (4.7 without), with a start that decreases 7; rows that each looked for
// themselves made padding cost its scan (8000 rows 9.5 -> 12 us).
template <int DT, int V, bool PAIRS, bool ALIGNED, bool MANY>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a, KvDiv by_units,
                                                          int units) {
  __shared__ float2 turn[kMaxHalf];
  const int half = a.rot / 2, dim = a.kv.dim, tid = threadIdx.x;
  const int turned = PAIRS ? half / V : 0;   // units of a head that are pairs
  const int heads = a.q ? a.kv.heads : 0;
  const int rotated = (heads + a.kv.kv_heads) * units;
  const int total = rotated + a.kv.kv_heads * (dim / V);
  const bool left_over = MANY && blockIdx.x < kLeftOver;
  if (left_over && starts_rise(a.kv)) return;
  const int first_row = MANY && !left_over ? blockIdx.x - kLeftOver : blockIdx.x;
  const int row_step = !MANY ? gridDim.x : left_over ? kLeftOver : gridDim.x - kLeftOver;
  for (int64_t at_row = first_row; at_row < a.kv.tokens; at_row += row_step) {
    const int t = (int)at_row;
    RowOf row = MANY ? request_of_many(a.kv, t) : request_of_few(a.kv, t);
    if (left_over) {
      if (row.q.n) continue;   // (alike in every wave)
      row = request_of_all(a.kv, t);
    }
    if (!row.q.n) continue;
    const int at = row.q.len - row.q.n + (t - row.q.start);
    if (tid < half) {
      // p freqs[i] in turns, reduced in fp64: far positions keep their angle
      const double p = a.positions ? a.positions[t] : at;
      double s = p * a.freqs[tid] * 0.15915494309189533577;
      s -= rint(s);
      float c, n;
      sincospif(2.f * (float)s, &n, &c);
      turn[tid] = make_float2(c, n);
    }
    const int in = kv_quotient(at, a.kv.by_page);
    const int page = a.kv.table[(int64_t)row.r * a.kv.table_pages + in];
    const bool there = (uint32_t)page < (uint32_t)a.kv.pages;
    __syncthreads();
    for (int u = tid; u < total; u += kThreads) {
      const bool value = u >= rotated;
      int head, e;
      if (value) {
        head = (u - rotated) / (dim / V);
        e = (u - rotated) - head * (dim / V);
      } else {
        head = kv_quotient(u, by_units);
        e = u - head * units;
      }
      const bool query = !value && head < heads;
      if (!value && !query) head -= heads;
      if (!query && !there) continue;
      const void *from = value ? a.v : query ? a.q : a.k;
      const int64_t stride = value ? a.v_stride : query ? a.q_stride : a.k_stride;
      const int64_t src = t * stride + (int64_t)head * dim;
      void *to = value ? a.v_cache : query ? a.q_out : a.k_cache;
      const int64_t dst =
          query ? ((int64_t)t * a.kv.heads + head) * dim
                : (((int64_t)page * a.kv.kv_heads + head) * a.kv.page_size +
                   (at - in * a.kv.page_size)) * dim;
      float x[V];
      if (PAIRS && !value && e < turned) {
        float y[V], z[V];
        read<DT, V, ALIGNED>(from, src + e * V, x);
        read<DT, V, ALIGNED>(from, src + half + e * V, y);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float2 w = turn[e * V + i];
          z[i] = x[i] * w.x - y[i] * w.y;
          y[i] = x[i] * w.y + y[i] * w.x;
        }
        write<DT, V, ALIGNED>(to, dst + e * V, z);
        write<DT, V, ALIGNED>(to, dst + half + e * V, y);
        continue;
      }
      const int d = PAIRS && !value ? a.rot + (e - turned) * V : e * V;
      read<DT, V, ALIGNED>(from, src + d, x);
      if constexpr (!PAIRS) {
        if (!value && d < a.rot)
#pragma unroll
          for (int i = 0; i + 1 < V; i += 2) {
            const float2 w = turn[(d + i) / 2];
            const float b = x[i];
            x[i] = b * w.x - x[i + 1] * w.y;
            x[i + 1] = b * w.y + x[i + 1] * w.x;
          }
      }
      write<DT, V, ALIGNED>(to, dst + d, x);
    }
    __syncthreads();
  }
}

template <int DT, bool MANY>
void append(const AppendArgs &a, hipStream_t stream) {
  constexpr int V = 16 / Elem<DT>::size;
  const unsigned grid = (unsigned)std::min(a.kv.tokens, 1 << 20) + (MANY ? kLeftOver : 0);
  const int dim = a.kv.dim;
  bool whole = a.k_stride % V == 0 && a.v_stride % V == 0 && (!a.q || a.q_stride % V == 0);
  auto run = [&](auto kernel, int units) {
    kernel<<<grid, kThreads, 0, stream>>>(a, kv_div(units), units);
  };
  if (a.interleaved) {
    whole = whole && a.rot % V == 0;
    if (whole)
      run(append_kernel<DT, V, false, true, MANY>, dim / V);
    else
      run(append_kernel<DT, 2, false, false, MANY>, dim / 2);
    return;
  }
  whole = whole && a.rot % (2 * V) == 0;
  if (whole)
    run(append_kernel<DT, V, true, true, MANY>, a.rot / 2 / V + (dim - a.rot) / V);
  else
    run(append_kernel<DT, 1, true, false, MANY>, a.rot / 2 + (dim - a.rot));
}
template <int DT>
void append(const AppendArgs &a, hipStream_t stream) {
  if (a.kv.requests > 64)
    append<DT, true>(a, stream);
  else
    append<DT, false>(a, stream);
}

// Accepted drafts of one (request, kv head) in the keys or values of `per` layers:
// the list of moves is made once for all of them.  All that a batch of vectors moves
// is in registers before any of it is written; a batch is a slice of columns, which
// no other batch touches.  64 requests, 8 heads, 16 layers, 5 moves: 8.7 us (4.3 TB/s).
__global__ __launch_bounds__(kThreads) void keep_kernel(KeepArgs a, int layers, int per,
                                                        int vectors) {
  constexpr int kHeld = 8;   // vectors a thread holds
  __shared__ int from[256], to[256];
  __shared__ int moves;
  char *cache = reinterpret_cast<char *>(blockIdx.z ? a.v_cache : a.k_cache);
  const int tid = threadIdx.x, layer0 = blockIdx.y * per, layer1 = min(layer0 + per, layers);
  const int64_t items = (int64_t)a.kv.requests * a.kv.kv_heads;
  for (int64_t i = blockIdx.x; i < items; i += gridDim.x) {
    const int r = (int)(i / a.kv.kv_heads), h = (int)(i - (int64_t)r * a.kv.kv_heads);
    const KvRequest q = kv_request(a.kv, r);
    const int kept = a.kept[r];
    if (!q.n || kept <= 0 || kept > a.most || kept > q.n) continue;   // (alike in all threads)
    if (tid == 0) moves = 0;
    __syncthreads();
    if (tid < kept) {
      const int n = a.keep[(int64_t)r * a.most + tid], base = q.len - q.n;
      if (n >= 0 && n < q.n && n != tid) {
        const int s = kv_row(a.kv, r, h, base + n), d = kv_row(a.kv, r, h, base + tid);
        if (s >= 0 && d >= 0) {
          const int at = atomicAdd(&moves, 1);   // (their order does not matter)
          from[at] = s, to[at] = d;
        }
      }
    }
    __syncthreads();
    const int n = moves, all = (layer1 - layer0) * vectors;   // columns of every layer, in a row
    const int cols = n ? min(all, kHeld * kThreads / n) : 0;
    for (int c0 = 0; c0 < all && cols; c0 += cols) {
      const int wide = min(cols, all - c0);
      u32x4 held[kHeld];
      int64_t dst[kHeld];
#pragma unroll
      for (int u = 0; u < kHeld; ++u) {
        const int e = tid + u * kThreads, j = e / wide, c = c0 + (e - j * wide);
        dst[u] = -1;
        if (j < n) {
          const int layer = c / vectors;
          const int64_t at = (layer0 + layer) * a.layer_bytes + 16 * (int64_t)(c - layer * vectors);
          held[u] = *reinterpret_cast<const u32x4 *>(cache + at + (int64_t)from[j] * vectors * 16);
          dst[u] = at + (int64_t)to[j] * vectors * 16;
        }
      }
      __builtin_amdgcn_s_waitcnt(vm_outstanding(0));   // every load has its value
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kHeld; ++u)
        if (dst[u] >= 0) *reinterpret_cast<u32x4 *>(cache + dst[u]) = held[u];
    }
    __syncthreads();
  }
}

}  // namespace

sparoa_status launch_kv_append(const AppendArgs &a, sparoa_dtype dt, hipStream_t stream) {
  switch (dt) {
    case SPAROA_F32: append<SPAROA_F32>(a, stream); break;
    case SPAROA_F16: append<SPAROA_F16>(a, stream); break;
    default: append<SPAROA_BF16>(a, stream); break;
  }
  SPAROA_LAUNCH_CHECK("kv_append");
  return SPAROA_OK;
}

sparoa_status launch_kv_keep(const KeepArgs &a, int64_t layers, sparoa_dtype dt,
                             hipStream_t stream) {
  const int64_t items = (int64_t)a.kv.requests * a.kv.kv_heads;
  // (the layers that fill a work-group's registers share its list: 64 requests of 8
  // heads, 16 layers, 6 drafts: 41 us with a work-group a layer)
  const int vectors = a.kv.dim * (int)elem_size(dt) / 16;
  const int per = (int)std::min<int64_t>(layers, std::max(1, 2048 / (a.most * vectors)));
  const dim3 grid((unsigned)std::min<int64_t>(items, 1 << 20), (unsigned)cdiv(layers, per), 2);
  keep_kernel<<<grid, kThreads, 0, stream>>>(a, (int)layers, per, vectors);
  SPAROA_LAUNCH_CHECK("kv_keep");
  return SPAROA_OK;
}

}  // namespace sparoa

// The norm between two blocks: r' = c r + gate * post(y), n = pre(r').
//
// One pass over memory: a row's elements stay in registers (fp32) from their
// load to both stores, so y and r are read once and r' and n written once.
// Sums run over lanes by cross-lane adds and, where a row takes several
// waves, once more through LDS; the layer norm's variance is taken from the
// registers around the mean (no E[v^2] - mean^2).
// Bound by HBM, 4 cols sizeof(dtype) bytes a row, up to 8192 columns: 8192 x 4096
// bf16 5.0 TB/s, 4096 x 8192 3.9, in fp32 5.0.  Longer rows are not: what a thread
// holds of them does not fit its registers (launch_dt).
#include <algorithm>

#include "block.h"
#include "dtype.h"

namespace sparoa {
namespace {

// Work-groups of 1024 threads that walk the rows of a long input (of 256: four
// times as many): two a CU.
constexpr int64_t kWalkers = 512;

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// Sum over the TPR threads of a row; red: one float per wave of the
// work-group, two halves used in turn so that one barrier per sum is enough.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float (*red)[16], int &turn) {
  v = wave_sum(v);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) red[turn][wave] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) v += red[turn][i];
    turn ^= 1;
  }
  return v;
}

// A row in registers: TPR threads, VPT pieces of V elements each: vectors of 16
// bytes, or single elements where cols is no multiple of a vector.  TPR = 64: a wave per row, four rows a work-group.  A
// work-group walks rows.  KEEP (where the registers allow it): the next row's y
// and r are sent for before the current one is summed, and the weights, biases
// and a gate that all rows share stay in registers from the first row on.
// 8192 x 4096 bf16: 53.6 us (5.0 TB/s); a work-group a row, its weights read
// again and behind the sums, 75.
template <int DT, int V, int TPR, int VPT, bool KEEP>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_rows_kernel(NormArgs a) {
  using E = Elem<DT>;
  using raw = typename E::raw;
  constexpr int RPW = TPR >= 256 ? 1 : 256 / TPR;   // rows per work-group
  __shared__ float red[2][16];
  const int t = TPR >= 256 ? threadIdx.x : threadIdx.x % TPR;
  const int cols = (int)a.cols, nv = cols / V;
  int turn = 0;
  const float inv = 1.f / (float)cols;

  struct alignas(V * E::size) Q {
    raw e[V];
  };
  auto load = [&](Q (&d)[VPT], const void *p, int64_t at) __attribute__((always_inline)) {
    const raw *src = reinterpret_cast<const raw *>(p) + at;
#pragma unroll
    for (int u = 0; u < VPT; ++u)   // (lanes past the row read its last vector, unused)
      d[u] = *reinterpret_cast<const Q *>(src + min(t + u * TPR, nv - 1) * V);
  };
  const int64_t step = (int64_t)gridDim.x * RPW;
  int64_t row = (int64_t)blockIdx.x * RPW + (TPR >= 256 ? 0 : threadIdx.x / TPR);
  if (row >= a.rows) return;   // (whole waves, and RPW > 1 has no barrier)
  Q yq[VPT], rq[VPT], ny[VPT], nr[VPT];
  Q post_w[VPT], post_b[VPT], gate[VPT], pre_w[VPT], pre_b[VPT];   // (KEEP)
  const bool post = a.y && a.post != SPAROA_NORM_NONE, pre = a.pre != SPAROA_NORM_NONE;
  const bool one_gate = a.gate && a.gate_rows >= a.rows;
  if (a.y) load(yq, a.y, row * a.cols);
  if (a.r) load(rq, a.r, row * a.cols);
  if constexpr (KEEP) {
    if (post && a.post_w) load(post_w, a.post_w, 0);
    if (post && a.post_b) load(post_b, a.post_b, 0);
    if (one_gate) load(gate, a.gate, 0);
    if (pre && a.pre_w) load(pre_w, a.pre_w, 0);
    if (pre && a.pre_b) load(pre_b, a.pre_b, 0);
  }
  for (;;) {
    const int64_t base = row * a.cols, next = row + step;
    if (KEEP && next < a.rows) {
      if (a.y) load(ny, a.y, next * a.cols);
      if (a.r) load(nr, a.r, next * a.cols);
    }
    if (KEEP && a.gate && !one_gate) load(gate, a.gate, row / a.gate_rows * a.cols);

    float v[VPT][V];
#pragma unroll
    for (int u = 0; u < VPT; ++u) {
      const bool in = t + u * TPR < nv;
#pragma unroll
      for (int e = 0; e < V; ++e) v[u][e] = (a.y && in) ? E::to_f32(yq[u].e[e]) : 0.f;
    }
    // v <- norm(v) * weight + bias
    auto normalise = [&](int kind, const void *wp, const void *bp, Q (&w)[VPT], Q (&b)[VPT])
                         __attribute__((always_inline)) {
      if constexpr (!KEEP) {
        if (wp) load(w, wp, 0);
        if (bp) load(b, bp, 0);
      }
      if (kind == SPAROA_NORM_LAYER) {
        float s = 0.f;
#pragma unroll
        for (int u = 0; u < VPT; ++u)
#pragma unroll
          for (int e = 0; e < V; ++e) s += v[u][e];
        const float mean = row_sum<TPR>(s, red, turn) * inv;
#pragma unroll
        for (int u = 0; u < VPT; ++u) {
          const bool in = t + u * TPR < nv;
#pragma unroll
          for (int e = 0; e < V; ++e) v[u][e] = in ? v[u][e] - mean : 0.f;
        }
      }
      float s = 0.f;
#pragma unroll
      for (int u = 0; u < VPT; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e) s += v[u][e] * v[u][e];
      const float k = 1.f / sqrtf(row_sum<TPR>(s, red, turn) * inv + a.eps);
#pragma unroll
      for (int u = 0; u < VPT; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          v[u][e] *= k;
          if (wp) v[u][e] *= E::to_f32(w[u].e[e]);
          if (bp) v[u][e] += E::to_f32(b[u].e[e]);
        }
    };
    auto store = [&](void *p) __attribute__((always_inline)) {
      raw *dst = reinterpret_cast<raw *>(p) + base;
#pragma unroll
      for (int u = 0; u < VPT; ++u) {
        Q o;
#pragma unroll
        for (int e = 0; e < V; ++e) o.e[e] = E::from_f32(v[u][e]);
        if (t + u * TPR < nv) *reinterpret_cast<Q *>(dst + (t + u * TPR) * V) = o;
      }
    };

    if (post) normalise(a.post, a.post_w, a.post_b, post_w, post_b);
    if (a.gate) {
      if constexpr (!KEEP) load(gate, a.gate, row / a.gate_rows * a.cols);
#pragma unroll
      for (int u = 0; u < VPT; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e) v[u][e] *= E::to_f32(gate[u].e[e]);
    }
    if (a.r) {
#pragma unroll
      for (int u = 0; u < VPT; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e) v[u][e] = fmaf(a.scale, E::to_f32(rq[u].e[e]), v[u][e]);
    }
    // lanes past the row hold what their clamped loads gave them: cleared
#pragma unroll
    for (int u = 0; u < VPT; ++u) {
      const bool in = t + u * TPR < nv;
#pragma unroll
      for (int e = 0; e < V; ++e) v[u][e] = in ? v[u][e] : 0.f;
    }
    if (a.r_out) store(a.r_out);
    if (pre) {
      normalise(a.pre, a.pre_w, a.pre_b, pre_w, pre_b);
      store(a.n_out);
    }
    if (next >= a.rows) return;
    row = next;
    if constexpr (KEEP) {
#pragma unroll
      for (int u = 0; u < VPT; ++u) yq[u] = ny[u], rq[u] = nr[u];
    } else {
      if (a.y) load(yq, a.y, row * a.cols);
      if (a.r) load(rq, a.r, row * a.cols);
    }
  }
}

// A row in LDS (fp32, cols * 4 bytes), any row length: for rows that are no
// multiple of a vector and too long for single elements in registers.  A thread
// keeps to its own columns, so only the sums need barriers.  1227 x 6811 fp16 36
// us, element by element from memory 81; 2000 x 3001 bf16 36, in registers 27.
constexpr int kLdsThreads = 512, kLdsCols = 16384;   // (64 KB)
template <int DT>
__global__ __launch_bounds__(kLdsThreads) void norm_lds_kernel(NormArgs a) {
  using E = Elem<DT>;
  using raw = typename E::raw;
  extern __shared__ float v[];
  __shared__ float red[2][16];
  int turn = 0;
  const int t = threadIdx.x, cols = (int)a.cols;
  const float inv = 1.f / (float)cols;
  const raw *gate = reinterpret_cast<const raw *>(a.gate);
  // f(column, v[column]) of this thread's columns, several loads in flight
  auto each = [&](auto f) __attribute__((always_inline)) {
#pragma unroll 8
    for (int c = t; c < cols; c += kLdsThreads) v[c] = f(c, v[c]);
  };
  // v <- (v - mean) / deviation, the weights' and biases' part left to the caller
  auto stats = [&](int kind, float &mean, float &k) __attribute__((always_inline)) {
    mean = 0.f;
    if (kind == SPAROA_NORM_LAYER) {
      float s = 0.f;
#pragma unroll 8
      for (int c = t; c < cols; c += kLdsThreads) s += v[c];
      mean = row_sum<kLdsThreads>(s, red, turn) * inv;
    }
    float s = 0.f;
#pragma unroll 8
    for (int c = t; c < cols; c += kLdsThreads) {
      const float d = v[c] - mean;
      s += d * d;
    }
    k = 1.f / sqrtf(row_sum<kLdsThreads>(s, red, turn) * inv + a.eps);
  };
  auto at = [&](const void *p, int64_t i) __attribute__((always_inline)) {
    return E::to_f32(reinterpret_cast<const raw *>(p)[i]);
  };
  const bool post = a.y && a.post != SPAROA_NORM_NONE, pre = a.pre != SPAROA_NORM_NONE;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int64_t base = row * a.cols, g0 = a.gate ? row / a.gate_rows * a.cols : 0;
    if (a.y) each([&](int c, float) { return at(a.y, base + c); });
    else each([&](int, float) { return 0.f; });
    float mean, k;
    if (post) {
      stats(a.post, mean, k);
      each([&](int c, float x) { return (x - mean) * k; });
      if (a.post_w) each([&](int c, float x) { return x * at(a.post_w, c); });
      if (a.post_b) each([&](int c, float x) { return x + at(a.post_b, c); });
    }
    if (a.gate) each([&](int c, float x) { return x * E::to_f32(gate[g0 + c]); });
    if (a.r) each([&](int c, float x) { return fmaf(a.scale, at(a.r, base + c), x); });
    raw *ro = reinterpret_cast<raw *>(a.r_out), *no = reinterpret_cast<raw *>(a.n_out);
    if (ro)
#pragma unroll 8
      for (int c = t; c < cols; c += kLdsThreads) ro[base + c] = E::from_f32(v[c]);
    if (!pre) continue;
    stats(a.pre, mean, k);
    each([&](int c, float x) { return (x - mean) * k; });
    if (a.pre_w) each([&](int c, float x) { return x * at(a.pre_w, c); });
    if (a.pre_b) each([&](int c, float x) { return x + at(a.pre_b, c); });
#pragma unroll 8
    for (int c = t; c < cols; c += kLdsThreads) no[base + c] = E::from_f32(v[c]);
  }
}

// Rows longer than that: element by element, a work-group per row,
// its elements read again for each statistic and computed again for the stores,
// which come last (so outputs may take an input's place).
template <int DT>
__global__ __launch_bounds__(256) void norm_any_kernel(NormArgs a) {
  using E = Elem<DT>;
  using raw = typename E::raw;
  __shared__ float red[2][16];
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int64_t base = row * a.cols;
    const raw *y = a.y ? reinterpret_cast<const raw *>(a.y) + base : nullptr;
    const raw *r = a.r ? reinterpret_cast<const raw *>(a.r) + base : nullptr;
    const raw *g = a.gate ? reinterpret_cast<const raw *>(a.gate) + row / a.gate_rows * a.cols
                          : nullptr;
    const raw *pw = reinterpret_cast<const raw *>(a.post_w);
    const raw *pb = reinterpret_cast<const raw *>(a.post_b);
    const raw *nw = reinterpret_cast<const raw *>(a.pre_w);
    const raw *nb = reinterpret_cast<const raw *>(a.pre_b);
    const float inv = 1.f / (float)a.cols;
    // mean (layer) and 1 / deviation of f(0 .. cols - 1)
    auto stats = [&](int kind, auto f, float &mean, float &k) {
      mean = 0.f;
      if (kind == SPAROA_NORM_LAYER) {
        float s = 0.f;
        for (int64_t c = threadIdx.x; c < a.cols; c += 256) s += f(c);
        mean = row_sum<256>(s, red, turn) * inv;
      }
      float s = 0.f;
      for (int64_t c = threadIdx.x; c < a.cols; c += 256) {
        const float d = f(c) - mean;
        s += d * d;
      }
      k = 1.f / sqrtf(row_sum<256>(s, red, turn) * inv + a.eps);
    };
    const bool post = y && a.post != SPAROA_NORM_NONE;
    float m0 = 0.f, k0 = 1.f, m1 = 0.f, k1 = 1.f;
    if (post) stats(a.post, [&](int64_t c) { return E::to_f32(y[c]); }, m0, k0);
    auto joined = [&](int64_t c) {
      float v = y ? E::to_f32(y[c]) : 0.f;
      if (post) {
        v = (v - m0) * k0;
        if (pw) v *= E::to_f32(pw[c]);
        if (pb) v += E::to_f32(pb[c]);
      }
      if (g) v *= E::to_f32(g[c]);
      return r ? fmaf(a.scale, E::to_f32(r[c]), v) : v;
    };
    const bool pre = a.pre != SPAROA_NORM_NONE;
    if (pre) stats(a.pre, joined, m1, k1);
    raw *ro = a.r_out ? reinterpret_cast<raw *>(a.r_out) + base : nullptr;
    raw *no = reinterpret_cast<raw *>(a.n_out) + base;
    for (int64_t c = threadIdx.x; c < a.cols; c += 256) {
      const float v = joined(c);
      if (ro) ro[c] = E::from_f32(v);
      if (!pre) continue;
      float n = (v - m1) * k1;
      if (nw) n *= E::to_f32(nw[c]);
      if (nb) n += E::to_f32(nb[c]);
      no[c] = E::from_f32(n);
    }
  }
}

template <int DT, int V, int TPR, int VPT, bool KEEP>
void launch_rows(const NormArgs &a, hipStream_t stream) {
  constexpr int RPW = TPR >= 256 ? 1 : 256 / TPR;
  const int64_t groups = cdiv(a.rows, RPW);
  const unsigned grid = (unsigned)std::min<int64_t>(groups, kWalkers * (TPR > 256 ? 1024 / TPR : 4));
  norm_rows_kernel<DT, V, TPR, VPT, KEEP><<<grid, TPR > 256 ? TPR : 256, 0, stream>>>(a);
}

template <int DT>
void launch_dt(const NormArgs &a, hipStream_t stream) {
  constexpr int V = 16 / Elem<DT>::size;
  const bool vec = a.cols % V == 0;
  const int64_t nv = vec ? a.cols / V : a.cols;
  if (nv > (vec ? 4096 : kLdsCols))
    norm_any_kernel<DT><<<(unsigned)std::min<int64_t>(a.rows, 1 << 20), 256, 0, stream>>>(a);
  else if (!vec) {
    if (nv <= 256) launch_rows<DT, 1, 64, 4, true>(a, stream);
    else if (nv <= 1024) launch_rows<DT, 1, 256, 4, true>(a, stream);
    else if (nv <= 4096) launch_rows<DT, 1, 512, 8, false>(a, stream);
    else   // (more in registers spill)
      norm_lds_kernel<DT><<<(unsigned)std::min<int64_t>(a.rows, 1 << 20), kLdsThreads,
                            (unsigned)(4 * nv), stream>>>(a);
  }
  else if (nv <= 64) launch_rows<DT, V, 64, 1, true>(a, stream);
  else if (nv <= 128) launch_rows<DT, V, 64, 2, true>(a, stream);
  else if (nv <= 256) launch_rows<DT, V, 256, 1, true>(a, stream);
  else if (nv <= 512) launch_rows<DT, V, 256, 2, true>(a, stream);
  else if (nv <= 1024) launch_rows<DT, V, 512, 2, true>(a, stream);
  // (spilled registers: 29 of 16-bit types, 2048 x 16384 bf16 95 us, 2.8 TB/s; then 190
  // and more, 1024 x 32768 223 us, 1.2 TB/s; in fp32 none, then 92, 2048 x 16384 190 us)
  else if (nv <= 2048) launch_rows<DT, V, 1024, 2, false>(a, stream);
  else launch_rows<DT, V, 1024, 4, false>(a, stream);
}

}  // namespace

sparoa_status launch_block_norm(const NormArgs &a, sparoa_dtype dt, hipStream_t stream) {
  switch (dt) {
    case SPAROA_F32: launch_dt<SPAROA_F32>(a, stream); break;
    case SPAROA_F16: launch_dt<SPAROA_F16>(a, stream); break;
    default: launch_dt<SPAROA_BF16>(a, stream); break;
  }
  SPAROA_LAUNCH_CHECK("block_norm");
  return SPAROA_OK;
}

}  // namespace sparoa

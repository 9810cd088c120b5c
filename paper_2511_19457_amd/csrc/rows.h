// What the row-product kernels share: MFMA over 16-byte operand pieces,
// activations, epilogue pieces.
#pragma once

#include "block.h"
#include "dtype.h"

namespace sparoa {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t kOut = 0x80000000u;   // an offset past every descriptor's range

// acc += W X^T of a 16 x 16 block over the 4 lanes' pieces of K: lane l holds
// 16 bytes of W's row l & 15 and of X's row l & 15, the same elements of K on
// both sides (a product over K asks for no order of them).  The result's lane
// holds W rows 4 (l >> 4) + i of X row l & 15.
template <int DT>
__device__ __forceinline__ f32x4 mma16(u32x4 w, u32x4 x, f32x4 acc) {
  if constexpr (DT == SPAROA_BF16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w),
                                                   __builtin_bit_cast(bf16x8, x), acc, 0, 0, 0);
  } else if constexpr (DT == SPAROA_F16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, w),
                                                  __builtin_bit_cast(f16x8, x), acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[i]), __uint_as_float(x[i]),
                                                 acc, 0, 0, 0);
    return acc;
  }
}

// relu and relu6 of a NaN are NaN here (apply_act gives 0).
__device__ __forceinline__ float row_act(float v, int act) {
  const float u = apply_act(v, act);
  return v == v ? u : v;
}

template <int DT>
__device__ __forceinline__ float block_act(float v, int act) {
  // (16-bit types: 2^x of a rounded product, off by |v| 2^-24, and a reciprocal are
  // below a rounding of u, in place of expf's and a division's dozens of instructions)
  if (act == SPAROA_ACT_SILU) {
    if constexpr (DT == SPAROA_F32) return v / (1.f + expf(-v));
    return v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -1.44269504088896341f));
  }
  // 1 + erf(v / sqrt 2), which cancels far below 0: by erf a tenth of the result at
  // -5, and 268 us against 282 for 4096 tokens over 16 fp16 experts of 1024 x 4096,
  // top 2
  if (act == SPAROA_ACT_GELU) return 0.5f * v * erfcf(v * -0.70710678118654752f);
  return row_act(v, act);
}

// V consecutive elements from an address aligned to them (V sizeof <= 16).
template <int DT, int V>
__device__ __forceinline__ void load_elems(const void *p, int64_t at, float (&v)[V]) {
  using E = Elem<DT>;
  using raw = typename E::raw;
  raw r[V];
  __builtin_memcpy(r, __builtin_assume_aligned(reinterpret_cast<const raw *>(p) + at,
                                               V * E::size), V * E::size);
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = E::to_f32(r[e]);
}
template <int DT, int V>
__device__ __forceinline__ void store_elems(void *p, int64_t at, const float (&v)[V]) {
  using E = Elem<DT>;
  using raw = typename E::raw;
  raw r[V];
#pragma unroll
  for (int e = 0; e < V; ++e) r[e] = E::from_f32(v[e]);
  __builtin_memcpy(__builtin_assume_aligned(reinterpret_cast<raw *>(p) + at, V * E::size), r,
                   V * E::size);
}

// A word every lane wants alike, by the scalar unit: memory that no kernel of
// this launch writes.
__device__ __forceinline__ int uniform_word(const int32_t *p) {
  return *reinterpret_cast<const __attribute__((address_space(4))) int32_t *>(
      reinterpret_cast<uintptr_t>(p));
}

// Eight elements as one 16-byte vector (16-bit types).
template <int DT>
__device__ __forceinline__ u32x4 pack8(const float (&v)[8]) {
  u32x4 w = {};
  if constexpr (DT != SPAROA_F32) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = Elem<DT>::pack2(v[2 * e], v[2 * e + 1]);
  }
  return w;
}

// Eight numbers in 16 bytes: fp16 multiples of 2^(code - 141), the largest of them
// in [2^14, 2^15], the last bit of each one a bit of the code (so 9 bits behind the
// point, for numbers down to 2^-28 of the largest; one below that is off by 2^-38 of
// the largest at most).  Rounded once: cut to fp16's 10 bits, half of the last bit
// kept added, cut there (a tie goes up, but the 13 bits cut first make ties rare;
// rounded to 10 bits first, every other number would be one and all of them grow by
// 3.5e-4).
// An infinity or NaN stays one by itself: the code is that of the largest finite
// number, so its neighbours keep their bits.
__device__ __forceinline__ u32x4 pack_scaled8(const float (&from)[8]) {
  float v[8];
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    v[e] = from[e];
    m = max(m, __float_as_uint(v[e]) & 0x7FFFFFFFu);
  }
  if (m >= 0x7F000000u) {   // (2^127; seldom)
    m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t b = __float_as_uint(v[e]) & 0x7FFFFFFFu;
      m = b < 0x7F800000u ? max(m, b) : m;
      // a NaN of all ones would not survive the rounding's carry, nor a finite
      // number the one to 2^128: the largest of 9 bits takes its place
      if (b > 0x7F800000u) v[e] = __uint_as_float(0x7FC00000u);
      else if (b > 0x7F7FC000u && b < 0x7F800000u)
        v[e] = copysignf(__uint_as_float(0x7F7FC000u), v[e]);
    }
  }
  const uint32_t code = max(m >> 23, 15u), half = 0x00010001u, spread = code | code << 15;
  const float scale = __uint_as_float((268 - code) << 23);
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t p = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(
                                                        v[2 * i] * scale, v[2 * i + 1] * scale)) +
                       half;
    w[i] = (p & 0xFFFEFFFEu) | (spread >> (2 * i) & 0x00010001u);
  }
  return w;
}
__device__ __forceinline__ void unpack_scaled8(u32x4 w, float (&v)[8]) {
  uint32_t s = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) s |= (w[i] & 0x00010001u) << (2 * i);
  const float scale = __uint_as_float((((s | s >> 15) & 255u) - 14u) << 23);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t h = (e & 1 ? w[e / 2] >> 16 : w[e / 2]) & 0xFFFEu;
    v[e] = Elem<SPAROA_F16>::to_f32((uint16_t)h) * scale;
  }
}

// The distinct values in [0, limit) among id[b] of every lane, in order, to LDS
// list; the whole wave.  Returns their number.
template <int BATCHES>
__device__ __forceinline__ int distinct_values(const int (&id)[BATCHES], int limit,
                                               int32_t *list) {
  const int lane = threadIdx.x & 63;
  uint64_t left[BATCHES];
#pragma unroll
  for (int b = 0; b < BATCHES; ++b) left[b] = __ballot((uint32_t)id[b] < (uint32_t)limit);
  int found = 0;
#pragma unroll
  for (int b = 0; b < BATCHES; ++b)
    while (left[b]) {
      const int a = __builtin_amdgcn_readlane(id[b], __builtin_ctzll(left[b]));
      if (lane == 0) list[found] = a;
      ++found;
#pragma unroll
      for (int c = b; c < BATCHES; ++c) left[c] &= ~__ballot(id[c] == a);
    }
  return found;
}

// The same of ids[0 .. n), n <= 64 BATCHES.
template <int BATCHES>
__device__ __forceinline__ int distinct_ids(const int32_t *ids, int n, int limit, int32_t *list) {
  int id[BATCHES];
#pragma unroll
  for (int b = 0; b < BATCHES; ++b) {
    const int i = 64 * b + (threadIdx.x & 63);
    id[b] = i < n ? ids[i] : -1;
  }
  return distinct_values<BATCHES>(id, limit, list);
}

}  // namespace sparoa

// Fragments of the paged cache for 16 stacked rows at a time, straight from global memory into registers: what the kernels over
// few rows (decoding, drafted tokens, short chunks) and over layouts without a tile kernel share.
//
// Rows are stacked as row = token * R + j, the memory order of [tokens][h * R + j][:]. With l16 = lane % 16, g = lane / 16, the
// matrix products of 16 x 16 results leave lane (l16, g) with column l16 and rows 4 g .. 4 g + 3. Which elements of the
// contraction a lane holds is free as long as both operands agree, so every layout below is the one whose loads are widest:
//   K   a lane holds key l16 of a tile of 16 keys and runs of 16 bytes of its head_dim (the query fragments likewise for rows);
//   V   a lane holds keys 4 g + r and the NE = D / 16 elements NE * l16 .. of each: a load of 16 lanes reads whole rows. As the
//       A operand of O^T += V^T P^T, product e takes d = NE * l16 + e, and P^T comes out of S^T = K Q^T in the lanes that
//       need it: nothing goes through LDS, and no lane exchanges anything;
//   O^T a lane ends up with the 4 NE = D / 4 neighbouring elements 4 NE * g .. of row l16.
// 16-bit elements come 32 keys at a time (two tiles; v_mfma_f32_16x16x32_bf16), f32 ones 16 (v_mfma_f32_16x16x4_f32, exact
// products). 8-bit elements are widened exactly to bf16.
#pragma once
#include "paged.h"

namespace qp {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 pr_bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float pr_f32x4;
typedef unsigned int pr_u32x4 __attribute__((ext_vector_type(4)));

// 8 E4M3 bytes -> 8 bf16 (exact)
__device__ __forceinline__ pr_u32x4 pr_widen8(unsigned lo, unsigned hi) {
  pr_u32x4 o;
  o.x = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false));
  o.y = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true));
  o.z = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false));
  o.w = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true));
  return o;
}

// What rows do not see must not reach them, but 0 times an infinity or NaN is NaN: where a block's V holds such values and not all
// rows see all of it, they leave the product (finite) and come back through sums of the numerators in front of them, which a row
// that does not see them has as 0. plus / minus: 1 where the element is +infinity / -infinity, both for NaN.
struct Split {
  float finite, plus, minus;
};
__device__ __forceinline__ bool pr_not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ Split pr_split(float x) {
  const bool bad = pr_not_finite(x);
  return Split{bad ? 0.f : x, bad && !(x < 0.f) ? 1.f : 0.f, bad && !(x > 0.f) ? 1.f : 0.f};
}
__device__ __forceinline__ void pr_split_pair(unsigned x, unsigned& finite, unsigned& plus, unsigned& minus) {
  const Split lo = pr_split(bf16lo_to_f32(x)), hi = pr_split(bf16hi_to_f32(x));
  finite = (__float_as_uint(lo.finite) >> 16) | __float_as_uint(hi.finite);  // exact: bf16 values
  plus = (__float_as_uint(lo.plus) >> 16) | __float_as_uint(hi.plus);
  minus = (__float_as_uint(lo.minus) >> 16) | __float_as_uint(hi.minus);
}
__device__ __forceinline__ void pr_join(float& sum, float plus, float minus) {
  if (plus > 0.f) sum += INFINITY;
  if (minus > 0.f) sum += -INFINITY;
}

// E: the pool's element: float, bf16_t or uint8_t (E4M3, with bf16 rows).
template <typename E, int D>
struct RowsLayout {
  static constexpr bool F32 = sizeof(E) == 4, F8 = sizeof(E) == 1;
  static constexpr int TILES = F32 ? 1 : 2;          // tiles of 16 keys in a block
  static constexpr int BK = 16 * TILES;              // keys per block
  static constexpr int NE = D / 16;                  // elements of a V row per lane, and products of one V block
  static constexpr int ROWB = D * (int)sizeof(E);    // bytes of a row of the pool
  static constexpr int QB = F32 ? 4 : 2;             // bytes of an element of q and out
  static constexpr int KL = ROWB / 64;               // 16-byte loads of a lane per key tile
  static constexpr int VK = F32 ? 4 : 8;             // keys of a lane's V fragments
  static constexpr int VW = NE * (int)sizeof(E) / 4; // dwords of each
  static constexpr int QF = D * QB / 64;             // 16-byte query fragments of a lane per row tile
};

// A lane's 16 bytes number u of a row, in the contraction's order (bytes from the row's start). Of an 8-bit row one load is two
// steps' elements, so the query's are taken in that order.
template <typename E, int D>
__device__ __forceinline__ int rows_k_byte(int u, int g) { return u * 64 + g * 16; }
template <typename E, int D>
__device__ __forceinline__ int rows_q_byte(int s, int g) {
  if (RowsLayout<E, D>::F8) return 2 * (64 * (s >> 1) + 16 * g + 8 * (s & 1));
  return s * 64 + g * 16;
}

template <typename E, int D>
__device__ __forceinline__ void rows_load_k(const unsigned char* base, int l16, int g, pr_u32x4 (&k)[RowsLayout<E, D>::KL]) {
  const unsigned at = (unsigned)(l16 * RowsLayout<E, D>::ROWB);
#pragma unroll
  for (int u = 0; u < RowsLayout<E, D>::KL; ++u) k[u] = *(const pr_u32x4*)(base + (at + rows_k_byte<E, D>(u, g)));
}

// Products of 16 keys (k) with 16 rows (q); KEYS_ARE_ROWS: result rows are keys and columns query rows (else the other way).
template <typename E, int D, bool KEYS_ARE_ROWS>
__device__ __forceinline__ pr_f32x4 rows_products(const pr_u32x4 (&k)[RowsLayout<E, D>::KL],
                                                  const pr_u32x4 (&q)[RowsLayout<E, D>::QF]) {
  using L = RowsLayout<E, D>;
  pr_f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if constexpr (L::F32) {
#pragma unroll
    for (int u = 0; u < L::KL; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = __uint_as_float(k[u][e]), y = __uint_as_float(q[u][e]);
        s = KEYS_ARE_ROWS ? __builtin_amdgcn_mfma_f32_16x16x4f32(x, y, s, 0, 0, 0)
                          : __builtin_amdgcn_mfma_f32_16x16x4f32(y, x, s, 0, 0, 0);
      }
  } else {
#pragma unroll
    for (int st = 0; st < L::QF; ++st) {
      pr_u32x4 raw;
      if constexpr (L::F8) raw = pr_widen8(k[st >> 1][2 * (st & 1)], k[st >> 1][2 * (st & 1) + 1]);
      else raw = k[st];
      const pr_bf16x8 x = __builtin_bit_cast(pr_bf16x8, raw), y = __builtin_bit_cast(pr_bf16x8, q[st]);
      s = KEYS_ARE_ROWS ? __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, s, 0, 0, 0)
                        : __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, x, s, 0, 0, 0);
    }
  }
  return s;
}

}  // namespace qp

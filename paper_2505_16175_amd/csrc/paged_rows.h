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

// A row's reference (log2 units) before its first visible entry, and its lowest one. c s - m is one multiply-add, so with m rounded from
// a product all numerators of a row carry the same factor, 2 to the power of what that rounding lost: it cancels as long as it is finite. A
// block of nothing but huge negative logits would make it 2^(2^-24 |m|), an infinity that no later reference takes back.
constexpr float PR_NONE = -0x1p29f;
constexpr float PR_LAZY = 8.f;

template <typename E, int D>
struct RowsBlock {
  using L = RowsLayout<E, D>;
  pr_u32x4 k[L::TILES][L::KL];
  unsigned v[L::VK][L::VW];
  int ok;  // bit t: tile t's page is there
};

// Online softmax of a wavefront's RT tiles of 16 stacked rows over blocks of keys.
template <typename E, int D, int RT>
struct RowsWave {
  using L = RowsLayout<E, D>;
  using Block = RowsBlock<E, D>;
  static constexpr int NE = L::NE;
  pr_u32x4 qf[RT][L::QF];
  pr_f32x4 acc[RT][NE];  // O^T: lane (l16, g) has elements 4 NE g + NE r + e of row l16 in acc[.][e][r]
  float m[RT], l[RT];    // reference (log2 units), and this lane's part of the denominator
  int lim[RT];           // last entry that this lane's row sees
  int lim_min;           // and the tile's first row
  int l16, g;

  // rows row0 .. row0 + n_rows - 1 (at most 16 RT) of the sequence's stacked rows of head h
  __device__ __forceinline__ void init(const PagedArgs& a, const PagedSeq& q, const void* queries, int h, int row0, int n_rows) {
    const int lane = threadIdx.x & 63, r_heads = a.h_q / a.h_kv;
    l16 = lane & 15;
    g = lane >> 4;
    lim_min = q.base + row0 / r_heads;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int row = row0 + min(16 * t + l16, n_rows - 1), i = row / r_heads;
      lim[t] = q.base + i;
      const unsigned char* p = (const unsigned char*)queries +
                               ((size_t)(q.row0 + i) * a.h_q + (size_t)h * r_heads + (row - i * r_heads)) * (D * L::QB);
#pragma unroll
      for (int u = 0; u < L::QF; ++u) qf[t][u] = *(const pr_u32x4*)(p + rows_q_byte<E, D>(u, g));
      m[t] = PR_NONE;
      l[t] = 0.f;
#pragma unroll
      for (int e = 0; e < NE; ++e) acc[t][e] = pr_f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }

  // Requests the block of keys from key0 on; page_of(key): the page number of the table, the same in all lanes.
  template <class PageOf>
  __device__ __forceinline__ void load(Block& b, const PagedArgs& a, int h, int key0, int k_end, PageOf page_of) const {
    b.ok = 0;
#pragma unroll
    for (int t = 0; t < L::TILES; ++t) {
      const int key = key0 + 16 * t;
      // a tile past the last entry takes the block's first page: read, never used
      const int page = page_of(key < k_end ? key : key0);
      const bool ok = paged_page_ok(page, a.n_pages);
      b.ok |= ok && key < k_end ? 1 << t : 0;
      const size_t at = paged_row(ok ? page : 0, h, key & ((1 << a.page_shift) - 1), a.h_kv, a.page_shift) * L::ROWB;
      rows_load_k<E, D>((const unsigned char*)a.k + at, l16, g, b.k[t]);
      const unsigned char* vb = (const unsigned char*)a.v + at;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const unsigned off = (unsigned)((4 * g + r) * L::ROWB + l16 * (NE * (int)sizeof(E)));
        if constexpr (L::VW == 2) {
          const uint2 raw = *(const uint2*)(vb + off);
          b.v[4 * t + r][0] = raw.x, b.v[4 * t + r][1] = raw.y;
        } else {
#pragma unroll
          for (int w = 0; w < L::VW; w += 4) {
            const pr_u32x4 raw = *(const pr_u32x4*)(vb + (off + 4 * w));
#pragma unroll
            for (int y = 0; y < 4; ++y) b.v[4 * t + r][w + y] = raw[y];
          }
        }
      }
    }
  }

  __device__ __forceinline__ void compute(Block& b, int key0, int k_end, float c2) {
    if (b.ok == 0) return;
    const bool whole = b.ok == (1 << L::TILES) - 1 && key0 + L::BK <= k_end && key0 + L::BK - 1 <= lim_min;
    if (!whole) {
      // V of entries that are not there may hold anything: 0 times it is not 0
#pragma unroll
      for (int j = 0; j < L::VK; ++j) {
        const bool there = ((b.ok >> (j >> 2)) & 1) && key0 + 16 * (j >> 2) + 4 * g + (j & 3) < k_end;
#pragma unroll
        for (int w = 0; w < L::VW; ++w) b.v[j][w] = there ? b.v[j][w] : 0u;
      }
    }
    float p[RT][L::VK];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
      for (int y = 0; y < L::TILES; ++y) {
        const pr_f32x4 st = rows_products<E, D, true>(b.k[y], qf[t]);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const bool seen = whole || (((b.ok >> y) & 1) && key0 + 16 * y + 4 * g + r <= min(lim[t], k_end - 1));
          p[t][4 * y + r] = seen ? st[r] : -INFINITY;
        }
      }
      float mx = p[t][0];
#pragma unroll
      for (int j = 1; j < L::VK; ++j) mx = fmaxf(mx, p[t][j]);
      mx *= c2;
      if (__any(mx > m[t] + PR_LAZY)) {
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(fmaxf(mx, __shfl_xor(mx, 32, 64)), m[t]);
        const float alpha = __builtin_amdgcn_exp2f(m[t] - mx);
        m[t] = mx;
        l[t] *= alpha;
#pragma unroll
        for (int e = 0; e < NE; ++e)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[t][e][r] *= alpha;
      }
#pragma unroll
      for (int j = 0; j < L::VK; ++j) {
        p[t][j] = __builtin_amdgcn_exp2f(fmaf(p[t][j], c2, -m[t]));
        l[t] += p[t][j];
      }
    }
    const pr_f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    if constexpr (L::F32) {
      bool bad = false;
      if (!whole) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int e = 0; e < NE; ++e) bad = bad || pr_not_finite(__uint_as_float(b.v[r][e]));
      }
      if (__any(bad)) {
#pragma unroll
        for (int e = 0; e < NE; ++e)
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            pr_f32x4 plus = zero, minus = zero;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const Split v = pr_split(__uint_as_float(b.v[r][e]));
              acc[t][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.finite, p[t][r], acc[t][e], 0, 0, 0);
              plus = __builtin_amdgcn_mfma_f32_16x16x4f32(v.plus, p[t][r], plus, 0, 0, 0);
              minus = __builtin_amdgcn_mfma_f32_16x16x4f32(v.minus, p[t][r], minus, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              float z = acc[t][e][r];
              pr_join(z, plus[r], minus[r]);
              acc[t][e][r] = z;
            }
          }
        return;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int e = 0; e < NE; ++e)
#pragma unroll
          for (int t = 0; t < RT; ++t)
            acc[t][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(b.v[r][e]), p[t][r], acc[t][e], 0, 0, 0);
    } else {
      pr_bf16x8 hi[RT], lo[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          hi[t][j] = (__bf16)p[t][j];
          lo[t][j] = (__bf16)(p[t][j] - (float)hi[t][j]);
        }
      auto pair = [&](int j, int y) {  // elements 2 y and 2 y + 1 of key j, as bf16
        if constexpr (L::F8) return (unsigned)__builtin_bit_cast(unsigned, (y & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b.v[j][y >> 1], 1.f, true)
                                                                                  : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b.v[j][y >> 1], 1.f, false));
        else return b.v[j][y];
      };
      bool bad = false;
      if (!whole) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int y = 0; y < NE / 2; ++y) {
            const unsigned w = pair(j, y);
            bad = bad || pr_not_finite(bf16lo_to_f32(w)) || pr_not_finite(bf16hi_to_f32(w));
          }
      }
      const bool guard = __any(bad);
      unsigned w[8];
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        if ((e & 1) == 0) {
#pragma unroll
          for (int j = 0; j < 8; ++j) w[j] = pair(j, e >> 1);
        }
        pr_u32x4 f;  // element e of the lane's 8 keys
#pragma unroll
        for (int y = 0; y < 4; ++y) f[y] = __builtin_amdgcn_perm(w[2 * y + 1], w[2 * y], (e & 1) ? 0x07060302u : 0x05040100u);
        if (guard) {
          pr_u32x4 finite, fp, fm;
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            unsigned x0, x1, x2;
            pr_split_pair(f[y], x0, x1, x2);
            finite[y] = x0, fp[y] = x1, fm[y] = x2;
          }
          f = finite;
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            const pr_f32x4 plus = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pr_bf16x8, fp), hi[t], zero, 0, 0, 0);
            const pr_f32x4 minus = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pr_bf16x8, fm), hi[t], zero, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              float z = acc[t][e][r];
              pr_join(z, plus[r], minus[r]);
              acc[t][e][r] = z;
            }
          }
        }
        const pr_bf16x8 vf = __builtin_bit_cast(pr_bf16x8, f);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          acc[t][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, hi[t], acc[t][e], 0, 0, 0);
          acc[t][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, lo[t], acc[t][e], 0, 0, 0);
        }
      }
    }
  }

  __device__ __forceinline__ float denominator(int t) const {
    float z = l[t] + __shfl_xor(l[t], 16, 64);
    return z + __shfl_xor(z, 32, 64);
  }
};

}  // namespace qp

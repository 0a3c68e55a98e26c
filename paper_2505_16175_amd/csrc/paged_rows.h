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

#include <type_traits>

namespace qp {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 pr_bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float pr_f32x4;
typedef unsigned int pr_u32x4 __attribute__((ext_vector_type(4)));

// 8 E4M3 bytes, times a power of two, -> 8 bf16 (exact)
__device__ __forceinline__ pr_u32x4 pr_widen8(unsigned lo, unsigned hi, float scale = 1.f) {
  pr_u32x4 o;
  o.x = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false));
  o.y = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true));
  o.z = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false));
  o.w = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true));
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

// E: the pool's element: float, bf16_t, uint8_t (E4M3, with bf16 rows) or ScaledCode (the same with scales). A tile of 16 keys is one
// block of those, so its scales are two numbers, which the widening takes along.
struct ScaledCode {
  uint8_t code;
};
template <typename E, int D>
struct RowsLayout {
  static constexpr bool F32 = sizeof(E) == 4, F8 = sizeof(E) == 1, SCALED = std::is_same_v<E, ScaledCode>;
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

// Products of 16 keys (k, codes times scale) with 16 rows (q): result rows are query rows, columns keys. The scale goes into the widening: codes' own
// products with a query may exceed f32 where the keys' do not.
template <typename E, int D>
__device__ __forceinline__ pr_f32x4 rows_products(const pr_u32x4 (&k)[RowsLayout<E, D>::KL], const pr_u32x4 (&q)[RowsLayout<E, D>::QF], float scale) {
  using L = RowsLayout<E, D>;
  pr_f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if constexpr (L::F32) {
#pragma unroll
    for (int u = 0; u < L::KL; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(q[u][e]), __uint_as_float(k[u][e]), s, 0, 0, 0);
  } else {
#pragma unroll
    for (int st = 0; st < L::QF; ++st) {
      pr_u32x4 raw;
      if constexpr (L::F8) raw = pr_widen8(k[st >> 1][2 * (st & 1)], k[st >> 1][2 * (st & 1) + 1], scale);
      else raw = k[st];
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pr_bf16x8, q[st]), __builtin_bit_cast(pr_bf16x8, raw), s, 0, 0, 0);
    }
  }
  return s;
}

// S^T of a block's tiles of keys with RT tiles of rows.
template <typename E, int D, int RT, class Block>
__device__ __forceinline__ void rows_scores(const Block& b, const pr_u32x4 (&q)[RT][RowsLayout<E, D>::QF],
                                            pr_f32x4 (&s)[RT][RowsLayout<E, D>::TILES]) {
  using L = RowsLayout<E, D>;
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int y = 0; y < L::TILES; ++y) s[t][y] = pr_f32x4{0.f, 0.f, 0.f, 0.f};
  if constexpr (L::F32) {
#pragma unroll
    for (int u = 0; u < L::KL; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int t = 0; t < RT; ++t)
          s[t][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(b.k[0][u][e]), __uint_as_float(q[t][u][e]), s[t][0], 0, 0, 0);
  } else {
#pragma unroll
    for (int st = 0; st < L::QF; ++st)
#pragma unroll
      for (int y = 0; y < L::TILES; ++y) {
        pr_u32x4 raw;
        if constexpr (L::F8) raw = pr_widen8(b.k[y][st >> 1][2 * (st & 1)], b.k[y][st >> 1][2 * (st & 1) + 1], b.key_scale(y));
        else raw = b.k[y][st];
#pragma unroll
        for (int t = 0; t < RT; ++t)
          s[t][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pr_bf16x8, raw), __builtin_bit_cast(pr_bf16x8, q[t][st]), s[t][y], 0, 0, 0);
      }
  }
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
  float scales;  // SCALED: lanes 0 and 1 (of every four) have those of the tiles' keys, 2 and 3 of their values
  int ok;        // bit t: tile t's page is there
  __device__ __forceinline__ float key_scale(int tile) const { return L::SCALED ? scale_of(tile, tile) : 1.f; }
  __device__ __forceinline__ float value_scale(int tile) const { return L::SCALED ? scale_of(tile, 2 + tile) : 1.f; }
  // Of a tile without entries any bits may be there, and 0 times a NaN is not 0.
  __device__ __forceinline__ float scale_of(int tile, int lane) const {
    const unsigned bits = (unsigned)__builtin_amdgcn_readlane(__float_as_uint(scales), lane);
    return __uint_as_float((ok >> tile) & 1 ? bits : 0x3f800000u);
  }
};

// Online softmax of a wavefront's RT tiles of 16 stacked rows over blocks of keys. WIN: rows see a window and the first entries.
template <typename E, int D, int RT, bool WIN = false>
struct RowsWave {
  using L = RowsLayout<E, D>;
  using Block = RowsBlock<E, D>;
  static constexpr int NE = L::NE;
  pr_u32x4 qf[RT][L::QF];
  pr_f32x4 acc[RT][NE];  // O^T: lane (l16, g) has elements 4 NE g + NE r + e of row l16 in acc[.][e][r]
  float m[RT], l[RT];    // reference (log2 units), and this lane's part of the denominator
  int lim[RT];           // last entry that this lane's row sees
  int lim_min;           // and the tile's first row
  int lim_max;           // and its last, WIN only
  int l16, g;

  // rows row0 .. row0 + n_rows - 1 (at most 16 RT) of the sequence's stacked rows of head h
  __device__ __forceinline__ void init(const PagedArgs& a, const PagedSeq& q, const void* queries, int h, int row0, int n_rows) {
    const int lane = threadIdx.x & 63, r_heads = a.h_q / a.h_kv;
    l16 = lane & 15;
    g = lane >> 4;
    lim_min = q.base + row0 / r_heads;
    if constexpr (WIN) lim_max = q.base + (row0 + n_rows - 1) / r_heads;
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
    size_t rows[L::TILES];
#pragma unroll
    for (int t = 0; t < L::TILES; ++t) {
      const int key = key0 + 16 * t;
      // a tile past the last entry takes the block's first page: read, never used
      const int page = page_of(key < k_end ? key : key0);
      const bool ok = paged_page_ok(page, a.n_pages);
      b.ok |= ok && key < k_end ? 1 << t : 0;
      const size_t row = paged_row(ok ? page : 0, h, key & ((1 << a.page_shift) - 1), a.h_kv, a.page_shift), at = row * L::ROWB;
      rows[t] = row;
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
    if constexpr (L::SCALED) {
      // One load of them all, in order with the others: as scalar loads, which end in any order, a block's were waited for together with the
      // next one's, just requested (four tokens of 16 sequences of the 72B heads over up to 32,768 entries 163 us).
      const int lane = threadIdx.x & 63;
      b.scales = ((lane & 2) ? a.v_scale : a.k_scale)[((lane & 1) ? rows[L::TILES - 1] : rows[0]) >> 4];
    }
  }

  // Whether some value of the block is an infinity or NaN: an element of which the exponent (of E4M3: everything but the sign) is all ones, to
  // which its least bit is added and makes the next. At the largest scale every code from 256 on stands for an infinity: such blocks, in which
  // hardly anything else is, count as if they had one.
  __device__ __forceinline__ bool values_not_finite(const Block& b) const {
    constexpr unsigned ONES = L::F32 ? 0x7f800000u : L::F8 ? 0x7f7f7f7fu : 0x7f807f80u, LEAST = L::F32 ? 0x00800000u : L::F8 ? 0x01010101u : 0x00800080u;
    unsigned found = 0;
    if constexpr (L::SCALED) {
      const int top = max((int)__float_as_uint(b.value_scale(0)), (int)__float_as_uint(b.value_scale(L::TILES - 1)));
      if (top >= (int)__float_as_uint(0x1p120f)) return true;
    }
#pragma unroll
    for (int j = 0; j < L::VK; ++j)
#pragma unroll
      for (int w = 0; w < L::VW; ++w) found |= (b.v[j][w] & ONES) + LEAST;
    return __any((found & (L::F32 ? 0x80000000u : L::F8 ? 0x80808080u : 0x80008000u)) != 0);
  }

  // Values that are not finite are looked for in blocks that every row sees whole, too: the second bf16 term of a numerator may be 0 or
  // negative, which times an infinity makes NaN of it. Looked for in the result instead, and its keys done again, one token over 46,125
  // entries of the 7B heads took 26.8 us, not 25.8.
  __device__ __forceinline__ void be_careful() { lim_min = -0x7fffffff - 1; }

  __device__ __forceinline__ void compute(Block& b, int key0, int k_end, float c2, int window = 0, int n_sink = 0) {
    if (b.ok == 0) return;
    bool whole = b.ok == (1 << L::TILES) - 1 && key0 + L::BK <= k_end && key0 + L::BK - 1 <= lim_min;
    if constexpr (WIN) whole = whole && (key0 > lim_max - window || key0 + L::BK <= n_sink);
    if (!whole) {
      // V of entries that are not there may hold anything: 0 times it is not 0
#pragma unroll
      for (int j = 0; j < L::VK; ++j) {
        const bool there = ((b.ok >> (j >> 2)) & 1) && key0 + 16 * (j >> 2) + 4 * g + (j & 3) < k_end;
#pragma unroll
        for (int w = 0; w < L::VW; ++w) b.v[j][w] = there ? b.v[j][w] : 0u;
      }
    }
    // The products' chains side by side, and masks behind a branch: an element's is six instructions, of few blocks.
    float p[RT][L::VK];
    {
      pr_f32x4 st[RT][L::TILES];
      rows_scores<E, D, RT>(b, qf, st);
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int j = 0; j < L::VK; ++j) p[t][j] = st[t][j >> 2][j & 3];
    }
    if (!whole) {
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int j = 0; j < L::VK; ++j) {
          const int key = key0 + 16 * (j >> 2) + 4 * g + (j & 3);
          bool seen = ((b.ok >> (j >> 2)) & 1) && key <= min(lim[t], k_end - 1);
          if constexpr (WIN) seen = seen && (key > lim[t] - window || key < n_sink);
          p[t][j] = seen ? p[t][j] : -INFINITY;
        }
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
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
      if (!whole && values_not_finite(b)) {
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
      const bool guard = !whole && values_not_finite(b);
      unsigned w[8];
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        pr_u32x4 f;  // element e of the lane's 8 keys
        if constexpr (L::F8) {  // bytes of two keys are put side by side and then widened, half as many moves as the other way
          if ((e & 1) == 0) {
#pragma unroll
            for (int y = 0; y < 4; ++y) w[y] = __builtin_amdgcn_perm(b.v[2 * y + 1][e >> 2], b.v[2 * y][e >> 2], (e & 2) ? 0x07030602u : 0x05010400u);
          }
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const float scale = b.value_scale(y >> 1);
            f[y] = (e & 1) ? __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[y], scale, true))
                           : __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[y], scale, false));
          }
        } else {
          if ((e & 1) == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = b.v[j][e >> 1];
          }
#pragma unroll
          for (int y = 0; y < 4; ++y) f[y] = __builtin_amdgcn_perm(w[2 * y + 1], w[2 * y], (e & 1) ? 0x07060302u : 0x05040100u);
        }
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

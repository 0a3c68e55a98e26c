// New rows on their way into the paged cache that are not only copied: keys (and the same tokens' queries) turned by their rotary
// angles, and entries of 8-bit pools whose blocks of 16 share a power of two.
//
// A workgroup has a block of 16 entries of a sequence (the entries that share scales, so nobody else writes those) and some of the
// heads; a wavefront takes one head's rows of the block at a time, whole rows by 16 lanes (of bf16 heads of 128) each, and a rotary pair's other element
// comes from the lane half a row away. For a scale the block's largest magnitude is one reduction over the wavefront.
//   Angles: pos * theta^(-2 i / d) in turns in f64, whose fraction is exact enough for f32 at any position that models reach, then an f32
// sine and cosine of at most an eighth of a turn. A frequency is the product of two of 16 numbers that come with the launch. Each angle is taken
// once per block and workgroup, through LDS, and held in registers over the heads.
//   Rotated in f32, rounded once, to what is stored. A rounded key is what qp_qkv_rope leaves except for that one rounding (it stores bf16,
// which an 8-bit pool would round again).
//   Bound by HBM from some thousand rows on, below by the host's call (9.8 us with the caller's slicing; 4 to 6 on the GPU). us: 7,744 tokens of the
// 7B heads with their queries 33.5 (4.3 TB/s); keys and values of 46,125 of the 72B heads out of a projection's rows of 80 heads, with scales 67.7, into
// 8-bit pages without 65.5, bf16 82; out of tensors of their own 65.6, 63.0, 80.0, as fast as qp_paged_append copies them.
//   Before: half rows per load (36.1, 71.0), four heads' rows loaded ahead of the first store (42, 90: half the wavefronts), two heads' in turn (44, 81),
// four blocks of entries per workgroup, one after the other (42, 77), workgroups of 8 blocks (39, 111).
#include "codes.h"
#include "paged.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace qp {

constexpr int PS_WAVES = 4;
constexpr int PS_THREADS = PS_WAVES * 64;
constexpr int PS_BLOCK = PAGED_BLOCK;

// Two values as bf16, nearest, ties to even; NaN stays NaN.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)lo, (__bf16)hi});
}
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// The 16 bytes of the lane D lanes away (lane ^ D).
template <int D>
__device__ __forceinline__ u32x4 from_lane_xor(const u32x4& x) {
  u32x4 o;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    if constexpr (D == 8) o[c] = (unsigned)__builtin_amdgcn_update_dpp(0, (int)x[c], 0x128, 0xf, 0xf, true);  // 16 lanes turned by 8
    else o[c] = (unsigned)__shfl_xor((int)x[c], D, 64);
  }
  return o;
}

// T: float or bf16_t rows. OUT: PS_SAME, PS_FP8 or PS_SCALED. ROPE: keys and queries are turned.
enum { PS_SAME = 0, PS_FP8 = 1, PS_SCALED = 2 };
template <typename T, int D, int OUT, bool ROPE>
__global__ __launch_bounds__(PS_THREADS, D * sizeof(T) > 256 ? 3 : 4) void paged_store_kernel(PagedArgs a, PagedStore src, int blocks_per_seq, int groups) {
  constexpr int EPL = Elem<T>::kPer16B;             // elements of a lane's 16 bytes
  constexpr int HALF = D / 2, LPR = D / EPL;        // lanes per row
  constexpr int TOKENS = 64 / LPR, PASSES = PS_BLOCK / TOKENS;
  constexpr int OUT_BYTES = OUT == PS_SAME ? 16 : EPL;
  // read 16 bytes at a time
  __shared__ __attribute__((aligned(16))) float lds_cos[ROPE ? PS_BLOCK : 1][HALF];
  __shared__ __attribute__((aligned(16))) float lds_sin[ROPE ? PS_BLOCK : 1][HALF];
  static_assert(__alignof__(lds_cos) >= 16 && __alignof__(lds_sin) >= 16 && HALF * sizeof(float) % 16 == 0, "vector reads of the angles");
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int unit = blockIdx.x / groups, group = blockIdx.x - unit * groups;
  const int s = unit / blocks_per_seq;
  const PagedSeq q = paged_seq_of(a, s);
  const int block = unit - s * blocks_per_seq;
  if (q.n == 0 || block > (q.n + PS_BLOCK - 2) / PS_BLOCK) return;
  const int e0 = ((q.base >> 4) + block) * PS_BLOCK;  // the block's first entry; below 0: rows without an entry
  if (e0 >= q.base + q.n) return;
  const int i0 = e0 - q.base;  // the sequence's row number of the block's first entry
  int page = -1;
  if (e0 >= 0 && e0 < q.len) page = a.table[(size_t)s * a.table_pages + (e0 >> a.page_shift)];
  const bool stored = paged_page_ok(page, a.n_pages);
  const int slot0 = e0 & ((1 << a.page_shift) - 1);

  // Heads of keys, then of values, then of queries, dealt to the groups and their wavefronts in runs: side by side the wavefronts of all
  // workgroups read a quarter of each token's heads at a time, which lie in a quarter of the memory's channels.
  const int items = src.q != nullptr ? 2 * a.h_kv + a.h_q : 2 * a.h_kv;
  const int first = (int)((long long)items * group / groups), last = (int)((long long)items * (group + 1) / groups);
  const int end = first + (last - first) * (wave + 1) / PS_WAVES;
  const int sub = lane % LPR, t_lane = lane / LPR;
  struct Rows {
    u32x4 raw[PASSES];
  };
  auto load = [&](Rows& r, int item) {
    if (item >= end) return;
    const bool is_q = item >= 2 * a.h_kv, is_v = !is_q && item >= a.h_kv;
    const int h = is_q ? item - 2 * a.h_kv : is_v ? item - a.h_kv : item;
    const unsigned char* const from = (const unsigned char*)(is_q ? src.q : is_v ? src.v : src.k) + (size_t)h * (is_q ? src.q_head_stride : src.head_stride);
    const size_t stride = is_q ? src.q_token_stride : src.token_stride;
    // rows that are not there repeat one of the block that is
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int i = min(max(i0 + p * TOKENS + t_lane, 0), q.n - 1);
      r.raw[p] = *(const u32x4*)(from + (size_t)(q.row0 + i) * stride + sub * 16);
    }
  };
  Rows r;
  int item = first + (last - first) * wave / PS_WAVES;
  load(r, item);

  if constexpr (ROPE) {
    const int f = tid % HALF;
    const int axis = f < src.s0 ? 0 : (f < src.s0 + src.s1 ? 1 : 2);
    const double turns = src.low[f & 7] * src.high[f >> 3];
#pragma unroll
    for (int t = tid / HALF; t < PS_BLOCK; t += PS_THREADS / HALF) {
      const int i = i0 + t;
      if (i < 0 || i >= q.n) continue;
      const double x = (double)src.axes[axis * src.axis_stride + q.row0 + i] * turns;
      const double quarters = (x - floor(x)) * 4.0, whole = rint(quarters);
      const float z = (float)(quarters - whole), zz = z * z;  // quarters of a turn, at most one half
      // Taylor's series of sine and cosine in quarter turns: the terms left out are below 2^-28
      const float sine = z * fmaf(zz, fmaf(zz, fmaf(zz, fmaf(zz, 1.6044118e-4f, -4.6817541e-3f), 7.9692626e-2f), -6.4596410e-1f), 1.5707963f);
      const float cosine = fmaf(zz, fmaf(zz, fmaf(zz, fmaf(zz, fmaf(zz, -2.5202042e-5f, 9.1926027e-4f), -2.0863480e-2f), 2.5366951e-1f), -1.2337005f), 1.f);
      const int turn = (int)whole & 3;
      const float c = turn & 1 ? sine : cosine, d = turn & 1 ? cosine : sine;
      lds_cos[t][f] = turn == 1 || turn == 2 ? -c : c;
      lds_sin[t][f] = turn >= 2 ? -d : d;
    }
    __syncthreads();
  }

  // full: all 16 entries are new and their page is there. The compiler then sees how many stores follow the next rows' loads, and does not
  // wait for them with those: with a branch around every store it did.
  auto store = [&](const Rows& r, int item, auto full) {
    constexpr bool FULL = decltype(full)::value;
    const bool is_q = item >= 2 * a.h_kv, is_v = !is_q && item >= a.h_kv;
    const int h = is_q ? item - 2 * a.h_kv : is_v ? item - a.h_kv : item;
    float unscale = 1.f, most_code = 448.f;
    const size_t row0 = FULL || stored ? paged_row(page, h, slot0, a.h_kv, a.page_shift) : 0;
    unsigned char* const pool = (unsigned char*)(is_v ? a.v : a.k);
    if constexpr (OUT == PS_SCALED) {
      if (!is_q && (FULL || stored)) {
        // The least e with every finite magnitude <= 448 2^e. Turning makes a key's at most sqrt(2) times as large, and 316 sqrt(2) <
        // 448: taken before it, the scale does not depend on the angles' last bits. Magnitudes of bf16 values are ordered as their bits are.
        u16x2 pairs = {0, 0};
#pragma unroll
        for (int p = 0; p < PASSES; ++p)
#pragma unroll
          for (int c = 0; c < 4; ++c) pairs = __builtin_elementwise_max(pairs, __builtin_bit_cast(u16x2, r.raw[p][c] & 0x7fff7fffu));
        unsigned most = max(pairs.x, pairs.y);
        if (__any(most >= 0x7f80u)) {  // infinities and NaN do not count
          most = 0;
#pragma unroll
          for (int p = 0; p < PASSES; ++p)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const unsigned lo = r.raw[p][c] & 0x7fffu, hi = (r.raw[p][c] >> 16) & 0x7fffu;
              most = max(most, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
            }
        }
        const unsigned bits = __builtin_amdgcn_readfirstlane(__float_as_uint(wave_max(__uint_as_float(most << 16))));
        const unsigned largest = ROPE && !is_v ? 0x1e0000u : 0x600000u;  // mantissas of 316 and 448
        int e = (int)(bits >> 23) - 135 + ((bits & 0x7fffffu) > largest);
        e = max(e, PAGED_SCALE_MIN);
        float* const scale = (is_v ? a.v_scale : a.k_scale) + (row0 >> 4);
        if (!FULL && e0 < q.base) {  // earlier entries of the block: its scale may only grow, and their codes go with it
          const int was = scale_exponent(*scale, PAGED_SCALE_MIN, PAGED_SCALE_MAX);
          e = __builtin_amdgcn_readfirstlane(max(e, was));
          if (e > was) {
            const float shrink = pow2f(max(was - e, -126));
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
              const int t = p * TOKENS + t_lane;
              if (i0 + t >= 0) continue;
              uint2* const at = (uint2*)(pool + (row0 + t) * D + sub * OUT_BYTES);
              uint2 c = *at;
              c.x = shrink4(c.x, shrink), c.y = shrink4(c.y, shrink);
              *at = c;
            }
          }
        }
        e = min(e, PAGED_SCALE_MAX);
        unscale = pow2f(-e);
        if (e == PAGED_SCALE_MAX) most_code = PAGED_SCALE_MAX_CODE;
        if (lane == 0) *scale = pow2f(e);
      }
    }
    const bool turned = ROPE && !is_v;
    const bool second = sub >= LPR / 2;  // the row's second half
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int t = p * TOKENS + t_lane, i = i0 + t;
      u32x4 other;
      if (turned) other = from_lane_xor<LPR / 2>(r.raw[p]);  // all lanes
      if (!FULL && (i < 0 || i >= q.n || (!is_q && (!stored || e0 + t < 0)))) continue;
      float x[EPL];
      widen16<T>(make_uint4(r.raw[p].x, r.raw[p].y, r.raw[p].z, r.raw[p].w), x);
      if constexpr (ROPE) {
        if (turned) {
          float y[EPL];
          widen16<T>(make_uint4(other.x, other.y, other.z, other.w), y);
          const float* const cs = &lds_cos[t][(sub % (LPR / 2)) * EPL];
          const float* const sn = &lds_sin[t][(sub % (LPR / 2)) * EPL];
#pragma unroll
          for (int c = 0; c < EPL; c += 4) {
            const float4 k = *(const float4*)(cs + c), l = *(const float4*)(sn + c);
            const float kk[4] = {k.x, k.y, k.z, k.w}, ll[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
            for (int z = 0; z < 4; ++z)  // as rotate_pair: lo c - (hi s), hi c + (lo s)
              x[c + z] = fmaf(x[c + z], kk[z], __fmul_rn(y[c + z], second ? ll[z] : -ll[z]));
          }
        }
      }
      const size_t row = (size_t)(q.row0 + i);
      if (OUT == PS_SAME || is_q) {
        T* const to = is_q ? (T*)src.q_out + (row * a.h_q + h) * D : (T*)pool + (row0 + t) * D;
        u32x4 o;
        if constexpr (EPL == 4) {
#pragma unroll
          for (int c = 0; c < 4; ++c) o[c] = __float_as_uint(x[c]);
        } else {
#pragma unroll
          for (int c = 0; c < 4; ++c) o[c] = pack_bf16(x[2 * c], x[2 * c + 1]);
        }
        *(u32x4*)(to + sub * EPL) = o;
      } else if constexpr (EPL == 8) {
        *(uint2*)(pool + (row0 + t) * D + sub * OUT_BYTES) =
            make_uint2(codes4(x[0] * unscale, x[1] * unscale, x[2] * unscale, x[3] * unscale, most_code),
                       codes4(x[4] * unscale, x[5] * unscale, x[6] * unscale, x[7] * unscale, most_code));
      }
    }
  };
  const bool full = stored && i0 >= 0 && i0 + PS_BLOCK <= q.n;
  while (item < end) {
    Rows next;
    load(next, item + 1);
    if (full) store(r, item, std::true_type());
    else store(r, item, std::false_type());
    r = next;
    ++item;
  }

  // the entries' positions, and no weight yet: the group's heads of keys
  if (!stored) return;
  for (int z = tid + first * PS_BLOCK; z < min(last, a.h_kv) * PS_BLOCK; z += PS_THREADS) {
    const int t = z % PS_BLOCK, h = z / PS_BLOCK, i = i0 + t;
    if (i < 0 || i >= q.n) continue;
    const size_t row = paged_row(page, h, slot0 + t, a.h_kv, a.page_shift);
    a.pos[row] = src.pos[(size_t)(q.row0 + i) * src.pos_token_stride + (size_t)h * src.pos_head_stride];
    if (a.weight != nullptr) a.weight[row] = 0.f;
  }
}

template <typename T, int D, int OUT, bool ROPE>
static bool store_as(const PagedArgs& a, const PagedStore& src, hipStream_t s) {
  const long long per_seq = ((long long)a.max_new + PS_BLOCK - 2) / PS_BLOCK + 1, blocks = per_seq * a.n_seqs;
  const int items = src.q != nullptr ? 2 * a.h_kv + a.h_q : 2 * a.h_kv;
  // Workgroups that share a block take its angles each, so no more of them than fill the card.
  const long long groups = std::min<long long>((items + PS_WAVES - 1) / PS_WAVES, std::max<long long>(1, 2048 / blocks));
  if (blocks * groups * PS_THREADS > PAGED_MAX_THREADS) return false;
  hipLaunchKernelGGL((paged_store_kernel<T, D, OUT, ROPE>), dim3((unsigned)(blocks * groups)), dim3(PS_THREADS), 0, s, a, src, (int)per_seq, (int)groups);
  return true;
}

bool launch_paged_store(const PagedArgs& a, const PagedStore& from, int dtype, int d, hipStream_t s) {
  PagedStore src = from;
  if (src.axes != nullptr) {
    // theta^(-2 f / d) / (2 pi) = low[f % 8] * high[f / 8]: as f64 powers on the device they took a third of a short launch
    const double step = -2.0 / d * std::log2((double)src.theta);
    for (int i = 0; i < 8; ++i) src.low[i] = std::exp2(i * step), src.high[i] = std::exp2(8 * i * step) * 0.15915494309189533577;
  }
  if (src.axes == nullptr) return store_as<bf16_t, 128, PS_SCALED, false>(a, src, s);  // without angles: pools with scales only
  if (a.fp8 == QP_CACHE_FP8_E4M3_SCALED) return store_as<bf16_t, 128, PS_SCALED, true>(a, src, s);
  if (a.fp8 == QP_CACHE_FP8_E4M3) return store_as<bf16_t, 128, PS_FP8, true>(a, src, s);
  if (dtype == QP_F32) return d == 64 ? store_as<float, 64, PS_SAME, true>(a, src, s) : store_as<float, 128, PS_SAME, true>(a, src, s);
  return d == 64 ? store_as<bf16_t, 64, PS_SAME, true>(a, src, s) : store_as<bf16_t, 128, PS_SAME, true>(a, src, s);
}

}  // namespace qp

// New rows on their way into the paged cache that are not only copied: keys (and the same tokens' queries) turned by their rotary
// angles, and entries of 8-bit pools whose blocks of 16 share a power of two.
//
// A workgroup has a block of 16 entries of a sequence (the entries that share scales, so nobody else writes those) and some of the
// heads; a wavefront takes one head's rows of the block at a time, whole: lane (t, c) has the 16 bytes c of a row's first half and those of
// its second half, so both elements of a rotary pair are its own. For a scale the block's largest magnitude is one reduction over the wavefront.
//   Angles: pos * theta^(-2 i / d) in quarter turns in f64, whose fraction is exact enough for f32 at any position, then one f32
// sine and cosine of at most an eighth of a turn. Each is taken once per block and workgroup, through LDS, and held in registers over the heads.
//   Rotated in f32, rounded once, to what is stored. A rounded key is what qp_qkv_rope leaves except for that one rounding (it stores bf16,
// which an 8-bit pool would round again).
#include "append.h"
#include "paged.h"

#include <algorithm>

namespace qp {

constexpr int PS_WAVES = 4;
constexpr int PS_THREADS = PS_WAVES * 64;
constexpr int PS_BLOCK = PAGED_BLOCK;

// 4 f32 values as E4M3 codes: nearest, ties to even; what is beyond +-448 saturates, NaN stays.
__device__ __forceinline__ unsigned codes4(float a, float b, float c, float d) {
  auto in = [](float x) { return __builtin_elementwise_minimum(__builtin_elementwise_maximum(x, -448.f), 448.f); };
  const unsigned lo = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(in(a), in(b), 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(in(c), in(d), (int)lo, true);
}
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }

// T: float or bf16_t rows. OUT: PS_SAME, PS_FP8 or PS_SCALED. ROPE: keys and queries are turned.
enum { PS_SAME = 0, PS_FP8 = 1, PS_SCALED = 2 };
template <typename T, int D, int OUT, bool ROPE>
__global__ __launch_bounds__(PS_THREADS) void paged_store_kernel(PagedArgs a, PagedStore src, int blocks_per_seq, int groups) {
  constexpr int EPL = Elem<T>::kPer16B;      // elements of a 16-byte piece
  constexpr int HALF = D / 2, LPR = HALF / EPL;  // lanes per row
  constexpr int TOKENS = 64 / LPR, PASSES = PS_BLOCK / TOKENS;
  __shared__ float lds_cos[ROPE ? PS_BLOCK : 1][HALF], lds_sin[ROPE ? PS_BLOCK : 1][HALF];
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

  // heads of keys, then of values, then of queries, dealt to the groups in equal runs
  const int items = src.q != nullptr ? 2 * a.h_kv + a.h_q : 2 * a.h_kv;
  const int per = (items + groups - 1) / groups;
  const int end = min(items, (group + 1) * per);
  const int sub = lane % LPR, t_lane = lane / LPR;
  u32x4 raw[PASSES][2];
  auto load = [&](int item) {
    const bool is_q = item >= 2 * a.h_kv, is_v = !is_q && item >= a.h_kv;
    const int h = is_q ? item - 2 * a.h_kv : is_v ? item - a.h_kv : item;
    const unsigned char* const from = (const unsigned char*)(is_q ? src.q : is_v ? src.v : src.k) + (size_t)h * (is_q ? src.q_head_stride : src.head_stride);
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int i = i0 + p * TOKENS + t_lane;
      raw[p][0] = raw[p][1] = u32x4{0u, 0u, 0u, 0u};
      if (i < 0 || i >= q.n) continue;
      const unsigned char* const at = from + (size_t)(q.row0 + i) * (is_q ? src.q_token_stride : src.token_stride) + sub * 16;
      raw[p][0] = *(const u32x4*)at;
      raw[p][1] = *(const u32x4*)(at + HALF * sizeof(T));
    }
  };
  int item = group * per + wave;
  if (item < end) load(item);

  float cs[ROPE ? PASSES : 1][EPL], sn[ROPE ? PASSES : 1][EPL];
  if constexpr (ROPE) {
    const int f = tid % HALF;
    const int axis = f < src.s0 ? 0 : (f < src.s0 + src.s1 ? 1 : 2);
    const double quarters = exp2(-(double)f / HALF * log2((double)src.theta)) * 0.63661977236758134308;  // 2 / pi
#pragma unroll
    for (int t = tid / HALF; t < PS_BLOCK; t += PS_THREADS / HALF) {
      const int i = i0 + t;
      if (i < 0 || i >= q.n) continue;
      const double x = (double)src.axes[axis * src.axis_stride + q.row0 + i] * quarters, whole = rint(x);
      float sine, cosine;
      sincospif((float)(x - whole) * 0.5f, &sine, &cosine);
      const int turn = (int)(whole - 4.0 * floor(whole * 0.25));
      const float c = turn & 1 ? sine : cosine, d = turn & 1 ? cosine : sine;
      lds_cos[t][f] = turn == 1 || turn == 2 ? -c : c;
      lds_sin[t][f] = turn >= 2 ? -d : d;
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
#pragma unroll
      for (int x = 0; x < EPL; x += 4) {
        const float4 c = *(const float4*)&lds_cos[p * TOKENS + t_lane][sub * EPL + x], d = *(const float4*)&lds_sin[p * TOKENS + t_lane][sub * EPL + x];
        cs[p][x] = c.x, cs[p][x + 1] = c.y, cs[p][x + 2] = c.z, cs[p][x + 3] = c.w;
        sn[p][x] = d.x, sn[p][x + 1] = d.y, sn[p][x + 2] = d.z, sn[p][x + 3] = d.w;
      }
  }

  for (; item < end; item += PS_WAVES) {
    const bool is_q = item >= 2 * a.h_kv, is_v = !is_q && item >= a.h_kv;
    const int h = is_q ? item - 2 * a.h_kv : is_v ? item - a.h_kv : item;
    float x[PASSES][2][EPL];
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
#pragma unroll
      for (int y = 0; y < 2; ++y) widen16<T>(make_uint4(raw[p][y].x, raw[p][y].y, raw[p][y].z, raw[p][y].w), x[p][y]);
    if (item + PS_WAVES < end) load(item + PS_WAVES);

    float unscale = 1.f;
    const size_t row0 = stored ? paged_row(page, h, slot0, a.h_kv, a.page_shift) : 0;
    unsigned char* const pool = (unsigned char*)(is_v ? a.v : a.k);
    if constexpr (OUT == PS_SCALED) {
      if (!is_q && stored) {
        // The least e with every finite magnitude <= 448 2^e. Turning makes a key's at most sqrt(2) times as large, and 316 sqrt(2) <
        // 448: taken before it, the scale does not depend on the angles' last bits.
        float most = 0.f;
#pragma unroll
        for (int p = 0; p < PASSES; ++p)
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int c = 0; c < EPL; ++c) {
              const float size = fabsf(x[p][y][c]);
              most = fmaxf(most, size < INFINITY ? size : 0.f);
            }
        const unsigned bits = __builtin_amdgcn_readfirstlane(__float_as_uint(wave_max(most)));
        const unsigned largest = ROPE && !is_v ? 0x1e0000u : 0x600000u;  // mantissas of 316 and 448
        int e = (int)(bits >> 23) - 135 + ((bits & 0x7fffffu) > largest);
        e = max(e, PAGED_SCALE_MIN);
        float* const scale = (is_v ? a.v_scale : a.k_scale) + (row0 >> 4);
        if (e0 < q.base) {  // earlier entries of the block: its scale may only grow, and their codes go with it
          const int was = min(max((int)((__float_as_uint(*scale) >> 23) & 255u) - 127, PAGED_SCALE_MIN), PAGED_SCALE_MAX);
          e = __builtin_amdgcn_readfirstlane(max(e, was));
          if (e > was) {
            const float shrink = pow2f(max(was - e, -126));
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
              const int t = p * TOKENS + t_lane;
              if (i0 + t >= 0) continue;
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                uint2* const at = (uint2*)(pool + (row0 + t) * D + y * HALF + sub * EPL);
                uint2 c = *at;
                auto smaller = [&](unsigned w) {
                  return codes4(__builtin_amdgcn_cvt_f32_fp8(w, 0) * shrink, __builtin_amdgcn_cvt_f32_fp8(w, 1) * shrink,
                                __builtin_amdgcn_cvt_f32_fp8(w, 2) * shrink, __builtin_amdgcn_cvt_f32_fp8(w, 3) * shrink);
                };
                c.x = smaller(c.x), c.y = smaller(c.y);
                *at = c;
              }
            }
          }
        }
        e = min(e, PAGED_SCALE_MAX);
        unscale = pow2f(-e);
        if (lane == 0) *scale = pow2f(e);
      }
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int t = p * TOKENS + t_lane, i = i0 + t;
      if (i < 0 || i >= q.n) continue;
      if constexpr (ROPE) {
        if (!is_v) {
#pragma unroll
          for (int c = 0; c < EPL; ++c) rotate_pair(x[p][0][c], x[p][1][c], cs[p][c], sn[p][c]);
        }
      }
      const size_t r = (size_t)(q.row0 + i);
      if (!is_q && (!stored || e0 + t < 0)) continue;
      if (OUT == PS_SAME || is_q) {
        T* const to = is_q ? (T*)src.q_out + (r * a.h_q + h) * D : (T*)pool + (row0 + t) * D;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          u32x4 o;
          if constexpr (EPL == 4) {
#pragma unroll
            for (int c = 0; c < 4; ++c) o[c] = __float_as_uint(x[p][y][c]);
          } else {
#pragma unroll
            for (int c = 0; c < 4; ++c) o[c] = (uint32_t)f32_to_bf16_rne(x[p][y][2 * c]) | ((uint32_t)f32_to_bf16_rne(x[p][y][2 * c + 1]) << 16);
          }
          *(u32x4*)(to + y * HALF + sub * EPL) = o;
        }
      } else if constexpr (EPL == 8) {
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          float* const z = x[p][y];
          *(uint2*)(pool + (row0 + t) * D + y * HALF + sub * EPL) =
              make_uint2(codes4(z[0] * unscale, z[1] * unscale, z[2] * unscale, z[3] * unscale), codes4(z[4] * unscale, z[5] * unscale, z[6] * unscale, z[7] * unscale));
        }
      }
      if (!is_q && !is_v && sub == 0) {
        a.pos[row0 + t] = src.pos[r * src.pos_token_stride + (size_t)h * src.pos_head_stride];
        if (a.weight != nullptr) a.weight[row0 + t] = 0.f;
      }
    }
  }
}

template <typename T, int D, int OUT, bool ROPE>
static bool store_as(const PagedArgs& a, const PagedStore& src, hipStream_t s) {
  const long long per_seq = ((long long)a.max_new + PS_BLOCK - 2) / PS_BLOCK + 1, blocks = per_seq * a.n_seqs;
  const int items = src.q != nullptr ? 2 * a.h_kv + a.h_q : 2 * a.h_kv;
  const long long groups = std::min<long long>((items + PS_WAVES - 1) / PS_WAVES, std::max<long long>(1, 2048 / blocks));
  if (blocks * groups * PS_THREADS > PAGED_MAX_THREADS) return false;
  hipLaunchKernelGGL((paged_store_kernel<T, D, OUT, ROPE>), dim3((unsigned)(blocks * groups)), dim3(PS_THREADS), 0, s, a, src, (int)per_seq, (int)groups);
  return true;
}

bool launch_paged_store(const PagedArgs& a, const PagedStore& src, int dtype, int d, hipStream_t s) {
  if (src.axes == nullptr) return store_as<bf16_t, 128, PS_SCALED, false>(a, src, s);  // without angles: pools with scales only
  if (a.fp8 == QP_CACHE_FP8_E4M3_SCALED) return store_as<bf16_t, 128, PS_SCALED, true>(a, src, s);
  if (a.fp8 == QP_CACHE_FP8_E4M3) return store_as<bf16_t, 128, PS_FP8, true>(a, src, s);
  if (dtype == QP_F32) return d == 64 ? store_as<float, 64, PS_SAME, true>(a, src, s) : store_as<float, 128, PS_SAME, true>(a, src, s);
  return d == 64 ? store_as<bf16_t, 64, PS_SAME, true>(a, src, s) : store_as<bf16_t, 128, PS_SAME, true>(a, src, s);
}

}  // namespace qp

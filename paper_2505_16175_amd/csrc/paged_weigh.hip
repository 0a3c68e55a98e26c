// The attention weight that the paged cache's entries received: w[j] (+)= sum over rows of exp2(c q.k_j - lse2), the column sums
// of the softmax whose row statistics qp_paged_attend left.
//
// A wavefront owns 64 entries (32 of f32) of a KV head, whose keys stay in registers, and walks the sequence's rows 16 at a time:
// S = Q K^T leaves a lane with one entry (column) and four rows, so the sum over rows stays in the lane until the end, and no
// two wavefronts meet in an entry: nothing to merge, no atomics. Few rows: bound by the keys' way from HBM, all of which is
// requested at once. Many rows: bound by the vector unit, 24 cycles per 64 pairs (an exponential, a multiply-add, an add)
// beside the products' 16.
#include "paged_rows.h"

#include <algorithm>

namespace qp {

constexpr int PW_NW = 4;
template <typename E>
constexpr int pw_tiles() { return sizeof(E) == 4 ? 2 : 4; }

template <typename E, int D>
__global__ __launch_bounds__(PW_NW * 64) void paged_weigh_kernel(PagedArgs a, const void* __restrict__ qp_, const float* __restrict__ lse,
                                                                int accumulate, int blocks) {
  using L = RowsLayout<E, D>;
  constexpr int KT = pw_tiles<E>();
  const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int x = blockIdx.x;
  const int h = x % a.h_kv;
  x /= a.h_kv;
  const int s = x % a.n_seqs;
  const long long first = ((long long)(x / a.n_seqs) * PW_NW + wave) * (16 * KT);
  const PagedSeq q = paged_seq_of(a, s);
  if (first >= q.len) return;
  const int key0 = (int)first;
  const int r_heads = a.h_q / a.h_kv;
  const int mask = (1 << a.page_shift) - 1;

  pr_u32x4 k[KT][L::KL];
  int page[KT];
#pragma unroll
  for (int t = 0; t < KT; ++t) {
    const int key = key0 + 16 * t;
    page[t] = key < q.len ? __builtin_amdgcn_readfirstlane(a.table[(size_t)s * a.table_pages + (key >> a.page_shift)]) : -1;
    if (!paged_page_ok(page[t], a.n_pages)) page[t] = -1;
    const size_t at = paged_row(max(page[t], 0), h, key & mask, a.h_kv, a.page_shift) * L::ROWB;
    rows_load_k<E, D>((const unsigned char*)a.k + at, l16, g, k[t]);
  }
  float w[KT];
#pragma unroll
  for (int t = 0; t < KT; ++t) w[t] = 0.f;
  const long long all_rows = (long long)q.n * r_heads;
  const float c2 = a.scale_log2;
  const int last = key0 + 16 * KT - 1;
  // rows before the first that sees key0 see none of these entries
  for (long long row0 = (long long)max(0, key0 - q.base) * r_heads / 16 * 16; row0 < all_rows; row0 += 16) {
    const int n = (int)min(all_rows - row0, 16ll);
    pr_u32x4 qf[L::QF];
    {
      const long long row = row0 + min(l16, n - 1);
      const int i = (int)(row / r_heads);
      const unsigned char* p = (const unsigned char*)qp_ +
                               ((size_t)(q.row0 + i) * a.h_q + (size_t)h * r_heads + (size_t)(row - (long long)i * r_heads)) * (D * L::QB);
#pragma unroll
      for (int u = 0; u < L::QF; ++u) qf[u] = *(const pr_u32x4*)(p + rows_q_byte<E, D>(u, g));
    }
    float neg[4];
    int lim[4];  // -1: a row that there is not, or that saw nothing
    bool all = true;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const long long row = row0 + min(4 * g + r, n - 1);
      const int i = (int)(row / r_heads);
      const float z = lse[(size_t)(h * r_heads + (int)(row - (long long)i * r_heads)) * a.n_rows + q.row0 + i];
      neg[r] = -z * 1.4426950408889634f;
      lim[r] = 4 * g + r < n && z != -INFINITY ? q.base + i : -1;
      all = all && lim[r] >= last;
    }
    const bool whole = __all(all);
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      const pr_f32x4 st = rows_products<E, D, false>(k[t], qf);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float p = __builtin_amdgcn_exp2f(fmaf(st[r], c2, neg[r]));
        w[t] += whole || key0 + 16 * t + l16 <= lim[r] ? p : 0.f;
      }
    }
  }
#pragma unroll
  for (int t = 0; t < KT; ++t) {
    w[t] += __shfl_xor(w[t], 16, 64);
    w[t] += __shfl_xor(w[t], 32, 64);
    const int key = key0 + 16 * t + l16;
    if (g == t && page[t] >= 0 && key < q.len) {
      float* const to = a.weight + paged_row(page[t], h, key & mask, a.h_kv, a.page_shift);
      *to = accumulate ? *to + w[t] : w[t];
    }
  }
}

size_t paged_weigh_workspace_bytes(int, int, int, int, int) { return 0; }

template <typename E, int D>
static bool weigh_as(const PagedArgs& a, const void* q, const float* lse, int accumulate, hipStream_t s) {
  constexpr int KEYS = PW_NW * 16 * pw_tiles<E>();
  const long long blocks = ((long long)a.max_len + KEYS - 1) / KEYS, all = blocks * a.n_seqs * a.h_kv;
  if (all * PW_NW * 64 > PAGED_MAX_THREADS) return false;
  hipLaunchKernelGGL((paged_weigh_kernel<E, D>), dim3((unsigned)all), dim3(PW_NW * 64), 0, s, a, q, lse, accumulate, (int)blocks);
  return true;
}

bool launch_paged_weigh(const PagedArgs& a, int dtype, int d, const void* q, const float* lse, int accumulate, void*, size_t,
                        hipStream_t s) {
  if (dtype == QP_F32) return d == 64 ? weigh_as<float, 64>(a, q, lse, accumulate, s) : weigh_as<float, 128>(a, q, lse, accumulate, s);
  if (a.fp8) return weigh_as<uint8_t, 128>(a, q, lse, accumulate, s);
  return d == 64 ? weigh_as<bf16_t, 64>(a, q, lse, accumulate, s) : weigh_as<bf16_t, 128>(a, q, lse, accumulate, s);
}

}  // namespace qp

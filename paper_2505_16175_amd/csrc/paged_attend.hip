// Attention of the paged cache's new tokens: online softmax over a sequence's pages.
//
// paged_rows_kernel: few stacked rows (tokens x query heads of a KV head; decoding, drafted tokens) against a long axis. What
// bounds it is HBM: K and V are read once and nothing is reused, and the products take a tenth of that time. So there is no LDS
// tile and no barrier in its loop: a workgroup takes a chunk of a sequence's entries for one KV head, its four wavefronts take
// blocks of 32 keys (16 of f32) in turn, each straight into registers (paged_rows.h) while the block before it is computed;
// chunks' partial results are merged by a second launch.
//   S^T = K Q^T, P^T = exp2(c S^T - m), O^T += V^T P^T; a lane holds one row and 8 of the block's keys. The reference m of a row
//   moves only when a logit exceeds it by 2^8, so that most blocks exchange nothing between lanes. Numerators are rounded to bf16
//   twice (their value, and what that lost), so that 16-bit results differ from exact ones by their own rounding: the second
//   product is hidden behind the loads. Denominators are summed from the unrounded ones.
#include "paged_rows.h"

#include <algorithm>

namespace qp {

constexpr int PR_NW = 4;               // wavefronts per workgroup
constexpr int PR_LIST = 512;           // page numbers kept in LDS: of a segment of 8192 entries in pages of 16
constexpr int PR_SEGMENT = PR_LIST * 16;
constexpr float PR_NONE = -3e38f;      // a row's reference (log2 units) before its first visible entry
constexpr float PR_LAZY = 8.f;

struct PagedOut {
  const void* q;   // [n_rows][h_q][d]
  void* out;
  float* lse;      // [h_q][n_rows] or nullptr
  float* part_o;   // [chunks][n_rows * h_q][d], chunks > 1
  float* part_lse; // [chunks][n_rows * h_q], log2 units
  int tiles, chunks, chunk_keys;
};

template <typename E, int D>
struct RowsBlock {
  using L = RowsLayout<E, D>;
  pr_u32x4 k[L::TILES][L::KL];
  unsigned v[L::VK][L::VW];
  int ok;  // bit t: tile t's page is there
};

// Two workgroups per compute unit where two blocks' rows fit half of the registers.
template <typename E, int D, int RT>
constexpr int pr_waves() { return D == 64 || (sizeof(E) < 4 && RT == 1) || sizeof(E) == 1 ? 2 : 1; }

template <typename E, int D, int RT>
__global__ __launch_bounds__(PR_NW * 64, (pr_waves<E, D, RT>())) void paged_rows_kernel(PagedArgs a, PagedOut o) {
  using L = RowsLayout<E, D>;
  using Block = RowsBlock<E, D>;
  constexpr int NE = L::NE, ROWS = 16 * RT, LD = D + 4;
  __shared__ int pages[PR_LIST];
  __shared__ float sm_m[PR_NW][ROWS], sm_l[PR_NW][ROWS];
  __shared__ __attribute__((aligned(16))) float slab[PR_NW][ROWS][LD];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // workgroup -> (chunk, sequence, row tile, head): one head's tiles of a chunk meet on few XCDs
  int x = blockIdx.x;
  const int h = x % a.h_kv;
  x /= a.h_kv;
  const int tile = x % o.tiles;
  x /= o.tiles;
  const int s = x % a.n_seqs, chunk = x / a.n_seqs;
  const PagedSeq q = paged_seq_of(a, s);
  const int r_heads = a.h_q / a.h_kv;
  const long long all_rows = (long long)q.n * r_heads;
  const int row0 = tile * ROWS;
  if (row0 >= all_rows) return;
  if (chunk > 0 && (long long)chunk * o.chunk_keys >= q.len) return;  // chunk 0 always answers
  const int n_rows = (int)(all_rows - row0 < ROWS ? all_rows - row0 : ROWS);
  // what the tile's rows see: the first of them least, the last most
  const int lim_min = q.base + row0 / r_heads, lim_max = q.base + (row0 + n_rows - 1) / r_heads;
  const int k_begin = chunk * o.chunk_keys;
  const int k_end = min(min(q.len, lim_max + 1), o.chunk_keys < q.len - k_begin ? k_begin + o.chunk_keys : q.len);

  int lim[RT];  // of this lane's row
  pr_u32x4 qf[RT][L::QF];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int row = row0 + min(16 * t + l16, n_rows - 1), i = row / r_heads;
    lim[t] = q.base + i;
    const unsigned char* p = (const unsigned char*)o.q +
                             ((size_t)(q.row0 + i) * a.h_q + (size_t)h * r_heads + (row - i * r_heads)) * (D * L::QB);
#pragma unroll
    for (int u = 0; u < L::QF; ++u) qf[t][u] = *(const pr_u32x4*)(p + rows_q_byte<E, D>(u, g));
  }
  pr_f32x4 acc[RT][NE];
  float m[RT], l[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    m[t] = PR_NONE;
    l[t] = 0.f;
#pragma unroll
    for (int e = 0; e < NE; ++e) acc[t][e] = pr_f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float c2 = a.scale_log2;
  const int mask = (1 << a.page_shift) - 1;
  int seg = k_begin;  // first entry of the segment whose pages are listed

  auto load = [&](Block& b, int key0) {
    b.ok = 0;
#pragma unroll
    for (int t = 0; t < L::TILES; ++t) {
      const int key = key0 + 16 * t;
      // a tile past the last entry takes the block's first page: read, never used
      const int page = __builtin_amdgcn_readfirstlane(pages[((key < k_end ? key : key0) >> a.page_shift) - (seg >> a.page_shift)]);
      const bool ok = paged_page_ok(page, a.n_pages);
      b.ok |= ok && key < k_end ? 1 << t : 0;
      const size_t at = paged_row(ok ? page : 0, h, key & mask, a.h_kv, a.page_shift) * L::ROWB;
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
  };

  auto compute = [&](Block& b, int key0) {
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
      unsigned w[8][NE / 2];  // V as pairs of bf16
      bool bad = false;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (L::F8) {
          const pr_u32x4 z = pr_widen8(b.v[j][0], b.v[j][1]);
#pragma unroll
          for (int y = 0; y < 4; ++y) w[j][y] = z[y];
        } else {
#pragma unroll
          for (int y = 0; y < NE / 2; ++y) w[j][y] = b.v[j][y];
        }
        if (!whole) {
#pragma unroll
          for (int y = 0; y < NE / 2; ++y)
            bad = bad || pr_not_finite(bf16lo_to_f32(w[j][y])) || pr_not_finite(bf16hi_to_f32(w[j][y]));
        }
      }
      const bool guard = __any(bad);
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        pr_u32x4 f;  // element e of the lane's 8 keys
#pragma unroll
        for (int y = 0; y < 4; ++y)
          f[y] = __builtin_amdgcn_perm(w[2 * y + 1][e >> 1], w[2 * y][e >> 1], (e & 1) ? 0x07060302u : 0x05040100u);
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
  };

  for (; seg < k_end; seg += PR_SEGMENT) {
    const int seg_end = min(k_end, k_end - seg > PR_SEGMENT ? seg + PR_SEGMENT : k_end);
    const int first = seg >> a.page_shift, count = ((seg_end - 1) >> a.page_shift) - first + 1;
    __syncthreads();  // the last segment's list has been read
    for (int i = tid; i < count; i += PR_NW * 64) pages[i] = a.table[(size_t)s * a.table_pages + first + i];
    __syncthreads();
    Block b0, b1;
    int key = seg + wave * L::BK;
    constexpr int STEP = PR_NW * L::BK;
    if (key < seg_end) load(b0, key);
    while (key < seg_end) {
      if (key + STEP < seg_end) load(b1, key + STEP);
      compute(b0, key);
      key += STEP;
      if (key >= seg_end) break;
      if (key + STEP < seg_end) load(b0, key + STEP);
      compute(b1, key);
      key += STEP;
    }
  }

  // the wavefronts' results meet in LDS
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    float z = l[t] + __shfl_xor(l[t], 16, 64);
    z += __shfl_xor(z, 32, 64);
    if (g == 0) {
      sm_m[wave][16 * t + l16] = m[t];
      sm_l[wave][16 * t + l16] = z;
    }
    float* const to = &slab[wave][16 * t + l16][4 * NE * g];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < NE; e += 4)
        *(float4*)(to + NE * r + e) = make_float4(acc[t][e][r], acc[t][e + 1][r], acc[t][e + 2][r], acc[t][e + 3][r]);
  }
  __syncthreads();
  const size_t total = (size_t)a.n_rows * a.h_q;
  for (int z = tid; z < n_rows * (D / 4); z += PR_NW * 64) {
    const int r = z / (D / 4), d = (z - r * (D / 4)) * 4;
    float big = sm_m[0][r];
#pragma unroll
    for (int w = 1; w < PR_NW; ++w) big = fmaxf(big, sm_m[w][r]);
    float den = 0.f;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < PR_NW; ++w) {
      const float wgt = __builtin_amdgcn_exp2f(sm_m[w][r] - big);
      const float4 v = *(const float4*)&slab[w][r][d];
      den = fmaf(wgt, sm_l[w][r], den);
      sum.x = fmaf(wgt, v.x, sum.x);
      sum.y = fmaf(wgt, v.y, sum.y);
      sum.z = fmaf(wgt, v.z, sum.z);
      sum.w = fmaf(wgt, v.w, sum.w);
    }
    const bool none = den == 0.f;
    const float inv = none ? 0.f : 1.f / den;
    if (none) sum = make_float4(0.f, 0.f, 0.f, 0.f);
    sum = make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv);
    const float lse2 = none ? -INFINITY : big + log2f(den);
    const int row = row0 + r, i = row / r_heads, qh = h * r_heads + (row - i * r_heads);
    const size_t at = (size_t)(q.row0 + i) * a.h_q + qh;
    if (o.chunks > 1) {
      const size_t p = (size_t)chunk * total + at;
      *(float4*)(o.part_o + p * D + d) = sum;
      if (d == 0) o.part_lse[p] = lse2;
    } else {
      if constexpr (L::F32) *(float4*)((float*)o.out + at * D + d) = sum;
      else
        *(uint2*)((bf16_t*)o.out + at * D + d) =
            make_uint2((uint32_t)f32_to_bf16_rne(sum.x) | ((uint32_t)f32_to_bf16_rne(sum.y) << 16),
                       (uint32_t)f32_to_bf16_rne(sum.z) | ((uint32_t)f32_to_bf16_rne(sum.w) << 16));
      if (o.lse != nullptr && d == 0) o.lse[(size_t)qh * a.n_rows + q.row0 + i] = lse2 * 0.6931471805599453f;
    }
  }
}

// Merge of the chunks' partial results of a row: out = sum_c 2^(lse_c - lse) O_c. W wavefronts share a row, each with up to 8 chunks'
// loads under way together; their results meet in LDS. One of 181 chunks per row alone took 42 us, a chain of 23 round trips.
constexpr int PM_WAVES = 4;  // rows of a workgroup where a wavefront has a row to itself
template <typename T, int D, int W>
__global__ __launch_bounds__((W == 1 ? PM_WAVES : W) * 64) void paged_merge_kernel(PagedArgs a, PagedOut o) {
  constexpr int PER = D / 64;  // elements of a lane
  constexpr int ROWS = W == 1 ? PM_WAVES : 1;
  __shared__ float red[W][64][PER], red_m[W], red_l[W];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int per_seq = (int)(((long long)a.max_new * a.h_q + ROWS - 1) / ROWS);
  const int s = blockIdx.x / per_seq;
  const PagedSeq q = paged_seq_of(a, s);
  const long long item = (long long)(blockIdx.x - s * per_seq) * ROWS + (W == 1 ? wave : 0);
  const int i = (int)(item / a.h_q), qh = (int)(item - (long long)i * a.h_q);
  if (i >= q.n) return;  // with W > 1: the whole workgroup
  const int n = q.len == 0 ? 1 : (q.len - 1) / o.chunk_keys + 1;  // chunks that answered
  const size_t total = (size_t)a.n_rows * a.h_q, at = (size_t)(q.row0 + i) * a.h_q + qh;
  constexpr int B = 8;
  float m = PR_NONE, den = 0.f, sum[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) sum[e] = 0.f;
  for (int c0 = W == 1 ? 0 : wave * B; c0 < n; c0 += B * W) {
    float ls[B], po[B][PER];
#pragma unroll
    for (int u = 0; u < B; ++u) {
      const size_t p = (size_t)min(c0 + u, n - 1) * total + at;
      ls[u] = o.part_lse[p];
#pragma unroll
      for (int e = 0; e < PER; ++e) po[u][e] = o.part_o[p * D + PER * lane + e];
      if (c0 + u >= n) {  // an infinity of the last chunk, with weight 0, would not be 0
        ls[u] = -INFINITY;
#pragma unroll
        for (int e = 0; e < PER; ++e) po[u][e] = 0.f;
      }
    }
    float mb = m;
#pragma unroll
    for (int u = 0; u < B; ++u) mb = fmaxf(mb, ls[u]);
    const float keep = __builtin_amdgcn_exp2f(m - mb);
    den *= keep;
#pragma unroll
    for (int e = 0; e < PER; ++e) sum[e] *= keep;
#pragma unroll
    for (int u = 0; u < B; ++u) {
      const float w = __builtin_amdgcn_exp2f(ls[u] - mb);
      den += w;
#pragma unroll
      for (int e = 0; e < PER; ++e) sum[e] = fmaf(w, po[u][e], sum[e]);
    }
    m = mb;
  }
  if constexpr (W > 1) {
#pragma unroll
    for (int e = 0; e < PER; ++e) red[wave][lane][e] = sum[e];
    if (lane == 0) {
      red_m[wave] = m;
      red_l[wave] = den;
    }
    __syncthreads();
    if (wave != 0) return;
    m = red_m[0];
#pragma unroll
    for (int w = 1; w < W; ++w) m = fmaxf(m, red_m[w]);
    den = 0.f;
#pragma unroll
    for (int e = 0; e < PER; ++e) sum[e] = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float wgt = __builtin_amdgcn_exp2f(red_m[w] - m);
      den = fmaf(wgt, red_l[w], den);
#pragma unroll
      for (int e = 0; e < PER; ++e) sum[e] = fmaf(wgt, red[w][lane][e], sum[e]);
    }
  }
  const bool none = den == 0.f;
  const float inv = none ? 0.f : 1.f / den;
#pragma unroll
  for (int e = 0; e < PER; ++e) store_elem<T>((T*)o.out + at * D + PER * lane + e, none ? 0.f : sum[e] * inv);
  if (o.lse != nullptr && lane == 0)
    o.lse[(size_t)qh * a.n_rows + q.row0 + i] = none ? -INFINITY : (m + log2f(den)) * 0.6931471805599453f;
}
// Eight wavefronts share a row of more than 16 chunks.
constexpr int PM_SHARE = 8;
static int merge_rows(int chunks) { return chunks > 16 ? 1 : PM_WAVES; }
static long long merge_blocks(const PagedArgs& a, int chunks) {
  const int rows = merge_rows(chunks);
  return (((long long)a.max_new * a.h_q + rows - 1) / rows) * a.n_seqs;
}

PagedPlan plan_paged_attend(const PagedArgs& a, int dtype, int d, size_t scratch_bytes) {
  PagedPlan p{};
  const long long rows = (long long)a.max_new * (a.h_q / a.h_kv);
  const int bk = dtype == QP_F32 ? 16 : 32;
  p.tile_rows = rows <= 16 ? 16 : 32;
  p.tiles = (int)((rows + p.tile_rows - 1) / p.tile_rows);
  const long long units = (long long)a.n_seqs * a.h_kv * p.tiles;
  // About two workgroups per compute unit and twice that for the shorter sequences; at least two blocks per wavefront.
  const long long want = std::max<long long>(1, (4ll * device_cu_count() + units - 1) / units);
  const long long least = 2 * PR_NW * bk;
  long long keys = std::max<long long>(((a.max_len + want - 1) / want + PR_NW * bk - 1) / (PR_NW * bk) * (PR_NW * bk), least);
  const size_t per_chunk = (size_t)a.n_rows * a.h_q * (d + 1) * sizeof(float);
  long long chunks = (a.max_len + keys - 1) / keys;
  const long long fit = (long long)(std::min(scratch_bytes, PAGED_ATTEND_SCRATCH) / per_chunk);
  if (chunks > fit) {
    chunks = fit >= 2 ? fit : 1;
    keys = ((a.max_len + chunks - 1) / chunks + bk - 1) / bk * bk;
    chunks = (a.max_len + keys - 1) / keys;
  }
  p.chunks = (int)std::max<long long>(chunks, 1);
  p.chunk_keys = (int)std::min<long long>(keys, 0x40000000);
  p.workgroups = units * p.chunks;
  p.scratch_bytes = p.chunks > 1 ? per_chunk * p.chunks : 0;
  return p;
}

template <typename E, typename T, int D>
static bool attend_as(const PagedArgs& a, const PagedOut& o, const PagedPlan& p, hipStream_t s) {
  const dim3 grid((unsigned)p.workgroups), block(PR_NW * 64);
  if (p.tile_rows == 16) hipLaunchKernelGGL((paged_rows_kernel<E, D, 1>), grid, block, 0, s, a, o);
  else hipLaunchKernelGGL((paged_rows_kernel<E, D, 2>), grid, block, 0, s, a, o);
  if (p.chunks > 1) {
    const dim3 merge((unsigned)merge_blocks(a, p.chunks));
    if (merge_rows(p.chunks) == 1) hipLaunchKernelGGL((paged_merge_kernel<T, D, PM_SHARE>), merge, dim3(PM_SHARE * 64), 0, s, a, o);
    else hipLaunchKernelGGL((paged_merge_kernel<T, D, 1>), merge, dim3(PM_WAVES * 64), 0, s, a, o);
  }
  return true;
}

bool launch_paged_attend(const PagedArgs& a, int dtype, int d, const void* q, void* out, float* lse, void* scratch,
                         size_t scratch_bytes, hipStream_t s) {
  const PagedPlan p = plan_paged_attend(a, dtype, d, scratch != nullptr ? scratch_bytes : 0);
  if (p.workgroups * PR_NW * 64 > PAGED_MAX_THREADS || merge_blocks(a, p.chunks) * PM_SHARE * 64 > PAGED_MAX_THREADS) return false;
  PagedOut o{};
  o.q = q, o.out = out, o.lse = lse;
  o.tiles = p.tiles, o.chunks = p.chunks, o.chunk_keys = p.chunk_keys;
  o.part_o = (float*)scratch;
  o.part_lse = o.part_o + (size_t)p.chunks * a.n_rows * a.h_q * d;
  if (dtype == QP_F32) return d == 64 ? attend_as<float, float, 64>(a, o, p, s) : attend_as<float, float, 128>(a, o, p, s);
  if (a.fp8) return attend_as<uint8_t, bf16_t, 128>(a, o, p, s);
  return d == 64 ? attend_as<bf16_t, bf16_t, 64>(a, o, p, s) : attend_as<bf16_t, bf16_t, 128>(a, o, p, s);
}

}  // namespace qp

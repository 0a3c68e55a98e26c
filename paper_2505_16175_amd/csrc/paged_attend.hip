// Attention of the paged cache's new tokens: online softmax over a sequence's pages.
//
// Chunks over bf16 heads of 128 (more than 32 stacked rows of a KV head) run the group attention's tile kernel over the pages
// (attend_mfma.hip); their chunks are merged here too.
//
// paged_rows_kernel: few stacked rows (tokens x query heads of a KV head; decoding, drafted tokens) against a long axis, and
// other layouts. What
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

struct PagedOut {
  const void* q;   // [n_rows][h_q][d]
  void* out;
  float* lse;      // [h_q][n_rows] or nullptr
  float* part_o;   // [chunks][n_rows * h_q][d], chunks > 1
  float* part_lse; // [chunks][n_rows * h_q], log2 units
  int tiles, chunks, chunk_keys;
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
  const int lim_max = q.base + (row0 + n_rows - 1) / r_heads;  // the last row sees most
  const int k_begin = chunk * o.chunk_keys;
  const int k_end = min(min(q.len, lim_max + 1), o.chunk_keys < q.len - k_begin ? k_begin + o.chunk_keys : q.len);

  RowsWave<E, D, RT> rows;
  rows.init(a, q, o.q, h, row0, n_rows);
  const float c2 = a.scale_log2;
  int seg = k_begin;  // first entry of the segment whose pages are listed

  auto load = [&](Block& b, int key0) {
    rows.load(b, a, h, key0, k_end,
              [&](int key) { return __builtin_amdgcn_readfirstlane(pages[(key >> a.page_shift) - (seg >> a.page_shift)]); });
  };
  auto compute = [&](Block& b, int key0) { rows.compute(b, key0, k_end, c2); };

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
    const float z = rows.denominator(t);
    if (g == 0) {
      sm_m[wave][16 * t + l16] = rows.m[t];
      sm_l[wave][16 * t + l16] = z;
    }
    float* const to = &slab[wave][16 * t + l16][4 * NE * g];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < NE; e += 4)
        *(float4*)(to + NE * r + e) = make_float4(rows.acc[t][e][r], rows.acc[t][e + 1][r], rows.acc[t][e + 2][r], rows.acc[t][e + 3][r]);
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

// Stacked rows above which bf16 heads of 128 take the tile kernel (attend_mfma.hip), and what its 32-bit arithmetic takes.
constexpr long long PT_FROM_ROWS = 32, PT_MOST_ROWS = 1 << 26;

PagedPlan plan_paged_attend(const PagedArgs& a, int dtype, int d, size_t scratch_bytes) {
  PagedPlan p{};
  const long long rows = (long long)a.max_new * (a.h_q / a.h_kv);
  const bool tiled = dtype == QP_BF16 && d == 128 && rows > PT_FROM_ROWS && rows <= PT_MOST_ROWS;
  const int step = tiled ? 64 : PR_NW * (dtype == QP_F32 ? 16 : 32);  // entries of a chunk are a multiple of it
  p.tile_rows = tiled ? PT_ROWS : rows <= 16 ? 16 : 32;
  p.tiles = (int)((rows + p.tile_rows - 1) / p.tile_rows);
  const long long units = (long long)a.n_seqs * a.h_kv * p.tiles;
  // Rows: one workgroup per compute unit, two over 8-bit pools, of at least two blocks per wavefront. us by workgroups per compute
  // unit 1 / 2 / 4: one token of the 7B heads over 46,125 entries 25.0 / 27.6 / 30.1, of 32 sequences over up to 9,840 84.8 / 89.8 /
  // 93.2; up to four of the 72B heads of 16 sequences over 8-bit pages of up to 32,768 251 / 180 / 187.
  // Tiles, one workgroup per compute unit at a time: four rounds of them, of at least 16 tiles of keys (four questions of up to
  // 300 tokens over up to 46,125 entries, one round 544, two 580, three 555, four 506, six 531).
  const int rounds = tiled ? 4 : a.fp8 ? 2 : 1;
  const long long want = std::max<long long>(1, ((long long)rounds * device_cu_count() + units - 1) / units);
  const long long least = tiled ? 16 * 64 : 2 * step;
  long long keys = std::max<long long>(((a.max_len + want - 1) / want + step - 1) / step * step, least);
  const size_t per_chunk = (size_t)a.n_rows * a.h_q * (d + 1) * sizeof(float);
  long long chunks = (a.max_len + keys - 1) / keys;
  const long long fit = (long long)(std::min(scratch_bytes, PAGED_ATTEND_SCRATCH) / per_chunk);
  if (chunks > fit) {
    chunks = fit >= 2 ? fit : 1;
    keys = ((a.max_len + chunks - 1) / chunks + step - 1) / step * step;
    chunks = (a.max_len + keys - 1) / keys;
  }
  p.chunks = (int)std::max<long long>(chunks, 1);
  p.chunk_keys = (int)std::min<long long>(keys, 0x40000000);
  p.workgroups = tiled ? paged_tile_blocks(a, p) : units * p.chunks;
  p.scratch_bytes = p.chunks > 1 ? per_chunk * p.chunks : 0;
  return p;
}

template <typename E, typename T, int D>
static bool attend_as(const PagedArgs& a, const PagedOut& o, const PagedPlan& p, hipStream_t s) {
  const dim3 grid((unsigned)p.workgroups), block(PR_NW * 64);
  if (p.tile_rows == PT_ROWS) launch_paged_tiles(a, p, o.q, o.out, o.lse, o.part_o, o.part_lse, s);
  else if (p.tile_rows == 16) hipLaunchKernelGGL((paged_rows_kernel<E, D, 1>), grid, block, 0, s, a, o);
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
  if (p.workgroups * (p.tile_rows == PT_ROWS ? 512 : PR_NW * 64) > PAGED_MAX_THREADS || merge_blocks(a, p.chunks) * PM_SHARE * 64 > PAGED_MAX_THREADS) return false;
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

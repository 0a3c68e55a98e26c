// Attention of the paged cache's new tokens: online softmax over a sequence's pages.
//
// Chunks over bf16 heads of 128 (more than 32 stacked rows of a KV head) run the group attention's tile kernel over the pages
// (attend_mfma.hip); their chunks are merged here too.
//
// paged_rows_kernel: few stacked rows (tokens x query heads of a KV head; decoding, drafted tokens) against a long axis, and
// other layouts. What
// bounds it is HBM: K and V are read once and nothing is reused, and the products take a tenth of that time. So there is no LDS
// tile and no barrier in its loop: a workgroup takes an equal share of the batch's entries for one KV head, its four wavefronts take
// blocks of 32 keys (16 of f32) in turn, each straight into registers (paged_rows.h) while the block before it is computed;
// partial results of sequences that shares cut are merged by a second launch.
//   S^T = K Q^T, P^T = exp2(c S^T - m), O^T += V^T P^T; a lane holds one row and 8 of the block's keys. The reference m of a row
//   moves only when a logit exceeds it by 2^8, so that most blocks exchange nothing between lanes. Numerators are rounded to bf16
//   twice (their value, and what that lost), so that 16-bit results differ from exact ones by their own rounding: the second
//   product is hidden behind the loads. Denominators are summed from the unrounded ones.
// What the vector unit does for a block of keys counts as soon as two row tiles meet 8-bit entries: it, not HBM, set the time of four tokens of 16
// sequences over up to 32,768 entries (163 us) until masks were left to the blocks that need them, the products' chains were put side by side, and
// two keys' bytes were paired before they are widened (141 us, a copy's rate).
// Windows: a row tile's workgroups walk the first entries and its tokens' windows as one axis without what lies between (RowsGap), each unit by
// workgroups of its own. us with the batch's blocks dealt evenly, as above / so: four tokens of 16 sequences of the 72B heads, window
// 2,000, 8-bit with scales 46 / 37 (31 now), of 64 112 / 87; one token of 32 of the 7B heads, window 4,096, 63 / 59 (57 now).
#include "paged_rows.h"

#include <algorithm>
#include <cmath>

namespace qp {

constexpr int PR_NW = 4;               // wavefronts per workgroup
constexpr int PR_LIST = 512;           // page numbers kept in LDS: of a segment of 8192 entries in pages of 16
constexpr int PR_SEGMENT = PR_LIST * 16;

struct PagedOut {
  const void* q;   // [n_rows][h_q][d]
  void* out;
  float* lse;      // [h_q][n_rows] or nullptr
  float* part_o;   // partial results: tile kernel [chunks][n_rows * h_q][d]; shares [h_kv][shares + units][rows of a tile][d]
  float* part_lse; // the same without d, log2 units
  int tiles, chunks, chunk_keys;
  int shares;      // workgroups of a KV head among which the batch's blocks are dealt; 0: one for each unit, or the tile kernel
  int per_unit;    // of a window: those of each unit, which share its blocks only
  int tile_rows;
  int span;        // keys in their row tile's own count that a sequence has at most, see RowsGap
  int2* info;      // [units]: first share of a unit and the shares that have blocks of it
};

// Two workgroups per compute unit for heads of 64 and over 8-bit pools, where two row tiles fill the registers (with scales 4 of them spill, 5 in windows, around
// the loop over the keys). Of bf16 heads of 128 one has the registers to itself: squeezed into half of them its results and
// addresses spill around the loop, one token over 46,125 entries 29.4 us, not 26. Of f32 heads of 128 too.
template <typename E, int D>
constexpr int pr_waves() { return D == 64 || sizeof(E) == 1 ? 2 : 1; }

// Where the workgroups' results meet. pages: page numbers; WIN: of every 16 keys, in the row tile's own count.
template <int D, int ROWS>
struct RowsLds {
  int pages[PR_LIST];
  float m[PR_NW][ROWS], l[PR_NW][ROWS];
  __attribute__((aligned(16))) float slab[PR_NW][ROWS][D + 4];
};

// Keys [k_begin, k_end) of one unit, a row tile of sequence s; slot: where its partial result goes, -1: it is the whole, and the output.
// WIN: keys in the unit's own count.
template <typename E, int D, int RT, bool WIN>
__device__ __forceinline__ void rows_unit(const PagedArgs& a, const PagedOut& o, RowsLds<D, 16 * RT>& lds, const PagedSeq& q, int s, int h,
                                          int row0, int n_rows, int k_begin, int k_end, const RowsGap& gap, long long slot) {
  using L = RowsLayout<E, D>;
  using Block = RowsBlock<E, D>;
  constexpr int NE = L::NE, ROWS = 16 * RT;
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r_heads = a.h_q / a.h_kv;
  RowsWave<E, D, RT, WIN> rows;
  rows.init(a, q, o.q, h, row0, n_rows);
  const float c2 = a.scale_log2;
  int seg = k_begin;  // first entry of the segment whose pages are listed

  const int entry_end = WIN ? gap.entry(k_end - 1) + 1 : k_end;
  auto load = [&](Block& b, int key0) {
    if constexpr (WIN) {
      const int entry0 = gap.entry(key0);
      rows.load(b, a, h, entry0, entry_end,
                [&](int entry) { return __builtin_amdgcn_readfirstlane(lds.pages[(key0 - seg + entry - entry0) >> 4]); });
    } else {
      rows.load(b, a, h, key0, k_end,
                [&](int key) { return __builtin_amdgcn_readfirstlane(lds.pages[(key >> a.page_shift) - (seg >> a.page_shift)]); });
    }
  };
  auto compute = [&](Block& b, int key0) {
    if constexpr (WIN) rows.compute(b, gap.entry(key0), entry_end, c2, a.window, a.n_sink);
    else rows.compute(b, key0, k_end, c2);
  };

  for (; seg < k_end; seg += PR_SEGMENT) {
    const int seg_end = min(k_end, k_end - seg > PR_SEGMENT ? seg + PR_SEGMENT : k_end);
    const int first = seg >> a.page_shift, count = WIN ? (seg_end - seg + 15) >> 4 : ((seg_end - 1) >> a.page_shift) - first + 1;
    __syncthreads();  // the last segment's list has been read
    for (int i = tid; i < count; i += PR_NW * 64)
      lds.pages[i] = a.table[(size_t)s * a.table_pages + (WIN ? gap.entry(seg + 16 * i) >> a.page_shift : first + i)];
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
      lds.m[wave][16 * t + l16] = rows.m[t];
      lds.l[wave][16 * t + l16] = z;
    }
    float* const to = &lds.slab[wave][16 * t + l16][4 * NE * g];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < NE; e += 4)
        *(float4*)(to + NE * r + e) = make_float4(rows.acc[t][e][r], rows.acc[t][e + 1][r], rows.acc[t][e + 2][r], rows.acc[t][e + 3][r]);
  }
  __syncthreads();
  for (int z = tid; z < n_rows * (D / 4); z += PR_NW * 64) {
    const int r = z / (D / 4), d = (z - r * (D / 4)) * 4;
    float big = lds.m[0][r];
#pragma unroll
    for (int w = 1; w < PR_NW; ++w) big = fmaxf(big, lds.m[w][r]);
    float den = 0.f;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < PR_NW; ++w) {
      const float wgt = __builtin_amdgcn_exp2f(lds.m[w][r] - big);
      const float4 v = *(const float4*)&lds.slab[w][r][d];
      den = fmaf(wgt, lds.l[w][r], den);
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
    if (slot >= 0) {
      const size_t p = (size_t)slot * ROWS + r;
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

// A unit is a row tile of a sequence that has rows; its blocks are the PR_NW wavefronts' keys up to the last that a row sees.
constexpr int PR_UNITS = 2048;  // units whose blocks a workgroup adds up
template <int RT, bool WIN>
__device__ __forceinline__ int unit_blocks(const PagedArgs& a, const PagedSeq& q, int tile, int step) {
  const int r_heads = a.h_q / a.h_kv;
  const long long all_rows = (long long)q.n * r_heads, row0 = (long long)tile * (16 * RT);
  if (row0 >= all_rows) return 0;
  const int last = (int)((min(row0 + 16 * RT, all_rows) - 1) / r_heads);
  int keys = min(q.len, q.base + last + 1);
  if constexpr (WIN) keys -= rows_gap(a.window, a.n_sink, q.base + (int)(row0 / r_heads), step / PR_NW).gap;
  return max(1, (keys + step - 1) / step);  // one at least: a unit that sees nothing has results too
}

template <typename E, int D, int RT, bool WIN>
__global__ __launch_bounds__(PR_NW * 64, (pr_waves<E, D>())) void paged_rows_kernel(PagedArgs a, PagedOut o) {
  constexpr int ROWS = 16 * RT, BK = RowsLayout<E, D>::BK, STEP = PR_NW * BK;
  __shared__ RowsLds<D, ROWS> lds;
  const int tid = threadIdx.x;
  const int r_heads = a.h_q / a.h_kv;
  const int h = blockIdx.x % a.h_kv;
  const bool shared = o.shares > 0;  // else the workgroup has a unit, and what follows one round of the loop
  // The blocks of all units, one after the other, in `shares` equal parts: lengths that differ, which only the device knows, leave
  // nobody waiting. Every workgroup adds the units up for itself; of up to 64 every wavefront does, without a barrier (all write the
  // same to LDS), and keeps what the device arrays say about their sequences.
  __shared__ int before[PR_UNITS + 1], wave_sum[PR_NW];
  __shared__ PagedSeq seqs[64];
  const int lane = tid & 63, wave = tid >> 6;
  const int share = blockIdx.x / a.h_kv, units = a.n_seqs * o.tiles;
  const bool few = !WIN && shared && units <= 64 && units > 1;
  int begin = 0, end = 1, u = share, all = 0, per = 0, more = 0;
  auto scan = [&](int sum) {
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
      const int y = __shfl_up(sum, x, 64);
      if (lane >= x) sum += y;
    }
    return sum;
  };
  if constexpr (WIN) {
    if (shared) {
      u = share / o.per_unit;
      all = unit_blocks<RT, WIN>(a, paged_seq_of(a, u / o.tiles), u % o.tiles, STEP);
      const int parts = min(o.per_unit, all), part = share - u * o.per_unit;
      if (part >= parts) return;
      if (part == 0 && h == 0 && tid == 0) o.info[u] = make_int2(u * o.per_unit, parts);
      per = all / parts;
      more = all - per * parts;
      begin = part * per + min(part, more);
      end = begin + per + (part < more);
    }
  } else if (few) {
    int n = 0;
    if (lane < units) {
      const PagedSeq q = paged_seq_of(a, lane / o.tiles);
      n = unit_blocks<RT, WIN>(a, q, lane % o.tiles, STEP);
      seqs[lane] = q;
    }
    const int sum = scan(n);
    if (lane < units) before[lane] = sum - n;
    if (lane == units - 1) before[units] = sum;
    all = __builtin_amdgcn_readlane(sum, units - 1);
  } else if (shared && units == 1) {  // one answer: nothing to add up
    all = unit_blocks<RT, WIN>(a, paged_seq_of(a, 0), 0, STEP);
  } else if (shared) {
    for (int u0 = 0; u0 < units; u0 += PR_NW * 64) {
      const int v = u0 + tid;
      const int n = v < units ? unit_blocks<RT, WIN>(a, paged_seq_of(a, v / o.tiles), v % o.tiles, STEP) : 0;
      const int sum = scan(n);
      if (lane == 63) wave_sum[wave] = sum;
      __syncthreads();
      int at = all;
#pragma unroll
      for (int w = 0; w < PR_NW; ++w) {
        if (w < wave) at += wave_sum[w];
        all += wave_sum[w];
      }
      if (v < units) before[v] = at + sum - n;
      __syncthreads();  // wave_sum has been read
    }
    if (tid == 0) before[units] = all;
    __syncthreads();
    all = __builtin_amdgcn_readfirstlane(all);  // the same in all lanes, which the compiler cannot see, nor of what comes from LDS
  }
  if (!WIN && shared) {
    const int shares = min(o.shares, all);  // each has a block at least
    if (share >= shares) return;
    per = all / shares;
    more = all - per * shares;  // the first ones have one more
    begin = share * per + min(share, more);
    end = begin + per + (share < more);
    // the unit with block `begin`: the last that starts there or before (units without rows have no blocks)
    u = 0;
    for (int step = units == 1 ? 0 : units > 64 ? PR_UNITS / 2 : 32; step > 0; step >>= 1)
      if (u + step <= units && __builtin_amdgcn_readfirstlane(before[u + step]) <= begin) u += step;
  }
  auto share_of = [&](int block) {
    const int longer = more * (per + 1);
    return block < longer ? block / (per + 1) : more + (block - longer) / per;
  };
  for (int at = begin; at < end; ++u) {
    const bool listed = !WIN && shared && units > 1;
    const int from = listed ? __builtin_amdgcn_readfirstlane(before[u]) : 0, to = listed ? __builtin_amdgcn_readfirstlane(before[u + 1]) : shared ? all : 1;
    if (from == to) continue;
    const int s = u / o.tiles, row0 = (u - s * o.tiles) * ROWS;
    PagedSeq q;
    if (few) {
      q.len = __builtin_amdgcn_readfirstlane(seqs[u].len);
      q.row0 = __builtin_amdgcn_readfirstlane(seqs[u].row0);
      q.n = __builtin_amdgcn_readfirstlane(seqs[u].n);
      q.base = __builtin_amdgcn_readfirstlane(seqs[u].base);
    } else {
      q = paged_seq_of(a, s);
    }
    const int n_rows = (int)min((long long)q.n * r_heads - row0, (long long)ROWS);
    if (n_rows <= 0) return;  // not shared: a tile without rows
    const int stop = min(to, end);
    const RowsGap gap = WIN ? rows_gap(a.window, a.n_sink, q.base + row0 / r_heads, BK) : RowsGap{0, 0};
    const int k_end = min(stop == to ? 0x7fffffff : (stop - from) * STEP, min(q.len, q.base + (row0 + n_rows - 1) / r_heads + 1) - gap.gap);
    const bool whole = at == from && stop == to;
    if (!WIN && shared && h == 0 && at == from && tid == 0) {
      const int first = share_of(from);
      o.info[u] = make_int2(first, share_of(to - 1) - first + 1);
    }
    __syncthreads();  // the last unit's results have been read
    rows_unit<E, D, RT, WIN>(a, o, lds, q, s, h, row0, n_rows, (at - from) * STEP, k_end, gap,
                             whole ? -1ll : (long long)h * (o.shares + units) + share + u);
    at = stop;
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
  const size_t at = (size_t)(q.row0 + i) * a.h_q + qh;
  int n = q.len == 0 ? 1 : (min(q.len, o.span) - 1) / o.chunk_keys + 1;  // chunks that answered
  size_t first = at, stride = (size_t)a.n_rows * a.h_q;     // their rows among the partial results
  if (o.shares > 0) {
    const int r_heads = a.h_q / a.h_kv, h = qh / r_heads;
    const long long row = (long long)i * r_heads + (qh - h * r_heads);
    const int tile = (int)(row / o.tile_rows), u = s * o.tiles + tile;
    const int2 info = o.info[u];
    n = info.y;
    if (n <= 1) return;  // one workgroup had the whole unit and wrote the output
    first = ((size_t)h * (o.shares + a.n_seqs * o.tiles) + info.x + u) * o.tile_rows + (size_t)(row - (long long)tile * o.tile_rows);
    stride = o.tile_rows;
  }
  constexpr int B = 8;
  float m = PR_NONE, den = 0.f, sum[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) sum[e] = 0.f;
  for (int c0 = W == 1 ? 0 : wave * B; c0 < n; c0 += B * W) {
    float ls[B], po[B][PER];
#pragma unroll
    for (int u = 0; u < B; ++u) {
      const size_t p = first + (size_t)min(c0 + u, n - 1) * stride;
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
// Eight wavefronts share a row of more than 16 chunks (of shares: so many per unit where all are as long as may be).
constexpr int PM_SHARE = 8;
static int merge_rows(const PagedArgs& a, const PagedPlan& p) {
  return (p.shares > 0 ? p.shares / ((long long)a.n_seqs * p.tiles) : p.chunks) > 16 ? 1 : PM_WAVES;
}
static long long merge_blocks(const PagedArgs& a, const PagedPlan& p) {
  const int rows = merge_rows(a, p);
  return (((long long)a.max_new * a.h_q + rows - 1) / rows) * a.n_seqs;
}

// Stacked rows above which bf16 heads of 128 take the tile kernel (attend_mfma.hip), and what its 32-bit arithmetic takes. A workgroup
// for few rows holds 32; more of them take the entries once for each 32. us few rows / tiles, 1, 4, 5, 8 and 12 tokens (of the 7B heads 28 rows are 4, of
// the 72B ones 32), one sequence over 46,125 entries: 7B heads, bf16 26.4 / 29.3, 29.6 / 30.5, 40.4 / 31.1, 41.8 / 32.3, 57.2 / 34.4, 8-bit 21.7 / 29.6,
// 25.0 / 31.1, 28.3 / 31.9, 29.7 / 33.1, 38.5 / 35.2; 72B heads, bf16 44.4 / 55.5, 47.8 / 57.4, 71.4 / 58.4, 72.9 / 60.7, 101 / 64.5, 8-bit 26.9 / 55.7,
// 32.5 / 57.6, 40.3 / 59.5, 42.0 / 61.7, 60.0 / 65.6. Of 16 sequences over up to 9,840 and over 8-bit pools, with scales or without, the tiles win later
// than the rule has it: 12 tokens of the 7B heads 76.5 / 81.7, 8-bit 47.1 / 88.6, with scales 52.3 / 91.2, of the 72B heads 140 / 102, 82.3 / 108, 91.5 / 111.
constexpr long long PT_FROM_ROWS = 32, PT_MOST_ROWS = 1 << 26;

PagedPlan plan_paged_attend(const PagedArgs& a, int dtype, int d, size_t scratch_bytes) {
  PagedPlan p{};
  const int r_heads = a.h_q / a.h_kv;
  const long long rows = (long long)a.max_new * r_heads;
  const bool tiled = dtype == QP_BF16 && d == 128 && rows > PT_FROM_ROWS && rows <= PT_MOST_ROWS;
  p.tile_rows = tiled ? PT_ROWS : rows <= 16 ? 16 : 32;
  p.tiles = (int)((rows + p.tile_rows - 1) / p.tile_rows);
  p.chunks = 1;
  // What a row tile has to look at: all entries, or the first ones and the windows of its tokens, each in whole blocks of keys
  int max_len = a.max_len;
  if (a.window > 0) {
    const int tokens = std::min(a.max_new, (p.tile_rows + r_heads - 2) / r_heads + 1);
    max_len = rows_span(a.window, a.n_sink, tokens, tiled ? 64 : dtype == QP_F32 ? 16 : 32, max_len);
  }
  p.span = p.chunk_keys = max_len;
  scratch_bytes = std::min(scratch_bytes, PAGED_ATTEND_SCRATCH);
  const long long units = (long long)a.n_seqs * p.tiles, cus = device_cu_count();
  if (!tiled) {
    // One workgroup per compute unit, two over 8-bit pools, whose blocks are longer chains over half the bytes, as long as each has
    // a block. us with the kernel as it was before masks went behind a branch (the first figure is 141 now, the second 76.5), equal
    // shares of all entries / equal chunks of the longest sequence (1, 2 and 4 workgroups per compute unit): up to
    // four tokens of 16 sequences of the 72B heads over 8-bit pages of up to 32,768 entries 163 / 251, 180, 187; one token of 32
    // sequences of the 7B heads over up to 9,840 79.0 / 84.8, 89.8, 93.2, of one over 46,125 26.0 / 25.0, 27.6, 30.1.
    const int step = PR_NW * (dtype == QP_F32 ? 16 : 32);
    const long long blocks = units * (((long long)max_len + step - 1) / step);
    p.workgroups = units * a.h_kv;
    long long shares = std::min(std::max<long long>(1, (a.fp8 ? 2 : 1) * cus / a.h_kv), blocks);
    // Of a few blocks a workgroup per unit makes no second launch. us with shares / without, one token: f32 heads of 64 over 128
    // entries 8.7 / 7.6, 256 11.4 / 8.7, 333 11.2 / 10.8, 600 12.0 / 14.6, 1,200 11.2 / 23.9; 7B heads over 256 8.4 / 8.4 (one launch
    // both), 333 14.0 / 12.7, 600 14.4 / 15.9, 1,200 15.4 / 22.4, over 8-bit pools 333 13.8 / 11.5, 600 13.9 / 14.2, 1,200 15.8 / 20.2.
    if (units > PR_UNITS || blocks > 0x7fffffff || max_len <= 2 * step) return p;
    const size_t per_share = (size_t)a.h_kv * p.tile_rows * (d + 1) * sizeof(float), info = (size_t)units * sizeof(int2);
    const long long fit = scratch_bytes < info ? 0ll : (long long)((scratch_bytes - info) / per_share) - units;
    if (a.window > 0) {
      // Windows are alike in length, so each unit has as many workgroups as the others: none has parts of two units, which costs it
      // the start and the end of both, and none adds up the others' blocks. As many as end first, in blocks of keys, with three for start and end.
      const long long n = (max_len + step - 1) / step, slots = shares;
      double least = 0;
      for (long long c = 1; c <= n && c * units <= std::min(4 * slots + units, PR_UNITS * 64ll); ++c) {
        const double cost = (double)((c * units + slots - 1) / slots) * ((n + c - 1) / c + 3) + (c > 1 ? 3 : 0);
        if (c * units <= std::max(fit, units) && (p.per_unit == 0 || cost < least)) p.per_unit = (int)c, least = cost;
      }
      if (p.per_unit <= 1) return p;
      shares = p.per_unit * units;
    }
    shares = std::min(shares, fit);
    if (shares < 2) return p;
    p.shares = (int)shares;
    p.workgroups = shares * a.h_kv;
    p.scratch_bytes = info + (size_t)(shares + units) * per_share;
    return p;
  }
  // One workgroup per compute unit at a time: four rounds of them, of at least 16 tiles of keys (four questions of up to 300
  // tokens over up to 46,125 entries: one round 544 us, two 580, three 555, four 506, six 531).
  const long long want = std::max<long long>(1, (4 * cus + units * a.h_kv - 1) / (units * a.h_kv));
  long long keys = std::max<long long>(((max_len + want - 1) / want + 63) / 64 * 64, 16 * 64);
  const size_t per_chunk = (size_t)a.n_rows * a.h_q * (d + 1) * sizeof(float);
  if (a.window > 0) {
    // Windows are alike in length, so a launch ends in rounds of workgroups, one per compute unit at a time, on each XCD's share of them
    // (see the mapping of workgroups there): as many chunks as end first. In tiles of keys, with seven for a workgroup's start and end and what
    // a second launch and the chunks' partial rows cost. us with 1 / 2 / 3 / 4 / 6 / 8 chunks of a window of 8,192 and 100 first entries, 7B heads: 300
    // tokens 241 / 137 / 104 / 87 / 68 / 89, of four sequences 240 / 254 / 213 / 227 / 231 / 222, up to 300 of four 240 / 162 / 197 / 165 / 180 / 184, 20 of
    // 16 226 / 131 / 99 / 84 / 105 / 95; up to 300 of four, window 4,096, 72B heads with scales 162 / 206 / 217 / 228 / 228 / 227.
    const long long n = (max_len + 63) / 64;
    const double blocks = std::min((double)p.tiles, std::ceil((double)a.n_rows * r_heads / PT_ROWS / a.n_seqs + 0.5));  // of rows, per sequence
    const int xcds = 8 % a.h_kv == 0 ? 8 / a.h_kv : 1, heads = a.h_kv % 8 == 0 ? a.h_kv / 8 : 1;                // of a head, of an XCD
    double least = 0;
    for (long long c = 1; c <= std::min<long long>(n, 64); ++c) {
      double wgs = (double)((a.n_seqs * c + xcds - 1) / xcds) * heads * blocks;  // on the XCD with most
      if (8 % a.h_kv != 0 && a.h_kv % 8 != 0) wgs = (double)a.n_seqs * c * a.h_kv * blocks / 8;
      const double cost = std::ceil(wgs * 8 / cus) * ((n + c - 1) / c + 7) + (c > 1 ? 3 + c * (double)per_chunk / 14e6 : 0);
      if (c == 1 || cost < least) keys = (n + c - 1) / c * 64, least = cost;
    }
  }
  long long chunks = (max_len + keys - 1) / keys;
  const long long fit = (long long)(scratch_bytes / per_chunk);
  if (chunks > fit) {
    chunks = fit >= 2 ? fit : 1;
    keys = ((max_len + chunks - 1) / chunks + 63) / 64 * 64;
    chunks = (max_len + keys - 1) / keys;
  }
  if (chunks > 1) p.chunks = (int)chunks, p.chunk_keys = (int)keys, p.scratch_bytes = per_chunk * p.chunks;
  p.workgroups = paged_tile_blocks(a, p);
  return p;
}

template <typename E, int D, bool WIN>
static void launch_rows(const PagedArgs& a, const PagedOut& o, const PagedPlan& p, hipStream_t s) {
  const dim3 grid((unsigned)p.workgroups), block(PR_NW * 64);
  if (p.tile_rows == 16) hipLaunchKernelGGL((paged_rows_kernel<E, D, 1, WIN>), grid, block, 0, s, a, o);
  else hipLaunchKernelGGL((paged_rows_kernel<E, D, 2, WIN>), grid, block, 0, s, a, o);
}

template <typename E, typename T, int D>
static bool attend_as(const PagedArgs& a, const PagedOut& o, const PagedPlan& p, hipStream_t s) {
  if (p.tile_rows == PT_ROWS) launch_paged_tiles(a, p, o.q, o.out, o.lse, o.part_o, o.part_lse, s);
  else if (a.window > 0) launch_rows<E, D, true>(a, o, p, s);
  else launch_rows<E, D, false>(a, o, p, s);
  if (p.chunks > 1 || p.shares > 0) {
    const dim3 merge((unsigned)merge_blocks(a, p));
    if (merge_rows(a, p) == 1) hipLaunchKernelGGL((paged_merge_kernel<T, D, PM_SHARE>), merge, dim3(PM_SHARE * 64), 0, s, a, o);
    else hipLaunchKernelGGL((paged_merge_kernel<T, D, 1>), merge, dim3(PM_WAVES * 64), 0, s, a, o);
  }
  return true;
}

bool launch_paged_attend(const PagedArgs& a, int dtype, int d, const void* q, void* out, float* lse, void* scratch,
                         size_t scratch_bytes, hipStream_t s) {
  const PagedPlan p = plan_paged_attend(a, dtype, d, scratch != nullptr ? scratch_bytes : 0);
  if (p.workgroups * (p.tile_rows == PT_ROWS ? 512 : PR_NW * 64) > PAGED_MAX_THREADS) return false;
  if ((p.chunks > 1 || p.shares > 0) && merge_blocks(a, p) * PM_SHARE * 64 > PAGED_MAX_THREADS) return false;
  PagedOut o{};
  o.q = q, o.out = out, o.lse = lse;
  o.tiles = p.tiles, o.chunks = p.chunks, o.chunk_keys = p.chunk_keys;
  o.shares = p.shares, o.tile_rows = p.tile_rows, o.span = p.span, o.per_unit = p.per_unit;
  const size_t part_rows = p.shares > 0 ? (size_t)(p.shares + a.n_seqs * p.tiles) * a.h_kv * p.tile_rows : (size_t)p.chunks * a.n_rows * a.h_q;
  o.part_o = (float*)scratch;
  o.part_lse = o.part_o + part_rows * d;
  o.info = (int2*)(o.part_lse + part_rows);  // part_rows is even
  if (dtype == QP_F32) return d == 64 ? attend_as<float, float, 64>(a, o, p, s) : attend_as<float, float, 128>(a, o, p, s);
  if (a.fp8 == QP_CACHE_FP8_E4M3_SCALED) return attend_as<ScaledCode, bf16_t, 128>(a, o, p, s);
  if (a.fp8) return attend_as<uint8_t, bf16_t, 128>(a, o, p, s);
  return d == 64 ? attend_as<bf16_t, bf16_t, 64>(a, o, p, s) : attend_as<bf16_t, bf16_t, 128>(a, o, p, s);
}

}  // namespace qp

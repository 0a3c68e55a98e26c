// The attention weight that the paged cache's entries received: w[j] (+)= sum over rows of exp2(c q.k_j - lse2), the column sums
// of the softmax whose row statistics qp_paged_attend left. No atomics: an entry's sum is one lane's, from the first row to the last.
//
// weigh_stream_kernel: few rows (decoding, drafted tokens). Queries and their statistics stay in registers, and a wavefront walks
// blocks of 32 keys (16 of f32), the next one requested while it works on this: S = Q K^T leaves a lane with one entry (column) and
// four rows. Bound by the keys' way from HBM: 3.7 TB/s, where wavefronts that take 64 keys at once and end reached 3.4 (54 us), and no
// more with fewer or more workgroups per compute unit. Attention of the same rows, whose workgroups have equal parts of all
// entries, reads at 5.0: these have up to `entries` of one sequence each and those behind its end have none.
//
// paged_weigh_kernel: chunks over layouts without a tile kernel. A wavefront owns 64 entries (32 of f32) of a KV head, whose keys stay
// in registers, and walks the sequence's rows 16 at a time.
//
// weigh_tile_kernel: chunks over bf16 heads of 128. Four wavefronts own 64 entries each, keys in registers, and walk the rows 32 at a
// time, which all of them read from LDS: tiles of queries go global -> LDS directly (XOR-swizzled 16-byte chunks), in a ring of four
// slots, three ahead, one barrier each. A pair costs a multiply-add, an exponential at a quarter of the rate and an add, 24 cycles per
// 64 pairs of the vector unit, beside the products' 16 on the matrix pipe: 98 and 66 us at 2.4 GHz for 500 tokens of the 7B heads over
// 46,125 entries (one question), which take 190. The clock stays at 2.4 GHz under it and the matrix pipe is busy for 34 % of the cycles
// (counters), so the two stand one behind the other and do not overlap. Products of 32 x 32 x 16 took 205-208, four wavefronts per
// SIMD instead of three 194-195, and before that two with a second set of scores, so that one tile's exponentials should have stood beside the
// next one's products, 217-222, with a barrier for every second tile the same.
#include "paged_rows.h"

#include <algorithm>

namespace qp {

constexpr int PW_NW = 4;
template <typename E>
constexpr int pw_tiles() { return sizeof(E) == 4 ? 2 : 4; }

template <typename E, int D>
__global__ __launch_bounds__(PW_NW * 64) void paged_weigh_kernel(PagedArgs a, const void* __restrict__ qp_, const float* __restrict__ lse,
                                                                int accumulate) {
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
  float scale[KT];  // of the tiles' codes
  int page[KT];
#pragma unroll
  for (int t = 0; t < KT; ++t) {
    const int key = key0 + 16 * t;
    page[t] = key < q.len ? __builtin_amdgcn_readfirstlane(a.table[(size_t)s * a.table_pages + (key >> a.page_shift)]) : -1;
    if (!paged_page_ok(page[t], a.n_pages)) page[t] = -1;
    const size_t row = paged_row(max(page[t], 0), h, key & mask, a.h_kv, a.page_shift);
    rows_load_k<E, D>((const unsigned char*)a.k + row * L::ROWB, l16, g, k[t]);
    scale[t] = L::SCALED ? a.k_scale[row >> 4] : 1.f;
  }
  float w[KT];
  float* to[KT];  // group g stores tile g: what was there is requested with the keys
  float before = 0.f;
#pragma unroll
  for (int t = 0; t < KT; ++t) {
    w[t] = 0.f;
    const int key = key0 + 16 * t + l16;
    to[t] = a.weight + paged_row(max(page[t], 0), h, key & mask, a.h_kv, a.page_shift);
    if (accumulate && g == t && page[t] >= 0 && key < q.len) before = *to[t];
  }
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
      const pr_f32x4 st = rows_products<E, D>(k[t], qf, scale[t]);
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
    if (g == t && page[t] >= 0 && key < q.len) *to[t] = before + w[t];
  }
}

// Entries of a workgroup: in pages of 16, at most one page number for each lane. One token of 32 sequences of the 7B heads over up to
// 9,840 entries (187 MB of keys): 128 entries 65 us, 256 54.0, 384 50.0, 512 50.4, 1024 51.5.
constexpr int WS_MOST = 512;
template <typename E, int D, int RT>
__global__ __launch_bounds__(PW_NW * 64, (RT == 1 ? 4 : 3)) void weigh_stream_kernel(PagedArgs a, const void* __restrict__ qp_, const float* __restrict__ lse,
                                                                               int accumulate, int entries) {
  using L = RowsLayout<E, D>;
  constexpr int STEP = PW_NW * L::BK;
  const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int x = blockIdx.x;
  const int h = x % a.h_kv;
  x /= a.h_kv;
  const int s = x % a.n_seqs;
  const PagedSeq q = paged_seq_of(a, s);
  const long long from = (long long)(x / a.n_seqs) * entries;
  if (from >= q.len) return;
  const int first = (int)from, end = min(q.len, first + entries);
  const int r_heads = a.h_q / a.h_kv, mask = (1 << a.page_shift) - 1, page0 = first >> a.page_shift;
  int list = -1;
  if (page0 + lane <= (end - 1) >> a.page_shift) list = a.table[(size_t)s * a.table_pages + page0 + lane];

  struct Block {
    pr_u32x4 k[L::TILES][L::KL];
    float* to;     // group t: the entry of tile t that this lane stores, nullptr: none
    float before;
    float scales;  // SCALED: that of tile t's codes in lane t, see RowsBlock
  };
  auto load = [&](Block& b, int key0) {
    b.to = nullptr;
    b.before = 0.f;
    size_t rows[L::TILES];
#pragma unroll
    for (int t = 0; t < L::TILES; ++t) {
      const int key = key0 + 16 * t;
      // a tile past the last entry takes the block's first page: read, never used
      const int page = __builtin_amdgcn_readlane(list, ((key < end ? key : key0) >> a.page_shift) - page0);
      const bool ok = paged_page_ok(page, a.n_pages);
      const size_t row = paged_row(ok ? page : 0, h, key & mask, a.h_kv, a.page_shift);
      rows[t] = row;
      rows_load_k<E, D>((const unsigned char*)a.k + row * L::ROWB, l16, g, b.k[t]);
      if (g == t && ok && key + l16 < end) b.to = a.weight + row + l16;
    }
    if constexpr (L::SCALED) b.scales = a.k_scale[((lane & 1) ? rows[L::TILES - 1] : rows[0]) >> 4];
    if (accumulate && b.to != nullptr) b.before = *b.to;
  };
  const int n_rows = q.n * r_heads;  // 16 RT at most
  pr_u32x4 qf[RT][L::QF];
  float neg[RT][4];
  int lim[RT][4];  // -1: a row that there is not, or that saw nothing
  Block b0, b1;
  int key = first + wave * L::BK;
  if (key < end) load(b0, key);
  bool all = true;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    if (n_rows > 0) {
      const int row = min(16 * t + l16, n_rows - 1), i = row / r_heads;
      const unsigned char* p = (const unsigned char*)qp_ + ((size_t)(q.row0 + i) * a.h_q + (size_t)h * r_heads + (row - i * r_heads)) * (D * L::QB);
#pragma unroll
      for (int u = 0; u < L::QF; ++u) qf[t][u] = *(const pr_u32x4*)(p + rows_q_byte<E, D>(u, g));
    } else {
#pragma unroll
      for (int u = 0; u < L::QF; ++u) qf[t][u] = pr_u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      neg[t][r] = -INFINITY;
      lim[t][r] = -1;
      const int row = 16 * t + 4 * g + r;
      if (row >= n_rows) continue;
      const int i = row / r_heads;
      const float z = lse[(size_t)(h * r_heads + row - i * r_heads) * a.n_rows + q.row0 + i];
      neg[t][r] = -z * 1.4426950408889634f;
      lim[t][r] = z != -INFINITY ? q.base + i : -1;
      all = all && lim[t][r] >= end - 1;
    }
    all = all && 16 * (t + 1) <= n_rows;
  }
  const bool whole = __all(all);
  const float c2 = a.scale_log2;
  auto compute = [&](Block& b, int key0) {
    float w = 0.f;
#pragma unroll
    for (int t = 0; t < L::TILES; ++t) {
      float sum = 0.f, scale = 1.f;
      if constexpr (L::SCALED) scale = __uint_as_float((unsigned)__builtin_amdgcn_readlane(__float_as_uint(b.scales), t));
#pragma unroll
      for (int y = 0; y < RT; ++y) {
        const pr_f32x4 st = rows_products<E, D>(b.k[t], qf[y], scale);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float p = __builtin_amdgcn_exp2f(fmaf(st[r], c2, neg[y][r]));
          sum += whole || key0 + 16 * t + l16 <= lim[y][r] ? p : 0.f;
        }
      }
      sum += __shfl_xor(sum, 16, 64);
      sum += __shfl_xor(sum, 32, 64);
      w = g == t ? sum : w;
    }
    if (b.to != nullptr) *b.to = b.before + w;
  };
  while (key < end) {
    if (key + STEP < end) load(b1, key + STEP);
    compute(b0, key);
    key += STEP;
    if (key >= end) break;
    if (key + STEP < end) load(b0, key + STEP);
    compute(b1, key);
    key += STEP;
  }
}

constexpr int WT_NW = 4;                 // wavefronts of a workgroup
constexpr int WT_KEYS = WT_NW * 64;      // and its entries
constexpr int WT_SLOTS = 4;
constexpr int WT_TILE = 32 * 256;        // bytes of 32 rows of queries
constexpr int WT_ROWS = 4096;            // rows whose statistics lie in LDS at a time
constexpr int WT_LDS = WT_SLOTS * WT_TILE;
constexpr int WT_MIN_TILES = 8;          // row tiles that a workgroup takes at least where rows are dealt to several

struct WeighTiles {
  const void* q;
  const float* lse;
  int accumulate;
  int splits;        // workgroups that share a block of entries' rows
  float* partial;    // [splits][n_seqs][h_kv][max_len], splits > 1
};

template <int N>
__device__ __forceinline__ void weigh_wait() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}

template <bool F8, bool SCALED>
__global__ __launch_bounds__(WT_NW * 64, 3) void weigh_tile_kernel(PagedArgs a, WeighTiles o) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  __shared__ __attribute__((aligned(16))) float neg[WT_ROWS];  // -lse of the segment's rows, base 2
  __shared__ int dead[WT_ROWS / 32];                           // a row of the tile saw nothing
  constexpr int ROWB = F8 ? 128 : 256;
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int x = blockIdx.x;
  const int h = x % a.h_kv;
  x /= a.h_kv;
  const int s = x % a.n_seqs;
  x /= a.n_seqs;
  const int split = x % o.splits;
  const long long wg_first = (long long)(x / o.splits) * WT_KEYS;
  const PagedSeq q = paged_seq_of(a, s);
  if (wg_first >= q.len) return;
  const int wg_key = (int)wg_first, key0 = wg_key + 64 * wave;
  const int r_heads = a.h_q / a.h_kv;
  const int rows = q.n * r_heads;
  const int mask = (1 << a.page_shift) - 1;

  // this lane's four entries: their keys, and the first row that sees them; it stores the one of tile g
  pr_u32x4 k[4][4];
  size_t mine_at = 0;
  bool mine = false;
  int first_row[4];
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const int key = key0 + 16 * b + l16, kc = min(key, q.len - 1);
    const int page = a.table[(size_t)s * a.table_pages + (kc >> a.page_shift)];
    const bool ok = paged_page_ok(page, a.n_pages);
    const size_t at = paged_row(ok ? page : 0, h, kc & mask, a.h_kv, a.page_shift);
    if (g == b) mine_at = at, mine = ok && key < q.len;
    first_row[b] = paged_clamp(key - q.base, 0, q.n) * r_heads;
    const unsigned char* p = (const unsigned char*)a.k + at * ROWB;
    const float scale = SCALED && ok ? a.k_scale[at >> 4] : 1.f;
#pragma unroll
    for (int st = 0; st < 4; ++st) {
      if constexpr (F8) {
        const uint2 raw = *(const uint2*)(p + 32 * st + 8 * g);
        k[b][st] = pr_widen8(raw.x, raw.y, scale);
      } else {
        k[b][st] = *(const pr_u32x4*)(p + 64 * st + 16 * g);
      }
    }
  }
  // rows from the first tile that sees the workgroup's first entry on, this workgroup's share of them
  const int tile_first = paged_clamp(wg_key - q.base, 0, q.n) * r_heads / 32, tile_end = (rows + 31) / 32;
  const int per = (tile_end - tile_first + o.splits - 1) / o.splits;
  const int begin = min(tile_first + split * per, tile_end), end = min(begin + per, tile_end);
  const int masked_below = paged_clamp(key0 + 63 - q.base, 0, q.n) * r_heads;  // rows below do not see all of the wavefront's entries

  int q_addr[4];  // query fragment of step st: row l16, chunk 4 st + g at position (4 st + g) ^ l16; rows 16 .. 31 alike
#pragma unroll
  for (int st = 0; st < 4; ++st) q_addr[st] = l16 * 256 + (((4 * st + g) ^ l16) << 4);
  const unsigned ring = lds_address(smem);
  const float c2 = a.scale_log2;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};

  for (int seg = begin; seg < end; seg += WT_ROWS / 32) {  // tiles of a segment
    const int seg_end = min(end, seg + WT_ROWS / 32);
    const int row0 = seg * 32;
    __syncthreads();  // the last segment's statistics and slots have been read
    if (tid < WT_ROWS / 32) dead[tid] = 0;
    __syncthreads();
    // queries: request i of a wavefront fills rows 8 wave + 4 i + (lane >> 4) of a slot, chunk lane & 15 of each from where the swizzle
    // has it; a row's offset goes on by 32 rows from tile to tile
    const int t_seg = row0 / r_heads;
    const unsigned char* const qb = (const unsigned char*)o.q + ((size_t)(q.row0 + t_seg) * a.h_q + (size_t)h * r_heads) * 256;
    const int last_row = min(rows, seg_end * 32) - 1;
    const unsigned last_off = (unsigned)(last_row / r_heads - t_seg) * (unsigned)a.h_q * 256u + (unsigned)(last_row % r_heads) * 256u;
    int rt[2], rj[2];
    unsigned swz[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = 8 * wave + 4 * i + (lane >> 4), full = row0 + r;
      rt[i] = full / r_heads - t_seg;
      rj[i] = full % r_heads;
      swz[i] = (unsigned)((((lane & 15) ^ (r & 15))) << 4);
    }
    const int step_t = 32 / r_heads, step_j = 32 % r_heads;
    auto request = [&](int slot) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        // rows past the last one repeat it: masked below
        const unsigned off = min((unsigned)rt[i] * ((unsigned)a.h_q * 256u) + (unsigned)rj[i] * 256u, last_off);
        lds_dma16_to(qb, off + swz[i], ring + slot * WT_TILE + (8 * wave + 4 * i) * 256);
        rt[i] += step_t;
        rj[i] += step_j;
        if (rj[i] >= r_heads) rj[i] -= r_heads, ++rt[i];
      }
    };
    const int n = seg_end - seg;
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < n) request(i);
    // the rows' statistics, six loads of a thread under way together
    {
      constexpr int STEP = WT_NW * 64, B = 6;
      const int rows_here = (seg_end - seg) * 32;
      int t = (row0 + tid) / r_heads, j = row0 + tid - t * r_heads;
      const int dt = STEP / r_heads, dj = STEP % r_heads;
      for (int r0 = tid; r0 < rows_here; r0 += B * STEP) {
        float z[B];
#pragma unroll
        for (int u = 0; u < B; ++u) {
          const int r = r0 + u * STEP;
          z[u] = r < rows_here && row0 + r < rows ? o.lse[(size_t)(h * r_heads + j) * a.n_rows + q.row0 + t] : -INFINITY;
          t += dt;
          j += dj;
          if (j >= r_heads) j -= r_heads, ++t;
        }
#pragma unroll
        for (int u = 0; u < B; ++u) {
          const int r = r0 + u * STEP;
          if (r >= rows_here) continue;
          neg[r] = z[u] == -INFINITY ? -INFINITY : -z[u] * 1.4426950408889634f;
          if (z[u] == -INFINITY && row0 + r < rows) dead[r >> 5] = 1;
        }
      }
    }
    for (int i = 0; i < n; ++i) {
      // tile i is there: two more may be under way. The statistics' loads were waited for by the compiler.
      if (i + 2 < n) weigh_wait<4>();
      else if (i + 1 < n) weigh_wait<2>();
      else weigh_wait<0>();
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this wavefront's statistics are written, its reads of tile i - 1 done
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (i + 3 < n) request((i + 3) & 3);
      const unsigned char* const slot = smem + (i & 3) * WT_TILE;
      const int tile_row = row0 + i * 32;
      const bool whole = tile_row >= masked_below && tile_row + 32 <= rows && __builtin_amdgcn_readfirstlane(dead[i]) == 0;
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        pr_u32x4 qf[4];
#pragma unroll
        for (int st = 0; st < 4; ++st) qf[st] = *(const pr_u32x4*)(slot + q_addr[st] + 4096 * y);
        const float4 ng = *(const float4*)&neg[i * 32 + 16 * y + 4 * g];
        pr_f32x4 sc[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) sc[b] = pr_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < 4; ++st)
#pragma unroll
          for (int b = 0; b < 4; ++b)
            sc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pr_bf16x8, qf[st]),
                                                            __builtin_bit_cast(pr_bf16x8, k[b][st]), sc[b], 0, 0, 0);
        if (whole) {
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[b][0], c2, ng.x)), p1 = __builtin_amdgcn_exp2f(fmaf(sc[b][1], c2, ng.y));
            const float p2 = __builtin_amdgcn_exp2f(fmaf(sc[b][2], c2, ng.z)), p3 = __builtin_amdgcn_exp2f(fmaf(sc[b][3], c2, ng.w));
            sum[b] += (p0 + p1) + (p2 + p3);
          }
        } else {
#pragma unroll
          for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float z = e == 0 ? ng.x : e == 1 ? ng.y : e == 2 ? ng.z : ng.w;
              const int r = tile_row + 16 * y + 4 * g + e;
              const bool seen = r >= first_row[b] && r < rows && z != -INFINITY;
              const float p = __builtin_amdgcn_exp2f(fmaf(sc[b][e], c2, z));
              sum[b] += seen ? p : 0.f;
            }
        }
      }
    }
  }
  float w = 0.f;
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    float x = sum[b] + __shfl_xor(sum[b], 16, 64);
    x += __shfl_xor(x, 32, 64);
    w = g == b ? x : w;
  }
  if (!mine) return;
  if (o.splits > 1) {
    o.partial[(((size_t)split * a.n_seqs + s) * a.h_kv + h) * a.max_len + key0 + lane] = w;
  } else {
    float* const to = a.weight + mine_at;
    *to = o.accumulate ? *to + w : w;
  }
}

// Adds the workgroups' shares in their order.
constexpr int WA_THREADS = 256;
__global__ __launch_bounds__(WA_THREADS) void weigh_add_kernel(PagedArgs a, WeighTiles o, int blocks) {
  const int sh = blockIdx.x / blocks, s = sh / a.h_kv, h = sh - s * a.h_kv;
  const long long key = (long long)(blockIdx.x - sh * blocks) * WA_THREADS + threadIdx.x;
  if (key >= paged_seq_of(a, s).len) return;
  const int page = a.table[(size_t)s * a.table_pages + ((int)key >> a.page_shift)];
  if (!paged_page_ok(page, a.n_pages)) return;
  float w = 0.f;
  for (int i = 0; i < o.splits; ++i) w += o.partial[((size_t)i * a.n_seqs * a.h_kv + sh) * a.max_len + key];
  float* const to = a.weight + paged_row(page, h, (int)key & ((1 << a.page_shift) - 1), a.h_kv, a.page_shift);
  *to = o.accumulate ? *to + w : w;
}

// Rows above which a call takes the tiles (stacked rows of a KV head), and what their 32-bit arithmetic takes. weigh_stream_kernel holds
// 32. us streamed / in tiles: 7B heads, one sequence over 46,125 entries, 1 token 12.1 / 12.6, 4 (28 rows) 15.0 / 12.5, 16 sequences over up
// to 9,840 28.8 / 31.5 and 34.5 / 31.5; 72B heads over 8-bit pools 12.6 / 20.5, 17.1 / 19.6, 28.8 / 50.1 and 36.9 / 49.7.
constexpr long long WT_FROM_ROWS = 32, WT_MOST_ROWS = 1 << 26;
constexpr int WT_MOST_HEADS = 1024;
static bool weigh_tiled(const PagedArgs& a, int dtype, int d) {
  const long long rows = (long long)a.max_new * (a.h_q / a.h_kv);
  return dtype == QP_BF16 && d == 128 && rows > WT_FROM_ROWS && rows <= WT_MOST_ROWS && a.h_kv <= WT_MOST_HEADS;
}
// Workgroups that share a block of entries' rows: as many as make two per compute unit, of WT_MIN_TILES row tiles and more.
static int weigh_splits(long long blocks, long long rows, size_t per_split, size_t scratch) {
  const long long want = 2ll * device_cu_count() / std::max<long long>(blocks, 1);
  const long long most = std::min<long long>(rows / (32 * WT_MIN_TILES), per_split > 0 ? (long long)(scratch / per_split) : 0);
  return (int)std::max<long long>(1, std::min<long long>(std::min<long long>(want, most), 32));
}
static size_t weigh_per_split(int n_seqs, int h_kv, int max_len) { return (size_t)n_seqs * h_kv * max_len * sizeof(float); }
static long long weigh_blocks(int n_seqs, int h_kv, int max_len) {
  return ((long long)max_len + WT_KEYS - 1) / WT_KEYS * n_seqs * h_kv;
}

size_t paged_weigh_workspace_bytes(int n_seqs, int h_q, int h_kv, int max_new, int max_len) {
  const long long rows = (long long)max_new * (h_q / h_kv);
  const size_t per = weigh_per_split(n_seqs, h_kv, max_len);
  const int splits = weigh_splits(weigh_blocks(n_seqs, h_kv, max_len), rows, per, ~(size_t)0);
  return splits > 1 ? splits * per : 0;
}

template <bool F8, bool SCALED>
static bool weigh_tiles_as(const PagedArgs& a, const void* q, const float* lse, int accumulate, void* scratch, size_t scratch_bytes,
                           hipStream_t s) {
  const long long blocks = weigh_blocks(a.n_seqs, a.h_kv, a.max_len);
  WeighTiles o{q, lse, accumulate, 1, (float*)scratch};
  if (scratch != nullptr)
    o.splits = weigh_splits(blocks, (long long)a.max_new * (a.h_q / a.h_kv), weigh_per_split(a.n_seqs, a.h_kv, a.max_len), scratch_bytes);
  if (blocks * o.splits * WT_NW * 64 > PAGED_MAX_THREADS) return false;
  hipLaunchKernelGGL((weigh_tile_kernel<F8, SCALED>), dim3((unsigned)(blocks * o.splits)), dim3(WT_NW * 64), WT_LDS, s, a, o);
  if (o.splits > 1) {
    const int per = (a.max_len + WA_THREADS - 1) / WA_THREADS;
    hipLaunchKernelGGL(weigh_add_kernel, dim3((unsigned)((long long)per * a.n_seqs * a.h_kv)), dim3(WA_THREADS), 0, s, a, o, per);
  }
  return true;
}

template <typename E, int D>
static bool weigh_as(const PagedArgs& a, const void* q, const float* lse, int accumulate, hipStream_t s) {
  const long long rows = (long long)a.max_new * (a.h_q / a.h_kv);
  if (rows <= WT_FROM_ROWS) {  // what weigh_stream_kernel holds
    constexpr int STEP = PW_NW * RowsLayout<E, D>::BK;
    const long long heads = (long long)a.n_seqs * a.h_kv;
    const long long want = (heads * a.max_len / (4ll * device_cu_count()) + STEP - 1) / STEP * STEP;  // four workgroups per compute unit
    const int entries = (int)std::max<long long>(STEP, std::min<long long>(want, WS_MOST));
    const long long all = ((long long)a.max_len + entries - 1) / entries * heads;
    if (all * PW_NW * 64 > PAGED_MAX_THREADS) return false;
    const dim3 grid((unsigned)all), block(PW_NW * 64);
    if (rows <= 16) hipLaunchKernelGGL((weigh_stream_kernel<E, D, 1>), grid, block, 0, s, a, q, lse, accumulate, entries);
    else hipLaunchKernelGGL((weigh_stream_kernel<E, D, 2>), grid, block, 0, s, a, q, lse, accumulate, entries);
    return true;
  }
  constexpr int KEYS = PW_NW * 16 * pw_tiles<E>();
  const long long all = ((long long)a.max_len + KEYS - 1) / KEYS * a.n_seqs * a.h_kv;
  if (all * PW_NW * 64 > PAGED_MAX_THREADS) return false;
  hipLaunchKernelGGL((paged_weigh_kernel<E, D>), dim3((unsigned)all), dim3(PW_NW * 64), 0, s, a, q, lse, accumulate);
  return true;
}

bool launch_paged_weigh(const PagedArgs& a, int dtype, int d, const void* q, const float* lse, int accumulate, void* scratch,
                        size_t scratch_bytes, hipStream_t s) {
  if (weigh_tiled(a, dtype, d))
    return a.fp8 == QP_CACHE_FP8_E4M3_SCALED ? weigh_tiles_as<true, true>(a, q, lse, accumulate, scratch, scratch_bytes, s)
           : a.fp8                           ? weigh_tiles_as<true, false>(a, q, lse, accumulate, scratch, scratch_bytes, s)
                                             : weigh_tiles_as<false, false>(a, q, lse, accumulate, scratch, scratch_bytes, s);
  if (dtype == QP_F32) return d == 64 ? weigh_as<float, 64>(a, q, lse, accumulate, s) : weigh_as<float, 128>(a, q, lse, accumulate, s);
  if (a.fp8 == QP_CACHE_FP8_E4M3_SCALED) return weigh_as<ScaledCode, 128>(a, q, lse, accumulate, s);
  if (a.fp8) return weigh_as<uint8_t, 128>(a, q, lse, accumulate, s);
  return d == 64 ? weigh_as<bf16_t, 64>(a, q, lse, accumulate, s) : weigh_as<bf16_t, 128>(a, q, lse, accumulate, s);
}

}  // namespace qp

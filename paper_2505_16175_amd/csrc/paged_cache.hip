// The paged cache's entries on their way: new rows stored in pages, and the entries of most weight moved to other pages.
//
// append   a copy: row r of head h -> its sequence's entry. Bound by HBM (2 rows in, 2 rows out per token and head) from a few
//          thousand rows on, by the launch below.
// evict    two launches. evict_select_kernel: one workgroup per (sequence, head) finds which entries stay, as order-preserving
//          keys (an entry that stays in any case above all weights, one on a missing page out of the search) through
//          select_threshold, and lists them in ascending order. evict_move_kernel: many workgroups copy the listed rows, which
//          is where the bytes are (4 rows of head_dim per kept entry against 4 bytes per entry for the selection).
#include "append.h"
#include "paged.h"
#include "select.h"

namespace qp {

// ---- append ----------------------------------------------------------------------------------------------------------

constexpr int PA_THREADS = 256;
// LPR: lanes per source row, 16 bytes each. CONVERT: bf16 rows (LPR 16) into an 8-bit pool. U: rows per thread, all requested before
// the first store.
template <int LPR, bool CONVERT, int U>
__global__ __launch_bounds__(PA_THREADS) void paged_append_kernel(PagedArgs a, PagedAppend src, int blocks_per_seq) {
  constexpr int ROWS = PA_THREADS / LPR;
  constexpr int OUT = CONVERT ? 8 : 16;  // bytes of a lane's piece in the pool
  const int s = blockIdx.x / blocks_per_seq, b = blockIdx.x - s * blocks_per_seq;
  const PagedSeq q = paged_seq_of(a, s);
  const int sub = threadIdx.x % LPR;
  const int mask = (1 << a.page_shift) - 1;
  u32x4 kk[U], vv[U];
  size_t row[U];
  int pos[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    // rows of a head side by side: they are neighbours in the page, and in a source with the heads outside
    const long long x = ((long long)b * U + u) * ROWS + threadIdx.x / LPR;
    const int h = (int)(x / a.max_new), i = (int)(x - (long long)h * a.max_new);
    row[u] = ~(size_t)0;
    const int j = q.base + i;
    if (h >= a.h_kv || i >= q.n || j < 0 || j >= q.len) continue;
    const int page = a.table[(size_t)s * a.table_pages + (j >> a.page_shift)];
    if (!paged_page_ok(page, a.n_pages)) continue;
    const size_t r = (size_t)(q.row0 + i);
    const size_t at = r * src.token_stride + (size_t)h * src.head_stride + sub * 16;
    kk[u] = *(const u32x4*)((const unsigned char*)src.k + at);
    vv[u] = *(const u32x4*)((const unsigned char*)src.v + at);
    pos[u] = sub == 0 ? src.pos[r * src.pos_token_stride + (size_t)h * src.pos_head_stride] : 0;
    row[u] = paged_row(page, h, j & mask, a.h_kv, a.page_shift);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (row[u] == ~(size_t)0) continue;
    const size_t at = row[u] * (LPR * OUT) + sub * OUT;
    if constexpr (CONVERT) {
      *(uint2*)((unsigned char*)a.k + at) = pack8_e4m3(kk[u]);
      *(uint2*)((unsigned char*)a.v + at) = pack8_e4m3(vv[u]);
    } else {
      *(u32x4*)((unsigned char*)a.k + at) = kk[u];
      *(u32x4*)((unsigned char*)a.v + at) = vv[u];
    }
    if (sub == 0) {
      a.pos[row[u]] = pos[u];
      if (a.weight != nullptr) a.weight[row[u]] = 0.f;
    }
  }
}

template <int LPR, bool CONVERT>
static bool append_as(const PagedArgs& a, const PagedAppend& src, hipStream_t s) {
  constexpr int U = 4;
  constexpr int ROWS = PA_THREADS / LPR;
  const long long rows = (long long)a.max_new * a.h_kv;
  const bool many = rows * a.n_seqs > 4096;  // enough rows to fill the card with four per thread
  const long long per = (rows + ROWS * (many ? U : 1) - 1) / (ROWS * (many ? U : 1));
  if (per * a.n_seqs * PA_THREADS > PAGED_MAX_THREADS) return false;
  const dim3 grid((unsigned)(per * a.n_seqs));
  if (many) hipLaunchKernelGGL((paged_append_kernel<LPR, CONVERT, U>), grid, dim3(PA_THREADS), 0, s, a, src, (int)per);
  else hipLaunchKernelGGL((paged_append_kernel<LPR, CONVERT, 1>), grid, dim3(PA_THREADS), 0, s, a, src, (int)per);
  return true;
}

bool launch_paged_append(const PagedArgs& a, const PagedAppend& src, int dtype, int d, hipStream_t s) {
  if (a.fp8 && !src.raw) return append_as<16, true>(a, src, s);  // bf16 heads of 128
  const int bytes = d * (src.raw ? 1 : dtype == QP_F32 ? 4 : 2);
  if (bytes == 128) return append_as<8, false>(a, src, s);
  if (bytes == 256) return append_as<16, false>(a, src, s);
  return append_as<32, false>(a, src, s);
}

// ---- evict -----------------------------------------------------------------------------------------------------------

constexpr int EV_LDS_KEYS = 32768;  // keys of longer sequences lie in the workspace
constexpr int EV_LOADS = 8;         // entries per thread whose weights are under way together
constexpr uint32_t EV_STAYS = 0xffffffffu;

size_t paged_evict_keys_bytes(int n_seqs, int h_kv, int max_len) {
  return max_len <= EV_LDS_KEYS ? 0 : (size_t)n_seqs * h_kv * max_len * sizeof(uint32_t);
}

// Keys: 0 an entry on a missing page, EV_STAYS one of the first or last, else the weight's order kept between the two.
template <bool IN_LDS>
__global__ __launch_bounds__(SEL_THREADS) void evict_select_kernel(PagedArgs a, PagedEvict e) {
  extern __shared__ uint32_t lds_keys[];
  __shared__ SelectLds lds;
  __shared__ uint32_t wave_b[SEL_WAVES], wave_min[SEL_WAVES], wave_max[SEL_WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int s = blockIdx.x / a.h_kv, h = blockIdx.x - s * a.h_kv;
  const int n = paged_len_of(a, s);
  const int mask = (1 << a.page_shift) - 1;
  uint32_t* const keys = IN_LDS ? lds_keys : e.keys + ((size_t)s * a.h_kv + h) * a.max_len;
  const int32_t* const table = a.table + (size_t)s * a.table_pages;

  uint32_t kmin = 0xffffffffu, kmax = 0u, present = 0;
  for (int j0 = tid; j0 < n; j0 += EV_LOADS * SEL_THREADS) {
    int page[EV_LOADS];
    float w[EV_LOADS];
#pragma unroll
    for (int u = 0; u < EV_LOADS; ++u) page[u] = j0 + u * SEL_THREADS < n ? table[(j0 + u * SEL_THREADS) >> a.page_shift] : -1;
#pragma unroll
    for (int u = 0; u < EV_LOADS; ++u) {
      const bool ok = paged_page_ok(page[u], a.n_pages);
      w[u] = ok ? a.weight[paged_row(page[u], h, (j0 + u * SEL_THREADS) & mask, a.h_kv, a.page_shift)] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < EV_LOADS; ++u) {
      const int j = j0 + u * SEL_THREADS;
      if (j >= n) continue;
      uint32_t key = 0;
      if (paged_page_ok(page[u], a.n_pages)) {
        key = j < e.n_first || j >= n - e.n_last ? EV_STAYS : min(max(order_key(w[u]), 1u), EV_STAYS - 1);
        kmin = min(kmin, key);
        kmax = max(kmax, key);
        ++present;
      }
      keys[j] = key;
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    kmin = min(kmin, (uint32_t)__shfl_xor((int)kmin, o, 64));
    kmax = max(kmax, (uint32_t)__shfl_xor((int)kmax, o, 64));
    present += (uint32_t)__shfl_xor((int)present, o, 64);
  }
  if (lane == 0) {
    wave_min[wave] = kmin;
    wave_max[wave] = kmax;
    wave_b[wave] = present;
  }
  lds.hist[2 * tid] = 0;
  lds.hist[2 * tid + 1] = 0;
  if (tid == 0) lds.list_n = 0;
  __syncthreads();  // also orders the keys in the workspace: one workgroup wrote them and reads them
  uint32_t lo = 0xffffffffu, hi = 0u, total = 0;
#pragma unroll
  for (int w = 0; w < SEL_WAVES; ++w) {
    lo = min(lo, wave_min[w]);
    hi = max(hi, wave_max[w]);
    total += wave_b[w];
  }
  const uint32_t count = min(total, (uint32_t)e.keep);
  uint32_t thr = 0, need = 0;  // every present entry stays
  if (count < total) select_threshold([&](int j) { return keys[j]; }, n, lo, hi, count, lds, thr, need);

  // list: wavefront w owns a run of entries and walks it 64 at a time
  const int run = ((n + SEL_WAVES - 1) / SEL_WAVES + 63) / 64 * 64;
  const int j_begin = min(wave * run, n), j_end = min(j_begin + run, n);
  uint32_t gt = 0, eq = 0;
  for (int j0 = j_begin; j0 < j_end; j0 += 64) {
    const bool in = j0 + lane < j_end;
    const uint32_t key = in ? keys[j0 + lane] : 0u;
    gt += (uint32_t)__popcll(__ballot(in && key > thr));
    eq += (uint32_t)__popcll(__ballot(in && key == thr));
  }
  __syncthreads();  // wave_min / wave_max have been read
  if (lane == 0) {
    wave_min[wave] = gt;
    wave_max[wave] = eq;
  }
  __syncthreads();
  uint32_t gt_before = 0, eq_run = 0;
#pragma unroll
  for (int w = 0; w < SEL_WAVES; ++w) {
    gt_before += w < wave ? wave_min[w] : 0u;
    eq_run += w < wave ? wave_max[w] : 0u;
  }
  uint32_t slot0 = gt_before + min(eq_run, need);
  int32_t* const kept = e.kept + ((size_t)s * a.h_kv + h) * e.keep;
  const unsigned long long below = (1ull << lane) - 1ull;
  for (int j0 = j_begin; j0 < j_end; j0 += 64) {
    const bool in = j0 + lane < j_end;
    const uint32_t key = in ? keys[j0 + lane] : 0u;
    const bool is_eq = in && key == thr;
    const unsigned long long be = __ballot(is_eq);
    const bool keep_it = (in && key > thr) || (is_eq && eq_run + (uint32_t)__popcll(be & below) < need);
    const unsigned long long bs = __ballot(keep_it);
    const uint32_t slot = slot0 + (uint32_t)__popcll(bs & below);
    if (keep_it && slot < (uint32_t)e.keep) kept[slot] = j0 + lane;
    slot0 += (uint32_t)__popcll(bs);
    eq_run += (uint32_t)__popcll(be);
  }
  for (uint32_t x = count + tid; x < (uint32_t)e.keep; x += SEL_THREADS) kept[x] = -1;
  if (h == 0 && tid == 0) e.to_len[s] = (int)count;
}

constexpr int EM_THREADS = 256;
constexpr int EM_UNROLL = 4;  // rows per lane group whose loads are under way together
template <int LPR>            // lanes per row, 16 bytes each
__global__ __launch_bounds__(EM_THREADS) void evict_move_kernel(PagedArgs a, PagedEvict e, int blocks_per_head) {
  constexpr int ROWS = EM_THREADS / LPR;
  const int sh = blockIdx.x / blocks_per_head, b = blockIdx.x - sh * blocks_per_head;
  const int s = sh / a.h_kv, h = sh - s * a.h_kv;
  const int sub = threadIdx.x % LPR;
  const int mask = (1 << a.page_shift) - 1;
  const int32_t* const kept = e.kept + (size_t)sh * e.keep;
  const int x0 = b * (ROWS * EM_UNROLL) + threadIdx.x / LPR;
  int from[EM_UNROLL];
#pragma unroll
  for (int u = 0; u < EM_UNROLL; ++u) from[u] = x0 + u * ROWS < e.keep ? kept[x0 + u * ROWS] : -1;
  size_t src[EM_UNROLL], dst[EM_UNROLL];
#pragma unroll
  for (int u = 0; u < EM_UNROLL; ++u) {
    dst[u] = ~(size_t)0;
    if (from[u] < 0) continue;
    const int x = x0 + u * ROWS;
    const int p = a.table[(size_t)s * a.table_pages + (from[u] >> a.page_shift)];
    const int t = e.to_table[(size_t)s * e.to_pages + (x >> a.page_shift)];
    if (!paged_page_ok(p, a.n_pages) || !paged_page_ok(t, a.n_pages)) continue;  // no destination: the entry is dropped
    src[u] = paged_row(p, h, from[u] & mask, a.h_kv, a.page_shift);
    dst[u] = paged_row(t, h, x & mask, a.h_kv, a.page_shift);
  }
  u32x4 kk[EM_UNROLL], vv[EM_UNROLL];
  int pos[EM_UNROLL];
  float w[EM_UNROLL];
#pragma unroll
  for (int u = 0; u < EM_UNROLL; ++u) {
    if (dst[u] == ~(size_t)0) continue;
    kk[u] = *(const u32x4*)((const unsigned char*)a.k + src[u] * (LPR * 16) + sub * 16);
    vv[u] = *(const u32x4*)((const unsigned char*)a.v + src[u] * (LPR * 16) + sub * 16);
    if (sub == 0) {
      pos[u] = a.pos[src[u]];
      w[u] = a.weight[src[u]];
    }
  }
#pragma unroll
  for (int u = 0; u < EM_UNROLL; ++u) {
    if (dst[u] == ~(size_t)0) continue;
    *(u32x4*)((unsigned char*)a.k + dst[u] * (LPR * 16) + sub * 16) = kk[u];
    *(u32x4*)((unsigned char*)a.v + dst[u] * (LPR * 16) + sub * 16) = vv[u];
    if (sub == 0) {
      a.pos[dst[u]] = pos[u];
      a.weight[dst[u]] = w[u];
    }
  }
}

template <int LPR>
static bool move_as(const PagedArgs& a, const PagedEvict& e, hipStream_t s) {
  constexpr int ROWS = EM_THREADS / LPR * EM_UNROLL;
  const long long per = ((long long)e.keep + ROWS - 1) / ROWS;
  const long long heads = (long long)a.n_seqs * a.h_kv;
  if (per * heads * EM_THREADS > PAGED_MAX_THREADS || heads * SEL_THREADS > PAGED_MAX_THREADS) return false;
  const bool in_lds = a.max_len <= EV_LDS_KEYS;
  if (in_lds) {
    static bool attr_set[QP_MAX_DEVICES] = {};
    const int dev = current_device();
    if (dev < 0 || !attr_set[dev]) {
      (void)hipFuncSetAttribute((const void*)evict_select_kernel<true>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                EV_LDS_KEYS * (int)sizeof(uint32_t));
      if (dev >= 0) attr_set[dev] = true;
    }
    hipLaunchKernelGGL(evict_select_kernel<true>, dim3((unsigned)heads), dim3(SEL_THREADS), (size_t)a.max_len * sizeof(uint32_t), s,
                       a, e);
  } else {
    hipLaunchKernelGGL(evict_select_kernel<false>, dim3((unsigned)heads), dim3(SEL_THREADS), 0, s, a, e);
  }
  hipLaunchKernelGGL(evict_move_kernel<LPR>, dim3((unsigned)(per * heads)), dim3(EM_THREADS), 0, s, a, e, (int)per);
  return true;
}

bool launch_paged_evict(const PagedArgs& a, const PagedEvict& e, int row_bytes, hipStream_t s) {
  return row_bytes == 128 ? move_as<8>(a, e, s) : row_bytes == 256 ? move_as<16>(a, e, s) : move_as<32>(a, e, s);
}

}  // namespace qp

// The paged cache's entries on their way: new rows stored in pages, and the entries of most weight moved to other pages.
//
// append   a copy: row r of head h -> its sequence's entry. Bound by HBM (2 rows in, 2 rows out per token and head) from a few
//          thousand rows on, by the launch below.
// evict    two launches. evict_select_kernel: one workgroup per (sequence, head) finds the threshold among order-preserving keys
//          (select_threshold) and lists the entries that stay, in order. evict_move_kernel: many workgroups copy the listed rows,
//          which is where the bytes are (4 rows of head_dim per kept entry against 4 bytes per entry for the selection).
#include "codes.h"
#include "paged.h"
#include "select.h"

#include <algorithm>

namespace qp {

// ---- append ----------------------------------------------------------------------------------------------------------

// pack8_e4m3's codes from the conversion instruction, which rounds to nearest even but does not saturate: clamped first, by minima and
// maxima that keep NaN. Some 35 instructions for 16 bytes, in integer arithmetic some 160: what an hour-long video left (46,125 entries
// of 8 heads) went into 8-bit pages in 82 us with those.
__device__ __forceinline__ unsigned convert_e4m3(unsigned pair, unsigned old, bool high) {
  const float x = __builtin_elementwise_minimum(__builtin_elementwise_maximum(bf16lo_to_f32(pair), -448.f), 448.f);
  const float y = __builtin_elementwise_minimum(__builtin_elementwise_maximum(bf16hi_to_f32(pair), -448.f), 448.f);
  return high ? (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(x, y, (int)old, true) : (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(x, y, (int)old, false);
}
__device__ __forceinline__ uint2 convert8_e4m3(const u32x4& b) {
  const uint2 r = make_uint2(convert_e4m3(b.y, convert_e4m3(b.x, 0u, false), true), convert_e4m3(b.w, convert_e4m3(b.z, 0u, false), true));
  // a code of seven ones is NaN, whose sign the instruction does not keep
  const unsigned nan = (((r.x & 0x7f7f7f7fu) + 0x01010101u) | ((r.y & 0x7f7f7f7fu) + 0x01010101u)) & 0x80808080u;
  return nan ? pack8_e4m3(b) : r;
}

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
      *(uint2*)((unsigned char*)a.k + at) = convert8_e4m3(kk[u]);
      *(uint2*)((unsigned char*)a.v + at) = convert8_e4m3(vv[u]);
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

// Keys of a (sequence, head): 0 an entry on a missing page (or none), EV_STAYS one of the first or last, else the weight's order, kept
// between the two. A thread takes four neighbours of a block of 4096: one page number and one load for the four.
constexpr uint32_t EV_STAYS = 0xffffffffu;
constexpr int EV_BLOCK = 4 * SEL_THREADS;
// Blocks whose keys the workgroup holds for itself; those of longer sequences lie in the workspace. us of a call held / by way of the
// workspace, 4 heads, a third kept: 3,000 entries 18.0 / 16.1, 9,840 22.1 / 21.9, 20,000 29.0 / 30.1, 46,125 48.0 / 57.6, 49,000 49.7 /
// 58.8; 16 sequences of 8 heads of up to 8,300 138.9 / 135.7. 60,000 entries, in the workspace, 67.5.
constexpr int EV_HELD = 12;

size_t paged_evict_keys_bytes(int n_seqs, int h_kv, int max_len) {
  const size_t blocks = ((size_t)max_len + EV_BLOCK - 1) / EV_BLOCK;
  return blocks <= EV_HELD ? 0 : (size_t)n_seqs * h_kv * blocks * EV_BLOCK * sizeof(uint32_t);
}

// One workgroup has a head to itself, so an instruction per entry costs time: 46,125 of them 0.3 us. us for 16,384 kept of
// 46,125 entries of 4 heads, one entry per thread and step, keys in the workspace 75, in LDS and registers 59; weights made into
// dense keys by a launch of their own 6 and 25. The search has HELD's keys in registers; the loop that writes the list is left rolled by
// the compiler and reads them back from scratch memory (208 bytes per thread), a block at a time.
template <bool HELD>
__global__ __launch_bounds__(SEL_THREADS) void evict_select_kernel(PagedArgs a, PagedEvict e) {
  __shared__ SelectLds lds;
  __shared__ uint32_t red[4][SEL_WAVES];
  constexpr int RUNS = HELD ? EV_HELD : 1;  // blocks whose wavefronts' counts are there at a time
  __shared__ __attribute__((aligned(16))) uint32_t run_gt[RUNS][SEL_WAVES], run_eq[RUNS][SEL_WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int sh = blockIdx.x, s = sh / a.h_kv, h = sh - s * a.h_kv;
  const int n = paged_len_of(a, s);
  const int mask = (1 << a.page_shift) - 1;
  const int32_t* const table = a.table + (size_t)s * a.table_pages;
  const int used = (n + EV_BLOCK - 1) / EV_BLOCK;
  uint32_t* const far = HELD ? nullptr : e.keys + (size_t)sh * (((size_t)a.max_len + EV_BLOCK - 1) / EV_BLOCK * EV_BLOCK);

  uint32_t v[4] = {0xffffffffu, 0u, 0u, 0u};  // smallest and largest key of those that compete, entries present, entries that stay
  auto load_page = [&](int u) { return u * EV_BLOCK + 4 * tid < n ? table[(u * EV_BLOCK + 4 * tid) >> a.page_shift] : -1; };
  auto load_weights = [&](int u, int page) {
    const int j = u * EV_BLOCK + 4 * tid;
    return paged_page_ok(page, a.n_pages) ? *(const float4*)(a.weight + paged_row(page, h, j & mask, a.h_kv, a.page_shift))
                                          : make_float4(0.f, 0.f, 0.f, 0.f);
  };
  auto key_of = [&](float w, int j, bool here) {
    if (!here || j >= n) return 0u;
    ++v[2];
    if (j < e.n_first || j >= n - e.n_last) {
      ++v[3];
      return EV_STAYS;
    }
    const uint32_t key = min(max(order_key(w), 1u), EV_STAYS - 1);
    v[0] = min(v[0], key);
    v[1] = max(v[1], key);
    return key;
  };
  auto keys_of = [&](int u, int page, const float4& w) {
    const int j = u * EV_BLOCK + 4 * tid;
    const bool here = paged_page_ok(page, a.n_pages);
    return make_uint4(key_of(w.x, j, here), key_of(w.y, j + 1, here), key_of(w.z, j + 2, here), key_of(w.w, j + 3, here));
  };
  uint4 held[HELD ? EV_HELD : 1];
  if constexpr (HELD) {
    int page[EV_HELD];
#pragma unroll
    for (int u = 0; u < EV_HELD; ++u) page[u] = load_page(u);
#pragma unroll
    for (int u0 = 0; u0 < EV_HELD; u0 += 6) {
      float4 w[6];
#pragma unroll
      for (int u = 0; u < 6; ++u) w[u] = load_weights(u0 + u, page[u0 + u]);
#pragma unroll
      for (int u = 0; u < 6; ++u) held[u0 + u] = keys_of(u0 + u, page[u0 + u], w[u]);
      __builtin_amdgcn_sched_barrier(0);  // or the second half's loads come first and push keys out of the registers
    }
  } else {
    for (int u0 = 0; u0 < used; u0 += 4) {
      int page[4];
      float4 w[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) page[u] = load_page(u0 + u);
#pragma unroll
      for (int u = 0; u < 4; ++u) w[u] = load_weights(u0 + u, page[u]);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (u0 + u < used) *(uint4*)(far + (size_t)(u0 + u) * EV_BLOCK + 4 * tid) = keys_of(u0 + u, page[u], w[u]);
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    v[0] = min(v[0], (uint32_t)__shfl_xor((int)v[0], o, 64));
    v[1] = max(v[1], (uint32_t)__shfl_xor((int)v[1], o, 64));
    v[2] += (uint32_t)__shfl_xor((int)v[2], o, 64);
    v[3] += (uint32_t)__shfl_xor((int)v[3], o, 64);
  }
  if (lane == 0) red[0][wave] = v[0], red[1][wave] = v[1], red[2][wave] = v[2], red[3][wave] = v[3];
  lds.hist[2 * tid] = 0;
  lds.hist[2 * tid + 1] = 0;
  if (tid == 0) lds.list_n = 0;
  __syncthreads();  // every thread reads the keys in the workspace that it wrote itself
  uint32_t lo = 0xffffffffu, hi = 0u, total = 0, stays = 0;
#pragma unroll
  for (int w = 0; w < SEL_WAVES; ++w) {
    lo = min(lo, red[0][w]);
    hi = max(hi, red[1][w]);
    total += red[2][w];
    stays += red[3][w];
  }
  auto key4 = [&](int u) { return u < used ? *(const uint4*)(far + (size_t)u * EV_BLOCK + 4 * tid) : make_uint4(0u, 0u, 0u, 0u); };
  auto each = [&](auto f) {
    if constexpr (HELD) {
#pragma unroll
      for (int u = 0; u < EV_HELD; ++u)
        if (u < used) f(held[u].x, true), f(held[u].y, true), f(held[u].z, true), f(held[u].w, true);
    } else {
      for (int u0 = 0; u0 < used; u0 += 8) {
        uint4 k[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) k[u] = key4(u0 + u);
#pragma unroll
        for (int u = 0; u < 8; ++u) f(k[u].x, true), f(k[u].y, true), f(k[u].z, true), f(k[u].w, true);
      }
    }
  };
  const uint32_t count = min(total, (uint32_t)e.keep);
  uint32_t thr = 0, need = 0;  // every present entry stays
  if (count < total) {
    thr = EV_STAYS - 1;        // only those that stay in any case
    if (count > stays) {       // and the largest of the others, whose keys alone the search spreads over its buckets
      bool many_low = true;
      if constexpr (HELD) {    // one in eight of a sample
        uint32_t low = 0;
#pragma unroll
        for (int u = 0; u < EV_HELD; ++u) low += (uint32_t)__popcll(__ballot(held[u].x == lo));
        many_low = low >= 8u * (uint32_t)used;
      }
      select_threshold<false>(each, each, lo, hi, count - stays, lds, thr, need, many_low);
    }
  }

  // The list, in order: an entry above the threshold stays, one equal to it if fewer than `need` of those lie before it, and its
  // slot is the number of survivors before it, gt + min(eq, need) of the keys above and equal there.
  int32_t* const kept = e.kept + (size_t)sh * e.keep;
  const unsigned long long below = (1ull << lane) - 1ull;
  auto tally = [&](const uint4& k, int r) {
    const uint32_t x = (uint32_t)(__popcll(__ballot(k.x > thr)) + __popcll(__ballot(k.y > thr)) + __popcll(__ballot(k.z > thr)) + __popcll(__ballot(k.w > thr)));
    const uint32_t y = (uint32_t)(__popcll(__ballot(k.x == thr)) + __popcll(__ballot(k.y == thr)) + __popcll(__ballot(k.z == thr)) + __popcll(__ballot(k.w == thr)));
    if (lane == 0) run_gt[r][wave] = x, run_eq[r][wave] = y;
  };
  auto emit = [&](const uint4& k, int j, uint32_t gt, uint32_t eq) {  // gt, eq: before this wavefront's run
    const uint32_t key[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      gt += (uint32_t)__popcll(__ballot(key[c] > thr) & below);
      eq += (uint32_t)__popcll(__ballot(key[c] == thr) & below);
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint32_t slot = gt + min(eq, need);
      if ((key[c] > thr || (key[c] == thr && eq < need)) && slot < (uint32_t)e.keep) kept[slot] = j + c;
      gt += key[c] > thr;
      eq += key[c] == thr;
    }
  };
  uint32_t gt = 0, eq = 0;  // before the block
  auto block = [&](const uint4& k, int u, int r) {
    uint32_t gt_w = gt, eq_w = eq;
#pragma unroll
    for (int w = 0; w < SEL_WAVES; w += 4) {
      const uint4 x = *(const uint4*)&run_gt[r][w], y = *(const uint4*)&run_eq[r][w];
      gt_w += (w < wave ? x.x : 0u) + (w + 1 < wave ? x.y : 0u) + (w + 2 < wave ? x.z : 0u) + (w + 3 < wave ? x.w : 0u);
      eq_w += (w < wave ? y.x : 0u) + (w + 1 < wave ? y.y : 0u) + (w + 2 < wave ? y.z : 0u) + (w + 3 < wave ? y.w : 0u);
      gt += x.x + x.y + x.z + x.w;
      eq += y.x + y.y + y.z + y.w;
    }
    emit(k, u * EV_BLOCK + 4 * tid, gt_w, eq_w);
  };
  if constexpr (HELD) {
#pragma unroll
    for (int u = 0; u < EV_HELD; ++u) {
      if (u < used) tally(held[u], u);
      else if (lane == 0) run_gt[u][wave] = run_eq[u][wave] = 0;
    }
    __syncthreads();
    // the first wavefront turns the runs' counts, in order, into what lies before each
    static_assert(EV_HELD * SEL_WAVES == 3 * 64, "three runs per lane");
    if (wave == 0) {
      uint32_t* const g = &run_gt[0][0] + 3 * lane;
      uint32_t* const q = &run_eq[0][0] + 3 * lane;
      const uint32_t g0 = g[0], g1 = g[1], g2 = g[2], q0 = q[0], q1 = q[1], q2 = q[2];
      uint32_t gs = g0 + g1 + g2, qs = q0 + q1 + q2;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t x = __shfl_up(gs, o, 64), y = __shfl_up(qs, o, 64);
        if (lane >= o) gs += x, qs += y;
      }
      if (lane == 63) red[0][0] = qs;
      gs -= g0 + g1 + g2;
      qs -= q0 + q1 + q2;
      g[0] = gs, g[1] = gs + g0, g[2] = gs + g0 + g1;
      q[0] = qs, q[1] = qs + q0, q[2] = qs + q0 + q1;
    }
    __syncthreads();
    // Nearly always all keys equal to the threshold stay, or none: then nobody asks which of them.
    const bool alike = need == 0 || red[0][0] == need;
#pragma unroll
    for (int u = 0; u < EV_HELD; ++u) {
      if (u >= used) break;
      const uint32_t gt_run = run_gt[u][wave], eq_run = run_eq[u][wave];
      const int j = u * EV_BLOCK + 4 * tid;
      if (!alike) {
        emit(held[u], j, gt_run, eq_run);
        continue;
      }
      const uint32_t key[4] = {held[u].x, held[u].y, held[u].z, held[u].w};
      uint32_t slot = gt_run + (need > 0 ? eq_run : 0u);
      const uint32_t least = need > 0 ? thr : thr + 1;  // thr < EV_STAYS; key 0 never stays
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const unsigned long long m = __ballot(key[c] >= least);
        slot = __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, slot));
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const bool stay = key[c] >= least;
        if (stay && slot < (uint32_t)e.keep) kept[slot] = j + c;
        slot += stay;
      }
    }
  } else {
    for (int u = 0; u < used; ++u) {
      const uint4 k = key4(u);
      __syncthreads();  // the counts of the block before have been read
      tally(k, 0);
      __syncthreads();
      block(k, u, 0);
    }
  }
  for (uint32_t x = count + tid; x < (uint32_t)e.keep; x += SEL_THREADS) kept[x] = -1;
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
  if (h == 0 && sub == 0) {
    // the new length is where the list ends: written here, since the heads' selections read the old one, which may be the same array
#pragma unroll
    for (int u = 0; u < EM_UNROLL; ++u) {
      const int x = x0 + u * ROWS;
      if (x >= e.keep) continue;
      if (from[u] < 0 && (x == 0 || kept[x - 1] >= 0)) e.to_len[s] = x;
      if (from[u] >= 0 && x == e.keep - 1) e.to_len[s] = e.keep;
    }
  }
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

// The move into a pool with scales: a wavefront has a block of 16 of the kept entries, which share scales that fit all of them: the largest of
// their old ones. 8 lanes have a row. Sixteen sequences of the 72B heads back to 4,096 entries 83.5 us, one of 46,125 of the 7B heads to 16,384 42.8;
// without scales 84.1 and 42.3.
__global__ __launch_bounds__(EM_THREADS) void evict_move_scaled_kernel(PagedArgs a, PagedEvict e, int blocks_per_head) {
  constexpr int NW = EM_THREADS / 64, LPR = 8, PASSES = 2;
  const int lane = threadIdx.x & 63, sub = lane % LPR;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int sh = blockIdx.x / blocks_per_head, b = (blockIdx.x - sh * blocks_per_head) * NW + wave;
  const int s = sh / a.h_kv, h = sh - s * a.h_kv;
  const int mask = (1 << a.page_shift) - 1;
  const int32_t* const kept = e.kept + (size_t)sh * e.keep;
  const long long x0 = (long long)b * PAGED_BLOCK;
  if (x0 >= e.keep) return;
  const int first = (int)x0, t = e.to_table[(size_t)s * e.to_pages + (first >> a.page_shift)];
  const bool there = paged_page_ok(t, a.n_pages);  // no destination: the entries are dropped
  const size_t to = paged_row(there ? t : 0, h, first & mask, a.h_kv, a.page_shift);
  int from[PASSES], ke = PAGED_SCALE_MIN, ve = PAGED_SCALE_MIN, k_exp[PASSES], v_exp[PASSES], pos[PASSES];
  float w[PASSES];
  u32x4 kk[PASSES], vv[PASSES];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int x = first + p * (64 / LPR) + lane / LPR;
    from[p] = x < e.keep ? kept[x] : -1;
    if (h == 0 && sub == 0 && x < e.keep) {  // the new length is where the list ends, as in evict_move_kernel
      if (from[p] < 0 && (x == 0 || kept[x - 1] >= 0)) e.to_len[s] = x;
      if (from[p] >= 0 && x == e.keep - 1) e.to_len[s] = e.keep;
    }
    if (from[p] < 0) continue;
    const int page = a.table[(size_t)s * a.table_pages + (from[p] >> a.page_shift)];
    if (!there || !paged_page_ok(page, a.n_pages)) {
      from[p] = -1;
      continue;
    }
    const size_t row = paged_row(page, h, from[p] & mask, a.h_kv, a.page_shift);
    kk[p] = *(const u32x4*)((const unsigned char*)a.k + row * (LPR * 16) + sub * 16);
    vv[p] = *(const u32x4*)((const unsigned char*)a.v + row * (LPR * 16) + sub * 16);
    k_exp[p] = scale_exponent(a.k_scale[row >> 4], PAGED_SCALE_MIN, PAGED_SCALE_MAX);
    v_exp[p] = scale_exponent(a.v_scale[row >> 4], PAGED_SCALE_MIN, PAGED_SCALE_MAX);
    ke = max(ke, k_exp[p]);
    ve = max(ve, v_exp[p]);
    if (sub == 0) {
      pos[p] = a.pos[row];
      w[p] = a.weight[row];
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    ke = max(ke, __shfl_xor(ke, o, 64));
    ve = max(ve, __shfl_xor(ve, o, 64));
  }
  if (!__any(from[0] >= 0 || from[1] >= 0)) return;
  if (lane == 0) {
    a.k_scale[to >> 4] = pow2f(ke);
    a.v_scale[to >> 4] = pow2f(ve);
  }
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    if (from[p] < 0) continue;
    const size_t row = to + p * (64 / LPR) + lane / LPR;
    const float kb = pow2f(max(k_exp[p] - ke, -126)), vb = pow2f(max(v_exp[p] - ve, -126));
    if (k_exp[p] < ke) {
#pragma unroll
      for (int c = 0; c < 4; ++c) kk[p][c] = shrink4(kk[p][c], kb);
    }
    if (v_exp[p] < ve) {
#pragma unroll
      for (int c = 0; c < 4; ++c) vv[p][c] = shrink4(vv[p][c], vb);
    }
    *(u32x4*)((unsigned char*)a.k + row * (LPR * 16) + sub * 16) = kk[p];
    *(u32x4*)((unsigned char*)a.v + row * (LPR * 16) + sub * 16) = vv[p];
    if (sub == 0) {
      a.pos[row] = pos[p];
      a.weight[row] = w[p];
    }
  }
}

template <int LPR>
static bool evict_as(const PagedArgs& a, const PagedEvict& e, hipStream_t s) {
  constexpr int ROWS = EM_THREADS / LPR * EM_UNROLL;
  const bool scaled = a.fp8 == QP_CACHE_FP8_E4M3_SCALED;
  const int rows = scaled ? EM_THREADS / 64 * PAGED_BLOCK : ROWS;
  const long long per = ((long long)e.keep + rows - 1) / rows;
  const long long heads = (long long)a.n_seqs * a.h_kv;
  if (per * heads * EM_THREADS > PAGED_MAX_THREADS || heads * SEL_THREADS > PAGED_MAX_THREADS) return false;
  const dim3 grid((unsigned)heads), block(SEL_THREADS);
  if (e.keys == nullptr) hipLaunchKernelGGL(evict_select_kernel<true>, grid, block, 0, s, a, e);
  else hipLaunchKernelGGL(evict_select_kernel<false>, grid, block, 0, s, a, e);
  if (scaled) hipLaunchKernelGGL(evict_move_scaled_kernel, dim3((unsigned)(per * heads)), dim3(EM_THREADS), 0, s, a, e, (int)per);
  else hipLaunchKernelGGL(evict_move_kernel<LPR>, dim3((unsigned)(per * heads)), dim3(EM_THREADS), 0, s, a, e, (int)per);
  return true;
}

bool launch_paged_evict(const PagedArgs& a, const PagedEvict& e, int row_bytes, hipStream_t s) {
  return row_bytes == 128 ? evict_as<8>(a, e, s) : row_bytes == 256 ? evict_as<16>(a, e, s) : evict_as<32>(a, e, s);
}

}  // namespace qp

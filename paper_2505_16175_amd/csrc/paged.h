// The paged cache's batch and pool as its kernels see them, and the arithmetic that keeps them inside: what the host cannot
// check (lengths, row numbers, page numbers are device values) is clamped here, in functions that run on the host too.
#pragma once
#include "qp_internal.h"
#include "qp_paged.h"

namespace qp {

struct PagedArgs {
  void* k;         // [n_pages][h_kv][1 << page_shift][d]
  void* v;
  int32_t* pos;    // [n_pages][h_kv][1 << page_shift]
  float* weight;
  const int32_t* table;      // [n_seqs][table_pages]
  const int32_t* len;        // [n_seqs]
  const int32_t* row_start;  // [n_seqs + 1]
  int n_pages, page_shift;
  int fp8;         // 1: the pool holds one E4M3 byte per element
  int n_seqs, table_pages, n_rows, max_new, max_len;
  int h_q, h_kv;
  float scale_log2;  // softmax scale * log2(e)
};

// One sequence of a batch: row i of its n new ones (from row0) sees the entries j <= base + i, j < len.
struct PagedSeq {
  int len, row0, n, base;
};
__host__ __device__ inline int paged_clamp(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }
// len, r0, r1: what the device arrays say. The table's end is limited to what an int holds.
__host__ __device__ inline PagedSeq paged_seq(int len, int r0, int r1, int n_rows, int max_new, int max_len, int table_pages,
                                              int page_shift) {
  const long long room = (long long)table_pages << page_shift;
  PagedSeq q;
  q.len = paged_clamp(len, 0, room < max_len ? (int)room : max_len);
  q.row0 = paged_clamp(r0, 0, n_rows);
  const int n = paged_clamp(r1, q.row0, n_rows) - q.row0;
  q.base = q.len - n;  // of all its new tokens, also those beyond max_new
  q.n = n < max_new ? n : max_new;
  return q;
}
__host__ __device__ inline bool paged_page_ok(int page, int n_pages) { return (unsigned)page < (unsigned)n_pages; }
// Row (of d elements, or one value) of entry `slot` of `page`, KV head h.
__host__ __device__ inline size_t paged_row(int page, int h, int slot, int h_kv, int page_shift) {
  return (((size_t)page * h_kv + h) << page_shift) + slot;
}

__device__ __forceinline__ PagedSeq paged_seq_of(const PagedArgs& a, int s) {
  return paged_seq(a.len[s], a.row_start[s], a.row_start[s + 1], a.n_rows, a.max_new, a.max_len, a.table_pages, a.page_shift);
}
__device__ __forceinline__ int paged_len_of(const PagedArgs& a, int s) {
  return paged_seq(a.len[s], 0, 0, 0, 0, a.max_len, a.table_pages, a.page_shift).len;
}

// Most workgroups of one launch: the runtime takes fewer than 2^32 threads.
constexpr long long PAGED_MAX_THREADS = 0xffffffffll;

struct PagedAppend {
  const void* k;
  const void* v;
  const int32_t* pos;
  long long token_stride, head_stride;  // bytes
  long long pos_token_stride, pos_head_stride;
  int raw;  // 1: the rows are E4M3 bytes already
};
bool launch_paged_append(const PagedArgs& a, const PagedAppend& src, int dtype, int d, hipStream_t s);

struct PagedPlan {
  int tile_rows, tiles;    // stacked rows per workgroup, tiles of max_new tokens
  int chunks, chunk_keys;  // tile kernel: key chunks of a sequence
  int shares;              // few rows: workgroups of a KV head among which all entries are dealt, 0: one per tile
  long long workgroups;
  size_t scratch_bytes;
};
PagedPlan plan_paged_attend(const PagedArgs& a, int dtype, int d, size_t scratch_bytes);
constexpr size_t PAGED_ATTEND_SCRATCH = (size_t)128 << 20;  // partial results take no more
// The tile kernel of attend_mfma.hip: 256 stacked rows per workgroup, keys in tiles of 64.
constexpr int PT_ROWS = 256;
long long paged_tile_blocks(const PagedArgs& a, const PagedPlan& p);  // workgroups, the padding of the XCD mapping included
void launch_paged_tiles(const PagedArgs& a, const PagedPlan& p, const void* q, void* out, float* lse, float* part_o, float* part_lse,
                        hipStream_t s);
bool launch_paged_attend(const PagedArgs& a, int dtype, int d, const void* q, void* out, float* lse, void* scratch,
                         size_t scratch_bytes, hipStream_t s);

size_t paged_weigh_workspace_bytes(int n_seqs, int h_q, int h_kv, int max_new, int max_len);
bool launch_paged_weigh(const PagedArgs& a, int dtype, int d, const void* q, const float* lse, int accumulate, void* scratch,
                        size_t scratch_bytes, hipStream_t s);

struct PagedEvict {
  int keep, n_first, n_last;
  const int32_t* to_table;
  int to_pages;
  int32_t* to_len;
  int32_t* kept;      // [n_seqs][h_kv][keep], the caller's or in the workspace
  uint32_t* keys;     // workspace of paged_evict_keys_bytes, nullptr where that is 0
};
size_t paged_evict_keys_bytes(int n_seqs, int h_kv, int max_len);  // 0 where a workgroup holds a head's keys
bool launch_paged_evict(const PagedArgs& a, const PagedEvict& e, int row_bytes, hipStream_t s);

}  // namespace qp

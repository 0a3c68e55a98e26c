// C-ABI entry points of the paged cache (qp_paged.h): validation, workspace carving, launches. Host code only.
#include <math.h>
#include <string.h>

#include "paged.h"

namespace {

inline bool aligned(const void* p, unsigned to) { return p != nullptr && (((uintptr_t)p) & (to - 1)) == 0; }
inline size_t round256(size_t x) { return (x + 255) / 256 * 256; }
constexpr int kMaxLen = 1 << 30;  // entries of a sequence, rows of a call: sums of two of them fit 32 bits

qp_status finish(bool launched) {
  if (!launched) return QP_ERR_UNSUPPORTED;  // more workgroups than a launch takes
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) {
    qp::note_hip_error((int)e);
    return QP_ERR_HIP;
  }
  return QP_OK;
}

qp_status check_layout(const qp_layout* L) {
  if (L == nullptr || L->n_q_heads <= 0 || L->n_kv_heads <= 0 || L->head_dim <= 0) return QP_ERR_INVALID_ARG;
  if (L->n_q_heads % L->n_kv_heads != 0 || (L->dtype != QP_F32 && L->dtype != QP_BF16)) return QP_ERR_INVALID_ARG;
  if (!(L->softmax_scale >= 0.f) || isinf(L->softmax_scale)) return QP_ERR_INVALID_ARG;
  if ((L->head_dim != 64 && L->head_dim != 128) || L->n_q_heads > 65535) return QP_ERR_UNSUPPORTED;
  return QP_OK;
}

qp_status check_sizes(int32_t n_seqs, int32_t n_rows, int32_t max_new, int32_t max_len) {
  if (n_seqs <= 0 || n_rows < 0 || max_new < 0 || max_len <= 0) return QP_ERR_INVALID_ARG;
  if (max_len > kMaxLen || n_rows > kMaxLen || max_new > kMaxLen || n_seqs > (1 << 20)) return QP_ERR_UNSUPPORTED;
  return QP_OK;
}

// Everything that does not depend on the call; rows: the call has new tokens.
qp_status check(const qp_layout* L, const qp_paged_cache* c, const qp_paged_batch* b, bool rows, qp::PagedArgs* a) {
  qp_status st = check_layout(L);
  if (st != QP_OK) return st;
  if (c == nullptr || b == nullptr) return QP_ERR_INVALID_ARG;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->pos, 4) || (c->weight != nullptr && !aligned(c->weight, 16)))
    return QP_ERR_INVALID_ARG;
  if (c->n_pages <= 0 || c->format < QP_CACHE_SAME || c->format > QP_CACHE_FP8_E4M3_SCALED) return QP_ERR_INVALID_ARG;
  const bool scaled = c->format == QP_CACHE_FP8_E4M3_SCALED;
  if (scaled && (!aligned(c->k_scale, 4) || !aligned(c->v_scale, 4))) return QP_ERR_INVALID_ARG;
  if (c->format != QP_CACHE_SAME && (L->dtype != QP_BF16 || L->head_dim != 128)) return QP_ERR_UNSUPPORTED;
  int shift = 4;
  while (shift < 8 && (1 << shift) != c->page_tokens) ++shift;
  if ((1 << shift) != c->page_tokens) return c->page_tokens <= 0 ? QP_ERR_INVALID_ARG : QP_ERR_UNSUPPORTED;
  if ((st = check_sizes(b->n_seqs, rows ? b->n_rows : 0, rows ? b->max_new : 0, b->max_len)) != QP_OK) return st;
  if (!aligned(b->page_table, 4) || !aligned(b->len, 4) || b->table_pages <= 0) return QP_ERR_INVALID_ARG;
  if (rows && (!aligned(b->row_start, 4) || b->n_rows == 0 || b->max_new == 0)) return QP_ERR_INVALID_ARG;
  memset(a, 0, sizeof(*a));
  a->k = c->k, a->v = c->v, a->pos = c->pos, a->weight = c->weight;
  a->table = b->page_table, a->len = b->len, a->row_start = b->row_start;
  a->n_pages = c->n_pages, a->page_shift = shift, a->fp8 = c->format;
  if (scaled) a->k_scale = c->k_scale, a->v_scale = c->v_scale;
  a->n_seqs = b->n_seqs, a->table_pages = b->table_pages;
  a->n_rows = rows ? b->n_rows : 0;
  a->max_new = rows ? (b->max_new < b->n_rows ? b->max_new : b->n_rows) : 0;
  a->max_len = b->max_len;
  a->h_q = L->n_q_heads, a->h_kv = L->n_kv_heads;
  const float scale = L->softmax_scale > 0.f ? L->softmax_scale : 1.0f / sqrtf((float)L->head_dim);
  a->scale_log2 = scale * 1.4426950408889634f;
  return QP_OK;
}

// Workspace of qp_paged_evict: [kept entries][keys of long sequences]
size_t evict_kept_bytes(int32_t n_seqs, int32_t h_kv, int32_t keep) { return round256((size_t)n_seqs * h_kv * keep * sizeof(int32_t)); }
size_t evict_bytes(int32_t n_seqs, int32_t h_kv, int32_t keep, int32_t max_len) {
  return evict_kept_bytes(n_seqs, h_kv, keep) + round256(qp::paged_evict_keys_bytes(n_seqs, h_kv, max_len));
}

// A source's strides in elements of `size` bytes, and those of its positions.
constexpr int64_t kMostStride = (int64_t)1 << 40;
qp_status check_strides(int64_t token_stride, int64_t head_stride, int64_t size) {
  if (token_stride < 0 || head_stride < 0) return QP_ERR_INVALID_ARG;
  if (token_stride > kMostStride || head_stride > kMostStride) return QP_ERR_UNSUPPORTED;
  return token_stride * size % 16 != 0 || head_stride * size % 16 != 0 ? QP_ERR_INVALID_ARG : QP_OK;
}
qp_status check_pos_strides(int64_t token_stride, int64_t head_stride) {
  if (token_stride < 0 || head_stride < 0) return QP_ERR_INVALID_ARG;
  return token_stride > kMostStride || head_stride > kMostStride ? QP_ERR_UNSUPPORTED : QP_OK;
}

bool bad_workspace(const void* p) { return p != nullptr && (((uintptr_t)p) & 255u) != 0; }

}  // namespace

extern "C" {

size_t qp_paged_workspace_bytes(const qp_layout* L, int32_t n_seqs, int32_t n_rows, int32_t max_new, int32_t max_len,
                                int32_t keep) {
  if (check_layout(L) != QP_OK || check_sizes(n_seqs, n_rows, max_new, max_len) != QP_OK || keep < 0 || keep > kMaxLen) return 0;
  size_t most = 256;
  if (n_rows > 0 && max_new > 0) {
    qp::PagedArgs a{};
    a.n_seqs = n_seqs, a.n_rows = n_rows, a.max_new = max_new < n_rows ? max_new : n_rows, a.max_len = max_len;
    a.h_q = L->n_q_heads, a.h_kv = L->n_kv_heads, a.page_shift = 8;
    size_t attend = 0;  // over a pool of either format
    for (a.fp8 = 0; a.fp8 < 2; ++a.fp8) {
      const size_t x = qp::plan_paged_attend(a, L->dtype, L->head_dim, qp::PAGED_ATTEND_SCRATCH).scratch_bytes;
      attend = x > attend ? x : attend;
    }
    const size_t weigh = qp::paged_weigh_workspace_bytes(n_seqs, a.h_q, a.h_kv, a.max_new, max_len);
    most = attend > most ? attend : most;
    most = weigh > most ? weigh : most;
  }
  if (keep > 0) {
    const size_t evict = evict_bytes(n_seqs, L->n_kv_heads, keep, max_len);
    most = evict > most ? evict : most;
  }
  return round256(most);
}

qp_status qp_paged_append(const qp_layout* L, const qp_paged_cache* cache, const qp_paged_batch* batch, const void* k,
                          const void* v, int64_t token_stride, int64_t head_stride, const int32_t* pos,
                          int64_t pos_token_stride, int64_t pos_head_stride, qp_cache_format source_format, void* hip_stream) {
  qp::PagedArgs a;
  const qp_status st = check(L, cache, batch, true, &a);
  if (st != QP_OK) return st;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(pos, 4)) return QP_ERR_INVALID_ARG;
  if (source_format != QP_CACHE_SAME && source_format != QP_CACHE_FP8_E4M3) return QP_ERR_INVALID_ARG;
  const bool raw = source_format == QP_CACHE_FP8_E4M3;
  if (raw && !a.fp8) return QP_ERR_UNSUPPORTED;
  if (raw && a.fp8 == QP_CACHE_FP8_E4M3_SCALED) return QP_ERR_UNSUPPORTED;
  const int64_t size = raw ? 1 : L->dtype == QP_F32 ? 4 : 2;
  qp_status stride = check_pos_strides(pos_token_stride, pos_head_stride);
  if (stride == QP_ERR_INVALID_ARG || token_stride < 0 || head_stride < 0) return QP_ERR_INVALID_ARG;
  if (stride == QP_OK) stride = check_strides(token_stride, head_stride, size);
  if (stride != QP_OK) return stride;
  if (a.fp8 == QP_CACHE_FP8_E4M3_SCALED) {
    qp::PagedStore store{};
    store.k = k, store.v = v, store.token_stride = token_stride * size, store.head_stride = head_stride * size;
    store.pos = pos, store.pos_token_stride = pos_token_stride, store.pos_head_stride = pos_head_stride;
    return finish(qp::launch_paged_store(a, store, L->dtype, L->head_dim, (hipStream_t)hip_stream));
  }
  const qp::PagedAppend src{k, v, pos, token_stride * size, head_stride * size, pos_token_stride, pos_head_stride, raw};
  return finish(qp::launch_paged_append(a, src, L->dtype, L->head_dim, (hipStream_t)hip_stream));
}

qp_status qp_paged_append_rope(const qp_layout* L, const qp_paged_cache* cache, const qp_paged_batch* batch, const qp_paged_rope* rope,
                               const void* q_or_null, int64_t q_token_stride, int64_t q_head_stride, const void* k, const void* v,
                               int64_t token_stride, int64_t head_stride, const int32_t* pos, int64_t pos_token_stride,
                               int64_t pos_head_stride, void* q_out, void* hip_stream) {
  qp::PagedArgs a;
  qp_status st = check(L, cache, batch, true, &a);
  if (st != QP_OK) return st;
  if (rope == nullptr || !aligned(rope->pos, 4) || rope->axis_stride < 0 || !(rope->theta > 0.f) || isinf(rope->theta))
    return QP_ERR_INVALID_ARG;
  int64_t sections = 0;
  for (int x = 0; x < 3; ++x) {
    if (rope->section[x] < 0) return QP_ERR_INVALID_ARG;
    sections += rope->section[x];
  }
  if (sections != L->head_dim / 2) return QP_ERR_INVALID_ARG;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(pos, 4)) return QP_ERR_INVALID_ARG;
  if ((q_or_null == nullptr) != (q_out == nullptr)) return QP_ERR_INVALID_ARG;
  const int64_t size = L->dtype == QP_F32 ? 4 : 2;
  if ((st = check_strides(token_stride, head_stride, size)) != QP_OK) return st;
  if ((st = check_pos_strides(pos_token_stride, pos_head_stride)) != QP_OK) return st;
  if (rope->axis_stride > kMostStride) return QP_ERR_UNSUPPORTED;
  qp::PagedStore store{};
  if (q_or_null != nullptr) {
    if (!aligned(q_or_null, 16) || !aligned(q_out, 16)) return QP_ERR_INVALID_ARG;
    if ((st = check_strides(q_token_stride, q_head_stride, size)) != QP_OK) return st;
    store.q = q_or_null, store.q_out = q_out, store.q_token_stride = q_token_stride * size, store.q_head_stride = q_head_stride * size;
  }
  store.k = k, store.v = v, store.token_stride = token_stride * size, store.head_stride = head_stride * size;
  store.pos = pos, store.pos_token_stride = pos_token_stride, store.pos_head_stride = pos_head_stride;
  store.axes = rope->pos, store.axis_stride = rope->axis_stride, store.theta = rope->theta;
  store.s0 = rope->section[0], store.s1 = rope->section[1];
  return finish(qp::launch_paged_store(a, store, L->dtype, L->head_dim, (hipStream_t)hip_stream));
}

qp_status qp_paged_attend(const qp_layout* L, const qp_paged_cache* cache, const qp_paged_batch* batch, const void* q, void* out,
                          float* lse_or_null, void* workspace, size_t workspace_bytes, void* hip_stream) {
  qp::PagedArgs a;
  const qp_status st = check(L, cache, batch, true, &a);
  if (st != QP_OK) return st;
  if (!aligned(q, 16) || !aligned(out, 16) || (lse_or_null != nullptr && !aligned(lse_or_null, 4)) || bad_workspace(workspace))
    return QP_ERR_INVALID_ARG;
  return finish(qp::launch_paged_attend(a, L->dtype, L->head_dim, q, out, lse_or_null, workspace, workspace_bytes,
                                        (hipStream_t)hip_stream));
}

qp_status qp_paged_attend_window(const qp_layout* L, const qp_paged_cache* cache, const qp_paged_batch* batch, int32_t window,
                                 int32_t n_sink, const void* q, void* out, float* lse_or_null, void* workspace, size_t workspace_bytes,
                                 void* hip_stream) {
  qp::PagedArgs a;
  const qp_status st = check(L, cache, batch, true, &a);
  if (st != QP_OK) return st;
  if (window < 1 || n_sink < 0) return QP_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 16) || (lse_or_null != nullptr && !aligned(lse_or_null, 4)) || bad_workspace(workspace))
    return QP_ERR_INVALID_ARG;
  a.window = window < a.max_len ? window : a.max_len;  // no entry is further from another
  a.n_sink = n_sink < a.max_len ? n_sink : a.max_len;
  return finish(qp::launch_paged_attend(a, L->dtype, L->head_dim, q, out, lse_or_null, workspace, workspace_bytes,
                                        (hipStream_t)hip_stream));
}

qp_status qp_paged_weigh(const qp_layout* L, const qp_paged_cache* cache, const qp_paged_batch* batch, const void* q,
                         const float* lse, int32_t accumulate, void* workspace, size_t workspace_bytes, void* hip_stream) {
  qp::PagedArgs a;
  const qp_status st = check(L, cache, batch, true, &a);
  if (st != QP_OK) return st;
  if (a.weight == nullptr || !aligned(q, 16) || !aligned(lse, 4) || bad_workspace(workspace)) return QP_ERR_INVALID_ARG;
  return finish(qp::launch_paged_weigh(a, L->dtype, L->head_dim, q, lse, accumulate != 0, workspace, workspace_bytes,
                                       (hipStream_t)hip_stream));
}

qp_status qp_paged_evict(const qp_layout* L, const qp_paged_cache* cache, const qp_paged_batch* batch, int32_t keep,
                         int32_t n_first, int32_t n_last, const int32_t* to_table, int32_t to_pages, int32_t* to_len,
                         int32_t* kept_or_null, void* workspace, size_t workspace_bytes, void* hip_stream) {
  qp::PagedArgs a;
  const qp_status st = check(L, cache, batch, false, &a);
  if (st != QP_OK) return st;
  if (a.weight == nullptr || keep <= 0 || n_first < 0 || n_last < 0 || n_first > keep || n_last > keep - n_first)
    return QP_ERR_INVALID_ARG;
  if (!aligned(to_table, 4) || !aligned(to_len, 4) || to_pages <= 0 || (kept_or_null != nullptr && !aligned(kept_or_null, 4)) ||
      bad_workspace(workspace))
    return QP_ERR_INVALID_ARG;
  if (keep > kMaxLen) return QP_ERR_UNSUPPORTED;
  if (((int64_t)to_pages << a.page_shift) < keep) return QP_ERR_CAPACITY;
  if (workspace == nullptr || workspace_bytes < evict_bytes(a.n_seqs, a.h_kv, keep, a.max_len)) return QP_ERR_CAPACITY;
  qp::PagedEvict e{};
  e.keep = keep, e.n_first = n_first, e.n_last = n_last;
  e.to_table = to_table, e.to_pages = to_pages, e.to_len = to_len;
  e.kept = kept_or_null != nullptr ? kept_or_null : (int32_t*)workspace;
  if (qp::paged_evict_keys_bytes(a.n_seqs, a.h_kv, a.max_len) > 0)
    e.keys = (uint32_t*)((unsigned char*)workspace + evict_kept_bytes(a.n_seqs, a.h_kv, keep));
  const int row_bytes = L->head_dim * (a.fp8 ? 1 : L->dtype == QP_F32 ? 4 : 2);
  return finish(qp::launch_paged_evict(a, e, row_bytes, (hipStream_t)hip_stream));
}

qp_status qp_paged_plan(const qp_layout* L, const qp_paged_cache* cache, const qp_paged_batch* batch, size_t workspace_bytes,
                        qp_paged_plan_info* out) {
  qp::PagedArgs a;
  const qp_status st = check(L, cache, batch, true, &a);
  if (st != QP_OK) return st;
  if (out == nullptr) return QP_ERR_INVALID_ARG;
  const qp::PagedPlan p = qp::plan_paged_attend(a, L->dtype, L->head_dim, workspace_bytes);
  memset(out, 0, sizeof(*out));
  if (p.workgroups > 0x7fffffffll) return QP_ERR_UNSUPPORTED;
  out->rows_per_tile = p.tile_rows;
  out->shares = p.shares;
  out->key_chunks = p.chunks;
  out->chunk_entries = p.chunk_keys;
  out->workgroups = (int32_t)p.workgroups;
  out->scratch_bytes = p.scratch_bytes;
  return QP_OK;
}

}  // extern "C"

/*
 * qp_paged.h -- C ABI of the paged pruned cache (gfx950): many sequences at once over one pool of pages.
 *
 * qp.h serves one sequence whose pruned cache (Sec. 3.2 of the QuickVideo paper) is one flat array and whose length the
 * host knows. The stages that follow video prefill (Sec. 2.1: the question's tokens, then decoding) are served to many
 * users at once, each over the entries of a video of their own or of a shared one, and an answer goes on until it ends.
 * Here entries live in pages of a pool, a table says which pages a sequence has, and lengths are DEVICE values, so that a
 * captured graph of a decoding step can be replayed while they grow:
 *   qp_paged_append   stores new keys and values (a step's, a chunk's, or what a video left in a flat cache) in the pages
 *   qp_paged_append_rope    the same with the keys turned by their rotary angles on the way, and the new tokens' queries too
 *   qp_paged_attend   attention of every sequence's new tokens over its entries
 *   qp_paged_attend_window  the same where a token sees a window of the last entries and the sequence's first ones
 *   qp_paged_weigh    the attention weight that every entry received from those tokens, taken anew or accumulated
 *   qp_paged_evict    keeps the entries of most weight (and the first and the last ones), packed into other pages
 *
 * Conventions as in qp.h: data pointers are DEVICE pointers, tensors dense and row-major unless strides are given, 16-byte
 * aligned (4-byte: int32 arrays and lse), the structs live in HOST memory, the library
 * allocates nothing, keeps no pointer and never waits for the GPU, all work is enqueued on `hip_stream` of the current
 * device, errors come back as qp_status and are found on the host before anything is launched. Same inputs (and the same
 * workspace size) give the same bits: nothing is summed by atomics.
 *   What the host cannot see is made harmless on the device: lengths and row numbers are brought into the limits that the
 * batch states, and a page number outside [0, n_pages) is a page that is not there: its entries are never read or
 * written, no row sees them. A caller may use that (-1) to give back pages in the middle of a sequence.
 *   A page may be in several sequences' tables (a video that several questions are about) in calls that only read it:
 * qp_paged_attend, and the source of qp_paged_evict. In a call that writes it (append, weigh, the destination of evict)
 * it may be there once: two writers of one entry race, and only its value is then unspecified.
 * Supported: dtype f32 or bf16, head_dim 64 or 128, pages of 16, 32, 64, 128 or 256 tokens; 8-bit pools (E4M3) as in qp.h.
 *   QP_CACHE_FP8_E4M3_SCALED: an 8-bit pool (bf16 layouts of head_dim 128) whose entries j / 16 of a sequence share a scale per KV head, one
 * for keys and one for values: an element is code * scale, scale a power of two from 2^-117 to 2^120 (at which codes beyond
 * +-240 are infinities, and appends saturate at 240). E4M3 codes alone hold magnitudes from 2^-9 to
 * 448: keys of channels with large offsets saturate. Codes are floating-point themselves, so a finer scale would not make them more exact; a power of two
 * is exact wherever it is applied. An append gives a block the least scale that holds its finite values (infinities saturate, NaN stays) and never
 * a smaller one than the block's earlier entries have; where it grows, their codes are divided with it, exactly down to 2^-6 of the new
 * scale and rounded below. So an append to a block that is partly full may write entries that were there before it, which with the other formats it never
 * does: sequences that share such a page have them rounded too, and a call on another stream that reads them meanwhile races with it (share pages up to a
 * multiple of 16 entries, and go on in a page of one's own). Tokens that are taken back, by a smaller len, leave their block's scale and its codes as they had
 * become; a block that is begun anew, from its first entry, has no past. Entries that qp_paged_evict moves join blocks of new neighbours, whose scale is the largest of theirs, their codes divided in the same way.
 */
#ifndef QP_PAGED_H_
#define QP_PAGED_H_

#include "qp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The pool. Entry e of KV head h in page p is row (p * n_kv_heads + h) * page_tokens + e of each array. */
typedef struct {
  void* k;             /* [n_pages][n_kv_heads][page_tokens][head_dim], layout dtype (or 1 byte, see format)   */
  void* v;
  int32_t* pos;        /* [n_pages][n_kv_heads][page_tokens]: the entry's token position                       */
  float* weight;       /* [n_pages][n_kv_heads][page_tokens]: attention weight it received; may be NULL where
                          neither qp_paged_weigh nor qp_paged_evict is called                                  */
  int32_t n_pages;
  int32_t page_tokens; /* 16, 32, 64, 128 or 256                                                               */
  int32_t format;      /* qp_cache_format of k and v                                                           */
  float* k_scale;      /* [n_pages][n_kv_heads][page_tokens / 16], QP_CACHE_FP8_E4M3_SCALED only: powers of two */
  float* v_scale;
} qp_paged_cache;

/* The sequences of a call. Sequence s has the entries 0 .. len[s] - 1, entry j in page page_table[s][j / page_tokens] at
 * j % page_tokens, and the new tokens of rows row_start[s] .. row_start[s + 1] - 1 (n_s of them, possibly none) of the call's
 * tensors, which are its LAST n_s entries: row i of s (from 0) is entry len[s] - n_s + i and sees the entries up to itself.
 * Rows before row_start[0] and from row_start[n_seqs] on belong to nobody and are left as they were. A length beyond max_len or the
 * end of the table counts as that end: the new tokens are then the last entries before it. */
typedef struct {
  const int32_t* page_table; /* device, [n_seqs][table_pages]                                                  */
  const int32_t* len;        /* device, [n_seqs]: entries, the new ones included                               */
  const int32_t* row_start;  /* device, [n_seqs + 1], not descending; NULL for qp_paged_evict                  */
  int32_t n_seqs;
  int32_t table_pages;       /* row length of page_table                                                       */
  int32_t n_rows;            /* rows that the call's tensors have, at least 1 (qp_paged_evict has none)        */
  int32_t max_new;           /* >= 1; no sequence has more new tokens: launches are sized by these two, and    */
  int32_t max_len;           /* what a sequence has beyond them (or beyond its table) is not looked at         */
} qp_paged_batch;

/* Workspace that every call below accepts for batches of these sizes (256-byte aligned where it is handed over): partial
 * results of qp_paged_attend (128 MiB at most) and qp_paged_weigh, the selection of qp_paged_evict with `keep` (0: none). Counted without
 * a window: qp_paged_attend_window would deal short windows, or those of many sequences, to more workgroups if it got more (up to the same 128 MiB). 0 on
 * bad arguments. */
size_t qp_paged_workspace_bytes(const qp_layout* layout, int32_t n_seqs, int32_t n_rows, int32_t max_new, int32_t max_len,
                                int32_t keep);

/* Stores the new tokens' keys and values: row r of KV head h is at k + (r * token_stride + h * head_stride) elements (v
 * alike), head_dim elements in a run, rows 16-byte aligned, so that a group's [rows][H_kv][d] tensors, slices of a fused QKV
 * result and a flat pruned cache's [H_kv][capacity][d] (token_stride d, head_stride capacity * d) can all be the source.
 *   pos: position of row r of head h at pos[r * pos_token_stride + h * pos_head_stride] (pos_head_stride 0: one per token)
 *   source_format: QP_CACHE_SAME, rows in the layout's dtype (rounded as qp_topk_compact rounds if the pool is 8-bit), or
 *     QP_CACHE_FP8_E4M3, rows that are E4M3 bytes already (8-bit pools without scales only; strides then count bytes)
 * The entries' weights, if the pool has them, become 0. */
qp_status qp_paged_append(const qp_layout* layout, const qp_paged_cache* cache, const qp_paged_batch* batch, const void* k,
                          const void* v, int64_t token_stride, int64_t head_stride, const int32_t* pos,
                          int64_t pos_token_stride, int64_t pos_head_stride, qp_cache_format source_format, void* hip_stream);

/* Rotary positions of a call's rows. Frequency i of head_dim / 2 is theta^(-2 i / head_dim); the first section[0] of them turn by the position
 * index on axis 0 (temporal), the next section[1] on axis 1 (height), the last section[2] on axis 2 (width). */
typedef struct {
  const int32_t* pos;   /* device: row r's index on axis a at pos[a * axis_stride + r]                        */
  int64_t axis_stride;  /* 0: the same index on all axes (text)                                               */
  float theta;
  int32_t section[3];   /* sum head_dim / 2                                                                   */
} qp_paged_rope;

/* qp_paged_append of keys that are not rotated yet (a plain projection's): pairs (i, i + head_dim / 2) of every key are turned by
 * pos * frequency on the way, and so are the queries of the same rows, if given. Angles as exact as f32 holds their sines and cosines,
 * f32 arithmetic, one rounding, to the pool's type (8-bit codes too) or, queries, the layout's. Positions up to 2^26 in
 * size; of larger ones the angles' last bits are lost.
 *   k, v: as in qp_paged_append (token_stride, head_stride in elements; rows of the layout's dtype)
 *   q_or_null: query head h of row r at q + (r * q_token_stride + h * q_head_stride), 16-byte aligned rows; q_out [n_rows][H_q][d], which
 *     may be q itself where that is dense. Rows of nobody are left as they were; both NULL: keys and values only
 *   pos, pos_token_stride, pos_head_stride: the entries' token positions, as in qp_paged_append */
qp_status qp_paged_append_rope(const qp_layout* layout, const qp_paged_cache* cache, const qp_paged_batch* batch,
                               const qp_paged_rope* rope, const void* q_or_null, int64_t q_token_stride, int64_t q_head_stride,
                               const void* k, const void* v, int64_t token_stride, int64_t head_stride, const int32_t* pos,
                               int64_t pos_token_stride, int64_t pos_head_stride, void* q_out, void* hip_stream);

/* Attention of the new tokens: q, out [n_rows][H_q][d] (layout dtype), lse_or_null [H_q][n_rows] f32 (natural log). A row that
 * sees no entry (the sequence has fewer than its new rows, or none of its pages is there) gets zeros and -infinity. Arithmetic as qp_group_attend: f32
 * products and sums; bf16 rows' softmax numerators are rounded to bf16 before the product with V (to two bf16 terms in calls of up to
 * 32 stacked rows, max_new * H_q / H_kv, and over heads of 64), never in the sums behind lse. All rows of a call take the same way, so
 * a row's last bits depend on max_new. What a row does not see does not reach its result, infinities and NaN included; an
 * infinite value that it sees makes its element infinite, or NaN. Values are summed in f32, each times a numerator of up to 2^8: where those that a row
 * sees add up to more than 2^119 in size, its element may be infinite too. Logits scale * q.k of
 * up to 2^28 in size are computed; those below -2^29 weigh nothing, as -infinity does, and a row that sees nothing else is one that sees
 * no entry; of a row with one above 2^28 nothing is promised.
 *   workspace: may be NULL. Where the rows would leave compute units idle, their entries are dealt to several workgroups
 *     whose partial results (f32) lie there until a second launch merges them; without it (or with less) to fewer. */
qp_status qp_paged_attend(const qp_layout* layout, const qp_paged_cache* cache, const qp_paged_batch* batch, const void* q,
                          void* out, float* lse_or_null, void* workspace, size_t workspace_bytes, void* hip_stream);

/* qp_paged_attend with a sliding window: the row that is entry p sees the entries j <= p with j > p - window or j < n_sink, so each
 * new token has a window of its own. window >= 1 entries, the row's own included; n_sink >= 0. What no row sees is not read: pages
 * between the first entries and the windows may have been given back (-1 in the table). Arguments, arithmetic and workspace otherwise as
 * qp_paged_attend; a window of max_len entries gives its results (a row's last bits may differ). */
qp_status qp_paged_attend_window(const qp_layout* layout, const qp_paged_cache* cache, const qp_paged_batch* batch, int32_t window,
                                 int32_t n_sink, const void* q, void* out, float* lse_or_null, void* workspace, size_t workspace_bytes,
                                 void* hip_stream);

/* weight[j] of KV head h = (accumulate ? weight[j] : 0) + the sum of exp(scale * q.k_j - lse) over the sequence's new rows that
 * see j and the H_q / H_kv query heads of h, for every entry j < len[s]: with the lse that qp_paged_attend (not qp_paged_attend_window) wrote for the same
 * rows, the attention weight that the entry received. Rows of lse = -infinity add nothing. f32 arithmetic. cache->weight must
 * be there. workspace: may be NULL; calls of many rows over few entries deal the rows to several workgroups where it is given. */
qp_status qp_paged_weigh(const qp_layout* layout, const qp_paged_cache* cache, const qp_paged_batch* batch, const void* q,
                         const float* lse, int32_t accumulate, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Keeps min(keep, present) entries of every sequence and KV head: of those that are present the ones among the first n_first
 * and the last n_last entries (n_first + n_last <= keep), and of the others those of the largest weight, equal weights (and
 * -0.0 == +0.0) by lower entry number; weights must not be NaN. They are stored in ascending order as entries 0, 1, ... of
 * the pages of to_table [n_seqs][to_pages], with their positions and weights, and to_len[s] becomes their number (the same for
 * all heads; to_len may be the batch's len). The old pages are only read: the caller gives them back (or keeps them, where others share them). A sequence of at
 * most `keep` entries is copied whole, without its missing pages.
 *   kept_or_null [n_seqs][H_kv][keep]: their old entry numbers, -1 behind the last
 *   workspace: qp_paged_workspace_bytes(..., keep) bytes, needed
 * No destination page may be one that the call reads. CAPACITY if to_pages * page_tokens < keep or the workspace is too small. */
qp_status qp_paged_evict(const qp_layout* layout, const qp_paged_cache* cache, const qp_paged_batch* batch, int32_t keep,
                         int32_t n_first, int32_t n_last, const int32_t* to_table, int32_t to_pages, int32_t* to_len,
                         int32_t* kept_or_null, void* workspace, size_t workspace_bytes, void* hip_stream);

/* How qp_paged_attend (without a window) would lay out a call (host arithmetic only). Few rows: `shares` workgroups of every KV head divide the entries
 * of all sequences evenly among them (0: a workgroup per sequence, head and row tile, no scratch). Chunks over bf16 heads of 128:
 * key_chunks of chunk_entries of every sequence (1: no scratch). */
typedef struct {
  int32_t rows_per_tile; /* stacked rows (tokens x query heads of a KV head) of one workgroup: 16, 32 or 256 */
  int32_t shares;
  int32_t key_chunks;
  int32_t chunk_entries;
  int32_t workgroups;
  size_t scratch_bytes;
} qp_paged_plan_info;
qp_status qp_paged_plan(const qp_layout* layout, const qp_paged_cache* cache, const qp_paged_batch* batch,
                        size_t workspace_bytes, qp_paged_plan_info* out);

#ifdef __cplusplus
}
#endif
#endif /* QP_PAGED_H_ */

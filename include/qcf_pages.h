/*
 * qcf_pages.h - decoding over the fused cache, kept in pages (conventions of qcf.h).
 *
 * After a prompt's cache has been fused, its answer is decoded token by token: the newest tokens' keys and values go behind
 * what their request holds, and their queries attend to all of it, or to the pages that a cheap score picks for each of them.
 *
 *   call order for one layer and one step:
 *     qcf_page_append -> [qcf_page_select ->] qcf_page_attn
 *   (all on one stream; the fused cache itself goes into pages with qcf_page_append, unrotated)
 *   (B is at most 65535 in each; a launch takes 2^32 threads at most, so selections of B * n_q * H_kv beyond 2^22 are refused)
 */
#ifndef QCF_PAGES_H
#define QCF_PAGES_H

#include "qcf.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A layer's cache in pages (host struct).  Token t of request b is in slot t % page_size of page table[b][t / page_size].
 * A table entry outside [0, n_pages) is a page that is not there: what would be written to it is dropped, its tokens are not
 * attended to.  Requests may share pages that none of them writes.
 * Slot s of page p, KV head g: d elements from p * page_stride + s * slot_stride + g * head_stride on, of k and of v.  Any order is
 * taken; pages that keep a head's tokens together are read 4 to 5 % faster than pages that keep a token's heads together.
 * The calls read lengths on the device and divide their work by max_pages: one request of 256 tokens is attended to in 7.0 us with a
 * table of 16 pages, 9.9 with one of 512 or 8192 (two launches); where contexts are long it makes no difference.
 * Strides are in elements, multiples of 8, at most 2^24 for slots and heads; rows of a page must not overlap, and page_stride
 * must be at least what a page spans. */
typedef struct qcf_page_cache {
  void* k;               /* DEVICE, element type desc->dtype */
  void* v;
  void* bounds;          /* DEVICE [n_pages, H_kv, 2, d]: least and largest stored key of a page, element by element; NULL = none */
  const int32_t* table;  /* DEVICE [B, max_pages] */
  int64_t page_stride;
  int64_t slot_stride;
  int64_t head_stride;
  int32_t n_pages;       /* > 0 */
  int32_t page_size;     /* 16, 32, 64, 128 or 256 tokens */
  int32_t max_pages;     /* > 0; max_pages * page_size at most 2^30 */
  int32_t reserved;      /* set to 0 */
} qcf_page_cache;

/* Rows [row_off[b], row_off[b+1]) of q, k and v become tokens len[b], len[b] + 1, ... of request b; len itself is not changed.
 * q [total_rows, H, d], k and v [total_rows, H_kv, d], the rows q_stride, k_stride and v_stride elements apart (multiples of 8,
 * at least a row): the three parts of one product's rows, for instance.  pos (NULL: no rotation): row m's keys and queries are
 * turned by pos[m] * theta_i, so pos holds the absolute positions of fresh rows or what a chunk's keys have to move by.
 * q and q_out [total_rows, H, d] (dense): both or neither; q_out may be q where the rows are dense.
 * Bounds (where the cache has them) are joined with the stored keys of the rows; a page whose slot 0 is written starts anew.
 * Rows whose token would lie beyond max_pages pages or before token 0, or whose page is not there, are not stored (their queries
 * are still turned).  Rows behind row_off[B] are left as they were, and so are slots that get no row.  A page that is written
 * must be in the table once only, and the rows must not lie in the cache.  A slot that is written again leaves its page's bounds
 * wider than they need be, until slot 0 is. */
qcf_status qcf_page_append(const qcf_layer_desc* desc, const qcf_page_cache* cache, int32_t B, const void* q, int64_t q_stride,
                           const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int64_t* row_off_dev,
                           int64_t total_rows, const int32_t* len_dev, const int32_t* pos_dev, void* q_out, void* stream);

/* The pages that each query's attention is cut down to.  q [B, n_q, H, d]: n_q new rows of each request, 1 <= n_q <= 16;
 * seen [B, n_q]: the number of leading tokens that a row sees (0: none, a row that fills up the batch).
 *   score[b, i, g, p] = max over the heads h of KV head g of sum_e max(q[b, i, h, e] lo[e], q[b, i, h, e] hi[e])
 * with lo and hi the bounds of page p of request b: no key of the page has a larger product with any of these queries.  The sum
 * is taken in 64 bits and rounded once to 32.  pages [B, n_q, H_kv, n_keep] gets the n_keep pages of the largest scores among
 * the ceil(seen / page_size) that the row sees, ascending, ties to the lower page, -1 behind the last.  The first n_first and
 * the last n_last of them rank before all others (n_first + n_last <= n_keep), then pages with a sum that is infinite or not a
 * number, of either sign (a key or a query that is not finite makes it so), and pages that are not in the table behind all
 * others.  A finite sum beyond the range of 32 bits counts as the largest or the least float. */
size_t qcf_page_select_workspace_bytes(const qcf_layer_desc* desc, const qcf_page_cache* cache, int32_t B, int32_t n_q, int32_t n_keep);
qcf_status qcf_page_select(const qcf_layer_desc* desc, const qcf_page_cache* cache, int32_t B, int32_t n_q, const void* q,
                           const int32_t* seen_dev, int32_t n_keep, int32_t n_first, int32_t n_last, int32_t* pages,
                           void* workspace, size_t workspace_bytes, void* stream);

/* o[b, i, h] = sum_t softmax_t( q[b, i, h] . k_t / sqrt(d) ) v_t over the tokens t < seen[b, i] of request b whose page is there,
 * k_t and v_t of KV head h / (H / H_kv).  q and o [B, n_q, H, d], seen [B, n_q], 1 <= n_q <= 16, as above; lse (may be NULL)
 * [B, n_q, H] float32, natural-log sum-exp of the scaled logits.  A row that sees nothing gets a zero output row and lse = -inf;
 * what is stored in slots that a row does not see, whatever it is, does not reach it.  A logit of -inf weighs nothing beside others,
and makes a row that has only such NaN; a logit that is NaN or +inf makes its row NaN.
 * pages (NULL: all pages; n_keep is then 0) [B, n_q, H_kv, n_keep]: only tokens of these pages, in any order; entries that are no
 * page of the row are passed over, a page that is listed twice counts twice.
 * The contexts are divided over the GPU by their lengths; the same call gives the same bits, and the last bits of a row depend on
 * the other rows' lengths. */
size_t qcf_page_attn_workspace_bytes(const qcf_layer_desc* desc, const qcf_page_cache* cache, int32_t B, int32_t n_q, int32_t n_keep);
qcf_status qcf_page_attn(const qcf_layer_desc* desc, const qcf_page_cache* cache, int32_t B, int32_t n_q, const void* q,
                         const int32_t* seen_dev, const int32_t* pages, int32_t n_keep, void* o_out, float* lse_out,
                         void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* QCF_PAGES_H */

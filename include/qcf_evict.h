/*
 * qcf_evict.h - a cache in pages cut down to the tokens that attention uses (conventions of qcf.h and qcf_pages.h).
 *
 * While an answer is decoded, qcf_page_weigh adds up the attention weights that every cached token gets, for each KV head by itself.
 * Once a request holds more than it should, qcf_page_evict moves the first tokens, the last ones and the heaviest of the others to
 * other pages, each head its own, and the pages they come from are free.
 *
 *   call order for one layer:
 *     every step  qcf_page_append -> qcf_page_attn (with lse) -> qcf_page_weigh
 *     now and then  qcf_page_evict
 *   (rows that may still be rejected, drafts, are weighed once it is known which of them stay, with a `seen` of 0 for the others)
 *
 * Both calls take pages of the layer's type (scales NULL) or 8-bit pages (qcf_pages8.h).  Weights are dense:
 *   weights  DEVICE [B, H_kv, max_pages * page_size] float32, token t of request b at its own place whatever page it is in.
 * Keys are stored rotated, so a token keeps its absolute position wherever it lies; lengths count what is held.
 */
#ifndef QCF_EVICT_H
#define QCF_EVICT_H

#include "qcf_pages8.h"

#ifdef __cplusplus
extern "C" {
#endif

/* weights[b, g, t] = alpha * weights[b, g, t] + beta * sum over rows i and heads h of KV head g of exp(q[b, i, h] . k_t / sqrt(d) - lse[b, i, h])
 * for the tokens t < max_i seen[b, i]; a row adds to the tokens that it sees (t < seen[b, i]) and whose page is there.  What is behind
 * them is left as it was.  q [B, n_q, H, d], seen [B, n_q] and lse [B, n_q, H] as in and from qcf_page_attn over all pages, 1 <= n_q <= 16.
 * old [B]: tokens of a request that have been weighed before; what is stored for others (fresh ones, whose places another token may have
 * had) counts as 0 (NULL: all have been).  alpha 0: nothing that is stored is read.  A weight that is NaN is stored as the positive one.
 * One sum to a token, in a fixed order: the same call gives the same bits. */
qcf_status qcf_page_weigh(const qcf_layer_desc* desc, const qcf_page_cache* cache, const float* scales, int32_t B, int32_t n_q,
                          const void* q, const int32_t* seen_dev, const float* lse, const int32_t* old_dev, float alpha, float beta,
                          float* weights, void* stream);

/* Each KV head of each request keeps n_keep > 0 of its len[b] tokens (all, where there are no more): the first n_first, the last n_last
 * (n_first + n_last <= n_keep) and, of the others, those with the largest weights, ties to the lower token, NaN (the positive one) before
 * all others.  kept [B, H_kv, n_keep] gets their numbers, ascending, -1 behind the last; token kept[b, g, j] becomes token j of the cache
 * `to`, its weight to_weights[b, g, j] (NULL: not wanted; otherwise [B, H_kv, to->max_pages * to->page_size], other memory than
 * weights), and to_len[b] (may be len) the number of tokens.  Slots of `to` behind them are left as they were.
 * `to` may lie in the same pools and have pages of another size; the pages that it lists must be none of the pages that `cache` lists for
 * these requests, and each once only.  Tokens of pages that are not there must not be among the first len[b] (they move as zeros);
 * what pages of `to` that are not there should get is dropped, and what goes beyond its max_pages (to_len counts it).  Bounds of `to`,
 * if it has any, are made anew; `cache` needs none.
 * 8-bit pages (scales and to_scales, both or neither): a block of `to` gets the scale that qcf_page8_append would give its tokens.
 * The choice is divided by the room of the table and not by the lengths, which the host does not know: in six launches, where a table has
 * room for more than 32768 tokens and B * H_kv is at most 128.  8 KV heads of 128 in 8 bits, requests of 2000 tokens to 1024: one takes
 * 13 us with room for 32768, 30 with more; 16 take 22, 47 with room for 33024 and 117 with room for 131072. */
size_t qcf_page_evict_workspace_bytes(const qcf_layer_desc* desc, const qcf_page_cache* cache, int32_t B, int32_t n_keep);
qcf_status qcf_page_evict(const qcf_layer_desc* desc, const qcf_page_cache* cache, const float* scales, int32_t B,
                          const int32_t* len_dev, const float* weights, int32_t n_keep, int32_t n_first, int32_t n_last,
                          const qcf_page_cache* to, float* to_scales, int32_t* kept, float* to_weights, int32_t* to_len_dev,
                          void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* QCF_EVICT_H */

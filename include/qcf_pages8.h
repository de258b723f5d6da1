/*
 * qcf_pages8.h - decoding over a cache in 8-bit pages (conventions of qcf.h and qcf_pages.h).
 *
 * The calls of qcf_pages.h over pages of half the size: k and v hold e4m3 codes (OCP: 1 sign, 4 exponent and 3 fraction bits, up to
 * 448, 0x7f and 0xff are NaN), and an element is its code times the scale of its block, the 16 tokens of a KV head that lie next to
 * each other in a page (slots 16 i to 16 i + 15).  Queries, new rows, outputs and bounds have the layer's type.
 *
 *   call order for one layer and one step:
 *     qcf_page8_append -> [qcf_page_select ->] qcf_page8_attn
 */
#ifndef QCF_PAGES8_H
#define QCF_PAGES8_H

#include "qcf_pages.h"

#ifdef __cplusplus
extern "C" {
#endif

#define QCF_PAGE8_BLOCK 16

/* The cache is described by a qcf_page_cache whose k and v point to codes (16-byte aligned; strides are in elements, which are bytes
 * here, and multiples of 16) and by
 *   scales  DEVICE [n_pages, H_kv, 2, page_size / 16] float32: those of a page's keys (0) and of its values (1); at most 2^31 of them.
 * Bounds, if there are any, have the layer's type; qcf_page_select takes such a cache as it is (it reads bounds and table only). */

/* qcf_page_append for 8-bit pages: the same arguments, and scales.  Keys are turned in 64 bits and rounded once, to their codes.  A
 * block's scale is the least power of two s, not less than 2^-100, with |x| <= 448 s for all elements that were stored into it since
 * its first slot was written.  Where rows make the scale of a block grow that has tokens in front of them, these are rounded again, to
 * the new scale (a value changes only where it comes beneath 2^-6 of it).  Elements that are not finite or beyond 2^100 are stored as
 * NaN and do not count for the scale.  Bounds contain the stored values, and are theirs but where older tokens were rounded again, which may
 * have come closer to 0 than they were: there they may be wider, until slot 0 of the page is written. */
qcf_status qcf_page8_append(const qcf_layer_desc* desc, const qcf_page_cache* cache, float* scales, int32_t B, const void* q,
                            int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                            const int64_t* row_off_dev, int64_t total_rows, const int32_t* len_dev, const int32_t* pos_dev, void* q_out,
                            void* stream);

/* qcf_page_attn over 8-bit pages: the same arguments, and scales (any from 2^-100 to 2^92, the least and the largest that are stored by
 * qcf_page8_append: beyond them sums may overflow, below them lose bits).  Products and sums are taken in 32 bits, codes enter them
 * exactly; a code that is NaN makes the rows NaN that see it.  The scale of a block none of whose tokens a row sees may be anything. */
size_t qcf_page8_attn_workspace_bytes(const qcf_layer_desc* desc, const qcf_page_cache* cache, int32_t B, int32_t n_q, int32_t n_keep);
qcf_status qcf_page8_attn(const qcf_layer_desc* desc, const qcf_page_cache* cache, const float* scales, int32_t B, int32_t n_q,
                          const void* q, const int32_t* seen_dev, const int32_t* pages, int32_t n_keep, void* o_out, float* lse_out,
                          void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* QCF_PAGES8_H */

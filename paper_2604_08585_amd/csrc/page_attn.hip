// Attention of the newest tokens over a cache in pages.
//
// One pass over the keys and values with a running reference point and sum of each row's softmax.  The contexts are divided into
// equal ranges, as many as the GPU holds at once; a second launch joins the partial results of contexts that several ranges have.
// Bound by memory: 4 d operations to a token and row against 4 d bytes (bf16) to a token and KV head, which is an operation a byte for
// each row, 4 to 32 of them.  32 / 8 heads of 128, 64 requests of 4K to 12K tokens: 395 us, 5.5 TB/s, the bytes of the keys and values
// and no more (counters; a copy of 1 GiB reaches 5.05 TB/s); one of 128K 101 us; one of 731 tokens 10.4 us, in two launches that depend on
// each other (6.9 and 4.5 us where a profiler keeps them apart).
//
// A wave takes 32 tokens (16 in float32) at a time, without LDS: the logits are products K Q^T of 16 tokens x 16 rows, so a lane
// owns a row and four tokens; the outputs are V^T P^T of 16 elements x 16 rows, in which the order of the tokens is free.  It
// is taken so that a lane's four tokens of the logits are its tokens of that product, and the elements of a head so that a lane
// loads 16 bytes of a value row.  What is left is a transposition inside the lane (bf16: 8 tokens x 8 elements, 32 v_perm).
#include "page_walk.h"

namespace qcf {

size_t page_attn_workspace(const qcf_layer_desc& L, const qcf_page_cache& c, int32_t B, int32_t n_q, int32_t n_keep) {
  return pages::workspace(L, pages::divide(L, c, B, n_q, n_keep));
}

qcf_status launch_page_attn(const qcf_layer_desc& L, const qcf_page_cache& c, int32_t B, int32_t n_q, const void* q,
                            const int32_t* seen, const int32_t* list, int32_t n_keep, void* o, float* lse, void* ws,
                            hipStream_t st) {
  return attend<false>(L, c, nullptr, B, n_q, q, seen, list, n_keep, o, lse, ws, st);
}

}  // namespace qcf

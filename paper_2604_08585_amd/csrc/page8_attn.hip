// Attention of the newest tokens over a cache in 8-bit pages: the walk of page_attn.hip, with codes that become bf16 (or float) in registers.
// o = sum_t softmax_t(q . k_t s_k / sqrt(d)) (s_v v_t): a key's scale is a factor of its block's logits, a value's of its block's weights.
// Bound by memory where contexts are long: 32 / 8 heads of 128, 64 requests of 4K to 12K tokens 203 us, 5.4 TB/s (a copy of 1 GiB reaches 5.1),
// 207 where a token's heads lie together (396 in bf16); one of 128K 59 us, 52 without the join.  The vector unit is busy for 33 % of that;
// with several new rows it is what counts: four drafts of 64 such requests, 64 / 8 heads, 262 us.
#include "page_walk.h"

namespace qcf {

size_t page8_attn_workspace(const qcf_layer_desc& L, const qcf_page_cache& c, int32_t B, int32_t n_q, int32_t n_keep) {
  return pages::workspace(L, pages::divide(L, c, B, n_q, n_keep, 1));
}

qcf_status launch_page8_attn(const qcf_layer_desc& L, const qcf_page_cache& c, const float* scales, int32_t B, int32_t n_q,
                             const void* q, const int32_t* seen, const int32_t* list, int32_t n_keep, void* o, float* lse, void* ws,
                             hipStream_t st) {
  return attend<true>(L, c, scales, B, n_q, q, seen, list, n_keep, o, lse, ws, st);
}

}  // namespace qcf

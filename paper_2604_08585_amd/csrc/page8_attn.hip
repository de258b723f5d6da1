// Attention of the newest tokens over a cache in 8-bit pages.
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

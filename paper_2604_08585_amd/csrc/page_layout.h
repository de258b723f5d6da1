// How the attention over a cache in pages divides its contexts: plain code of the host and the device, which tests compile.
#pragma once

#include <stdint.h>
#include <stddef.h>

#include "qcf_pages.h"

#ifdef __HIP__
#define QCF_BOTH __host__ __device__ inline
#else
#define QCF_BOTH inline
#endif

namespace qcf {
int compute_unit_count();
namespace pages {

constexpr int kWaves = 4;                 // of a workgroup; each takes every fourth tile of its part of a context
constexpr int kGrain = 32;                // contexts are divided at multiples of this many tokens
constexpr int kLeast = 4;                 // grains of a range: a tile for every wave

// The contexts, laid end to end in grains (one at least for each), are cut into equal ranges, one to a workgroup, as many as the
// GPU holds at once: a range may end inside a context, and may hold several.  (Units of equal length within each context, the last
// one shorter, left the workgroups unequal where lengths differ: 64 requests of 4K to 12K 480 us, 16 of 1K to 8K 84; @ and @ so.)
struct Division {
  int contexts;                           // B, or B * n_q where every row has pages of its own
  int rows;                               // rows of a context and KV head: (new rows) * heads of the group
  int row_tiles;                          // of 16 rows, in a workgroup: 1 or 2
  int row_blocks;                         // workgroups that take the rows of a context and KV head
  int inner;                              // workgroups of a range: KV heads x row blocks
  int slots;                              // ranges at most
  int64_t most;                           // grains at most
};

inline Division divide(const qcf_layer_desc& L, const qcf_page_cache& c, int32_t B, int32_t n_q, int32_t n_keep) {
  Division d;
  const int G = L.n_q_heads / L.n_kv_heads;
  d.contexts = n_keep ? B * n_q : B;
  d.rows = n_keep ? G : n_q * G;
  d.row_tiles = d.rows > 16 ? 2 : 1;
  d.row_blocks = (d.rows + 16 * d.row_tiles - 1) / (16 * d.row_tiles);
  d.inner = L.n_kv_heads * d.row_blocks;
  d.slots = 2 * compute_unit_count() / d.inner;
  if (d.slots < 1) d.slots = 1;
  const int64_t longest = (int64_t)(n_keep && n_keep < c.max_pages ? n_keep : c.max_pages) * c.page_size;
  d.most = (int64_t)d.contexts * ((longest + kGrain - 1) / kGrain);
  const int64_t ranges = (d.most + kLeast - 1) / kLeast;
  if (d.slots > ranges) d.slots = (int)ranges;
  return d;
}

// Grains of a context and of a range, where there are `total` of them in all.
QCF_BOTH int64_t grains_of(int64_t tokens) { return tokens <= kGrain ? 1 : (tokens + kGrain - 1) / kGrain; }
QCF_BOTH int64_t range_of(int64_t total, int slots) {
  const int64_t even = total >> 31 ? (total + slots - 1) / slots : (int64_t)(((uint32_t)total + (uint32_t)slots - 1u) / (uint32_t)slots);
  return even > kLeast ? even : kLeast;
}

// Partial results, [2 * range + 1 where the context starts in the range, + 0 where it started before][inner][rows of a workgroup]: d
// sums each, then pairs (reference point, sum of the weights).  A range has at most one context of each kind that it does not
// hold as a whole.
inline int part_rows(const Division& d) { return d.rows < 16 * d.row_tiles ? d.rows : 16 * d.row_tiles; }
inline size_t parts(const Division& d) { return (size_t)2 * d.slots * d.inner * part_rows(d); }
inline size_t sums_bytes(const qcf_layer_desc& L, const Division& d) { return parts(d) * L.head_dim * sizeof(float); }
// (one range: nothing is left to be joined)
inline bool divides(const Division& d) { return d.slots > 1; }
inline size_t workspace(const qcf_layer_desc& L, const Division& d) {
  return divides(d) ? sums_bytes(L, d) + parts(d) * 2 * sizeof(float) : 0;
}

}  // namespace pages
}  // namespace qcf

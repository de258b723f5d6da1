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

constexpr int kWaves = 4;                 // of a workgroup; each takes every fourth tile of its unit
constexpr int kUnitStep = 128;            // tokens of a unit are a multiple of this: a tile of 32 for every wave

// Contexts, and the parts of the grid that all of them have.
struct Division {
  int contexts;                           // B, or B * n_q where every row has pages of its own
  int rows;                               // rows of a context and KV head: (new rows) * heads of the group
  int row_tiles;                          // of 16 rows, in a workgroup: 1 or 2
  int row_blocks;                         // workgroups that take the rows of a context and KV head
  int inner;                              // workgroups of a unit: KV heads x row blocks
  int slots;                              // units (of `inner` workgroups) that the GPU holds at once
  int64_t max_units;
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
  const int64_t most = (int64_t)d.contexts * ((longest + kUnitStep - 1) / kUnitStep);
  d.max_units = (int64_t)d.slots + d.contexts;
  if (d.max_units > most) d.max_units = most;
  return d;
}

// Tokens of a unit for `total` tokens in all contexts: no more than slots + contexts units come of it, a context having one at least.
QCF_BOTH int64_t unit_tokens(int64_t total, int slots) {
  const int64_t even = (total + slots - 1) / slots;
  return even <= kUnitStep ? kUnitStep : (even + kUnitStep - 1) / kUnitStep * kUnitStep;
}
QCF_BOTH int64_t units_of(int64_t tokens, int64_t unit) { return tokens <= unit ? 1 : (tokens + unit - 1) / unit; }

// Partial results: [unit][inner][rows of a workgroup] of d sums, then pairs (reference point, sum of the weights).
inline int part_rows(const Division& d) { return d.rows < 16 * d.row_tiles ? d.rows : 16 * d.row_tiles; }
inline size_t sums_bytes(const qcf_layer_desc& L, const Division& d) {
  return (size_t)d.max_units * d.inner * part_rows(d) * L.head_dim * sizeof(float);
}
// (without a second unit anywhere nothing is left to be joined)
inline bool divides(const Division& d) { return d.max_units > d.contexts; }
inline size_t workspace(const qcf_layer_desc& L, const Division& d) {
  return divides(d) ? sums_bytes(L, d) + (size_t)d.max_units * d.inner * part_rows(d) * 2 * sizeof(float) : 0;
}

}  // namespace pages
}  // namespace qcf

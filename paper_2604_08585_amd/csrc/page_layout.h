// How the calls over a cache in pages divide their work: plain code of the host and the device, which tests compile.
#pragma once

#include <stdint.h>
#include <stddef.h>
#include <algorithm>

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
constexpr int kWholeWaves = 8;            // of a workgroup that has a context as a whole
constexpr int kGrain = 32;                // contexts are divided at multiples of this many tokens
constexpr int64_t kThreadsAtMost = 0xffffffff;               // of a launch: a dispatch counts them in 32 bits
constexpr int kTopThreads = 1024;         // of a workgroup that chooses a row's pages
constexpr int kShared = 16 << 20;         // bytes of keys and values from which on two tiles of rows share a workgroup

// Grains of a range: a tile of 32 tokens (bf16) or 16 for every wave.
inline int least_range(const qcf_layer_desc& L) { return L.dtype == QCF_DTYPE_BF16 ? 4 : 2; }

// The contexts, laid end to end in grains (one at least for each), are cut into equal ranges, one to a workgroup, as many as the
// GPU holds at once: a range may end inside a context, and may hold several.  (Units of equal length within each context, the last
// one shorter, left the workgroups unequal where lengths differ: 64 requests of 4K to 12K 480 us, 16 of 1K to 8K 84; 399 and 71
// with ranges when they came in, 395 and 70 now.)
struct Division {
  int contexts;                           // B, or B * n_q where every row has pages of its own
  int rows;                               // rows of a context and KV head: (new rows) * heads of the group
  int row_tiles;                          // of 16 rows, in a workgroup: 1 or 2
  int row_blocks;                         // workgroups that take the rows of a context and KV head
  int inner;                              // workgroups of a range: KV heads x row blocks
  int slots;                              // ranges at most
  int least;                              // grains of a range at least (a power of two)
  int pad;                                // grains that the beginning of a context counts for
  int64_t most;                           // grains at most
  bool whole;                             // a workgroup to every context, KV head and row block: nothing is divided
};

// Whether workgroups of eight waves take whole contexts, in one launch, or four waves each range of them, in two.  The second launch
// takes 4 to 5 us, a compute unit reads 50 to 60 GB/s at most; what is saved by dividing shrinks as more workgroups share the
// memory.  us on the GPU, whole and divided.  Heads of 128 in bf16: 8 workgroups (a request, 8 KV heads) of 512 tokens 10.0 and 9.5, of
// 1024 15.3 and 10.3; 64 of up to 768 12.8 and 12.5, 1024 16.0 and 13.4; 128 of up to 1024 17.6 and 20.6, 1536 21.4 and 23.5, 2048 27.9 and
// 28.7, 4096 48.1 and 42.1; 512 of up to 1024 40.0 and 42.7, 4096 161 and 159.  Heads of 64: 16 of up to 1024 11.0 and 12.9, 1536 12.8 and
// 13.1, 2048 16.3 and 11.1.  In float32, heads of 64: 2 of 512 10.8 and 9.7, 4 of up to 512 10.9 and 12.3, 1024 15.9 and 10.5.  Over eight
// shapes, 1 to 64 requests and 256 to 8192 tokens the rule is 0.5 % behind the better of the two on average (272 KB in place of 290:
// 0.6 %, 350: 0.9 %); at its border it takes the worse one by up to 11 % (19 % in float32), and by 25 % for 2048 workgroups of up to 256 tokens.
inline bool takes_whole(const qcf_layer_desc& L, int64_t workgroups, int64_t longest) {
  const int64_t bytes = longest * 2 * L.head_dim * (L.dtype == QCF_DTYPE_BF16 ? 2 : 4);
  const int64_t alone = std::max<int64_t>(30, 200 - workgroups * 256 / compute_unit_count());      // of 200
  return bytes * alone <= (int64_t)((L.dtype == QCF_DTYPE_BF16 ? 290 : 240) << 10) * 200;
}

inline Division divide(const qcf_layer_desc& L, const qcf_page_cache& c, int32_t B, int32_t n_q, int32_t n_keep) {
  Division d;
  const int G = L.n_q_heads / L.n_kv_heads;
  d.contexts = n_keep ? B * n_q : B;
  d.rows = n_keep ? G : n_q * G;
  // More than 16 rows: two tiles of them share what a wave reads, unless there is little to read in all (by the width of the table):
  // then a second workgroup finds it in the L2, and the first is done sooner.  64 / 2 heads of 128, us, two tiles and one: one request of
  // 4096 tokens 14.6 and 12.5, of 16384 18.9 and 19.5; 8 of up to 1024 15.9 and 13.5, of up to 4096 18.9 and 23.5.  32 / 1 heads: one
  // request of 16384 tokens 18.1 and 16.0, 8 of up to 4096 16.6 and 16.4, 64 of up to 1024 19.2 and 16.6, of up to 4096 32.6 and 43.7.
  const int64_t longest = (int64_t)(n_keep && n_keep < c.max_pages ? n_keep : c.max_pages) * c.page_size;
  const double read = (double)d.contexts * (double)longest * L.n_kv_heads * 2 * L.head_dim * (L.dtype == QCF_DTYPE_BF16 ? 2 : 4);
  d.row_tiles = d.rows > 16 && read > kShared ? 2 : 1;
  d.row_blocks = (d.rows + 16 * d.row_tiles - 1) / (16 * d.row_tiles);
  d.inner = L.n_kv_heads * d.row_blocks;
  d.slots = (d.row_tiles == 1 || L.head_dim == 64 ? 2 : 1) * compute_unit_count() / d.inner;       // (two waves to a SIMD, or one)
  if (d.slots < 1) d.slots = 1;
  d.most = (int64_t)d.contexts * ((longest + kGrain - 1) / kGrain);
  d.least = least_range(L);
  // (four drafts of 8 requests of 2K to 6K tokens, 32 rows, before later steps, which brought 47 to 44 us: 53.0 us without, 48.1 with 12,
  // 47.1 with 18, 50.0 with 28; two workgroups on a compute unit cover for each other, 0 to 9 are the same there)
  d.pad = d.contexts > 1 && d.row_tiles == 2 ? 16 : 0;
  d.whole = d.row_tiles == 1 && takes_whole(L, (int64_t)d.contexts * d.inner, longest);
  const int64_t ranges = (d.most + d.least - 1) / d.least;
  if (d.slots > ranges) d.slots = (int)ranges;
  return d;
}

// Grains of a context and of a range, where there are `total` of them in all.
QCF_BOTH int64_t grains_of(int64_t tokens) { return tokens <= kGrain ? 1 : (tokens + kGrain - 1) / kGrain; }
QCF_BOTH int64_t range_of(int64_t total, int slots, int least) {
  const int64_t even = total >> 31 ? (total + slots - 1) / slots : (int64_t)(((uint32_t)total + (uint32_t)slots - 1u) / (uint32_t)slots);
  return even > least ? even : least;
}

// Partial results, [2 * range + 1 where the context starts in the range, + 0 where it started before][inner][rows of a workgroup]: d
// sums each, then pairs (reference point, sum of the weights).  A range has at most one context of each kind that it does not
// hold as a whole.
inline int part_rows(const Division& d) { return d.rows < 16 * d.row_tiles ? d.rows : 16 * d.row_tiles; }
inline size_t parts(const Division& d) { return (size_t)2 * d.slots * d.inner * part_rows(d); }
inline size_t sums_bytes(const qcf_layer_desc& L, const Division& d) { return parts(d) * L.head_dim * sizeof(float); }
// (one range: nothing is left to be joined)
inline bool divides(const Division& d) { return !d.whole && d.slots > 1; }
inline size_t workspace(const qcf_layer_desc& L, const Division& d) {
  return divides(d) ? sums_bytes(L, d) + parts(d) * 2 * sizeof(float) : 0;
}

// Units of an append, one to each page that gets rows: those of request b start at row_off[b] / page + 2 b, which leaves room for
// every page that its rows can touch (n rows touch at most floor((n - 1) / page) + 2).
inline int64_t append_units(const qcf_page_cache& c, int32_t B, int64_t total_rows) { return total_rows / c.page_size + 2 * (int64_t)B; }

// KV heads of an append's workgroup: a power of two of them, whose vectors of a row fill a wave at most, as long as every compute
// unit has a workgroup (two where a page has 256 rows).  More share their (cos, sin) and whole rows, fewer give a short call more
// workgroups: 8 KV heads of 128, us, with one head, by this rule and with all eight: 500 rows 7.9, 8.1 and 14.8, 8000 in pages of 64
// 53.1, 43.8 and 80.8, 256 requests of one row 20.0, 8.7 and 9.4; 16 requests of 1000 to 2000 in pages of 256 163 (208 with one workgroup
// to a compute unit), in pages of 128 143 (156 with two).  About three workgroups to a compute unit, which fill it once, are slower
// than twice as many: 4 requests of 2000 to 4000 rows in pages of 16 84 and 75, 32 of 1000 to 2000 in pages of 64 303 and 270.
inline int append_heads(const qcf_layer_desc& L, const qcf_page_cache& c, int64_t units) {
  const int per_row = L.head_dim / 2 / (L.dtype == QCF_DTYPE_BF16 ? 8 : 4);            // 16-byte vectors of half a row
  const int cus = compute_unit_count(), wanted = (c.page_size >= 256 ? 2 : 1) * cus;
  int heads = 1;
  while (L.n_kv_heads % (2 * heads) == 0 && 2 * heads * per_row <= 64 && units * (L.n_kv_heads / (2 * heads)) >= wanted)
    heads *= 2;
  const int64_t groups = units * (L.n_kv_heads / heads);
  if (heads > 1 && 2 * groups > 5 * cus && groups < 4 * cus) heads /= 2;
  return heads;
}

}  // namespace pages
}  // namespace qcf

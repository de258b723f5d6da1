// How the calls over a cache in pages divide their work: plain code of the host and the device, which tests compile.
#pragma once

#include <stdint.h>
#include <stddef.h>
#include <algorithm>

#include "qcf_pages8.h"

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

// Bytes of an element of the layer; the pages' own may be smaller.
inline int layer_elem(const qcf_layer_desc& L) { return L.dtype == QCF_DTYPE_BF16 ? 2 : 4; }

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
  int inner;                              // KV heads x row blocks of a range
  int heads;                              // KV heads that a workgroup of a range takes side by side
  int slots;                              // ranges at most
  int least;                              // grains of a range at least (a power of two)
  int pad;                                // grains that the beginning of a context counts for
  int64_t most;                           // grains at most
  bool whole;                             // a workgroup to every context, KV head and row block: nothing is divided
};

// Workgroups of four waves that a compute unit holds at once.  (8-bit heads of 64 leave room for a third: 64 requests of 4K to 12K tokens 113
// us, 123 with two.  Those of 128 would spill registers: 234 us, 203 with two.)
constexpr int at_once(int head_dim, int row_tiles, bool eight) {
  return head_dim == 64 ? (eight && row_tiles == 1 ? 3 : 2) : row_tiles == 1 || eight ? 2 : 1;
}

// KV heads whose rows lie next to each other and are read side by side, by the waves of a workgroup: 256 bytes in a row, as a row of bf16
// has.  read: bytes of the keys and values at most; where they are few, the joins of twice as many parts cost more.  us, pages that keep a
// token's 8-bit heads together, a head to a workgroup and side by side: heads of 128, 64 requests of 4K to 12K tokens 239 and 206, one of 128K
// 70 and 61, of 30K (61 MB) 23.3 and 22.9, four new rows 250 and 221, 71 and 65, 8 requests of up to 6K 32.1 and 32.5;
// heads of 64 191 and 130, one of 30K 22.3 and 20.5, of 3K 11.9 and 14.5.
inline int side_by_side(const qcf_layer_desc& L, const qcf_page_cache& c, int elem, double read) {
  const int heads = 256 / L.head_dim;
  const bool worth = read > (L.head_dim == 128 ? 4.0 : 1.0) * kShared;
  return elem == 1 && worth && c.head_stride == L.head_dim && L.n_kv_heads % heads == 0 ? heads : 1;
}

// Whether workgroups of eight waves take whole contexts, in one launch, or four waves each range of them, in two.  The second launch
// takes 4 to 5 us, a compute unit reads 50 to 60 GB/s at most; what is saved by dividing shrinks as more workgroups share the
// memory.  us on the GPU, whole and divided.  Heads of 128 in bf16: 8 workgroups (a request, 8 KV heads) of 512 tokens 10.0 and 9.5, of
// 1024 15.3 and 10.3; 64 of up to 768 12.8 and 12.5, 1024 16.0 and 13.4; 128 of up to 1024 17.6 and 20.6, 1536 21.4 and 23.5, 2048 27.9 and
// 28.7, 4096 48.1 and 42.1; 512 of up to 1024 40.0 and 42.7, 4096 161 and 159.  Heads of 64: 16 of up to 1024 11.0 and 12.9, 1536 12.8 and
// 13.1, 2048 16.3 and 11.1.  In float32, heads of 64: 2 of 512 10.8 and 9.7, 4 of up to 512 10.9 and 12.3, 1024 15.9 and 10.5.  Over eight
// shapes, 1 to 64 requests and 256 to 8192 tokens the rule is 0.5 % behind the better of the two on average (272 KB in place of 290:
// 0.6 %, 350: 0.9 %); at its border it takes the worse one by up to 11 % (19 % in float32), and by 25 % for 2048 workgroups of up to 256 tokens.
// 8-bit pages: a wave's tile takes about as long whatever its width, so that the rule goes by tokens; and where there are more workgroups
// than compute units, whose second round leaves some idle, it divides from fewer on.  us, whole and divided, lengths from a quarter of the
// longest on.  One new row, bf16, heads of 128: 8 workgroups of up to 1024 tokens 11.0 and 11.3, 2048 15.0 and 11.2; 192 of up to 2000 22.0
// and 23.8, 4000 39.7 and 36.4; 320 of up to 1000 22.9 and 22.2, 4000 64.4 and 53.9; 512 of up to 1000 26.8 and 30.3, 8000 150 and 134; 1024 of
// up to 1000 53.4 and 54.9, 2000 84.0 and 80.9.  Heads of 64: 8 of 1024 8.7 and 10.7, 2048 11.8 and 11.0; 128 of up to 3000 22.2 and 20.9; 320
// of up to 2000 21.7 and 22.3, 4000 38.8 and 32.6; 1024 of up to 2000 45.7 and 50.9, 8000 151 and 141.  float32, half as many tokens: heads of
// 64, 320 of up to 500 16.1 and 18.3, 1500 34.8 and 29.8; of 128, 1024 of up to 500 54.4 and 58.4, 1000 91.6 and 84.8.
// Several new rows, which a join takes longer for: 512 workgroups, heads of 128, of up to 2000 53.2 and 58.2, 4000 88.1 and 89.4; 320 of up
// to 4000 70.0 and 64.1; heads of 64, 512 of up to 4000 50.3 and 53.7.
// Heads that only ranges take side by side, one row: heads of 128, 256 of up to 5000 63.7 and 54.6, 320 of up to 4000 73.9 and 53.8, 2048 of
// up to 300 57.9 and 47.4; of 64, 256 of up to 2500 26.4 and 25.8, 320 of up to 1000 17.4 and 19.0, 1024 of up to 1000 33.9 and 32.0, 4000 120
// and 89.1.  Four rows, heads of 128: 256 of up to 2500 38.2 and 43.4, 4000 54.6 and 55.3; 512 of up to 1000 34.8 and 37.5, 3000 80.6 and
// 76.9; 2048 of up to 300 78.9 and 73.2, 2000 200 and 182.  At its borders the rule takes the worse one by up to 6 % (float32, heads of 64:
// 15 %).
inline bool takes_whole(const qcf_layer_desc& L, int64_t workgroups, int64_t longest, int elem, int heads, bool several) {
  if (elem == 1) {
    const int64_t units = compute_unit_count();
    const bool one_round = workgroups <= units, wide = L.head_dim == 128;
    int64_t most = one_round ? 1400 * 200 / (200 - workgroups * 154 / units) : several ? (wide ? 3072 : 4096) : wide ? 1024 : 3072;
    if (heads > 1 && !several) most = std::min<int64_t>(most, one_round ? 2048 : wide ? 0 : 1024);
    if (heads > 1 && several && wide) most = std::min(most, one_round ? 4096 : 2048 * units / workgroups);
    return (L.dtype == QCF_DTYPE_BF16 ? longest : 2 * longest) <= most;
  }
  const int64_t bytes = longest * 2 * L.head_dim * elem;
  const int64_t alone = std::max<int64_t>(30, 200 - workgroups * 256 / compute_unit_count());      // of 200
  return bytes * alone <= (int64_t)((L.dtype == QCF_DTYPE_BF16 ? 290 : 240) << 10) * 200;
}

// elem: bytes of a stored element
inline Division divide(const qcf_layer_desc& L, const qcf_page_cache& c, int32_t B, int32_t n_q, int32_t n_keep, int elem) {
  Division d;
  const int G = L.n_q_heads / L.n_kv_heads;
  d.contexts = n_keep ? B * n_q : B;
  d.rows = n_keep ? G : n_q * G;
  // More than 16 rows: two tiles of them share what a wave reads, unless there is little to read in all (by the width of the table):
  // then a second workgroup finds it in the L2, and the first is done sooner.  64 / 2 heads of 128, us, two tiles and one: one request of
  // 4096 tokens 14.6 and 12.5, of 16384 18.9 and 19.5; 8 of up to 1024 15.9 and 13.5, of up to 4096 18.9 and 23.5.  32 / 1 heads: one
  // request of 16384 tokens 18.1 and 16.0, 8 of up to 4096 16.6 and 16.4, 64 of up to 1024 19.2 and 16.6, of up to 4096 32.6 and 43.7.
  const int64_t longest = (int64_t)(n_keep && n_keep < c.max_pages ? n_keep : c.max_pages) * c.page_size;
  const double read = (double)d.contexts * (double)longest * L.n_kv_heads * 2 * L.head_dim * elem;
  // (8-bit heads of 128: from more bytes on.  64 / 8 heads, us, two tiles and one: four drafts of 8 requests of 2K to 6K tokens 38.4 and 36.6,
  // of 64 of 4K to 12K 262 and 301, of one of 128K 76.4 and 80.6; 32 / 8 heads, 8 drafts of 16 requests of up to 8K 60.0 and 63.9.)
  const bool wide8 = elem == 1 && L.head_dim == 128;
  d.row_tiles = d.rows > 16 && read > (wide8 ? 8.0 : 1.0) * kShared ? 2 : 1;
  d.row_blocks = (d.rows + 16 * d.row_tiles - 1) / (16 * d.row_tiles);
  d.inner = L.n_kv_heads * d.row_blocks;
  d.heads = n_keep || d.row_tiles > 1 ? 1 : side_by_side(L, c, elem, read);
  d.slots = at_once(L.head_dim, d.row_tiles, elem == 1) * compute_unit_count() * d.heads / d.inner;       // (two waves to a SIMD, or one)
  if (d.slots < 1) d.slots = 1;
  d.most = (int64_t)d.contexts * ((longest + kGrain - 1) / kGrain);
  d.least = least_range(L);
  // (four drafts of 8 requests of 2K to 6K tokens, 32 rows, before later steps, which brought 47 to 44 us: 53.0 us without, 48.1 with 12,
  // 47.1 with 18, 50.0 with 28; two workgroups on a compute unit cover for each other, 0 to 9 are the same there)
  d.pad = d.contexts > 1 && d.row_tiles == 2 ? 16 : 0;
  d.whole = d.row_tiles == 1 && takes_whole(L, (int64_t)d.contexts * d.inner, longest, elem, d.heads, n_q > 1 && !n_keep);
  const int64_t ranges = (d.most + d.least - 1) / d.least;
  if (d.slots > ranges) d.slots = (int)ranges;
  return d;
}
inline Division divide(const qcf_layer_desc& L, const qcf_page_cache& c, int32_t B, int32_t n_q, int32_t n_keep) {
  return divide(L, c, B, n_q, n_keep, layer_elem(L));
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

// Units of an append to 8-bit pages: blocks of 16 tokens; where the pages have bounds, which one workgroup joins, pages.  (24K rows of 16
// requests in pages of 256, 32 / 8 heads of 128: 118 us, 133 in parts of 64 tokens, 145 in pages.)
inline int append8_tokens(const qcf_page_cache& c) { return c.bounds ? c.page_size : QCF_PAGE8_BLOCK; }
inline int64_t append8_units(const qcf_page_cache& c, int32_t B, int64_t total_rows) { return total_rows / append8_tokens(c) + 2 * (int64_t)B; }
// KV heads of its workgroup: they share (cos, sin) and whole rows; fewer give a short call, and long pages, more workgroups.  us with one, two
// and four (32 / 8 heads of 128, blocks): 36K rows 191, 156, 158; 256 requests of one row 18.5, 12.8, 10.7; 32 of 50 to 100 17.2, 15.1,
// 15.2 (two by this rule); 500 rows 9.6, 9.6, 10.4 (one); pages with 256 rows, 24K of them 145, 173, 233 (one), with 64, 6K of them 42.8, 42.3, 55.7 (one).
inline int append8_heads(const qcf_layer_desc& L, const qcf_page_cache& c, int32_t B, int64_t total_rows) {
  const int tokens = append8_tokens(c);
  const int64_t workgroups = (total_rows / tokens + B) * L.n_kv_heads;               // that get rows, about, one head each
  const int64_t wanted = (int64_t)(tokens > QCF_PAGE8_BLOCK && total_rows > 16 * (int64_t)B ? 8 : 2) * compute_unit_count();
  int heads = 1;
  while (heads < kWaves && L.n_kv_heads % (2 * heads) == 0 && workgroups / (2 * heads) >= wanted) heads *= 2;
  return heads;
}

}  // namespace pages
}  // namespace qcf

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
#include "qcf_internal.h"
#include "page_layout.h"

namespace qcf {
namespace {

constexpr float kLn2 = 0.6931471805599453f;
// A row's reference point moves where a logit is more than 8 above it (in powers of two): weights are up to 256 then, and most
// tiles neither exchange their maxima nor scale what has been summed.
constexpr float kRoom = 8.f;

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

enum Mode { kOne = 0, kList = 1, kSeveral = 2 };         // one new row to a context, pages of its own, or several new rows

struct PageAttnArgs {
  qcf_page_cache c;
  const void* q;
  const int32_t* seen;
  const int32_t* list;
  int n_keep, n_q, H, Hkv, G, log2_page;
  int contexts, rows, inner, slots, least, pad, part_rows;
  float scale, scale_low;                                // log2(e) / sqrt(d), rounded down, and what that leaves (positive, so that a
                                                         // product that is infinite keeps its sign)
  void* o;
  float* lse;
  float* part_o;
  float2* part_ml;
};

// Tokens that context x covers: what its rows see, or as many entries of its list as the row sees pages.  What a list has behind
// these is mostly empty; the last part of a context looks through it (list_end).  16 rows of 32 to 3000 tokens with lists of 256
// pages of 16: selection and attention 37.4 us without that, 39.6 with it, 47.5 with the lists divided as a whole.
__device__ __forceinline__ int64_t context_tokens(const PageAttnArgs& a, int x) {
  const int64_t most = (int64_t)a.c.max_pages << a.log2_page;
  if (a.list) {
    const int64_t seen = min((int64_t)max(a.seen[x], 0), most);
    return min((seen + a.c.page_size - 1) >> a.log2_page, (int64_t)a.n_keep) << a.log2_page;
  }
  int seen = 0;
  for (int i0 = 0; i0 < a.n_q; i0 += 4)                  // (four loads on their way together)
#pragma unroll
    for (int i = 0; i < 4; ++i) seen = max(seen, a.seen[(int64_t)x * a.n_q + min(i0 + i, a.n_q - 1)]);
  return min((int64_t)seen, most);
}

// The end of the last part of a context of `tokens`.
template <int MODE>
__device__ __forceinline__ int64_t list_end(const PageAttnArgs& a, int64_t tokens) {
  return MODE == kList && tokens > 0 ? (int64_t)a.n_keep << a.log2_page : tokens;
}

template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}
// Inclusive sum over the lanes of a wave: within rows (row_shr), then across them (row_bcast).
__device__ __forceinline__ uint32_t wave_incl(uint32_t x) {
  x += dpp<0x111>(x); x += dpp<0x112>(x); x += dpp<0x114>(x); x += dpp<0x118>(x);
  x += dpp<0x142, 0xa>(x);
  return x + dpp<0x143, 0xc>(x);
}
__device__ __forceinline__ uint32_t from_lane(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }

// The contexts in grains, end to end, `pad` of them in front of each: what a workgroup that has begun one context pays for another.
// Every wave works them out by itself; the first 64 stay in its lanes.
struct Contexts {
  uint32_t tokens, grains;             // of context `lane`
  uint32_t room, incl;                 // grains with the padding, and the sum so far (64 of less than 2^26)
  int64_t range;                       // grains of a range
  int pad;
  bool apart;                          // no range has two contexts
};
struct Place {
  int x;                               // context
  int64_t start, grains;               // its first grain (behind the padding), and how many it has
};

__device__ __forceinline__ Contexts contexts_of(const PageAttnArgs& a, int lane) {
  Contexts c;
  c.pad = a.pad;
  c.apart = false;
  if (a.contexts == 1) {                                 // (the latency of one request: no sums over the lanes)
    c.tokens = (uint32_t)context_tokens(a, 0);
    c.grains = c.room = c.incl = (uint32_t)pages::grains_of(c.tokens);
    c.range = pages::range_of(c.grains, a.slots, a.least);
    return c;
  }
  c.tokens = lane < a.contexts ? (uint32_t)context_tokens(a, lane) : 0u;
  c.grains = lane < a.contexts ? (uint32_t)pages::grains_of(c.tokens) : 0u;
  c.room = lane < a.contexts ? c.grains + a.pad : 0u;
  c.incl = wave_incl(c.room);
  if (a.contexts <= 64) {
    // little work: every context begins a range of its own if there are enough of them (two parts in a row take a workgroup
    // twice the latency: five requests of up to 600 tokens in float32 13.6 us, 10.4 so)
    const uint32_t room = (c.grains + a.least - 1) & ~(uint32_t)(a.least - 1), incl = wave_incl(room);
    if (from_lane(incl, 63) <= (uint64_t)a.least * a.slots) {
      c.room = room;
      c.incl = incl;
      c.pad = 0;
      c.apart = true;
    }
  }
  int64_t total = from_lane(c.incl, 63);
  for (int x0 = 64; x0 < a.contexts; x0 += 64)
    total += from_lane(wave_incl(x0 + lane < a.contexts ? (uint32_t)pages::grains_of(context_tokens(a, x0 + lane)) + a.pad : 0u), 63);
  c.range = pages::range_of(total, a.slots, a.least);
  return c;
}
// The context whose grain or padding a position is (x -1: none), or context x itself.
template <bool OF>
__device__ __forceinline__ Place place_of(const PageAttnArgs& a, const Contexts& c, int64_t at, int x, int lane) {
  Place p = {-1, 0, 0};
  uint32_t n = c.grains, room = c.room, incl = c.incl;
  for (int x0 = 0; x0 < a.contexts; x0 += 64) {
    if (x0 > 0) {
      n = x0 + lane < a.contexts ? (uint32_t)pages::grains_of(context_tokens(a, x0 + lane)) : 0u;
      room = n > 0u ? n + a.pad : 0u;
      incl = wave_incl(room);
    }
    const uint64_t hit = __ballot(n > 0u && (OF ? x0 + lane == x : at < p.start + incl));
    if (hit) {
      const int l = __builtin_ctzll(hit);
      p.x = x0 + l;
      p.grains = from_lane(n, l);
      p.start += from_lane(incl, l) - from_lane(room, l) + (uint32_t)c.pad;
      return p;
    }
    p.start += from_lane(incl, 63);
  }
  return p;
}

// 64 entries of a context's pages, one to a lane, and the tile's part of them.
struct Window {
  int first;               // index of lane 0's page in the context's order
  int phys, page;          // lane's page: number in the pool (-1: not there), and in the request
};

template <typename T, int D, int RT, int MODE, int WAVES>
struct Walk {
  static constexpr bool kHalf = sizeof(T) == 2;
  static constexpr int kSub = kHalf ? 2 : 1;             // parts of 16 tokens of a tile; a part lies in one page
  static constexpr int kTokens = 16 * kSub, kS = 4 * kSub;             // tokens of a tile, logits of a lane
  static constexpr int kLoads = kHalf ? D / 32 : D / 16;               // 16-byte loads of a lane for 16 tokens' keys
  static constexpr int kE = D / 16;                                    // 16-element slices of the output
  static constexpr int kV = kHalf ? 8 : 4 * (D / 64);                  // value loads of a lane
  static constexpr int kVWords = kHalf && D == 64 ? 2 : 4;
  static constexpr int kStep = WAVES * kTokens;                        // tokens that the workgroup's waves take side by side
  typedef uint32_t vec_v __attribute__((ext_vector_type(kVWords)));

  struct Tile {
    u32x4 k[kSub][kLoads];
    vec_v v[kV];
    int base[kSub];                                      // request's number of its first token (-1: not there)
  };

  const PageAttnArgs& a;
  const int lane, quad, col, g;
  int x, b;                                              // context, request
  int64_t end;                                           // of the workgroup's part, in the context's order
  int count;                                             // pages that a row sees (listed pages of higher numbers are none)
  Window w;
  u32x4 q[RT][kLoads];
  int lim[RT];                                           // tokens that the lane's row sees
  int lim_lo, lim_hi;                                    // least and largest of the rows that see anything
  float m[RT], l[RT];
  bool any[RT];
  floatx4 acc[RT][kE];

  __device__ __forceinline__ Walk(const PageAttnArgs& args, int lane_, int g_)
      : a(args), lane(lane_), quad(lane_ >> 4), col(lane_ & 15), g(g_) {}

  __device__ __forceinline__ void open(int first) {
    w.first = first;
    int p = first + lane;
    if constexpr (MODE == kList) p = p < a.n_keep ? a.list[((int64_t)x * a.Hkv + g) * a.n_keep + p] : -1;
    // (the table is asked before it is known how many of its pages are seen)
    const int phys = p >= 0 && p < a.c.max_pages ? a.c.table[(int64_t)b * a.c.max_pages + p] : -1;
    w.page = p;
    w.phys = p < count && phys < a.c.n_pages ? phys : -1;
  }

  // where the parts of a tile are; a page that is not there: page 0 is read instead, and nothing of it used
  struct Where {
    int base[kSub];
    int64_t off[kSub];
  };
  __device__ __forceinline__ Where find(int64_t at) {
    const int mask = a.c.page_size - 1;
    const int last = (int)((at + kTokens - 1) >> a.log2_page);
    if (last - w.first >= 64) open((int)(at >> a.log2_page));
    Where r;
#pragma unroll
    for (int h = 0; h < kSub; ++h) {
      const int64_t mine = at + 16 * h;
      const int i = (int)(mine >> a.log2_page) - w.first;
      const int slot = (int)mine & mask;
      const int phys = __builtin_amdgcn_readlane(w.phys, i);
      const int page = __builtin_amdgcn_readlane(w.page, i);
      r.base[h] = phys >= 0 && mine < end ? (page << a.log2_page) + slot : -1;
      r.off[h] = max(phys, 0) * a.c.page_stride + g * a.c.head_stride + slot * a.c.slot_stride;
    }
    return r;
  }
  __device__ __forceinline__ void load_keys(Tile& t, const Where& r) const {
    const uint32_t stride = (uint32_t)a.c.slot_stride * sizeof(T);
#pragma unroll
    for (int h = 0; h < kSub; ++h) {
      const char* k = reinterpret_cast<const char*>(static_cast<const T*>(a.c.k) + r.off[h]);
#pragma unroll
      for (int f = 0; f < kLoads; ++f) t.k[h][f] = *reinterpret_cast<const u32x4*>(k + (col * stride + 16 * quad + 64 * f));
    }
  }
  __device__ __forceinline__ void load_values(Tile& t, const Where& r) const {
    const uint32_t stride = (uint32_t)a.c.slot_stride * sizeof(T);
#pragma unroll
    for (int h = 0; h < kSub; ++h) {
      const char* v = reinterpret_cast<const char*>(static_cast<const T*>(a.c.v) + r.off[h]);
      t.base[h] = r.base[h];
#pragma unroll
      for (int j = 0; j < kV / kSub; ++j) {
        const int token = kHalf ? j : j & 3, part = kHalf ? 0 : j >> 2;
        t.v[kHalf ? 4 * h + j : j] =
            *reinterpret_cast<const vec_v*>(v + ((4 * quad + token) * stride + col * (uint32_t)sizeof(vec_v) + 256 * part));
      }
    }
  }
  __device__ __forceinline__ void load(Tile& t, int64_t at) {
    const Where r = find(at);
    load_keys(t, r);
    load_values(t, r);
  }

  // The wave's tile at `at`; of a list, the next one before `stop` that has a page.
  __device__ __forceinline__ int64_t tile_at(int64_t at, int64_t stop) {
    if constexpr (MODE == kList)
      for (; at < stop; at += kStep) {
        const Where r = find(at);
        if (r.base[0] >= 0 || r.base[kSub - 1] >= 0) break;
      }
    return at;
  }

  // products of the tile's values with the weights, added to c
  template <int N>
  __device__ __forceinline__ void values(const Tile& t, const float (&p)[N][kS], floatx4 (&c)[N][kE]) const {
    if constexpr (kHalf) {
      // weights as three bf16 terms, which add up to the float: cut off, what that left cut off, and the rest.  (The second and the
      // third term of a weight that is not 0 are kept from being 0, so that an infinite value comes out infinite and not NaN.)  With
      // two terms, 16 bits, five to seventeen times as many results were off the nearest bf16 value (16 requests of 1K to 8K tokens:
      // 0.41 % and 0.04 %, one of 128K 0.42 % and 0.02 %) in 0 to 1 % less time (64 of 4K to 12K 397.3 and 398.1 us).
      bf16x8 term[3][N];
#pragma unroll
      for (int r = 0; r < N; ++r) {
        u32x4 w[3];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x = p[r][2 * i], y = p[r][2 * i + 1];
          const float least_x = fminf(x, 0x1p-126f), least_y = fminf(y, 0x1p-126f);
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            w[n][i] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
            x = fmaxf(x - __uint_as_float(__float_as_uint(x) & 0xffff0000u), least_x);
            y = fmaxf(y - __uint_as_float(__float_as_uint(y) & 0xffff0000u), least_y);
          }
          w[2][i] = cvt_pk_bf16(x, y);
        }
#pragma unroll
        for (int n = 0; n < 3; ++n) term[n][r] = __builtin_bit_cast(bf16x8, w[n]);
      }
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        u32x4 vt;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          vt[i] = __builtin_amdgcn_perm(t.v[2 * i + 1][e / 2], t.v[2 * i][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
        const bf16x8 va = __builtin_bit_cast(bf16x8, vt);
#pragma unroll
        for (int r = 0; r < N; ++r)
#pragma unroll
          for (int n = 0; n < 3; ++n) c[r][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, term[n][r], c[r][e], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int j = 0; j < kV; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int r = 0; r < N; ++r)
            c[r][4 * (j >> 2) + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.v[j][e]), p[r][j & 3], c[r][4 * (j >> 2) + e], 0, 0, 0);
    }
  }

  __device__ __forceinline__ int token(const Tile& t, int i) const { return t.base[i >> 2] + 4 * quad + (i & 3); }

  // values of tokens from `limit` on, and of pages that are not there, become 0
  __device__ __forceinline__ void clear(Tile& t, int limit) const {
#pragma unroll
    for (int j = 0; j < kV; ++j) {
      const int i = kHalf ? j : j & 3;
      const bool ok = t.base[i >> 2] >= 0 && token(t, i) < limit;
#pragma unroll
      for (int e = 0; e < kVWords; ++e) t.v[j][e] = ok ? t.v[j][e] : 0u;
    }
  }

  // CAREFUL: the tile may have tokens that only some of the rows see
  // (after_logits(): the keys' registers are free)
  template <bool CAREFUL, typename F>
  __device__ __forceinline__ void step(Tile& t, F&& after_logits) {
    float s[RT][kS];
#pragma unroll
    for (int h = 0; h < kSub; ++h)
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        floatx4 z = {0.f, 0.f, 0.f, 0.f};
        if constexpr (kHalf) {
#pragma unroll
          for (int f = 0; f < kLoads; ++f)
            z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, t.k[h][f]), __builtin_bit_cast(bf16x8, q[r][f]), z, 0, 0, 0);
        } else {
          // (two sums side by side: half the chain, and less rounding)
          floatx4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int f = 0; f < kLoads; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              floatx4& sum = e & 1 ? y : z;
              sum = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.k[h][f][e]), __uint_as_float(q[r][f][e]), sum, 0, 0, 0);
            }
          z += y;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s[r][4 * h + i] = z[i];
      }
    after_logits();
    // a tile that every row sees as a whole needs no mask
    bool whole = true;
#pragma unroll
    for (int h = 0; h < kSub; ++h) whole = whole && t.base[h] >= 0 && t.base[h] + 16 <= lim_lo;
    if (!whole) clear(t, lim_hi);
    float p[RT][kS];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      if (whole) any[r] = true;
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < kS; ++i) {
        if (!whole) {
          const bool ok = t.base[i >> 2] >= 0 && token(t, i) < lim[r];
          any[r] = any[r] || ok;
          top = ok ? fmaxf(top, s[r][i]) : top;
        } else {
          top = fmaxf(top, s[r][i]);
        }
      }
      top *= a.scale;
      if (__any(top > m[r] + kRoom)) {
        typedef unsigned u2v __attribute__((ext_vector_type(2)));
        u2v y = __builtin_amdgcn_permlane16_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = fmaxf(__uint_as_float(y.x), __uint_as_float(y.y));
        y = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = fmaxf(__uint_as_float(y.x), __uint_as_float(y.y));
        const float next = top > m[r] + kRoom ? top : m[r];          // (each row by itself)
        const float f = next == m[r] ? 1.f : __builtin_amdgcn_exp2f(m[r] - next);
        m[r] = next;
        l[r] *= f;
#pragma unroll
        for (int e = 0; e < kE; ++e) acc[r][e] *= f;
      }
      const float ref = m[r] == -INFINITY ? 0.f : m[r];               // (all logits so far -inf: weights of 0, not NaN)
#pragma unroll
      for (int i = 0; i < kS; ++i) {
        // (float32: the scale as two floats, so that a large logit does not lose the bits behind the first)
        const float from = kHalf ? -ref : __builtin_fmaf(s[r][i], a.scale_low, -ref);
        float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r][i], a.scale, from));
        if (!whole) e = t.base[i >> 2] >= 0 && token(t, i) < lim[r] ? e : 0.f;
        p[r][i] = e;
        l[r] += e;
      }
    }
    if (!CAREFUL || whole) {
      values(t, p, acc);
      return;
    }
    // one new row after the other, with the values that it does not see cleared: 0 times a value that is not finite is not 0
    const int last = min(row0 + 16 * RT, a.rows) - 1;
    for (int i = row0 / a.G; i <= last / a.G; ++i) {
      const int at = max(i * a.G, row0) - row0;          // a row of it in the workgroup
      Tile mine = t;
      clear(mine, __builtin_amdgcn_readlane(RT == 2 && at >= 16 ? lim[RT - 1] : lim[0], at & 15));
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const bool here = row_of(r) / a.G == i;
        if (!__any(here)) continue;
        float one[1][kS];
        floatx4 c[1][kE];
#pragma unroll
        for (int y = 0; y < kS; ++y) one[0][y] = p[r][y];
#pragma unroll
        for (int e = 0; e < kE; ++e) c[0][e] = floatx4{0.f, 0.f, 0.f, 0.f};
        values(mine, one, c);
#pragma unroll
        for (int e = 0; e < kE; ++e)
#pragma unroll
          for (int y = 0; y < 4; ++y) acc[r][e][y] += here ? c[0][e][y] : 0.f;
      }
    }
  }

  // Tiles from token `at` on, every WAVES-th: those that all rows see as far as they see them, then, without a second tile on its
  // way (its registers hold what each row's product takes there), those that only some of them see.
  __device__ __forceinline__ void run(int64_t at) {
    const int64_t shared = MODE == kSeveral && lim_lo < lim_hi ? min(end, (int64_t)(lim_lo & -kTokens)) : end;
    auto nothing = [] {};
    at = tile_at(at, shared);
    if constexpr (RT == 2 && D == 128) {
      // (no registers for a second tile: the next keys are asked for once the logits are there, the next values after the products)
      if (at < shared) {
        Tile t;
        load(t, at);
        while (at < shared) {
          Where next;
          at = tile_at(at + kStep, shared);
          const bool more = at < shared;
          step<false>(t, [&] {
            if (more) {
              next = find(at);
              load_keys(t, next);
            }
          });
          if (more) load_values(t, next);
        }
      }
    } else if (at < shared) {
      Tile t0, t1;
      load(t0, at);
      while (true) {
        at = tile_at(at + kStep, shared);
        if (at < shared) load(t1, at);
        step<false>(t0, nothing);
        if (at >= shared) break;
        at = tile_at(at + kStep, shared);
        if (at < shared) load(t0, at);
        step<false>(t1, nothing);
        if (at >= shared) break;
      }
    }
    if constexpr (MODE == kSeveral) {
      for (; at < end; at += kStep) {
        Tile t;
        load(t, at);
        step<true>(t, nothing);
      }
    }
  }

  int row0;                                              // first row of the workgroup
  __device__ __forceinline__ int row_of(int r) const { return row0 + 16 * r + col; }

  __device__ __forceinline__ void start(int context, int first_row, int64_t begin, int64_t end_) {
    x = context;
    b = MODE == kList ? x / a.n_q : x;
    end = end_;
    row0 = first_row;
    const int64_t most = (int64_t)a.c.max_pages << a.log2_page;
    int lo = 0x7fffffff, hi = 0;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int row = row_of(r);
      const bool there = row < a.rows;
      const int i = there ? row / a.G : 0;
      const int64_t out = MODE == kList ? x : (int64_t)x * a.n_q + i;
      lim[r] = there ? (int)min((int64_t)max(a.seen[out], 0), most) : 0;
      if (lim[r] > 0) { lo = min(lo, lim[r]); hi = max(hi, lim[r]); }
      const T* src = static_cast<const T*>(a.q) + (out * a.H + g * a.G + (there ? row - i * a.G : 0)) * D;
      const u32x4 zero = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int f = 0; f < kLoads; ++f)
        q[r][f] = there ? *reinterpret_cast<const u32x4*>(src + (4 * f + quad) * (16 / (int)sizeof(T))) : zero;
      m[r] = -INFINITY;
      l[r] = 0.f;
      any[r] = false;
#pragma unroll
      for (int e = 0; e < kE; ++e) acc[r][e] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    if constexpr (MODE == kSeveral) {
#pragma unroll
      for (int d = 8; d >= 1; d >>= 1) { lo = min(lo, __shfl_xor(lo, d, 64)); hi = max(hi, __shfl_xor(hi, d, 64)); }
      lim_lo = hi > 0 ? __builtin_amdgcn_readfirstlane(lo) : 0;
      lim_hi = __builtin_amdgcn_readfirstlane(hi);
    } else {
      lim_lo = lim_hi = __builtin_amdgcn_readfirstlane(lim[0]);       // (row 0 is always there)
    }
    count = (int)(((int64_t)lim_hi + a.c.page_size - 1) >> a.log2_page);
    open((int)(begin >> a.log2_page));
  }
};

// One row's result: four elements of its sums over the sum of its weights.
template <typename T, int D>
__device__ __forceinline__ void store_row(const PageAttnArgs& a, int x, int g, int row, int e, float top, float l, floatx4 o) {
  const int i = row / a.G;
  const int64_t out = (a.list ? x : (int64_t)x * a.n_q + i) * a.H + g * a.G + (row - i * a.G);
  const bool nothing = top == -INFINITY && l == 0.f;
  const float inv = 1.f / l;
#pragma unroll
  for (int y = 0; y < 4; ++y) o[y] = nothing ? 0.f : o[y] * inv;
  T* dst = static_cast<T*>(a.o) + out * D + e;
  if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2*>(dst) = u32x2{cvt_pk_bf16(o[0], o[1]), cvt_pk_bf16(o[2], o[3])};
  else *reinterpret_cast<floatx4*>(dst) = o;
  if (a.lse && e == 0) a.lse[out] = nothing ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * kLn2;
}

// Joins the waves of a workgroup: their sums go through LDS, scaled to the largest of their reference points, and leave as rows of
// the output, or as partial result `part`.
template <typename T, int D, int RT, int MODE, int WAVES>
__device__ __forceinline__ void finish(const PageAttnArgs& a, Walk<T, D, RT, MODE, WAVES>& w, float (&s_o)[WAVES][16 * RT][D + 4],
                                       float (&s_m)[WAVES][16 * RT], float (&s_l)[WAVES][16 * RT], int in, int row0, int64_t part) {
  typedef Walk<T, D, RT, MODE, WAVES> W;
  constexpr int kRows = 16 * RT, kThreads = 64 * WAVES;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    if (w.lim[r] == 0) { w.m[r] = -INFINITY; w.l[r] = 0.f; w.any[r] = false; }       // (beside rows that see whole tiles)
    float l = w.l[r];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    bool any = w.any[r];
    any = __shfl_xor((int)any, 16, 64) || any;
    any = __shfl_xor((int)any, 32, 64) || any;
    // without a reference point: only logits of -inf (l is 0), which make the row NaN where no other part has more, or some that are
    // NaN (l is NaN), which make it NaN whatever the others have: with a finite point the joins take that l with them
    if (l != l) w.m[r] = w.m[r] == -INFINITY ? 0.f : w.m[r];
    else if (any && w.m[r] == -INFINITY) l = NAN;
    if (lane < 16) { s_m[wave][16 * r + lane] = w.m[r]; s_l[wave][16 * r + lane] = l; }
    if (row0 + 16 * r + w.col >= a.rows) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < W::kE; e += 4) {
        const int dim = W::kHalf ? D / 16 * (4 * w.quad + i) + e : 16 * e + 4 * (4 * w.quad + i);
        *reinterpret_cast<floatx4*>(&s_o[wave][16 * r + w.col][dim]) =
            any ? floatx4{w.acc[r][e][i], w.acc[r][e + 1][i], w.acc[r][e + 2][i], w.acc[r][e + 3][i]} : floatx4{0.f, 0.f, 0.f, 0.f};
      }
  }
  __syncthreads();
  const int rows = min(kRows, a.rows - row0);
  for (int item = tid; item < rows * (D / 4); item += kThreads) {
    const int r = item / (D / 4), e = item % (D / 4) * 4;
    float top = s_m[0][r];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) top = fmaxf(top, s_m[i][r]);
    float l = 0.f;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      const float mi = s_m[i][r], li = s_l[i][r];
      const floatx4 oi = *reinterpret_cast<const floatx4*>(&s_o[i][r][e]);
      // (what saw nothing or only logits of -inf weighs nothing beside others; the latter make a row NaN that has nothing else.  Their
      // sums are 0, or NaN where a value is not finite)
      if (mi == -INFINITY) { l = top == -INFINITY ? l + li : l; o += oi; continue; }
      const float f = mi == top ? 1.f : __builtin_amdgcn_exp2f(mi - top);
      l += f * li;
      o += f * oi;
    }
    if (part >= 0) {
      const int64_t at = (part * a.inner + in) * a.part_rows + r;
      *reinterpret_cast<floatx4*>(a.part_o + at * D + e) = o;
      if (e == 0) a.part_ml[at] = make_float2(top, l);
      continue;
    }
    store_row<T, D>(a, w.x, w.g, row0 + r, e, top, l, o);
  }
}

// WHOLE: a workgroup has a context as a whole, and nothing is joined.
template <typename T, int D, int RT, int MODE, int WAVES, bool WHOLE>
__global__ __launch_bounds__(64 * WAVES, RT == 1 || D == 64 ? 2 : 1) void page_attn_kernel(PageAttnArgs a) {
  typedef Walk<T, D, RT, MODE, WAVES> W;
  constexpr int kRows = 16 * RT;
  __shared__ __align__(16) float s_o[WAVES][kRows][D + 4];         // (rows 4 banks apart)
  __shared__ float s_m[WAVES][kRows], s_l[WAVES][kRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t r = blockIdx.x / a.inner;
  const int in = (int)(blockIdx.x - r * a.inner), g = in % a.Hkv, row0 = in / a.Hkv * kRows;
  W w(a, lane, g);
  if constexpr (WHOLE) {
    w.start((int)r, row0, 0, list_end<MODE>(a, context_tokens(a, (int)r)));
    w.run(wave * W::kTokens);
    finish(a, w, s_o, s_m, s_l, in, row0, -1);
    return;
  }
  const Contexts all = contexts_of(a, lane);
  const int64_t from = r * all.range, to = from + all.range;
  Place here = place_of<false>(a, all, from, 0, lane);
  if (here.x < 0) return;
  while (true) {
    // its grains in the range, counted from its first
    const int64_t g0 = max(from - here.start, (int64_t)0), g1 = min(to - here.start, here.grains);
    if (g1 > g0) {
      const int64_t tokens = here.x < 64 ? from_lane(all.tokens, here.x) : context_tokens(a, here.x);
      w.start(here.x, row0, g0 * pages::kGrain, g1 == here.grains ? list_end<MODE>(a, tokens) : g1 * pages::kGrain);
      w.run(g0 * pages::kGrain + wave * W::kTokens);
      finish(a, w, s_o, s_m, s_l, in, row0, g1 - g0 == here.grains ? -1 : 2 * r + (g0 == 0));
    }
    here.start += here.grains + all.pad;
    if (here.start >= to || all.apart || ++here.x >= a.contexts) return;
    here.grains = here.x < 64 ? (int64_t)from_lane(all.grains, here.x) : pages::grains_of(context_tokens(a, here.x));
    __syncthreads();                                     // (before the sums in LDS are written again)
  }
}

// Joins the parts of a context: a workgroup per (context, KV head and row block, rows), or, where there are more contexts than
// ranges, per range for the context that starts in it and goes on behind it.  SHARED: the groups of threads share a row's parts, one
// row to a workgroup; otherwise each has a row.
template <typename T, int D, bool SHARED>
__global__ __launch_bounds__(256) void page_join_kernel(PageAttnArgs a, int row_steps) {
  constexpr int kVecs = D / 4, kGroups = 256 / kVecs, kStep = SHARED ? kGroups : 1, kAt = 4;
  __shared__ __align__(16) float s_o[kGroups][D];
  __shared__ float s_l[kGroups], s_m[kGroups];
  const int tid = threadIdx.x, lane = tid & 63, group = tid / kVecs, e = tid % kVecs * 4;
  const int64_t rest = blockIdx.x / row_steps, item = rest / a.inner;
  const int r = SHARED ? (int)(blockIdx.x - rest * row_steps) : (int)(blockIdx.x - rest * row_steps) * kGroups + group;
  const int in = (int)(rest - item * a.inner), row = in / a.Hkv * a.part_rows + r;
  const Contexts all = contexts_of(a, lane);
  const bool few = a.contexts <= a.slots;
  const Place p = few ? place_of<true>(a, all, 0, (int)item, lane) : place_of<false>(a, all, (item + 1) * all.range - 1, 0, lane);
  if (p.x < 0 || r >= a.part_rows || row >= a.rows) return;             // (SHARED: of the workgroup)
  auto range_at = [&](int64_t grain) {
    return (grain | all.range) >> 31 ? grain / all.range : (int64_t)((uint32_t)grain / (uint32_t)all.range);
  };
  const int64_t first = range_at(p.start), last = range_at(p.start + p.grains - 1);
  if (last == first || (!few && first != item)) return;
  const int count = (int)(last - first) + 1;
  auto part = [&](int j) { return ((2 * (first + j) + (j == 0)) * a.inner + in) * a.part_rows + r; };
  float top = -INFINITY, l = 0.f;
  floatx4 o = {0.f, 0.f, 0.f, 0.f};
  // part j: (ml, v) beside what there is; what has only logits of -inf weighs nothing beside others, and makes a row NaN alone
  auto add = [&](float2 ml, floatx4 v) {
    if (ml.x == -INFINITY) { l = top == -INFINITY ? l + ml.y : l; o += v; return; }
    if (top == -INFINITY) l = 0.f;
    const float next = fmaxf(top, ml.x);
    const float f = top == next ? 1.f : __builtin_amdgcn_exp2f(top - next), g = ml.x == next ? 1.f : __builtin_amdgcn_exp2f(ml.x - next);
    l = l * f + ml.y * g;
    o = o * f + v * g;
    top = next;
  };
  for (int j0 = SHARED ? group : 0; j0 < count; j0 += kAt * kStep) {
    float2 ml[kAt];
    floatx4 v[kAt];
#pragma unroll
    for (int i = 0; i < kAt; ++i) {
      const int64_t at = part(min(j0 + i * kStep, count - 1));
      ml[i] = a.part_ml[at];
      v[i] = *reinterpret_cast<const floatx4*>(a.part_o + at * D + e);
    }
#pragma unroll
    for (int i = 0; i < kAt; ++i)
      if (j0 + i * kStep < count) add(ml[i], v[i]);
  }
  if constexpr (SHARED) {
    *reinterpret_cast<floatx4*>(&s_o[group][e]) = o;
    if (e == 0) { s_l[group] = l; s_m[group] = top; }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int j = 1; j < kGroups; ++j) add(make_float2(s_m[j], s_l[j]), *reinterpret_cast<const floatx4*>(&s_o[j][e]));
  }
  store_row<T, D>(a, p.x, in % a.Hkv, row, e, top, l, o);
}

template <typename T, int D>
qcf_status launch(const PageAttnArgs& a, const pages::Division& d, hipStream_t st) {
  const int64_t blocks = (int64_t)(d.whole ? d.contexts : d.slots) * d.inner;
  // groups of a joining workgroup share a row where contexts have more than four parts on average
  const bool shared = (int64_t)d.contexts * 4 < d.slots;
  const int row_steps = shared ? a.part_rows : (a.part_rows + 1024 / D - 1) / (1024 / D);
  const int64_t joins = (int64_t)std::min(d.contexts, d.slots) * d.inner * row_steps;
  if (blocks > pages::kThreadsAtMost / (64 * (d.whole ? pages::kWholeWaves : pages::kWaves)) || joins > pages::kThreadsAtMost / 256)
    return fail(QCF_ERR_UNSUPPORTED, "page attention: too many rows");
  const dim3 grid((unsigned)blocks);
#define QCF_LAUNCH(RT, MODE, WAVES, WHOLE) page_attn_kernel<T, D, RT, MODE, WAVES, WHOLE><<<grid, dim3(64 * WAVES), 0, st>>>(a)
#define QCF_ROWS(MODE)                                                                          \
  do {                                                                                          \
    if (d.row_tiles == 1) {                                                                     \
      if (d.whole) QCF_LAUNCH(1, MODE, pages::kWholeWaves, true);                               \
      else QCF_LAUNCH(1, MODE, pages::kWaves, false);                                           \
    } else {                                                                                    \
      QCF_LAUNCH(2, MODE, pages::kWaves, false);                                                \
    }                                                                                           \
  } while (0)
  if (a.list) QCF_ROWS(kList);
  else if (a.n_q == 1) QCF_ROWS(kOne);
  else QCF_ROWS(kSeveral);
#undef QCF_ROWS
#undef QCF_LAUNCH
  QCF_TRY_LAUNCH("page attention");
  if (!pages::divides(d)) return QCF_OK;
  if (shared) page_join_kernel<T, D, true><<<dim3((unsigned)joins), dim3(256), 0, st>>>(a, row_steps);
  else page_join_kernel<T, D, false><<<dim3((unsigned)joins), dim3(256), 0, st>>>(a, row_steps);
  return check_launch("page attention join");
}

}  // namespace

size_t page_attn_workspace(const qcf_layer_desc& L, const qcf_page_cache& c, int32_t B, int32_t n_q, int32_t n_keep) {
  return pages::workspace(L, pages::divide(L, c, B, n_q, n_keep));
}

qcf_status launch_page_attn(const qcf_layer_desc& L, const qcf_page_cache& c, int32_t B, int32_t n_q, const void* q,
                            const int32_t* seen, const int32_t* list, int32_t n_keep, void* o, float* lse, void* ws,
                            hipStream_t st) {
  const pages::Division d = pages::divide(L, c, B, n_q, n_keep);
  PageAttnArgs a;
  a.c = c; a.q = q; a.seen = seen; a.list = list; a.n_keep = n_keep;
  a.n_q = n_q; a.H = L.n_q_heads; a.Hkv = L.n_kv_heads; a.G = a.H / a.Hkv;
  a.log2_page = __builtin_ctz((unsigned)c.page_size);
  a.contexts = d.contexts; a.rows = d.rows; a.inner = d.inner; a.slots = d.slots; a.least = d.least; a.pad = d.pad;
  a.part_rows = pages::part_rows(d);
  const double scale = 1.4426950408889634 / std::sqrt((double)L.head_dim);
  a.scale = (float)scale;
  if (a.scale > scale) a.scale = std::nextafterf(a.scale, 0.f);
  a.scale_low = (float)(scale - a.scale);
  a.o = o; a.lse = lse;
  a.part_o = static_cast<float*>(ws);
  a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + (pages::divides(d) ? pages::sums_bytes(L, d) : 0));
  if (L.dtype == QCF_DTYPE_BF16) return L.head_dim == 128 ? launch<bf16_t, 128>(a, d, st) : launch<bf16_t, 64>(a, d, st);
  return L.head_dim == 128 ? launch<float, 128>(a, d, st) : launch<float, 64>(a, d, st);
}

}  // namespace qcf

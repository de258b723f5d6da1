// What the tokens of a cache in pages get of their requests' attention, added up step by step.
//
// w_t = alpha w_t + beta sum_rows exp(z_t - lse): the softmax's sums are known, so a token's weights need its logits and nothing of other tokens,
// and one pass over the keys is all.  A wave takes 32 tokens (16 in float32) at a time as in the attention, whose division of the contexts
// this has too, with the product's operands the other way round: a lane owns a token and four rows of each 16, so that the sum over the
// rows is three additions and two exchanges between lanes (136 us with a row to a lane, four exchanges to each token; 129).  Bound by memory: the
// keys, and 8 bytes of weights to a token and KV head: 16 requests of 1K to 16K tokens in bf16 72 us, 4.7 TB/s; 64 of 4K to 12K in 8 bits 130, 4.5.
#include "page_walk.h"

namespace qcf {
namespace {

struct WeighArgs {
  PageAttnArgs a;
  const float* lse;
  const int32_t* old;
  float alpha, beta;
  float* weights;
  int64_t stride;                                        // tokens of a head's weights
  int row_blocks;
};

// Workgroups on a compute unit, of four waves each: as many as the registers allow.  (us, 8 bits, 64 requests of 4K to 12K tokens: heads of 128
// 132 with two, 129 with three, 139 with four, whose registers spill, 133 with two and tiles of 64 tokens; heads of 64 92 with two, 79.9 with
// three, 76.0 with four.  16 of 1K to 16K in bf16: 73.0, 72.5 and 95.)
constexpr int at_once(bool eight, int row_tiles, int head_dim) { return !eight || row_tiles > 1 ? 2 : head_dim == 64 ? 4 : 3; }

template <typename T, int D, int RT, bool EIGHT, int HEADS>
struct Weigher : Walk<T, D, RT, kSeveral, pages::kWaves / HEADS, EIGHT> {
  typedef Walk<T, D, RT, kSeveral, pages::kWaves / HEADS, EIGHT> W;
  typedef typename W::Tile Tile;
  static constexpr float kLog2e = 1.4426950408889634f, kLog2eLow = 1.925963033500e-8f;
  const WeighArgs& w_;
  float ref[RT][4], ref_low[RT][4];                      // lse in powers of two of rows 4 quad to 4 quad + 3 (float32: as two floats)
  int sees[RT][4];                                       // tokens that they see
  float* out;                                            // this lane's place among the weights: token col of part `quad` of a tile
  int known;                                             // tokens weighed before
  int tokens;                                            // that any row of the context sees

  __device__ __forceinline__ Weigher(const WeighArgs& args, int lane, int g) : W(args.a, lane, g), w_(args) {}

  __device__ __forceinline__ void prepare(int context, int row0, int64_t begin, int64_t end, int tokens_) {
    this->start(context, row0, begin, end);
    tokens = tokens_;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = row0 + 16 * r + 4 * this->quad + i;
        sees[r][i] = __shfl(this->lim[r], 4 * this->quad + i, 64);
        const int at = row / this->a.G, head = this->g * this->a.G + (row - at * this->a.G);
        const float l = sees[r][i] > 0 ? w_.lse[((int64_t)context * this->a.n_q + at) * this->a.H + head] : INFINITY;
        ref[r][i] = l * kLog2e;                          // (a row that sees nothing: infinite, its weights are 0)
        ref_low[r][i] = __builtin_isfinite(ref[r][i]) ? __builtin_fmaf(l, kLog2e, -ref[r][i]) + l * kLog2eLow : 0.f;
      }
    known = w_.old ? w_.old[context] : 0x7fffffff;
    out = w_.weights + ((int64_t)context * this->a.Hkv + this->g) * w_.stride + this->lane;
  }

  __device__ __forceinline__ bool mine(int64_t at) const { return this->quad < W::kSub && at + this->lane < tokens; }
  __device__ __forceinline__ void load(Tile& t, float& was, int64_t at, bool first) {
    const typename W::Where r = this->find(at);
    this->load_keys(t, r);
#pragma unroll
    for (int h = 0; h < W::kSub; ++h) t.base[h] = r.base[h];
    was = 0.f;
    if ((!first || w_.alpha != 0.f) && mine(at)) was = out[at];
  }
  __device__ __forceinline__ void weigh(const Tile& t, float was, int64_t at, bool first) {
    float s[RT][W::kS], sum = 0.f;
    this->template logits<true>(t, s);
    bool whole = true;
#pragma unroll
    for (int h = 0; h < W::kSub; ++h) whole = whole && t.base[h] >= 0 && t.base[h] + 16 <= this->lim_lo;
#pragma unroll
    for (int h = 0; h < W::kSub; ++h) {
      float part = 0.f;
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float z = s[r][4 * h + i];
          float x = __builtin_fmaf(z, this->a.scale, -ref[r][i]);
          // (bf16: 2^-24 of the logit and of lse less, beside what the products of rounded queries and keys have lost)
          if constexpr (!W::kHalf) x += __builtin_fmaf(z, this->a.scale_low, -ref_low[r][i]);
          float e = __builtin_amdgcn_exp2f(x);
          // (a row that sees nothing may hold anything)
          e = whole ? (sees[r][i] > 0 ? e : 0.f) : t.base[h] >= 0 && t.base[h] + this->col < sees[r][i] ? e : 0.f;
          part += e;
        }
      typedef unsigned u2v __attribute__((ext_vector_type(2)));
      u2v y = __builtin_amdgcn_permlane16_swap(__float_as_uint(part), __float_as_uint(part), false, false);
      part = __uint_as_float(y.x) + __uint_as_float(y.y);
      y = __builtin_amdgcn_permlane32_swap(__float_as_uint(part), __float_as_uint(part), false, false);
      part = __uint_as_float(y.x) + __uint_as_float(y.y);
      sum = h == this->quad ? part : sum;
    }
    if (!mine(at)) return;
    const float before = !first ? was : at + this->lane < known && w_.alpha != 0.f ? w_.alpha * was : 0.f;
    const float now = before + w_.beta * sum;
    out[at] = now != now ? NAN : now;
  }
  __device__ __forceinline__ void run(int64_t at, bool first) {
    if (at >= this->end) return;
    Tile t0, t1;
    float w0, w1;
    load(t0, w0, at, first);
    while (true) {
      int64_t next = at + W::kStep;
      if (next < this->end) load(t1, w1, next, first);
      weigh(t0, w0, at, first);
      if (next >= this->end) return;
      at = next + W::kStep;
      if (at < this->end) load(t0, w0, at, first);
      weigh(t1, w1, next, first);
      if (at >= this->end) return;
    }
  }
};

// (HEADS: KV heads that the waves take side by side)
template <typename T, int D, int RT, bool EIGHT, int HEADS>
__global__ __launch_bounds__(64 * pages::kWaves, at_once(EIGHT, RT, D)) void page_weigh_kernel(WeighArgs args) {
  typedef Weigher<T, D, RT, EIGHT, HEADS> W;
  const PageAttnArgs& a = args.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t r = blockIdx.x / a.inner;
  const int g = (int)(blockIdx.x - r * a.inner) * HEADS + wave % HEADS;
  W w(args, lane, g);
  const Contexts all = contexts_of(a, lane);
  const int64_t from = r * all.range, to = from + all.range;
  Place here = place_of<false>(a, all, from, 0, lane);
  if (here.x < 0) return;
  while (true) {
    const int64_t g0 = max(from - here.start, (int64_t)0), g1 = min(to - here.start, here.grains);
    if (g1 > g0) {
      const int64_t tokens = here.x < 64 ? from_lane(all.tokens, here.x) : context_tokens(a, here.x);
      const int64_t begin = g0 * pages::kGrain, end = g1 == here.grains ? tokens : g1 * pages::kGrain;
      // (each wave's tokens are its own, and so are their weights: the second block of rows finds what the first one stored)
      for (int block = 0; block < args.row_blocks; ++block) {
        w.prepare(here.x, block * 16 * RT, begin, end, (int)tokens);
        w.run(begin + wave / HEADS * W::W::kTokens, block == 0);
      }
    }
    here.start += here.grains + all.pad;
    if (here.start >= to || all.apart || ++here.x >= a.contexts) return;
    here.grains = here.x < 64 ? (int64_t)from_lane(all.grains, here.x) : pages::grains_of(context_tokens(a, here.x));
  }
}

}  // namespace

qcf_status launch_page_weigh(const qcf_layer_desc& L, const qcf_page_cache& c, const float* scales, int32_t B, int32_t n_q, const void* q,
                             const int32_t* seen, const float* lse, const int32_t* old, float alpha, float beta, float* weights,
                             hipStream_t st) {
  WeighArgs w;
  const int rows = n_q * (L.n_q_heads / L.n_kv_heads), row_tiles = rows > 16 ? 2 : 1;
  fill_args(w.a, L, c, scales, n_q, q, seen);
  w.a.contexts = B;
  w.a.rows = rows;
  w.stride = (int64_t)c.max_pages * c.page_size;
  const int heads = pages::side_by_side(L, c, scales ? 1 : 2, (double)B * (double)w.stride * L.n_kv_heads * 2 * L.head_dim);
  w.a.inner = L.n_kv_heads / heads;
  w.a.least = pages::least_range(L);
  w.a.pad = 0;
  w.lse = lse; w.old = old; w.alpha = alpha; w.beta = beta;
  w.weights = weights;
  w.row_blocks = (rows + 16 * row_tiles - 1) / (16 * row_tiles);
  const int64_t ranges = ((int64_t)B * ((w.stride + pages::kGrain - 1) / pages::kGrain) + w.a.least - 1) / w.a.least;
  w.a.slots = (int)std::min<int64_t>(ranges, std::max(1, at_once(scales != nullptr, row_tiles, L.head_dim) * compute_unit_count() / w.a.inner));
  const dim3 grid((unsigned)((int64_t)w.a.slots * w.a.inner)), block(64 * pages::kWaves);
#define QCF_LAUNCH(T, D, RT, EIGHT)                                                          \
  do {                                                                                       \
    if (heads > 1) page_weigh_kernel<T, D, RT, EIGHT, EIGHT ? 256 / D : 1><<<grid, block, 0, st>>>(w); \
    else page_weigh_kernel<T, D, RT, EIGHT, 1><<<grid, block, 0, st>>>(w);                   \
  } while (0)
#define QCF_ROWS(T, D, EIGHT) do { if (row_tiles == 1) QCF_LAUNCH(T, D, 1, EIGHT); else QCF_LAUNCH(T, D, 2, EIGHT); } while (0)
#define QCF_PAGES(T, D) do { if (scales) QCF_ROWS(T, D, true); else QCF_ROWS(T, D, false); } while (0)
  if (L.dtype == QCF_DTYPE_BF16) {
    if (L.head_dim == 128) QCF_PAGES(bf16_t, 128); else QCF_PAGES(bf16_t, 64);
  } else {
    if (L.head_dim == 128) QCF_PAGES(float, 128); else QCF_PAGES(float, 64);
  }
#undef QCF_PAGES
#undef QCF_ROWS
#undef QCF_LAUNCH
  return check_launch("page weights");
}

}  // namespace qcf

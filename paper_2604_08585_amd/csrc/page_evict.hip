// A cache in pages cut down to the tokens that attention uses: the choice is qcf_page_select's, over tokens; here the rows move.
#include "qcf_internal.h"
#include "page_layout.h"
#include "append_common.h"
#include "eight.h"

namespace qcf {
namespace {

struct EvictArgs {
  qcf_page_cache from, to;
  const float* scales;
  float* to_scales;
  const float* weights;
  float* to_weights;
  const int32_t* kept;
  int32_t* to_len;
  int Hkv, n_keep, log2_from, log2_to;
  int units, tokens;                                     // workgroups of a head, and tokens of each
};

// ---- the choice among many tokens: all of the GPU on each row ------------------------------------------------------------------------
// launch_page_top has one workgroup to a row, which reads it again and again (131072 tokens 104 us).  Here a row is cut into segments of
// kSegment tokens, one workgroup each, and its threshold is found digit by digit: histograms of 11, 11 and 10 bits of the weights' order
// keys, added up over the segments by integer atomics (sums do not depend on their order), each launch finding the digit of the one
// before it.  Then the segments' counts, and the tokens in order.  The same tokens as launch_page_top's, bit for bit.
// (8 rows of 131072 tokens, the whole eviction, us: segments of 4096 with 512 threads 63.6, 256 67.7, 1024 62.9 but 64 rows of 65536 101
// and not 86; of 2048 with 256 64.6, of 8192 with 512 69.8)
constexpr int kSegment = 4096, kThreadsOf = 512, kEach = kSegment / kThreadsOf;
constexpr int kBits[3] = {11, 11, 10}, kShift[3] = {21, 10, 0};
constexpr int kHist = 2048 + 2048 + 1024, kHistAt[3] = {0, 2048, 4096};

// Per row: the histograms, the digits found so far (prefix, how many of its keys are still wanted), and per segment how many keys are
// beyond the threshold and how many equal it.
struct TopArgs {
  const float* weights;
  const int32_t* len;
  int64_t stride;                        // tokens of a row
  int Hkv, n_keep, n_first, n_last, segments;
  uint32_t* hist;                        // [rows][kHist]
  uint2* state;                          // [rows][2]
  uint2* counts;                         // [rows][segments]
  int32_t* kept;
};
struct TopRow {
  int count, n;                          // tokens, and how many stay
  int lo, hi;                            // tokens that are chosen from
  int wanted;                            // of them
};
__device__ __forceinline__ TopRow top_row(const TopArgs& a, int64_t row) {
  TopRow r;
  r.count = (int)min((int64_t)max(a.len[row / a.Hkv], 0), a.stride);
  r.n = min(r.count, a.n_keep);
  r.lo = a.n_first;
  r.hi = r.count - a.n_last;
  r.wanted = r.count > a.n_keep ? r.n - a.n_first - a.n_last : 0;          // (0: nothing is to be found)
  return r;
}
__device__ __forceinline__ uint32_t order_key(float s) {
  uint32_t u = __float_as_uint(s);
  if (u == 0x80000000u) u = 0u;          // -0 and +0 are the same weight
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
// This thread's keys, in order; what is not chosen from has none.
__device__ __forceinline__ uint32_t read_keys(const TopArgs& a, const TopRow& r, int64_t row, int t0, uint32_t (&key)[kEach]) {
  const float* w = a.weights + row * a.stride;
  uint32_t there = 0;
#pragma unroll
  for (int q = 0; q < kEach; q += 4) {
    const int t = t0 + q;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (t < r.hi) v = *reinterpret_cast<const float4*>(w + t);             // (rows are multiples of 16 long)
    const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      key[q + i] = order_key(f[i]);
      there |= (uint32_t)(t + i >= r.lo && t + i < r.hi) << (q + i);
    }
  }
  return there;
}
// Inclusive sum over the threads of a workgroup.
__device__ __forceinline__ uint32_t block_incl(uint32_t x, uint32_t (&s_wave)[kThreadsOf / 64]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t y = __shfl_up(x, d, 64);
    if (lane >= d) x += y;
  }
  __syncthreads();
  if (lane == 63) s_wave[wave] = x;
  __syncthreads();
  for (int i = 0; i < wave; ++i) x += s_wave[i];
  return x;
}
// The digit, counted from the largest, in which the `wanted`-th largest key lies, and how many keys are wanted of it.
template <int LEVEL>
__device__ __forceinline__ uint2 find_digit(const uint32_t* hist, uint32_t wanted, uint32_t (&s_wave)[kThreadsOf / 64], uint2& s_found) {
  constexpr int kBins = 1 << kBits[LEVEL], kPer = kBins / kThreadsOf;
  uint32_t n[kPer], sum = 0;
  const int top = kBins - 1 - (int)threadIdx.x * kPer;                     // this thread's largest digit
#pragma unroll
  for (int i = 0; i < kPer; ++i) sum += n[i] = hist[kHistAt[LEVEL] + top - i];
  uint32_t before = block_incl(sum, s_wave) - sum;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (before < wanted && before + n[i] >= wanted) s_found = make_uint2((uint32_t)(top - i), wanted - before);
    before += n[i];
  }
  __syncthreads();
  return s_found;
}

__global__ __launch_bounds__(256) void top_clear_kernel(uint32_t* hist, int64_t n) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i < n) *reinterpret_cast<uint4*>(hist + i) = make_uint4(0u, 0u, 0u, 0u);
}

template <int LEVEL>
__global__ __launch_bounds__(kThreadsOf) void top_count_kernel(TopArgs a) {
  constexpr int kBins = 1 << kBits[LEVEL];
  __shared__ uint32_t s_hist[kBins], s_wave[kThreadsOf / 64];
  __shared__ uint2 s_found;
  const int64_t row = blockIdx.x / a.segments;
  const int seg = (int)(blockIdx.x - row * a.segments), tid = threadIdx.x;
  const TopRow r = top_row(a, row);
  if (r.wanted <= 0 || seg * kSegment >= r.hi) return;
  uint32_t* hist = a.hist + row * kHist;
  uint32_t prefix = 0, wanted = (uint32_t)r.wanted;
  for (int i = tid; i < kBins; i += kThreadsOf) s_hist[i] = 0u;
  uint32_t key[kEach];
  const uint32_t there = read_keys(a, r, row, seg * kSegment + tid * kEach, key);
  if constexpr (LEVEL > 0) {
    if constexpr (LEVEL > 1) {
      const uint2 s = a.state[row * 2];
      prefix = s.x;
      wanted = s.y;
    }
    const uint2 found = find_digit<LEVEL - 1>(hist, wanted, s_wave, s_found);
    prefix |= found.x << kShift[LEVEL - 1];
    if (seg == 0 && tid == 0) a.state[row * 2 + LEVEL - 1] = make_uint2(prefix, found.y);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    constexpr int kFound = kShift[LEVEL == 0 ? 0 : LEVEL - 1];
    const bool mine = (there >> i & 1) && (LEVEL == 0 || key[i] >> kFound == prefix >> kFound);
    const uint32_t digit = key[i] >> kShift[LEVEL] & (kBins - 1);
    // (keys that are all alike, weights of 0 above all, are counted at once)
    const uint64_t all = __ballot(mine);
    const uint32_t first = (uint32_t)__builtin_amdgcn_readlane((int)digit, all ? __builtin_ctzll(all) : 0);
    if (__ballot(mine && digit == first) == all) {
      if (all && (threadIdx.x & 63) == 0) atomicAdd(&s_hist[first], (uint32_t)__popcll(all));
    } else if (mine) {
      atomicAdd(&s_hist[digit], 1u);
    }
  }
  __syncthreads();
  for (int i = tid; i < kBins; i += kThreadsOf)
    if (s_hist[i]) atomicAdd(hist + kHistAt[LEVEL] + i, s_hist[i]);
}

// (WRITE: the tokens, after a launch without it has counted each segment's)
template <bool WRITE>
__global__ __launch_bounds__(kThreadsOf) void top_keep_kernel(TopArgs a) {
  __shared__ uint32_t s_wave[kThreadsOf / 64], s_wave2[kThreadsOf / 64];
  __shared__ uint2 s_found;
  const int64_t row = blockIdx.x / a.segments;
  const int seg = (int)(blockIdx.x - row * a.segments), tid = threadIdx.x;
  const TopRow r = top_row(a, row);
  int32_t* kept = a.kept + row * a.n_keep;
  if constexpr (WRITE) {
    // what needs no choice: all tokens, or the first and the last ones, and nothing behind them
    const int t0 = seg * kSegment, t1 = seg + 1 == a.segments ? 0x7fffffff : t0 + kSegment;
    if (r.count <= a.n_keep) {
      for (int j = t0 + tid; j < min(t1, a.n_keep); j += kThreadsOf) kept[j] = j < r.count ? j : -1;
      return;
    }
    if (seg == 0) {
      for (int j = tid; j < a.n_first; j += kThreadsOf) kept[j] = j;
      for (int j = tid; j < a.n_last; j += kThreadsOf) kept[r.n - a.n_last + j] = r.count - a.n_last + j;
    }
  }
  if (r.wanted <= 0 || seg * kSegment >= r.hi) return;
  uint32_t key[kEach];
  const int t0 = seg * kSegment + tid * kEach;
  const uint32_t there = read_keys(a, r, row, t0, key);
  const uint2 s = a.state[row * 2 + 1];
  const uint2 found = find_digit<2>(a.hist + row * kHist, s.y, s_wave, s_found);
  const uint32_t least = s.x | found.x;                                    // the least key that stays, and how many of its kind
  uint32_t more = 0, same = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    more |= (uint32_t)((there >> i & 1) && key[i] > least) << i;
    same |= (uint32_t)((there >> i & 1) && key[i] == least) << i;
  }
  const uint32_t n_more = block_incl((uint32_t)__popc(more), s_wave), n_same = block_incl((uint32_t)__popc(same), s_wave2);
  uint2* counts = a.counts + row * a.segments;
  if constexpr (!WRITE) {
    if (tid == kThreadsOf - 1) counts[seg] = make_uint2(n_more, n_same);
    return;
  }
  uint32_t before_more = 0, before_same = 0;                               // in the segments in front of this one
  for (int i = tid; i < seg; i += kThreadsOf) {
    before_more += counts[i].x;
    before_same += counts[i].y;
  }
  __shared__ uint32_t s_sum[2];
  if (tid < 2) s_sum[tid] = 0u;
  __syncthreads();
  if (before_more) atomicAdd(&s_sum[0], before_more);
  if (before_same) atomicAdd(&s_sum[1], before_same);
  __syncthreads();
  uint32_t at_same = s_sum[1] + n_same - (uint32_t)__popc(same);
  uint32_t at = (uint32_t)a.n_first + s_sum[0] + n_more - (uint32_t)__popc(more) + min(at_same, found.y);
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const bool tie = same >> i & 1;
    if ((more >> i & 1) || (tie && at_same < found.y)) kept[at++] = t0 + i;
    at_same += tie;
  }
}

// ---- the rows ------------------------------------------------------------------------------------------------------------------------------
// A wave takes a block of 16 tokens of the new cache: their numbers, their pages and then the rows, all of a block on their way together.  A
// workgroup has four blocks; with bounds a page of the new cache, which its waves join.  Bound by memory, every kept row is read and written
// once: 16 requests to 2048 tokens of 32 / 8 heads of 128 in bf16 60 us, 4.5 TB/s (a copy of 1 GiB 5.1); one to 32768 in 8 bits, rows of 128
// bytes from anywhere, 32 us, 4.2 (without a kernel of their own for pages without bounds, 35 registers more, 34).  Two or four blocks to a wave,
// with the next one's numbers and pages on their way, take 1 to 8 % longer.
template <typename T, int D, bool EIGHT, bool BOUNDS>
__global__ __launch_bounds__(256) void evict_kernel(EvictArgs a) {
  constexpr int kSize = EIGHT ? 1 : (int)sizeof(T), kIn = 16 / kSize;                // elements of a 16-byte vector
  constexpr int VPR = D * kSize / 16, RPI = 64 / VPR, ITS = kBlock / RPI;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int64_t head = blockIdx.x / a.units;             // (request, KV head)
  const int64_t b = head / a.Hkv;
  const int g = (int)(head - b * a.Hkv), first = (int)(blockIdx.x - head * a.units) * a.tokens;
  const int32_t* kept = a.kept + head * a.n_keep;
  auto entry = [&](int j) { return j < a.n_keep ? kept[j] : -1; };
  float lo[BOUNDS ? kIn : 1], hi[BOUNDS ? kIn : 1];
  if constexpr (BOUNDS) {
#pragma unroll
    for (int e = 0; e < kIn; ++e) { lo[e] = INFINITY; hi[e] = -INFINITY; }
  }
  const int row = lane / VPR, part = lane % VPR;         // of this lane in each step of RPI rows
  // lane l % 16 has token l % 16 of a block: its number, and the page that it is in (-1: not there)
  auto number = [&](int j0) { return entry(j0 + (lane & 15)); };
  auto page_of = [&](int t) {
    const int p = t >> a.log2_from;
    return t >= 0 && p < a.from.max_pages ? a.from.table[b * a.from.max_pages + p] : -1;
  };
  auto new_page = [&](int j0) {
    const int p = j0 >> a.log2_to;
    return j0 < a.n_keep && p < a.to.max_pages ? a.to.table[b * a.to.max_pages + p] : -1;
  };
  const int end = min(first + a.tokens, a.n_keep);
  for (int j0 = first + wave * kBlock; j0 < end; j0 += waves * kBlock) {
    const int t = number(j0), from = page_of(t), to = new_page(j0);
    const int count = (int)__popcll(__ballot(t >= 0) & 0xffffu);
    // (the entry behind a full block: the next block's first)
    if (g == 0 && lane == 0 && (count > 0 || j0 == 0) && (count < kBlock || entry(j0 + kBlock) < 0)) a.to_len[b] = j0 + count;
    if (count == 0) break;                               // (of the wave: a block without tokens has no scale either)
    const int s = t & (a.from.page_size - 1), slot = j0 & (a.to.page_size - 1);
    const bool found = from >= 0 && from < a.from.n_pages, there = to >= 0 && to < a.to.n_pages;
    const int64_t src = found ? (from * a.from.page_stride + s * a.from.slot_stride + g * a.from.head_stride) * kSize : -1;
    if (a.to_weights && lane < count && j0 >> a.log2_to < a.to.max_pages)
      a.to_weights[(head * a.to.max_pages << a.log2_to) + j0 + lane] = found ? a.weights[(head * a.from.max_pages << a.log2_from) + t] : 0.f;
    if (there) {
      float scale[2] = {0.f, 0.f};
      if constexpr (EIGHT) {
#pragma unroll
        for (int which = 0; which < 2; ++which)
          if (found) scale[which] = a.scales[scale_at(from, a.Hkv, g, which, s, a.log2_from)];
      }
      u32x4 x[2][ITS];
#pragma unroll
      for (int it = 0; it < ITS; ++it) {
        const int64_t at = __shfl(src, it * RPI + row, 64);
#pragma unroll
        for (int which = 0; which < 2; ++which)
          x[which][it] = at >= 0 ? *reinterpret_cast<const u32x4*>(static_cast<const char*>(which ? a.from.v : a.from.k) + at + part * 16)
                                 : mk4(0u, 0u, 0u, 0u);
      }
      const int64_t dst = (to * a.to.page_stride + slot * a.to.slot_stride + g * a.to.head_stride) * kSize + part * 16;
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        char* out = static_cast<char*>(which ? a.to.v : a.to.k) + dst;
        float now = 0.f;
        if constexpr (EIGHT) {
          float amax = 0.f, f[kIn];
#pragma unroll
          for (int it = 0; it < ITS; ++it) {
            const float was = __shfl(scale[which], it * RPI + row, 64);
#pragma unroll
            for (int w = 0; w < 4; ++w) values_of(x[which][it][w], f + 4 * w);
            if (it * RPI + row < count) {
#pragma unroll
              for (int e = 0; e < kIn; ++e) amax = fmaxf(amax, __builtin_fabsf(f[e] * was));
            }
          }
          amax = wave_max(amax);
          now = scale_for(amax);
          const float inv = 1.f / now;
          if (lane == 0) a.to_scales[scale_at(to, a.Hkv, g, which, slot, a.log2_to)] = now;
#pragma unroll
          for (int it = 0; it < ITS; ++it) {
            const float was = __shfl(scale[which], it * RPI + row, 64);
            if (was == now) continue;                    // (the codes stay)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              values_of(x[which][it][w], f);
              x[which][it][w] = codes_of(f[0] * was * inv, f[1] * was * inv, f[2] * was * inv, f[3] * was * inv);
            }
          }
        }
#pragma unroll
        for (int it = 0; it < ITS; ++it) {
          const int r = it * RPI + row;
          if (r >= count) continue;
          *reinterpret_cast<u32x4*>(out + r * a.to.slot_stride * kSize) = x[which][it];
          if (BOUNDS && which == 0) {
            float f[kIn];
            if constexpr (EIGHT) {
#pragma unroll
              for (int w = 0; w < 4; ++w) values_of(x[0][it][w], f + 4 * w);
#pragma unroll
              for (int e = 0; e < kIn; ++e) f[e] *= now;
            } else {
              Vec16<T>::unpack(x[0][it], f);
            }
#pragma unroll
            for (int e = 0; e < kIn; ++e) {
              const int i = BOUNDS ? e : 0;
              lo[i] = least(lo[i], f[e]);
              hi[i] = largest(hi[i], f[e]);
            }
          }
        }
      }
    }
  }
  if constexpr (BOUNDS) {
    __shared__ float s_bound[2][4][D];
    const int page = first < a.n_keep && entry(first) >= 0 ? new_page(first) : -1;
    if (page < 0 || page >= a.to.n_pages) return;        // (of the workgroup)
#pragma unroll
    for (int d = VPR; d < 64; d *= 2)
#pragma unroll
      for (int e = 0; e < kIn; ++e) {
        lo[e] = least(lo[e], __shfl_xor(lo[e], d, 64));
        hi[e] = largest(hi[e], __shfl_xor(hi[e], d, 64));
      }
    if (lane < VPR) {
#pragma unroll
      for (int e = 0; e < kIn; ++e) {
        s_bound[0][wave][part * kIn + e] = lo[e];
        s_bound[1][wave][part * kIn + e] = hi[e];
      }
    }
    __syncthreads();
    T* bounds = static_cast<T*>(a.to.bounds) + ((int64_t)page * a.Hkv + g) * 2 * D;
    for (int item = threadIdx.x; item < 2 * D; item += blockDim.x) {
      const bool low = item < D;
      float v = s_bound[low ? 0 : 1][0][item % D];
      for (int w = 1; w < waves; ++w) v = low ? least(v, s_bound[0][w][item % D]) : largest(v, s_bound[1][w][item % D]);
      Elem<T>::store(bounds + item, v);
    }
  }
}

// Whether the choice is divided over the GPU: six launches and five passes over the weights, so long rows and not too many of them.  Eviction
// of 8-bit heads of 64 to an eighth, us, divided and not: 8 rows of 32768 tokens 36 and 25, 49152 38 and 43, 131072 44 and 108; 64 rows of
// 32768 58 and 45, 49152 75 and 76, 131072 150 and 203; 256 rows of 65536 270 and 237.  (By the room of the table: the host does not know the
// lengths.  Short requests in wide tables pay for it, 16 of 2000 tokens 47 us with room for 33024 and 117 with room for 131072, 22 undivided.)
bool splits_choice(const qcf_page_cache& c, int64_t rows) { return (int64_t)c.max_pages * c.page_size > 32768 && rows <= 128; }

}  // namespace

size_t page_evict_workspace(const qcf_layer_desc& L, const qcf_page_cache& c, int32_t B) {
  const int64_t heads = (int64_t)B * L.n_kv_heads;
  if (!splits_choice(c, heads)) return 0;
  const int64_t segments = ((int64_t)c.max_pages * c.page_size + kSegment - 1) / kSegment;
  return (size_t)(heads * (kHist * (int64_t)sizeof(uint32_t) + (2 + segments) * (int64_t)sizeof(uint2)));
}

qcf_status launch_page_evict(const qcf_layer_desc& L, const qcf_page_cache& c, const float* scales, int32_t B, const int32_t* len,
                             const float* weights, int32_t n_keep, int32_t n_first, int32_t n_last, const qcf_page_cache& to,
                             float* to_scales, int32_t* kept, float* to_weights, int32_t* to_len, void* ws, hipStream_t st) {
  EvictArgs a;
  a.from = c; a.to = to; a.scales = scales; a.to_scales = to_scales;
  a.weights = weights; a.to_weights = to_weights; a.kept = kept; a.to_len = to_len;
  a.Hkv = L.n_kv_heads; a.n_keep = n_keep;
  a.log2_from = __builtin_ctz((unsigned)c.page_size);
  a.log2_to = __builtin_ctz((unsigned)to.page_size);
  const int64_t heads = (int64_t)B * L.n_kv_heads;
  const int threads = to.bounds ? 64 * std::min(4, to.page_size / kBlock) : 256;
  a.tokens = to.bounds ? to.page_size : 4 * kBlock;
  a.units = (n_keep + a.tokens - 1) / a.tokens;
  const int64_t blocks = heads * a.units;
  if (blocks > pages::kThreadsAtMost / threads || heads > pages::kThreadsAtMost / pages::kTopThreads)
    return fail(QCF_ERR_UNSUPPORTED, "page evict: too many rows");
  if (splits_choice(c, heads)) {
    TopArgs t;
    t.weights = weights; t.len = len;
    t.stride = (int64_t)c.max_pages * c.page_size;
    t.Hkv = L.n_kv_heads; t.n_keep = n_keep; t.n_first = n_first; t.n_last = n_last;
    t.segments = (int)((t.stride + kSegment - 1) / kSegment);
    t.hist = static_cast<uint32_t*>(ws);
    t.state = reinterpret_cast<uint2*>(t.hist + heads * kHist);
    t.counts = t.state + heads * 2;
    t.kept = kept;
    const int64_t groups = heads * t.segments;
    if (groups > pages::kThreadsAtMost / kThreadsOf) return fail(QCF_ERR_UNSUPPORTED, "page evict: too many rows");
    const dim3 grid((unsigned)groups), block(kThreadsOf);
    top_clear_kernel<<<dim3((unsigned)((heads * kHist + 1023) / 1024)), dim3(256), 0, st>>>(t.hist, heads * kHist);
    QCF_TRY_LAUNCH("page evict");
    top_count_kernel<0><<<grid, block, 0, st>>>(t);
    top_count_kernel<1><<<grid, block, 0, st>>>(t);
    top_count_kernel<2><<<grid, block, 0, st>>>(t);
    top_keep_kernel<false><<<grid, block, 0, st>>>(t);
    top_keep_kernel<true><<<grid, block, 0, st>>>(t);
    QCF_TRY_LAUNCH("page evict: tokens");
  } else {
    // (a page of one token: the choice between pages is one between tokens)
    QCF_TRY(launch_page_top(weights, len, B, L.n_kv_heads, 1, c.max_pages * c.page_size, n_keep, n_first, n_last, kept, st));
  }
#define QCF_LAUNCH(T, D, EIGHT)                                                                              \
  do {                                                                                                       \
    if (to.bounds) evict_kernel<T, D, EIGHT, true><<<dim3((unsigned)blocks), dim3(threads), 0, st>>>(a);     \
    else evict_kernel<T, D, EIGHT, false><<<dim3((unsigned)blocks), dim3(threads), 0, st>>>(a);              \
  } while (0)
#define QCF_PAGES(T, D) do { if (scales) QCF_LAUNCH(T, D, true); else QCF_LAUNCH(T, D, false); } while (0)
  if (L.dtype == QCF_DTYPE_BF16) {
    if (L.head_dim == 128) QCF_PAGES(bf16_t, 128); else QCF_PAGES(bf16_t, 64);
  } else {
    if (L.head_dim == 128) QCF_PAGES(float, 128); else QCF_PAGES(float, 64);
  }
#undef QCF_PAGES
#undef QCF_LAUNCH
  return check_launch("page evict");
}

}  // namespace qcf

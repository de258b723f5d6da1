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
  int Hkv, n_keep, log2_from, log2_to, pages;            // pages of `to` that n_keep tokens fill
};

// One workgroup per (request, KV head, page of the new cache), a wave of it to a block of 16 tokens: their numbers, their pages and then
// the rows, all of a block on their way together.  Bound by memory: every kept row is read and written once.
template <typename T, int D, bool EIGHT>
__global__ __launch_bounds__(256) void evict_kernel(EvictArgs a) {
  constexpr int kSize = EIGHT ? 1 : (int)sizeof(T), kIn = 16 / kSize;                // elements of a 16-byte vector
  constexpr int VPR = D * kSize / 16, RPI = 64 / VPR, ITS = kBlock / RPI;
  __shared__ float s_bound[2][4][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int64_t head = blockIdx.x / a.pages;             // (request, KV head)
  const int page = (int)(blockIdx.x - head * a.pages);
  const int64_t b = head / a.Hkv;
  const int g = (int)(head - b * a.Hkv), first = page << a.log2_to;
  const int32_t* kept = a.kept + head * a.n_keep;
  auto entry = [&](int j) { return j < a.n_keep ? kept[j] : -1; };
  const int dst_page = a.to.table[b * a.to.max_pages + page];
  const bool there = dst_page >= 0 && dst_page < a.to.n_pages;
  float lo[kIn], hi[kIn];
#pragma unroll
  for (int e = 0; e < kIn; ++e) { lo[e] = INFINITY; hi[e] = -INFINITY; }
  const int row = lane / VPR, part = lane % VPR;         // of this lane in each step of RPI rows
  for (int slot = wave * kBlock; slot < a.to.page_size; slot += waves * kBlock) {
    const int j0 = first + slot;
    if (j0 > 0 && entry(j0) < 0) break;                  // (of the wave)
    // lane l % 16 has token l % 16 of the block
    const int t = entry(j0 + (lane & 15));
    const int count = (int)__popcll(__ballot(t >= 0) & 0xffffu);
    if (g == 0 && lane == 0 && (count < kBlock || entry(j0 + kBlock) < 0)) a.to_len[b] = j0 + count;
    const int p = t >> a.log2_from, s = t & (a.from.page_size - 1);
    const int phys = t >= 0 && p < a.from.max_pages ? a.from.table[b * a.from.max_pages + p] : -1;
    const bool found = phys >= 0 && phys < a.from.n_pages;
    const int64_t src = found ? (phys * a.from.page_stride + s * a.from.slot_stride + g * a.from.head_stride) * kSize : -1;
    if (a.to_weights && lane < count)
      a.to_weights[(head * a.to.max_pages << a.log2_to) + j0 + lane] = found ? a.weights[(head * a.from.max_pages << a.log2_from) + t] : 0.f;
    if (!there) continue;
    float scale[2] = {0.f, 0.f};
    if constexpr (EIGHT) {
#pragma unroll
      for (int which = 0; which < 2; ++which)
        if (found) scale[which] = a.scales[scale_at(phys, a.Hkv, g, which, s, a.log2_from)];
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
    const int64_t dst = (dst_page * a.to.page_stride + slot * a.to.slot_stride + g * a.to.head_stride) * kSize + part * 16;
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
        if (lane == 0) a.to_scales[scale_at(dst_page, a.Hkv, g, which, slot, a.log2_to)] = now;
#pragma unroll
        for (int it = 0; it < ITS; ++it) {
          const float was = __shfl(scale[which], it * RPI + row, 64);
          if (was == now) continue;                      // (the codes stay)
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
        if (which == 0 && a.to.bounds) {
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
          for (int e = 0; e < kIn; ++e) { lo[e] = least(lo[e], f[e]); hi[e] = largest(hi[e], f[e]); }
        }
      }
    }
  }
  if (!there || !a.to.bounds || entry(first) < 0) return;              // (of the workgroup)
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
  T* bounds = static_cast<T*>(a.to.bounds) + ((int64_t)dst_page * a.Hkv + g) * 2 * D;
  for (int item = threadIdx.x; item < 2 * D; item += blockDim.x) {
    const bool low = item < D;
    float v = s_bound[low ? 0 : 1][0][item % D];
    for (int w = 1; w < waves; ++w) v = low ? least(v, s_bound[0][w][item % D]) : largest(v, s_bound[1][w][item % D]);
    Elem<T>::store(bounds + item, v);
  }
}

}  // namespace

qcf_status launch_page_evict(const qcf_layer_desc& L, const qcf_page_cache& c, const float* scales, int32_t B, const int32_t* len,
                             const float* weights, int32_t n_keep, int32_t n_first, int32_t n_last, const qcf_page_cache& to,
                             float* to_scales, int32_t* kept, float* to_weights, int32_t* to_len, hipStream_t st) {
  EvictArgs a;
  a.from = c; a.to = to; a.scales = scales; a.to_scales = to_scales;
  a.weights = weights; a.to_weights = to_weights; a.kept = kept; a.to_len = to_len;
  a.Hkv = L.n_kv_heads; a.n_keep = n_keep;
  a.log2_from = __builtin_ctz((unsigned)c.page_size);
  a.log2_to = __builtin_ctz((unsigned)to.page_size);
  a.pages = (n_keep + to.page_size - 1) / to.page_size;
  const int threads = 64 * std::min(4, to.page_size / kBlock);
  const int64_t heads = (int64_t)B * L.n_kv_heads, blocks = heads * a.pages;
  if (blocks > pages::kThreadsAtMost / threads || heads > pages::kThreadsAtMost / pages::kTopThreads)
    return fail(QCF_ERR_UNSUPPORTED, "page evict: too many rows");
  // (a page of one token: the choice between pages is one between tokens)
  QCF_TRY(launch_page_top(weights, len, B, L.n_kv_heads, 1, c.max_pages * c.page_size, n_keep, n_first, n_last, kept, st));
#define QCF_LAUNCH(T, D, EIGHT) evict_kernel<T, D, EIGHT><<<dim3((unsigned)blocks), dim3(threads), 0, st>>>(a)
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

// Attention of the newest tokens over a cache in pages.
#include "qcf_internal.h"

namespace qcf {
namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct PageAttnArgs {
  qcf_page_cache c;
  const void* q;
  const int32_t* seen;
  const int32_t* pages;
  int n_keep, B, n_q, H, Hkv, log2_page;
  void* o;
  float* lse;
};

// One workgroup per (row, head); a wave takes every fourth token, its lanes the elements of the head.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void page_attn_kernel(PageAttnArgs a) {
  constexpr int E = D / 64, WAVES = kThreads / 64;
  __shared__ float s_m[WAVES], s_l[WAVES], s_o[WAVES][D];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = blockIdx.x / a.H;                  // (request, new row)
  const int h = (int)(blockIdx.x - row * a.H), g = h / (a.H / a.Hkv), b = (int)(row / a.n_q);
  const int64_t seen = min((int64_t)max(a.seen[row], 0), (int64_t)a.c.max_pages << a.log2_page);
  const int count = (int)((seen + a.c.page_size - 1) >> a.log2_page);
  const int32_t* list = a.pages ? a.pages + (row * a.Hkv + g) * a.n_keep : nullptr;
  const int n_pages = list ? a.n_keep : count;
  float x[E], o[E];
  const T* q = static_cast<const T*>(a.q) + (row * a.H + h) * D;
#pragma unroll
  for (int e = 0; e < E; ++e) { x[e] = Elem<T>::load(q + lane + 64 * e); o[e] = 0.f; }
  const float scale = kLog2e / sqrtf((float)D);
  float m = -INFINITY, l = 0.f;
  bool any = false;
  for (int i = 0; i < n_pages; ++i) {
    const int p = list ? list[i] : i;
    if (p < 0 || p >= count) continue;
    const int phys = a.c.table[(int64_t)b * a.c.max_pages + p];
    if (phys < 0 || phys >= a.c.n_pages) continue;
    const int n = (int)min((int64_t)a.c.page_size, seen - ((int64_t)p << a.log2_page));
    const int64_t at = phys * a.c.page_stride + g * a.c.head_stride;
    for (int s = wave; s < n; s += WAVES) {
      const T* k = static_cast<const T*>(a.c.k) + at + s * a.c.slot_stride;
      const T* v = static_cast<const T*>(a.c.v) + at + s * a.c.slot_stride;
      float dot = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) dot += x[e] * Elem<T>::load(k + lane + 64 * e);
      const float logit = wave_sum(dot) * scale;
      any = true;
      const float top = fmaxf(m, logit);
      const float ref = top == -INFINITY ? 0.f : top;     // (all logits so far -inf: their weights are 0, not NaN)
      const float keep = m == top ? 1.f : exp2f(m - ref), w = exp2f(logit - ref);
      m = top;
      l = l * keep + w;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = o[e] * keep + w * Elem<T>::load(v + lane + 64 * e);
    }
  }
  if (any && m == -INFINITY) l = NAN;
  if (lane == 0) { s_m[wave] = m; s_l[wave] = l; }
#pragma unroll
  for (int e = 0; e < E; ++e) s_o[wave][lane + 64 * e] = o[e];
  __syncthreads();
  if (wave > 0) return;
  float top = s_m[0];
  for (int w = 1; w < WAVES; ++w) top = fmaxf(top, s_m[w]);
  float total = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  for (int w = 0; w < WAVES; ++w) {
    // (a part whose logits are all -inf weighs nothing beside others, and makes the row NaN alone)
    if (s_m[w] == -INFINITY && !(top == -INFINITY && s_l[w] != 0.f)) continue;
    const float f = s_m[w] == top ? 1.f : exp2f(s_m[w] - top);
    total += f * s_l[w];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] += f * s_o[w][lane + 64 * e];
  }
  const bool nothing = top == -INFINITY && total == 0.f;
  T* out = static_cast<T*>(a.o) + (row * a.H + h) * D;
#pragma unroll
  for (int e = 0; e < E; ++e) Elem<T>::store(out + lane + 64 * e, nothing ? 0.f : o[e] / total);
  if (a.lse && lane == 0) a.lse[row * a.H + h] = nothing ? -INFINITY : (top + log2f(total)) * kLn2;
}

}  // namespace

size_t page_attn_workspace(const qcf_layer_desc&, const qcf_page_cache&, int32_t, int32_t, int32_t) { return 0; }

qcf_status launch_page_attn(const qcf_layer_desc& L, const qcf_page_cache& c, int32_t B, int32_t n_q, const void* q,
                            const int32_t* seen, const int32_t* pages, int32_t n_keep, void* o, float* lse, void*,
                            hipStream_t st) {
  PageAttnArgs a;
  a.c = c; a.q = q; a.seen = seen; a.pages = pages; a.n_keep = n_keep;
  a.B = B; a.n_q = n_q; a.H = L.n_q_heads; a.Hkv = L.n_kv_heads;
  a.log2_page = __builtin_ctz((unsigned)c.page_size);
  a.o = o; a.lse = lse;
  const dim3 grid((unsigned)((int64_t)B * n_q * L.n_q_heads)), block(kThreads);
  if (L.dtype == QCF_DTYPE_BF16) {
    if (L.head_dim == 128) page_attn_kernel<bf16_t, 128><<<grid, block, 0, st>>>(a);
    else page_attn_kernel<bf16_t, 64><<<grid, block, 0, st>>>(a);
  } else {
    if (L.head_dim == 128) page_attn_kernel<float, 128><<<grid, block, 0, st>>>(a);
    else page_attn_kernel<float, 64><<<grid, block, 0, st>>>(a);
  }
  return check_launch("page attention");
}

}  // namespace qcf

// Decoding over a cache in pages: new rows into their pages, and the scores of a request's pages for its new queries.
#include "qcf_internal.h"

namespace qcf {
namespace {

constexpr int kThreads = 256;

// theta_i / 2 pi of a layer's rotary pairs, computed on the host: exp2 in float64 in front of every workgroup's first row would
// take longer than a decoding step's whole append.
struct Turns {
  double of[64];
};

struct AppendArgs {
  const void* q;
  const void* k;
  const void* v;
  int64_t q_stride, k_stride, v_stride;
  const int64_t* row_off;
  int64_t total_rows;
  const int32_t* len;
  const int32_t* pos;
  void* q_out;
  qcf_page_cache c;
  int B, H, Hkv, log2_page;
};

// (cos, sin) of `positions` times a frequency given in turns per position.  The product is rounded at 2^-53 of up to 2^31
// turns; its fraction is exact in float64 and loses less than 2^-25 of a turn as a float.
template <typename T>
__device__ __forceinline__ float2 turn_at(double positions, double turns) {
  const double t = positions * turns;
  const float f = (float)(t - __builtin_rint(t));
  float sn, cn;
  sincospif(2.f * f, &sn, &cn);
  return make_float2(cn, sn);
}

// The least and the largest of two values, not a number if either is not.
__device__ __forceinline__ float least(float a, float b) { return __builtin_elementwise_minimum(a, b); }
__device__ __forceinline__ float largest(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// Request of a unit: units of request b start at row_off[b] / page + 2 b, which leaves room for every page that its rows can touch
// (n rows touch at most floor((n - 1) / page) + 2), so that no sum over the requests stands in front of the rows.  Every wave
// counts the requests that start at or before the unit.
__device__ __forceinline__ int request_of(const AppendArgs& a, int64_t unit, int lane) {
  int before = 0;
  for (int b0 = 1; b0 < a.B; b0 += 64) {
    const int b = b0 + lane;
    const int64_t off = a.row_off[min(b, a.B - 1)];
    const int64_t first = (min(max(off, (int64_t)0), a.total_rows) >> a.log2_page) + 2 * (int64_t)b;
    before += (int)__popcll(__ballot(b < a.B && first <= unit));
  }
  return before;
}

// One workgroup per (page that gets rows, KV head): its keys, turned and rounded, their bounds, its values, and the queries of
// the head's group.  A thread takes VEC rotary pairs of a row, two 16-byte vectors.
template <typename T, int D, int STYLE>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a, Turns turns) {
  constexpr int VEC = Elem<T>::kVec, TPR = D / 2 / VEC, SLOTS = kThreads / TPR, WAVES = kThreads / 64;
  __shared__ float s_lo[WAVES][D], s_hi[WAVES][D];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t unit = blockIdx.x / a.Hkv;
  const int g = (int)(blockIdx.x - unit * a.Hkv), G = a.H / a.Hkv;
  const int b = request_of(a, unit, lane);
  const int64_t r0 = min(max(a.row_off[b], (int64_t)0), a.total_rows);
  const int64_t r1 = min(max(a.row_off[b + 1], r0), a.total_rows);
  const int64_t len = a.len[b], page = a.c.page_size;
  const int64_t p = (len >> a.log2_page) + unit - ((r0 >> a.log2_page) + 2 * (int64_t)b);
  const int64_t t0 = max(p * page, len), t1 = min((p + 1) * page, len + (r1 - r0));
  if (t0 >= t1) return;
  const int n = (int)(t1 - t0);
  const int64_t row0 = r0 + (t0 - len);
  const int64_t phys = p >= 0 && p < a.c.max_pages ? a.c.table[(int64_t)b * a.c.max_pages + p] : -1;
  const bool there = phys >= 0 && phys < a.c.n_pages;
  const int slot0 = (int)(t0 - p * page);
  const int64_t at = there ? phys * a.c.page_stride + g * a.c.head_stride + slot0 * a.c.slot_stride : 0;

  const int i0 = tid % TPR * VEC;                       // first pair
  const int e0 = STYLE == 0 ? i0 : 2 * i0, e1 = STYLE == 0 ? i0 + D / 2 : 2 * i0 + VEC;
  auto turned = [&](const T* src, int64_t row, u32x4& ra, u32x4& rb) {
    ra = *reinterpret_cast<const u32x4*>(src + e0);
    rb = *reinterpret_cast<const u32x4*>(src + e1);
    if (!a.pos) return;
    const double pos = (double)a.pos[row];
    float f[2 * VEC], o[2 * VEC];
    Vec16<T>::unpack(ra, f);
    Vec16<T>::unpack(rb, f + VEC);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const int ia = STYLE == 0 ? i : 2 * i, ib = STYLE == 0 ? i + VEC : 2 * i + 1;
      turn_pair(f[ia], f[ib], turn_at<T>(pos, turns.of[i0 + i]), o[ia], o[ib]);
    }
    ra = Vec16<T>::pack(o);
    rb = Vec16<T>::pack(o + VEC);
  };

  if (there) {
    float lo[2 * VEC], hi[2 * VEC];
#pragma unroll
    for (int e = 0; e < 2 * VEC; ++e) { lo[e] = INFINITY; hi[e] = -INFINITY; }
    const T* k = static_cast<const T*>(a.k) + row0 * a.k_stride + g * D;
    const T* v = static_cast<const T*>(a.v) + row0 * a.v_stride + g * D;
    T* kc = static_cast<T*>(a.c.k) + at;
    T* vc = static_cast<T*>(a.c.v) + at;
    for (int j = tid / TPR; j < n; j += SLOTS) {
      u32x4 ra, rb;
      turned(k + j * a.k_stride, row0 + j, ra, rb);
      *reinterpret_cast<u32x4*>(kc + j * a.c.slot_stride + e0) = ra;
      *reinterpret_cast<u32x4*>(kc + j * a.c.slot_stride + e1) = rb;
      *reinterpret_cast<u32x4*>(vc + j * a.c.slot_stride + e0) = *reinterpret_cast<const u32x4*>(v + j * a.v_stride + e0);
      *reinterpret_cast<u32x4*>(vc + j * a.c.slot_stride + e1) = *reinterpret_cast<const u32x4*>(v + j * a.v_stride + e1);
      float f[2 * VEC];
      Vec16<T>::unpack(ra, f);
      Vec16<T>::unpack(rb, f + VEC);
#pragma unroll
      for (int e = 0; e < 2 * VEC; ++e) { lo[e] = least(lo[e], f[e]); hi[e] = largest(hi[e], f[e]); }
    }
    if (a.c.bounds) {
#pragma unroll
      for (int x = TPR; x < 64; x *= 2)
#pragma unroll
        for (int e = 0; e < 2 * VEC; ++e) {
          lo[e] = least(lo[e], __shfl_xor(lo[e], x, 64));
          hi[e] = largest(hi[e], __shfl_xor(hi[e], x, 64));
        }
      if (lane < TPR) {
#pragma unroll
        for (int e = 0; e < 2 * VEC; ++e) {
          const int col = e < VEC ? e0 + e : e1 + e - VEC;
          s_lo[wave][col] = lo[e];
          s_hi[wave][col] = hi[e];
        }
      }
      __syncthreads();                                  // (by all threads: `there` is the workgroup's)
      for (int col = tid; col < 2 * D; col += kThreads) {
        T* bound = static_cast<T*>(a.c.bounds) + (phys * a.Hkv + g) * 2 * D + col;
        const bool low = col < D;
        float x = low ? s_lo[0][col] : s_hi[0][col - D];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) x = low ? least(x, s_lo[w][col]) : largest(x, s_hi[w][col - D]);
        if (slot0 > 0) {
          const float old = Elem<T>::load(bound);
          x = low ? least(x, old) : largest(x, old);
        }
        Elem<T>::store(bound, x);
      }
    }
  }
  if (a.q) {
    for (int item = tid / TPR; item < n * G; item += SLOTS) {
      const int j = item / G, h = g * G + item - j * G;
      const int64_t row = row0 + j;
      u32x4 ra, rb;
      turned(static_cast<const T*>(a.q) + row * a.q_stride + h * D, row, ra, rb);
      T* out = static_cast<T*>(a.q_out) + (row * a.H + h) * D;
      *reinterpret_cast<u32x4*>(out + e0) = ra;
      *reinterpret_cast<u32x4*>(out + e1) = rb;
    }
  }
}

// Scores of pages (the definition is in qcf_pages.h): one wave per (page, row, KV head).  Products of two stored values are exact
// in float64 and so, for values within 2^29 of each other, are their sums: the order of the sum does not decide between pages.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void page_score_kernel(qcf_page_cache c, const T* __restrict__ q,
                                                              const int32_t* __restrict__ seen, int n_q, int H, int Hkv,
                                                              int log2_page, float* __restrict__ score) {
  const int lane = threadIdx.x & 63;
  const int64_t row = blockIdx.y;                       // (request, new row)
  const int b = (int)(row / n_q), G = H / Hkv;
  const int64_t item = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  const int g = (int)(item % Hkv);
  const int64_t p = item / Hkv;
  const int count = (int)(((int64_t)max(seen[row], 0) + c.page_size - 1) >> log2_page);
  if (p >= min(count, c.max_pages)) return;
  const int phys = c.table[(int64_t)b * c.max_pages + p];
  float best = -INFINITY;
  if (phys >= 0 && phys < c.n_pages) {
    const T* lo = static_cast<const T*>(c.bounds) + ((int64_t)phys * Hkv + g) * 2 * D;
    for (int h = 0; h < G; ++h) {
      const T* x = q + (row * H + g * G + h) * D;
      double sum = 0.0;
#pragma unroll
      for (int e = lane; e < D; e += 64) {
        const double f = (double)Elem<T>::load(x + e);
        sum += fmin(f, 0.0) * (double)Elem<T>::load(lo + e) + fmax(f, 0.0) * (double)Elem<T>::load(lo + D + e);
        if (f != f) sum = f;
      }
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d, 64);
      const float s = (float)sum;
      best = fmaxf(best, s == s ? fmaxf(s, -3.402823466e38f) : INFINITY);
    }
  }
  if (lane == 0) score[(row * Hkv + g) * c.max_pages + p] = best;
}

}  // namespace

qcf_status launch_page_append(const qcf_layer_desc& L, const qcf_page_cache& c, int32_t B, const void* q, int64_t q_stride,
                              const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int64_t* row_off,
                              int64_t total_rows, const int32_t* len, const int32_t* pos, void* q_out, hipStream_t st) {
  AppendArgs a;
  a.q = q; a.k = k; a.v = v;
  a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride;
  a.row_off = row_off; a.total_rows = total_rows; a.len = len; a.pos = pos; a.q_out = q_out;
  a.c = c;
  a.B = B; a.H = L.n_q_heads; a.Hkv = L.n_kv_heads;
  a.log2_page = __builtin_ctz((unsigned)c.page_size);
  Turns turns;
  const double log2_base = std::log2(L.rope_base);
  for (int i = 0; i < L.head_dim / 2; ++i) turns.of[i] = std::exp2(-2.0 * i / L.head_dim * log2_base) * 0.15915494309189533577;
  const int64_t blocks = ((total_rows >> a.log2_page) + 2 * (int64_t)B) * L.n_kv_heads;
  if (blocks > 0x7fffffff) return fail(QCF_ERR_UNSUPPORTED, "page append: too many rows");
#define QCF_LAUNCH(T, D, S) append_kernel<T, D, S><<<dim3((unsigned)blocks), dim3(kThreads), 0, st>>>(a, turns)
#define QCF_STYLE(T, D) do { if (L.rope_style == 0) QCF_LAUNCH(T, D, 0); else QCF_LAUNCH(T, D, 1); } while (0)
  if (L.dtype == QCF_DTYPE_BF16) {
    if (L.head_dim == 128) QCF_STYLE(bf16_t, 128); else QCF_STYLE(bf16_t, 64);
  } else {
    if (L.head_dim == 128) QCF_STYLE(float, 128); else QCF_STYLE(float, 64);
  }
#undef QCF_STYLE
#undef QCF_LAUNCH
  return check_launch("page append");
}

size_t page_select_workspace(const qcf_layer_desc& L, const qcf_page_cache& c, int32_t B, int32_t n_q) {
  return align_up((size_t)B * n_q * L.n_kv_heads * c.max_pages * sizeof(float), 256);
}

qcf_status launch_page_select(const qcf_layer_desc& L, const qcf_page_cache& c, int32_t B, int32_t n_q, const void* q,
                              const int32_t* seen, int32_t n_keep, int32_t n_first, int32_t n_last, int32_t* pages, void* ws,
                              hipStream_t st) {
  float* score = static_cast<float*>(ws);
  const int64_t rows = (int64_t)B * n_q, items = (int64_t)c.max_pages * L.n_kv_heads, blocks = (items + 3) / 4;
  if (rows * L.n_kv_heads > 0x7fffffff || blocks > 0x7fffffff) return fail(QCF_ERR_UNSUPPORTED, "page select: too many rows");
  const int log2_page = __builtin_ctz((unsigned)c.page_size);
  if (rows > 65535) return fail(QCF_ERR_UNSUPPORTED, "page select: %lld rows > 65535", (long long)rows);
#define QCF_LAUNCH(T, D)                                                                                                  \
  page_score_kernel<T, D><<<dim3((unsigned)blocks, (unsigned)rows), dim3(kThreads), 0, st>>>(c, static_cast<const T*>(q), \
                                                                                              seen, n_q, L.n_q_heads, L.n_kv_heads, log2_page, score)
  if (L.dtype == QCF_DTYPE_BF16) {
    if (L.head_dim == 128) QCF_LAUNCH(bf16_t, 128); else QCF_LAUNCH(bf16_t, 64);
  } else {
    if (L.head_dim == 128) QCF_LAUNCH(float, 128); else QCF_LAUNCH(float, 64);
  }
#undef QCF_LAUNCH
  QCF_TRY_LAUNCH("page scores");
  return launch_page_top(score, seen, rows, L.n_kv_heads, c.page_size, c.max_pages, n_keep, n_first, n_last, pages, st);
}

}  // namespace qcf

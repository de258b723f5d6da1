// What the appends to pages (pages.hip) and to 8-bit pages (page8_append.hip) share: the rows of a unit, rounding, bounds.
#pragma once

#include "qcf_internal.h"
#include "page_layout.h"

namespace qcf {
namespace {

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
  int log2_unit;                  // tokens of a unit: a page's, or fewer
  double neg2_over_d_log2base;
};

// (cos, sin) of `positions` times a frequency given in turns per position.  The product is rounded at 2^-53 of up to 2^31
// turns; its fraction is exact in float64 and loses less than 2^-25 of a turn as a float.
template <typename T>
__device__ __forceinline__ float2 turn_at(double positions, double turns) {
  const double t = positions * turns;
  const float f = (float)(t - __builtin_rint(t));
  // bf16: the hardware's sine and cosine of a fraction of a turn, at most 1.3e-7 off (731 rows with heads of 64, in pages of 64:
  // 10.8 us with sincospif and rounding by integers, 8.1 with both in hardware)
  if constexpr (sizeof(T) == 2) return make_float2(__builtin_amdgcn_cosf(f), __builtin_amdgcn_sinf(f));
  float sn, cn;
  sincospif(2.f * f, &sn, &cn);
  return make_float2(cn, sn);
}

// sixteen bytes of rounded elements
template <typename T>
__device__ __forceinline__ u32x4 rounded(const float* f) {
  if constexpr (sizeof(T) == 4) return Vec16<T>::pack(f);
  else return mk4(cvt_pk_bf16(f[0], f[1]), cvt_pk_bf16(f[2], f[3]), cvt_pk_bf16(f[4], f[5]), cvt_pk_bf16(f[6], f[7]));
}

// The least and the largest of two values, not a number if either is not.
__device__ __forceinline__ float least(float a, float b) { return __builtin_elementwise_minimum(a, b); }
__device__ __forceinline__ float largest(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// Request of a unit (a page that gets rows): units of request b start at row_off[b] / page + 2 b (pages::append_units), so that no sum
// over the requests stands in front of the rows.  Every wave looks for the last request that starts at or before the unit; offsets and lengths of the
// first 64 are on their way together.
struct Request {
  int b;
  int64_t r0, r1, len, unit0;     // its rows, the tokens that it holds, its first unit
};
__device__ __forceinline__ Request request_of(const AppendArgs& a, int64_t unit, int lane) {
  auto clamped = [&](int64_t off) { return min(max(off, (int64_t)0), a.total_rows); };
  auto first = [&](int b, int64_t off) { return (off >> a.log2_unit) + 2 * (int64_t)b; };
  const int mine = min(lane, a.B - 1);
  const int64_t off = clamped(a.row_off[mine]), next = clamped(a.row_off[mine + 1]);
  const int len = a.len[mine];
  int before = (int)__popcll(__ballot(lane >= 1 && lane < a.B && first(lane, off) <= unit));
  if (a.B > 64) {
    // the request lies in [at, end): 64 places of that are looked at a time
    int at = 0, end = a.B;
    while (end - at > 1) {
      const int step = (end - at + 63) / 64, b = at + lane * step;
      const int64_t o = clamped(a.row_off[min(b, a.B - 1)]);
      const int n = (int)__popcll(__ballot(b < end && first(b, o) <= unit));
      at += max(n - 1, 0) * step;
      end = min(end, at + step);
    }
    before = at;
  }
  Request r;
  r.b = before;
  if (before < 64) {
    // (rows are at most 2^30)
    r.r0 = __builtin_amdgcn_readlane((int)off, before);
    r.r1 = __builtin_amdgcn_readlane((int)next, before);
    r.len = __builtin_amdgcn_readlane(len, before);
  } else {
    r.r0 = clamped(a.row_off[before]);
    r.r1 = clamped(a.row_off[before + 1]);
    r.len = a.len[before];
  }
  r.r1 = max(r.r1, r.r0);
  r.unit0 = first(before, r.r0);
  return r;
}

inline AppendArgs append_args(const qcf_layer_desc& L, const qcf_page_cache& c, int32_t B, const void* q, int64_t q_stride,
                              const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int64_t* row_off,
                              int64_t total_rows, const int32_t* len, const int32_t* pos, void* q_out) {
  AppendArgs a;
  a.q = q; a.k = k; a.v = v;
  a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride;
  a.row_off = row_off; a.total_rows = total_rows; a.len = len; a.pos = pos; a.q_out = q_out;
  a.c = c;
  a.B = B; a.H = L.n_q_heads; a.Hkv = L.n_kv_heads;
  a.log2_page = a.log2_unit = __builtin_ctz((unsigned)c.page_size);
  a.neg2_over_d_log2base = -2.0 / L.head_dim * std::log2(L.rope_base);
  return a;
}

}  // namespace
}  // namespace qcf

// Decoding over a cache in 8-bit pages: new rows into their pages.
#include <type_traits>

#include "qcf_internal.h"
#include "page_layout.h"
#include "append_common.h"
#include "eight.h"

namespace qcf {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

// (cos, sin) of `positions` times a frequency in turns, in 64 bits: a rotated key is rounded to a code as the formula has it.  (In float32
// 32 to 40 of 34 million codes were a whole step off, elements within an error of 2^-24 of the middle between two codes.)  The angle is
// reduced to an eighth of a turn around a quarter; Taylor's series are 2^-45 off there.  (731 rows 10.2 us, 9.6 in
// float32; 8 rows 6.7 in the kernel, 6.0; 36K 159 both ways.)
__device__ __forceinline__ double2 exact_turn(double positions, double turns) {
  const double t = positions * turns, r = t - __builtin_rint(t), quarters = __builtin_rint(4.0 * r);
  const double x = (r - 0.25 * quarters) * 6.283185307179586477, y = x * x;
  double sn = 1.0 / 6227020800, cn = -1.0 / 87178291200;                 // 1 / 13!, -1 / 14!
  constexpr double kSin[] = {-1.0 / 39916800, 1.0 / 362880, -1.0 / 5040, 1.0 / 120, -1.0 / 6, 1.0};
  constexpr double kCos[] = {1.0 / 479001600, -1.0 / 3628800, 1.0 / 40320, -1.0 / 720, 1.0 / 24, -0.5, 1.0};
#pragma unroll
  for (int i = 0; i < 6; ++i) sn = __builtin_fma(sn, y, kSin[i]);
#pragma unroll
  for (int i = 0; i < 7; ++i) cn = __builtin_fma(cn, y, kCos[i]);
  sn *= x;
  const int q = (int)quarters & 3;
  const double c = q & 1 ? sn : cn, s = q & 1 ? cn : sn;
  return make_double2(q == 1 || q == 2 ? -c : c, q & 2 ? -s : s);
}

// x as a float of 21 bits that lies on the same side of every code, and of every middle between two, as x does: what these bits cannot hold
// makes the last one odd.
__device__ __forceinline__ float odd(double x) {
  const uint64_t bits = (uint64_t)__double_as_longlong(x);
  const uint32_t high = (uint32_t)(bits >> 32) | min((uint32_t)bits, 1u);
  return (float)__longlong_as_double((int64_t)((uint64_t)high << 32));
}

// One workgroup per (unit that gets rows, `heads` KV heads of it): a block of 16 tokens, or, where the pages have bounds, a page.  A wave
// takes a block for one head as a whole, keys and values: it turns the keys, finds both largest elements, hence the scales, and stores
// the codes.  Where the block has tokens already and its scale grows, these are rounded again.  (heads: 1, 2 or 4; the waves of a head
// take its blocks in turn.)  Bound by memory where many rows come (36K rows, 32 / 8 heads of 128: 159 us, 5.1 TB/s of what
// is read and written, a copy's rate), by the chain offsets -> table and positions -> factors -> largest elements -> codes where few do (8
// rows 6.7 us).
template <typename T, int D, int STYLE>
__global__ __launch_bounds__(kThreads) void append8_kernel(AppendArgs a, float* __restrict__ scales, int heads) {
  constexpr int VEC = Elem<T>::kVec, TPR = D / 2 / VEC, PAIRS = D / 2, ROWS = 4096 / D;
  constexpr int RPI = 64 / TPR, ITS = kBlock / RPI;                      // rows of a block side by side in a wave, and how often
  constexpr int kWords = VEC / 4;                                        // words of half a lane's codes
  typedef uint32_t codes_t __attribute__((ext_vector_type(kWords)));
  // (the pairs of a lane TPR apart, rows 16 * TPR bytes more than theirs: lanes read what lies side by side, in banks of their own)
  __shared__ __align__(16) double2 s_turn[ROWS][PAIRS + TPR];
  __shared__ float s_bound[2][kWaves][D];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int parts = a.Hkv / heads;
  const int64_t unit = blockIdx.x / parts;
  const int g0 = (int)(blockIdx.x - unit * parts) * heads, G = a.H / a.Hkv;
  const Request rq = request_of(a, unit, lane);
  const double turns = exp2(a.neg2_over_d_log2base * (double)(tid % PAIRS)) * 0.15915494309189533577;
  const int64_t page = a.c.page_size, len = rq.len;
  const int64_t begin = ((len >> a.log2_unit) + unit - rq.unit0) << a.log2_unit, p = begin >> a.log2_page;
  const int64_t t0 = max(begin, len), t1 = min(begin + ((int64_t)1 << a.log2_unit), len + (rq.r1 - rq.r0));
  if (t0 >= t1) return;
  const int64_t phys = p >= 0 && p < a.c.max_pages ? a.c.table[(int64_t)rq.b * a.c.max_pages + p] : -1;
  const bool there = phys >= 0 && phys < a.c.n_pages;
  const int slot0 = (int)(t0 - p * page), slot1 = (int)(t1 - p * page);
  const int64_t row0 = rq.r0 + (t0 - len) - slot0;                       // row of slot s: row0 + s

  const int place = lane % TPR, i0 = place * VEC;
  const int e0 = STYLE == 0 ? i0 : 2 * i0, e1 = STYLE == 0 ? i0 + PAIRS : 2 * i0 + VEC;
  auto read = [&](const T* src, float* f) {
    Vec16<T>::unpack(*reinterpret_cast<const u32x4*>(src + e0), f);
    Vec16<T>::unpack(*reinterpret_cast<const u32x4*>(src + e1), f + VEC);
  };
  // (exact: of a key, which will be coded)
  auto turn = [&](auto exact, int j, float* f) {
    if (!a.pos) return;
    float o[2 * VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const int ia = STYLE == 0 ? i : 2 * i, ib = STYLE == 0 ? i + VEC : 2 * i + 1;
      const double2 w = s_turn[j][i * TPR + place];
      if constexpr (exact.value) {
        o[ia] = odd(f[ia] * w.x - f[ib] * w.y);
        o[ib] = odd(f[ib] * w.x + f[ia] * w.y);
      } else {
        turn_pair(f[ia], f[ib], make_float2((float)w.x, (float)w.y), o[ia], o[ib]);
      }
    }
#pragma unroll
    for (int e = 0; e < 2 * VEC; ++e) f[e] = o[e];
  };
  auto store_codes = [&](uint8_t* dst, const float* f, float inv, codes_t (&c)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int w = 0; w < kWords; ++w) {
        const float* x = f + h * VEC + 4 * w;
        c[h][w] = codes_of(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
      }
      *reinterpret_cast<codes_t*>(dst + (h ? e1 : e0)) = c[h];
    }
  };

  const int head = wave % heads, turn_of = wave / heads, turns_of = kWaves / heads, g = g0 + head;
  float lo[2 * VEC], hi[2 * VEC];
#pragma unroll
  for (int e = 0; e < 2 * VEC; ++e) { lo[e] = INFINITY; hi[e] = -INFINITY; }
  for (int c0 = slot0 / ROWS * ROWS; c0 < slot1; c0 += ROWS) {
    const int first = max(slot0, c0), last = min(slot1, c0 + ROWS);       // slots of the chunk that get rows
    if (a.pos) {
      if (c0 > slot0) __syncthreads();
      // (a block's at a time: positions and factors on their way together; rows behind the last one are that one again)
      constexpr int kStep = kThreads / PAIRS, kAt = kBlock / kStep;
      for (int s0 = first + tid / PAIRS; s0 < last; s0 += kBlock) {
        int32_t pos[kAt];
#pragma unroll
        for (int i = 0; i < kAt; ++i) pos[i] = a.pos[row0 + min(s0 + i * kStep, last - 1)];
#pragma unroll
        for (int i = 0; i < kAt; ++i)
          s_turn[min(s0 + i * kStep, last - 1) - c0][tid % VEC * TPR + tid % PAIRS / VEC] = exact_turn((double)pos[i], turns);
      }
      __syncthreads();
    }
    for (int b0 = (first / kBlock + turn_of) * kBlock; there && b0 < last; b0 += turns_of * kBlock) {
      const bool joins = b0 < slot0;                     // the block has tokens already
      const int64_t cell = phys * a.c.page_stride + g * a.c.head_stride;
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        const T* src = static_cast<const T*>(which ? a.v : a.k) + g * D;
        const int64_t stride = which ? a.v_stride : a.k_stride;
        uint8_t* dst = static_cast<uint8_t*>(which ? a.c.v : a.c.k) + cell;
        float* scale = scales + scale_at(phys, a.Hkv, g, which, b0, a.log2_page);
        const float was = joins ? *scale : 0.f;
        float f[ITS][2 * VEC];
#pragma unroll
        for (int it = 0; it < ITS; ++it) {
          const int s = b0 + it * RPI + lane / TPR;
          read(src + (row0 + min(max(s, first), last - 1)) * stride, f[it]);
        }
        float amax = 0.f;
#pragma unroll
        for (int it = 0; it < ITS; ++it) {
          const int s = b0 + it * RPI + lane / TPR;
          const bool mine = s >= first && s < last;
          if (which == 0) turn(std::true_type{}, min(max(s, first), last - 1) - c0, f[it]);
#pragma unroll
          for (int e = 0; e < 2 * VEC; ++e) {
            if (!storable(f[it][e])) f[it][e] = NAN;
            amax = mine ? fmaxf(amax, __builtin_fabsf(f[it][e])) : amax;
          }
        }
        amax = wave_max(amax);
        const float now = fmaxf(scale_for(amax), was), inv = 1.f / now;
        if (lane == 0) *scale = now;
        const bool again = joins && now > was;
#pragma unroll
        for (int it = 0; it < ITS; ++it) {
          const int s = b0 + it * RPI + lane / TPR;
          uint8_t* at = dst + s * a.c.slot_stride;
          float scaled = inv;
          bool mine = s >= first && s < last;
          if (again && s < slot0) {                      // rounded again
            mine = true;
            scaled = was * inv;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const codes_t old = *reinterpret_cast<const codes_t*>(at + (h ? e1 : e0));
#pragma unroll
              for (int w = 0; w < kWords; ++w) values_of(old[w], f[it] + h * VEC + 4 * w);
            }
          }
          if (!mine) continue;
          codes_t c[2];
          store_codes(at, f[it], scaled, c);
          if (which == 0 && a.c.bounds) {
#pragma unroll
            for (int e = 0; e < 2 * VEC; e += 4) {
              float x[4];
              values_of(c[e / VEC][e % VEC / 4], x);
#pragma unroll
              for (int i = 0; i < 4; ++i) { lo[e + i] = least(lo[e + i], x[i] * now); hi[e + i] = largest(hi[e + i], x[i] * now); }
            }
          }
        }
      }
    }
    if (a.q) {
      const int q_vecs = heads * G * TPR, items = (last - first) * q_vecs;
      const T* q = static_cast<const T*>(a.q) + g0 * G * D;
      T* q_out = static_cast<T*>(a.q_out) + g0 * G * D;
      for (int at = tid; at < items; at += kThreads) {   // (kThreads is a multiple of TPR: the place stays)
        const int j = at / q_vecs, h = (at - j * q_vecs) / TPR, s = first + j;
        float f[2 * VEC];
        read(q + (row0 + s) * a.q_stride + h * D, f);
        turn(std::false_type{}, s - c0, f);
        T* dst = q_out + ((row0 + s) * a.H + h) * D;
        *reinterpret_cast<u32x4*>(dst + e0) = rounded<T>(f);
        *reinterpret_cast<u32x4*>(dst + e1) = rounded<T>(f + VEC);
      }
    }
  }
  if (!there || !a.c.bounds) return;                     // (of the workgroup)
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
      s_bound[0][wave][col] = lo[e];
      s_bound[1][wave][col] = hi[e];
    }
  }
  __syncthreads();
  T* bounds = static_cast<T*>(a.c.bounds) + (phys * a.Hkv + g0) * 2 * D;
  for (int item = tid; item < heads * 2 * D; item += kThreads) {
    const int h = item / (2 * D), col = item % D;
    const bool low = item % (2 * D) < D;
    float x = s_bound[low ? 0 : 1][h][col];
    for (int w = h + heads; w < kWaves; w += heads) x = low ? least(x, s_bound[0][w][col]) : largest(x, s_bound[1][w][col]);
    if (slot0 > 0) {
      const float was = Elem<T>::load(bounds + item);
      x = low ? least(x, was) : largest(x, was);
    }
    Elem<T>::store(bounds + item, x);
  }
}

}  // namespace

qcf_status launch_page8_append(const qcf_layer_desc& L, const qcf_page_cache& c, float* scales, int32_t B, const void* q,
                               int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                               const int64_t* row_off, int64_t total_rows, const int32_t* len, const int32_t* pos, void* q_out,
                               hipStream_t st) {
  AppendArgs a = append_args(L, c, B, q, q_stride, k, k_stride, v, v_stride, row_off, total_rows, len, pos, q_out);
  if (!c.bounds) a.log2_unit = __builtin_ctz((unsigned)kBlock);
  const int64_t units = pages::append8_units(c, B, total_rows);
  const int heads = pages::append8_heads(L, c, B, total_rows);
  const int64_t blocks = units * (L.n_kv_heads / heads);
  if (blocks > pages::kThreadsAtMost / kThreads) return fail(QCF_ERR_UNSUPPORTED, "page append: too many rows");
#define QCF_LAUNCH(T, D, S) append8_kernel<T, D, S><<<dim3((unsigned)blocks), dim3(kThreads), 0, st>>>(a, scales, heads)
#define QCF_STYLE(T, D) do { if (L.rope_style == 0) QCF_LAUNCH(T, D, 0); else QCF_LAUNCH(T, D, 1); } while (0)
  if (L.dtype == QCF_DTYPE_BF16) {
    if (L.head_dim == 128) QCF_STYLE(bf16_t, 128); else QCF_STYLE(bf16_t, 64);
  } else {
    if (L.head_dim == 128) QCF_STYLE(float, 128); else QCF_STYLE(float, 64);
  }
#undef QCF_STYLE
#undef QCF_LAUNCH
  return check_launch("page append in 8 bits");
}

}  // namespace qcf

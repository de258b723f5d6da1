// Decoding over a cache in pages: new rows into their pages, and the scores of a request's pages for its new queries.
#include "qcf_internal.h"
#include "page_layout.h"

namespace qcf {
namespace {

constexpr int kThreads = 256;

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

// Request of a unit: units of request b start at row_off[b] / page + 2 b (pages::append_units), so that no sum over the requests
// stands in front of the rows.  Every wave looks for the last request that starts at or before the unit; offsets and lengths of the
// first 64 are on their way together.
struct Request {
  int b;
  int64_t r0, r1, len, unit0;     // its rows, the tokens that it holds, its first unit
};
__device__ __forceinline__ Request request_of(const AppendArgs& a, int64_t unit, int lane) {
  auto clamped = [&](int64_t off) { return min(max(off, (int64_t)0), a.total_rows); };
  auto first = [&](int b, int64_t off) { return (off >> a.log2_page) + 2 * (int64_t)b; };
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

// One workgroup per (page that gets rows, `heads` KV heads of it): their keys, turned and rounded, the bounds, the values, and the
// queries of the heads' groups.  A thread takes VEC rotary pairs of a row, two 16-byte vectors.  The (cos, sin) of ROWS rows are
// kept in LDS for all heads: formed for every vector anew they took the vector unit longer than the rows took memory (32K rows, 8
// KV heads of 128: 238 us, 190 with them, 181 or 4.95 TB/s now).  Bound by memory there, and by the chain offsets -> rows, page and
// positions -> factors -> stores where few rows come (8 rows 5.2 us): what needs no factors is asked for in front of them.
template <typename T, int D, int STYLE>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a, int heads, int log2_lanes) {
  constexpr int VEC = Elem<T>::kVec, TPR = D / 2 / VEC, WAVES = kThreads / 64, PAIRS = D / 2, ROWS = 4096 / D, AHEAD = 2;
  typedef float2 turn_rows[ROWS][PAIRS];
  typedef float bound_rows[2][WAVES][64 / TPR][D];
  __shared__ __align__(16) char s_mem[sizeof(turn_rows) > sizeof(bound_rows) ? sizeof(turn_rows) : sizeof(bound_rows)];
  turn_rows& s_turn = *reinterpret_cast<turn_rows*>(s_mem);
  bound_rows& s_bound = *reinterpret_cast<bound_rows*>(s_mem);          // (after the last factors have been used)
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int parts = a.Hkv / heads;
  const int64_t unit = blockIdx.x / parts;
  const int g0 = (int)(blockIdx.x - unit * parts) * heads, G = a.H / a.Hkv;
  const Request rq = request_of(a, unit, lane);
  // (a thread forms the factors of one pair; its frequency, in turns per position, needs nothing from memory)
  const double turns = exp2(a.neg2_over_d_log2base * (double)(tid % PAIRS)) * 0.15915494309189533577;
  const int64_t page = a.c.page_size, len = rq.len;
  const int64_t p = (len >> a.log2_page) + unit - rq.unit0;
  const int64_t t0 = max(p * page, len), t1 = min((p + 1) * page, len + (rq.r1 - rq.r0));
  if (t0 >= t1) return;
  const int n = (int)(t1 - t0);
  const int64_t row0 = rq.r0 + (t0 - len);
  const int64_t phys = p >= 0 && p < a.c.max_pages ? a.c.table[(int64_t)rq.b * a.c.max_pages + p] : -1;
  const int slot0 = (int)(t0 - p * page);

  // columns of a thread's pairs in a head; tid = (row, head, place in the head)
  const int place = tid % TPR, i0 = place * VEC;
  const int e0 = STYLE == 0 ? i0 : 2 * i0, e1 = STYLE == 0 ? i0 + PAIRS : 2 * i0 + VEC;
  struct Pairs {
    u32x4 a, b;
  };
  auto read = [&](const T* src) {
    return Pairs{*reinterpret_cast<const u32x4*>(src + e0), *reinterpret_cast<const u32x4*>(src + e1)};
  };
  auto write = [&](T* dst, const Pairs& x) {
    *reinterpret_cast<u32x4*>(dst + e0) = x.a;
    *reinterpret_cast<u32x4*>(dst + e1) = x.b;
  };
  auto turn = [&](int j, Pairs& x) {
    if (!a.pos) return;
    float f[2 * VEC], o[2 * VEC];
    Vec16<T>::unpack(x.a, f);
    Vec16<T>::unpack(x.b, f + VEC);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const int ia = STYLE == 0 ? i : 2 * i, ib = STYLE == 0 ? i + VEC : 2 * i + 1;
      turn_pair(f[ia], f[ib], s_turn[j][i0 + i], o[ia], o[ib]);
    }
    x.a = rounded<T>(o);
    x.b = rounded<T>(o + VEC);
  };
  const int slots = kThreads >> log2_lanes, slot = tid >> log2_lanes;          // rows side by side; heads * TPR threads to a row
  const int head = (tid & ((1 << log2_lanes) - 1)) / TPR;
  const T* k = static_cast<const T*>(a.k) + row0 * a.k_stride + (g0 + head) * D;
  const T* v = static_cast<const T*>(a.v) + row0 * a.v_stride + (g0 + head) * D;
  const int q_vecs = heads * G * TPR;
  const T* q = static_cast<const T*>(a.q) + row0 * a.q_stride + g0 * G * D;
  T* q_out = static_cast<T*>(a.q_out) + (row0 * a.H + g0 * G) * D;
  // the next AHEAD rows of keys and values from row j on, and AHEAD vectors of queries from item `at` on, of rows before `end`
  Pairs kk[AHEAD], vv[AHEAD], qq[AHEAD];
  auto read_rows = [&](int j, int end) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int64_t r = min(j + i * slots, end - 1);
      kk[i] = read(k + r * a.k_stride);
      vv[i] = read(v + r * a.v_stride);
    }
  };
  auto query = [&](int at, int& j, int& h) { j = at / q_vecs; h = (at - j * q_vecs) / TPR; };     // (kThreads is a multiple of TPR: the place stays)
  auto read_queries = [&](int at, int items, int j0) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      int j, h;
      query(min(at + i * kThreads, items - TPR + place), j, h);
      qq[i] = read(q + (j0 + j) * a.q_stride + h * D);
    }
  };
  read_rows(slot, n);
  if (a.q) read_queries(tid, min(n, ROWS) * q_vecs, 0);

  const bool there = phys >= 0 && phys < a.c.n_pages;
  const int64_t dst = there ? phys * a.c.page_stride + slot0 * a.c.slot_stride + (g0 + head) * a.c.head_stride : 0;
  T* kc = static_cast<T*>(a.c.k) + dst;
  T* vc = static_cast<T*>(a.c.v) + dst;
  T* bounds = static_cast<T*>(a.c.bounds) + (phys * a.Hkv + g0) * 2 * D;
  const bool join = there && a.c.bounds && slot0 > 0;
  const float old = join && tid < heads * 2 * D ? Elem<T>::load(bounds + tid) : 0.f;       // (the others' follow where they are used)
  float lo[2 * VEC], hi[2 * VEC];
#pragma unroll
  for (int e = 0; e < 2 * VEC; ++e) { lo[e] = INFINITY; hi[e] = -INFINITY; }
  for (int j0 = 0; j0 < n; j0 += ROWS) {
    const int rows = min(n - j0, ROWS);
    if (a.pos) {
      if (j0 > 0) __syncthreads();
      for (int j = tid / PAIRS; j < rows; j += kThreads / PAIRS)
        s_turn[j][tid % PAIRS] = turn_at<T>((double)a.pos[row0 + j0 + j], turns);
      __syncthreads();
    }
    for (int j = slot; j < rows; j += AHEAD * slots) {
      if (j0 > 0 || j > slot) read_rows(j0 + j, n);
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int mine = j + i * slots;
        if (mine >= rows || !there) continue;
        turn(mine, kk[i]);
        write(kc + (int64_t)(j0 + mine) * a.c.slot_stride, kk[i]);
        write(vc + (int64_t)(j0 + mine) * a.c.slot_stride, vv[i]);
        float f[2 * VEC];
        Vec16<T>::unpack(kk[i].a, f);
        Vec16<T>::unpack(kk[i].b, f + VEC);
#pragma unroll
        for (int e = 0; e < 2 * VEC; ++e) { lo[e] = least(lo[e], f[e]); hi[e] = largest(hi[e], f[e]); }
      }
    }
    if (a.q) {
      const int items = rows * q_vecs;
      for (int at = tid; at < items; at += AHEAD * kThreads) {
        if (j0 > 0 || at > tid) read_queries(at, items, j0);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
          if (at + i * kThreads >= items) continue;
          int j, h;
          query(at + i * kThreads, j, h);
          turn(j, qq[i]);
          write(q_out + ((int64_t)(j0 + j) * a.H + h) * D, qq[i]);
        }
      }
    }
  }
  if (!there || !a.c.bounds) return;                      // (of the workgroup)
  for (int x = 1 << log2_lanes; x < 64 && x >> log2_lanes < n; x *= 2)     // (rows side by side in a wave, as many as there are)
#pragma unroll
    for (int e = 0; e < 2 * VEC; ++e) {
      lo[e] = least(lo[e], __shfl_xor(lo[e], x, 64));
      hi[e] = largest(hi[e], __shfl_xor(hi[e], x, 64));
    }
  __syncthreads();
  if (lane >> log2_lanes == 0) {
#pragma unroll
    for (int e = 0; e < 2 * VEC; ++e) {
      const int col = e < VEC ? e0 + e : e1 + e - VEC;
      s_bound[0][wave][head][col] = lo[e];
      s_bound[1][wave][head][col] = hi[e];
    }
  }
  __syncthreads();
  for (int item = tid; item < heads * 2 * D; item += kThreads) {
    const int h = item / (2 * D), col = item % D;
    const bool low = item % (2 * D) < D;
    const float(*b)[64 / TPR][D] = s_bound[low ? 0 : 1];
    float x = b[0][h][col];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) x = low ? least(x, b[w][h][col]) : largest(x, b[w][h][col]);
    if (join) {
      const float was = item == tid ? old : Elem<T>::load(bounds + item);
      x = low ? least(x, was) : largest(x, was);
    }
    Elem<T>::store(bounds + item, x);
  }
}

// Scores of pages (the definition is in qcf_pages.h), 16 pages to a wave, in float64 products of 4 pages x 4 queries x 4 elements,
// four of them side by side: score = sum of min(q, 0) lo + max(q, 0) hi.  Products of two stored bf16 values are exact in float64,
// and so are their sums where the terms are within 2^29 of each other: the order of the sum does not decide between pages.
// Bound by memory (512 bytes to a page and KV head of 128) and by its float64 work, a conversion and a product to each value: 32
// contexts of 1024 pages on average, 8 KV heads, 41.6 us with the queries in registers, two waves to a SIMD (30 of it without the
// products, with more chains of sums no change), 38.9 with the queries in LDS, four waves of up to four tiles, the next on its way,
// 35.7 with their table entries asked for at once, 31.4 (4.3 TB/s) with one tile at a time, six waves.  A lane has page lane % 16 and
// every fourth 16-byte vector of its bounds; of the result, query lane % 4 and page 4 (lane / 4 % 4) + lane / 16.
constexpr int kScorePages = 16, kScoreStep = kScorePages * kThreads / 64;           // pages of a wave, of a workgroup
template <typename T, int D>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 4 : 2) void page_score_kernel(
    qcf_page_cache c, const T* __restrict__ q, const int32_t* __restrict__ seen, int n_q, int H, int Hkv, int log2_page, int parts,
    float* __restrict__ score) {
  constexpr int VEC = Elem<T>::kVec, LOADS = D / (4 * VEC);
  typedef double pair_t __attribute__((ext_vector_type(2)));
  // min(q, 0) and max(q, 0) of two elements of four queries, in the order in which the lanes read them
  __shared__ pair_t s_q[2][D / 8][16];
  const int tid = threadIdx.x, lane = tid & 63, quad = lane >> 4, col = lane & 15, j = lane & 3;
  const int g = (int)(blockIdx.x % Hkv), G = H / Hkv;
  const int64_t rest = blockIdx.x / Hkv, row = rest / parts;            // (request, new row)
  const int64_t b = row / n_q;
  const int first = (int)(rest - row * parts) * kScoreStep, p0 = first + kScorePages * __builtin_amdgcn_readfirstlane(tid >> 6);
  const int step = parts * kScoreStep;                  // (at most max_pages and 64 more)
  const int32_t* table = c.table + b * c.max_pages;
  auto entry = [&](int p) { return p + col < c.max_pages ? table[p + col] : -1; };
  const int phys0 = entry(p0);                          // (asked for with the count)
  const int count = (int)min(((int64_t)max(seen[row], 0) + c.page_size - 1) >> log2_page, (int64_t)c.max_pages);
  if (first >= count) return;                           // (the workgroup)
  float* out = score + (row * Hkv + g) * c.max_pages;
  const T* bounds = static_cast<const T*>(c.bounds);
  auto load = [&](int phys, u32x4 (&l)[LOADS], u32x4 (&h)[LOADS]) {
    const T* src = bounds + ((int64_t)(phys >= 0 && phys < c.n_pages ? phys : 0) * Hkv + g) * 2 * D + quad * VEC;
#pragma unroll
    for (int f = 0; f < LOADS; ++f) {
      l[f] = *reinterpret_cast<const u32x4*>(src + 4 * f * VEC);
      h[f] = *reinterpret_cast<const u32x4*>(src + D + 4 * f * VEC);
    }
  };
  for (int h0 = 0; h0 < G; h0 += 4) {                   // four queries at a time
    u32x4 lo[LOADS], hi[LOADS];
    int phys = phys0;
    if (p0 < count) load(phys, lo, hi);
    if (h0 > 0) __syncthreads();
    for (int i = tid; i < 4 * D; i += kThreads) {
      const int h = i / D, e = i % D;                   // element e is in vector e / VEC: load vector / 4, quad vector % 4
      const float v = Elem<T>::load(q + (row * H + g * G + min(h0 + h, G - 1)) * D + e);
      const int at = (e / (4 * VEC) * VEC + e % VEC) / 2, lanes = e / VEC % 4 * 4 + h;
      s_q[0][at][lanes][e & 1] = v > 0.f ? 0.0 : (double)v;
      s_q[1][at][lanes][e & 1] = v < 0.f ? 0.0 : (double)v;
    }
    __syncthreads();
    for (int p = p0; p < count;) {
      const uint64_t mask = __ballot(phys >= 0 && phys < c.n_pages);
      const int next = p + step;
      if (next < count) phys = entry(next);
      double a0 = 0.0, a1 = 0.0;
      int query = 4 * quad + j;
      asm volatile("" : "+v"(query));                   // (read from LDS for every tile: kept, they would be spilled)
#pragma unroll
      for (int f = 0; f < LOADS; ++f) {
        float l[VEC], h[VEC];
        Vec16<T>::unpack(lo[f], l);
        Vec16<T>::unpack(hi[f], h);
#pragma unroll
        for (int e = 0; e < VEC; e += 2) {
          const pair_t down = s_q[0][(f * VEC + e) / 2][query], up = s_q[1][(f * VEC + e) / 2][query];
          a0 = __builtin_amdgcn_mfma_f64_4x4x4f64((double)l[e], down[0], a0, 0, 0, 0);
          a1 = __builtin_amdgcn_mfma_f64_4x4x4f64((double)h[e], up[0], a1, 0, 0, 0);
          a0 = __builtin_amdgcn_mfma_f64_4x4x4f64((double)l[e + 1], down[1], a0, 0, 0, 0);
          a1 = __builtin_amdgcn_mfma_f64_4x4x4f64((double)h[e + 1], up[1], a1, 0, 0, 0);
        }
      }
      if (next < count) load(phys, lo, hi);
      // (a sum that is not finite ranks first; what is beyond the floats stays above pages that are not there, and below those)
      const double sum = a0 + a1;
      float s = __builtin_isfinite(sum) ? __builtin_amdgcn_fmed3f((float)sum, -3.402823466e38f, 3.402823466e38f) : INFINITY;
      if (h0 + j >= G) s = -INFINITY;
      s = fmaxf(s, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(s), 0xb1, 0xf, 0xf, false)));    // the four queries
      s = fmaxf(s, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(s), 0x4e, 0xf, 0xf, false)));
      const int mine = 4 * (lane >> 2 & 3) + quad;
      if (j == 0 && p + mine < count) {
        s = mask >> mine & 1 ? s : -INFINITY;
        out[p + mine] = h0 > 0 ? fmaxf(out[p + mine], s) : s;           // (written by this lane)
      }
      p = next;
    }
  }
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
  a.neg2_over_d_log2base = -2.0 / L.head_dim * std::log2(L.rope_base);
  const int64_t units = pages::append_units(c, B, total_rows);
  const int heads = pages::append_heads(L, c, units);
  const int per_row = L.head_dim / 2 / (16 / elem_size(L.dtype));
  const int log2_lanes = __builtin_ctz((unsigned)(heads * per_row));
  const int64_t blocks = units * (L.n_kv_heads / heads);
  if (blocks > pages::kThreadsAtMost / kThreads) return fail(QCF_ERR_UNSUPPORTED, "page append: too many rows");
#define QCF_LAUNCH(T, D, S) append_kernel<T, D, S><<<dim3((unsigned)blocks), dim3(kThreads), 0, st>>>(a, heads, log2_lanes)
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
  // A workgroup to every 64 pages of a table's row, but not more than the GPU holds at a time (six to a compute unit with bf16 heads
  // of 128): these take turns.  Scores and choice, us, with four / six / eight / sixteen / any number to a compute unit: 32 contexts
  // of 512 to 1536 pages 39.3, 38.7, 38.9, 39.8, 42.0; 64 of 1024 to 2048 pages 43.5, 42.5, 42.7, 43.1, 44.8; 32 of 94 to 188 pages
  // in a table of 8192 15.1, 13.9, 17.4, 17.9, 24.8 (64 to a compute unit).
  const int64_t rows = (int64_t)B * n_q, steps = ((int64_t)c.max_pages + kScoreStep - 1) / kScoreStep;
  const int64_t most = 6 * (int64_t)compute_unit_count() / (rows * L.n_kv_heads);
  const int64_t parts = std::min(steps, std::max<int64_t>(most, 1)), blocks = rows * L.n_kv_heads * parts;
  if (blocks > pages::kThreadsAtMost / kThreads || rows * L.n_kv_heads > pages::kThreadsAtMost / pages::kTopThreads)
    return fail(QCF_ERR_UNSUPPORTED, "page select: too many rows");
  const int log2_page = __builtin_ctz((unsigned)c.page_size);
#define QCF_LAUNCH(T, D)                                                                                              \
  page_score_kernel<T, D><<<dim3((unsigned)blocks), dim3(kThreads), 0, st>>>(c, static_cast<const T*>(q), seen, n_q,  \
                                                                             L.n_q_heads, L.n_kv_heads, log2_page, (int)parts, score)
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

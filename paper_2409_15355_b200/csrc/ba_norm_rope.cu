// What lies between a layer's projections and its attention: norms of queries and keys for each head and the position rotation
// (Section 2.3, Eq. 1, at the tokens' prompt positions) in one pass, its gradients, and the same on the way into a paged cache.
//
//   y = R(p) (x r w),  r = 1 / sqrt(mean(x^2) + eps)         (no weights: y = R(p) x)
//   g = R(-p) dy,  h = g w,  dx = r h - x r^3 mean(h x),  dw = sum over rows and heads of g x r
//
// All of it is bound by HBM: a value is read once, kept in registers in fp32 and rounded once when it is written.  A head is held by
// head_dim / 8 lanes (16 bytes a lane), a warp has 256 / head_dim heads at a time (a step), several steps in flight; sums over a head
// are shuffles.  Queries, keys and values are sides of a call with CTAs of their own, as many as their steps are worth, so that a
// thread keeps one side's weights and sums.  One (cos, sin) pair of a row serves all of its heads: a warp that has a row folds its four
// pairs a lane into the weights and walks the heads; with few rows the heads of a row are shared out among warps instead.  The values
// of two rotary pairs are kept side by side, first members and second members, for arithmetic on two floats at a time.
//
// Kernels are launched early (ba_pdl_wait), so that tables, positions and sums may be written by the kernel before while one is alive already:
// they are read by plain loads, not through the read-only path, which wants data that nobody writes in a kernel's lifetime.
//
// Measured, heads of 128: 131072 rows of 32 + 8 heads 476 us (5.65 TB/s, 86 % of a copy), their gradients at 32768 rows 190 us (5.3 TB/s) and
// 5 us for the weights' sums; 64 passages of 1000 rows into pages 109 us (4.8 TB/s); one row each of 16 sequences 4 us.
#include <string.h>

#include <algorithm>
#include <type_traits>

#include "ba_common.cuh"
#include "ba_sm100.cuh"

using sm100::add2;
using sm100::fma2;
using sm100::pack2;
using sm100::unpack2;

namespace {

constexpr int kNormThreads = 256;
constexpr int kNormWarps = kNormThreads / 32;
// Steps in flight a warp, and CTAs an SM: more of the one leave registers for fewer of the other.  131072 rows, us: 4 x 3 476, 4 x 4 482, 3 x 4 508,
// 2 x 5 555, 8 x 2 629; gradients of 32768 rows: 4 x 2 190, 2 x 2 221, 1 x 4 227, 2 x 3 254, 3 x 3 315.
constexpr int kAhead = 4, kBwdAhead = 4;
constexpr int kFwdCtas = 3, kBwdCtas = kBaNormBwdCtas;

// One side of a call: rows of `heads` heads, `stride` elements apart.
struct NormSide {
  const __nv_bfloat16 *x;
  const __nv_bfloat16 *w;       // [D] or null: not normed
  void *y;                      // forward: packed rows, or the pool.  Gradients: dx
  const void *dy;               // gradients: packed rows
  float *dw;
  long long stride, y_stride;
  int heads;
  int cta0, n_ctas;             // its CTAs
  int rows_a_unit;              // a warp's rows, one behind the other; or
  int parts, steps_a_part;      // the steps of a row are shared out among `parts` warps
};
constexpr int kQ = 0, kK = 1, kV = 2;

struct NormParams {
  NormSide side[3];             // queries, keys, values (append only: copied); n_ctas 0: left out
  const int32_t *pos;           // null: position 0, no rotation
  int n_rows;
  float eps;
  // append: rows seq_cu[s] .. seq_cu[s + 1] - 1 go to places seq_start[s] .. of list s
  const int32_t *seq_cu, *seq_start, *page_cu, *page_idx;
  int n_seqs, page_lg, n_pages;
  int32_t *status;
  float *dw_part;               // gradients: [gridDim.x][D], every CTA's sums
  double turns[64];             // theta_m / (2 pi)
};

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t both(float x) { return pack2(x, x); }
__device__ __forceinline__ float sum_of(uint64_t v) {
  float a, b;
  unpack2(v, a, b);
  return a + b;
}

// The eight values of lane `l` of a head: four rotary pairs, 4 l .. 4 l + 3.  a: their first members, two and two; b: their second ones.  In
// the adjacent layout they are elements 8 l .. 8 l + 7, in the half layout 4 l .. and D / 2 + 4 l ..
struct Eight { uint64_t a[2], b[2]; };

template <int D, int kLayout>
__device__ __forceinline__ int second_four(int l) { return kLayout == BA_ROPE_ADJACENT ? 8 * l + 4 : D / 2 + 4 * l; }
template <int kLayout>
__device__ __forceinline__ int first_four(int l) { return kLayout == BA_ROPE_ADJACENT ? 8 * l : 4 * l; }

struct Raw16 { uint2 a, b; };
template <int D, int kLayout>
__device__ __forceinline__ Raw16 load_raw(const __nv_bfloat16 *head, int l) {
  Raw16 r;
  if (kLayout == BA_ROPE_ADJACENT) {
    const uint4 u = __ldcs(reinterpret_cast<const uint4 *>(head + 8 * l));
    r.a = make_uint2(u.x, u.y); r.b = make_uint2(u.z, u.w);
  } else {
    r.a = __ldcs(reinterpret_cast<const uint2 *>(head + 4 * l));
    r.b = __ldcs(reinterpret_cast<const uint2 *>(head + D / 2 + 4 * l));
  }
  return r;
}
template <int D, int kLayout>
__device__ __forceinline__ void store_raw(__nv_bfloat16 *head, int l, const Raw16 &r) {
  if (kLayout == BA_ROPE_ADJACENT) {
    *reinterpret_cast<uint4 *>(head + 8 * l) = make_uint4(r.a.x, r.a.y, r.b.x, r.b.y);
  } else {
    *reinterpret_cast<uint2 *>(head + 4 * l) = r.a;
    *reinterpret_cast<uint2 *>(head + D / 2 + 4 * l) = r.b;
  }
}
__device__ __forceinline__ float lo_f(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float hi_f(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}
template <int kLayout>
__device__ __forceinline__ Eight to_eight(const Raw16 &r) {
  Eight e;
  if (kLayout == BA_ROPE_ADJACENT) {
    e.a[0] = pack2(lo_f(r.a.x), lo_f(r.a.y)); e.b[0] = pack2(hi_f(r.a.x), hi_f(r.a.y));
    e.a[1] = pack2(lo_f(r.b.x), lo_f(r.b.y)); e.b[1] = pack2(hi_f(r.b.x), hi_f(r.b.y));
  } else {
    e.a[0] = pack2(lo_f(r.a.x), hi_f(r.a.x)); e.a[1] = pack2(lo_f(r.a.y), hi_f(r.a.y));
    e.b[0] = pack2(lo_f(r.b.x), hi_f(r.b.x)); e.b[1] = pack2(lo_f(r.b.y), hi_f(r.b.y));
  }
  return e;
}
// in memory order: the first four elements, then the other four
template <int kLayout>
__device__ __forceinline__ void in_order(const Eight &e, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float a0, a1, b0, b1;
    unpack2(e.a[i], a0, a1);
    unpack2(e.b[i], b0, b1);
    if (kLayout == BA_ROPE_ADJACENT) { f[4 * i] = a0; f[4 * i + 1] = b0; f[4 * i + 2] = a1; f[4 * i + 3] = b1; }
    else { f[2 * i] = a0; f[2 * i + 1] = a1; f[4 + 2 * i] = b0; f[4 + 2 * i + 1] = b1; }
  }
}
struct Raw32 { float4 a, b; };
template <int D, int kLayout>
__device__ __forceinline__ Raw32 load_raw(const float *head, int l) {
  return {__ldcs(reinterpret_cast<const float4 *>(head + first_four<kLayout>(l))), __ldcs(reinterpret_cast<const float4 *>(head + second_four<D, kLayout>(l)))};
}
template <int kLayout>
__device__ __forceinline__ Eight to_eight(const Raw32 &r) {
  Eight e;
  if (kLayout == BA_ROPE_ADJACENT) {
    e.a[0] = pack2(r.a.x, r.a.z); e.b[0] = pack2(r.a.y, r.a.w);
    e.a[1] = pack2(r.b.x, r.b.z); e.b[1] = pack2(r.b.y, r.b.w);
  } else {
    e.a[0] = pack2(r.a.x, r.a.y); e.a[1] = pack2(r.a.z, r.a.w);
    e.b[0] = pack2(r.b.x, r.b.y); e.b[1] = pack2(r.b.z, r.b.w);
  }
  return e;
}
template <typename T> struct RawOf { using Type = Raw16; };
template <> struct RawOf<float> { using Type = Raw32; };
template <int D, int kLayout>
__device__ __forceinline__ void store_eight(__nv_bfloat16 *head, int l, const Eight &e) {
  float f[8];
  in_order<kLayout>(e, f);
  Raw16 r;
  r.a = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
  r.b = make_uint2(pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
  store_raw<D, kLayout>(head, l, r);
}
template <int D, int kLayout>
__device__ __forceinline__ void store_eight(float *head, int l, const Eight &e) {
  float f[8];
  in_order<kLayout>(e, f);
  *reinterpret_cast<float4 *>(head + first_four<kLayout>(l)) = make_float4(f[0], f[1], f[2], f[3]);
  *reinterpret_cast<float4 *>(head + second_four<D, kLayout>(l)) = make_float4(f[4], f[5], f[6], f[7]);
}
template <int D, int kLayout>
__device__ __forceinline__ Eight load_weights(const __nv_bfloat16 *w, int l) {
  if (w) return to_eight<kLayout>(load_raw<D, kLayout>(w, l));
  return {{both(1.f), both(1.f)}, {both(1.f), both(1.f)}};
}

// (cos, sin) of the four pairs of lane `l` of a head at position `p`.  The angle is reduced in turns in fp64 -- p theta / 2 pi reaches
// thousands of turns, of which fp32 keeps no fraction worth having -- and its fraction fits fp32 to 2e-7 radians.
__device__ __forceinline__ void row_angles(const double *turns, int p, int l, uint64_t (&c)[2], uint64_t (&s)[2]) {
  float cc[4], ss[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    double t = (double)p * turns[4 * l + j];
    t -= rint(t);
    sincospif(2.f * (float)t, &ss[j], &cc[j]);
  }
  c[0] = pack2(cc[0], cc[1]); c[1] = pack2(cc[2], cc[3]);
  s[0] = pack2(ss[0], ss[1]); s[1] = pack2(ss[2], ss[3]);
}
__device__ __forceinline__ uint64_t negative(uint64_t v) { return v ^ 0x8000000080000000ull; }

__device__ __forceinline__ float squares(const Eight &x) {
  return sum_of(fma2(x.b[1], x.b[1], fma2(x.b[0], x.b[0], fma2(x.a[1], x.a[1], mul2(x.a[0], x.a[0])))));
}
__device__ __forceinline__ float products(const Eight &x, const Eight &y) {
  return sum_of(fma2(x.b[1], y.b[1], fma2(x.b[0], y.b[0], fma2(x.a[1], y.a[1], mul2(x.a[0], y.a[0])))));
}
// Sum over the lanes of a head.
template <int D>
__device__ __forceinline__ float head_sum(float x) {
#pragma unroll
  for (int o = D / 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// Places of rows in their sequences' page lists -> pool rows, for a warp that walks rows one behind the other: tables are looked up where a
// sequence or a page begins (64 passages of 1000 tokens, looked up for every row: 123 us, so 109).
struct AppendWalk {
  int s = -1, first = 0, end = 0;        // sequence, its rows
  int list = 0, n_list = 0;              // its pages
  long long start = 0, page_at = -1;     // place of its first row; page of the list that the last row lay on
  long long page_row = -1;               // pool row of that page; negative: there is none
  // -1: nowhere (recorded), -2: a row behind the last sequence or between them (padding)
  __device__ __forceinline__ long long pool_row(const NormParams &p, int row, bool query) {
    if (row >= end || s < 0) {
      page_at = -1;
      if (p.seq_cu) {
        int lo = 0, hi = p.n_seqs + 1;                     // first index whose start lies behind the row
        while (lo < hi) { const int mid = (lo + hi) >> 1; if (p.seq_cu[mid] <= row) lo = mid + 1; else hi = mid; }
        s = lo - 1;
        if (s < 0 || s >= p.n_seqs) { s = -1; return -2; }
        first = p.seq_cu[s]; end = p.seq_cu[s + 1];
      } else {
        s = first = row; end = row + 1;
      }
      if (!query) {
        start = p.seq_start[s];
        list = p.page_cu[s];
        n_list = list >= 0 ? p.page_cu[s + 1] - list : 0;    // (a list that begins before the table has no pages)
      }
    }
    if (query) return row;
    const long long place = start + (row - first), nth = place >> p.page_lg;
    if (nth != page_at || page_at < 0) {
      page_at = nth;
      const int page = nth >= 0 && nth < n_list ? p.page_idx[list + nth] : -1;
      page_row = page >= 0 && page < p.n_pages ? (long long)page << p.page_lg : -1;
    }
    if (page_row < 0) {
      if ((threadIdx.x & 31) == 0) ba_record_status(p.status, BA_ERR_INVALID_ARG);
      return -1;
    }
    return page_row + (place & ((1 << p.page_lg) - 1));
  }
};

__device__ __forceinline__ int my_side(const NormParams &p) {
  const int b = (int)blockIdx.x;
  return b < p.side[kK].cta0 ? kQ : b < p.side[kV].cta0 ? kK : kV;
}
// Rows and steps of unit u.
struct NormUnit { int row, row_end, step, step_end; };
__device__ __forceinline__ int units_of(const NormSide &side, int n_rows) { return side.parts > 1 ? n_rows * side.parts : (n_rows + side.rows_a_unit - 1) / side.rows_a_unit; }
__device__ __forceinline__ NormUnit unit_at(const NormSide &side, int n_rows, int steps, int u) {
  NormUnit x;
  if (side.parts > 1) {
    x.row = u / side.parts; x.row_end = x.row + 1;
    x.step = (u - x.row * side.parts) * side.steps_a_part; x.step_end = min(steps, x.step + side.steps_a_part);
  } else {
    x.row = u * side.rows_a_unit; x.row_end = min(n_rows, x.row + side.rows_a_unit);
    x.step = 0; x.step_end = steps;
  }
  return x;
}

// kAppend: keys and values go through the page table.
template <int D, int kLayout, bool kAppend>
__global__ void __launch_bounds__(kNormThreads, kFwdCtas)
ba_norm_rope_kernel(const __grid_constant__ NormParams p) {
  constexpr int kLanes = D / 8, kHeads = 32 / kLanes;
  __shared__ double turns[D / 2];
  const int lane = threadIdx.x & 31, l = lane % kLanes, sub = lane / kLanes;
  if (threadIdx.x < D / 2) turns[threadIdx.x] = p.turns[threadIdx.x];
  const int which = my_side(p);
  const NormSide &side = p.side[which];
  const int steps = (side.heads + kHeads - 1) / kHeads;
  ba_pdl_wait();
  ba_pdl_trigger();
  __syncthreads();
  const bool normed = side.w != nullptr;
  const Raw16 raw_w = normed ? load_raw<D, kLayout>(side.w, l) : Raw16{make_uint2(0x3f803f80u, 0x3f803f80u), make_uint2(0x3f803f80u, 0x3f803f80u)};    // (ones)
  const int units = units_of(side, p.n_rows), stride = side.n_ctas * kNormWarps;
  for (int u = ((int)blockIdx.x - side.cta0) * kNormWarps + (threadIdx.x >> 5); u < units; u += stride) {
    const NormUnit un = unit_at(side, p.n_rows, steps, u);
    const int begin = un.step, end = un.step_end;
    AppendWalk walk;
    for (int row = un.row; row < un.row_end; ++row) {
      const __nv_bfloat16 *src = side.x + row * side.stride + sub * D;
      long long to = row;
      const int pos = p.pos ? p.pos[row] : 0;
      Eight wc, ws;                        // weights x cos, weights x sin
      for (int i0 = begin; i0 < end; i0 += kAhead) {
        Raw16 raw[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
          raw[a] = {make_uint2(0, 0), make_uint2(0, 0)};
          if (i0 + a < end && (i0 + a) * kHeads + sub < side.heads) raw[a] = load_raw<D, kLayout>(src + (i0 + a) * kHeads * D, l);
        }
        if (i0 == begin) {                 // (while the loads are on their way)
          if (kAppend) to = walk.pool_row(p, row, which == kQ);
          if (which != kV) {
            const Eight w = to_eight<kLayout>(raw_w);
            uint64_t c[2], s[2];
            row_angles(turns, pos, l, c, s);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              wc.a[i] = mul2(w.a[i], c[i]); wc.b[i] = mul2(w.b[i], c[i]);
              ws.a[i] = mul2(w.a[i], s[i]); ws.b[i] = negative(mul2(w.b[i], s[i]));
            }
          }
        }
        if (to < 0) break;
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
          const int i = i0 + a;
          if (i >= end) break;                               // (the whole warp)
          if (!kAppend || which != kV) {
            const Eight x = to_eight<kLayout>(raw[a]);
            const float r = normed ? rsqrtf(head_sum<D>(squares(x)) * (1.f / D) + p.eps) : 1.f;
            Eight y;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              y.a[k] = mul2(both(r), fma2(x.b[k], ws.b[k], mul2(x.a[k], wc.a[k])));
              y.b[k] = mul2(both(r), fma2(x.b[k], wc.b[k], mul2(x.a[k], ws.a[k])));
            }
            float f[8];
            in_order<kLayout>(y, f);
            raw[a].a = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
            raw[a].b = make_uint2(pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
          }
          const int h = i * kHeads + sub;
          if (h < side.heads) store_raw<D, kLayout>(reinterpret_cast<__nv_bfloat16 *>(side.y) + (to * side.heads + h) * D, l, raw[a]);
        }
      }
    }
  }
}

// Gradients.  Units are shared out among warps once and for all, each lane sums the weights' gradients of its columns in fp32, the
// CTA adds its warps in order and a second kernel the CTAs: no atomics, the same bits every run.
template <int D, int kLayout, typename T>
__global__ void __launch_bounds__(kNormThreads, kBwdCtas)
ba_norm_rope_bwd_kernel(const __grid_constant__ NormParams p) {
  constexpr int kLanes = D / 8, kHeads = 32 / kLanes;
  __shared__ double turns[D / 2];
  __shared__ float sums[kNormWarps][D];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane % kLanes, sub = lane / kLanes;
  if (threadIdx.x < D / 2) turns[threadIdx.x] = p.turns[threadIdx.x];
  const NormSide &side = p.side[my_side(p)];
  const int steps = (side.heads + kHeads - 1) / kHeads;
  ba_pdl_wait();
  ba_pdl_trigger();
  __syncthreads();
  const bool normed = side.w != nullptr;
  const Eight w = load_weights<D, kLayout>(side.w, l);
  Eight dw = {{0ull, 0ull}, {0ull, 0ull}};
  const int units = units_of(side, p.n_rows), stride = side.n_ctas * kNormWarps;
  for (int u = ((int)blockIdx.x - side.cta0) * kNormWarps + warp; u < units; u += stride) {
    const NormUnit un = unit_at(side, p.n_rows, steps, u);
    const int begin = un.step, end = un.step_end;
    for (int row = un.row; row < un.row_end; ++row) {
      const int pos = p.pos ? p.pos[row] : 0;
      const __nv_bfloat16 *src = side.x + row * side.stride + sub * D;
      const T *dy = reinterpret_cast<const T *>(side.dy) + ((long long)row * side.heads + sub) * D;
      T *dx = reinterpret_cast<T *>(side.y) + row * side.y_stride + sub * D;
      uint64_t c[2], s[2];
      for (int i0 = begin; i0 < end; i0 += kBwdAhead) {
        Raw16 rx[kBwdAhead];
        typename RawOf<T>::Type rd[kBwdAhead];
#pragma unroll
        for (int a = 0; a < kBwdAhead; ++a) {
          rx[a] = {};
          rd[a] = {};
          if (i0 + a < end && (i0 + a) * kHeads + sub < side.heads) {
            if (normed) rx[a] = load_raw<D, kLayout>(src + (i0 + a) * kHeads * D, l);
            rd[a] = load_raw<D, kLayout>(dy + (i0 + a) * kHeads * D, l);
          }
        }
        if (i0 == begin) row_angles(turns, pos, l, c, s);    // (while the loads are on their way)
#pragma unroll
        for (int a = 0; a < kBwdAhead; ++a) {
          const int i = i0 + a;
          if (i >= end) break;                               // (the whole warp)
          const bool there = i * kHeads + sub < side.heads;
          const Eight d = to_eight<kLayout>(rd[a]);
          Eight g;
#pragma unroll
          for (int k = 0; k < 2; ++k) {                      // R(-p)
            g.a[k] = fma2(d.b[k], s[k], mul2(d.a[k], c[k]));
            g.b[k] = fma2(d.a[k], negative(s[k]), mul2(d.b[k], c[k]));
          }
          if (normed) {
            const Eight x = to_eight<kLayout>(rx[a]);
            Eight h;
#pragma unroll
            for (int k = 0; k < 2; ++k) { h.a[k] = mul2(g.a[k], w.a[k]); h.b[k] = mul2(g.b[k], w.b[k]); }
            const float ss = head_sum<D>(squares(x)), hx = head_sum<D>(products(h, x));
            const float r = there ? rsqrtf(ss * (1.f / D) + p.eps) : 0.f;        // (no head there: 0 r is NaN for eps 0)
            const uint64_t r2 = both(r), t2 = both(-hx * (1.f / D) * r * r);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              dw.a[k] = fma2(mul2(g.a[k], x.a[k]), r2, dw.a[k]);
              dw.b[k] = fma2(mul2(g.b[k], x.b[k]), r2, dw.b[k]);
              g.a[k] = mul2(r2, fma2(x.a[k], t2, h.a[k]));
              g.b[k] = mul2(r2, fma2(x.b[k], t2, h.b[k]));
            }
          }
          if (there) store_eight<D, kLayout>(dx + (long long)i * kHeads * D, l, g);
        }
      }
    }
  }
  if (!p.dw_part) return;
  // a warp's heads, then the CTA's warps, in order
  float f[8];
  in_order<kLayout>(dw, f);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
#pragma unroll
    for (int o = kLanes; o < 32; o <<= 1) f[e] += __shfl_xor_sync(0xffffffffu, f[e], o);
    if (sub == 0) sums[warp][(e < 4 ? first_four<kLayout>(l) : second_four<D, kLayout>(l)) + (e & 3)] = f[e];
  }
  __syncthreads();
  if (threadIdx.x < D) {
    float t = 0.f;
    for (int k = 0; k < kNormWarps; ++k) t += sums[k][threadIdx.x];
    p.dw_part[(size_t)blockIdx.x * D + threadIdx.x] = t;
  }
}

// dw = the CTAs' sums, added in a fixed order: 32 columns of a side a CTA, 32 runs of CTAs side by side.
template <int D>
__global__ void __launch_bounds__(1024)
ba_norm_dw_kernel(const float *part, int n_q, int n_k, float *dw_q, float *dw_k) {
  __shared__ float sums[32][33];
  ba_pdl_wait();
  ba_pdl_trigger();
  const int side = blockIdx.x / (D / 32), col = blockIdx.x % (D / 32) * 32 + (threadIdx.x & 31), run = threadIdx.x >> 5;
  const int first = side ? n_q : 0, n = side ? n_k : n_q;
  float *dw = side ? dw_k : dw_q;
  if (!dw) return;
  float t = 0.f;
#pragma unroll 4
  for (int b = run; b < n; b += 32) t += part[(size_t)(first + b) * D + col];
  sums[run][threadIdx.x & 31] = t;
  __syncthreads();
  t = sums[threadIdx.x & 31][run];                         // (column `run` of the 32, a run of CTAs a lane)
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  if ((threadIdx.x & 31) == 0) dw[col - (threadIdx.x & 31) + run] = t;
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// One side's tensor: present, aligned, rows apart far enough for whole 16-byte vectors.  `stride` 0: packed rows.
bool side_ok(const void *x, int64_t *stride, int row, int elements_16_bytes) {
  if (*stride == 0) *stride = row;
  return x && aligned16(x) && *stride >= row && *stride % elements_16_bytes == 0;
}
bool eps_ok(float eps, const void *w_q, const void *w_k) { return (!w_q && !w_k) || (eps >= 0.f && eps <= 1e30f); }

// Lays out the CTAs of a call: `room` of them at a time, shared out by the sides' steps.  A warp with a whole row computes its angles
// once (131072 rows); few rows are cut up until every SM has eight warps (50 rows of 16 steps: one warp each would walk them alone).
int lay_out(const ba_ctx *ctx, NormParams &p, int ctas_a_sm, const bool (&there)[3]) {
  const int heads_a_step = 256 / ctx->cfg.head_dim;
  int steps[3], all = 0, cta = 0;
  for (int i = 0; i < 3; ++i) all += steps[i] = there[i] ? (p.side[i].heads + heads_a_step - 1) / heads_a_step : 0;
  const long long room = (long long)ctx->sm_count * ctas_a_sm;
  for (int i = 0; i < 3; ++i) {
    NormSide &s = p.side[i];
    s.cta0 = cta; s.n_ctas = 0;
    if (!there[i]) continue;
    long long parts = ((long long)ctx->sm_count * 8 + p.n_rows - 1) / p.n_rows;
    if (parts > steps[i]) parts = steps[i];
    s.steps_a_part = (int)((steps[i] + parts - 1) / parts);
    s.parts = (steps[i] + s.steps_a_part - 1) / s.steps_a_part;
    long long most = room * steps[i] / all * kNormWarps;   // warps
    if (most < kNormWarps) most = kNormWarps;
    s.rows_a_unit = (int)((p.n_rows + most - 1) / most);
    const long long units = s.parts > 1 ? (long long)p.n_rows * s.parts : (p.n_rows + s.rows_a_unit - 1) / s.rows_a_unit;
    s.n_ctas = (int)((std::min(units, most) + kNormWarps - 1) / kNormWarps);
    cta += s.n_ctas;
  }
  return cta;
}

template <bool kAppend>
ba_status launch_norm_rope(ba_ctx *ctx, NormParams &p, const bool (&there)[3], cudaStream_t stream) {
  if (there[kK]) {                                         // keys that a queued re-encoding is to write
    const size_t row = (size_t)p.side[kK].heads * ctx->cfg.head_dim;
    const ba_status st = ba_flush_pending_into(ctx, p.side[kK].x, ((size_t)(p.n_rows - 1) * p.side[kK].stride + row) * 2, stream);
    if (st != BA_OK) return st;
  }
  p.status = ctx->dev_status;
  memcpy(p.turns, ctx->turns, sizeof(p.turns));
  const int grid = lay_out(ctx, p, kFwdCtas, there);
  auto launch = [&](auto kern) { return ba_launch(kern, dim3((unsigned)grid), kNormThreads, 0, stream, true, p); };
  const bool half = ctx->cfg.rope_layout == BA_ROPE_HALF;
  if (ctx->cfg.head_dim == 128) BA_CUDA_TRY(half ? launch(ba_norm_rope_kernel<128, BA_ROPE_HALF, kAppend>) : launch(ba_norm_rope_kernel<128, BA_ROPE_ADJACENT, kAppend>));
  else BA_CUDA_TRY(half ? launch(ba_norm_rope_kernel<64, BA_ROPE_HALF, kAppend>) : launch(ba_norm_rope_kernel<64, BA_ROPE_ADJACENT, kAppend>));
  ctx->launches += 1;
  return BA_OK;
}

}  // namespace

extern "C" {

ba_status ba_qk_norm_rope(ba_ctx *ctx, const void *q, int64_t q_stride, const void *k, int64_t k_stride, int32_t n_rows,
                          const int32_t *pos, const void *w_q, const void *w_k, float eps, void *q_out, void *k_out, void *stream) {
  if (!ctx || n_rows < 0 || (!q && !k) || !q != !q_out || !k != !k_out) return BA_ERR_INVALID_ARG;
  const int D = ctx->cfg.head_dim, q_row = ctx->cfg.n_q_heads * D, k_row = ctx->cfg.n_kv_heads * D;
  if ((q && !side_ok(q, &q_stride, q_row, 8)) || (k && !side_ok(k, &k_stride, k_row, 8))) return BA_ERR_INVALID_ARG;
  if (!aligned16(q_out) || !aligned16(k_out) || !aligned16(w_q) || !aligned16(w_k) || !eps_ok(eps, w_q, w_k)) return BA_ERR_INVALID_ARG;
  if ((q && q == q_out && q_stride != q_row) || (k && k == k_out && k_stride != k_row)) return BA_ERR_INVALID_ARG;
  if (q && k && (q_out == k_out || q_out == k || k_out == q)) return BA_ERR_INVALID_ARG;       // (the sides run side by side)
  if (n_rows == 0) return BA_OK;
  BA_CUDA_TRY(cudaSetDevice(ctx->device));
  NormParams p = {};
  p.side[kQ] = {(const __nv_bfloat16 *)q, (const __nv_bfloat16 *)w_q, q_out, nullptr, nullptr, q_stride, q_row, ctx->cfg.n_q_heads};
  p.side[kK] = {(const __nv_bfloat16 *)k, (const __nv_bfloat16 *)w_k, k_out, nullptr, nullptr, k_stride, k_row, ctx->cfg.n_kv_heads};
  p.pos = pos; p.n_rows = n_rows; p.eps = eps;
  return launch_norm_rope<false>(ctx, p, {q != nullptr, k != nullptr, false}, (cudaStream_t)stream);
}

ba_status ba_append_paged(ba_ctx *ctx, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                          int32_t n_rows, const int32_t *pos, const void *w_q, const void *w_k, float eps, const int32_t *seq_cu,
                          const int32_t *seq_start, int32_t n_seqs, void *q_out, void *k_pool, void *v_pool, const ba_page_table *pages,
                          void *stream) {
  ba_status st = ba_check_pages(pages);
  if (st != BA_OK) return st;
  if (!ctx || n_rows < 0 || n_seqs < 0 || !k || !v || !k_pool || !v_pool || !seq_start || !q != !q_out) return BA_ERR_INVALID_ARG;
  const int D = ctx->cfg.head_dim, q_row = ctx->cfg.n_q_heads * D, k_row = ctx->cfg.n_kv_heads * D;
  if ((q && !side_ok(q, &q_stride, q_row, 8)) || !side_ok(k, &k_stride, k_row, 8) || !side_ok(v, &v_stride, k_row, 8)) return BA_ERR_INVALID_ARG;
  if (!aligned16(q_out) || !aligned16(k_pool) || !aligned16(v_pool) || !aligned16(w_q) || !aligned16(w_k) || !eps_ok(eps, w_q, w_k))
    return BA_ERR_INVALID_ARG;
  if (k == k_pool || v == v_pool || k_pool == v_pool || (q && q == q_out && q_stride != q_row)) return BA_ERR_INVALID_ARG;
  if (q && (q_out == k_pool || q_out == v_pool || q_out == k || q_out == v)) return BA_ERR_INVALID_ARG;
  if (!seq_cu && n_seqs != n_rows) return BA_ERR_SHAPE;
  if (n_rows == 0 || n_seqs == 0) return BA_OK;
  BA_CUDA_TRY(cudaSetDevice(ctx->device));
  NormParams p = {};
  p.side[kQ] = {(const __nv_bfloat16 *)q, (const __nv_bfloat16 *)w_q, q_out, nullptr, nullptr, q_stride, q_row, ctx->cfg.n_q_heads};
  p.side[kK] = {(const __nv_bfloat16 *)k, (const __nv_bfloat16 *)w_k, k_pool, nullptr, nullptr, k_stride, k_row, ctx->cfg.n_kv_heads};
  p.side[kV] = {(const __nv_bfloat16 *)v, nullptr, v_pool, nullptr, nullptr, v_stride, k_row, ctx->cfg.n_kv_heads};
  p.pos = pos; p.n_rows = n_rows; p.eps = eps;
  p.seq_cu = seq_cu; p.seq_start = seq_start; p.n_seqs = n_seqs;
  p.page_cu = pages->page_cu; p.page_idx = pages->page_idx; p.n_pages = pages->n_pages;
  while ((1 << p.page_lg) < pages->page_rows) ++p.page_lg;
  return launch_norm_rope<true>(ctx, p, {q != nullptr, true, true}, (cudaStream_t)stream);
}

ba_status ba_qk_norm_rope_bwd(ba_ctx *ctx, const void *q, int64_t q_stride, const void *k, int64_t k_stride, int32_t n_rows,
                              const int32_t *pos, const void *w_q, const void *w_k, float eps, const void *dy_q, const void *dy_k,
                              void *dq, int64_t dq_stride, void *dk, int64_t dk_stride, float *dw_q, float *dw_k,
                              ba_out_dtype grad_dtype, void *stream) {
  if (!ctx || n_rows < 0 || (!dq && !dk) || !dy_q != !dq || !dy_k != !dk) return BA_ERR_INVALID_ARG;
  if (grad_dtype != BA_OUT_BF16 && grad_dtype != BA_OUT_F32) return BA_ERR_INVALID_ARG;
  const int D = ctx->cfg.head_dim, q_row = ctx->cfg.n_q_heads * D, k_row = ctx->cfg.n_kv_heads * D, vec = grad_dtype == BA_OUT_F32 ? 4 : 8;
  // (the input itself counts only under a norm)
  if ((w_q && !dq) || (w_k && !dk) || (w_q && !side_ok(q, &q_stride, q_row, 8)) || (w_k && !side_ok(k, &k_stride, k_row, 8)))
    return BA_ERR_INVALID_ARG;
  if ((dq && !side_ok(dq, &dq_stride, q_row, vec)) || (dk && !side_ok(dk, &dk_stride, k_row, vec))) return BA_ERR_INVALID_ARG;
  if (!aligned16(dy_q) || !aligned16(dy_k) || !aligned16(w_q) || !aligned16(w_k) || !eps_ok(eps, w_q, w_k)) return BA_ERR_INVALID_ARG;
  if (!w_q != !dw_q || !w_k != !dw_k) return BA_ERR_INVALID_ARG;
  if ((dq && dq == dy_q && dq_stride != q_row) || (dk && dk == dy_k && dk_stride != k_row)) return BA_ERR_INVALID_ARG;
  // the place of the inputs, too, if they lie row on row and value on value
  const bool wide = grad_dtype == BA_OUT_F32;
  if ((w_q && dq == q && (wide || dq_stride != q_stride)) || (w_k && dk == k && (wide || dk_stride != k_stride))) return BA_ERR_INVALID_ARG;
  if (dq && dk && (dq == dk || dq == dy_k || dk == dy_q || (w_q && dk == q) || (w_k && dq == k))) return BA_ERR_INVALID_ARG;
  const bool sums = w_q || w_k;
  if (n_rows == 0 && !sums) return BA_OK;
  const size_t need = sums ? ba_norm_sums_bytes(ctx->sm_count, D) : 0;
  if (sums && (!ctx->workspace || ba_scratch_offset(ctx) + need + ctx->pending_table_bytes > ctx->workspace_bytes)) return BA_ERR_WORKSPACE;
  if (dw_q && dw_q == dw_k) return BA_ERR_INVALID_ARG;
  BA_CUDA_TRY(cudaSetDevice(ctx->device));
  const cudaStream_t cs = (cudaStream_t)stream;
  NormParams p = {};
  p.side[kQ] = {(const __nv_bfloat16 *)q, (const __nv_bfloat16 *)w_q, dq, dy_q, dw_q, q_stride, dq_stride, ctx->cfg.n_q_heads};
  p.side[kK] = {(const __nv_bfloat16 *)k, (const __nv_bfloat16 *)w_k, dk, dy_k, dw_k, k_stride, dk_stride, ctx->cfg.n_kv_heads};
  p.pos = pos; p.n_rows = n_rows; p.eps = eps;
  p.dw_part = sums ? (float *)((char *)ctx->workspace + ba_scratch_offset(ctx)) : nullptr;
  memcpy(p.turns, ctx->turns, sizeof(p.turns));
  if (n_rows > 0) {
    const int grid = lay_out(ctx, p, kBwdCtas, {dq != nullptr, dk != nullptr, false});
    auto launch = [&](auto kern) { return ba_launch(kern, dim3((unsigned)grid), kNormThreads, 0, cs, true, p); };
    auto pick = [&](auto layout, auto value) {
      constexpr int kL = decltype(layout)::value;
      using T = decltype(value);
      return D == 128 ? launch(ba_norm_rope_bwd_kernel<128, kL, T>) : launch(ba_norm_rope_bwd_kernel<64, kL, T>);
    };
    auto by_type = [&](auto layout) { return grad_dtype == BA_OUT_F32 ? pick(layout, float{}) : pick(layout, __nv_bfloat16{}); };
    BA_CUDA_TRY(ctx->cfg.rope_layout == BA_ROPE_HALF ? by_type(std::integral_constant<int, BA_ROPE_HALF>{})
                                                    : by_type(std::integral_constant<int, BA_ROPE_ADJACENT>{}));
    ctx->launches += 1;
  }
  if (sums) {
    auto kern = D == 128 ? ba_norm_dw_kernel<128> : ba_norm_dw_kernel<64>;
    BA_CUDA_TRY(ba_launch(kern, dim3((unsigned)(2 * D / 32)), 1024, 0, cs, true, p.dw_part, p.side[kQ].n_ctas, p.side[kK].n_ctas, dw_q, dw_k));
    ctx->launches += 1;
  }
  return BA_OK;
}

}  // extern "C"

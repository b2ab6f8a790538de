// What lies between a layer's projections and its attention: norms of queries and keys for each head and the position rotation
// (Section 2.3, Eq. 1, at the tokens' prompt positions) in one pass, its gradients, and the same on the way into a paged cache.
//
//   y = R(p) (x r w),  r = 1 / sqrt(mean(x^2) + eps)         (no weights: y = R(p) x)
//   g = R(-p) dy,  h = g w,  dx = r h - x r^3 mean(h x),  dw = sum over rows and heads of g x r
//
// All of it is bound by HBM: a value is read once, kept in registers in fp32 and rounded once when it is written.  A head is held by
// head_dim / 8 lanes (16 bytes a lane), a warp has 256 / head_dim heads at a time, kAhead of these steps in flight; sums over a head
// are shuffles.  One (cos, sin) pair of a row serves all of its heads, so the warp that has a row keeps its four pairs a lane in
// registers and walks the heads; with few rows the heads of a row are shared out among warps instead.
#include "ba_common.cuh"

namespace {

constexpr int kNormThreads = 256;
constexpr int kNormWarps = kNormThreads / 32;
constexpr int kAhead = 4;                 // loads in flight a lane
constexpr int kNormGridMax = kBaNormGridMax;

// A side's heads in a row-strided tensor: bf16 [n_rows, heads, D], rows `stride` elements apart.
struct NormSide {
  const __nv_bfloat16 *x;
  const __nv_bfloat16 *w;       // [D] or null: not normed
  long long stride;
  int heads;
};

struct NormParams {
  NormSide q, k, v;             // x null: side absent.  v (append only) is copied
  __nv_bfloat16 *q_out, *k_out; // packed rows
  const int32_t *pos;           // null: position 0, no rotation
  int n_rows;
  float eps;
  int parts, steps_a_part;      // a row's steps (256 / D heads each) are shared out among `parts` warps
  // append: rows seq_cu[s] .. seq_cu[s + 1] - 1 go to places seq_start[s] .. of list s
  const int32_t *seq_cu, *seq_start, *page_cu, *page_idx;
  __nv_bfloat16 *k_pool, *v_pool;
  int n_seqs, page_lg, n_pages;
  int32_t *status;
  double turns[64];             // theta_m / (2 pi)
};

struct NormBwdParams {
  NormSide q, k;
  const void *dy_q, *dy_k;      // packed rows
  void *dq, *dk;
  long long dq_stride, dk_stride;
  const int32_t *pos;
  int n_rows;
  float eps;
  int parts, steps_a_part;
  float *dw_part;               // [gridDim.x][2][D]: every CTA's sums for the weights of the queries and of the keys
  double turns[64];
};

// (cos, sin) of the four pairs of lane `l` of a head at position `p`.  The angle is reduced in turns in fp64 -- p theta / 2 pi reaches
// thousands of turns, of which fp32 keeps no fraction worth having -- and its fraction fits fp32 to 6e-8 radians.
__device__ __forceinline__ void row_angles(const double *turns, int p, int l, float (&c)[4], float (&s)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    double t = (double)p * turns[4 * l + j];
    t -= rint(t);
    sincospif(2.f * (float)t, &s[j], &c[j]);
  }
}

// The eight values of lane `l` of a head, as four rotary pairs: v[2 j], v[2 j + 1].  In the half layout pair m is (m, m + D / 2).
template <int D, int kLayout>
__device__ __forceinline__ int lane_column(int l, int half) { return kLayout == BA_ROPE_ADJACENT ? 8 * l + 4 * half : (D / 2) * half + 4 * l; }

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
// words of a, b in memory order -> pairs
template <int kLayout>
__device__ __forceinline__ void to_pairs(const Raw16 &r, float (&v)[8]) {
  const float f[8] = {lo_f(r.a.x), hi_f(r.a.x), lo_f(r.a.y), hi_f(r.a.y), lo_f(r.b.x), hi_f(r.b.x), lo_f(r.b.y), hi_f(r.b.y)};
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = kLayout == BA_ROPE_ADJACENT ? f[i] : f[(i >> 1) + 4 * (i & 1)];
}
template <int kLayout>
__device__ __forceinline__ Raw16 from_pairs(const float (&v)[8]) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[kLayout == BA_ROPE_ADJACENT ? i : (i >> 1) + 4 * (i & 1)] = v[i];
  Raw16 r;
  r.a = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
  r.b = make_uint2(pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
  return r;
}
template <int D, int kLayout>
__device__ __forceinline__ void load_pairs(const float *head, int l, float (&v)[8]) {
  const float4 a = __ldcs(reinterpret_cast<const float4 *>(head + lane_column<D, kLayout>(l, 0)));
  const float4 b = __ldcs(reinterpret_cast<const float4 *>(head + lane_column<D, kLayout>(l, 1)));
  const float f[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = kLayout == BA_ROPE_ADJACENT ? f[i] : f[(i >> 1) + 4 * (i & 1)];
}
template <int D, int kLayout>
__device__ __forceinline__ void load_pairs(const __nv_bfloat16 *head, int l, float (&v)[8]) {
  to_pairs<kLayout>(load_raw<D, kLayout>(head, l), v);
}
template <int D, int kLayout>
__device__ __forceinline__ void store_pairs(float *head, int l, const float (&v)[8]) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[kLayout == BA_ROPE_ADJACENT ? i : (i >> 1) + 4 * (i & 1)] = v[i];
  *reinterpret_cast<float4 *>(head + lane_column<D, kLayout>(l, 0)) = make_float4(f[0], f[1], f[2], f[3]);
  *reinterpret_cast<float4 *>(head + lane_column<D, kLayout>(l, 1)) = make_float4(f[4], f[5], f[6], f[7]);
}
template <int D, int kLayout>
__device__ __forceinline__ void store_pairs(__nv_bfloat16 *head, int l, const float (&v)[8]) {
  store_raw<D, kLayout>(head, l, from_pairs<kLayout>(v));
}
// Sum over the lanes of a head.
template <int D>
__device__ __forceinline__ float head_sum(float x) {
#pragma unroll
  for (int o = D / 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
template <int D, int kLayout>
__device__ __forceinline__ void load_weights(const __nv_bfloat16 *w, int l, float (&v)[8]) {
  if (w) {
    load_pairs<D, kLayout>(w, l, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 1.f;
  }
}

// Place of a row in its sequence's page list -> pool row; negative: nowhere.
struct AppendPlace { long long pool_row; bool covered; };
__device__ __forceinline__ AppendPlace find_place(const NormParams &p, int row, int lane) {
  int s = row, first = row;
  if (p.seq_cu) {
    int lo = 0, hi = p.n_seqs + 1;                         // first index whose start lies behind the row
    while (lo < hi) { const int mid = (lo + hi) >> 1; if (__ldg(p.seq_cu + mid) <= row) lo = mid + 1; else hi = mid; }
    s = lo - 1;
    if (s < 0 || s >= p.n_seqs) return {-1, false};        // a row behind the last sequence: padding
    first = __ldg(p.seq_cu + s);
  }
  const long long place = (long long)__ldg(p.seq_start + s) + (row - first);
  const int list = __ldg(p.page_cu + s);
  const long long nth = place >> p.page_lg;
  int page = -1;
  if (place >= 0 && nth < (long long)__ldg(p.page_cu + s + 1) - list) page = __ldg(p.page_idx + list + nth);
  if (page < 0 || page >= p.n_pages) {
    if (lane == 0) ba_record_status(p.status, BA_ERR_INVALID_ARG);
    return {-1, true};
  }
  return {((long long)page << p.page_lg) + (place & ((1 << p.page_lg) - 1)), true};
}

// kAppend: keys and values go through the page table.  A step is 256 / D heads; the steps of a row: queries, keys, values.
template <int D, int kLayout, bool kAppend>
__global__ void __launch_bounds__(kNormThreads)
ba_norm_rope_kernel(const __grid_constant__ NormParams p) {
  constexpr int kLanes = D / 8, kHeads = 32 / kLanes;
  __shared__ double turns[D / 2];
  const int lane = threadIdx.x & 31, l = lane % kLanes, sub = lane / kLanes;
  if (threadIdx.x < D / 2) turns[threadIdx.x] = p.turns[threadIdx.x];
  ba_pdl_wait();
  ba_pdl_trigger();
  __syncthreads();
  float wq[8], wk[8];
  load_weights<D, kLayout>(p.q.w, l, wq);
  load_weights<D, kLayout>(p.k.w, l, wk);
  const int steps_q = p.q.x ? (p.q.heads + kHeads - 1) / kHeads : 0, steps_k = p.k.x ? (p.k.heads + kHeads - 1) / kHeads : 0;
  const int steps_v = kAppend ? steps_k : 0, steps = steps_q + steps_k + steps_v;
  const long long units = (long long)p.n_rows * p.parts, stride = (long long)gridDim.x * kNormWarps;
  for (long long u = (long long)blockIdx.x * kNormWarps + (threadIdx.x >> 5); u < units; u += stride) {
    const int row = (int)(u / p.parts), part = (int)(u - (long long)row * p.parts);
    const int begin = part * p.steps_a_part, end = min(steps, begin + p.steps_a_part);
    const int pos = p.pos ? __ldg(p.pos + row) : 0;
    AppendPlace at = {0, true};
    if (kAppend) {
      at = find_place(p, row, lane);
      if (!at.covered) continue;
    }
    float c[4], s[4];
    bool have_angles = false;
    for (int i0 = begin; i0 < end; i0 += kAhead) {
      Raw16 raw[kAhead];
      const __nv_bfloat16 *src[kAhead];
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        const int i = i0 + a;
        src[a] = nullptr;
        if (i < end) {
          const bool is_q = i < steps_q, is_k = !is_q && (!kAppend || i < steps_q + steps_k);
          const NormSide &side = is_q ? p.q : is_k ? p.k : p.v;
          const int h = (i - (is_q ? 0 : is_k ? steps_q : steps_q + steps_k)) * kHeads + sub;
          if (h < side.heads) src[a] = side.x + (long long)row * side.stride + h * D;
        }
        if (src[a]) raw[a] = load_raw<D, kLayout>(src[a], l);
        else raw[a] = {make_uint2(0, 0), make_uint2(0, 0)};
      }
      if (!have_angles) { row_angles(turns, pos, l, c, s); have_angles = true; }       // (while the loads are on their way)
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        const int i = i0 + a;
        if (i >= end) break;                               // (the whole warp)
        const bool is_q = i < steps_q, is_k = !is_q && (!kAppend || i < steps_q + steps_k);
        const int h = (i - (is_q ? 0 : is_k ? steps_q : steps_q + steps_k)) * kHeads + sub;
        __nv_bfloat16 *dst;
        if (is_q) dst = p.q_out + ((long long)row * p.q.heads + h) * D;
        else if (!kAppend) dst = p.k_out + ((long long)row * p.k.heads + h) * D;
        else if (at.pool_row < 0) continue;
        else dst = (is_k ? p.k_pool : p.v_pool) + (at.pool_row * p.k.heads + h) * D;
        if (is_q || is_k) {
          float x[8];
          to_pairs<kLayout>(raw[a], x);
          if (is_q ? p.q.w != nullptr : p.k.w != nullptr) {
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
            const float r = rsqrtf(head_sum<D>(ss) * (1.f / D) + p.eps);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= r * (is_q ? wq[e] : wk[e]);
          }
          float y[8];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            y[2 * j] = x[2 * j] * c[j] - x[2 * j + 1] * s[j];
            y[2 * j + 1] = x[2 * j] * s[j] + x[2 * j + 1] * c[j];
          }
          raw[a] = from_pairs<kLayout>(y);
        }
        if (src[a]) store_raw<D, kLayout>(dst, l, raw[a]);
      }
    }
  }
}

// Gradients.  Units are shared out among warps once and for all, each lane sums the weights' gradients of its columns in fp32, the
// CTA adds its warps in order and a second kernel the CTAs: no atomics, the same bits every run.
template <int D, int kLayout, typename T>
__global__ void __launch_bounds__(kNormThreads)
ba_norm_rope_bwd_kernel(const __grid_constant__ NormBwdParams p) {
  constexpr int kLanes = D / 8, kHeads = 32 / kLanes;
  constexpr int kBwdAhead = 2;
  __shared__ double turns[D / 2];
  __shared__ float sums[kNormWarps][2][D];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane % kLanes, sub = lane / kLanes;
  if (threadIdx.x < D / 2) turns[threadIdx.x] = p.turns[threadIdx.x];
  ba_pdl_wait();
  ba_pdl_trigger();
  __syncthreads();
  float wq[8], wk[8], dwq[8], dwk[8];
  load_weights<D, kLayout>(p.q.w, l, wq);
  load_weights<D, kLayout>(p.k.w, l, wk);
#pragma unroll
  for (int e = 0; e < 8; ++e) dwq[e] = dwk[e] = 0.f;
  const int steps_q = p.q.x ? (p.q.heads + kHeads - 1) / kHeads : 0, steps_k = p.k.x ? (p.k.heads + kHeads - 1) / kHeads : 0;
  const int steps = steps_q + steps_k;
  const long long units = (long long)p.n_rows * p.parts, stride = (long long)gridDim.x * kNormWarps;
  for (long long u = (long long)blockIdx.x * kNormWarps + warp; u < units; u += stride) {
    const int row = (int)(u / p.parts), part = (int)(u - (long long)row * p.parts);
    const int begin = part * p.steps_a_part, end = min(steps, begin + p.steps_a_part);
    const int pos = p.pos ? __ldg(p.pos + row) : 0;
    float c[4], s[4];
    bool have_angles = false;
    for (int i0 = begin; i0 < end; i0 += kBwdAhead) {
      float x[kBwdAhead][8], g[kBwdAhead][8];
      bool valid[kBwdAhead];
#pragma unroll
      for (int a = 0; a < kBwdAhead; ++a) {
        const int i = i0 + a;
        const bool is_q = i < steps_q;
        const NormSide &side = is_q ? p.q : p.k;
        const int h = (i - (is_q ? 0 : steps_q)) * kHeads + sub;
        valid[a] = i < end && h < side.heads;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[a][e] = g[a][e] = 0.f;
        if (valid[a]) {
          if (side.w) load_pairs<D, kLayout>(side.x + (long long)row * side.stride + h * D, l, x[a]);
          load_pairs<D, kLayout>(reinterpret_cast<const T *>(is_q ? p.dy_q : p.dy_k) + ((long long)row * side.heads + h) * D, l, g[a]);
        }
      }
      if (!have_angles) { row_angles(turns, pos, l, c, s); have_angles = true; }
#pragma unroll
      for (int a = 0; a < kBwdAhead; ++a) {
        const int i = i0 + a;
        if (i >= end) break;                               // (the whole warp)
        const bool is_q = i < steps_q;
        const NormSide &side = is_q ? p.q : p.k;
        const int h = (i - (is_q ? 0 : steps_q)) * kHeads + sub;
#pragma unroll
        for (int j = 0; j < 4; ++j) {                      // R(-p)
          const float u0 = g[a][2 * j], u1 = g[a][2 * j + 1];
          g[a][2 * j] = u0 * c[j] + u1 * s[j];
          g[a][2 * j + 1] = u1 * c[j] - u0 * s[j];
        }
        if (side.w) {
          float ss = 0.f, hx = 0.f, hw[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            ss = fmaf(x[a][e], x[a][e], ss);
            hw[e] = g[a][e] * (is_q ? wq[e] : wk[e]);
            hx = fmaf(hw[e], x[a][e], hx);
          }
          const float r = rsqrtf(head_sum<D>(ss) * (1.f / D) + p.eps);
          const float t = head_sum<D>(hx) * (1.f / D) * r * r;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float gx = g[a][e] * (x[a][e] * r);
            if (is_q) dwq[e] += valid[a] ? gx : 0.f; else dwk[e] += valid[a] ? gx : 0.f;    // (no head there: 0 r is NaN for eps 0)
            g[a][e] = r * (hw[e] - x[a][e] * t);
          }
        }
        if (valid[a]) {
          T *dst = reinterpret_cast<T *>(is_q ? p.dq : p.dk) + (long long)row * (is_q ? p.dq_stride : p.dk_stride) + h * D;
          store_pairs<D, kLayout>(dst, l, g[a]);
        }
      }
    }
  }
  // a warp's heads, then the CTA's warps, in order
#pragma unroll
  for (int e = 0; e < 8; ++e) {
#pragma unroll
    for (int o = kLanes; o < 32; o <<= 1) {
      dwq[e] += __shfl_xor_sync(0xffffffffu, dwq[e], o);
      dwk[e] += __shfl_xor_sync(0xffffffffu, dwk[e], o);
    }
    const int col = lane_column<D, kLayout>(l, kLayout == BA_ROPE_ADJACENT ? e >> 2 : e & 1) + (kLayout == BA_ROPE_ADJACENT ? e & 3 : e >> 1);
    if (sub == 0) { sums[warp][0][col] = dwq[e]; sums[warp][1][col] = dwk[e]; }
  }
  __syncthreads();
  if (p.dw_part && threadIdx.x < 2 * D) {
    float t = 0.f;
    for (int w = 0; w < kNormWarps; ++w) t += sums[w][threadIdx.x / D][threadIdx.x % D];
    p.dw_part[(size_t)blockIdx.x * 2 * D + threadIdx.x] = t;
  }
}

// dw = the CTAs' sums, added in a fixed order: 32 columns a CTA, eight runs of CTAs side by side.
template <int D>
__global__ void __launch_bounds__(256)
ba_norm_dw_kernel(const float *part, int n, float *dw_q, float *dw_k) {
  __shared__ float sums[8][32];
  ba_pdl_wait();
  ba_pdl_trigger();
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), run = threadIdx.x >> 5;
  float t = 0.f;
  for (int b = run; b < n; b += 8) t += __ldg(part + (size_t)b * 2 * D + col);
  sums[run][threadIdx.x & 31] = t;
  __syncthreads();
  if (run == 0) {
    for (int k = 1; k < 8; ++k) t += sums[k][threadIdx.x & 31];
    float *dw = col < D ? dw_q : dw_k;
    if (dw) dw[col % D] = t;
  }
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// One side's tensor: present, aligned, rows apart far enough for whole 16-byte vectors.  `stride` 0: packed rows.
bool side_ok(const void *x, int64_t *stride, int row, int elements_16_bytes) {
  if (*stride == 0) *stride = row;
  return x && aligned16(x) && *stride >= row && *stride % elements_16_bytes == 0;
}

void fill_turns(const ba_ctx *ctx, double *turns) {
  const int half = ctx->cfg.head_dim / 2;
  for (int m = 0; m < half; ++m) turns[m] = pow(ctx->cfg.rope_theta, -(double)m / half) / 6.283185307179586476925286766559;
}

// Warps a row's steps are shared out among, and the grid.  A warp with a whole row computes its angles once (131072 rows); few rows
// are cut up until every SM has eight warps (50 rows of 20 steps: one warp each would walk them alone).
struct NormShape { int parts, steps_a_part, grid; };
NormShape norm_shape(const ba_ctx *ctx, int n_rows, int steps, int ctas_a_sm) {
  NormShape sh;
  const long long warps = (long long)ctx->sm_count * 8;
  long long parts = (warps + n_rows - 1) / n_rows;
  if (parts > steps) parts = steps;
  sh.steps_a_part = (int)((steps + parts - 1) / parts);
  sh.parts = (steps + sh.steps_a_part - 1) / sh.steps_a_part;
  const long long ctas = ((long long)n_rows * sh.parts + kNormWarps - 1) / kNormWarps, most = (long long)ctx->sm_count * ctas_a_sm;
  sh.grid = (int)(ctas < most ? ctas : most);
  return sh;
}

template <bool kAppend>
ba_status launch_norm_rope(ba_ctx *ctx, NormParams &p, cudaStream_t stream) {
  const int D = ctx->cfg.head_dim, heads = 256 / D;
  auto steps_of = [&](const NormSide &s) { return s.x ? (s.heads + heads - 1) / heads : 0; };
  const NormShape sh = norm_shape(ctx, p.n_rows, steps_of(p.q) + steps_of(p.k) * (kAppend ? 2 : 1), 8);
  p.parts = sh.parts; p.steps_a_part = sh.steps_a_part;
  p.status = ctx->dev_status;
  fill_turns(ctx, p.turns);
  auto launch = [&](auto kern) { return ba_launch(kern, dim3((unsigned)sh.grid), kNormThreads, 0, stream, true, p); };
  const bool half = ctx->cfg.rope_layout == BA_ROPE_HALF;
  if (D == 128) BA_CUDA_TRY(half ? launch(ba_norm_rope_kernel<128, BA_ROPE_HALF, kAppend>) : launch(ba_norm_rope_kernel<128, BA_ROPE_ADJACENT, kAppend>));
  else BA_CUDA_TRY(half ? launch(ba_norm_rope_kernel<64, BA_ROPE_HALF, kAppend>) : launch(ba_norm_rope_kernel<64, BA_ROPE_ADJACENT, kAppend>));
  ctx->launches += 1;
  return BA_OK;
}

bool eps_ok(float eps, const void *w_q, const void *w_k) { return (!w_q && !w_k) || (eps >= 0.f && eps <= 1e30f); }

}  // namespace

extern "C" {

ba_status ba_qk_norm_rope(ba_ctx *ctx, const void *q, int64_t q_stride, const void *k, int64_t k_stride, int32_t n_rows,
                          const int32_t *pos, const void *w_q, const void *w_k, float eps, void *q_out, void *k_out, void *stream) {
  if (!ctx || n_rows < 0 || (!q && !k) || !q != !q_out || !k != !k_out) return BA_ERR_INVALID_ARG;
  const int D = ctx->cfg.head_dim, q_row = ctx->cfg.n_q_heads * D, k_row = ctx->cfg.n_kv_heads * D;
  if ((q && !side_ok(q, &q_stride, q_row, 8)) || (k && !side_ok(k, &k_stride, k_row, 8))) return BA_ERR_INVALID_ARG;
  if (!aligned16(q_out) || !aligned16(k_out) || !aligned16(w_q) || !aligned16(w_k) || !eps_ok(eps, w_q, w_k)) return BA_ERR_INVALID_ARG;
  if ((q && q == q_out && q_stride != q_row) || (k && k == k_out && k_stride != k_row)) return BA_ERR_INVALID_ARG;
  if (n_rows == 0) return BA_OK;
  BA_CUDA_TRY(cudaSetDevice(ctx->device));
  NormParams p = {};
  p.q = {(const __nv_bfloat16 *)q, (const __nv_bfloat16 *)w_q, q_stride, ctx->cfg.n_q_heads};
  p.k = {(const __nv_bfloat16 *)k, (const __nv_bfloat16 *)w_k, k_stride, ctx->cfg.n_kv_heads};
  p.q_out = (__nv_bfloat16 *)q_out; p.k_out = (__nv_bfloat16 *)k_out;
  p.pos = pos; p.n_rows = n_rows; p.eps = eps;
  return launch_norm_rope<false>(ctx, p, (cudaStream_t)stream);
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
  if (!seq_cu && n_seqs != n_rows) return BA_ERR_SHAPE;
  if (n_rows == 0 || n_seqs == 0) return BA_OK;
  BA_CUDA_TRY(cudaSetDevice(ctx->device));
  NormParams p = {};
  p.q = {(const __nv_bfloat16 *)q, (const __nv_bfloat16 *)w_q, q_stride, ctx->cfg.n_q_heads};
  p.k = {(const __nv_bfloat16 *)k, (const __nv_bfloat16 *)w_k, k_stride, ctx->cfg.n_kv_heads};
  p.v = {(const __nv_bfloat16 *)v, nullptr, v_stride, ctx->cfg.n_kv_heads};
  p.q_out = (__nv_bfloat16 *)q_out;
  p.k_pool = (__nv_bfloat16 *)k_pool; p.v_pool = (__nv_bfloat16 *)v_pool;
  p.pos = pos; p.n_rows = n_rows; p.eps = eps;
  p.seq_cu = seq_cu; p.seq_start = seq_start; p.n_seqs = n_seqs;
  p.page_cu = pages->page_cu; p.page_idx = pages->page_idx; p.n_pages = pages->n_pages;
  while ((1 << p.page_lg) < pages->page_rows) ++p.page_lg;
  return launch_norm_rope<true>(ctx, p, (cudaStream_t)stream);
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
  if (n_rows == 0 && !w_q && !w_k) return BA_OK;
  const bool sums = w_q || w_k;
  const size_t need = sums ? (size_t)kNormGridMax * 2 * D * sizeof(float) : 0;
  if (sums && (!ctx->workspace || ba_scratch_offset(ctx) + need + ctx->pending_table_bytes > ctx->workspace_bytes)) return BA_ERR_WORKSPACE;
  BA_CUDA_TRY(cudaSetDevice(ctx->device));
  const cudaStream_t cs = (cudaStream_t)stream;
  NormBwdParams p = {};
  p.q = {(const __nv_bfloat16 *)(dq ? (w_q ? q : dy_q) : nullptr), (const __nv_bfloat16 *)w_q, q_stride, ctx->cfg.n_q_heads};
  p.k = {(const __nv_bfloat16 *)(dk ? (w_k ? k : dy_k) : nullptr), (const __nv_bfloat16 *)w_k, k_stride, ctx->cfg.n_kv_heads};
  p.dy_q = dy_q; p.dy_k = dy_k; p.dq = dq; p.dk = dk; p.dq_stride = dq_stride; p.dk_stride = dk_stride;
  p.pos = pos; p.n_rows = n_rows; p.eps = eps;
  p.dw_part = sums ? (float *)((char *)ctx->workspace + ba_scratch_offset(ctx)) : nullptr;
  fill_turns(ctx, p.turns);
  int grid = 0;
  if (n_rows > 0) {
    const int heads = 256 / D;
    NormShape sh = norm_shape(ctx, n_rows, (dq ? (ctx->cfg.n_q_heads + heads - 1) / heads : 0) + (dk ? (ctx->cfg.n_kv_heads + heads - 1) / heads : 0), 4);
    if (sh.grid > kNormGridMax) sh.grid = kNormGridMax;
    p.parts = sh.parts; p.steps_a_part = sh.steps_a_part;
    grid = sh.grid;
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
    BA_CUDA_TRY(ba_launch(kern, dim3((unsigned)(2 * D / 32)), 256, 0, cs, true, p.dw_part, grid, dw_q, dw_k));
    ctx->launches += 1;
  }
  return BA_OK;
}

}  // extern "C"

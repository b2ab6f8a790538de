// Attention of a batch whose sequences share prefixes, over a paged cache (the steps after a prompt).
//
// Work.  An entry is a prefix with the query rows of its whole group, or a sequence's own rows with its queries.  The rows of an entry
// are (token, head of a KV group) pairs, 32 to a row tile; entry x KV head x row tile is an item, its keys come in tiles of 128.  The key
// tiles of all items, laid end to end, are one stream that is cut into equal runs, one per SM, so that one long sequence, many short
// ones and a prefix of 32K keep every SM equally long.  The cut pieces of an item leave partial results (normalised rows and their
// log-sum-exp) that a second kernel merges, prefix and own rows alike; an item that is whole, of a sequence without prefix, is
// written straight to the output.  The stream is laid out on the device from the caller's tables by every CTA for itself: the lengths
// of a captured launch change from replay to replay.
//
// Structure of a CTA (384 threads, one per SM): warp 8 asks the copy engine for key and value tiles (a ring of stages, one box per page);
// warps 0-7 take 16 keys of a tile each.  With few rows a key (a decode step has one token x the heads of a group) everything is bound by
// the bytes of the cache, so the products need no more than mma.sync on operands from shared memory: S = Q K^T, softmax with
// maxima and sums of the warp's own keys, O += P V with P from registers.  The warps share nothing until the end of a piece, where
// their maxima, sums and accumulators are merged through shared memory.
//
// Rounding: P to bf16 (the products' type; 2^-9 relative, the sums of the softmax are taken before it), o once at the end.
#include <algorithm>

#include "ba_common.cuh"
#include "ba_sm100.cuh"

using namespace sm100;

bool ba_tensor_map(ba_ctx *ctx, CUtensorMap *out, const void *ptr, int heads, long long rows, int box_heads, int box_rows);

namespace {

constexpr int kTile = 128;            // keys per tile
constexpr int kRows = 32;             // rows per row tile
constexpr int kWarps = 8;             // consumer warps
constexpr int kThreads = 32 * kWarps + 128;
// Registers after launch (168 a thread): 256 * 224 + 128 * 56 = 384 * 168.  Two row tiles of 16 keep 128 accumulators and 64 words of queries.
constexpr int kConsumerRegs = 224, kCopyRegs = 56;
constexpr int kMaxEntries = BA_SHARED_MAX;
constexpr float kRescale = 8.f;       // O is rescaled when a maximum grows by more than 2^8: exact in real arithmetic, values stay bounded

struct SharedParams {
  const __nv_bfloat16 *q;
  void *o;
  float *lse;
  int32_t *status;
  int out_f32, Hq, Hkv, G;
  float scale_log2;
  int n_q_rows, batch, n_groups;
  const int32_t *group_cu, *prefix_cu, *q_cu, *own_len;
  int n_prefix_rows;                  // packed prefixes
  int prefix_paged;
  const int32_t *prefix_page_cu, *prefix_page_idx, *page_cu, *page_idx;
  int prefix_page_lg, page_lg, prefix_pages, n_pages;
  float *part;                        // partial results: a slot is [kRows][D] values and [kRows] log-sum-exps
  int n_slots;
  int4 *meta;                         // [n_groups + batch]: first unit, tiles, row tiles, first item; then one of units a CTA, validity
};

template <int D>
struct SharedLayout {
  static constexpr int kChunks = D / 64;
  static constexpr int kTileBytes = kTile * D * 2;
  static constexpr int kStages = D == 128 ? 5 : 10;
  static constexpr int kRegion = kTile * 128;
  static constexpr int kBufStride = 68;                                // floats a row: rows of a quad's lanes in different banks
  static constexpr int kBuf = kStages * kTileBytes;                    // [kWarps][16][kBufStride]
  static constexpr int kStat = kBuf + kWarps * 16 * kBufStride * 4;    // [kWarps][kRows] (maximum, sum)
  static constexpr int kUnits = kStat + kWarps * kRows * 8;            // [kMaxEntries + 1]
  static constexpr int kItems = kUnits + (kMaxEntries + 4) * 4;        // [kMaxEntries + 1]
  static constexpr int kCtrl = kItems + (kMaxEntries + 4) * 4;
  static constexpr int kBytes = kCtrl + 512 + 1024;
  static constexpr int kSlot = kRows * (D + 1);                        // floats
};
static_assert(SharedLayout<128>::kBytes <= 227 * 1024, "shared memory");

struct SharedCtrl {
  uint64_t full[10], empty[10];
  int abort_flag, invalid;
  int warp_units[kThreads / 32], warp_items[kThreads / 32];
};
static_assert(sizeof(SharedCtrl) <= 512, "control area");

// An entry, looked up by the thread that asks: rows q_row0 .. of the queries, `len` keys.
struct Entry { int q_row0, rows, len; };
__device__ __forceinline__ int q_begin(const SharedParams &p, int s) { return p.q_cu ? __ldg(p.q_cu + s) : s; }
__device__ __forceinline__ Entry get_entry(const SharedParams &p, int e) {
  Entry x;
  if (e < p.n_groups) {
    const int a = p.group_cu ? __ldg(p.group_cu + e) : 0, b = p.group_cu ? __ldg(p.group_cu + e + 1) : p.batch;
    x.q_row0 = q_begin(p, a); x.rows = q_begin(p, b) - x.q_row0;
    x.len = __ldg(p.prefix_cu + e + 1) - __ldg(p.prefix_cu + e);
  } else {
    const int s = e - p.n_groups;
    x.q_row0 = q_begin(p, s); x.rows = q_begin(p, s + 1) - x.q_row0;
    x.len = __ldg(p.own_len + s);
  }
  return x;
}
// The tables of entry e hold: nothing else of them is read where they do not.
__device__ __forceinline__ bool entry_holds(const SharedParams &p, int e) {
  if (e < p.n_groups) {
    if (p.group_cu) {
      const int a = __ldg(p.group_cu + e), b = __ldg(p.group_cu + e + 1);
      if (a < 0 || b < a || b > p.batch) return false;
    }
    const int r0 = __ldg(p.prefix_cu + e), r1 = __ldg(p.prefix_cu + e + 1);
    if (r0 < 0 || r1 < r0) return false;
    if (!p.prefix_paged) return r1 <= p.n_prefix_rows;
    return (long long)(r1 - r0) <= ((long long)__ldg(p.prefix_page_cu + e + 1) - __ldg(p.prefix_page_cu + e)) << p.prefix_page_lg;
  }
  const int s = e - p.n_groups, a = q_begin(p, s), b = q_begin(p, s + 1), len = __ldg(p.own_len + s);
  if (a < 0 || b < a || b > p.n_q_rows || len < 0) return false;
  return len == 0 || (long long)len <= ((long long)__ldg(p.page_cu + s + 1) - __ldg(p.page_cu + s)) << p.page_lg;
}
__device__ __forceinline__ int tiles_of(const Entry &x) { return (x.len + kTile - 1) / kTile; }
__device__ __forceinline__ int row_tiles_of(const SharedParams &p, const Entry &x) { return (int)(((long long)x.rows * p.G + kRows - 1) / kRows); }

// Last index in x[0 .. n] whose value is at most v (x[0] = 0 <= v).
__device__ __forceinline__ int last_at_most(const int *x, int n, int v) {
  int lo = 0, hi = n + 1;
  while (lo < hi) { const int mid = (lo + hi) >> 1; if (x[mid] <= v) lo = mid + 1; else hi = mid; }
  return lo - 1;
}
// The group of sequence s, or -1.
__device__ __forceinline__ int group_of(const SharedParams &p, int s) {
  if (p.n_groups == 0) return -1;
  if (!p.group_cu) return 0;
  int lo = 0, hi = p.n_groups + 1;
  while (lo < hi) { const int mid = (lo + hi) >> 1; if (__ldg(p.group_cu + mid) <= s) lo = mid + 1; else hi = mid; }
  return lo - 1 < p.n_groups ? lo - 1 : -1;
}

// A piece of the stream: key tiles tile0 .. tile0 + n - 1 of an item.
struct Piece {
  int e, head, row_tile, tile0, n, tiles, slot;
  Entry x;
};
// The piece that starts at unit `at` of this CTA's run, which ends at `end`.
__device__ __forceinline__ Piece piece_at(const SharedParams &p, const int *units, const int *items, int n_entries, int at, int end) {
  Piece k;
  k.e = last_at_most(units, n_entries, at);
  k.x = get_entry(p, k.e);
  k.tiles = tiles_of(k.x);
  const int local = at - units[k.e], item = local / k.tiles, rts = row_tiles_of(p, k.x);
  k.tile0 = local - item * k.tiles;
  k.head = item / rts; k.row_tile = item - k.head * rts;
  k.n = min(k.tiles - k.tile0, end - at);
  k.slot = items[k.e] + item + (int)blockIdx.x;
  return k;
}

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory"); }

// One piece of an item with kM x 16 rows: the consumer warps' work.  Returns with the ring position moved on.
template <int D, int kM>
__device__ __forceinline__ void consume_piece(const SharedParams &p, const Piece &k, uint8_t *smem, SharedCtrl *ctrl, int &ring, bool &ok, bool direct) {
  using L = SharedLayout<D>;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quad = lane >> 2, in_quad = lane & 3;
  volatile int *abort_flag = &ctrl->abort_flag;
  const bool own = k.e >= p.n_groups;
  const int n_rows = min(kRows, k.x.rows * p.G - k.row_tile * kRows);
  // queries as A operands, straight from memory; rows past the item's are zeros
  uint32_t qa[kM][D / 16][4];
  int limit[kM][2];                      // keys that the lane's rows see
#pragma unroll
  for (int m = 0; m < kM; ++m)
#pragma unroll
    for (int hi = 0; hi < 2; ++hi) {
      const int r = m * 16 + hi * 8 + quad;
      const bool there = r < n_rows;
      const int rr = k.row_tile * kRows + (there ? r : 0), tok = rr / p.G, h = k.head * p.G + rr - tok * p.G;
      const uint32_t *src = reinterpret_cast<const uint32_t *>(p.q + ((size_t)(k.x.q_row0 + tok) * p.Hq + h) * D) + in_quad;
      limit[m][hi] = own ? k.x.len - (k.x.rows - 1 - tok) : k.x.len;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        qa[m][c][hi] = there ? __ldg(src + c * 8) : 0u;
        qa[m][c][hi + 2] = there ? __ldg(src + c * 8 + 4) : 0u;
      }
    }
  float o[kM][D / 8][4], mx[kM][2], sum[kM][2];
#pragma unroll
  for (int m = 0; m < kM; ++m) {
#pragma unroll
    for (int c = 0; c < D / 8; ++c) o[m][c][0] = o[m][c][1] = o[m][c][2] = o[m][c][3] = 0.f;
    mx[m][0] = mx[m][1] = -INFINITY; sum[m][0] = sum[m][1] = 0.f;
  }
  const float sl = p.scale_log2;
  const int k_row = warp * 16 + ((lane >> 4) & 1) * 8 + (lane & 7), k_col = (lane >> 3) & 1;
  const int v_row = warp * 16 + ((lane >> 3) & 1) * 8 + (lane & 7), v_col = (lane >> 4) & 1;
  for (int j = 0; j < k.n; ++j, ring += 2) {
    const int key0 = (k.tile0 + j) * kTile + warp * 16;    // this warp's keys
    const int left = k.x.len - key0;
    const int ks = ring % L::kStages, vs = (ring + 1) % L::kStages;
    if (ok) ok = mbar_wait(&ctrl->full[ks], (ring / L::kStages) & 1, abort_flag);
    float s[kM][2][4];
    if (ok && left > 0) {
      const uint32_t tile = smem_u32(smem + ks * L::kTileBytes) + k_row * 128;
#pragma unroll
      for (int m = 0; m < kM; ++m)
#pragma unroll
        for (int n = 0; n < 2; ++n) s[m][n][0] = s[m][n][1] = s[m][n][2] = s[m][n][3] = 0.f;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        uint32_t b[4];
        const int col = c * 2 + k_col;
        ldsm4(b, tile + (col >> 3) * L::kRegion + (((col & 7) ^ (k_row & 7)) << 4));
#pragma unroll
        for (int m = 0; m < kM; ++m) { mma_16816(s[m][0], qa[m][c], b[0], b[1]); mma_16816(s[m][1], qa[m][c], b[2], b[3]); }
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&ctrl->empty[ks]);
    uint32_t pa[kM][4];
    if (ok && left > 0) {
#pragma unroll
      for (int m = 0; m < kM; ++m) {
        const bool masked = key0 + 16 > min(limit[m][0], limit[m][1]);
        float top[2];
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
          if (masked) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (key0 + (i >> 1) * 8 + in_quad * 2 + (i & 1) >= limit[m][hi]) s[m][i >> 1][hi * 2 + (i & 1)] = -INFINITY;
          }
          top[hi] = fmaxf(fmaxf(s[m][0][hi * 2], s[m][0][hi * 2 + 1]), fmaxf(s[m][1][hi * 2], s[m][1][hi * 2 + 1]));
          top[hi] = fmaxf(top[hi], __shfl_xor_sync(0xffffffffu, top[hi], 1));
          top[hi] = fmaxf(top[hi], __shfl_xor_sync(0xffffffffu, top[hi], 2));
          top[hi] = fmaxf(top[hi], mx[m][hi]);
        }
        const bool grow = (top[0] > mx[m][0] && !((top[0] - mx[m][0]) * sl <= kRescale)) || (top[1] > mx[m][1] && !((top[1] - mx[m][1]) * sl <= kRescale));
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
          for (int hi = 0; hi < 2; ++hi) {
            const float alpha = mx[m][hi] == -INFINITY ? 0.f : ex2((mx[m][hi] - top[hi]) * sl);     // (nothing summed so far)
            mx[m][hi] = top[hi];
            sum[m][hi] *= alpha;
#pragma unroll
            for (int c = 0; c < D / 8; ++c) { o[m][c][hi * 2] *= alpha; o[m][c][hi * 2 + 1] *= alpha; }
          }
        }
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
          const float neg = mx[m][hi] == -INFINITY ? 0.f : -mx[m][hi] * sl;
          float e[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) e[i] = ex2(fmaf(s[m][i >> 1][hi * 2 + (i & 1)], sl, neg));
          sum[m][hi] += (e[0] + e[1]) + (e[2] + e[3]);
          pa[m][hi] = pack_bf16(e[0], e[1]);
          pa[m][hi + 2] = pack_bf16(e[2], e[3]);
        }
      }
    }
    if (ok) ok = mbar_wait(&ctrl->full[vs], ((ring + 1) / L::kStages) & 1, abort_flag);
    if (ok && left > 0) {
      uint8_t *tile = smem + vs * L::kTileBytes;
      if (left < 16) {
        // values behind the end may be anything, and zero times a NaN is a NaN
        for (int i = lane; i < (16 - left) * (D / 8); i += 32) {
          const int row = warp * 16 + left + i / (D / 8), col = i % (D / 8);
          *reinterpret_cast<uint4 *>(tile + (col >> 3) * L::kRegion + row * 128 + ((col & 7) << 4)) = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async();                               // (the copy engine writes the stage next)
        __syncwarp();
      }
      const uint32_t base = smem_u32(tile) + v_row * 128;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        uint32_t b[4];
        const int col = c * 2 + v_col;
        ldsm4_t(b, base + (col >> 3) * L::kRegion + (((col & 7) ^ (v_row & 7)) << 4));
#pragma unroll
        for (int m = 0; m < kM; ++m) { mma_16816(o[m][2 * c], pa[m], b[0], b[1]); mma_16816(o[m][2 * c + 1], pa[m], b[2], b[3]); }
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&ctrl->empty[vs]);
  }
  // The warps' results: rows' maxima and sums are exchanged, every accumulator is scaled to the common maximum and divided by the
  // common sum, and the eight are added 64 columns at a time.
  float2 *stat = reinterpret_cast<float2 *>(smem + L::kStat);
  float *buf = reinterpret_cast<float *>(smem + L::kBuf);
#pragma unroll
  for (int m = 0; m < kM; ++m)
#pragma unroll
    for (int hi = 0; hi < 2; ++hi) {
      sum[m][hi] += __shfl_xor_sync(0xffffffffu, sum[m][hi], 1);
      sum[m][hi] += __shfl_xor_sync(0xffffffffu, sum[m][hi], 2);
      if (in_quad == 0) stat[warp * kRows + m * 16 + hi * 8 + quad] = make_float2(mx[m][hi], sum[m][hi]);
    }
  consumers_sync();
  float *slot = p.part + (size_t)k.slot * L::kSlot;
  const bool fits = k.slot < p.n_slots;                    // (always, by the host's count; a table that changes meanwhile would not)
#pragma unroll
  for (int m = 0; m < kM; ++m) {
    float f[2];
#pragma unroll
    for (int hi = 0; hi < 2; ++hi) {
      const int r = m * 16 + hi * 8 + quad;
      float top = -INFINITY, den = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, stat[w * kRows + r].x);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float2 v = stat[w * kRows + r];
        if (v.x != -INFINITY) den += v.y * ex2((v.x - top) * sl);
      }
      f[hi] = mx[m][hi] != -INFINITY && den > 0.f ? ex2((mx[m][hi] - top) * sl) / den : 0.f;
      if (ok && warp == 0 && in_quad == 0 && r < n_rows) {
        const float lse = den > 0.f ? (top * sl + log2f(den)) * 0.6931471805599453f : -INFINITY;
        if (!direct) {
          if (fits) slot[kRows * D + r] = lse;
        } else if (p.lse) {
          const int rr = k.row_tile * kRows + r, tok = rr / p.G;
          p.lse[(size_t)(k.x.q_row0 + tok) * p.Hq + k.head * p.G + rr - tok * p.G] = lse;
        }
      }
    }
#pragma unroll
    for (int half = 0; half < D / 64; ++half) {
      float *mine = buf + warp * 16 * L::kBufStride;
#pragma unroll
      for (int c = 0; c < 8; ++c)
#pragma unroll
        for (int hi = 0; hi < 2; ++hi)
          *reinterpret_cast<float2 *>(mine + (hi * 8 + quad) * L::kBufStride + c * 8 + in_quad * 2) =
              make_float2(o[m][half * 8 + c][hi * 2] * f[hi], o[m][half * 8 + c][hi * 2 + 1] * f[hi]);
      consumers_sync();
      const int r = threadIdx.x >> 4, col = (threadIdx.x & 15) * 4;
      if (ok && m * 16 + r < n_rows) {
        float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float4 v = *reinterpret_cast<const float4 *>(buf + (w * 16 + r) * L::kBufStride + col);
          t.x += v.x; t.y += v.y; t.z += v.z; t.w += v.w;
        }
        if (!direct) {
          if (fits) *reinterpret_cast<float4 *>(slot + (m * 16 + r) * D + half * 64 + col) = t;
        } else {
          const int rr = k.row_tile * kRows + m * 16 + r, tok = rr / p.G;
          const size_t at = ((size_t)(k.x.q_row0 + tok) * p.Hq + k.head * p.G + rr - tok * p.G) * D + half * 64 + col;
          if (p.out_f32) *reinterpret_cast<float4 *>(reinterpret_cast<float *>(p.o) + at) = t;
          else *reinterpret_cast<uint2 *>(reinterpret_cast<__nv_bfloat16 *>(p.o) + at) = make_uint2(pack_bf16(t.x, t.y), pack_bf16(t.z, t.w));
        }
      }
      consumers_sync();
    }
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
ba_shared_attend_kernel(const __grid_constant__ CUtensorMap tmap_kx, const __grid_constant__ CUtensorMap tmap_vx,
                        const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                        const __grid_constant__ SharedParams p) {
  using L = SharedLayout<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  SharedCtrl *ctrl = reinterpret_cast<SharedCtrl *>(smem + L::kCtrl);
  int *units = reinterpret_cast<int *>(smem + L::kUnits), *items = reinterpret_cast<int *>(smem + L::kItems);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_entries = p.n_groups + p.batch;
  if (tid == 0) {
    for (int s = 0; s < L::kStages; ++s) { mbar_init(&ctrl->full[s], 1); mbar_init(&ctrl->empty[s], kWarps); }
    ctrl->abort_flag = 0; ctrl->invalid = 0;
    fence_barrier_init();
  }
  if (warp == kWarps && elect_one()) { prefetch_tmap(&tmap_k); prefetch_tmap(&tmap_v); prefetch_tmap(&tmap_kx); prefetch_tmap(&tmap_vx); }
  ba_pdl_wait();
  ba_pdl_trigger();
  __syncthreads();
  // The stream: units (key tiles) and items of every entry, summed up.  A thread takes neighbouring entries.
  {
    const int per = (n_entries + kThreads - 1) / kThreads, e0 = min(n_entries, tid * per), e1 = min(n_entries, e0 + per);
    bool good = true;
    for (int e = e0; e < e1; ++e) good = good && entry_holds(p, e);
    if (!good) ctrl->invalid = 1;
    __syncthreads();
    long long nu = 0, ni = 0;
    if (!ctrl->invalid) {                                  // (groups read the queries' table of other threads' sequences)
      for (int e = e0; e < e1; ++e) {
        const Entry x = get_entry(p, e);
        const long long it = (long long)row_tiles_of(p, x) * p.Hkv;
        nu += it * tiles_of(x); ni += it;
      }
      if (nu > INT32_MAX || ni > INT32_MAX) { nu = ni = 0; ctrl->invalid = 1; }
    }
    // sums over the warp, then over the warps, in doubles: whole numbers up to 2^53, so that an overflow shows
    double su = (double)nu, si = (double)ni;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const double a = __shfl_up_sync(0xffffffffu, su, d), b = __shfl_up_sync(0xffffffffu, si, d);
      if (lane >= d) { su += a; si += b; }
    }
    if (su > 2e9 || si > 2e9) ctrl->invalid = 1;
    if (lane == 31) { ctrl->warp_units[warp] = su > 2e9 ? 0 : (int)su; ctrl->warp_items[warp] = si > 2e9 ? 0 : (int)si; }
    __syncthreads();
    for (int w = 0; w < warp; ++w) { su += ctrl->warp_units[w]; si += ctrl->warp_items[w]; }
    if (su > 2e9 || si > 2e9) ctrl->invalid = 1;
    __syncthreads();
    if (!ctrl->invalid) {
      int u = (int)(su - (double)nu), i = (int)(si - (double)ni);
      for (int e = e0; e < e1; ++e) {
        units[e] = u; items[e] = i;
        const Entry x = get_entry(p, e);
        const int it = row_tiles_of(p, x) * p.Hkv, tiles = tiles_of(x);
        if (blockIdx.x == 0) p.meta[e] = make_int4(u, tiles, row_tiles_of(p, x), i);
        u += it * tiles; i += it;
      }
      if (tid == kThreads - 1) { units[n_entries] = (int)su; items[n_entries] = (int)si; }
    }
    __syncthreads();
  }
  const bool valid = !ctrl->invalid;
  const int total = valid ? units[n_entries] : 0;
  const int run = (total + (int)gridDim.x - 1) / (int)gridDim.x;
  if (blockIdx.x == 0 && tid == 0) {
    p.meta[n_entries] = make_int4(run, valid, 0, 0);
    if (!valid) ba_record_status(p.status, BA_ERR_INVALID_ARG);
  }
  const int begin = (int)min((long long)total, (long long)run * blockIdx.x), end = min(total, begin + run);
  if (begin < end) {
    int ring = 0;
    bool ok = true;
    if (warp >= kWarps) {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kCopyRegs));
      if (warp == kWarps) {
        // ------------------------------------------------------------ copies
        for (int at = begin; at < end && ok;) {
          const Piece k = piece_at(p, units, items, n_entries, at, end);
          at += k.n;
          const bool own = k.e >= p.n_groups, paged = own || p.prefix_paged;
          const CUtensorMap *mk = own ? &tmap_k : &tmap_kx, *mv = own ? &tmap_v : &tmap_vx;
          const int lg = own ? p.page_lg : p.prefix_page_lg, n_pages = own ? p.n_pages : p.prefix_pages;
          const int sub_rows = paged ? min(kTile, 1 << lg) : kTile;
          const int list = own ? __ldg(p.page_cu + k.e - p.n_groups) : paged ? __ldg(p.prefix_page_cu + k.e) : 0;
          const int32_t *idx = own ? p.page_idx : p.prefix_page_idx;
          const int first = paged ? 0 : __ldg(p.prefix_cu + k.e);
          // lane i has box i of a tile, a box per page; the row of its next box is looked up a tile ahead
          auto row_of = [&](int tile) -> int {
            const int t = tile * kTile + lane * sub_rows;
            if (lane * sub_rows >= kTile || t >= k.x.len) return -1;
            if (!paged) return first + t;
            const int page = __ldg(idx + list + (t >> lg));
            if (page < 0 || page >= n_pages) {
              ba_record_status(p.status, BA_ERR_INVALID_ARG);
              return n_pages << lg;                          // behind the pool: the copy engine fills in zeros
            }
            return (page << lg) + (t & ((1 << lg) - 1));
          };
          int next = row_of(k.tile0);
          for (int j = 0; j < k.n && ok; ++j) {
            const int row = next;
            if (j + 1 < k.n) next = row_of(k.tile0 + j + 1);
            const unsigned boxes = __popc(__ballot_sync(0xffffffffu, row >= 0));
            for (int kv = 0; kv < 2; ++kv, ++ring) {
              const int stage = ring % L::kStages;
              ok = mbar_wait(&ctrl->empty[stage], ((ring / L::kStages) & 1) ^ 1, &ctrl->abort_flag);
              ok = __all_sync(0xffffffffu, ok);
              if (!ok) break;
              if (lane == 0) mbar_arrive_expect_tx(&ctrl->full[stage], boxes * sub_rows * D * 2);
              __syncwarp();
              if (row >= 0) {
                uint8_t *dst = smem + stage * L::kTileBytes + lane * sub_rows * 128;
                for (int c = 0; c < L::kChunks; ++c) tma_load_3d(dst + c * L::kRegion, kv ? mv : mk, &ctrl->full[stage], c * 64, k.head, row);
              }
              __syncwarp();
            }
          }
        }
        if (!ok) {
          // leave no copy in flight: wait (bounded) for the tiles already requested
          for (int i = max(0, ring - L::kStages); i < ring; ++i)
            for (uint32_t spin = 0; spin < (1u << 20); ++spin)
              if (mbar_try_wait(&ctrl->full[i % L::kStages], (i / L::kStages) & 1)) break;
        }
      }
    } else {
      asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kConsumerRegs));
      for (int at = begin; at < end;) {                    // (to the end even after a wait that expired: the warps meet at barriers)
        const Piece k = piece_at(p, units, items, n_entries, at, end);
        at += k.n;
        bool direct = k.e >= p.n_groups && k.n == k.tiles;
        if (direct) {
          const int g = group_of(p, k.e - p.n_groups);
          direct = g < 0 || units[g + 1] == units[g];
        }
        if (min(kRows, k.x.rows * p.G - k.row_tile * kRows) <= 16) consume_piece<D, 1>(p, k, smem, ctrl, ring, ok, direct);
        else consume_piece<D, 2>(p, k, smem, ctrl, ring, ok, direct);
      }
    }
  }
  __syncthreads();
  if (tid == 0 && ctrl->abort_flag) ba_record_status(p.status, BA_ERR_TIMEOUT);
}

// The partial results of every (row, head): those of its group's prefix and of its own rows, weighted by their denominators.  A warp
// has a row of 128 values, or two of 64.
template <int D>
__global__ void __launch_bounds__(256)
ba_shared_merge_kernel(const __grid_constant__ SharedParams p) {
  using L = SharedLayout<D>;
  constexpr int kLanes = D / 4, kAt = 256 / kLanes;
  ba_pdl_wait();
  ba_pdl_trigger();
  const int4 head = p.meta[p.n_groups + p.batch];          // (plain loads: the kernel before wrote them)
  if (!head.y) return;
  const int run = head.x;
  const long long u = (long long)blockIdx.x * kAt + threadIdx.x / kLanes;
  const int c = threadIdx.x % kLanes;
  if (u >= (long long)p.n_q_rows * p.Hq) return;
  const int row = (int)(u / p.Hq), hq = (int)(u - (long long)row * p.Hq), h = hq / p.G;
  int s = row;
  if (p.q_cu) {
    int lo = 0, hi = p.batch + 1;
    while (lo < hi) { const int mid = (lo + hi) >> 1; if (__ldg(p.q_cu + mid) <= row) lo = mid + 1; else hi = mid; }
    s = lo - 1;
  }
  if (s < 0 || s >= p.batch) return;
  const int g = group_of(p, s);
  float top = -INFINITY, den = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  int pieces = 0;
#pragma unroll 1
  for (int side = 0; side < 2; ++side) {
    const int e = side == 0 ? g : p.n_groups + s;
    if (e < 0) continue;
    const int4 m = p.meta[e];
    if (m.y == 0) continue;
    const int row0 = side == 0 ? q_begin(p, p.group_cu ? __ldg(p.group_cu + g) : 0) : q_begin(p, s);
    const int r = (row - row0) * p.G + hq - h * p.G, rt = r / kRows, item = h * m.z + rt;
    const int a = m.x + item * m.y, c0 = a / run, c1 = (a + m.y - 1) / run;
    if (side == 1 && pieces == 0 && c0 == c1) return;      // whole, and nothing beside it: written where it was computed
    for (int k = c0; k <= c1; ++k, ++pieces) {
      const int at = m.w + item + k;
      if (at >= p.n_slots) return;
      const float *slot = p.part + (size_t)at * L::kSlot;
      const float lse = slot[kRows * D + r - rt * kRows];
      if (lse == -INFINITY) continue;
      const float4 x = __ldcs(reinterpret_cast<const float4 *>(slot + (r - rt * kRows) * D) + c);
      const float t = fmaxf(top, lse), fa = top == -INFINITY ? 0.f : __expf(top - t), fx = __expf(lse - t);
      top = t;
      den = den * fa + fx;
      acc.x = acc.x * fa + x.x * fx; acc.y = acc.y * fa + x.y * fx; acc.z = acc.z * fa + x.z * fx; acc.w = acc.w * fa + x.w * fx;
    }
  }
  const float inv = den > 0.f ? 1.f / den : 0.f;
  const size_t out = (size_t)u * D + c * 4;
  if (p.out_f32) *reinterpret_cast<float4 *>(reinterpret_cast<float *>(p.o) + out) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
  else *reinterpret_cast<uint2 *>(reinterpret_cast<__nv_bfloat16 *>(p.o) + out) = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
  if (p.lse && c == 0) p.lse[u] = den > 0.f ? top + logf(den) : -INFINITY;
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Slots: a piece per item, and one more for every cut (one per CTA at most).  Items: row tiles of prefixes and of own rows, each
// entry with one that is not full.
long long slots_for(const ba_config &c, int batch, int n_groups, int n_q_rows, int n_ctas) {
  const long long G = c.n_q_heads / c.n_kv_heads, rows = (long long)n_q_rows * G;
  return (2 * (rows / kRows) + n_groups + batch) * c.n_kv_heads + n_ctas;
}
size_t meta_bytes(int n_entries) { return ba_align_up((size_t)(n_entries + 1) * sizeof(int4), 256); }
constexpr int kMostCtas = 256;        // sizing without a device

}  // namespace

ba_status ba_shared_sm100_setup() {
  BA_CUDA_TRY(cudaFuncSetAttribute(ba_shared_attend_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, SharedLayout<128>::kBytes));
  BA_CUDA_TRY(cudaFuncSetAttribute(ba_shared_attend_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, SharedLayout<64>::kBytes));
  return BA_OK;
}

extern "C" {

ba_status ba_shared_prefix_bytes(const ba_config *cfg, int32_t batch, int32_t n_groups, int32_t n_q_rows, size_t *bytes) {
  size_t least;
  ba_status st = ba_workspace_bytes(cfg, 1, 0, &least);    // (checks the configuration)
  if (st != BA_OK) return st;
  if (!bytes || batch < 1 || n_groups < 0 || n_q_rows < 0) return BA_ERR_INVALID_ARG;
  if ((long long)batch + n_groups > BA_SHARED_MAX) return BA_ERR_UNSUPPORTED;
  *bytes = ba_scratch_offset(nullptr) + meta_bytes(batch + n_groups) +
           (size_t)slots_for(*cfg, batch, n_groups, n_q_rows, kMostCtas) * kRows * (cfg->head_dim + 1) * sizeof(float) + 256;
  return BA_OK;
}

ba_status ba_shared_prefix_attend(ba_ctx *ctx, const void *q, int32_t n_q_rows, const void *k_prefix, const void *v_prefix,
                                  int32_t n_prefix_rows, const ba_page_table *prefix_pages, const void *k_pool, const void *v_pool,
                                  const ba_page_table *pages, const ba_shared_batch *b, void *o, float *lse,
                                  ba_out_dtype out_dtype, void *stream) {
  ba_status st = ba_check_pages(pages);
  if (st != BA_OK) return st;
  if (!ctx || !b || n_q_rows < 0 || n_prefix_rows < 0 || b->batch < 0 || b->n_groups < 0) return BA_ERR_INVALID_ARG;
  if (out_dtype != BA_OUT_BF16 && out_dtype != BA_OUT_F32) return BA_ERR_INVALID_ARG;
  if ((long long)b->batch + b->n_groups > BA_SHARED_MAX) return BA_ERR_UNSUPPORTED;
  if (b->batch > 0 && (!b->own_len || !k_pool || !v_pool || !aligned16(k_pool) || !aligned16(v_pool))) return BA_ERR_INVALID_ARG;
  if (!b->q_cu && b->batch != n_q_rows) return BA_ERR_SHAPE;
  if (n_q_rows > 0 && (!q || !o || !aligned16(q) || !aligned16(o))) return BA_ERR_INVALID_ARG;
  if (b->n_groups > 0) {
    if (!b->prefix_cu || (!b->group_cu && b->n_groups != 1)) return BA_ERR_INVALID_ARG;
    if (prefix_pages && (st = ba_check_pages(prefix_pages)) != BA_OK) return st;
    // (packed prefixes without a row: nothing to read)
    if ((prefix_pages || n_prefix_rows > 0) && (!k_prefix || !v_prefix || !aligned16(k_prefix) || !aligned16(v_prefix))) return BA_ERR_INVALID_ARG;
  }
  if (b->batch == 0 || n_q_rows == 0) return BA_OK;
  const int D = ctx->cfg.head_dim, n_entries = b->batch + b->n_groups;
  const long long n_slots = slots_for(ctx->cfg, b->batch, b->n_groups, n_q_rows, ctx->sm_count);
  const size_t need = meta_bytes(n_entries) + (size_t)n_slots * kRows * (D + 1) * sizeof(float);
  if (!ctx->workspace || ba_scratch_offset(ctx) + need + ctx->pending_table_bytes > ctx->workspace_bytes) return BA_ERR_WORKSPACE;
  if (n_slots > INT32_MAX || (long long)n_q_rows * ctx->cfg.n_q_heads > INT32_MAX) return BA_ERR_SHAPE;
  BA_CUDA_TRY(cudaSetDevice(ctx->device));
  auto lg_of = [](const ba_page_table *t) { int lg = 0; while ((1 << lg) < t->page_rows) ++lg; return lg; };
  SharedParams p = {};
  p.q = (const __nv_bfloat16 *)q; p.o = o; p.lse = lse; p.status = ctx->dev_status;
  p.out_f32 = out_dtype == BA_OUT_F32;
  p.Hq = ctx->cfg.n_q_heads; p.Hkv = ctx->cfg.n_kv_heads; p.G = p.Hq / p.Hkv;
  p.scale_log2 = ctx->scale * 1.4426950408889634f;
  p.n_q_rows = n_q_rows; p.batch = b->batch; p.n_groups = b->n_groups;
  p.group_cu = b->group_cu; p.prefix_cu = b->prefix_cu; p.q_cu = b->q_cu; p.own_len = b->own_len;
  p.n_prefix_rows = n_prefix_rows;
  p.page_cu = pages->page_cu; p.page_idx = pages->page_idx; p.page_lg = lg_of(pages); p.n_pages = pages->n_pages;
  const bool has_prefix = b->n_groups > 0 && (prefix_pages || n_prefix_rows > 0);
  if (b->n_groups > 0 && prefix_pages) {
    p.prefix_paged = 1;
    p.prefix_page_cu = prefix_pages->page_cu; p.prefix_page_idx = prefix_pages->page_idx;
    p.prefix_page_lg = lg_of(prefix_pages); p.prefix_pages = prefix_pages->n_pages;
  }
  char *scratch = (char *)ctx->workspace + ba_scratch_offset(ctx);
  p.meta = (int4 *)scratch;
  p.part = (float *)(scratch + meta_bytes(n_entries));
  p.n_slots = (int)n_slots;
  CUtensorMap tk, tv, tkx, tvx;
  const long long rows = (long long)pages->n_pages * pages->page_rows;
  const int box = std::min(kTile, pages->page_rows);
  if (!ba_tensor_map(ctx, &tk, k_pool, p.Hkv, rows, 1, box) || !ba_tensor_map(ctx, &tv, v_pool, p.Hkv, rows, 1, box)) return BA_ERR_CUDA;
  tkx = tk; tvx = tv;
  if (has_prefix) {
    const long long prows = prefix_pages ? (long long)prefix_pages->n_pages * prefix_pages->page_rows : n_prefix_rows;
    const int pbox = prefix_pages ? std::min(kTile, prefix_pages->page_rows) : kTile;
    if (!ba_tensor_map(ctx, &tkx, k_prefix, p.Hkv, prows, 1, pbox) || !ba_tensor_map(ctx, &tvx, v_prefix, p.Hkv, prows, 1, pbox)) return BA_ERR_CUDA;
  }
  const dim3 grid((unsigned)ctx->sm_count);
  const cudaStream_t cs = (cudaStream_t)stream;
  const unsigned merge = (unsigned)(((long long)n_q_rows * p.Hq * (D / 4) + 255) / 256);
  if (D == 128) {
    BA_CUDA_TRY(ba_launch(ba_shared_attend_kernel<128>, grid, kThreads, SharedLayout<128>::kBytes, cs, true, tkx, tvx, tk, tv, p));
    BA_CUDA_TRY(ba_launch(ba_shared_merge_kernel<128>, dim3(merge), 256, 0, cs, true, p));
  } else {
    BA_CUDA_TRY(ba_launch(ba_shared_attend_kernel<64>, grid, kThreads, SharedLayout<64>::kBytes, cs, true, tkx, tvx, tk, tv, p));
    BA_CUDA_TRY(ba_launch(ba_shared_merge_kernel<64>, dim3(merge), 256, 0, cs, true, p));
  }
  ctx->launches += 2;
  return BA_OK;
}

}  // extern "C"

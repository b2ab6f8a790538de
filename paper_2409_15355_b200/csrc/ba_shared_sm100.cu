// Attention of a batch whose sequences share prefixes, over a paged cache (the steps after a prompt).
//
// Work.  An entry is a prefix with the query rows of its whole group, or a sequence's own rows with its queries.  The rows of an entry
// are (token, head of a KV group) pairs; its keys come in tiles of 128.  Entries are of two kinds, by their rows:
//   few  (at most 16): a key is used by few rows, the bytes of the cache are all that counts.  An item is entry x KV head.
//   many (more): a matrix product.  An item is entry x KV head x 256 rows (two tiles of 128), for the tensor core.
// The key tiles of all items of a kind, laid end to end (an item begins with a few units that stand for what it costs besides them), are
// a stream that is cut into equal runs, one per CTA; the CTAs are shared out
// among the two streams by their cost.  So one long sequence, many short ones and a prefix of 32K keep every SM equally long.
// An item that a cut divides leaves partial results (normalised rows and their log-sum-exp), in the rows of its queries for its first
// piece and in a place of the CTA for the others (a run starts with one such piece at most); a second kernel merges them, prefix
// and own rows alike.  An item of few rows that is whole, of a sequence without prefix, is written straight to the output.  The streams are
// laid out on the device from the caller's tables by every CTA for itself: the lengths of a captured launch change from replay to replay.
//
// A CTA has 384 threads, one CTA runs on an SM.
// Few rows: warps 8 and 9 ask the copy engine for key and value tiles (a ring of stages for both, one box per page); warps 0-7 take 16 keys of a tile
// each, with mma.sync on operands from shared memory: S = Q K^T, softmax with maxima and sums of the warp's own keys, O += P V with P from
// registers.  The warps share nothing until the end of a piece, where their maxima, sums and accumulators are merged.
// Many rows: tcgen05 with accumulators in tensor memory, warps 0-3 and 4-7 softmax (a thread a row), warps 8 and 10 copy keys
// (and queries) and values, warp 9 issues the products (a thread for each softmax group: their products get into one another's way, 24 questions
// over 16384 tokens 308 -> 329 us).  Items of more than 128 rows: the two softmax groups have a tile of queries each and share key
// tiles; items of fewer: they share the query tile and take key tiles in turn, each with an accumulator of its own, so that products and
// exponentials overlap there too; the merge counts them as two results.
//
// Measured, 32 heads over 8 KV heads of 128: 64 sequences of 1500-7000 rows of their own 160 us of kernel for 161 of the bytes at a copy's rate;
// 16 sequences of one token over a prefix of 32000 keys 36 us (20 of them the prefix's bytes); 24 questions of 17-64 tokens over 16384 keys 280 us,
// 50 % of the tensor pipe: a pair of tiles takes 3270 cycles, its products 2100, the chain from scores over softmax to scores is what is left.
//
// A score that is NaN or +infinity leaves a NaN in its row's sum (the maximum does not show it), as in the formula.  So a sum of zero is what
// marks a row that saw no key; any other is divided by, and a NaN goes through to o and lse whatever the cuts.
//
// Rounding: P to bf16 (the products' type; 2^-8 relative at most, the sums of the softmax are taken before it), o once at the end.
#include <algorithm>

#include "ba_common.cuh"
#include "ba_sm100.cuh"

using namespace sm100;

bool ba_tensor_map(ba_ctx *ctx, CUtensorMap *out, const void *ptr, int heads, long long rows, int box_heads, int box_rows);

namespace {

constexpr int kTile = 128;            // keys per tile
constexpr int kRows = 16;             // most rows of an entry of few: one tile of mma.sync
constexpr int kManyRows = 256;        // rows of an item of many
constexpr int kWarps = 8;             // consumer warps
constexpr int kThreads = 32 * kWarps + 128;
// Registers after launch (168 a thread): 256 * 224 + 128 * 56 = 384 * 168.  A thread keeps 64 accumulators and 32 words of queries.
constexpr int kConsumerRegs = 224, kCopyRegs = 56;
constexpr int kMaxEntries = BA_SHARED_MAX;
constexpr int kSoftmaxRegs = 208, kServiceRegs = 88;     // of CTAs for many rows: 256 * 208 + 128 * 88
// Units of the streams.  A key tile counts for one in the stream of few rows and, in the other, for three with two query tiles and two with
// one; an item counts besides for what begins and ends it (queries, the pipeline's filling, the rows' way out).  Measured, us: few rows' 1, 4, 8
// units: 16 requests over 32000 tokens 61.7, 49.1, 48.7, 160 requests in seven groups 200, 192, 211, 64 apart 180, 177, 181; many rows' 3, 10, 20:
// 24 questions over 16384 tokens 451, 308, 312, the seven groups 197, 192, 193.
constexpr int kTileFew = 1, kTilePair = 3, kTileSolo = 2, kFrontFew = 4, kFrontMany = 10;
// What a unit costs, to share out the CTAs between the streams.  2, 3, 4.5 for few rows against 2: the 16 requests 53.5, 49.1, 48.5 us, the seven
// groups 210, 192, 232, the others, of one kind nearly alone, the same.
constexpr float kCostFew = 3.f, kCostMany = 2.f;
constexpr long long kMostUnits = 2000000000;               // of a stream: places in it are 32 bits
constexpr float kRescale = 8.f;       // O is rescaled when a maximum grows by more than 2^8: exact in real arithmetic, values stay bounded

struct SharedParams {
  const __nv_bfloat16 *q;
  void *o;
  float *lse;
  int32_t *status;
  int out_f32, Hq, Hkv, G;
  int q_boxes;                        // 128 is a multiple of G: the copy engine fetches query tiles
  float scale_log2;
  int n_q_rows, batch, n_groups;
  const int32_t *group_cu, *prefix_cu, *q_cu, *own_len;
  int n_prefix_rows;                  // packed prefixes
  int prefix_paged;
  const int32_t *prefix_page_cu, *prefix_page_idx, *page_cu, *page_idx;
  int prefix_page_lg, page_lg, prefix_pages, n_pages;
  // partial results, normalised: [n_part][D] values, then [n_part] log-sum-exps.  First pieces of items: four arrays indexed as o (own
  // rows, prefixes, and the second softmax group's share of each); then kManyRows for every CTA.
  float *part;
  long long n_part;
  int4 *meta;                         // [n_groups + batch]: first unit in its stream, tiles, rows, many; then runs of the two kinds, CTAs for many, validity
};

constexpr int kCtrlBytes = 1360;

template <int D>
struct SharedLayout {
  static constexpr int kTileBytes = kTile * D * 2;
  static constexpr int kRegion = kTile * 128;
  // few rows
  static constexpr int kStages = D == 128 ? 5 : 10;
  static constexpr int kBufStride = 68;                                // floats a row: rows of a quad's lanes in different banks
  static constexpr int kBuf = kStages * kTileBytes;                    // [kWarps][16][kBufStride]
  static constexpr int kStat = kBuf + kWarps * 16 * kBufStride * 4;    // [kWarps][kRows] (maximum, sum)
  static constexpr int kFewEnd = kStat + kWarps * kRows * 8;
  // many rows: query tiles, key tiles, value tiles, write-out
  static constexpr int kDepth = D == 128 ? 2 : 4;                      // stages of keys, and of values
  static constexpr int kKeys = 2 * kTileBytes, kValues = kKeys + kDepth * kTileBytes;
  static constexpr int kOut = kValues + kDepth * kTileBytes;           // [kWarps][32 rows][16 columns]
  static constexpr int kManyEnd = kOut + kWarps * 32 * 16 * 4;
  static constexpr int kEnd = kFewEnd > kManyEnd ? kFewEnd : kManyEnd;
  static constexpr int kUnits = (kEnd + 15) / 16 * 16;                 // [2][kMaxEntries + 4]: units before an entry, by kind
  static constexpr int kCtrl = kUnits + 2 * (kMaxEntries + 4) * 4;
  static constexpr int kBytes = kCtrl + kCtrlBytes + 1024;
};
static_assert(SharedLayout<128>::kBytes <= 227 * 1024, "shared memory");

struct SharedCtrl {
  uint64_t full[10], empty[10];       // few: the ring
  uint64_t k_full[5], k_empty[5], v_full[4], v_empty[4];                       // many
  uint64_t q_full, q_empty, s_full[2], p_full[2][2], o_done[2], o_free[2];
  int abort_flag, invalid;
  uint32_t tmem_base;
  uint32_t prefixed[kMaxEntries / 32];         // a bit a sequence: it has a prefix
  uint32_t pairs[kMaxEntries / 32];   // a bit an entry: it has items of more than 128 rows
  longlong2 warp_sums[kThreads / 32]; // units of few rows, of many
};
static_assert(sizeof(SharedCtrl) <= kCtrlBytes, "control area");

// Tables and queries may come from the kernel before (ba_segment, ba_append_paged), beside which this one is launched: plain loads throughout, as the
// read-only path wants data that nobody writes in a kernel's lifetime.
// An entry, looked up by the thread that asks: rows q_row0 .. of the queries, `len` keys.
struct Entry { int q_row0, rows, len; };
__device__ __forceinline__ int q_begin(const SharedParams &p, int s) { return p.q_cu ? p.q_cu[s] : s; }
__device__ __forceinline__ Entry get_entry(const SharedParams &p, int e) {
  Entry x;
  if (e < p.n_groups) {
    const int a = p.group_cu ? p.group_cu[e] : 0, b = p.group_cu ? p.group_cu[e + 1] : p.batch;
    x.q_row0 = q_begin(p, a); x.rows = q_begin(p, b) - x.q_row0;
    x.len = p.prefix_cu[e + 1] - p.prefix_cu[e];
  } else {
    const int s = e - p.n_groups;
    x.q_row0 = q_begin(p, s); x.rows = q_begin(p, s + 1) - x.q_row0;
    x.len = p.own_len[s];
  }
  return x;
}
// The same with its tables checked: false, and nothing read by their values, where they do not hold.
__device__ __forceinline__ bool load_entry(const SharedParams &p, int e, Entry &x) {
  x.q_row0 = x.rows = x.len = 0;
  int a, b;
  if (e < p.n_groups) {
    a = p.group_cu ? p.group_cu[e] : 0; b = p.group_cu ? p.group_cu[e + 1] : p.batch;
    const int r0 = p.prefix_cu[e], r1 = p.prefix_cu[e + 1], list = p.prefix_paged ? p.prefix_page_cu[e] : 0;
    const long long room = p.prefix_paged ? ((long long)p.prefix_page_cu[e + 1] - list) << p.prefix_page_lg : (long long)p.n_prefix_rows - r0;
    if (a < 0 || b < a || b > p.batch || r0 < 0 || r1 < r0 || list < 0 || r1 - r0 > room) return false;
    x.len = r1 - r0;
  } else {
    const int s = e - p.n_groups, len = p.own_len[s], list = p.page_cu[s];
    const long long room = ((long long)p.page_cu[s + 1] - list) << p.page_lg;
    if (len < 0 || list < 0 || len > room) return false;
    a = s; b = s + 1; x.len = len;
  }
  const int first = q_begin(p, a), last = q_begin(p, b);   // (their difference may not fit where they do not hold)
  if (first < 0 || last < first || last > p.n_q_rows || x.len > INT32_MAX - 2 * kTile) { x.len = 0; return false; }
  x.q_row0 = first; x.rows = last - first;
  return true;
}
__device__ __forceinline__ int tiles_of(const Entry &x) { return (x.len + kTile - 1) / kTile; }
__device__ __forceinline__ bool is_many(const SharedParams &p, const Entry &x) { return x.rows * p.G > kRows; }
// Units of a tile of an item of n rows.
__device__ __forceinline__ int tile_units(bool many, int n_rows) { return !many ? kTileFew : n_rows > 128 ? kTilePair : kTileSolo; }
// How an entry's items lie in its stream: head by head, row tile by row tile, each `front` units and those of its tiles.
struct Lay {
  int tiles, rts, front, full, last;   // row tiles; units of an item that is not a head's last one, and of one that is
  __device__ __forceinline__ Lay(int tiles_, int rows, bool many) : tiles(tiles_) {
    rts = many ? (rows + kManyRows - 1) / kManyRows : rows > 0;
    front = many ? kFrontMany : kFrontFew;
    full = front + tiles * tile_units(many, kManyRows);
    last = front + tiles * tile_units(many, rows - (rts - 1) * kManyRows);
  }
  __device__ __forceinline__ long long a_head() const { return tiles > 0 && rts > 0 ? (long long)(rts - 1) * full + last : 0; }
};
__device__ __forceinline__ Lay lay_of(const SharedParams &p, const Entry &x) { return Lay(tiles_of(x), x.rows * p.G, is_many(p, x)); }
// Rows of an item: row r is head h of token tok of its queries (tok x heads + h) from `at` on.
struct RowMap {
  long long at;         // of its first token and head, as o is indexed without the head's values
  int g0, G, Hq;
  float inv;
  __device__ __forceinline__ RowMap(const SharedParams &p, const Entry &x, int row0, int head) : G(p.G), Hq(p.Hq), inv(1.f / (float)p.G) {
    const int tok0 = row0 / p.G;
    g0 = row0 - tok0 * p.G;
    at = (long long)(x.q_row0 + tok0) * p.Hq + head * p.G;
  }
  // tokens from the first one to row r's (whole numbers below G + 256: exact)
  __device__ __forceinline__ int token(int r) const { return (int)(((float)(g0 + r) + 0.5f) * inv); }
  __device__ __forceinline__ long long row(int r) const { const int t = token(r); return at + (long long)t * Hq + (g0 + r - t * G); }
};
// First pieces leave their results at the rows of their queries: `which` 0 own rows, 1 a prefix, + 2 the second softmax group's; other pieces
// at their CTA's.
__device__ __forceinline__ long long first_part(const SharedParams &p, int which) { return (long long)which * p.n_q_rows * p.Hq; }
__device__ __forceinline__ long long cut_part(const SharedParams &p, int cta) { return 4ll * p.n_q_rows * p.Hq + (long long)cta * kManyRows; }

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
  while (lo < hi) { const int mid = (lo + hi) >> 1; if (p.group_cu[mid] <= s) lo = mid + 1; else hi = mid; }
  return lo - 1 < p.n_groups ? lo - 1 : -1;
}

// A piece of a stream: key tiles tile0 .. tile0 + n - 1 of an item, rows row0 .. row0 + n_rows - 1 of its entry.
struct Piece {
  int e, head, row0, n_rows, tile0, n, tiles, units;
  Entry x;
};
// The piece that starts at unit `at` of this CTA's run, which ends at `end`; units is where it stops.  n = 0: only units in front of the tiles.
__device__ __forceinline__ Piece piece_at(const SharedParams &p, const int *units, int n_entries, int at, int end) {
  Piece k;
  k.e = last_at_most(units, n_entries, at);
  k.x = get_entry(p, k.e);
  k.tiles = tiles_of(k.x);
  const Lay lay = lay_of(p, k.x);
  const int a_head = (int)lay.a_head(), local = at - units[k.e];
  k.head = local / a_head;
  const int in_head = local - k.head * a_head, rt = min(in_head / lay.full, lay.rts - 1), from = in_head - rt * lay.full;
  k.row0 = rt * kManyRows;
  k.n_rows = min(kManyRows, k.x.rows * p.G - k.row0);
  const int to = min(rt + 1 < lay.rts ? lay.full : lay.last, from + end - at), w = tile_units(is_many(p, k.x), k.n_rows);
  k.units = to - from;
  // tile t is worked on where its first unit lies
  k.tile0 = max(0, from - lay.front + w - 1) / w;
  k.n = max(0, to - lay.front + w - 1) / w - k.tile0;
  return k;
}
// Where the keys of a piece lie.  Lane i of the copying warp has box i of a tile, a box per page.
struct Source {
  const int32_t *idx;
  int lg, n_pages, sub_rows, list, first, len;
  bool paged;
};
__device__ __forceinline__ Source source_of(const SharedParams &p, const Piece &k) {
  const bool own = k.e >= p.n_groups;
  Source s;
  s.paged = own || p.prefix_paged;
  s.lg = own ? p.page_lg : p.prefix_page_lg; s.n_pages = own ? p.n_pages : p.prefix_pages;
  s.sub_rows = s.paged ? min(kTile, 1 << s.lg) : kTile;
  s.list = own ? p.page_cu[k.e - p.n_groups] : s.paged ? p.prefix_page_cu[k.e] : 0;
  s.idx = own ? p.page_idx : p.prefix_page_idx;
  s.first = s.paged ? 0 : p.prefix_cu[k.e];
  s.len = k.x.len;
  return s;
}
// First row of this lane's box of a tile; -1: it has none, or nothing lies there.
__device__ __forceinline__ int box_row(const SharedParams &p, const Source &s, int tile) {
  const int lane = threadIdx.x & 31, t = tile * kTile + lane * s.sub_rows;
  if (lane * s.sub_rows >= kTile || t >= s.len) return -1;
  if (!s.paged) return s.first + t;
  const int page = s.idx[s.list + (t >> s.lg)];
  if (page < 0 || page >= s.n_pages) {
    ba_record_status(p.status, BA_ERR_INVALID_ARG);
    return s.n_pages << s.lg;                              // behind the pool: the copy engine fills in zeros
  }
  return (page << s.lg) + (t & ((1 << s.lg) - 1));
}
// One tile into shared memory, by the whole copying warp.
template <int D>
__device__ __forceinline__ void copy_tile(const Source &s, const CUtensorMap *m, uint8_t *dst, uint64_t *bar, int head, int row) {
  const unsigned boxes = __popc(__ballot_sync(0xffffffffu, row >= 0));
  if ((threadIdx.x & 31) == 0) mbar_arrive_expect_tx(bar, boxes * s.sub_rows * D * 2);
  __syncwarp();
  if (row >= 0) {
    dst += (threadIdx.x & 31) * s.sub_rows * 128;
    for (int c = 0; c < D / 64; ++c) tma_load_3d(dst + c * SharedLayout<D>::kRegion, m, bar, c * 64, head, row);
  }
  __syncwarp();
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

// Queries of a piece of an item of few rows as the A operand, straight from memory (rows past the item's are zeros), and how many
// keys the lane's two rows see.
template <int D>
__device__ __forceinline__ void load_queries(const SharedParams &p, const Piece &k, uint32_t (&qa)[D / 16][4], int (&limit)[2]) {
  const int lane = threadIdx.x & 31, quad = lane >> 2, in_quad = lane & 3;
  const bool own = k.e >= p.n_groups;
  const RowMap map(p, k.x, 0, k.head);
#pragma unroll
  for (int hi = 0; hi < 2; ++hi) {
    const int r = hi * 8 + quad;
    const bool there = r < k.n_rows;
    const uint32_t *src = reinterpret_cast<const uint32_t *>(p.q + map.row(there ? r : 0) * D) + in_quad;
    limit[hi] = own ? k.x.len - (k.x.rows - 1 - map.token(there ? r : 0)) : k.x.len;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      qa[c][hi] = there ? src[c * 8] : 0u;
      qa[c][hi + 2] = there ? src[c * 8 + 4] : 0u;
    }
  }
}

// The pieces of a run of few rows, one by one: the consumer warps' view of it.
struct FewRun {
  const int *units;
  int n_entries, at, end;
  __device__ __forceinline__ bool next(const SharedParams &p, Piece &k) {
    while (at < end) {
      k = piece_at(p, units, n_entries, at, end);
      at += k.units;
      if (k.n > 0) return true;
    }
    return false;
  }
};

// The consumer warps' work on a run of few rows.
template <int D>
__device__ __forceinline__ void consume_run(const SharedParams &p, FewRun run, uint8_t *smem, SharedCtrl *ctrl) {
  using L = SharedLayout<D>;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quad = lane >> 2, in_quad = lane & 3;
  volatile int *abort_flag = &ctrl->abort_flag;
  int ring = 0;
  bool ok = true;
  uint32_t qa[D / 16][4];
  int limit[2];
  Piece k;
  bool more = run.next(p, k);
  if (more) load_queries<D>(p, k, qa, limit);
  while (more) {                         // (to the end even after a wait that expired: the warps meet at barriers)
    const bool own = k.e >= p.n_groups;
    const bool direct = own && k.n == k.tiles && !(ctrl->prefixed[(k.e - p.n_groups) >> 5] >> ((k.e - p.n_groups) & 31) & 1);
    const int n_rows = k.n_rows;
    float o[D / 8][4], mx[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < D / 8; ++c) o[c][0] = o[c][1] = o[c][2] = o[c][3] = 0.f;
    const float sl = p.scale_log2;
    const int k_row = warp * 16 + ((lane >> 4) & 1) * 8 + (lane & 7), k_col = (lane >> 3) & 1;
    const int v_row = warp * 16 + ((lane >> 3) & 1) * 8 + (lane & 7), v_col = (lane >> 4) & 1;
    for (int j = 0; j < k.n; ++j, ring += 2) {
      const int key0 = (k.tile0 + j) * kTile + warp * 16;    // this warp's keys
      const int left = k.x.len - key0;
      const int ks = ring % L::kStages, vs = (ring + 1) % L::kStages;
      if (ok) ok = mbar_wait(&ctrl->full[ks], (ring / L::kStages) & 1, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
      if (ok && left > 0) {
        const uint32_t tile = smem_u32(smem + ks * L::kTileBytes) + k_row * 128;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
          uint32_t b[4];
          const int col = c * 2 + k_col;
          ldsm4(b, tile + (col >> 3) * L::kRegion + (((col & 7) ^ (k_row & 7)) << 4));
          mma_16816(s[0], qa[c], b[0], b[1]);
          mma_16816(s[1], qa[c], b[2], b[3]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctrl->empty[ks]);
      uint32_t pa[4];
      if (ok && left > 0) {
        float top[2];
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
          if (key0 + 16 > limit[hi]) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (key0 + (i >> 1) * 8 + in_quad * 2 + (i & 1) >= limit[hi]) s[i >> 1][hi * 2 + (i & 1)] = -INFINITY;
          }
          top[hi] = fmaxf(fmaxf(s[0][hi * 2], s[0][hi * 2 + 1]), fmaxf(s[1][hi * 2], s[1][hi * 2 + 1]));
          top[hi] = fmaxf(top[hi], __shfl_xor_sync(0xffffffffu, top[hi], 1));
          top[hi] = fmaxf(top[hi], __shfl_xor_sync(0xffffffffu, top[hi], 2));
          top[hi] = fmaxf(top[hi], mx[hi]);
        }
        // (from -inf: yes, unless nothing has been seen yet)
        const bool grow = (top[0] > mx[0] && !((top[0] - mx[0]) * sl <= kRescale)) || (top[1] > mx[1] && !((top[1] - mx[1]) * sl <= kRescale));
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
          for (int hi = 0; hi < 2; ++hi) {
            const float alpha = mx[hi] == -INFINITY ? 0.f : ex2((mx[hi] - top[hi]) * sl);     // (nothing summed so far)
            mx[hi] = top[hi];
            sum[hi] *= alpha;
#pragma unroll
            for (int c = 0; c < D / 8; ++c) { o[c][hi * 2] *= alpha; o[c][hi * 2 + 1] *= alpha; }
          }
        }
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
          const float neg = mx[hi] == -INFINITY ? 0.f : -mx[hi] * sl;
          float e[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) e[i] = ex2(fmaf(s[i >> 1][hi * 2 + (i & 1)], sl, neg));
          sum[hi] += (e[0] + e[1]) + (e[2] + e[3]);
          pa[hi] = pack_bf16(e[0], e[1]);
          pa[hi + 2] = pack_bf16(e[2], e[3]);
        }
      }
      if (ok) ok = mbar_wait(&ctrl->full[vs], ((ring + 1) / L::kStages) & 1, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
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
          mma_16816(o[2 * c], pa, b[0], b[1]);
          mma_16816(o[2 * c + 1], pa, b[2], b[3]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctrl->empty[vs]);
    }
    // the next piece's queries are on their way while this one is finished
    const Piece done = k;
    more = run.next(p, k);
    if (more) load_queries<D>(p, k, qa, limit);
    // The warps' results: rows' maxima and sums are exchanged, every accumulator is scaled to the common maximum and divided by the
    // common sum, and the eight are added 64 columns at a time.
    const RowMap map(p, done.x, 0, done.head);
    float2 *stat = reinterpret_cast<float2 *>(smem + L::kStat);
    float *buf = reinterpret_cast<float *>(smem + L::kBuf);
#pragma unroll
    for (int hi = 0; hi < 2; ++hi) {
      sum[hi] += __shfl_xor_sync(0xffffffffu, sum[hi], 1);
      sum[hi] += __shfl_xor_sync(0xffffffffu, sum[hi], 2);
      if (in_quad == 0) stat[warp * kRows + hi * 8 + quad] = make_float2(mx[hi], sum[hi]);
    }
    consumers_sync();
    // a row's place: in the output, among the first pieces, or in the CTA's own
    auto place = [&](int r) -> long long {
      return direct ? map.row(r) : done.tile0 == 0 ? first_part(p, own ? 0 : 1) + map.row(r) : cut_part(p, (int)blockIdx.x) + r;
    };
    float f[2];
#pragma unroll
    for (int hi = 0; hi < 2; ++hi) {
      const int r = hi * 8 + quad;
      float top = -INFINITY, den = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, stat[w * kRows + r].x);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float2 v = stat[w * kRows + r];
        if (v.y != 0.f) den += v.y * ex2((v.x - top) * sl);
      }
      f[hi] = sum[hi] != 0.f ? ex2((mx[hi] - top) * sl) / den : 0.f;
      if (ok && warp == 0 && in_quad == 0 && r < n_rows) {
        const float lse = den != 0.f ? (top * sl + log2f(den)) * 0.6931471805599453f : -INFINITY;
        if (!direct) p.part[p.n_part * D + place(r)] = lse;
        else if (p.lse) p.lse[place(r)] = lse;
      }
    }
    // up to eight rows: the buffer's other eight rows take the other 64 columns, and one round does
    const bool compact = n_rows <= 8;
    float *mine = buf + warp * 16 * L::kBufStride;
    const int r16 = threadIdx.x >> 4, col = (threadIdx.x & 15) * 4;
#pragma unroll
    for (int half = 0; half < D / 64; ++half) {
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        *reinterpret_cast<float2 *>(mine + ((compact ? half * 8 : 0) + quad) * L::kBufStride + c * 8 + in_quad * 2) =
            make_float2(o[half * 8 + c][0] * f[0], o[half * 8 + c][1] * f[0]);
        if (!compact)
          *reinterpret_cast<float2 *>(mine + (8 + quad) * L::kBufStride + c * 8 + in_quad * 2) =
              make_float2(o[half * 8 + c][2] * f[1], o[half * 8 + c][3] * f[1]);
      }
      if (compact && half + 1 < D / 64) continue;
      consumers_sync();
      const int r = compact ? r16 & 7 : r16, h = compact ? r16 >> 3 : half;
      if (ok && r < n_rows && h < D / 64) {
        float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float4 v = *reinterpret_cast<const float4 *>(buf + (w * 16 + r16) * L::kBufStride + col);
          t.x += v.x; t.y += v.y; t.z += v.z; t.w += v.w;
        }
        const long long at = place(r) * D + h * 64 + col;
        if (!direct) *reinterpret_cast<float4 *>(p.part + at) = t;
        else if (p.out_f32) *reinterpret_cast<float4 *>(reinterpret_cast<float *>(p.o) + at) = t;
        else *reinterpret_cast<uint2 *>(reinterpret_cast<__nv_bfloat16 *>(p.o) + at) = make_uint2(pack_bf16(t.x, t.y), pack_bf16(t.z, t.w));
      }
      consumers_sync();
    }
  }
}

// A CTA for few rows: units [begin, end) of that stream.
template <int D>
__device__ __forceinline__ void few_rows(const SharedParams &p, const CUtensorMap *tmap_kx, const CUtensorMap *tmap_vx, const CUtensorMap *tmap_k,
                                         const CUtensorMap *tmap_v, uint8_t *smem, SharedCtrl *ctrl, const int *units, int n_entries, int begin, int end) {
  using L = SharedLayout<D>;
  const int warp = threadIdx.x >> 5;
  int ring = 0;
  bool ok = true;
  if (warp >= kWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kCopyRegs));
    if (warp < kWarps + 2) {
      const int kv = warp - kWarps;                        // keys and values are asked for by a warp each: a tile is up to 16 boxes
      ring = kv;
      for (int at = begin; at < end && ok;) {
        const Piece k = piece_at(p, units, n_entries, at, end);
        at += k.units;
        if (k.n == 0) continue;
        const bool own = k.e >= p.n_groups;
        const Source src = source_of(p, k);
        int next = box_row(p, src, k.tile0);               // (looked up a tile ahead)
        for (int j = 0; j < k.n && ok; ++j) {
          const int row = next;
          if (j + 1 < k.n) next = box_row(p, src, k.tile0 + j + 1);
          const int stage = ring % L::kStages;
          ok = __all_sync(0xffffffffu, mbar_wait(&ctrl->empty[stage], ((ring / L::kStages) & 1) ^ 1, &ctrl->abort_flag));
          if (!ok) break;
          copy_tile<D>(src, own ? (kv ? tmap_v : tmap_k) : (kv ? tmap_vx : tmap_kx), smem + stage * L::kTileBytes, &ctrl->full[stage], k.head, row);
          ring += 2;
        }
      }
      if (!ok) {
        // leave no copy in flight: wait (bounded) for the tiles already requested
        for (int i = max(kv, ring - 2 * ((L::kStages + 1) / 2)); i < ring; i += 2)
          for (uint32_t spin = 0; spin < (1u << 20); ++spin)
            if (mbar_try_wait(&ctrl->full[i % L::kStages], (i / L::kStages) & 1)) break;
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kConsumerRegs));
    consume_run<D>(p, {units, n_entries, begin, end}, smem, ctrl);
  }
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ void copy_16_or_zero(uint32_t dst, const void *src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}

// The ring of key tiles of a CTA for many rows.  The second query tile's place is one more stage where the run has no pairs: a stage is
// refilled once its product is done and needed one softmax later, which HBM under load outlasts (160 requests in seven groups: the CTAs for
// many rows waited 1500 of 6500 cycles for keys).
template <int D>
struct KeyRing {
  using L = SharedLayout<D>;
  bool deep;
  __device__ __forceinline__ int stage(int i) const { return deep ? i % (L::kDepth + 1) : i % L::kDepth; }
  __device__ __forceinline__ int phase(int i) const { return (deep ? i / (L::kDepth + 1) : i / L::kDepth) & 1; }
  __device__ __forceinline__ int depth() const { return L::kDepth + (deep ? 1 : 0); }
  static __device__ __forceinline__ int offset(int stage) { return stage < L::kDepth ? L::kKeys + stage * L::kTileBytes : L::kTileBytes; }
};

// A CTA for many rows: units [begin, end) of that stream.  Softmax group t has, of the n key tiles of a piece, all (a piece of more
// than 128 rows: pair) or t, t + 2, ..
template <int D>
__device__ __forceinline__ void many_rows(const SharedParams &p, const CUtensorMap *tmap_kx, const CUtensorMap *tmap_vx, const CUtensorMap *tmap_k,
                                          const CUtensorMap *tmap_v, const CUtensorMap *tmap_q, uint8_t *smem, SharedCtrl *ctrl, const int *units,
                                         int n_entries, int begin, int end) {
  using L = SharedLayout<D>;
  constexpr int kDepth = L::kDepth;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t tmem = ctrl->tmem_base;
  volatile int *abort_flag = &ctrl->abort_flag;
  uint64_t *k_full = ctrl->k_full, *v_full = ctrl->v_full, *k_empty = ctrl->k_empty, *v_empty = ctrl->v_empty;
  bool ok = true, any_pair = false;
  for (int e = last_at_most(units, n_entries, begin), last = last_at_most(units, n_entries, end - 1); e <= last; ++e)
    any_pair = any_pair || (ctrl->pairs[e >> 5] >> (e & 31) & 1);
  const KeyRing<D> keys = {!any_pair};
  if (warp == 8) {
    // ------------------------------------------------------------ copies of queries and keys
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kServiceRegs));
    int nk = 0, n_pieces = 0, n_q = 0;                     // key tiles requested, pieces begun; pieces whose queries the copy engine fetches
    for (int at = begin; at < end && ok;) {
      const Piece k = piece_at(p, units, n_entries, at, end);
      at += k.units;
      if (k.n == 0) continue;
      // the queries, once the piece before has no use for their place
      auto load_queries = [&]() -> bool {
        if (!__all_sync(0xffffffffu, mbar_wait(&ctrl->q_empty, (n_pieces & 1) ^ 1, abort_flag))) return false;
        ++n_pieces;
        const int tile_rows = k.n_rows > 128 ? 256 : 128;
        if (p.q_boxes) {                                   // the heads of a group divide a tile: boxes of whole tokens
          if (lane == 0) {
            mbar_arrive_expect_tx(&ctrl->q_full, tile_rows * D * 2);
            for (int t = 0; t * 128 < tile_rows; ++t)
              for (int c = 0; c < D / 64; ++c)
                tma_load_3d(smem + t * L::kTileBytes + c * L::kRegion, tmap_q, &ctrl->q_full, c * 64, k.head * p.G, k.x.q_row0 + (k.row0 + t * 128) / p.G);
          }
          n_q = n_pieces;
        } else {                                           // 16 bytes a copy, into the tiles' swizzled layout
          constexpr int kVecs = D / 8;
          const int c = lane % kVecs;
          const RowMap map(p, k.x, k.row0, k.head);
          const uint32_t base = smem_u32(smem) + (c >> 3) * L::kRegion;
#pragma unroll 8
          for (int r = lane / kVecs; r < tile_rows; r += 32 / kVecs) {
            const bool there = r < k.n_rows;               // (rows that are not there are zeros)
            copy_16_or_zero(base + (r >> 7) * L::kTileBytes + (r & 127) * 128 + (((c & 7) ^ (r & 7)) << 4), p.q + map.row(there ? r : 0) * D + c * 8, there);
          }
          asm volatile("cp.async.wait_all;" ::: "memory");
          fence_proxy_async();                             // the tensor core reads through the async proxy
          __syncwarp();
          if (lane == 0) mbar_arrive(&ctrl->q_full);
        }
        __syncwarp();
        return true;
      };
      const Source src = source_of(p, k);
      int next = box_row(p, src, k.tile0);                 // (looked up a tile ahead)
      for (int j = 0; j < k.n; ++j, ++nk) {
        const int row = next, st = keys.stage(nk);
        if (j + 1 < k.n) next = box_row(p, src, k.tile0 + j + 1);
        ok = __all_sync(0xffffffffu, mbar_wait(&k_empty[st], keys.phase(nk) ^ 1, abort_flag));
        if (!ok) break;
        copy_tile<D>(src, k.e >= p.n_groups ? tmap_k : tmap_kx, smem + KeyRing<D>::offset(st), &k_full[st], k.head, row);
        if (j == 0) ok = load_queries();                   // (behind the first keys, whose place is free sooner)
        if (!ok) { ++nk; break; }
      }
    }
    if (!ok) {
      // leave no copy in flight: wait (bounded) for what was requested
      for (int i = max(0, nk - keys.depth()); i < nk; ++i)
        for (uint32_t spin = 0; spin < (1u << 20); ++spin)
          if (mbar_try_wait(&k_full[keys.stage(i)], keys.phase(i))) break;
      if (n_q > 0)
        for (uint32_t spin = 0; spin < (1u << 20); ++spin)
          if (mbar_try_wait(&ctrl->q_full, (n_q - 1) & 1)) break;
    }
  } else if (warp == 9) {
    // ------------------------------------------------------------ products
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kServiceRegs));
    if (elect_one()) {
      constexpr uint32_t idesc_qk = make_idesc_bf16(128, kTile, 0), idesc_pv = make_idesc_bf16(128, D, 1);
      const uint64_t q_desc = make_smem_desc(smem_u32(smem), 16, 1024);
      const uint64_t v_desc = make_smem_desc(smem_u32(smem + L::kValues), L::kRegion, 1024);
      int nk = 0, nv = 0, n_pieces = 0;                    // tiles of all earlier pieces; pieces
      int p_uses[2] = {0, 0}, o_uses[2] = {0, 0};
      for (int at = begin; at < end && ok;) {
        const Piece k = piece_at(p, units, n_entries, at, end);
        at += k.units;
        if (k.n == 0) continue;
        const bool pair = k.n_rows > 128;
        const int n = k.n, step = pair ? 1 : 2;
        auto wait_k = [&](int j) { return mbar_wait(&k_full[keys.stage(nk + j)], keys.phase(nk + j), abort_flag); };
        auto wait_v = [&](int j) { return mbar_wait(&v_full[(nv + j) % kDepth], ((nv + j) / kDepth) & 1, abort_flag); };
        auto issue_qk = [&](int t, int j) {
          const uint64_t qd = q_desc + (uint64_t)((pair && t ? L::kTileBytes : 0) >> 4);
          const int st = keys.stage(nk + j);
          const uint64_t kd = q_desc + (uint64_t)(KeyRing<D>::offset(st) >> 4);
#pragma unroll
          for (int c = 0; c < D / 16; ++c) {
            const uint64_t off = (uint64_t)(((c >> 2) * L::kRegion + (c & 3) * 32) >> 4);
            mma_ss(tmem + t * 128, qd + off, kd + off, idesc_qk, c > 0);
          }
          mma_commit(&ctrl->s_full[t]);
          if (!pair || t) mma_commit(&k_empty[st]);
          if (j + 1 == n && (!pair || t)) mma_commit(&ctrl->q_empty);         // that was the piece's last product with the queries
        };
        auto issue_pv = [&](int t, int j, bool first, int half) {
          const uint64_t vd = v_desc + (uint64_t)((((nv + j) % kDepth) * L::kTileBytes) >> 4);
#pragma unroll
          for (int c = half * 4; c < half * 4 + 4; ++c)
            mma_ts(tmem + 256 + t * 128, tmem + t * 128 + c * 8, vd + (uint64_t)((c * 2048) >> 4), idesc_pv, (!first || c > 0) ? 1u : 0u);
        };
        ok = mbar_wait(&ctrl->q_full, n_pieces & 1, abort_flag);
        ++n_pieces;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int j = pair ? 0 : t;
          if (!ok || j >= n) continue;
          if (!pair || t == 0) ok = wait_k(j);
          if (!ok) continue;
          tc_fence_after();
          issue_qk(t, j);
        }
        for (int i = 0; ok && i * step < n; ++i) {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const int j = pair ? i : 2 * i + t, jn = j + step;
            if (!ok || j >= n) continue;
            const bool last = jn >= n;
            if (!pair || t == 0) ok = wait_v(j);           // (a wait costs this thread some 220 cycles: none twice)
            // the first product of a piece overwrites O_t: the rows before it must have been read out
            if (ok && i == 0) ok = mbar_wait(&ctrl->o_free[t], (o_uses[t] & 1) ^ 1, abort_flag);
            if (ok) ok = mbar_wait(&ctrl->p_full[t][0], p_uses[t] & 1, abort_flag);
            if (!ok) continue;
            tc_fence_after();
            issue_pv(t, j, i == 0, 0);
            if (!last && (!pair || t == 0)) ok = wait_k(jn);                   // (needed right after; off the critical path here)
            if (ok) ok = mbar_wait(&ctrl->p_full[t][1], p_uses[t] & 1, abort_flag);
            if (!ok) continue;
            tc_fence_after();
            issue_pv(t, j, false, 1);
            ++p_uses[t];
            if (last) { mma_commit(&ctrl->o_done[t]); ++o_uses[t]; }
            if (!pair || t) mma_commit(&v_empty[(nv + j) % kDepth]);
            if (!last) issue_qk(t, jn);
          }
        }
        nk += n; nv += n;
      }
    }
  } else if (warp == 10) {
    // ------------------------------------------------------------ copies of values
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kServiceRegs));
    int nv = 0;
    for (int at = begin; at < end && ok;) {
      const Piece k = piece_at(p, units, n_entries, at, end);
      at += k.units;
      if (k.n == 0) continue;
      const Source src = source_of(p, k);
      int next = box_row(p, src, k.tile0);
      for (int j = 0; j < k.n; ++j, ++nv) {
        const int row = next, st = nv % kDepth;
        if (j + 1 < k.n) next = box_row(p, src, k.tile0 + j + 1);
        ok = __all_sync(0xffffffffu, mbar_wait(&v_empty[st], ((nv / kDepth) & 1) ^ 1, abort_flag));
        if (!ok) break;
        copy_tile<D>(src, k.e >= p.n_groups ? tmap_v : tmap_vx, smem + L::kValues + st * L::kTileBytes, &v_full[st], k.head, row);
      }
    }
    if (!ok) {
      for (int i = max(0, nv - kDepth); i < nv; ++i)
        for (uint32_t spin = 0; spin < (1u << 20); ++spin)
          if (mbar_try_wait(&v_full[i % kDepth], (i / kDepth) & 1)) break;
    }
  } else if (warp == 11) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kServiceRegs));
  } else {
    // ------------------------------------------------------------ softmax, a thread a row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    const int t = warp >> 2, r = threadIdx.x & 127;
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + t * 128 + lane_off, tO = tmem + 256 + t * 128 + lane_off;
    const float sl = p.scale_log2;
    int s_uses = 0, o_uses = 0, nv = 0;
    for (int at = begin; at < end && ok;) {
      const Piece k = piece_at(p, units, n_entries, at, end);
      at += k.units;
      if (k.n == 0) continue;
      const bool pair = k.n_rows > 128, own = k.e >= p.n_groups;
      const int step = pair ? 1 : 2, row = pair ? t * 128 + r : r;             // of the item
      const int limit = own ? k.x.len - (k.x.rows - 1 - min(k.x.rows - 1, (k.row0 + row) / p.G)) : k.x.len;
      float m_used = -INFINITY, l = 0.f;
      const int j0 = pair ? 0 : t;
      for (int j = j0; j < k.n; j += step) {
        ok = __all_sync(0xffffffffu, mbar_wait(&ctrl->s_full[t], s_uses & 1, abort_flag));
        if (!ok) break;
        ++s_uses;
        tc_fence_after();
        const int key0 = (k.tile0 + j) * kTile, lim = limit - key0;            // columns 0 .. lim - 1 are seen
        uint32_t s[128];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld_32x32b_x32(tS + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&s[c * 32]));
        tmem_wait_ld();
        if (lim < 128) {
#pragma unroll
          for (int c = 0; c < 128; ++c)
            if (c >= lim) s[c] = 0xff800000u;                                  // -inf
        }
        const float *sf = reinterpret_cast<const float *>(s);
        float l1[43], l2[15], l3[5];
#pragma unroll
        for (int i = 0; i < 43; ++i) l1[i] = 3 * i + 2 < 128 ? max3(sf[3 * i], sf[3 * i + 1], sf[3 * i + 2]) : fmaxf(sf[126], sf[127]);
#pragma unroll
        for (int i = 0; i < 15; ++i) l2[i] = 3 * i + 2 < 43 ? max3(l1[3 * i], l1[3 * i + 1], l1[3 * i + 2]) : l1[42];
#pragma unroll
        for (int i = 0; i < 5; ++i) l3[i] = max3(l2[3 * i], l2[3 * i + 1], l2[3 * i + 2]);
        const float m_new = fmaxf(m_used, fmaxf(max3(l3[0], l3[1], l3[2]), fmaxf(l3[3], l3[4])));
        if (j == j0) {
          m_used = m_new;
        } else {
          // (from -inf: yes; rows that are not the item's have no say, so that results do not depend on what lies there)
          const bool grow = row < k.n_rows && (m_new - m_used) * sl > kRescale;
          if (__any_sync(0xffffffffu, grow)) {
            // 1 when this row's maximum did not move (also when the row has seen no key yet)
            const float alpha = (m_new == -INFINITY) ? 1.f : ex2((m_used - m_new) * sl);
            m_used = m_new;
            l *= alpha;
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
              uint32_t o[32];
              tmem_ld_32x32b_x32(tO + c * 32, o);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
              tmem_st_32x32b_x32(tO + c * 32, o);
            }
          }
        }
        const float neg_m = (m_used == -INFINITY) ? 0.f : -m_used * sl;        // no key seen so far: every p is 0
        const uint64_t sl2 = pack2(sl, sl), negm2 = pack2(neg_m, neg_m);
        uint64_t sum2[4] = {0ull, 0ull, 0ull, 0ull};
        // P is handed over in two halves, so that the product starts on the first 64 keys while the others are exponentiated
        uint32_t pk[32], pk1[32];
        auto expo = [&](int e0, uint32_t &dst, int i) {
          const uint64_t x2 = fma2(pack2(__uint_as_float(s[e0]), __uint_as_float(s[e0 + 1])), sl2, negm2);
          float x0, x1;
          unpack2(x2, x0, x1);
          const float p0 = ex2(x0), p1 = ex2(x1);
          sum2[i & 3] = add2(sum2[i & 3], pack2(p0, p1));
          dst = pack_bf16(p0, p1);
        };
#pragma unroll
        for (int i = 0; i < 32; ++i) expo(2 * i, pk[i], i);
        tmem_st_32x32b_x32(tS, pk);
#pragma unroll
        for (int i = 0; i < 16; ++i) expo(64 + 2 * i, pk1[i], i);
        const int valid = k.x.len - key0;
        if (valid < kTile) {
          // values behind the end may be anything, and zero times a NaN is a NaN: zeros there, before the product may start.  (These
          // scores were issued after the products with what lay in that stage before, so that the barrier's phase is the one meant.)
          const int jv = nv + j;
          ok = __all_sync(0xffffffffu, mbar_wait(&v_full[jv % kDepth], (jv / kDepth) & 1, abort_flag));
          if (!ok) break;
          uint8_t *tile = smem + L::kValues + (jv % kDepth) * L::kTileBytes;
          for (int i = r; i < (kTile - valid) * (D / 8); i += 128) {
            const int vr = valid + i / (D / 8), c = i % (D / 8);
            *reinterpret_cast<uint4 *>(tile + (c >> 3) * L::kRegion + vr * 128 + ((c & 7) << 4)) = make_uint4(0, 0, 0, 0);
          }
          fence_proxy_async();
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&ctrl->p_full[t][0]);
#pragma unroll
        for (int i = 16; i < 32; ++i) expo(64 + 2 * i, pk1[i], i);
        tmem_st_32x32b_x32(tS + 32, pk1);
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&ctrl->p_full[t][1]);
        float sum[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack2(sum2[i], sum[2 * i], sum[2 * i + 1]);
        l += ((sum[0] + sum[1]) + (sum[2] + sum[3])) + ((sum[4] + sum[5]) + (sum[6] + sum[7]));
      }
      nv += k.n;
      if (!ok) break;
      // The rows leave through shared memory, 16 columns at a time, so that a store writes 64 bytes of each of eight rows.
      const RowMap map(p, k.x, k.row0, k.head);
      const long long base = k.tile0 == 0 ? first_part(p, (own ? 0 : 1) + (pair ? 0 : 2 * t)) : cut_part(p, (int)blockIdx.x) + (pair ? 0 : t * 128);
      auto place = [&](int rr) { return base + (k.tile0 == 0 ? map.row(rr) : rr); };
      const float lse = l != 0.f ? (m_used * sl + log2f(l)) * 0.6931471805599453f : -INFINITY;
      if (row < k.n_rows) p.part[p.n_part * D + place(row)] = lse;
      if (j0 >= k.n) continue;                             // (no tile for this group)
      const float inv = l != 0.f ? 1.f / l : 0.f;
      ok = __all_sync(0xffffffffu, mbar_wait(&ctrl->o_done[t], o_uses & 1, abort_flag));
      ++o_uses;
      if (!ok) break;
      tc_fence_after();
      float *stage = reinterpret_cast<float *>(smem + L::kOut) + warp * 32 * 16;
      float *dst[4];                                       // of the lane's rows of the warp's 32
#pragma unroll
      for (int it = 0; it < 4; ++it) {
        const int rr = row - lane + it * 8 + (lane >> 2);
        dst[it] = rr < k.n_rows ? p.part + place(rr) * D + (lane & 3) * 4 : nullptr;
      }
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c) {
        uint32_t o[32];
        tmem_ld_32x32b_x32(tO + c * 32, o);
        tmem_wait_ld();
        if (c + 1 == D / 32) { tc_fence_before(); mbar_arrive(&ctrl->o_free[t]); }     // O_t has been read out
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
          for (int v = 0; v < 4; ++v)
            *reinterpret_cast<float4 *>(stage + lane * 16 + ((v ^ ((lane >> 1) & 3)) << 2)) =
                make_float4(__uint_as_float(o[half * 16 + v * 4]) * inv, __uint_as_float(o[half * 16 + v * 4 + 1]) * inv,
                            __uint_as_float(o[half * 16 + v * 4 + 2]) * inv, __uint_as_float(o[half * 16 + v * 4 + 3]) * inv);
          __syncwarp();
#pragma unroll
          for (int it = 0; it < 4; ++it) {
            const int rr = it * 8 + (lane >> 2), v = lane & 3;
            if (dst[it]) *reinterpret_cast<float4 *>(dst[it] + c * 32 + half * 16) = *reinterpret_cast<const float4 *>(stage + rr * 16 + ((v ^ ((rr >> 1) & 3)) << 2));
          }
          __syncwarp();
        }
      }
    }
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
ba_shared_attend_kernel(const __grid_constant__ CUtensorMap tmap_kx, const __grid_constant__ CUtensorMap tmap_vx,
                        const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                        const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ SharedParams p) {
  using L = SharedLayout<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  SharedCtrl *ctrl = reinterpret_cast<SharedCtrl *>(smem + L::kCtrl);
  int *units = reinterpret_cast<int *>(smem + L::kUnits);  // of entries of few rows; those of many behind them
  int *units_many = units + kMaxEntries + 4;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_entries = p.n_groups + p.batch, n_ctas = (int)gridDim.x;
  if (tid == 0) {
    for (int i = 0; i < L::kStages; ++i) { mbar_init(&ctrl->full[i], 1); mbar_init(&ctrl->empty[i], kWarps); }
    for (int i = 0; i <= L::kDepth; ++i) { mbar_init(&ctrl->k_full[i], 1); mbar_init(&ctrl->k_empty[i], 1); }
    for (int i = 0; i < L::kDepth; ++i) { mbar_init(&ctrl->v_full[i], 1); mbar_init(&ctrl->v_empty[i], 1); }
    mbar_init(&ctrl->q_full, 1); mbar_init(&ctrl->q_empty, 1);
    for (int t = 0; t < 2; ++t) {
      mbar_init(&ctrl->s_full[t], 1); mbar_init(&ctrl->p_full[t][0], 128); mbar_init(&ctrl->p_full[t][1], 128);
      mbar_init(&ctrl->o_done[t], 1); mbar_init(&ctrl->o_free[t], 128);
    }
    ctrl->abort_flag = 0; ctrl->invalid = 0;
    fence_barrier_init();
  }
  if (tid >= 32 && tid < 32 + kMaxEntries / 32) { ctrl->prefixed[tid - 32] = 0; ctrl->pairs[tid - 32] = 0; }
  if (warp == 9) { tmem_alloc(&ctrl->tmem_base, 512); tmem_relinquish(); }
  if (warp == kWarps && elect_one()) { prefetch_tmap(&tmap_k); prefetch_tmap(&tmap_v); prefetch_tmap(&tmap_kx); prefetch_tmap(&tmap_vx); prefetch_tmap(&tmap_q); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  ba_pdl_wait();
  ba_pdl_trigger();
  // The streams: units before every entry, by kind, and what the entries of many rows cost.  A thread takes neighbouring entries.
  const int per = (n_entries + kThreads - 1) / kThreads, e0 = min(n_entries, tid * per), e1 = min(n_entries, e0 + per);
  long long sum[2] = {0, 0};
  Entry one;                                               // (a thread's only entry, where there are no more than threads)
  for (int e = e0; e < e1; ++e) {
    if (!load_entry(p, e, one)) { ctrl->invalid = 1; break; }
    sum[is_many(p, one)] += lay_of(p, one).a_head() * p.Hkv;
    if (one.rows * p.G > 128) atomicOr(&ctrl->pairs[e >> 5], 1u << (e & 31));
    if (e < p.n_groups && one.len > 0) {                   // its sequences do not write their rows straight to the output
      const int a = p.group_cu ? p.group_cu[e] : 0, b = p.group_cu ? p.group_cu[e + 1] : p.batch;
      for (int w = a >> 5; w <= (b - 1) >> 5 && a < b; ++w) {
        const unsigned from = w == a >> 5 ? ~0u << (a & 31) : ~0u, to = w == (b - 1) >> 5 ? ~0u >> (31 - ((b - 1) & 31)) : ~0u;
        atomicOr(&ctrl->prefixed[w], from & to);
      }
    }
  }
  const long long mine[2] = {sum[0], sum[1]};
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long a = __shfl_up_sync(0xffffffffu, sum[0], d), b = __shfl_up_sync(0xffffffffu, sum[1], d);
    if (lane >= d) { sum[0] += a; sum[1] += b; }
  }
  if (lane == 31) ctrl->warp_sums[warp] = make_longlong2(sum[0], sum[1]);
  __syncthreads();
  long long total[2] = {0, 0};
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    const longlong2 v = ctrl->warp_sums[w];
    if (w < warp) { sum[0] += v.x; sum[1] += v.y; }
    total[0] += v.x; total[1] += v.y;
  }
  const bool valid = !ctrl->invalid && total[0] <= kMostUnits && total[1] <= kMostUnits;
  // CTAs for many rows
  int n_many = 0;
  if (valid && total[1] > 0) {
    const float few = (float)total[0] * kCostFew, more = (float)total[1] * kCostMany;
    n_many = (int)((float)n_ctas * more / (more + few) + 0.5f);
    n_many = max(1, min(n_many, total[0] > 0 ? n_ctas - 1 : n_ctas));
  }
  const int n_few = n_ctas - n_many;
  // (a run is a tile at least: every CTA between an item's first and last tile has one of it)
  auto run_of = [&](int kind) {
    const unsigned n = (unsigned)(kind ? n_many : n_few);
    return valid && n > 0 ? max(kind ? kTilePair : kTileFew, (int)(((unsigned)total[kind] + n - 1) / n)) : 0;     // (fits: total is checked)
  };
  if (valid) {
    int u[2] = {(int)(sum[0] - mine[0]), (int)(sum[1] - mine[1])};
    for (int e = e0; e < e1; ++e) {
      units[e] = u[0]; units_many[e] = u[1];
      const Entry x = per == 1 ? one : get_entry(p, e);
      const bool many = is_many(p, x);
      if (blockIdx.x == 0) p.meta[e] = make_int4(u[many], tiles_of(x), x.rows * p.G, many);
      u[many] += (int)lay_of(p, x).a_head() * p.Hkv;
    }
    if (tid == kThreads - 1) { units[n_entries] = (int)total[0]; units_many[n_entries] = (int)total[1]; }
  }
  if (blockIdx.x == 0 && tid == 0) {
    p.meta[n_entries] = make_int4(run_of(0), run_of(1), n_many, valid);
    if (!valid) ba_record_status(p.status, BA_ERR_INVALID_ARG);
  }
  const bool many = (int)blockIdx.x < n_many;
  const int nth = many ? (int)blockIdx.x : (int)blockIdx.x - n_many, all = valid ? (int)total[many] : 0;
  const int run = run_of(many);
  const int begin = (int)min((long long)all, (long long)run * nth), end = (int)min((long long)all, (long long)begin + run);
  __syncthreads();
  if (begin < end) {
    if (many) many_rows<D>(p, &tmap_kx, &tmap_vx, &tmap_k, &tmap_v, &tmap_q, smem, ctrl, units_many, n_entries, begin, end);
    else few_rows<D>(p, &tmap_kx, &tmap_vx, &tmap_k, &tmap_v, smem, ctrl, units, n_entries, begin, end);
  }
  tc_fence_before();
  __syncthreads();
  if (tid == 0 && ctrl->abort_flag) ba_record_status(p.status, BA_ERR_TIMEOUT);
  if (warp == 9) tmem_dealloc(ctrl->tmem_base, 512);
}

// The partial results of every (row, head): those of its group's prefix and of its own rows, weighted by their denominators.  What a row
// waits for is a chain of look-ups, so rows go side by side: eight lanes a row (32600 rows: 34 us with a warp each), or, with few rows,
// whose long prefixes leave many results, a warp or four (the figures are at the launch).
template <int D, int kL>
__global__ void __launch_bounds__(256)
ba_shared_merge_kernel(const __grid_constant__ SharedParams p, int warps_a_row) {
  constexpr int kVec = D / kL < 4 ? D / kL : 4, kChunks = D / (kL * kVec);     // a lane has kChunks x kVec columns
  constexpr int kV = kVec * kChunks, kBatch = kL == 32 ? 4 : 2;                // results whose values are on their way at a time
  __shared__ float others[kL == 32 ? 8 : 1][32 * kV + 2];
  const int lane = threadIdx.x % kL, warp = threadIdx.x >> 5;
  const int share = kL == 32 ? warp & (warps_a_row - 1) : 0;                   // this warp's share of the row's results
  const long long u = ((long long)blockIdx.x * (256 / kL) + threadIdx.x / kL) / warps_a_row;
  // Whose row this is, while the kernel before is still at work: the caller's tables are not that kernel's, and what wrote them had
  // completed when it let this one start.
  const bool there = u < (long long)p.n_q_rows * p.Hq;
  const int row = there ? (int)u / p.Hq : 0, hq = there ? (int)u - row * p.Hq : 0, h = hq / p.G;
  int s = row, g = -1, row0[2] = {0, 0};
  if (there && p.q_cu) {
    int lo = 0, hi = p.batch + 1;
    while (lo < hi) { const int mid = (lo + hi) >> 1; if (p.q_cu[mid] <= row) lo = mid + 1; else hi = mid; }
    s = lo - 1;
  }
  // (lanes whose row is not there or complete go on without results: the warps of a CTA meet)
  bool needed = there && s >= 0 && s < p.batch;
  if (needed) {
    g = group_of(p, s);
    row0[1] = q_begin(p, s);
    if (g >= 0 && p.group_cu) { const int a = p.group_cu[g]; row0[0] = a >= 0 && a <= p.batch ? q_begin(p, a) : 0; }    // (not checked yet)
    else if (g >= 0) row0[0] = q_begin(p, 0);
  }
  ba_pdl_wait();
  ba_pdl_trigger();
  const int4 head = p.meta[p.n_groups + p.batch];          // (plain loads: the kernel before wrote them)
  needed = needed && head.w;
  // results of this row: first pieces, then those of CTAs, of its prefix (0) and of its own rows (1)
  int n[2] = {0, 0}, c0[2] = {0, 0}, per[2] = {1, 1}, tile_row[2] = {0, 0};
  if (needed) {
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      if (side == 0 && g < 0) continue;
      const int e = side == 0 ? g : p.n_groups + s;
      const int4 m = p.meta[e];
      if (m.y == 0) continue;
      const int r = (row - row0[side]) * p.G + hq - h * p.G, rt = m.w ? r / kManyRows : 0, run = m.w ? head.y : head.x;
      const Lay lay(m.y, m.z, m.w != 0);
      const int first_tile = m.x + h * (int)lay.a_head() + rt * lay.full + lay.front;
      const int w = tile_units(m.w != 0, m.z - rt * kManyRows);
      c0[side] = first_tile / run;
      const int pieces = (first_tile + (m.y - 1) * w) / run - c0[side] + 1;
      if (side == 1 && n[0] == 0 && pieces == 1 && !m.w) { needed = false; continue; }       // whole, and nothing beside it: written where it was computed
      c0[side] += m.w ? 0 : head.z;
      per[side] = m.w && m.z - rt * kManyRows <= 128 ? 2 : 1;                  // each softmax group left a result
      n[side] = pieces * per[side];
      tile_row[side] = r - rt * kManyRows;
    }
  }
  const long long here = (long long)row * p.Hq + hq;
  const int total = n[0] + n[1], i_begin = share * total / warps_a_row, i_end = (share + 1) * total / warps_a_row;
  float top = -INFINITY, den = 0.f, acc[kV];
#pragma unroll
  for (int v = 0; v < kV; ++v) acc[v] = 0.f;
  // everything so far and `mx`, which may be -infinity like `top`, on a common scale
  auto rescale = [&](float mx) {
    const float f = top == -INFINITY ? 0.f : __expf(top - mx);
    top = mx;
    den *= f;
#pragma unroll
    for (int v = 0; v < kV; ++v) acc[v] *= f;
  };
  // A lane looks up one result of kL; what is not empty is added.  (The rows of a warp take as many rounds as its longest.)
  const int rounds = __reduce_max_sync(0xffffffffu, i_end - i_begin);
  for (int i0 = 0; i0 < rounds; i0 += kL) {
    const int i = i_begin + i0 + lane;
    long long at = -1;                                     // (of an empty result: it holds no values at all)
    float lse = -INFINITY;
    if (i < i_end) {
      const int side = i >= n[0], k = i - (side ? n[0] : 0), two = (side ? per[1] : per[0]) - 1, piece = k >> two, second = k & two;
      at = piece == 0 ? first_part(p, (side ? 0 : 1) + 2 * second) + here
                      : cut_part(p, (side ? c0[1] : c0[0]) + piece) + (side ? tile_row[1] : tile_row[0]) + 128 * second;
      lse = p.part[p.n_part * D + at];
      if (lse == -INFINITY) at = -1;
    }
    float mx = fmaxf(lse, top);
#pragma unroll
    for (int d = kL / 2; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
    const float w = at < 0 ? 0.f : __expf(lse - mx);       // (a NaN stays one)
    rescale(mx);
    for (int k0 = 0; k0 < min(kL, rounds - i0); k0 += kBatch) {
      float wk[kBatch], f[kBatch][kV];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        wk[k] = __shfl_sync(0xffffffffu, w, (k0 + k) & (kL - 1), kL);          // (kL is a multiple of kBatch)
        const long long from = __shfl_sync(0xffffffffu, at, (k0 + k) & (kL - 1), kL);
        const float *x = p.part + from * D + lane * kVec;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          if (kVec == 4) {
            const float4 v = from < 0 ? make_float4(0.f, 0.f, 0.f, 0.f) : __ldcs(reinterpret_cast<const float4 *>(x + c * kL * kVec));
            f[k][c * kVec] = v.x; f[k][c * kVec + 1] = v.y; f[k][c * kVec + 2 % kVec] = v.z; f[k][c * kVec + 3 % kVec] = v.w;
          } else {
            const float2 v = from < 0 ? make_float2(0.f, 0.f) : __ldcs(reinterpret_cast<const float2 *>(x + c * kL * kVec));
            f[k][c * kVec] = v.x; f[k][c * kVec + 1] = v.y;
          }
        }
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        den += wk[k];
#pragma unroll
        for (int v = 0; v < kV; ++v) acc[v] = fmaf(wk[k], f[k][v], acc[v]);
      }
    }
  }
  if (kL == 32 && warps_a_row > 1) {                       // the row's first warp adds the others' shares, in order
    if (share > 0) {
#pragma unroll
      for (int v = 0; v < kV; ++v) others[warp][lane * kV + v] = acc[v];
      if (lane == 0) { others[warp][32 * kV] = top; others[warp][32 * kV + 1] = den; }
    }
    __syncthreads();
    if (share > 0) return;
    for (int k = 1; k < warps_a_row; ++k) {
      const float t = others[warp + k][32 * kV], d = others[warp + k][32 * kV + 1];
      if (d == 0.f) continue;
      rescale(fmaxf(top, t));
      const float f = __expf(t - top);
      den = fmaf(d, f, den);
#pragma unroll
      for (int v = 0; v < kV; ++v) acc[v] = fmaf(others[warp + k][lane * kV + v], f, acc[v]);
    }
  }
  if (!needed) return;
  const float inv = den != 0.f ? 1.f / den : 0.f;
#pragma unroll
  for (int v = 0; v < kV; ++v) acc[v] *= inv;
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const long long out = here * D + c * kL * kVec + lane * kVec;
    const float *a = acc + c * kVec;
    if (p.out_f32) {
      float *o = reinterpret_cast<float *>(p.o) + out;
      if (kVec == 4) *reinterpret_cast<float4 *>(o) = make_float4(a[0], a[1], a[2 % kVec], a[3 % kVec]);
      else *reinterpret_cast<float2 *>(o) = make_float2(a[0], a[1]);
    } else {
      __nv_bfloat16 *o = reinterpret_cast<__nv_bfloat16 *>(p.o) + out;
      if (kVec == 4) *reinterpret_cast<uint2 *>(o) = make_uint2(pack_bf16(a[0], a[1]), pack_bf16(a[2 % kVec], a[3 % kVec]));
      else *reinterpret_cast<uint32_t *>(o) = pack_bf16(a[0], a[1]);
    }
  }
  if (p.lse && lane == 0) p.lse[here] = den != 0.f ? top + logf(den) : -INFINITY;
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Rows of partial results: four for every (query row, head), and kManyRows a CTA.
long long part_rows(const ba_config &c, int n_q_rows, int n_ctas) { return 4ll * n_q_rows * c.n_q_heads + (long long)n_ctas * kManyRows; }
size_t meta_bytes(int n_entries) { return ba_align_up((size_t)(n_entries + 1) * sizeof(int4), 256); }

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
           (size_t)part_rows(*cfg, n_q_rows, kBaMostSms) * (cfg->head_dim + 1) * sizeof(float) + 256;
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
  const long long n_part = part_rows(ctx->cfg, n_q_rows, ctx->sm_count);
  const size_t need = meta_bytes(n_entries) + (size_t)n_part * (D + 1) * sizeof(float);
  if (!ctx->workspace || ba_scratch_offset(ctx) + need + ctx->pending_table_bytes > ctx->workspace_bytes) return BA_ERR_WORKSPACE;
  if ((long long)n_q_rows * ctx->cfg.n_q_heads > INT32_MAX) return BA_ERR_SHAPE;
  BA_CUDA_TRY(cudaSetDevice(ctx->device));
  const cudaStream_t cs = (cudaStream_t)stream;
  const size_t kv_row = (size_t)ctx->cfg.n_kv_heads * D * 2;
  st = ba_flush_pending_into(ctx, k_pool, kv_row * pages->n_pages * pages->page_rows, cs);
  if (st == BA_OK && b->n_groups > 0)
    st = ba_flush_pending_into(ctx, k_prefix, kv_row * (prefix_pages ? (size_t)prefix_pages->n_pages * prefix_pages->page_rows : n_prefix_rows), cs);
  if (st != BA_OK) return st;
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
  p.n_part = n_part;
  CUtensorMap tk, tv, tkx, tvx, tq;
  const long long rows = (long long)pages->n_pages * pages->page_rows;
  const int box = std::min(kTile, pages->page_rows);
  if (!ba_tensor_map(ctx, &tk, k_pool, p.Hkv, rows, 1, box) || !ba_tensor_map(ctx, &tv, v_pool, p.Hkv, rows, 1, box)) return BA_ERR_CUDA;
  tkx = tk; tvx = tv; tq = tk;
  p.q_boxes = p.G <= 128 && 128 % p.G == 0;
  if (p.q_boxes && !ba_tensor_map(ctx, &tq, q, p.Hq, n_q_rows, p.G, 128 / p.G)) return BA_ERR_CUDA;
  if (has_prefix) {
    const long long prows = prefix_pages ? (long long)prefix_pages->n_pages * prefix_pages->page_rows : n_prefix_rows;
    const int pbox = prefix_pages ? std::min(kTile, prefix_pages->page_rows) : kTile;
    if (!ba_tensor_map(ctx, &tkx, k_prefix, p.Hkv, prows, 1, pbox) || !ba_tensor_map(ctx, &tvx, v_prefix, p.Hkv, prows, 1, pbox)) return BA_ERR_CUDA;
  }
  const dim3 grid((unsigned)ctx->sm_count);
  // How many lanes a row gets in the merge: what decides is rows x results, but results follow from lengths that the host does not read.  Calls of
  // 32 heads over a shared prefix of 2000 / 32000 keys, us with 8 lanes, a warp, four warps a row: 512 rows 33.2, 24.4, 22.8 / 86.0, 50.1, 46.1;
  // 1024 rows 32.1, 27.4, 26.5 / 87.7, 55.0, 53.5; 2048 rows 38.5, 36.0, 39.7 / 86.9, 69.5, 72.5; 4096 rows 49.8, 49.1, 58.8 / 118, 132, 134;
  // 6144 rows 77.6, 75.5, 91.6 / 162, 182, 202; 8192 rows 88.4, 95.8, 111 / 202, 230, 262.  Without a prefix a warp a row is as good or better up
  // to 6144 rows (300 keys each: 2048 rows 34.0, 32.3, 33.9; 6144 rows 78.2, 76.9, 83.6; 12288 rows 140.4, 140.9, 154.7).
  const long long rows_out = (long long)n_q_rows * p.Hq;
  const bool wide = rows_out <= 6144;
  const int warps_a_row = rows_out <= 1024 ? 4 : 1;
  const unsigned merge = (unsigned)((rows_out * warps_a_row * (wide ? 32 : 8) + 255) / 256);
  if (D == 128) {
    BA_CUDA_TRY(ba_launch(ba_shared_attend_kernel<128>, grid, kThreads, SharedLayout<128>::kBytes, cs, true, tkx, tvx, tk, tv, tq, p));
    BA_CUDA_TRY(ba_launch(wide ? ba_shared_merge_kernel<128, 32> : ba_shared_merge_kernel<128, 8>, dim3(merge), 256, 0, cs, true, p, warps_a_row));
  } else {
    BA_CUDA_TRY(ba_launch(ba_shared_attend_kernel<64>, grid, kThreads, SharedLayout<64>::kBytes, cs, true, tkx, tvx, tk, tv, tq, p));
    BA_CUDA_TRY(ba_launch(wide ? ba_shared_merge_kernel<64, 32> : ba_shared_merge_kernel<64, 8>, dim3(merge), 256, 0, cs, true, p, warps_a_row));
  }
  ctx->launches += 2;
  return BA_OK;
}

}  // extern "C"

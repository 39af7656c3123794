// Attention of a batch whose sequences share long prefixes.
//
//   out[t][h] = sum_j p_j v_j / sum_j p_j,   j over the prefix of t's sequence, its own positions and the rows that t sees
//
// The softmax of a row falls apart into parts (reference, sum, output) that are joined by their log-sum-exp.  What a
// prefix contributes is one large product for all rows that share it: with 256 rows of a KV head in a tile the cache of the
// prefix is read once per tile, and the tensor core, not the cache, bounds the work.  What the sequences' own positions
// contribute is a few rows over a short stretch each, bound by the cache.  One launch does both at once: some CTAs take the
// prefixes (tensor memory), the others the own positions (a stream for every warp), in shares that cost about the same,
// so that the memory system works for the ones while the tensor cores work for the others.  prefix_join_kernel joins the
// parts in ascending order: the same lengths give the same bits.
//
// A CTA of the prefixes.  Warp 8 copies keys and values page by page into a ring, warps 9 and 11 issue the products of a
// group each, warp 10 plans, and two groups of four warps have an accumulator of 128 rows each, one thread per row: a thread
// takes 64 scores of its row at a time from tensor memory, maximum, exponentials, and puts the probabilities where the scores
// were, while the tensor core computes the next 64 beside them.  Nothing is exchanged between threads; a row's reference
// moves only when a score exceeds the maximum that set it by a factor of 2^8, and then the thread rescales its output by itself
// once the products under way have ended.
// In a tile of at most 128 rows both groups have the same rows and every other unit, and join their halves at the end.
// Every row of a tile sees the whole prefix, so masks are only needed at its end and at bad pages, and are the same for
// all rows.  P is rounded to the cache's type as in tree attention.
//
// 192 rows of 64 and 8 heads of 128 over 32,765 positions: 264 to 272 us in a burst, 315 in a long run under the power limit (0.66
// PFLOP/s); products alone 123 and 145 at the measured rates.  Neither unit is full: the tensor pipe is active 40% of the time (a 128 x 128 x 16 product takes 64 cycles, a 128 x 64 x 16 one 48),
// the special-function units need half of a block's cycles, and the groups run in step and share both.  Slower, at the same
// point: 128 positions a block 303, one thread for the products of both groups 317, two threads a row 291, a part of the
// exponentials by polynomial 270, the next scores asked for before the exponentials 307 and more.  Smaller calls are bound by
// latency: plan and queries 7 to 9 us, the end of a segment 4 to 5, the joining kernel 5 to 8.
#include <algorithm>
#include <cmath>
#include <cstdio>

#include "paged_device.cuh"

namespace prima {
namespace {

constexpr int kPrefixThreads = 384;
constexpr int kBlock = 64;              // positions whose scores are one product
constexpr int kPlanned = 4;            // segments ahead
// In places.  With 1, 4, 8: 64 rows over 8192 positions 61, 58, 59 us, three prefixes 36, 35, 35 (heads of 64), 56, 48, 46 (of 128), 192
// rows over 32,765 positions 268, 264, 264, of heads of 64 229, 228, 250.
constexpr int kPrefixSegmentCost = 4;
// Registers of a thread: the two groups that hold scores (or the fragments of the streaming body), and the third one.  Their
// sum is what the block is launched with: 384 x 168 = 256 x 208 + 128 x 88.  18 to 20 registers are
// spilled (half of the joining kernel's forms spill one or two).
constexpr int kManyRegisters = 208, kFewRegisters = 88;

// What a step of 16 own positions costs, in 64ths of a prefix's place.  Heads of 128, 6, 10 and 16: three prefixes 50, 48, 52 us, 64
// rows over 8192 positions 59, 58, 66, 192 rows over 32,765 positions 309, 264, 272; 32 requests of 900 to 1900 positions behind 2000,
// which are mostly own ones, 58, 67, 84.  Heads of 64, 3, 6 and 10, the same: 44, 35, 35; 51, 40, 43; 420, 228, 225; 43, 42, 51.
constexpr int kOwnCost128 = 10, kOwnCost64 = 6;

struct PrefixView {
  int n;
  const int32_t* seq_begin;
  const int32_t* len;
  const int32_t* table;
  int64_t table_stride;
};

// Parts: of a source (0: prefixes, 1: own positions) and of every KV head, row R = token * group + query head in the group.
// What a worker has whole lies at [head][D/4][rows][4]; what it has of something that is cut, at
// [2 * worker + (it begins here)][D/4][tile rows][4].
struct PrefixArgs {
  PoolView pool;
  BatchView b;
  PrefixView prefix;
  PrefixShape shape;
  int64_t capacity;          // positions that a row of the sequences' table can name
  int layer, n_q_heads, group;
  uint32_t group_inverse;    // small_inverse(group)
  float scale_log2;
  const void* q;
  void* out;
  float* lse;
  int own_cost;              // 0: the own positions' attention is done in front
  int64_t rows;              // n_tok * group
  int n_cta;                 // workers there are at most: of the prefixes; eight times as many stream
  float* whole_o[2];
  float2* whole_ml[2];       // [head][rows]: reference, sum
  int2* note[2];             // [head][rows]: first worker, number of parts
  int4* place;               // [n_tok], see write_places
  float* part_o;             // of the prefixes' workers
  float2* part_ml;
  float* own_part_o;         // of the streaming ones
  float2* own_part_ml;
};

struct PrefixWork {
  int prefix, head, row0, rows;        // rows row0 .. row0 + rows - 1 of the (prefix, KV head)
  long long first;                     // row R of the first of all
  int unit0, n;
  int kind;                            // 0: whole; 1: continues; 2: begins here and goes on
  int last_worker;
  long long limit;                     // positions that are seen
  __device__ __forceinline__ bool both() const { return rows > kPrefixRows / 2; }      // accumulators per unit
  __device__ __forceinline__ int units_of(int group_of_warps) const { return prefix_group_units(both(), n, group_of_warps); }
};

struct PrefixControl {
  unsigned long long full[12], empty[12], s_ready[4], p_ready[4], pv_done[4], q_ready[2], q_first, drained;
  unsigned long long seg_full[kPlanned], seg_empty[kPlanned];
  PrefixWork seg[kPlanned];
  long long places, own_places;
  uint32_t tmem;
  int give_up;
  int edge[16];                        // of the last units: not all positions are seen (the ring holds fewer)
  uint32_t seen[16][4];
  float2 ml[2][128];                   // a group's reference and sum, for the other one
};

// The range of a prefix: rows of the step that share it, or none.  Reads device memory; false: the numbers are bad.
struct PrefixRange {
  int first = 0, rows = 0, len = 0;    // rows: of the step
};
__device__ __forceinline__ bool prefix_range(const PrefixArgs& a, int p, PrefixRange* out) {
  const BatchView& b = a.b;
  const int s0 = a.prefix.seq_begin[p], s1 = a.prefix.seq_begin[p + 1], len = a.prefix.len[p];
  *out = PrefixRange();
  if (s0 < 0 || s1 < s0 || s1 > b.n_seq || len < 0) return false;
  if (s1 == s0) return true;
  const int first = b.row_begin[s0], end = b.row_begin[s1];
  if (first < 0 || end < first || end > b.n_tok) return false;
  out->first = first;
  out->rows = end - first;
  out->len = len;
  return true;
}

// The prefixes' line, 32 prefixes at a time, one per lane of a warp: its length, then a worker's share of it.
struct PrefixCursor {
  const PrefixArgs& a;
  const int lane;
  int worker = 0, p0 = 0;              // p0: first prefix of the window
  long long total = 0, u = 0, u_end = 0, window = 0, before = 0, per_head = 0, places = 0;
  TreeShares shares{};
  PrefixRange range;

  __device__ __forceinline__ bool read(int p) {
    const bool ok = prefix_range(a, p, &range);
    per_head = prefix_places(a.shape, static_cast<long long>(range.rows) * a.group, prefix_units(a.shape, range.len));
    places = per_head * a.pool.n_kv_heads;
    return ok;
  }
  __device__ void load(long long in_front, bool has_read = false) {
    if (!has_read) {
      per_head = places = 0;
      range = PrefixRange();
      if (p0 + lane < a.prefix.n) read(p0 + lane);
    }
    long long x = places;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    before = in_front + x - places;
    window = in_front + __shfl_sync(0xffffffffu, x, 31);
  }
  __device__ __forceinline__ PrefixCursor(const PrefixArgs& args, int lane_) : a(args), lane(lane_) {}
  __device__ __forceinline__ void add_up(bool reports) {
    for (int p = lane; p < a.prefix.n; p += 32) {
      const bool ok = read(p);
      total += places;
      if (reports) {
        if (!ok) raise(a.pool.status, kBadRows);
        else if (range.rows && range.len > a.shape.capacity) raise(a.pool.status, kBadSlot);
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  }
  __device__ __forceinline__ void begin(int worker_, int n_workers) {
    worker = worker_;
    shares = tree_shares(total, n_workers);
    u = tree_share_begin(shares, worker);
    u_end = tree_share_begin(shares, worker + 1);
    load(0, a.prefix.n <= 32);      // what add_up has read last
  }
  __device__ bool next(PrefixWork* s) {
    while (u < u_end) {
      unsigned hit;
      while (!(hit = __ballot_sync(0xffffffffu, u >= before && u < before + places))) {      // ends: u is below the total
        p0 += 32;
        load(window);
      }
      const int src = __ffs(hit) - 1;
      const long long in_front = __shfl_sync(0xffffffffu, before, src), mine = __shfl_sync(0xffffffffu, per_head, src);
      const int first = __shfl_sync(0xffffffffu, range.first, src), n_rows = __shfl_sync(0xffffffffu, range.rows, src), len = __shfl_sync(0xffffffffu, range.len, src);
      const long long rows = static_cast<long long>(n_rows) * a.group, units = prefix_units(a.shape, len);
      const PrefixSegment t = prefix_segment(a.shape, rows, units, mine, u - in_front, u_end - in_front);
      s->prefix = p0 + src;
      s->head = t.head;
      s->row0 = static_cast<int>(t.row_tile * kPrefixRows);
      s->rows = static_cast<int>(min(rows - s->row0, static_cast<long long>(kPrefixRows)));
      s->first = static_cast<long long>(first) * a.group;
      s->unit0 = t.unit0;
      s->n = t.unit1 - t.unit0;
      s->kind = t.unit0 ? 1 : t.unit1 < units ? 2 : 0;
      s->last_worker = s->kind == 2 ? tree_cta_of(shares, in_front + t.last) : worker;
      s->limit = min(static_cast<long long>(len), static_cast<long long>(a.shape.capacity));
      u += t.places;
      if (s->n) return true;
    }
    return false;
  }
};

// ---- the sequences' own positions ------------------------------------------------------------------------------------
// A worker is a warp: it copies 16 positions at a time through a ring of its own, a few steps ahead and on into its next
// segments, and applies them with m16n8k16 products, queries and output in registers; nothing waits for another warp.
template <int D> struct OwnGeometry {
  static constexpr int kWarps = 8, kStages = D == 128 ? 3 : 6;
  static constexpr int kHalf = kFewPos * D * 2;                // keys or values of a step
  static constexpr int kStage = 2 * kHalf;
  static constexpr int kPanel = kFewPos * 128;                 // 64 columns of either
  static constexpr int kWarpBytes = kStages * kStage;
};
struct OwnWork {
  int seq, first, nodes, ctx, head, row0, rows, step0, n;      // rows row0 .. of the (sequence, KV head)
  int kind, last_worker;               // as PrefixWork
  long long limit;                     // positions there are
};
constexpr int kWindows = 1024;         // of the sequences, for which their places are added up
struct OwnControl {                    // behind the warps' rings
  long long before[kWindows];          // places in front of a window
  unsigned long long full[8][6];
  OwnWork fifo[8][8];                  // segments between a warp's copies (at most five steps ahead) and its products
};
// Sequences of a window: 32, or a multiple where there are too many.
__device__ __forceinline__ int window_of(int n_seq) { return 32 * ((n_seq + 32 * kWindows - 1) / (32 * kWindows)); }

// A sequence as the own positions' line counts it.
struct OwnSeq {
  int first = 0, nodes = 0, ctx = 0;
  long long limit = 0, per_head = 0;
};
__device__ __forceinline__ bool own_seq(const PrefixArgs& a, int i, OwnSeq* s) {
  const int f = a.b.row_begin[i], e = a.b.row_begin[i + 1], c = a.b.ctx_len[i];
  *s = OwnSeq();
  if (f < 0 || e < f || e > a.b.n_tok || c < 0) return false;
  s->first = f;
  s->nodes = e - f;
  s->ctx = c;
  s->limit = min(static_cast<long long>(c) + s->nodes, static_cast<long long>(a.capacity));
  s->per_head = own_places(s->nodes * a.group, s->limit);
  return true;
}
// Places of each window of sequences, by all warps; their sums by the first one.  Two barriers.
__device__ void add_up_own(const PrefixArgs& a, OwnControl* own, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, size = window_of(a.b.n_seq), n = (a.b.n_seq + size - 1) / size;
  for (int w = warp; w < n; w += kPrefixThreads / 32) {
    long long sum = 0;
    for (int i = w * size + lane; i < min((w + 1) * size, a.b.n_seq); i += 32) {
      OwnSeq s;
      const bool ok = own_seq(a, i, &s);
      sum += s.per_head * a.pool.n_kv_heads;
      if (blockIdx.x == 0) {
        if (!ok) raise(a.pool.status, kBadRows);
        else if (s.nodes && static_cast<long long>(s.ctx) + s.nodes > a.capacity) raise(a.pool.status, kBadSlot);
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) own->before[w] = sum;
  }
  __syncthreads();
  if (warp == 0) {
    long long front = 0;
    for (int w0 = 0; w0 < n; w0 += 32) {
      const long long mine = w0 + lane < n ? own->before[w0 + lane] : 0;
      long long x = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      if (w0 + lane < n) own->before[w0 + lane] = front + x - mine;
      front += __shfl_sync(0xffffffffu, x, 31);
    }
    if (lane == 0) *total = front;
  }
  __syncthreads();
}

// Walks a worker's share of the own positions, 32 sequences at a time, one per lane.
struct OwnCursor {
  const PrefixArgs& a;
  const int lane, worker;
  const TreeShares shares;
  long long u, u_end, window = 0, front = 0;      // front: places in front of the lane's sequence
  int w0 = 0;
  OwnSeq mine;

  __device__ __forceinline__ void load(long long in_front) {
    mine = OwnSeq();
    if (w0 + lane < a.b.n_seq) own_seq(a, w0 + lane, &mine);
    long long x = mine.per_head * a.pool.n_kv_heads;
    const long long places = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    front = in_front + x - places;
    window = in_front + __shfl_sync(0xffffffffu, x, 31);
  }
  __device__ OwnCursor(const PrefixArgs& args, const OwnControl* own, int lane_, int worker_, int n_workers, long long total)
      : a(args), lane(lane_), worker(worker_), shares(tree_shares(total, n_workers)) {
    u = tree_share_begin(shares, worker);
    u_end = tree_share_begin(shares, worker + 1);
    if (u >= u_end) return;
    const int size = window_of(a.b.n_seq);
    int lo = 0, hi = (a.b.n_seq + size - 1) / size;
    while (hi - lo > 1) {      // the last window with at most u places in front
      const int at = (lo + hi) / 2;
      if (own->before[at] <= u) lo = at;
      else hi = at;
    }
    w0 = lo * size;
    load(own->before[lo]);
  }
  __device__ __forceinline__ bool next(OwnWork* s) {
    while (u < u_end) {
      unsigned hit;
      while (!(hit = __ballot_sync(0xffffffffu, u >= front && u < front + mine.per_head * a.pool.n_kv_heads))) {      // ends: u is below the total
        w0 += 32;
        load(window);
      }
      const int src = __ffs(hit) - 1;
      const long long in_front = __shfl_sync(0xffffffffu, front, src), per_head = __shfl_sync(0xffffffffu, mine.per_head, src);
      s->first = __shfl_sync(0xffffffffu, mine.first, src);
      s->nodes = __shfl_sync(0xffffffffu, mine.nodes, src);
      s->ctx = __shfl_sync(0xffffffffu, mine.ctx, src);
      s->limit = __shfl_sync(0xffffffffu, mine.limit, src);
      const OwnSegment t = own_segment(s->limit, per_head, u - in_front, u_end - in_front);
      s->seq = w0 + src;
      s->head = t.head;
      s->row0 = t.tile * kFewRows;
      s->rows = min(s->nodes * a.group - s->row0, kFewRows);
      s->step0 = t.step0;
      s->n = t.step1 - t.step0;
      s->kind = t.step0 ? 1 : t.step1 < own_steps(s->limit) ? 2 : 0;
      s->last_worker = s->kind == 2 ? tree_cta_of(shares, in_front + t.last) : worker;
      u += t.places;
      if (s->n) return true;
    }
    return false;
  }
};

template <typename T, int D>
__device__ __forceinline__ void own_share(const CUtensorMap* k_map, const CUtensorMap* v_map, const PrefixArgs& a, uint8_t* smem, OwnControl* own, int* give_up, int worker,
                                          int n_workers, long long total) {
  using Geo = OwnGeometry<D>;
  constexpr bool kBf16 = !__is_same(T, __half);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
  int* const status = a.pool.status;
  const uint32_t ring_addr = smem_u32(smem + warp * Geo::kWarpBytes), bar_full = smem_u32(own->full[warp]);
  const int shift = a.pool.page_shift;
  // Copies of a step: lane i < boxes takes 64 columns of box_rows positions of keys or values.
  const int box_rows = min(1 << shift, kFewPos), halves = kFewPos / box_rows, boxes = 2 * (D / 64) * halves;
  const int is_v = lane / (boxes / 2), panel = lane % (boxes / 2) / halves, half = lane % halves;
  const CUtensorMap* const map = is_v ? v_map : k_map;
  const uint32_t box_at = ring_addr + is_v * Geo::kHalf + panel * Geo::kPanel + half * box_rows * 128;

  // Only here, where it is known that this CTA streams: in the others copies write over this memory.
  if (lane < Geo::kStages) mbar_init(bar_full + 8 * lane, 1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  __syncwarp();
  OwnCursor cursor(a, own, lane, worker, n_workers, total);
  RingPlace<Geo::kStages> put, get;
  uint32_t bad_stages = 0, planned = 0, begun = 0;
  // The segment that is copied, its next step, the page that this lane's box of that step lies on
  OwnWork from{};
  int step = 0, page = -1;
  bool more = false;
  auto read_page = [&]() {
    const long long pos = static_cast<long long>(from.step0 + step) * kFewPos + half * box_rows;
    page = more && lane < boxes && pos < from.limit ? a.b.table[from.seq * a.b.table_stride + (pos >> shift)] : -1;
  };
  auto plan = [&]() {
    more = cursor.next(&from);
    step = 0;
    if (more) {
      __syncwarp();
      if (lane == 0) own->fifo[warp][planned & 7] = from;
      __syncwarp();
      ++planned;
    }
  };
  auto copy = [&]() {
    if (!more) return;
    const long long pos = static_cast<long long>(from.step0 + step) * kFewPos + half * box_rows;
    const bool wanted = lane < boxes && pos < from.limit, good = static_cast<unsigned>(page) < static_cast<unsigned>(a.pool.n_pages);
    if (wanted && !good) raise(status, kBadPage);
    const uint32_t copies = __ballot_sync(0xffffffffu, wanted && good);
    const bool bad = __any_sync(0xffffffffu, wanted && !good);
    bad_stages = (bad_stages & ~(1u << put.slot)) | (bad ? 1u << put.slot : 0u);
    if (lane == 0) mbar_expect(bar_full + 8 * put.slot, static_cast<uint32_t>(__popc(copies)) * box_rows * 128);
    __syncwarp();
    // below 2^31 rows (prima_paged_create)
    const int row = (((a.layer * a.pool.n_pages + page) * a.pool.n_kv_heads + from.head) << shift) + (static_cast<int>(pos) & ((1 << shift) - 1));
    if (wanted && good) tma_load_2d(box_at + put.slot * Geo::kStage, map, panel * 64, row, bar_full + 8 * put.slot);
    put.step(1);
    if (++step == from.n) plan();
    read_page();
  };
  plan();
  read_page();
#pragma unroll 1
  for (int i = 0; i < Geo::kStages - 1; ++i) copy();

  while (begun < planned) {
    const OwnWork s = own->fifo[warp][begun & 7];
    ++begun;
    const int t0 = s.row0 / a.group, rem0 = s.row0 - t0 * a.group;
    // Fragments of the queries: rows g and g + 8, columns 2 t4, + 1, + 8, + 9 of every 16
    uint32_t qf[D / 16][4];
    int node[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int x = 8 * h + g, y = rem0 + x, n = small_div(y, a.group_inverse);
      node[h] = x < s.rows ? t0 + n : -1;
      const uint32_t* src = reinterpret_cast<const uint32_t*>(static_cast<const T*>(a.q) + (static_cast<int64_t>(s.first + t0 + n) * a.n_q_heads + s.head * a.group + (y - n * a.group)) * D) + t4;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        qf[k][h] = x < s.rows ? src[8 * k] : 0u;
        qf[k][2 + h] = x < s.rows ? src[8 * k + 4] : 0u;
      }
    }
    float o[D / 8][4], ref[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
#pragma unroll
    for (int n = 0; n < D / 8; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[n][e] = 0.f;
#pragma unroll 1
    for (int i = 0; i < s.n; ++i) {
      __syncwarp();      // all have read the step whose place is filled again
      copy();
      wait_for(bar_full + 8 * get.slot, get.phase, give_up, status);
      const uint32_t kk = ring_addr + get.slot * Geo::kStage, vv = kk + Geo::kHalf;
      const long long pos0 = static_cast<long long>(s.step0 + i) * kFewPos;
      const bool bad = bad_stages >> get.slot & 1, edge = bad || pos0 + kFewPos > min(static_cast<long long>(s.ctx), s.limit);
      const SegmentView view{a.b, a.pool, s.first, s.nodes, s.ctx, s.limit, a.b.table + s.seq * a.b.table_stride, bad};
      if (edge) {
        // Values at positions that no row sees may be anything, and 0 x NaN is NaN: clear them.
        const uint32_t seen = view.seen_by_any(pos0, lane);
        if (lane < kFewPos && !(seen >> lane & 1)) {
#pragma unroll
          for (int c = 0; c < D / 8; ++c)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(vv + c / 8 * Geo::kPanel + lane * 128 + c % 8 * 16), "r"(0) : "memory");
        }
        fence_async_smem();
        __syncwarp();
      }
      float sc[2][4];
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[n][e] = 0.f;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        uint32_t b[4];      // positions 0..7 and 8..15, two halves of 8 columns each
        const int row = (lane >> 4) * 8 + (lane & 7), chunk = 2 * k + (lane >> 3 & 1);
        ldsm4(b, kk + chunk / 8 * Geo::kPanel + row * 128 + (chunk % 8 ^ (row & 7)) * 16);
        mma16816<kBf16>(sc[0], qf[k], b[0], b[1]);
        mma16816<kBf16>(sc[1], qf[k], b[2], b[3]);
      }
      if (edge) {      // positions that the row does not see, or on a bad page
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t seen = node[h] >= 0 ? view.seen_by(node[h], pos0) : 0u;
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              if (!(seen >> (8 * n + 2 * t4 + e) & 1)) sc[n][2 * h + e] = -INFINITY;
        }
      }
      float top[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) top[h] = fmaxf(fmaxf(sc[0][2 * h], sc[0][2 * h + 1]), fmaxf(sc[1][2 * h], sc[1][2 * h + 1])) * a.scale_log2;
      if (__any_sync(0xffffffffu, top[0] > ref[0] + kSlack || top[1] > ref[1] + kSlack)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float x = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 1));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
          const float r = x > ref[h] + kSlack ? x - kHeadroom : ref[h];
          const float f = r == ref[h] ? 1.f : ex2(ref[h] - r);
          ref[h] = r;
          sum[h] *= f;
#pragma unroll
          for (int n = 0; n < D / 8; ++n) {
            o[n][2 * h] *= f;
            o[n][2 * h + 1] *= f;
          }
        }
      }
      uint32_t p[4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float down = ref[h] == -INFINITY ? 0.f : -ref[h];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const float x = ex2(fmaf(sc[n][2 * h], a.scale_log2, down)), y = ex2(fmaf(sc[n][2 * h + 1], a.scale_log2, down));
          sum[h] += x + y;
          p[2 * n + h] = Half2Of<T>::pack(x, y);
        }
      }
#pragma unroll
      for (int n = 0; n < D / 16; ++n) {
        uint32_t b[4];      // 16 positions, columns 16 n .. + 7 and + 8 .. + 15
        const int row = (lane >> 3 & 1) * 8 + (lane & 7), chunk = 2 * n + (lane >> 4);
        ldsm4_t(b, vv + chunk / 8 * Geo::kPanel + row * 128 + (chunk % 8 ^ (row & 7)) * 16);
        mma16816<kBf16>(o[2 * n], p, b[0], b[1]);
        mma16816<kBf16>(o[2 * n + 1], p, b[2], b[3]);
      }
      get.step(1);
    }
    // ---- the segment's part ----
    const int64_t slot = 2 * static_cast<int64_t>(worker) + (s.kind == 2), at = static_cast<int64_t>(s.first) * a.group + s.row0;
    float* const dst = s.kind == 0 ? a.whole_o[1] + (static_cast<int64_t>(s.head) * (D / 4) * a.rows + at) * 4 : a.own_part_o + slot * (D / 4) * kFewRows * 4;
    const int64_t stride = 4 * (s.kind == 0 ? a.rows : kFewRows);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int x = 8 * h + g;
      float z = sum[h] + __shfl_xor_sync(0xffffffffu, sum[h], 1);
      z += __shfl_xor_sync(0xffffffffu, z, 2);
      if (x >= s.rows) continue;
#pragma unroll
      for (int n = 0; n < D / 8; ++n) *reinterpret_cast<float2*>(dst + (2 * n + (t4 >> 1)) * stride + 4 * x + 2 * (t4 & 1)) = make_float2(o[n][2 * h], o[n][2 * h + 1]);
      if (t4 == 0) {
        const int64_t row = static_cast<int64_t>(s.head) * a.rows + at + x;
        if (s.kind == 0) a.whole_ml[1][row] = make_float2(ref[h], z);
        else a.own_part_ml[slot * kFewRows + x] = make_float2(ref[h], z);
        if (s.kind != 1) a.note[1][row] = make_int2(worker, s.last_worker - worker + 1);
      }
    }
  }
  // A wait that gave up may have left copies under way: they end before the memory is given back.
  if (*static_cast<volatile int*>(give_up))
    for (uint32_t i = 0; i < Geo::kStages; ++i)
      for (int j = 0; j < (1 << 16) && !mbar_test(bar_full + 8 * i, i < put.slot ? put.phase : put.phase ^ 1); ++j) {}
}

// Where the joining kernel finds what belongs to a token, written here for all tokens (nothing of what it reads depends on
// the attention): whether it is any sequence's, that sequence's first row of the step, and the first row of those that share
// its prefix, -1 without one.
__device__ __forceinline__ void write_places(const PrefixArgs& a, int warp, int n_warps) {
  const int lane = threadIdx.x & 31;
  for (int t0 = 32 * warp; t0 < a.b.n_tok; t0 += 32 * n_warps) {
    const int t = t0 + lane;
    // the warp looks the first token's sequence and prefix up, the others are not far behind
    int s = seq_of_row(a.b, t0, lane), p = 0;
    for (int i = lane; i < a.prefix.n; i += 32) p += a.prefix.seq_begin[i + 1] <= s ? 1 : 0;
    p = __reduce_add_sync(0xffffffffu, p);
    if (t >= a.b.n_tok) continue;
    while (s < a.b.n_seq && a.b.row_begin[s + 1] <= t) ++s;
    OwnSeq seq;
    int4 x = make_int4(0, 0, -1, 0);
    if (s < a.b.n_seq && own_seq(a, s, &seq) && t >= seq.first) {
      while (p < a.prefix.n && a.prefix.seq_begin[p + 1] <= s) ++p;
      PrefixRange range;
      const bool shares = p < a.prefix.n && a.prefix.seq_begin[p] <= s && prefix_range(a, p, &range) && prefix_units(a.shape, range.len) > 0;
      x = make_int4(1, seq.first, shares ? range.first : -1, 0);
    }
    a.place[t] = x;
  }
}

// What the warps of a prefixes' CTA share.
template <int D>
struct PrefixCta {
  static constexpr int kSlots = Geometry<D>::kSlots;
  const PrefixArgs& a;
  uint8_t* smem;
  PrefixControl* ctl;
  int n_workers;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  int* const give_up = &ctl->give_up;
  int* const status = a.pool.status;
  uint8_t* const s_q = smem;
  uint8_t* const s_ring = smem + 2 * Geometry<D>::kQBytes;
  const uint32_t bar_full = smem_u32(ctl->full), bar_empty = smem_u32(ctl->empty), bar_s = smem_u32(ctl->s_ready), bar_p = smem_u32(ctl->p_ready),
                 bar_pv = smem_u32(ctl->pv_done), bar_seg = smem_u32(ctl->seg_full), bar_seg_empty = smem_u32(ctl->seg_empty), bar_q = smem_u32(ctl->q_ready),
                 bar_first = smem_u32(&ctl->q_first);
  const uint32_t tmem = ctl->tmem;      // scores of accumulator 0 and 1: columns 0, 128; their outputs: 256, 256 + D
  RingPlace<kSlots> ring;               // the place that the segment begins with
  uint32_t copies_before = 0;           // copies: places used so far, up to kSlots (the ring is empty at first)

  // Segment i of this CTA, or nothing when there are no more; the caller's warp gives it back with done_with(i).
  __device__ __forceinline__ const PrefixWork* segment(uint32_t i) const {
    const PrefixWork* s = &ctl->seg[i % kPlanned];
    if (!wait_segment(bar_seg + 8 * (i % kPlanned), i / kPlanned & 1)) {
      if (lane == 0) raise(status, kGaveUp);
      return nullptr;
    }
    return s->n ? s : nullptr;
  }
  __device__ __forceinline__ void done_with(uint32_t i) const {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar_seg_empty + 8 * (i % kPlanned));
  }
  template <typename T> __device__ __forceinline__ void feed(const Maps& maps, PrefixCursor& cursor);
  template <typename T> __device__ __forceinline__ void softmax();
  __device__ __forceinline__ void drain();
};

// Warps 8 to 11.
template <int D>
template <typename T>
__device__ __forceinline__ void PrefixCta<D>::feed(const Maps& maps, PrefixCursor& cursor) {
  using Geo = Geometry<D>;
  constexpr bool kBf16 = !__is_same(T, __half);
  const PoolView& pool = a.pool;
  if (warp == 10) {
    // ---- the plan ----
    cursor.begin(blockIdx.x, n_workers);
    PrefixWork s;
    for (uint32_t i = 0;; ++i) {
      const bool more = cursor.next(&s);
      if (i >= kPlanned && !__all_sync(0xffffffffu, wait_segment(bar_seg_empty + 8 * (i % kPlanned), (i / kPlanned - 1) & 1))) {      // never seen; what others may still read stays
        if (lane == 0) raise(status, kGaveUp);
        break;
      }
      if (lane == 0) {
        ctl->seg[i % kPlanned] = s;
        if (!more) ctl->seg[i % kPlanned].n = 0;
        mbar_arrive(bar_seg + 8 * (i % kPlanned));
      }
      __syncwarp();
      if (!more) break;
    }
  } else if (warp == 8) {
    // ---- copies ----
    const int shift = pool.page_shift;
    const int box_rows = min(1 << shift, kTilePos);
    const int boxes = kTilePos / box_rows;           // per 64 columns of a unit
    const int box = lane % boxes, panel = lane / boxes;
    const uint32_t dst = smem_u32(s_ring) + panel * Geo::kPanel + box * box_rows * 128;
    bool started = false;
    uint32_t n_read = 0;      // units
    const PrefixWork* seg;
    for (uint32_t si = 0; (seg = segment(si)); ++si) {
      const PrefixWork s = *seg;
      done_with(si);
      const int32_t* table = a.prefix.table + s.prefix * a.prefix.table_stride;
      for (int t = 0; t < s.n; ++t) {
        const long long unit = static_cast<long long>(s.unit0 + t) * kTilePos, pos = unit + box * box_rows;
        int64_t row = -1;
        bool bad = false;
        if (panel < D / 64 && pos < s.limit) {
          const int64_t r = find_slot(pool, table, a.prefix.table_stride, a.layer, pos);
          bad = r < 0;
          if (bad) raise(status, static_cast<int>(-r));
          else row = r + (static_cast<int64_t>(s.head) << shift);
        }
        const int n_copies = __popc(__ballot_sync(0xffffffffu, row >= 0));
        const bool edge = __any_sync(0xffffffffu, bad) || unit + kTilePos > s.limit;
        uint32_t seen = 0xffffffffu;
        if (edge) {
#pragma unroll 1
          for (int i = 0; i < 4; ++i) {
            const long long at = unit + 32 * i + lane;
            const uint32_t word = __ballot_sync(0xffffffffu, at < s.limit && find_slot(pool, table, a.prefix.table_stride, a.layer, at) >= 0);
            if (lane == i) seen = word;
          }
        }
#pragma unroll
        for (int is_v = 0; is_v < 2; ++is_v) {
          bool ok = true;
          if (copies_before >= kSlots) ok = wait_for(bar_empty + 8 * ring.slot, ring.phase ^ 1, give_up, status);
          ok = __all_sync(0xffffffffu, ok);
          if (ok) {
            if (!is_v && lane < 4) ctl->seen[n_read % 16][lane] = seen;
            if (!is_v && lane == 0) ctl->edge[n_read % 16] = edge;
            __syncwarp();
            if (lane == 0) mbar_expect(bar_full + 8 * ring.slot, static_cast<uint32_t>(n_copies) * box_rows * 128);
            __syncwarp();
            if (row >= 0) tma_load_2d(dst + ring.slot * Geo::kSlotBytes, is_v ? &maps.v : &maps.k, panel * 64, static_cast<int>(row), bar_full + 8 * ring.slot);
          }
          // Queries before the rest of the first places, as in tree attention.
          if (!started) wait_for(bar_first, 0, give_up, status);
          started = true;
          ring.step(1);
          if (copies_before < kSlots) ++copies_before;
        }
        ++n_read;
      }
    }
  } else if (warp == 9 || warp == 11) {
    // ---- products of a group ----
    // Blocks of 64 positions, two per unit, with a buffer of scores each: the scores of the group's next block are computed
    // while it has the exponentials of this one.  They follow the product with the probabilities of the block before last,
    // which lay in the same columns (one thread's products run in order).  A thread for each group: waiting for barriers,
    // issuing and committing takes it longer than the tensor core takes for its products (830 and 640 cycles a block).
    constexpr uint32_t kDescS = mma_f16_desc(kBf16, false, 128, kBlock), kDescO = mma_f16_desc(kBf16, true, 128, D);
    const uint32_t h = warp == 11, ring_addr = uniform(smem_u32(s_ring));
    const uint32_t t_s = uniform(tmem + h * kTilePos), t_o = uniform(tmem + 256 + h * D);
    const SmemOperand qq = smem_operand(uniform(smem_u32(s_q) + h * Geo::kQBytes), 16), k_all = smem_operand(ring_addr, 16), v_all = smem_operand(ring_addr, Geo::kPanel);
    const uint32_t my_s = bar_s + 16 * h, my_p = bar_p + 16 * h, my_pv = bar_pv + 16 * h;
    if (elect_one()) {
      uint32_t turn = 0, tiles = 0;      // blocks so far; tiles of queries
      bool ok = true;
      auto wait = [&](uint32_t bar, uint32_t parity) { ok = wait_for(bar, parity, give_up, status) && ok; };
      for (uint32_t si = 0;; ++si) {
        const uint32_t at = si % kPlanned;
        if (!wait_segment(bar_seg + 8 * at, si / kPlanned & 1)) {
          raise(status, kGaveUp);
          break;
        }
        const bool both = ctl->seg[at].both();
        const int n = ctl->seg[at].n, count = 2 * ctl->seg[at].units_of(h);
        if (n == 0) break;
        mbar_arrive(bar_seg_empty + 8 * at);
        if (count) wait(bar_q + 8 * h, tiles++ & 1);      // without a unit the group loads none
        // The places of the next scores' keys and of the next product's values.  Where only one group takes a unit it gives its
        // places back twice.
        RingPlace<kSlots> pk = ring, pv;
        if (!both && h) pk.step(2);
        pv = pk;
        pv.step(1);
        auto give_back = [&](uint32_t slot) {
          tc_commit(bar_empty + 8 * slot);
          if (!both) tc_commit(bar_empty + 8 * slot);
        };
        auto scores = [&](uint32_t half) {      // S = Q K^T
          if (!half) wait(bar_full + 8 * pk.slot, pk.phase);
          if (ok) {
            tc_fence_after();
            const SmemOperand kk = k_all + (pk.slot * Geo::kSlotBytes + half * (kBlock * 128));
#pragma unroll
            for (int k = 0; k < D / 16; ++k) mma_ss(t_s + kBlock * half, qq + (k / 4 * Geo::kPanel + k % 4 * 32), kk + (k / 4 * Geo::kPanel + k % 4 * 32), kDescS, k > 0);
            tc_commit(my_s + 8 * half);
            if (half) give_back(pk.slot);
          }
          if (half) pk.step(both ? 2 : 4);
        };
        auto outputs = [&](uint32_t half, bool add) {      // O += P V
          if (!half) wait(bar_full + 8 * pv.slot, pv.phase);
          wait(my_p + 8 * half, turn++ >> 1 & 1);
          if (ok) {
            tc_fence_after();
            const SmemOperand vv = v_all + (pv.slot * Geo::kSlotBytes + half * (kBlock * 128));
#pragma unroll
            for (int k = 0; k < kBlock / 16; ++k) mma_ts(t_o, t_s + kBlock * half + 8 * k, vv + k * (16 * 128), kDescO, add || k > 0);
            tc_commit(my_pv + 8 * half);
            if (half) give_back(pv.slot);
          }
          if (half) pv.step(both ? 2 : 4);
        };
        if (count) {
          scores(0);
          scores(1);
        }
        for (int j = 0; j < count; j += 2) {
          outputs(0, j > 0);
          if (j + 2 < count) scores(0);
          outputs(1, true);
          if (j + 2 < count) scores(1);
        }
        ring.skip(2 * n);
      }
    }
    __syncwarp();
  }
}

// ---- softmax: warps 0 to 7, a group of four per accumulator, one thread per row ----
template <int D>
template <typename T>
__device__ __forceinline__ void PrefixCta<D>::softmax() {
  using Geo = Geometry<D>;
  const int w = warp >> 2, quarter = warp & 3, r = quarter * 32 + lane;
  const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
  const uint32_t t_s = tmem + lanes + kTilePos * w, t_o = tmem + lanes + 256;
  const int group = a.group, n_q_heads = a.n_q_heads;
  uint32_t n_block = 0, unit_base = 0;      // blocks of this accumulator, units before
  bool loaded = false;                               // the queries of the segment are on their way already

  // Queries of a segment into this group's tile, in the background.  Its products have read what was there before: the
  // caller has seen the last scores.
  auto load_queries = [&](const PrefixWork& g) {
    const int from = g.both() ? w * 128 : 0;
    const long long r0 = g.first + g.row0 + from, t0 = div_small(r0, group);
    load_query_tile<T, D>(smem_u32(s_q) + w * Geo::kQBytes, Geo::kPanel, static_cast<const T*>(a.q) + (t0 * n_q_heads + g.head * group) * D, static_cast<int>(r0 - t0 * group),
                          group, static_cast<int64_t>(n_q_heads) * D, g.rows - from, r);
  };
  auto queries_ready = [&]() {
    asm volatile("cp.async.wait_all;" ::: "memory");
    fence_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive(bar_q + 8 * w);
  };

  const PrefixWork* seg;
  for (uint32_t si = 0; (seg = segment(si)); ++si) {
    const PrefixWork& s = *seg;
    const bool both = s.both();
    const int count = s.units_of(w);
    // A group loads the queries of the segments that it has units of, and of no other: what orders a phase of the barrier
    // behind the wait for the one before it is that the group has seen the scores between the two.
    if (!loaded && count) {
      load_queries(s);
      queries_ready();
    }
    if (si == 0 && lane == 0) mbar_arrive(bar_first);
    bool next_loads = false;
    auto load_next = [&]() {
      const PrefixWork* next = segment(si + 1);
      if (!next || !next->units_of(w)) return;
      load_queries(*next);
      next_loads = true;
    };
    const int in_tile = (both ? w * 128 : 0) + r;
    const bool live = in_tile - lane < s.rows, mine = in_tile < s.rows;
    float m = -INFINITY;
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll 1
    for (int i = 0; i < 2 * count; ++i, ++n_block) {
      const int t = both ? i >> 1 : (i & ~1) + w, half = i & 1;
      wait_for(bar_s + 16 * w + 8 * half, n_block >> 1 & 1, give_up, status);
      tc_fence_after();
      if (i == 2 * count - 1) load_next();
      const bool edge = *static_cast<volatile int*>(&ctl->edge[(unit_base + t) % 16]) != 0;
      const volatile uint32_t* seen = ctl->seen[(unit_base + t) % 16] + 2 * half;
      if (edge) {
        // Values at positions that are not seen may be anything, and 0 x NaN is NaN: clear them (each group for its own
        // product, which may come first).
        RingPlace<kSlots> pv = ring;
        pv.skip(2 * t + 1);
        wait_for(bar_full + 8 * pv.slot, pv.phase, give_up, status);
        if (!(seen[quarter & 1] >> lane & 1)) {
          uint8_t* row = s_ring + pv.slot * Geo::kSlotBytes + (kBlock * half + (r & 63)) * 128;
          constexpr int kHalfRow = D / 16;      // 16-byte pieces
#pragma unroll
          for (int c = 0; c < kHalfRow; ++c) {
            const int piece = (r >> 6) * kHalfRow + c;
            *reinterpret_cast<uint4*>(row + piece / 8 * Geo::kPanel + piece % 8 * 16) = make_uint4(0, 0, 0, 0);
          }
        }
        fence_async_smem();
      }
      if (live) {
        uint32_t sc[2][32];
#pragma unroll
        for (int c = 0; c < 2; ++c) tmem_load(sc[c], t_s + kBlock * half + 32 * c);
        tmem_wait_load();
#pragma unroll
        for (int c = 0; c < 2; ++c) tmem_use(sc[c]);
        if (edge) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const uint32_t word = seen[c];
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (!(word >> j & 1)) sc[c][j] = 0xff800000u;
          }
        }
        const float top = max_of(sc[1], max_of(sc[0], -INFINITY)) * a.scale_log2;
        if (__any_sync(0xffffffffu, top > m + kSlack)) {
          const float m_new = top > m + kSlack ? top - kHeadroom : m;
          const float f = m == m_new ? 1.f : ex2(m - m_new);
          m = m_new;
          sum.x *= f;
          sum.y *= f;
          if (i > 0) {
            // behind the last product into this accumulator (the one before it is done: these scores came behind it)
            wait_for(bar_pv + 16 * w + 8 * (half ^ 1), (n_block - 1) >> 1 & 1, give_up, status);
            tc_fence_after();
#pragma unroll 1
            for (int k = 0; k < D / 16; ++k) {
              uint32_t y[16];
              const uint32_t at = t_o + w * D + 16 * k;
              tmem_load(y, at);
              tmem_wait_load();
              tmem_use(y);
#pragma unroll
              for (int j = 0; j < 16; ++j) y[j] = __float_as_uint(__uint_as_float(y[j]) * f);
              tmem_store(at, y);
            }
            tmem_wait_store();
          }
        }
        const float2 scale = make_float2(a.scale_log2, a.scale_log2), shift = m == -INFINITY ? make_float2(0.f, 0.f) : make_float2(-m, -m);
        uint32_t packed[32];
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            float2 p = fma2(make_float2(__uint_as_float(sc[c][2 * j]), __uint_as_float(sc[c][2 * j + 1])), scale, shift);
            p = make_float2(ex2(p.x), ex2(p.y));
            sum = add2(sum, p);
            packed[16 * c + j] = Half2Of<T>::pack(p.x, p.y);
          }
        tmem_store(t_s + kBlock * half, packed);
        tmem_wait_store();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_p + 16 * w + 8 * half);
    }
    // ---- the segment's part ----
    if (next_loads) queries_ready();
    loaded = next_loads;
    unit_base += s.n;
    ring.skip(2 * s.n);
    if (count > 0) wait_for(bar_pv + 16 * w + 8, (n_block / 2 - 1) & 1, give_up, status);      // the last product
    tc_fence_after();
    const int64_t head = s.head, at = s.first + s.row0 + in_tile;
    const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x) + (s.kind == 2);
    float4* const dst = s.kind == 0 ? reinterpret_cast<float4*>(a.whole_o[0]) + head * (D / 4) * a.rows + at
                                    : reinterpret_cast<float4*>(a.part_o) + slot * (D / 4) * kPrefixRows + in_tile;
    const int64_t step = s.kind == 0 ? a.rows : kPrefixRows;
    float total = sum.x + sum.y, f0 = 1.f, f1 = 1.f;
    if (!both) {
      // Both groups hold parts of the same rows; each writes half of the columns.
      ctl->ml[w][r] = make_float2(m, total);
      tc_fence_before();
      asm volatile("bar.sync 3, 256;" ::: "memory");
      tc_fence_after();
      const float2 x = ctl->ml[0][r], y = ctl->ml[1][r];
      m = fmaxf(x.x, y.x);
      f0 = x.x == -INFINITY ? 0.f : ex2(x.x - m);
      f1 = y.x == -INFINITY ? 0.f : ex2(y.x - m);
      total = x.y * f0 + y.y * f1;
    }
    if (live) {
      constexpr int kChunk = 16;
#pragma unroll 1
      for (int c = both ? 0 : w * (D / 2 / kChunk); c < (both ? D : (w + 1) * (D / 2)) / kChunk; ++c) {
        uint32_t x[kChunk], y[kChunk];
        tmem_load(x, t_o + (both ? w * D : 0) + kChunk * c);
        if (!both) tmem_load(y, t_o + D + kChunk * c);
        tmem_wait_load();
        tmem_use(x);
        if (!both) {
          tmem_use(y);
          // an accumulator without a unit holds anything
#pragma unroll
          for (int j = 0; j < kChunk; ++j)
            x[j] = __float_as_uint((f0 == 0.f ? 0.f : __uint_as_float(x[j]) * f0) + (f1 == 0.f ? 0.f : __uint_as_float(y[j]) * f1));
        }
        if (mine) {
#pragma unroll
          for (int j = 0; j < kChunk / 4; ++j)
            dst[(c * (kChunk / 4) + j) * step] = make_float4(__uint_as_float(x[4 * j]), __uint_as_float(x[4 * j + 1]), __uint_as_float(x[4 * j + 2]), __uint_as_float(x[4 * j + 3]));
        }
      }
    }
    if (mine && (both || w == 0)) {
      if (s.kind == 0) a.whole_ml[0][head * a.rows + at] = make_float2(m, total);
      else a.part_ml[slot * kPrefixRows + in_tile] = make_float2(m, total);
      if (s.kind != 1) a.note[0][head * a.rows + at] = make_int2(blockIdx.x, s.last_worker - static_cast<int>(blockIdx.x) + 1);
    }
    tc_fence_before();
    if (!both) asm volatile("bar.sync 3, 256;" ::: "memory");      // the other group's next product overwrites what was read here
    done_with(si);
  }
}

// A wait that gave up may have left products or copies under way: they end before the memory is given back.
template <int D>
__device__ __forceinline__ void PrefixCta<D>::drain() {
  if (!ctl->give_up) return;
  if ((warp == 9 || warp == 11) && elect_one()) {
    tc_commit(smem_u32(&ctl->drained));
    for (int i = 0; i < (1 << 22) && !mbar_test(smem_u32(&ctl->drained), 0); ++i) {}
  }
  if (tid == 8 * 32)
    for (uint32_t p = 0; p < copies_before; ++p) {      // the last places
      ring.phase ^= ring.slot == 0;
      ring.slot = ring.slot == 0 ? kSlots - 1 : ring.slot - 1;
      for (int i = 0; i < (1 << 16) && !mbar_test(bar_full + 8 * ring.slot, ring.phase); ++i) {}
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(kPrefixThreads, 1) prefix_kernel(const __grid_constant__ Maps maps, const __grid_constant__ PrefixArgs a) {
  using Geo = Geometry<D>;
  using Own = OwnGeometry<D>;
  constexpr int kRingBytes = 2 * Geo::kQBytes + Geo::kSlots * Geo::kSlotBytes;
  static_assert(Own::kWarps * Own::kWarpBytes + sizeof(OwnControl) <= kRingBytes, "the streaming warps' memory fits where the ring is");
  extern __shared__ __align__(1024) uint8_t smem[];
  if (smem_u32(smem) & 1023) {      // never seen, as in tree attention; the joining kernel does without what is not there
    pdl_wait();
    if (threadIdx.x == 0) raise(a.pool.status, kGaveUp);
    return;
  }
  PrefixControl* const ctl = reinterpret_cast<PrefixControl*>(smem + kRingBytes);
  OwnControl* const own = reinterpret_cast<OwnControl*>(smem + Own::kWarps * Own::kWarpBytes);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_trigger();
  if (tid == 0) {
    for (int i = 0; i < 12; ++i) {
      mbar_init(smem_u32(&ctl->full[i]), 1);
      mbar_init(smem_u32(&ctl->empty[i]), 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&ctl->s_ready[2 * i]), 1);
      mbar_init(smem_u32(&ctl->s_ready[2 * i + 1]), 1);
      mbar_init(smem_u32(&ctl->p_ready[2 * i]), 4);
      mbar_init(smem_u32(&ctl->p_ready[2 * i + 1]), 4);
      mbar_init(smem_u32(&ctl->pv_done[2 * i]), 1);
      mbar_init(smem_u32(&ctl->pv_done[2 * i + 1]), 1);
      mbar_init(smem_u32(&ctl->q_ready[i]), 4);
    }
    for (int i = 0; i < kPlanned; ++i) {
      mbar_init(smem_u32(&ctl->seg_full[i]), 1);
      mbar_init(smem_u32(&ctl->seg_empty[i]), 11);
    }
    mbar_init(smem_u32(&ctl->q_first), 8);
    mbar_init(smem_u32(&ctl->drained), 2);
    ctl->give_up = 0;
    ctl->own_places = 0;
    tma_prefetch_map(&maps.k);
    tma_prefetch_map(&maps.v);
  }
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  if (warp == 9) tmem_alloc(smem_u32(&ctl->tmem), 512);
  pdl_wait();
  PrefixCursor cursor(a, lane);
  if (warp == 10) {
    cursor.add_up(blockIdx.x == 0);
    if (lane == 0) ctl->places = cursor.total;
  }
  if (a.own_cost) add_up_own(a, own, &ctl->own_places);
  fence_async_smem();      // the ring's copies follow where the sums were
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const long long places = ctl->places, own_places = ctl->own_places;
  const int n_prefix = prefix_workers(places, own_places, a.own_cost, gridDim.x);
  const bool is_prefix = static_cast<int>(blockIdx.x) < n_prefix;
  PrefixCta<D> cta{a, smem, ctl, n_prefix};
  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyRegisters));
    if (is_prefix) cta.template softmax<T>();
    else if (own_places > 0)
      own_share<T, D>(&maps.k_few, &maps.v_few, a, smem, own, &ctl->give_up, 8 * (static_cast<int>(blockIdx.x) - n_prefix) + warp, 8 * (static_cast<int>(gridDim.x) - n_prefix), own_places);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegisters));
    if (is_prefix) cta.template feed<T>(maps, cursor);
    if (warp == 10) write_places(a, blockIdx.x, gridDim.x);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (is_prefix) cta.drain();
  __syncthreads();
  if (warp == 9) tmem_free(ctl->tmem, 512);
}

// ---- joining the parts ----------------------------------------------------------------------------------------------
// blockIdx.y = KV head, blockIdx.x = 32 of its rows, one per lane; a warp has 4 columns, blockIdx.z 32 of them: reads of the
// parts are contiguous across the rows, eight parts of a thread in flight.  kOwnRows: the own positions' attention is done, its
// outputs lie as rows and its log-sum-exps behind one another.
template <typename Out, int D, bool kOwnRows>
__global__ void __launch_bounds__(256) prefix_join_kernel(const __grid_constant__ PrefixArgs a) {
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, quad = blockIdx.z * 8 + (threadIdx.x >> 5), group = a.group, head = blockIdx.y;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * 32 + lane;
  if (row >= a.rows) return;
  const int t = static_cast<int>(row / group);
  const int64_t at = static_cast<int64_t>(head) * a.rows + row;
  const int4 place = __ldcg(a.place + t);
  const int2 far = __ldcg(a.note[0] + at), near = kOwnRows ? make_int2(0, 1) : __ldcg(a.note[1] + at);
  if (!place.x) return;
  // Parts 0 .. n0 - 1 of the prefix, then n1 of the own positions
  int n0 = 0, n1 = near.y, x0 = 0, x1 = 0;
  const int w0 = far.x, w1 = near.x;
  if (place.z >= 0 && far.x >= 0 && far.y > 0 && far.y <= a.n_cta - far.x) {
    n0 = far.y;
    x0 = static_cast<int>((row - static_cast<int64_t>(place.z) * group) % kPrefixRows);
  }
  if (!kOwnRows) {
    if (near.x < 0 || near.y < 0 || near.y > 8 * a.n_cta - near.x) n1 = 0;
    x1 = static_cast<int>((row - static_cast<int64_t>(place.y) * group) % kFewRows);
  }
  const int64_t out_row = static_cast<int64_t>(t) * a.n_q_heads + head * group + (row - static_cast<int64_t>(t) * group);
  auto stats = [&](int i) {
    if (i < n0) return n0 == 1 ? __ldcg(a.whole_ml[0] + at) : __ldcg(a.part_ml + (2 * static_cast<int64_t>(w0 + i) + (i == 0)) * kPrefixRows + x0);
    i -= n0;
    if (kOwnRows) {
      const float lse = __ldcg(reinterpret_cast<const float*>(a.whole_ml[1]) + out_row);
      return make_float2(lse * kLog2e, lse == -INFINITY ? 0.f : 1.f);
    }
    return n1 == 1 ? __ldcg(a.whole_ml[1] + at) : __ldcg(a.own_part_ml + (2 * static_cast<int64_t>(w1 + i) + (i == 0)) * kFewRows + x1);
  };
  auto columns = [&](int i) {
    if (i < n0) {
      return n0 == 1 ? __ldcg(reinterpret_cast<const float4*>(a.whole_o[0]) + (static_cast<int64_t>(head) * (D / 4) + quad) * a.rows + row)
                     : __ldcg(reinterpret_cast<const float4*>(a.part_o) + ((2 * static_cast<int64_t>(w0 + i) + (i == 0)) * (D / 4) + quad) * kPrefixRows + x0);
    }
    i -= n0;
    if (kOwnRows) return __ldcg(reinterpret_cast<const float4*>(a.whole_o[1]) + out_row * (D / 4) + quad);
    return n1 == 1 ? __ldcg(reinterpret_cast<const float4*>(a.whole_o[1]) + (static_cast<int64_t>(head) * (D / 4) + quad) * a.rows + row)
                   : __ldcg(reinterpret_cast<const float4*>(a.own_part_o) + ((2 * static_cast<int64_t>(w1 + i) + (i == 0)) * (D / 4) + quad) * kFewRows + x1);
  };
  const int n = n0 + n1;
  float m = -INFINITY, total = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  constexpr int kFlight = 8;
  for (int i0 = 0; i0 < n; i0 += kFlight) {
    float2 ml[kFlight];
    float4 x[kFlight];
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      ml[j] = make_float2(-INFINITY, 0.f);
      if (i0 + j < n) {
        ml[j] = stats(i0 + j);
        x[j] = columns(i0 + j);
      }
    }
    float top = m;
#pragma unroll
    for (int j = 0; j < kFlight; ++j) top = fmaxf(top, ml[j].x);
    const float f = m == -INFINITY ? 0.f : ex2(m - top);
    m = top;
    total *= f;
    o.x *= f;
    o.y *= f;
    o.z *= f;
    o.w *= f;
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      if (ml[j].y == 0.f) continue;      // nothing was seen: its columns may be anything.  (All scores NaN: reference -infinity, sum NaN.)
      const float g = ex2(ml[j].x - m);
      total += ml[j].y * g;
      o.x += x[j].x * g;
      o.y += x[j].y * g;
      o.z += x[j].z * g;
      o.w += x[j].w * g;
    }
  }
  const float inv = inverse_of(total);
  store4(static_cast<Out*>(a.out) + out_row * D + 4 * quad, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
  if (a.lse && quad == 0) a.lse[out_row] = log_sum(m, total);
}

constexpr int64_t kAlign = 256;
int64_t padded(int64_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

template <typename T, typename Out, int D>
cudaError_t launch_prefix(const prima_paged& pool, const PrefixArgs& a, cudaStream_t st) {
  using Geo = Geometry<D>;
  constexpr size_t kSmem = 2 * Geo::kQBytes + Geo::kSlots * Geo::kSlotBytes + sizeof(PrefixControl);
  static_assert(kSmem <= 232448, "shared memory of a CTA");
  static bool done[kMaxDevices] = {};
  auto kernel = prefix_kernel<T, D>;
  cudaError_t e = allow_smem(kernel, kSmem, done);
  const Maps* maps = static_cast<const Maps*>(pool.maps);
  if (e == cudaSuccess) e = launch_pdl(kernel, dim3(pool.sm_count), dim3(kPrefixThreads), kSmem, st, *maps, a);
  if (e != cudaSuccess) return e;
  const dim3 grid(static_cast<unsigned>((a.rows + 31) / 32), static_cast<unsigned>(pool.cfg.n_kv_heads), D / 32);
  return launch_pdl(a.own_cost ? prefix_join_kernel<Out, D, false> : prefix_join_kernel<Out, D, true>, grid, dim3(256), 0, st, a);
}

}  // namespace
}  // namespace prima

using namespace prima;

extern "C" {

int64_t prima_prefix_attention_workspace(const prima_paged* p, int n_seq, int n_tok, int n_q_heads) {
  if (!p || n_seq < 1 || n_tok < 1 || n_q_heads < 1) return PRIMA_ERR_ARG;
  const int64_t rows = static_cast<int64_t>(n_tok) * n_q_heads, dim = p->cfg.head_dim, sm = p->sm_count;
  if (rows > 2147483647) return PRIMA_ERR_ARG;
  const int64_t whole = 2 * (padded(rows * dim * 4) + padded(rows * 8) + padded(rows * 8));
  const int64_t parts = padded(2 * sm * kPrefixRows * dim * 4) + padded(2 * sm * kPrefixRows * 8), own = padded(16 * sm * kFewRows * dim * 4) + padded(16 * sm * kFewRows * 8);
  return padded(static_cast<int64_t>(n_tok) * 16) + whole + parts + std::max(own, prima_tree_attention_workspace(p, n_seq, n_tok, n_q_heads));
}

int prima_prefix_attention(prima_paged* p, int layer, const prima_paged_batch* batch, const prima_prefix* prefix, const void* q, int n_q_heads,
                           float scale, void* out, int out_dtype, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  const int rc = check_batch(p, batch, "prima_prefix_attention");
  if (rc != PRIMA_OK) return rc;
  auto refuse = [](const char* what) {
    char msg[160];
    snprintf(msg, sizeof msg, "prima_prefix_attention: %s", what);
    return call_fail(PRIMA_ERR_ARG, msg);
  };
  const prima_paged_config& c = p->cfg;
  if (layer < 0 || layer >= c.n_layers) return refuse("layer out of range");
  if (!prefix || prefix->n_prefix < 1 || !prefix->seq_begin || !prefix->len || !prefix->table) return refuse("a prefix with seq_begin, len and table is needed");
  if (prefix->table_stride < 1 || prefix->table_stride > 2147483647) return refuse("the prefix's table_stride is out of range");
  if (!aligned_to(prefix->seq_begin, 4) || !aligned_to(prefix->len, 4) || !aligned_to(prefix->table, 4)) return refuse("an array of the prefix is not 4-byte aligned");
  if (!q || !out) return refuse("null q or out");
  if (n_q_heads < 1 || n_q_heads % c.n_kv_heads || n_q_heads / c.n_kv_heads > 64) return refuse("n_q_heads must be a multiple of n_kv_heads, at most 64 times it");
  if (static_cast<int64_t>(batch->n_tok) * n_q_heads > 2147483647) return refuse("n_tok * n_q_heads reaches 2^31");
  if (!(scale > 0.f) || std::isinf(scale)) return refuse("scale must be positive and finite");
  if (out_dtype != PRIMA_DT_F32 && out_dtype != c.dtype) return refuse("out_dtype is neither fp32 nor the cache's type");
  if (!aligned_to(q, 16) || !aligned_to(out, 16)) return refuse("q and out must be 16-byte aligned");
  if (!aligned_to(lse, 4)) return refuse("lse must be 4-byte aligned");
  if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < prima_prefix_attention_workspace(p, batch->n_seq, batch->n_tok, n_q_heads))
    return refuse("workspace too small or not 256-byte aligned");
  CallDevice dev(c.device);
  if (!dev.ok) return call_fail(PRIMA_ERR_CUDA, "cudaSetDevice failed");
  PrefixArgs a;
  a.pool = view_of(*p);
  a.b = view_of(*batch);
  const int group = n_q_heads / c.n_kv_heads;
  a.capacity = batch->table_stride << p->page_shift;
  a.layer = layer;
  a.n_q_heads = n_q_heads;
  a.group = group;
  a.group_inverse = small_inverse(group);
  a.scale_log2 = scale * kLog2e;
  a.q = q;
  a.out = out;
  a.lse = lse;
  a.prefix = {prefix->n_prefix, prefix->seq_begin, prefix->len, prefix->table, prefix->table_stride};
  a.shape = {c.n_kv_heads, prefix->table_stride << p->page_shift, kPrefixSegmentCost};
  a.rows = static_cast<int64_t>(batch->n_tok) * group;
  a.n_cta = p->sm_count;
  const int64_t rows = a.rows * c.n_kv_heads, dim = c.head_dim, sm = p->sm_count;
  char* ws = static_cast<char*>(workspace);
  auto take = [&](int64_t bytes) {
    char* at = ws;
    ws += padded(bytes);
    return at;
  };
  a.place = reinterpret_cast<int4*>(take(batch->n_tok * static_cast<int64_t>(16)));
  for (int i = 0; i < 2; ++i) {
    a.whole_o[i] = reinterpret_cast<float*>(take(rows * dim * 4));
    a.whole_ml[i] = reinterpret_cast<float2*>(take(rows * 8));
    a.note[i] = reinterpret_cast<int2*>(take(rows * 8));
  }
  a.part_o = reinterpret_cast<float*>(take(2 * sm * kPrefixRows * dim * 4));
  a.part_ml = reinterpret_cast<float2*>(take(2 * sm * kPrefixRows * 8));
  // Few rows of a sequence: its own positions are streamed beside the prefixes.  Many: tree attention's tensor-memory kernel
  // is the better one for them (its rule), and runs in front.  Beside against in front, 8 KV heads of 128: 16 sequences of 500
  // behind 4096 positions, 16 rows 31 and 45 us, 32 rows 42 and 54, 64 rows 69 and 70; 64 of 300 behind 2000, 32 rows 90 and
  // 103, 64 rows 160 and 140.  Own positions longer than the prefix, which the host does not know, would like it earlier: 16 of
  // 3000 behind 1000, 4 rows 73 and 65, 32 rows 122 and 91 (heads of 64: 59 and 66).
  a.own_cost = streams(a.b, group) ? (dim == 128 ? kOwnCost128 : kOwnCost64) : 0;
  if (a.own_cost) {
    a.own_part_o = reinterpret_cast<float*>(take(16 * sm * kFewRows * dim * 4));
    a.own_part_ml = reinterpret_cast<float2*>(take(16 * sm * kFewRows * 8));
  } else {
    a.own_part_o = nullptr;
    a.own_part_ml = nullptr;
    const int tree = prima_tree_attention(p, layer, batch, q, n_q_heads, scale, a.whole_o[1], PRIMA_DT_F32, reinterpret_cast<float*>(a.whole_ml[1]), ws,
                                          static_cast<char*>(workspace) + workspace_bytes - ws, stream);
    if (tree != PRIMA_OK) return tree;
  }
  using launcher = cudaError_t (*)(const prima_paged&, const PrefixArgs&, cudaStream_t);
  static const launcher table[2][2][2] = {{{launch_prefix<__half, float, 64>, launch_prefix<__half, float, 128>}, {launch_prefix<__half, __half, 64>, launch_prefix<__half, __half, 128>}},
                                          {{launch_prefix<__nv_bfloat16, float, 64>, launch_prefix<__nv_bfloat16, float, 128>},
                                           {launch_prefix<__nv_bfloat16, __nv_bfloat16, 64>, launch_prefix<__nv_bfloat16, __nv_bfloat16, 128>}}};
  const cudaError_t e = table[c.dtype == PRIMA_DT_BF16][out_dtype != PRIMA_DT_F32][c.head_dim == 128](*p, a, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? PRIMA_OK : call_cuda_fail(e, "prima_prefix_attention");
}

}  // extern "C"

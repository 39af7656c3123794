// Attention of a batch whose sequences share long prefixes.
//
//   out[t][h] = sum_j p_j v_j / sum_j p_j,   j over the prefix of t's sequence, its own positions and the rows that t sees
//
// The softmax of a row falls apart into parts (reference, sum, output) that are joined by their log-sum-exp.  What a
// prefix contributes is one large product for all rows that share it: with 256 rows of a KV head in a tile the cache of the
// prefix is read once per tile, and the tensor core, not the cache, bounds the work.  What the sequences' own positions
// contribute is a few rows over a short stretch each, bound by the cache.  One launch does both at once: some CTAs take the
// prefixes (tensor memory), the others the own positions (streaming, tree_device.cuh), in shares that cost about the same,
// so that the memory system works for the ones while the tensor cores work for the others.  prefix_join_kernel joins the
// parts in ascending order: the same lengths give the same bits.
//
// A CTA of the prefixes.  Warp 8 copies keys and values page by page into a ring, warp 9 issues the products, warp 10
// plans, and two groups of four warps have an accumulator of 128 rows each, one thread per row: a thread takes the 128
// scores of its row from tensor memory, maximum, exponentials, and puts the probabilities where the scores were.  The
// groups take turns at the tensor core: while it multiplies for one, the other has its exponentials.  Nothing is exchanged
// between threads; a row's reference moves only when a score exceeds the maximum that set it by a factor of 2^8, and
// then the thread rescales its output by itself (the scores of a unit come behind all earlier products of the accumulator).
// In a tile of at most 128 rows both groups have the same rows and every other unit, and join their halves at the end.
// Every row of a tile sees the whole prefix, so masks are only needed at its end and at bad pages, and are the same for
// all rows.  P is rounded to the cache's type as in tree attention.
#include <algorithm>
#include <cmath>
#include <cstdio>

#include "tree_device.cuh"

namespace prima {
namespace {

constexpr int kGroupThreads = 128, kPrefixThreads = 3 * kGroupThreads;
constexpr int kPlanned = 4;            // segments ahead
constexpr int kPrefixSegmentCost = 4;  // in places
// Registers of a thread: the two groups that hold scores (or the fragments of the streaming body), and the third one.  Their
// sum is what the block is launched with: 384 x 168 = 256 x 208 + 128 x 88.
constexpr int kManyRegisters = 208, kFewRegisters = 88;

// What a unit of 128 own positions costs, in eighths of a prefix's place.
constexpr int kOwnCost128 = 16, kOwnCost64 = 8;

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
  TreeArgs own;              // part_o, part_ml: of the streaming workers
  PrefixView prefix;
  PrefixShape shape;
  int own_cost;
  int64_t rows;              // n_tok * group
  int n_cta;                 // workers there are at most: of the prefixes; twice as many stream
  float* whole_o[2];
  float2* whole_ml[2];       // [head][rows]: reference, sum
  int2* note[2];             // [head][rows]: first worker, number of parts
  float* part_o;             // of the prefixes' workers
  float2* part_ml;
};

struct PrefixWork {
  int prefix, head, row0, rows;        // rows row0 .. row0 + rows - 1 of the (prefix, KV head)
  long long first;                     // row R of the first of all
  int unit0, n;
  int kind;                            // 0: whole; 1: continues; 2: begins here and goes on
  int last_worker;
  long long limit;                     // positions that are seen
  __device__ __forceinline__ bool both() const { return rows > kPrefixRows / 2; }      // accumulators per unit
};

struct PrefixControl {
  unsigned long long full[12], empty[12], s_ready[2], p_ready[4], pv_done[2], q_ready[2], q_first, drained;
  unsigned long long seg_full[kPlanned], seg_empty[kPlanned];
  PrefixWork seg[kPlanned];
  long long places, own_places;
  uint32_t tmem;
  int give_up;
  int edge[16];                        // of the last units: not all positions are seen (the ring holds at most six)
  uint32_t seen[16][4];
  union {
    float2 ml[2][128];                 // a group's reference and sum, for the other one
    struct {                           // of the streaming groups, in the CTAs that have these
      Segment seg[2];
      float2 ml[2][4][16];
    } own;
  };
};

// The range of a prefix: rows of the step that share it, or none.  Reads device memory; false: the numbers are bad.
struct PrefixRange {
  int first = 0, rows = 0, len = 0;    // rows: of the step
};
__device__ __forceinline__ bool prefix_range(const PrefixArgs& a, int p, PrefixRange* out) {
  const BatchView& b = a.own.b;
  const int s0 = __ldg(a.prefix.seq_begin + p), s1 = __ldg(a.prefix.seq_begin + p + 1), len = __ldg(a.prefix.len + p);
  *out = PrefixRange();
  if (s0 < 0 || s1 < s0 || s1 > b.n_seq || len < 0) return false;
  if (s1 == s0) return true;
  const int first = __ldg(b.row_begin + s0), end = __ldg(b.row_begin + s1);
  if (first < 0 || end < first || end > b.n_tok) return false;
  out->first = first;
  out->rows = end - first;
  out->len = len;
  return true;
}

// Walks the share of a prefixes' worker, 32 prefixes at a time, one per lane.
struct PrefixCursor {
  const PrefixArgs& a;
  const int lane, worker, n_workers;
  const long long total;
  long long u, u_end;
  int p0 = 0;                          // first prefix of the window
  long long window = 0, before = 0, per_head = 0, places = 0;
  PrefixRange range;

  __device__ void load(long long in_front) {
    per_head = 0;
    range = PrefixRange();
    if (p0 + lane < a.prefix.n) {
      prefix_range(a, p0 + lane, &range);
      per_head = prefix_places(a.shape, static_cast<long long>(range.rows) * a.own.shape.group, prefix_units(a.shape, range.len));
    }
    places = per_head * a.shape.n_kv_heads;
    long long x = places;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    before = in_front + x - places;
    window = in_front + __shfl_sync(0xffffffffu, x, 31);
  }
  __device__ PrefixCursor(const PrefixArgs& args, int lane_, int worker_, int n_workers_, long long total_)
      : a(args), lane(lane_), worker(worker_), n_workers(n_workers_), total(total_) {
    const TreeShares shares = tree_shares(total, n_workers);
    u = tree_share_begin(shares, worker);
    u_end = tree_share_begin(shares, worker + 1);
    load(0);
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
      const long long rows = static_cast<long long>(n_rows) * a.own.shape.group, units = prefix_units(a.shape, len);
      const PrefixSegment t = prefix_segment(a.shape, rows, units, mine, u - in_front, u_end - in_front);
      s->prefix = p0 + src;
      s->head = t.head;
      s->row0 = static_cast<int>(t.row_tile * kPrefixRows);
      s->rows = static_cast<int>(min(rows - s->row0, static_cast<long long>(kPrefixRows)));
      s->first = static_cast<long long>(first) * a.own.shape.group;
      s->unit0 = t.unit0;
      s->n = t.unit1 - t.unit0;
      s->kind = t.unit0 ? 1 : t.unit1 < units ? 2 : 0;
      s->last_worker = s->kind == 2 ? tree_cta_of(tree_shares(total, n_workers), in_front + t.last) : worker;
      s->limit = min(static_cast<long long>(len), static_cast<long long>(a.shape.capacity));
      u += t.places;
      if (s->n) return true;
    }
    return false;
  }
};

// The results of the streaming groups.
struct OwnEnv {
  static constexpr bool kFinal = false;
  const PrefixArgs& a;
  int tid, worker, n_workers;
  bool reports;
  uint8_t* smem;
  Segment* seg;
  float2 (*ml)[16];
  int barrier, dim;
  __device__ __forceinline__ void sync() const { asm volatile("bar.sync %0, 128;" ::"r"(barrier) : "memory"); }
  // Row x of the segment as row R of its KV head
  __device__ __forceinline__ int64_t row_of(const Segment& s, int x) const {
    return static_cast<int64_t>(s.head) * a.rows + static_cast<int64_t>(s.first) * a.own.shape.group + s.row0 + x;
  }
  __device__ __forceinline__ void whole(const Segment& s, int x, int64_t, int quad, float4 y, float top, float total) const {
    const int64_t row = row_of(s, x), head = s.head;
    reinterpret_cast<float4*>(a.whole_o[1])[(head * (dim / 4) + quad) * a.rows + (row - head * a.rows)] = y;
    if (quad == 0) {
      a.whole_ml[1][row] = make_float2(top, total);
      a.note[1][row] = make_int2(worker, 1);
    }
  }
  __device__ __forceinline__ void begins(const Segment& s, int x) const { a.note[1][row_of(s, x)] = make_int2(worker, s.last_worker - worker + 1); }
  __device__ __forceinline__ void ends(const Cursor&, const Segment&) const {}
};
template <int D> struct OwnStream { static constexpr int kStages = D == 128 ? 3 : 6; };

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
  int* const status = a.own.pool.status;
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
  template <typename T> __device__ __forceinline__ void feed(const CUtensorMap* k_map, const CUtensorMap* v_map);
  template <typename T> __device__ __forceinline__ void softmax();
  __device__ __forceinline__ void drain();
};

// Warps 8 to 10.
template <int D>
template <typename T>
__device__ __forceinline__ void PrefixCta<D>::feed(const CUtensorMap* k_map, const CUtensorMap* v_map) {
  using Geo = Geometry<D>;
  constexpr bool kBf16 = !__is_same(T, __half);
  const PoolView& pool = a.own.pool;
  if (warp == 10) {
    // ---- the plan ----
    PrefixCursor cursor(a, lane, blockIdx.x, n_workers, ctl->places);
    PrefixWork s;
    for (uint32_t i = 0;; ++i) {
      const bool more = cursor.next(&s);
      if (i >= kPlanned) wait_segment(bar_seg_empty + 8 * (i % kPlanned), (i / kPlanned - 1) & 1);
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
          const int64_t r = find_slot(pool, table, a.prefix.table_stride, a.own.layer, pos);
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
            const uint32_t word = __ballot_sync(0xffffffffu, at < s.limit && find_slot(pool, table, a.prefix.table_stride, a.own.layer, at) >= 0);
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
            if (row >= 0) tma_load_2d(dst + ring.slot * Geo::kSlotBytes, is_v ? v_map : k_map, panel * 64, static_cast<int>(row), bar_full + 8 * ring.slot);
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
  } else if (warp == 9) {
    // ---- products ----
    constexpr uint32_t kDescS = mma_f16_desc(kBf16, false, 128, kTilePos), kDescO = mma_f16_desc(kBf16, true, 128, D);
    const uint32_t u_tmem = uniform(tmem);
    const uint32_t ring_addr = uniform(smem_u32(s_ring)), q_addr = uniform(smem_u32(s_q));
    const SmemOperand k_all = smem_operand(ring_addr, 16), v_all = smem_operand(ring_addr, Geo::kPanel);
    uint32_t turns[2] = {0, 0};      // probabilities of an accumulator so far
    const PrefixWork* seg;
    for (uint32_t si = 0; (seg = segment(si)); ++si) {
      const uint32_t both = uniform(seg->rows) > kPrefixRows / 2 ? 1 : 0;
      const int count = uniform(seg->n) << both;
      done_with(si);
      bool ok = wait_for(bar_q, si & 1, give_up, status);
      ok = wait_for(bar_q + 8, si & 1, give_up, status) && ok;
      RingPlace<kSlots> pk = ring, pv = ring;      // of the unit whose keys, whose values are due
      pv.step(1);
      // Sub-unit i: accumulator i % 2 and unit i, or unit i / 2 where a unit takes both
      auto scores = [&](int i) {                   // S = Q K^T
        const uint32_t h = i & 1;
        const bool last = !both || h == 1;
        if (!both || h == 0) ok = wait_for(bar_full + 8 * pk.slot, pk.phase, give_up, status) && ok;
        tc_fence_after();
        if (__all_sync(0xffffffffu, ok) && elect_one()) {
          const SmemOperand qq = smem_operand(q_addr + h * Geo::kQBytes, 16), kk = k_all + pk.slot * Geo::kSlotBytes;
#pragma unroll
          for (int k = 0; k < D / 16; ++k) mma_ss(u_tmem + h * kTilePos, qq + (k / 4 * Geo::kPanel + k % 4 * 32), kk + (k / 4 * Geo::kPanel + k % 4 * 32), kDescS, k > 0);
          tc_commit(bar_s + 8 * h);
          if (last) tc_commit(bar_empty + 8 * pk.slot);
        }
        __syncwarp();
        if (last) pk.step(2);
      };
      for (int i = 0; i < min(count, 2); ++i) scores(i);
      for (int i = 0; i < count; ++i) {
        const uint32_t h = i & 1, phase = (h ? turns[1]++ : turns[0]++) & 1;
        const bool first = i < 2, last = !both || h == 1;
        if (!both || h == 0) ok = wait_for(bar_full + 8 * pv.slot, pv.phase, give_up, status) && ok;
        // O += P V, each half of the positions when its P is there; the first product of a segment overwrites O, which its
        // group has read by then (its P says so)
        const SmemOperand vv = v_all + pv.slot * Geo::kSlotBytes;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          ok = wait_for(bar_p + 16 * h + 8 * w, phase, give_up, status) && ok;
          tc_fence_after();
          if (__all_sync(0xffffffffu, ok) && elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              mma_ts(u_tmem + 256 + h * D, u_tmem + h * kTilePos + 32 * w + 8 * k, vv + (4 * w + k) * (16 * 128), kDescO, !first || w > 0 || k > 0);
            if (w) {
              if (i + 2 >= count) tc_commit(bar_pv + 8 * h);
              if (last) tc_commit(bar_empty + 8 * pv.slot);
            }
          }
          __syncwarp();
        }
        if (last) pv.step(2);
        // P lies over S: the next scores are written behind the product that reads it (one warp's products run in order)
        if (i + 2 < count) scores(i + 2);
      }
      ring.skip(2 * (count >> both));
    }
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
  const int group = a.own.shape.group, n_q_heads = a.own.n_q_heads;
  uint32_t n_sub = 0, n_seg = 0, unit_base = 0;      // sub-units of this accumulator, segments that had some, units before
  bool loaded = false;                               // the queries of the segment are on their way already

  // Queries of a segment into this group's tile, in the background.  Its products have read what was there before: the
  // caller has seen the last scores.
  auto load_queries = [&](const PrefixWork& g) {
    constexpr int kPieces = D / 8;
    const int from = g.both() ? w * 128 : 0;
    const long long r0 = g.first + g.row0 + from;
    const long long t0 = r0 / group;
    const int rem0 = static_cast<int>(r0 - t0 * group);
#pragma unroll 4
    for (int idx = r; idx < 128 * kPieces; idx += 128) {
      const int row = idx / kPieces, piece = idx % kPieces;
      const bool there = from + row < g.rows;
      const int y = there ? rem0 + row : rem0, t = small_div(y, a.own.group_inverse);
      copy16(smem_u32(s_q) + w * Geo::kQBytes + piece / 8 * Geo::kPanel + row * 128 + ((piece % 8) ^ (row & 7)) * 16,
             static_cast<const T*>(a.own.q) + ((t0 + t) * n_q_heads + g.head * group + (y - t * group)) * D + piece * 8, there);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
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
    if (!loaded) {
      load_queries(s);
      queries_ready();
      if (si == 0 && lane == 0) mbar_arrive(bar_first);
    }
    bool next_loads = false;
    auto load_next = [&]() {
      const PrefixWork* next = segment(si + 1);
      if (!next) return;
      load_queries(*next);
      next_loads = true;
    };
    const bool both = s.both();
    const int count = both ? s.n : (s.n + 1 - w) >> 1;
    const int in_tile = (both ? w * 128 : 0) + r;
    const bool live = in_tile - lane < s.rows, mine = in_tile < s.rows;
    float m = -INFINITY;
    float2 sum = make_float2(0.f, 0.f);
    // (without a unit the next queries wait for the other group's end: the barrier of the queries may be one phase ahead of
    // the warp that issues the products, not two)
#pragma unroll 1
    for (int i = 0; i < count; ++i, ++n_sub) {
      const int t = both ? i : 2 * i + w;
      wait_for(bar_s + 8 * w, n_sub & 1, give_up, status);
      tc_fence_after();
      if (i == count - 1) load_next();
      const bool edge = *static_cast<volatile int*>(&ctl->edge[(unit_base + t) % 16]) != 0;
      const volatile uint32_t* seen = ctl->seen[(unit_base + t) % 16];
      if (edge && (!both || w == 0)) {
        // Values at positions that are not seen may be anything, and 0 x NaN is NaN: clear them.
        RingPlace<kSlots> pv = ring;
        pv.skip(2 * t + 1);
        wait_for(bar_full + 8 * pv.slot, pv.phase, give_up, status);
        if (!(seen[quarter] >> lane & 1)) {
          uint8_t* row = s_ring + pv.slot * Geo::kSlotBytes + r * 128;
#pragma unroll
          for (int c = 0; c < D / 8; ++c) *reinterpret_cast<uint4*>(row + c / 8 * Geo::kPanel + c % 8 * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_async_smem();
      }
      uint32_t sc[4][32];
      float2 scale, shift;
      if (live) {
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_load(sc[c], t_s + 32 * c);
        tmem_wait_load();
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_use(sc[c]);
        if (edge) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint32_t word = seen[c];
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (!(word >> j & 1)) sc[c][j] = 0xff800000u;
          }
        }
        const float top = fmaxf(max_of(sc[1], max_of(sc[0], -INFINITY)), max_of(sc[3], max_of(sc[2], -INFINITY))) * a.own.scale_log2;
        if (__any_sync(0xffffffffu, top > m + kSlack)) {
          const float m_new = top > m + kSlack ? top - kHeadroom : m;
          const float f = m == m_new ? 1.f : ex2(m - m_new);
          m = m_new;
          sum.x *= f;
          sum.y *= f;
          if (i > 0) {
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
        scale = make_float2(a.own.scale_log2, a.own.scale_log2);
        shift = m == -INFINITY ? make_float2(0.f, 0.f) : make_float2(-m, -m);
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (live) {
          uint32_t packed[32];
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              float2 p = fma2(make_float2(__uint_as_float(sc[2 * half + c][2 * j]), __uint_as_float(sc[2 * half + c][2 * j + 1])), scale, shift);
              p = make_float2(ex2(p.x), ex2(p.y));
              sum = add2(sum, p);
              packed[16 * c + j] = Half2Of<T>::pack(p.x, p.y);
            }
          tmem_store(t_s + 32 * half, packed);
          tmem_wait_store();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_p + 16 * w + 8 * half);
      }
    }
    // ---- the segment's part ----
    if (next_loads) queries_ready();
    loaded = next_loads;
    unit_base += s.n;
    ring.skip(2 * s.n);
    if (count > 0) {
      wait_for(bar_pv + 8 * w, n_seg & 1, give_up, status);
      ++n_seg;
    }
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
  if (tid == 9 * 32) {
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
__global__ void __launch_bounds__(kPrefixThreads, 1) prefix_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                                                                   const __grid_constant__ PrefixArgs a) {
  using Geo = Geometry<D>;
  using Stream = StreamGeometry<D, OwnStream<D>::kStages>;
  constexpr int kRingBytes = 2 * Geo::kQBytes + Geo::kSlots * Geo::kSlotBytes;
  static_assert(2 * Stream::kBytes <= kRingBytes, "two streaming groups fit where the ring is");
  extern __shared__ __align__(1024) uint8_t smem[];
  if (smem_u32(smem) & 1023) {      // never seen, as in tree attention; the joining kernel does without what is not there
    pdl_wait();
    if (threadIdx.x == 0) raise(a.own.pool.status, kGaveUp);
    return;
  }
  PrefixControl* ctl = reinterpret_cast<PrefixControl*>(smem + kRingBytes);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_trigger();
  if (tid == 0) {
    for (int i = 0; i < 12; ++i) {
      mbar_init(smem_u32(&ctl->full[i]), 1);
      mbar_init(smem_u32(&ctl->empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&ctl->s_ready[i]), 1);
      mbar_init(smem_u32(&ctl->p_ready[2 * i]), 4);
      mbar_init(smem_u32(&ctl->p_ready[2 * i + 1]), 4);
      mbar_init(smem_u32(&ctl->pv_done[i]), 1);
      mbar_init(smem_u32(&ctl->q_ready[i]), 4);
    }
    for (int i = 0; i < kPlanned; ++i) {
      mbar_init(smem_u32(&ctl->seg_full[i]), 1);
      mbar_init(smem_u32(&ctl->seg_empty[i]), 10);
    }
    mbar_init(smem_u32(&ctl->q_first), 8);
    mbar_init(smem_u32(&ctl->drained), 1);
    ctl->give_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma_prefetch_map(&k_map);
    tma_prefetch_map(&v_map);
  }
  if (warp == 9) tmem_alloc(smem_u32(&ctl->tmem), 512);
  pdl_wait();
  if (warp == 10) {      // places of all prefixes
    long long n = 0;
    for (int p = lane; p < a.prefix.n; p += 32) {
      PrefixRange range;
      const bool ok = prefix_range(a, p, &range);
      n += prefix_places(a.shape, static_cast<long long>(range.rows) * a.own.shape.group, prefix_units(a.shape, range.len)) * a.own.shape.n_kv_heads;
      if (blockIdx.x == 0) {
        if (!ok) raise(a.own.pool.status, kBadRows);
        else if (range.rows && range.len > a.shape.capacity) raise(a.own.pool.status, kBadSlot);
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
    if (lane == 0) ctl->places = n;
  } else if (warp == 11) {      // and of the own positions
    const long long n = a.own_cost ? Cursor(a.own, lane, 0, 1, blockIdx.x == 0).total : 0;
    if (lane == 0) ctl->own_places = n;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const long long places = ctl->places, own_places = ctl->own_places;
  const int n_prefix = prefix_workers(places, own_places, a.own_cost, gridDim.x);
  const bool is_prefix = static_cast<int>(blockIdx.x) < n_prefix;
  PrefixCta<D> cta{a, smem, ctl, n_prefix};
  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyRegisters));
    if (is_prefix) {
      cta.template softmax<T>();
    } else if (own_places > 0) {
      const int g = warp >> 2, worker = 2 * (static_cast<int>(blockIdx.x) - n_prefix) + g;
      stream_share<T, D, OwnStream<D>::kStages>(a.own, OwnEnv{a, tid & 127, worker, 2 * (static_cast<int>(gridDim.x) - n_prefix), false, smem + g * Stream::kBytes,
                                                              &ctl->own.seg[g], ctl->own.ml[g], 1 + g, D});
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegisters));
    if (is_prefix) cta.template feed<T>(&k_map, &v_map);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (is_prefix) cta.drain();
  __syncthreads();
  if (warp == 9) tmem_free(ctl->tmem, 512);
}

// ---- joining the parts ----------------------------------------------------------------------------------------------
// blockIdx.y = KV head, blockIdx.x = 32 of its rows, one per lane; the eight warps share the columns, four at a time, so
// that reads of the parts are contiguous across the rows.  kOwnRows: the own positions' attention is done, its outputs lie
// as rows and its log-sum-exps behind one another.
template <typename Out, int D, bool kOwnRows>
__global__ void __launch_bounds__(256) prefix_join_kernel(const __grid_constant__ PrefixArgs a) {
  pdl_trigger();
  pdl_wait();
  const BatchView& b = a.own.b;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, group = a.own.shape.group, head = blockIdx.y;
  const int64_t first_row = static_cast<int64_t>(blockIdx.x) * 32, row = first_row + lane;
  const int t0 = static_cast<int>(first_row / group);
  const int t = t0 + static_cast<int>(first_row - static_cast<int64_t>(t0) * group + lane) / group;
  // The sequence of the row and its prefix: the warp looks the first row's up, the others are not far behind.
  int s = seq_of_row(b, min(t0, b.n_tok - 1), lane), p = 0;
  while (s < b.n_seq && __ldg(b.row_begin + s + 1) <= t) ++s;
  const int s_first = __shfl_sync(0xffffffffu, s, 0);
  for (int i = lane; i < a.prefix.n; i += 32) p += __ldg(a.prefix.seq_begin + i + 1) <= s_first ? 1 : 0;
  p = __reduce_add_sync(0xffffffffu, p);
  if (t >= b.n_tok || s >= b.n_seq) return;
  const int first = __ldg(b.row_begin + s);
  if (first < 0 || t < first || __ldg(b.row_begin + s + 1) > b.n_tok || __ldg(b.ctx_len + s) < 0) return;
  while (p < a.prefix.n && __ldg(a.prefix.seq_begin + p + 1) <= s) ++p;

  // Parts 0 .. n0 - 1 of the prefix, then n1 of the own positions: addresses of their first columns and statistics
  const int64_t at = static_cast<int64_t>(head) * a.rows + row;
  int n0 = 0, n1 = 1, w0 = 0, w1 = 0, x0 = 0, x1 = 0;
  PrefixRange range;
  if (p < a.prefix.n && __ldg(a.prefix.seq_begin + p) <= s && prefix_range(a, p, &range) && prefix_units(a.shape, range.len) > 0) {
    const int2 note = __ldcg(a.note[0] + at);
    if (note.x >= 0 && note.y > 0 && note.y <= a.n_cta - note.x) {
      w0 = note.x;
      n0 = note.y;
    }
    x0 = static_cast<int>((row - static_cast<int64_t>(range.first) * group) % kPrefixRows);
  }
  if (!kOwnRows) {
    const int2 note = __ldcg(a.note[1] + at);
    w1 = note.x;
    n1 = note.x >= 0 && note.y > 0 && note.y <= 2 * a.n_cta - note.x ? note.y : 0;
    x1 = static_cast<int>((row - static_cast<int64_t>(first) * group) % 16);
  }
  const int64_t out_row = static_cast<int64_t>(t) * a.own.n_q_heads + head * group + (row - static_cast<int64_t>(t) * group);
  auto stats = [&](int i) {
    if (i < n0) return n0 == 1 ? __ldcg(a.whole_ml[0] + at) : __ldcg(a.part_ml + (2 * static_cast<int64_t>(w0 + i) + (i == 0)) * kPrefixRows + x0);
    i -= n0;
    if (kOwnRows) {
      const float lse = __ldcg(reinterpret_cast<const float*>(a.whole_ml[1]) + out_row);
      return make_float2(lse * kLog2e, lse == -INFINITY ? 0.f : 1.f);
    }
    return n1 == 1 ? __ldcg(a.whole_ml[1] + at) : __ldcg(a.own.part_ml + (2 * static_cast<int64_t>(w1 + i) + (i == 0)) * 16 + x1);
  };
  auto columns = [&](int i, int quad) {
    if (i < n0) {
      return n0 == 1 ? __ldcg(reinterpret_cast<const float4*>(a.whole_o[0]) + (static_cast<int64_t>(head) * (D / 4) + quad) * a.rows + row)
                     : __ldcg(reinterpret_cast<const float4*>(a.part_o) + ((2 * static_cast<int64_t>(w0 + i) + (i == 0)) * (D / 4) + quad) * kPrefixRows + x0);
    }
    i -= n0;
    if (kOwnRows) return __ldcg(reinterpret_cast<const float4*>(a.whole_o[1]) + out_row * (D / 4) + quad);
    return n1 == 1 ? __ldcg(reinterpret_cast<const float4*>(a.whole_o[1]) + (static_cast<int64_t>(head) * (D / 4) + quad) * a.rows + row)
                   : __ldcg(reinterpret_cast<const float4*>(a.own.part_o) + ((2 * static_cast<int64_t>(w1 + i) + (i == 0)) * (D / 4) + quad) * 16 + x1);
  };
  const int n = n0 + n1;
  constexpr int kQuads = D / 32;      // of a warp
  float m = -INFINITY, total = 0.f;
  float4 o[kQuads];
#pragma unroll
  for (int k = 0; k < kQuads; ++k) o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
  constexpr int kFlight = 4;
  for (int i0 = 0; i0 < n; i0 += kFlight) {
    float2 ml[kFlight];
    float4 x[kFlight][kQuads];
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      ml[j] = make_float2(-INFINITY, 0.f);
      if (i0 + j < n) {
        ml[j] = stats(i0 + j);
#pragma unroll
        for (int k = 0; k < kQuads; ++k) x[j][k] = columns(i0 + j, warp * kQuads + k);
      }
    }
    float top = m;
#pragma unroll
    for (int j = 0; j < kFlight; ++j) top = fmaxf(top, ml[j].x);
    const float f = m == -INFINITY ? 0.f : ex2(m - top);
    m = top;
    total *= f;
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
      o[k].x *= f;
      o[k].y *= f;
      o[k].z *= f;
      o[k].w *= f;
    }
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      if (ml[j].x == -INFINITY) continue;      // nothing was seen: its columns may be anything
      const float g = ex2(ml[j].x - m);
      total += ml[j].y * g;
#pragma unroll
      for (int k = 0; k < kQuads; ++k) {
        o[k].x += x[j][k].x * g;
        o[k].y += x[j][k].y * g;
        o[k].z += x[j][k].z * g;
        o[k].w += x[j][k].w * g;
      }
    }
  }
  const float inv = inverse_of(total);
  Out* const dst = static_cast<Out*>(a.own.out) + out_row * D;
#pragma unroll
  for (int k = 0; k < kQuads; ++k)
    store4(dst + 4 * (warp * kQuads + k), make_float4(o[k].x * inv, o[k].y * inv, o[k].z * inv, o[k].w * inv));
  if (a.own.lse && warp == 0) a.own.lse[out_row] = log_sum(m, total);
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
  if (e == cudaSuccess) e = launch_pdl(kernel, dim3(pool.sm_count), dim3(kPrefixThreads), kSmem, st, maps->k, maps->v, a);
  if (e != cudaSuccess) return e;
  const dim3 grid(static_cast<unsigned>((a.rows + 31) / 32), static_cast<unsigned>(pool.cfg.n_kv_heads));
  return launch_pdl(a.own_cost ? prefix_join_kernel<Out, D, false> : prefix_join_kernel<Out, D, true>, grid, dim3(256), 0, st, a);
}

}  // namespace
}  // namespace prima

using namespace prima;

extern "C" {

int64_t prima_prefix_attention_workspace(const prima_paged* p, int n_seq, int n_tok, int n_q_heads) {
  if (!p || n_seq < 1 || n_tok < 1 || n_q_heads < 1) return PRIMA_ERR_ARG;
  const int64_t rows = static_cast<int64_t>(n_tok) * n_q_heads, dim = p->cfg.head_dim, sm = p->sm_count;
  const int64_t whole = 2 * (padded(rows * dim * 4) + padded(rows * 8) + padded(rows * 8));
  const int64_t parts = padded(2 * sm * kPrefixRows * dim * 4) + padded(2 * sm * kPrefixRows * 8) + padded(4 * sm * 16 * dim * 4) + padded(4 * sm * 16 * 8);
  return whole + std::max(parts, parts - padded(4 * sm * 16 * dim * 4) - padded(4 * sm * 16 * 8) + prima_tree_attention_workspace(p, n_seq, n_tok, n_q_heads));
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
  if (!(scale > 0.f) || std::isinf(scale)) return refuse("scale must be positive and finite");
  if (out_dtype != PRIMA_DT_F32 && out_dtype != c.dtype) return refuse("out_dtype is neither fp32 nor the cache's type");
  if (!aligned_to(q, 16) || !aligned_to(out, 16)) return refuse("q and out must be 16-byte aligned");
  if (!aligned_to(lse, 4)) return refuse("lse must be 4-byte aligned");
  if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < prima_prefix_attention_workspace(p, batch->n_seq, batch->n_tok, n_q_heads))
    return refuse("workspace too small or not 256-byte aligned");
  CallDevice dev(c.device);
  if (!dev.ok) return call_fail(PRIMA_ERR_CUDA, "cudaSetDevice failed");
  PrefixArgs a;
  TreeArgs& own = a.own;
  own.pool = view_of(*p);
  own.b = view_of(*batch);
  const int group = n_q_heads / c.n_kv_heads;
  own.shape = {c.n_kv_heads, group, batch->mask == nullptr, batch->table_stride << p->page_shift, kStreamSegmentCost, 16};
  own.layer = layer;
  own.n_q_heads = n_q_heads;
  own.scale_log2 = scale * kLog2e;
  own.group_inverse = small_inverse(group);
  own.q = q;
  own.out = out;
  own.lse = lse;
  own.notes = nullptr;
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
  for (int i = 0; i < 2; ++i) {
    a.whole_o[i] = reinterpret_cast<float*>(take(rows * dim * 4));
    a.whole_ml[i] = reinterpret_cast<float2*>(take(rows * 8));
    a.note[i] = reinterpret_cast<int2*>(take(rows * 8));
  }
  a.part_o = reinterpret_cast<float*>(take(2 * sm * kPrefixRows * dim * 4));
  a.part_ml = reinterpret_cast<float2*>(take(2 * sm * kPrefixRows * 8));
  // Few rows of a sequence: its own positions are streamed beside the prefixes.  Many: tree attention's tensor-memory kernel
  // is the better one for them (its rule), and runs in front.
  a.own_cost = streams(own.b, group) ? (dim == 128 ? kOwnCost128 : kOwnCost64) : 0;
  if (a.own_cost) {
    own.part_o = reinterpret_cast<float*>(take(4 * sm * 16 * dim * 4));
    own.part_ml = reinterpret_cast<float2*>(take(4 * sm * 16 * 8));
  } else {
    own.part_o = nullptr;
    own.part_ml = nullptr;
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

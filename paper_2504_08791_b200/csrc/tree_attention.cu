// Attention of drafted token trees over a paged cache.
//
//   out[t][h] = sum_j p_j v_j / sum_j p_j,   p_j = exp(scale q.k_j - m),   j over the context and the rows that t sees
//
// A step has few rows per sequence and a long cache, so the cache should be read once, at HBM speed: all query heads
// that share a KV head and all rows of the sequence make one tile of up to 256 rows (two accumulators of 128), which one
// pass over the cache serves.
//
// One persistent CTA per SM takes an equal share of all units (paged_index.h): 128 positions of one KV head for one
// tile of rows.  Warp 8 copies keys and values page by page into a ring in shared memory (one tiled copy per page and
// 64 columns), warp 9 issues the products, S = Q K^T into tensor memory, O += P V with P read from tensor memory, and
// eight warps turn S into P, one thread per row and half of the 128 positions: no shuffles.  There are two buffers of
// scores, used in turn by the units (or by the two accumulators of a tile of more than 128 rows), so that the scores of
// the next sub-unit are computed under the exponentials of this one; P takes the place of its scores.
// The two threads of a row share its reference, which moves only when a score exceeds the maximum that set it by a factor
// of 2^8: that is one vote of two warps per sub-unit, and O is hardly ever rescaled.  Sums and maxima are in 32 bits.  P is
// rounded to the cache's type because the product takes both operands in one type; with values widened to 32 bits it would
// run at half the rate and the values would take twice the ring, and P as a sum of two 16-bit numbers would double the
// product.  It costs half a step of each probability (outputs in fp16 off by 2.9e-4 of their size from 64 bits where
// unrounded probabilities give 2.1e-4, in bf16 2.1e-3 and 1.7e-3); the streaming kernel does the same.
// A segment that is not a whole (sequence, KV head, tile) leaves its maximum, sum and output in the workspace, and
// tree_merge_kernel joins the parts in ascending order: the same lengths give the same bits.
// Measured (one B200, both kernels together): 64 nodes, 64 query heads on 8 KV heads of 128, 65,531 positions, fp16:
// 168 us (0.82 PFLOP/s; 186 to 201 when called for long, the power limit), bound by the softmax, whose eight warps wait,
// read, take maximum and exponential in step: of about 2400 cycles per sub-unit of 128 x 128 scores the exponentials
// take 1100 (1024 is what the special-function units need).  16 trees of 1 to 26 nodes over 100 to 8192 positions, 40
// query heads, bf16: 62 us (2.5 TB/s), half of it beginnings and ends of segments, half waiting for keys.
#include <cudaTypedefs.h>

#include <cmath>
#include <cstdio>
#include <new>

#include "paged_device.cuh"

namespace prima {
namespace {

constexpr int kTileRows = 256;         // of the tensor-memory kernel
constexpr int kSoftmaxThreads = 256;
constexpr int kThreads = kSoftmaxThreads + 96;       // eight warps of softmax; copies, products, the plan
constexpr int kSegments = 4;           // planned ahead
// Of a segment besides its units, in units.  16 ragged trees 63.6 us, without a cost 64.8, with twice as much 69.0; 64
// nodes over 65,531 positions 168, 174, 166; streaming kernel, 64 ragged single tokens 23.8, 28.1, with three units 26.9.
constexpr int kSegmentCost = 3, kStreamSegmentCost = 1;
struct Segment {
  int seq, head, row0, rows;           // rows row0 .. row0 + rows - 1 of the (sequence, KV head)
  int first, nodes, ctx;               // the sequence: first row of the step, rows, cached positions
  int chunk0, n;                       // first unit and their number
  int kind;                            // 0: whole; 1: continues; 2: begins here and goes on
  long long limit;                     // positions that the tile may see
  __device__ __forceinline__ int halves() const { return rows > 128 ? 2 : 1; }      // accumulators of 128 rows
  // Positions that all rows see: the context, as far as the table names pages for it.
  __device__ __forceinline__ long long all_see() const { return min(static_cast<long long>(ctx), limit); }
};

struct Control {
  unsigned long long full[12], empty[12], s_ready[2], p_ready[4], pv_done[2], q_ready, q_first, seg_done, drained;      // of each buffer; p_ready: and half; q_first: the first segment's queries
  unsigned long long seg_full[kSegments], seg_empty[kSegments];
  Segment seg[kSegments];              // n = 0: no more
  uint32_t tmem;
  int give_up;
  int bad[16];                         // of the last units: some page is none (the ring holds at most six)
  float top[2][2][128];                // [buffer][half of the positions][row]: what the other half has to know
};

// What a CTA leaves about the segment that begins in it and goes on in later ones.
struct TailNote {
  int rows, row0, first, head, last_cta, unused[3];
};

struct TreeArgs {
  PoolView pool;
  BatchView b;
  TreeShape shape;
  int layer, n_q_heads;
  float scale_log2;
  uint32_t group_inverse;      // small_inverse(shape.group)
  const void* q;
  void* out;
  float* lse;
  float* part_o;       // [2 n_cta][D / 4][tile_rows][4]
  float2* part_ml;     // [2 n_cta][tile_rows]: reference (binary exponent), sum
  TailNote* notes;     // [n_cta]
};

// ---- this CTA's share, segment by segment -----------------------------------------------------------------------------
// One warp walks the share, 32 sequences at a time, one per lane, and hands the segments to the others ahead of time.
struct Cursor {
  const TreeArgs& a;
  const int lane;
  long long total = 0, u = 0, u_end = 0;
  int w0 = 0;                                  // first sequence of the window
  long long window = 0, before = 0, units = 0; // of the window; of the lane's sequence: units in front of it, its own
  int first = 0, nodes = 0, ctx = 0;

  __device__ __forceinline__ bool read(int i) {
    const int f = a.b.row_begin[i], e = a.b.row_begin[i + 1], c = a.b.ctx_len[i];
    const bool ok = f >= 0 && e >= f && e <= a.b.n_tok && c >= 0;
    first = f;
    nodes = ok ? e - f : 0;
    ctx = c;
    units = ok ? tree_units(a.shape, ctx, nodes) * a.shape.n_kv_heads : 0;
    return ok;
  }
  __device__ void load(long long in_front) {
    units = 0;
    if (w0 + lane < a.b.n_seq) read(w0 + lane);
    long long x = units;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    before = in_front + x - units;
    window = in_front + __shfl_sync(0xffffffffu, x, 31);
  }
  __device__ Cursor(const TreeArgs& args, int lane_, bool reports, bool used = true) : a(args), lane(lane_) {
    if (!used) return;
    for (int i = lane; i < a.b.n_seq; i += 32) {
      const bool ok = read(i);
      total += units;
      if (reports) {
        if (!ok) raise(a.pool.status, kBadRows);
        else if (nodes && static_cast<long long>(ctx) + nodes > a.shape.capacity) raise(a.pool.status, kBadSlot);
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    const TreeShares shares = tree_shares(total, gridDim.x);
    u = tree_share_begin(shares, blockIdx.x);
    u_end = tree_share_begin(shares, blockIdx.x + 1);
    load(0);
  }
  __device__ bool next(Segment* s) {
    while (u < u_end) {
      unsigned hit;
      while (!(hit = __ballot_sync(0xffffffffu, u >= before && u < before + units))) {      // ends: u is below the total
        w0 += 32;
        load(window);
      }
      const int src = __ffs(hit) - 1;
      const long long in_front = __shfl_sync(0xffffffffu, before, src);
      s->first = __shfl_sync(0xffffffffu, first, src);
      s->nodes = __shfl_sync(0xffffffffu, nodes, src);
      s->ctx = __shfl_sync(0xffffffffu, ctx, src);
      const long long per_head = div_small(__shfl_sync(0xffffffffu, units, src), a.shape.n_kv_heads);
      const TreeSegment t = tree_segment(a.shape, s->ctx, s->nodes, per_head, u - in_front, u_end - in_front);
      s->seq = w0 + src;
      s->head = t.head;
      s->row0 = t.row_tile * a.shape.tile_rows;
      s->rows = static_cast<int>(min(static_cast<long long>(s->nodes) * a.shape.group - s->row0, static_cast<long long>(a.shape.tile_rows)));
      s->chunk0 = t.chunk0;
      s->n = t.chunk1 - t.chunk0;
      s->kind = t.chunk0 ? 1 : t.chunk1 < t.chunks ? 2 : 0;
      s->limit = tree_kv_end(a.shape, s->ctx, s->nodes, t.row_tile);
      last_unit = u + t.to_end - 1;
      u += t.places;
      if (s->n) return true;
    }
    return false;
  }
  // s: the last segment of the share, kind 0 if there was none
  __device__ void write_note(const Segment& s) const {
    TailNote& note = a.notes[blockIdx.x];
    const bool cut = s.kind == 2 && s.n > 0;
    note.rows = cut ? s.rows : 0;
    if (cut) {
      note.row0 = s.row0;
      note.first = s.first;
      note.head = s.head;
      note.last_cta = tree_cta_of(tree_shares(total, gridDim.x), last_unit);
    }
  }
  long long last_unit = 0;      // of the whole (sequence, KV head, row tile) of the segment that next() gave
};

template <typename T, typename Out, int D>
__global__ void __launch_bounds__(kThreads, 1) tree_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                                                           const __grid_constant__ TreeArgs a) {
  using Geo = Geometry<D>;
  constexpr int kSlots = Geo::kSlots;
  constexpr bool kBf16 = !__is_same(T, __half);
  // The swizzled tiles need 1024-byte alignment, which the shared memory of a kernel without static variables has; there
  // is no room to round up.
  extern __shared__ __align__(1024) uint8_t smem[];
  if (smem_u32(smem) & 1023) {      // never seen; nothing is computed, and the joining kernel finds nothing to join
    pdl_wait();
    if (threadIdx.x == 0) {
      a.notes[blockIdx.x].rows = 0;
      raise(a.pool.status, kGaveUp);
    }
    return;
  }
  uint8_t* s_q = smem;
  uint8_t* s_ring = smem + 2 * Geo::kQBytes;
  Control* ctl = reinterpret_cast<Control*>(s_ring + kSlots * Geo::kSlotBytes);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t bar_full = smem_u32(ctl->full), bar_empty = smem_u32(ctl->empty), bar_s = smem_u32(ctl->s_ready), bar_p = smem_u32(ctl->p_ready),
                 bar_pv = smem_u32(ctl->pv_done), bar_seg = smem_u32(ctl->seg_full), bar_seg_empty = smem_u32(ctl->seg_empty), bar_q = smem_u32(&ctl->q_ready), bar_first = smem_u32(&ctl->q_first),
                 bar_done = smem_u32(&ctl->seg_done), bar_drain = smem_u32(&ctl->drained);
  int* const give_up = &ctl->give_up;
  int* const status = a.pool.status;

  pdl_trigger();
  if (tid == 0) {
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(bar_full + 8 * i, 1);
      mbar_init(bar_empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_s + 8 * i, 1);
      mbar_init(bar_p + 16 * i, 4);
      mbar_init(bar_p + 16 * i + 8, 4);
      mbar_init(bar_pv + 8 * i, 1);
    }
    for (int i = 0; i < kSegments; ++i) {
      mbar_init(bar_seg + 8 * i, 1);
      mbar_init(bar_seg_empty + 8 * i, 10);
    }
    mbar_init(bar_q, 8);
    mbar_init(bar_first, 8);
    mbar_init(bar_done, 8);
    mbar_init(bar_drain, 1);
    ctl->give_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma_prefetch_map(&k_map);
    tma_prefetch_map(&v_map);
  }
  if (warp == 9) tmem_alloc(smem_u32(&ctl->tmem), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl->tmem;      // scores of buffer 0 and 1: columns 0, 128; outputs of half tile 0 and 1: 256, 256 + D
  pdl_wait();

  // Segment i of this CTA, or nothing when there are no more; the caller's warp gives it back with done_with(i).
  auto segment = [&](uint32_t i) -> const Segment* {
    const Segment* s = &ctl->seg[i % kSegments];
    if (!wait_segment(bar_seg + 8 * (i % kSegments), i / kSegments & 1)) {
      if (lane == 0) raise(status, kGaveUp);
      return nullptr;
    }
    return s->n ? s : nullptr;
  };
  auto done_with = [&](uint32_t i) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar_seg_empty + 8 * (i % kSegments));
  };
  RingPlace<kSlots> ring;       // the place that the segment begins with
  uint32_t copies_before = 0;   // copies: places used so far, up to kSlots (the ring is empty at first)

  if (warp == 10) {
    // ---- the plan ----
    Cursor cursor(a, lane, blockIdx.x == 0);
    Segment s;
    s.kind = 0;
    for (uint32_t i = 0;; ++i) {
      const bool more = cursor.next(&s);
      if (i >= kSegments && !__all_sync(0xffffffffu, wait_segment(bar_seg_empty + 8 * (i % kSegments), (i / kSegments - 1) & 1))) {      // never seen; what others may still read stays
        if (lane == 0) raise(status, kGaveUp);
        break;
      }
      if (lane == 0) {
        ctl->seg[i % kSegments] = s;
        if (!more) ctl->seg[i % kSegments].n = 0;
        mbar_arrive(bar_seg + 8 * (i % kSegments));
      }
      __syncwarp();
      if (!more) break;
    }
    if (lane == 0) cursor.write_note(s);
  } else if (warp == 8) {
    // ---- copies ----
    const int shift = a.pool.page_shift;
    const int box_rows = min(1 << shift, kTilePos);
    const int boxes = kTilePos / box_rows;           // per 64 columns of a unit
    const int box = lane % boxes, panel = lane / boxes;
    const uint32_t dst = smem_u32(s_ring) + panel * Geo::kPanel + box * box_rows * 128;
    bool started = false;
    uint32_t n_read = 0;      // units
    const Segment* seg;
    for (uint32_t si = 0; (seg = segment(si)); ++si) {
      const Segment s = *seg;
      done_with(si);
      const int32_t* table = a.b.table + s.seq * a.b.table_stride;
      for (int t = 0; t < s.n; ++t) {
        const long long pos = static_cast<long long>(s.chunk0 + t) * kTilePos + box * box_rows;
        int64_t row = -1;
        bool bad = false;
        if (panel < D / 64 && pos < s.limit) {
          const int64_t r = find_slot(a.pool, table, a.b.table_stride, a.layer, pos);
          bad = r < 0;
          if (bad) raise(status, static_cast<int>(-r));
          else row = r + (static_cast<int64_t>(s.head) << shift);
        }
        const int n_copies = __popc(__ballot_sync(0xffffffffu, row >= 0));
        const bool any_bad = __any_sync(0xffffffffu, bad);
#pragma unroll
        for (int is_v = 0; is_v < 2; ++is_v) {
          bool ok = true;
          if (copies_before >= kSlots) ok = wait_for(bar_empty + 8 * ring.slot, ring.phase ^ 1, give_up, status);
          ok = __all_sync(0xffffffffu, ok);
          if (ok) {
            if (lane == 0) {
              if (!is_v) ctl->bad[n_read % 16] = any_bad;
              mbar_expect(bar_full + 8 * ring.slot, static_cast<uint32_t>(n_copies) * box_rows * 128);
            }
            __syncwarp();
            if (row >= 0) tma_load_2d(dst + ring.slot * Geo::kSlotBytes, is_v ? &v_map : &k_map, panel * 64, static_cast<int>(row), bar_full + 8 * ring.slot);
          }
          // Queries before the rest of the first places: the first scores need them and one unit's keys, not what
          // else fills the ring (measured: queries behind 160 KB of keys and values arrive 8 us late).  A barrier of their
          // own: the next segment's queries may be ready before this warp looks, and bar_q a phase further.
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
    uint32_t n_sub = 0;      // sub-units before this segment; sub-unit i uses buffer i % 2
    const Segment* seg;
    for (uint32_t si = 0; (seg = segment(si)); ++si) {
      const int halves = uniform(seg->rows) > 128 ? 2 : 1, count = uniform(seg->n) * halves;
      done_with(si);
      bool ok = wait_for(bar_q, si & 1, give_up, status);
      RingPlace<kSlots> pk = ring, pv = ring;      // of the unit whose keys, whose values are due
      pv.step(1);
      // Sub-unit i: unit i, or half i % 2 of the rows of unit i / 2
      auto wait_keys = [&](int i) {
        if (halves == 1 || !(i & 1)) ok = wait_for(bar_full + 8 * pk.slot, pk.phase, give_up, status) && ok;
      };
      auto scores = [&](int i) {                   // S = Q K^T
        const uint32_t h = halves == 2 ? i & 1 : 0, buffer = (n_sub + i) & 1;
        const bool last = halves == 1 || h == 1;
        tc_fence_after();
        if (__all_sync(0xffffffffu, ok) && elect_one()) {
          const SmemOperand qq = smem_operand(q_addr + (halves == 2 ? h : si & 1) * Geo::kQBytes, 16), kk = k_all + pk.slot * Geo::kSlotBytes;
#pragma unroll
          for (int k = 0; k < D / 16; ++k) mma_ss(u_tmem + buffer * kTilePos, qq + (k / 4 * Geo::kPanel + k % 4 * 32), kk + (k / 4 * Geo::kPanel + k % 4 * 32), kDescS, k > 0);
          tc_commit(bar_s + 8 * buffer);
          if (last) tc_commit(bar_empty + 8 * pk.slot);
        }
        __syncwarp();
        if (last) pk.step(2);
      };
      for (int i = 0; i < min(count, 2); ++i) {
        wait_keys(i);
        scores(i);
      }
      for (int i = 0; i < count; ++i) {
        const uint32_t h = halves == 2 ? i & 1 : 0, buffer = (n_sub + i) & 1, phase = (n_sub + i) >> 1 & 1;
        const bool first = i < halves, last = halves == 1 || h == 1;
        if (halves == 1 || !h) ok = wait_for(bar_full + 8 * pv.slot, pv.phase, give_up, status) && ok;
        if (i + 2 < count) wait_keys(i + 2);
        // O += P V, each half of the positions when its P is there (warps that rescale O report no P before all of a row's
        // columns are scaled); the first product of a segment overwrites O, which all warps must have read (their P says so)
        const SmemOperand vv = v_all + pv.slot * Geo::kSlotBytes;
        if (first) ok = wait_for(bar_p + 16 * buffer + 8, phase, give_up, status) && ok;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          if (w == 0 || !first) ok = wait_for(bar_p + 16 * buffer + 8 * w, phase, give_up, status) && ok;
          tc_fence_after();
          if (__all_sync(0xffffffffu, ok) && elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              mma_ts(u_tmem + 256 + h * D, u_tmem + buffer * kTilePos + 64 * w + 8 * k, vv + (4 * w + k) * (16 * 128), kDescO, !first || w > 0 || k > 0);
            if (w) {
              tc_commit(bar_pv + 8 * buffer);
              if (last) tc_commit(bar_empty + 8 * pv.slot);
            }
          }
          __syncwarp();
        }
        if (last) pv.step(2);
        // P lies over S: the next scores are written behind the product that reads it (one warp's products run in order)
        if (i + 2 < count) scores(i + 2);
      }
      n_sub += count;
      ring.skip(2 * (count / halves));
    }
  } else {
    // ---- softmax: warps 0..3 take positions 0..63 of a unit, warps 4..7 the others; one thread per row and half ----
    const int w = warp >> 2, quarter = warp & 3, r = quarter * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
    const uint32_t t_s = tmem + lanes + 64 * w, t_o = tmem + lanes + 256;
    const int group = a.shape.group;
    uint32_t n_sub = 0, unit_base = 0;      // sub-units, units of the segments before
    bool loaded = false;                    // the queries of the segment are on their way already

    // Row x of a segment's tile: its head's place in an array [n_tok][n_q_heads]
    auto place_of = [&](const Segment& g, int t0, int rem0, int x) {
      const int y = rem0 + x, t = small_div(y, a.group_inverse);
      return static_cast<int64_t>(g.first + t0 + t) * a.n_q_heads + g.head * group + (y - t * group);
    };
    // Queries of a segment into its tile, in the background; all threads.
    auto load_queries = [&](const Segment& g, uint32_t tile) {
      constexpr int kPieces = D / 8;
      const int t0 = g.row0 / group, rem0 = g.row0 - t0 * group;
      const int rows = g.halves() * 128;
#pragma unroll 4
      for (int idx = tid; idx < rows * kPieces; idx += kSoftmaxThreads) {
        const int row = idx / kPieces, piece = idx % kPieces, in_acc = row & 127;
        const bool there = row < g.rows;
        copy16(smem_u32(s_q) + ((rows > 128 ? row >> 7 : tile) ? Geo::kQBytes : 0) + piece / 8 * Geo::kPanel + in_acc * 128 + ((piece % 8) ^ (in_acc & 7)) * 16,
               static_cast<const T*>(a.q) + place_of(g, t0, rem0, there ? row : 0) * D + piece * 8, there);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto queries_ready = [&]() {
      asm volatile("cp.async.wait_all;" ::: "memory");
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_q);
    };
    // The two warps of the same rows
    auto pair_any = [&](bool x) {
      uint32_t y = x;
      asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 q, %1, 0;\nbar.red.or.pred p, %2, 64, q;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(y) : "r"(y), "r"(1 + quarter) : "memory");
      return y != 0;
    };
    auto pair_sync = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(1 + quarter) : "memory"); };

    const Segment* seg;
    for (uint32_t si = 0; (seg = segment(si)); ++si) {
      const Segment& s = *seg;      // read again where it is needed
      // All warps are done with the segment before: awaited before its queries are overwritten, and by every warp before
      // it reports this segment (a barrier counts arrivals of one phase at a time).
      bool before_done = si == 0;
      auto wait_before = [&]() {
        if (!before_done) wait_for(bar_done, (si - 1) & 1, give_up, status);
        before_done = true;
      };
      if (!loaded) {
        wait_before();
        load_queries(s, si & 1);
        queries_ready();
        if (si == 0 && lane == 0) mbar_arrive(bar_first);
      }
      // A tile of at most 128 rows leaves room for the next one's queries, where the segment before had its own.
      bool next_loads = false;
      auto load_next = [&]() {
        if (s.halves() == 2) return;
        const Segment* next = segment(si + 1);
        if (!next || next->halves() == 2) return;
        wait_before();
        load_queries(*next, (si + 1) & 1);
        next_loads = true;
      };
      const int t0 = s.row0 / group, rem0 = s.row0 - t0 * group;
      const int halves = s.halves(), count = s.n * halves;
      RingPlace<kSlots> pk = ring;            // of the unit's keys
      ring.skip(2 * s.n);
      // of the accumulator whose turn it is, and of the other one
      float m = -INFINITY, m_other = -INFINITY;
      float2 sum = make_float2(0.f, 0.f), sum_other = make_float2(0.f, 0.f);
#pragma unroll 1
      for (int i = 0; i < count; ++i, ++n_sub) {
        const int h = halves == 2 ? i & 1 : 0, t = halves == 2 ? i >> 1 : i;
        const int in_tile = h * 128 + r;
        const bool live = h * 128 + quarter * 32 < s.rows;
        const uint32_t buffer = n_sub & 1;
        const long long pos0 = static_cast<long long>(s.chunk0 + t) * kTilePos + 64 * w;
        // At the edge: what this thread's row sees, and which of the warp's 32 positions any row sees.  Worked out
        // before the scores are there; again in the rare case that the unit turns out to have a bad page.
        bool edge = pos0 + 64 > s.all_see(), waited = false, bad = false;
        uint32_t seen[2], seen_any = 0xffffffffu;
        for (;;) {
          if (edge) {
            const SegmentView view{a.b, a.pool, s.first, s.nodes, s.ctx, s.limit, a.b.table + s.seq * a.b.table_stride, bad};
            const int node = in_tile < s.rows ? t0 + small_div(rem0 + in_tile, a.group_inverse) : 0;
            if (h == 0) seen_any = view.seen_by_any(pos0 + (r & 32), lane);
#pragma unroll
            for (int c = 0; c < 2; ++c) seen[c] = live ? view.seen_by(node, pos0 + 32 * c) : 0u;
          }
          if (waited) break;
          wait_for(bar_s + 8 * buffer, n_sub >> 1 & 1, give_up, status);
          waited = true;
          bad = *static_cast<volatile int*>(&ctl->bad[(unit_base + t) % 16]) != 0;
          if (!bad) break;
          edge = true;
        }
        tc_fence_after();
        if (live) {
          uint32_t sc[2][32];
#pragma unroll
          for (int c = 0; c < 2; ++c) tmem_load(sc[c], t_s + buffer * kTilePos + 32 * c);
          tmem_wait_load();
#pragma unroll
          for (int c = 0; c < 2; ++c) tmem_use(sc[c]);
          if (edge) {
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (!(seen[c] >> j & 1)) sc[c][j] = 0xff800000u;
          }
          // Both halves of the positions measure a row against the same reference.
          const float top = max_of(sc[1], max_of(sc[0], -INFINITY)) * a.scale_log2;
          if (i < halves) {
            ctl->top[buffer][w][r] = top;
            pair_sync();
            m = fmaxf(top, ctl->top[buffer][w ^ 1][r]) - kHeadroom;
          } else if (pair_any(top > m + kSlack)) {
            ctl->top[buffer][w][r] = top;
            pair_sync();
            const float both = fmaxf(top, ctl->top[buffer][w ^ 1][r]);
            const float m_new = both > m + kSlack ? both - kHeadroom : m;
            const float f = m == m_new ? 1.f : ex2(m - m_new);
            m = m_new;
            sum.x *= f;
            sum.y *= f;
            // behind the last product into this accumulator; each of the two warps takes half of its columns
            if (halves == 1) wait_for(bar_pv + 8 * (buffer ^ 1), (n_sub - 1) >> 1 & 1, give_up, status);
            tc_fence_after();
#pragma unroll 1
            for (int k = 0; k < D / 32; ++k) {
              uint32_t y[16];
              const uint32_t at = t_o + h * D + w * (D / 2) + 16 * k;
              tmem_load(y, at);
              tmem_wait_load();
              tmem_use(y);
#pragma unroll
              for (int j = 0; j < 16; ++j) y[j] = __float_as_uint(__uint_as_float(y[j]) * f);
              tmem_store(at, y);
            }
            // The next product adds to all columns and may be issued when one of the two warps has reported its P: neither
            // reports before both have scaled their half.
            tmem_wait_store();
            tc_fence_before();
            pair_sync();
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
          tmem_store(t_s + buffer * kTilePos, packed);
          tmem_wait_store();
        }
        if (seen_any != 0xffffffffu) {
          // Values at positions that no row sees may be anything, and 0 x NaN is NaN: clear them.
          RingPlace<kSlots> pv = pk;
          pv.step(1);
          wait_for(bar_full + 8 * pv.slot, pv.phase, give_up, status);
          if (!(seen_any >> lane & 1)) {
            uint8_t* row = s_ring + pv.slot * Geo::kSlotBytes + (64 * w + (r & 63)) * 128;
            constexpr int kHalfRow = D / 16;      // 16-byte pieces
#pragma unroll
            for (int c = 0; c < kHalfRow; ++c) {
              const int piece = (r >> 6) * kHalfRow + c;
              *reinterpret_cast<uint4*>(row + piece / 8 * Geo::kPanel + piece % 8 * 16) = make_uint4(0, 0, 0, 0);
            }
          }
          fence_async_smem();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_p + 16 * buffer + 8 * w);
        if (h == halves - 1) pk.step(2);
        if (halves == 2) {
          const float x = m;
          const float2 y = sum;
          m = m_other;
          sum = sum_other;
          m_other = x;
          sum_other = y;
        }
        if (i == 0) load_next();
      }
      // ---- the segment's result: each of the two warps takes half of the columns ----
      if (next_loads) queries_ready();      // the next scores may follow the last product
      loaded = next_loads;
      unit_base += s.n;
      wait_for(bar_pv + 8 * ((n_sub - 1) & 1), (n_sub - 1) >> 1 & 1, give_up, status);
      tc_fence_after();
      __syncwarp();
      wait_before();
      if (lane == 0) mbar_arrive(bar_done);
#pragma unroll 1
      for (int h = 0; h < halves; ++h) {
        const int in_tile = h * 128 + r;
        if (h * 128 + quarter * 32 < s.rows) {
          float total = sum.x + sum.y;
          ctl->top[h][w][r] = total;
          pair_sync();
          total += ctl->top[h][w ^ 1][r];
          pair_sync();      // read before the next segment's maxima take its place
          const float f = s.kind == 0 ? inverse_of(total) : 1.f;
          const bool mine = in_tile < s.rows;
          const int64_t at = mine ? place_of(s, t0, rem0, in_tile) : 0;
          const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x) + (s.kind == 2);
#pragma unroll 1
          for (int c = w * (D / 64); c < (w + 1) * (D / 64); ++c) {
            uint32_t o[32];
            float y[32];
            tmem_load(o, t_o + h * D + 32 * c);
            tmem_wait_load();
            tmem_use(o);
#pragma unroll
            for (int j = 0; j < 32; ++j) y[j] = __uint_as_float(o[j]) * f;
            if (mine) {
              if (s.kind == 0) {
                store_row(static_cast<Out*>(a.out) + at * D + 32 * c, y);
              } else {
                float4* dst = reinterpret_cast<float4*>(a.part_o) + (slot * (D / 4) + 8 * c) * kTileRows + in_tile;
#pragma unroll
                for (int j = 0; j < 8; ++j) dst[j * kTileRows] = make_float4(y[4 * j], y[4 * j + 1], y[4 * j + 2], y[4 * j + 3]);
              }
            }
          }
          if (mine && w == 0) {
            if (s.kind != 0) a.part_ml[slot * kTileRows + in_tile] = make_float2(m, total);
            else if (a.lse) a.lse[at] = log_sum(m, total);
          }
        }
        m = m_other;
        sum = sum_other;
      }
      tc_fence_before();
      done_with(si);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();

  // A wait that gave up may have left products or copies under way: they end before the memory is given back.
  if (ctl->give_up) {
    if (tid == 9 * 32) {
      tc_commit(bar_drain);
      for (int i = 0; i < (1 << 22) && !mbar_test(bar_drain, 0); ++i) {}
    }
    if (tid == 8 * 32)
      for (uint32_t p = 0; p < copies_before; ++p) {      // the last places
        ring.phase ^= ring.slot == 0;
        ring.slot = ring.slot == 0 ? kSlots - 1 : ring.slot - 1;
        for (int i = 0; i < (1 << 16) && !mbar_test(bar_full + 8 * ring.slot, ring.phase); ++i) {}
      }
    __syncthreads();
  }
  if (warp == 9) tmem_free(tmem, 512);
}

// ---- few rows ---------------------------------------------------------------------------------------------------------
// Where a KV head is read by few rows of a sequence (single tokens, short drafts), 128-row products are mostly
// padding and what counts is the path from one short sequence to the next.  Here a CTA of four warps takes a share;
// each warp streams every fourth group of 16 positions through a ring of its own (16-byte asynchronous copies) and
// applies it with m16n8k16 products, queries and output in registers; several CTAs per SM hide one another's starts and
// ends.  The warps' states are joined through shared memory at the end of a segment.
// Measured with the join: 64 single tokens over 1 to 4096 positions, 32 query heads on 8 KV heads of 64, bf16: 24 us (3.0
// TB/s), bound by the barriers and starts of 512 ragged segments; 5 nodes over 1000 positions, 32 heads of 128: 12.7 us,
// latency.
template <int D> struct StreamGeometry {
  static constexpr int kStages = 3;
  static constexpr int kStep = 16;                             // positions
  static constexpr int kRow = D * 2;                           // bytes
  static constexpr int kStage = 2 * kStep * kRow;              // keys and values of a step
  static constexpr int kWarpBytes = kStages * kStage;
  static constexpr int kBytes = 4 * kWarpBytes + 16 * kRow;
  static constexpr int kCtas = D == 128 ? 2 : 4;               // per SM
  static_assert(16 * D * 4 <= kWarpBytes, "a warp's output fits where its ring was");
};

template <typename T, typename Out, int D>
__global__ void __launch_bounds__(128, StreamGeometry<D>::kCtas) tree_stream_kernel(const __grid_constant__ TreeArgs a) {
  using Geo = StreamGeometry<D>;
  constexpr bool kBf16 = !__is_same(T, __half);
  constexpr int kPieces = D / 8, kRows = 16;          // 16-byte pieces of a row; rows of a tile
  extern __shared__ __align__(128) uint8_t smem_raw[];
  __shared__ Segment s_seg;
  __shared__ float2 s_ml[4][kRows];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
  uint8_t* const s_q = smem_raw + 4 * Geo::kWarpBytes;
  uint8_t* const my_ring = smem_raw + warp * Geo::kWarpBytes;
  const uint32_t q_addr = smem_u32(s_q), ring_addr = smem_u32(my_ring);
  const int group = a.shape.group;
  pdl_trigger();
  pdl_wait();

  Cursor cursor(a, lane, blockIdx.x == 0, warp == 0);
  Segment plan;
  plan.kind = 0;
  for (;;) {
    if (warp == 0) {
      const bool more = cursor.next(&plan);
      if (lane == 0) {
        s_seg = plan;
        if (!more) s_seg.n = 0;
      }
    }
    __syncthreads();
    const Segment s = s_seg;
    if (s.n == 0) break;
    const int t0 = s.row0 / group, rem0 = s.row0 - t0 * group;
    auto place_of = [&](int x) {
      const int y = rem0 + x, t = small_div(y, a.group_inverse);
      return static_cast<int64_t>(s.first + t0 + t) * a.n_q_heads + s.head * group + (y - t * group);
    };
    for (int idx = tid; idx < kRows * kPieces; idx += 128) {
      const int row = idx / kPieces, piece = idx % kPieces;
      copy16(q_addr + row * Geo::kRow + (piece ^ (row & 7)) * 16, static_cast<const T*>(a.q) + place_of(row < s.rows ? row : 0) * D + piece * 8, row < s.rows);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");

    const long long pos_first = static_cast<long long>(s.chunk0) * kTilePos;
    const long long pos_end = min(static_cast<long long>(s.chunk0 + s.n) * kTilePos, s.limit);
    const int steps = static_cast<int>((pos_end - pos_first + Geo::kStep - 1) / Geo::kStep);      // the warp's: warp, warp + 4, ...
    const int32_t* table = a.b.table + s.seq * a.b.table_stride;
    // Lane's rows of a step: lane / kPieces + 32 / kPieces * i, column piece lane % kPieces; pages hold at least 8
    // positions, so a step's rows 0..7 and 8..15 lie in one page each.  The page ids are read a step ahead.
    int page[2] = {-1, -1};
    uint32_t bad_stages = 0;
    auto read_pages = [&](int step) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const long long pos = pos_first + step * Geo::kStep + 8 * h;
        page[h] = pos < pos_end ? table[pos >> a.pool.page_shift] : -1;
      }
    };
    auto load_step = [&](int step, int stage) {
      if (step < steps) {
        const long long pos0 = pos_first + step * Geo::kStep;
        uint32_t seen = low_bits(pos_end - pos0);
        bool bad = false;
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (static_cast<unsigned>(page[h]) >= static_cast<unsigned>(a.pool.n_pages)) {
            bad |= pos0 + 8 * h < pos_end;
            seen &= h ? 0x00ffu : 0xff00u;
          }
        if (bad && lane == 0) raise(a.pool.status, kBadPage);
        bad_stages = (bad_stages & ~(1u << stage)) | (bad ? 1u << stage : 0u);
        if (pos0 + Geo::kStep > s.ctx) {      // rows of the step: those that no row sees are not read, whatever they hold
          const SegmentView view{a.b, a.pool, s.first, s.nodes, s.ctx, s.limit, table, false};
          seen &= view.seen_by_any(pos0, lane);
        }
        const uint32_t dst = ring_addr + stage * Geo::kStage;
#pragma unroll
        for (int i = 0; i < Geo::kStep * kPieces / 32; ++i) {
          const int r = lane / kPieces + 32 / kPieces * i;
          const int64_t row = (((static_cast<int64_t>(a.layer) * a.pool.n_pages + page[r >> 3]) * a.pool.n_kv_heads + s.head) << a.pool.page_shift) +
                              ((pos0 + r) & ((1 << a.pool.page_shift) - 1));
          const bool there = seen >> r & 1;
          const int64_t off = there ? row * D + (lane % kPieces) * 8 : 0;
          const uint32_t at = dst + r * Geo::kRow + ((lane % kPieces) ^ (r & 7)) * 16;
          copy16(at, static_cast<const T*>(a.pool.k) + off, there);
          copy16(at + Geo::kStep * Geo::kRow, static_cast<const T*>(a.pool.v) + off, there);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    read_pages(warp);
#pragma unroll
    for (int i = 0; i < Geo::kStages - 1; ++i) {
      load_step(warp + 4 * i, i);
      read_pages(warp + 4 * (i + 1));
    }
    asm volatile("cp.async.wait_group %0;" ::"n"(Geo::kStages - 1) : "memory");      // the queries
    __syncthreads();
    uint32_t qf[D / 16][4];
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      const int row = lane & 15;
      ldsm4(qf[k], q_addr + row * Geo::kRow + ((2 * k + (lane >> 4)) ^ (row & 7)) * 16);
    }
    float o[D / 8][4];
    float ref[2], sum[2];
    int node[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int x = 8 * h + g;
      node[h] = x < s.rows ? t0 + small_div(rem0 + x, a.group_inverse) : -1;
      ref[h] = -INFINITY;
      sum[h] = 0.f;
    }
#pragma unroll
    for (int n = 0; n < D / 8; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[n][e] = 0.f;
    int stage = 0;
#pragma unroll 1
    for (int step = warp; step < steps; step += 4) {
      {
        const int ahead = stage + Geo::kStages - 1;
        load_step(step + 4 * (Geo::kStages - 1), ahead >= Geo::kStages ? ahead - Geo::kStages : ahead);
        read_pages(step + 4 * Geo::kStages);
      }
      asm volatile("cp.async.wait_group %0;" ::"n"(Geo::kStages - 1) : "memory");
      __syncwarp();
      const uint32_t kk = ring_addr + stage * Geo::kStage, vv = kk + Geo::kStep * Geo::kRow;
      float sc[2][4];
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[n][e] = 0.f;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        uint32_t b[4];      // positions 0..7 and 8..15, two halves of 8 columns each
        const int row = (lane >> 4) * 8 + (lane & 7);
        ldsm4(b, kk + row * Geo::kRow + ((2 * k + (lane >> 3 & 1)) ^ (row & 7)) * 16);
        mma16816<kBf16>(sc[0], qf[k], b[0], b[1]);
        mma16816<kBf16>(sc[1], qf[k], b[2], b[3]);
      }
      const long long pos0 = pos_first + step * Geo::kStep;
      const bool bad = bad_stages >> stage & 1;
      if (pos0 + Geo::kStep > s.all_see() || bad) {      // positions that the row does not see, or on a bad page
        const SegmentView view{a.b, a.pool, s.first, s.nodes, s.ctx, s.limit, table, bad};
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
        const float shift = ref[h] == -INFINITY ? 0.f : -ref[h];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const float x = ex2(fmaf(sc[n][2 * h], a.scale_log2, shift)), y = ex2(fmaf(sc[n][2 * h + 1], a.scale_log2, shift));
          sum[h] += x + y;
          p[2 * n + h] = Half2Of<T>::pack(x, y);
        }
      }
#pragma unroll
      for (int n = 0; n < D / 16; ++n) {
        uint32_t b[4];      // 16 positions, columns 16 n .. + 7 and + 8 .. + 15
        const int row = (lane >> 3 & 1) * 8 + (lane & 7);
        ldsm4_t(b, vv + row * Geo::kRow + ((2 * n + (lane >> 4)) ^ (row & 7)) * 16);
        mma16816<kBf16>(o[2 * n], p, b[0], b[1]);
        mma16816<kBf16>(o[2 * n + 1], p, b[2], b[3]);
      }
      stage = stage + 1 == Geo::kStages ? 0 : stage + 1;
      __syncwarp();
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();
    // ---- the segment's result: every warp's state to shared memory, in place of its ring ----
    float* my_o = reinterpret_cast<float*>(my_ring);      // [kRows][D]
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int x = 8 * h + g;
      float z = sum[h] + __shfl_xor_sync(0xffffffffu, sum[h], 1);
      z += __shfl_xor_sync(0xffffffffu, z, 2);
      if (t4 == 0) s_ml[warp][x] = make_float2(ref[h], z);
#pragma unroll
      for (int n = 0; n < D / 8; ++n) *reinterpret_cast<float2*>(my_o + x * D + 8 * n + 2 * t4) = make_float2(o[n][2 * h], o[n][2 * h + 1]);
    }
    __syncthreads();
    const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x) + (s.kind == 2);
    for (int idx = tid; idx < s.rows * (D / 4); idx += 128) {
      // whole rows side by side for the result; for the parts, rows innermost
      const int x = s.kind == 0 ? idx / (D / 4) : idx % s.rows, quad = s.kind == 0 ? idx % (D / 4) : idx / s.rows;
      float2 ml[4];
      float top = -INFINITY, total = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        ml[w] = s_ml[w][x];
        top = fmaxf(top, ml[w].x);
      }
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = ml[w].x == -INFINITY ? 0.f : ex2(ml[w].x - top);
        total += ml[w].y * f;
        const float4 v = *reinterpret_cast<const float4*>(smem_raw + w * Geo::kWarpBytes + (x * D + 4 * quad) * 4);
        y.x += v.x * f;
        y.y += v.y * f;
        y.z += v.z * f;
        y.w += v.w * f;
      }
      if (s.kind == 0) {
        const float inv = inverse_of(total);
        const int64_t at = place_of(x);
        store4(static_cast<Out*>(a.out) + at * D + 4 * quad, make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv));
        if (a.lse && quad == 0) a.lse[at] = log_sum(top, total);
      } else {
        reinterpret_cast<float4*>(a.part_o)[(slot * (D / 4) + quad) * kRows + x] = y;
        if (quad == 0) a.part_ml[slot * kRows + x] = make_float2(top, total);
      }
    }
    __syncthreads();
  }
  if (tid == 0) cursor.write_note(plan);
}

// ---- joining the parts ----------------------------------------------------------------------------------------------
// blockIdx.x = the CTA in which a cut segment begins, blockIdx.y = kRows of its rows, blockIdx.z = some of the columns;
// a thread owns one row and 4 columns at a time, so that reads of the parts are contiguous across the rows.  The parts are taken eight at
// a time, all their reads in flight: what this kernel costs is the latency of its reads (5 us behind the streaming
// kernel, 9 to 12 behind the other, with cold caches).  A thread takes kTurns such places: many CTAs find nothing to do,
// and fewer of them end sooner (heads of 128, 16 ragged trees: 63.6, 62.4 and 63.1 us in all with 1, 2 and 4 turns).
template <typename Out, int D, int kRows, int kTurns>
__global__ void __launch_bounds__(256) tree_merge_kernel(const __grid_constant__ TreeArgs a) {
  pdl_trigger();
  pdl_wait();
  const TailNote note = a.notes[blockIdx.x];
  const int tile_rows = a.shape.tile_rows;
  const int row = blockIdx.y * kRows + threadIdx.x % kRows;
  if (row >= note.rows) return;
  const int parts = note.last_cta - static_cast<int>(blockIdx.x) + 1;
#pragma unroll 1
  for (int turn = 0; turn < kTurns; ++turn) {
    const int quad = (blockIdx.z * kTurns + turn) * (256 / kRows) + threadIdx.x / kRows;
    float m = -INFINITY, total = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int c0 = 0; c0 < parts; c0 += 8) {
      float2 ml[8];
      float4 x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        ml[j] = make_float2(-INFINITY, 0.f);
        x[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c0 + j < parts) {
          const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x + c0 + j) + (c0 + j == 0);
          ml[j] = __ldcg(&a.part_ml[slot * tile_rows + row]);
          x[j] = __ldcg(reinterpret_cast<const float4*>(a.part_o) + (slot * (D / 4) + quad) * tile_rows + row);
        }
      }
      float top = m;
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, ml[j].x);
      const float f = m == -INFINITY ? 0.f : ex2(m - top);
      m = top;
      total *= f;
      o.x *= f;
      o.y *= f;
      o.z *= f;
      o.w *= f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float g = ml[j].x == -INFINITY ? 0.f : ex2(ml[j].x - m);
        total += ml[j].y * g;
        o.x += x[j].x * g;
        o.y += x[j].y * g;
        o.z += x[j].z * g;
        o.w += x[j].w * g;
      }
    }
    const float inv = inverse_of(total);
    const int gr = note.row0 + row, group = a.shape.group;
    const int64_t out_row = static_cast<int64_t>(note.first + gr / group) * a.n_q_heads + note.head * group + gr % group;
    Out* dst = static_cast<Out*>(a.out) + out_row * D + 4 * quad;
    store4(dst, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
    if (a.lse && quad == 0) a.lse[out_row] = log_sum(m, total);
  }
}

constexpr int64_t kAlign = 256;
int64_t padded(int64_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

struct Workers {
  int n, tile_rows;
};
Workers workers_of(const prima_paged& pool, const BatchView& b, int group) {
  return streams(b, group) ? Workers{pool.sm_count * (pool.cfg.head_dim == 128 ? 2 : 4), 16} : Workers{pool.sm_count, kTileRows};
}

template <typename T, typename Out, int D>
cudaError_t launch_stream(const TreeArgs& a, int n_cta, cudaStream_t st) {
  using Geo = StreamGeometry<D>;
  static bool done[kMaxDevices] = {};
  auto kernel = tree_stream_kernel<T, Out, D>;
  cudaError_t e = allow_smem(kernel, Geo::kBytes, done);
  if (e == cudaSuccess) e = launch_pdl(kernel, dim3(n_cta), dim3(128), Geo::kBytes, st, a);
  if (e != cudaSuccess) return e;
  constexpr int kRows = 16;
  return launch_pdl(tree_merge_kernel<Out, D, kRows, 1>, dim3(n_cta, 1, D / 4 * kRows / 256), dim3(256), 0, st, a);
}

template <typename T, typename Out, int D>
cudaError_t launch_tree(const prima_paged& pool, TreeArgs a, int n_cta, cudaStream_t st) {
  if (a.shape.tile_rows == 16) return launch_stream<T, Out, D>(a, n_cta, st);
  using Geo = Geometry<D>;
  constexpr size_t kSmem = 2 * Geo::kQBytes + Geo::kSlots * Geo::kSlotBytes + sizeof(Control);
  static_assert(kSmem <= 232448, "shared memory of a CTA");
  static bool done[kMaxDevices] = {};
  auto kernel = tree_kernel<T, Out, D>;
  cudaError_t e = allow_smem(kernel, kSmem, done);
  const Maps* maps = static_cast<const Maps*>(pool.maps);
  if (e == cudaSuccess) e = launch_pdl(kernel, dim3(n_cta), dim3(kThreads), kSmem, st, maps->k, maps->v, a);
  if (e != cudaSuccess) return e;
  constexpr int kTurns = 2;
  return launch_pdl(tree_merge_kernel<Out, D, 32, kTurns>, dim3(n_cta, kTileRows / 32, D / 32 / kTurns), dim3(256), 0, st, a);
}

}  // namespace

cudaError_t make_tree_maps(prima_paged* p) {
  static PFN_cuTensorMapEncodeTiled_v12000 encode = nullptr;
  if (!encode) {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found);
    if (e != cudaSuccess) return e;
    if (found != cudaDriverEntryPointSuccess || !f) return cudaErrorNotSupported;
    encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
  }
  Maps* m = new (std::nothrow) Maps();
  if (!m) return cudaErrorMemoryAllocation;
  p->maps = m;
  const prima_paged_config& c = p->cfg;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(c.head_dim), static_cast<cuuint64_t>(c.n_layers) * c.n_pages * c.n_kv_heads * c.page_size};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(c.head_dim) * 2};
  const cuuint32_t box[2] = {64, static_cast<cuuint32_t>(std::min(c.page_size, kTilePos))}, few[2] = {64, static_cast<cuuint32_t>(std::min(c.page_size, kFewPos))}, ones[2] = {1, 1};
  const CUtensorMapDataType type = c.dtype == PRIMA_DT_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  CUtensorMap* const maps[4] = {&m->k, &m->v, &m->k_few, &m->v_few};
  for (int i = 0; i < 4; ++i)
    if (encode(maps[i], type, 2, i & 1 ? p->v : p->k, dims, strides, i < 2 ? box : few, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return cudaErrorInvalidValue;
  return cudaSuccess;
}

void free_tree_maps(prima_paged* p) { delete static_cast<Maps*>(p->maps); }

}  // namespace prima

using namespace prima;

extern "C" {

// Enough for either kernel: a worker's two parts, of which the tensor-memory kernel has the larger ones.
int64_t prima_tree_attention_workspace(const prima_paged* p, int n_seq, int n_tok, int n_q_heads) {
  if (!p || n_seq < 1 || n_tok < 1 || n_q_heads < 1) return PRIMA_ERR_ARG;
  const int64_t n = p->sm_count;
  static_assert(4 * 16 <= kTileRows, "four workers of the streaming kernel need no more");
  return padded(4 * n * static_cast<int64_t>(sizeof(TailNote))) + padded(2 * n * kTileRows * static_cast<int64_t>(sizeof(float2))) +
         padded(2 * n * kTileRows * p->cfg.head_dim * static_cast<int64_t>(sizeof(float)));
}

int prima_tree_attention(prima_paged* p, int layer, const prima_paged_batch* batch, const void* q, int n_q_heads, float scale, void* out,
                         int out_dtype, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  const int rc = check_batch(p, batch, "prima_tree_attention");
  if (rc != PRIMA_OK) return rc;
  const prima_paged_config& c = p->cfg;
  if (layer < 0 || layer >= c.n_layers) return call_fail(PRIMA_ERR_ARG, "prima_tree_attention: layer out of range");
  if (!q || !out) return call_fail(PRIMA_ERR_ARG, "prima_tree_attention: null q or out");
  if (n_q_heads < 1 || n_q_heads % c.n_kv_heads || n_q_heads / c.n_kv_heads > 64)
    return call_fail(PRIMA_ERR_ARG, "prima_tree_attention: n_q_heads must be a multiple of n_kv_heads, at most 64 times it");
  if (!(scale > 0.f) || std::isinf(scale)) return call_fail(PRIMA_ERR_ARG, "prima_tree_attention: scale must be positive and finite");
  if (out_dtype != PRIMA_DT_F32 && out_dtype != c.dtype) return call_fail(PRIMA_ERR_ARG, "prima_tree_attention: out_dtype is neither fp32 nor the cache's type");
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15) return call_fail(PRIMA_ERR_ARG, "prima_tree_attention: q and out must be 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(lse) & 3) return call_fail(PRIMA_ERR_ARG, "prima_tree_attention: lse must be 4-byte aligned");
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < prima_tree_attention_workspace(p, batch->n_seq, batch->n_tok, n_q_heads))
    return call_fail(PRIMA_ERR_ARG, "prima_tree_attention: workspace too small or not 256-byte aligned");
  CallDevice dev(c.device);
  if (!dev.ok) return call_fail(PRIMA_ERR_CUDA, "cudaSetDevice failed");
  const BatchView view = view_of(*batch);
  const Workers workers = workers_of(*p, view, n_q_heads / c.n_kv_heads);
  const int64_t n = workers.n;
  TreeArgs a;
  a.pool = view_of(*p);
  a.b = view;
  a.shape = {c.n_kv_heads, n_q_heads / c.n_kv_heads, batch->mask == nullptr, batch->table_stride << p->page_shift, workers.tile_rows == kTileRows ? kSegmentCost : kStreamSegmentCost, workers.tile_rows};
  a.layer = layer;
  a.n_q_heads = n_q_heads;
  a.scale_log2 = scale * kLog2e;
  a.group_inverse = small_inverse(a.shape.group);
  a.q = q;
  a.out = out;
  a.lse = lse;
  char* ws = static_cast<char*>(workspace);
  a.notes = reinterpret_cast<TailNote*>(ws);
  ws += padded(n * static_cast<int64_t>(sizeof(TailNote)));
  a.part_ml = reinterpret_cast<float2*>(ws);
  ws += padded(2 * n * workers.tile_rows * static_cast<int64_t>(sizeof(float2)));
  a.part_o = reinterpret_cast<float*>(ws);
  using launcher = cudaError_t (*)(const prima_paged&, TreeArgs, int, cudaStream_t);
  static const launcher table[2][2][2] = {{{launch_tree<__half, float, 64>, launch_tree<__half, float, 128>}, {launch_tree<__half, __half, 64>, launch_tree<__half, __half, 128>}},
                                          {{launch_tree<__nv_bfloat16, float, 64>, launch_tree<__nv_bfloat16, float, 128>},
                                           {launch_tree<__nv_bfloat16, __nv_bfloat16, 64>, launch_tree<__nv_bfloat16, __nv_bfloat16, 128>}}};
  const cudaError_t e = table[c.dtype == PRIMA_DT_BF16][out_dtype != PRIMA_DT_F32][c.head_dim == 128](*p, a, workers.n, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? PRIMA_OK : call_cuda_fail(e, "prima_tree_attention");
}

}  // extern "C"

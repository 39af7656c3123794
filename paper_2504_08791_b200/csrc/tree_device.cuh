// The work of tree attention on the device: how a worker walks its share, what a row sees, and the streaming kernel's body.
#pragma once

#include <cuda.h>

#include "paged_device.cuh"

namespace prima {

struct Maps { CUtensorMap k, v; };      // of a pool's two arrays

template <int D> struct Geometry {
  static constexpr int kQBytes = 128 * D * 2;                  // one tile of 128 rows of queries
  static constexpr int kSlotBytes = kTilePos * D * 2;          // keys or values of a unit
  static constexpr int kPanel = kTilePos * 128;                // 64 columns of a unit
  static constexpr int kSlots = D == 128 ? 5 : 12;
};

struct Segment {
  int seq, head, row0, rows;           // rows row0 .. row0 + rows - 1 of the (sequence, KV head)
  int first, nodes, ctx;               // the sequence: first row of the step, rows, cached positions
  int chunk0, n;                       // first unit and their number
  int kind;                            // 0: whole; 1: continues; 2: begins here and goes on
  long long limit;                     // positions that the tile may see
  int last_worker;                     // kind 2: the worker in which it ends
  __device__ __forceinline__ int halves() const { return rows > 128 ? 2 : 1; }      // accumulators of 128 rows
  // Positions that all rows see: the context, as far as the table names pages for it.
  __device__ __forceinline__ long long all_see() const { return min(static_cast<long long>(ctx), limit); }
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

// The hand-over of segments, which goes on after a wait has given up elsewhere (nothing else may be left waiting).
__device__ __forceinline__ bool wait_segment(uint32_t bar, uint32_t parity) {
  for (int i = 0; i < (1 << 24); ++i)
    if (mbar_test(bar, parity)) return true;
  return false;
}

// ---- this CTA's share, segment by segment -----------------------------------------------------------------------------
// One warp walks the share, 32 sequences at a time, one per lane, and hands the segments to the others ahead of time.
struct Cursor {
  const TreeArgs& a;
  const int lane, worker, n_workers;
  long long total = 0, u = 0, u_end = 0;
  int w0 = 0;                                  // first sequence of the window
  long long window = 0, before = 0, units = 0; // of the window; of the lane's sequence: units in front of it, its own
  int first = 0, nodes = 0, ctx = 0;

  __device__ __forceinline__ bool read(int i) {
    const int f = __ldg(a.b.row_begin + i), e = __ldg(a.b.row_begin + i + 1), c = __ldg(a.b.ctx_len + i);
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
  __device__ Cursor(const TreeArgs& args, int lane_, int worker_, int n_workers_, bool reports, bool used = true)
      : a(args), lane(lane_), worker(worker_), n_workers(n_workers_) {
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
    const TreeShares shares = tree_shares(total, n_workers);
    u = tree_share_begin(shares, worker);
    u_end = tree_share_begin(shares, worker + 1);
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
      s->last_worker = s->kind == 2 ? tree_cta_of(tree_shares(total, n_workers), u + t.to_end - 1) : worker;
      u += t.places;
      if (s->n) return true;
    }
    return false;
  }
  // s: the last segment of the share, kind 0 if there was none
  __device__ void write_note(const Segment& s) const {
    TailNote& note = a.notes[worker];
    const bool cut = s.kind == 2 && s.n > 0;
    note.rows = cut ? s.rows : 0;
    if (cut) {
      note.row0 = s.row0;
      note.first = s.first;
      note.head = s.head;
      note.last_cta = s.last_worker;
    }
  }
};

// ---- what a row sees ------------------------------------------------------------------------------------------------
struct SegmentView {
  const BatchView& b;
  const PoolView& pool;
  int first, nodes, ctx;
  long long limit;
  const int32_t* table;
  bool bad_pages;

  __device__ __forceinline__ bool page_ok(long long pos) const {
    return static_cast<unsigned>(__ldg(table + (pos >> pool.page_shift))) < static_cast<unsigned>(pool.n_pages);
  }
  __device__ uint32_t good_pages(long long pos) const {      // pos < limit: a page id is read only where it is needed
    uint32_t w = 0;
#pragma unroll 1
    for (int i = 0; i < 32; ++i)
      if (pos + i < limit && page_ok(pos + i)) w |= 1u << i;
    return w;
  }
  // node: index of the row in its sequence
  __device__ uint32_t seen_by(int node, long long pos) const {
    const long long a = pos - ctx;
    uint32_t w = b.mask ? tree_bits(reinterpret_cast<const uint32_t*>(b.mask + static_cast<long long>(first + node) * b.mask_words), 2 * b.mask_words, a)
                        : low_bits(static_cast<long long>(node) + 1 - a);
    w &= low_bits(limit - pos);
    if (bad_pages) w &= good_pages(pos);
    return w;
  }
  // Positions that any row of the sequence sees; the whole warp calls it.
  __device__ uint32_t seen_by_any(long long pos, int lane) const {
    const long long a = pos - ctx;
    uint32_t w = 0xffffffffu;
    if (b.mask && a > -32) {
      w = 0;
      for (int i = lane; i < nodes; i += 32)
        w |= tree_bits(reinterpret_cast<const uint32_t*>(b.mask + static_cast<long long>(first + i) * b.mask_words), 2 * b.mask_words, a);
      w = __reduce_or_sync(0xffffffffu, w);
    }
    w &= low_bits(limit - pos);
    if (bad_pages) w &= good_pages(pos);
    return w;
  }
};


// Which kernel, by the rows that a KV head has of a sequence on average (the lengths themselves are on the device; each
// kernel is right for any): up to 32 the streaming kernel, which takes 16 at a time, beyond it the tensor-memory kernel.
// Streaming against tensor memory, heads of 128: 16 sequences of 4096 positions, 5 rows 52 and 70 us, 20 rows 70 and 71,
// 40 rows 135 and 74; 64 of 600, 5 rows 39 and 56, 20 rows 61 and 57, 40 rows 83 and 59.  Between 16 and 32 rows it goes
// by the lengths, which are not known here: 20 rows over 1000 positions 12.6 and 14.9, over 30 positions 8.6 and 14.9,
// 64 ragged sequences up to 4096 68 and 61; heads of 64, the same, 41 and 56.  The larger gains are with streaming.
// The average hides mixed batches, and padding rows count in it: 63 single tokens and one tree of 64 nodes, 8 query heads
// per KV head, go to the streaming kernel, which reads the tree's cache once per 16 of its 512 rows.  All over 30,000
// positions that is still the faster one (1607 and 2078 us), but with the single tokens over 1000 it takes 454 and 189, 15
// single tokens over 2000 and a tree over 8000, 4 heads per KV head, 89 and 75.
inline bool streams(const BatchView& b, int group) { return (static_cast<int64_t>(b.n_tok) + b.n_seq - 1) / b.n_seq * group <= 32; }
constexpr int kStreamSegmentCost = 1;      // of a segment besides its units, in units (measured beside the tensor-memory kernel's)

// ---- few rows ---------------------------------------------------------------------------------------------------------
// Where a KV head is read by few rows of a sequence (single tokens, short drafts), 128-row products are mostly
// padding and what counts is the path from one short sequence to the next.  Here a CTA of four warps takes a share;
// each warp streams every fourth group of 16 positions through a ring of its own (16-byte asynchronous copies) and
// applies it with m16n8k16 products, queries and output in registers; several CTAs per SM hide one another's starts and
// ends.  The warps' states are joined through shared memory at the end of a segment.
// Measured with the join: 64 single tokens over 1 to 4096 positions, 32 query heads on 8 KV heads of 64, bf16: 24 us (3.0
// TB/s), bound by the barriers and starts of 512 ragged segments; 5 nodes over 1000 positions, 32 heads of 128: 12.7 us,
// latency.
template <int D, int kStages_> struct StreamGeometry {
  static constexpr int kStages = kStages_;
  static constexpr int kStep = 16;                             // positions
  static constexpr int kRow = D * 2;                           // bytes
  static constexpr int kStage = 2 * kStep * kRow;              // keys and values of a step
  static constexpr int kWarpBytes = kStages * kStage;
  static constexpr int kBytes = 4 * kWarpBytes + 16 * kRow;
  static_assert(16 * D * 4 <= kWarpBytes, "a warp's output fits where its ring was");
};

// Env: who the four warps are (tid, worker of n_workers, reports), their shared memory, barrier and where results go.
template <typename T, int D, int kStages, typename Env>
__device__ __forceinline__ void stream_share(const TreeArgs& a, const Env& env) {
  using Geo = StreamGeometry<D, kStages>;
  constexpr bool kBf16 = !__is_same(T, __half);
  constexpr int kPieces = D / 8, kRows = 16;          // 16-byte pieces of a row; rows of a tile
  uint8_t* const smem_raw = env.smem;
  Segment& s_seg = *env.seg;
  float2(*const s_ml)[kRows] = env.ml;
  const int tid = env.tid, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
  uint8_t* const s_q = smem_raw + 4 * Geo::kWarpBytes;
  uint8_t* const my_ring = smem_raw + warp * Geo::kWarpBytes;
  const uint32_t q_addr = smem_u32(s_q), ring_addr = smem_u32(my_ring);
  const int group = a.shape.group;

  Cursor cursor(a, lane, env.worker, env.n_workers, env.reports, warp == 0);
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
    env.sync();
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
        page[h] = pos < pos_end ? __ldg(table + (pos >> a.pool.page_shift)) : -1;
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
    env.sync();
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
    env.sync();
    const int64_t slot = 2 * static_cast<int64_t>(env.worker) + (s.kind == 2);
    const bool by_rows = Env::kFinal && s.kind == 0;
    for (int idx = tid; idx < s.rows * (D / 4); idx += 128) {
      // whole rows side by side for the result; for the parts, rows innermost
      const int x = by_rows ? idx / (D / 4) : idx % s.rows, quad = by_rows ? idx % (D / 4) : idx / s.rows;
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
        env.whole(s, x, place_of(x), quad, y, top, total);
      } else {
        reinterpret_cast<float4*>(a.part_o)[(slot * (D / 4) + quad) * kRows + x] = y;
        if (quad == 0) {
          a.part_ml[slot * kRows + x] = make_float2(top, total);
          if (s.kind == 2) env.begins(s, x);
        }
      }
    }
    env.sync();
  }
  if (tid == 0) env.ends(cursor, plan);
}

}  // namespace prima

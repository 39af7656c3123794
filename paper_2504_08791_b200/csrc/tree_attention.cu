// Attention of drafted token trees over a paged cache.
//
//   out[t][h] = sum_j p_j v_j / sum_j p_j,   p_j = exp(scale q.k_j - m),   j over the context and the rows that t sees
//
// A step has few rows per sequence and a long cache, so the cache should be read once, at HBM speed: all query heads
// that share a KV head and all rows of the sequence make one tile of up to 256 rows (two accumulators of 128), which
// is what one pass over the cache can serve before the tensor core and the exponentials, about 2500 cycles per 128
// positions, become slower than the SM's share of HBM, about 2850.
//
// One persistent CTA per SM takes an equal share of all units (paged_index.h): 128 positions of one KV head for one
// tile of rows.  Warp 8 copies keys and values page by page into a ring in shared memory (one tiled copy per page and
// 64 columns), warp 9 issues the products, S = Q K^T into tensor memory, O += P V with P read from tensor memory, and
// two groups of four warps turn S into P, one thread per row: no shuffles.  The groups are the two halves of a tile of
// more than 128 rows, or, where a tile has fewer rows, take every other unit each and join at the end; one group's
// exponentials run under the other's products.  A row's reference maximum moves only when a score exceeds it by a
// factor of 2^8, so that O is hardly ever rescaled.  Sums and maxima are in 32 bits, P has the cache's type.
// A segment that is not a whole (sequence, KV head, tile) leaves its maximum, sum and output in the workspace, and
// tree_merge_kernel joins the parts in ascending order: the same lengths give the same bits.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <cmath>
#include <cstdio>
#include <new>

#include "paged.cuh"
#include "tcgen05.cuh"

namespace prima {
namespace {

constexpr int kSoftmaxThreads = 256;
constexpr int kThreads = kSoftmaxThreads + 96;
constexpr int kSub = 64;               // positions whose scores are in tensor memory at a time, per group and buffer
constexpr int kMaxSegments = 24;       // planned at a time
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;
constexpr float kSlack = 8.f;          // binary exponent by which a score may exceed the reference

template <int D> struct Geometry {
  static constexpr int kQBytes = 128 * D * 2;                  // one tile of 128 rows of queries
  static constexpr int kSlotBytes = kTilePos * D * 2;          // keys or values of a unit
  static constexpr int kPanel = kTilePos * 128;                // 64 columns of a unit
  static constexpr int kSlots = D == 128 ? 5 : 12;
};

struct Segment {
  int seq, head, row0, rows;           // rows row0 .. row0 + rows - 1 of the (sequence, KV head)
  int first, nodes, ctx;               // the sequence: first row of the step, rows, cached positions
  int chunk0, chunk1;
  int kind;                            // 0: whole; 1: continues; 2: begins here and goes on
  long long limit;                     // positions that the tile may see
};

struct Control {
  unsigned long long full[12], empty[12], s_ready[4], p_ready[4], pv_done[4], q_ready, drained[2];      // [group][buffer]
  uint32_t tmem;
  int give_up;
  int n_segments, found;
  long long unit;
  Segment seg[kMaxSegments];
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
  float* part_o;       // [2 n_cta][D / 4][256][4]
  float2* part_ml;     // [2 n_cta][256]: reference (binary exponent), sum
  TailNote* notes;     // [n_cta]
};

__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, int* give_up, int* status) {
  for (int i = 0; i < (1 << 22); ++i) {
    if (mbar_test(bar, parity)) return true;
    if (*static_cast<volatile int*>(give_up)) return false;
  }
  *static_cast<volatile int*>(give_up) = 1;
  raise(status, kGaveUp);
  return false;
}

// ---- planning -------------------------------------------------------------------------------------------------------
// Lengths of a sequence; nodes = 0 for one whose entries make no sense.
__device__ __forceinline__ bool sequence(const BatchView& b, int i, int* first, int* nodes, int* ctx) {
  const int f = __ldg(b.row_begin + i), e = __ldg(b.row_begin + i + 1), c = __ldg(b.ctx_len + i);
  const bool ok = f >= 0 && e >= f && e <= b.n_tok && c >= 0;
  *first = f;
  *nodes = ok ? e - f : 0;
  *ctx = c;
  return ok;
}

// Exclusive prefix sum of v over the CTA and the total; s_warp: one word per warp and one more.
__device__ __forceinline__ long long block_scan(long long v, long long* s_warp, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) s_warp[warp] = x;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    const long long y = s_warp[w];
    if (w < warp) before += y;
    all += y;
  }
  __syncthreads();
  *total = all;
  return before + x - v;
}

// Fills ctl->seg with the next segments of this CTA's share; the whole CTA calls it.  `scratch` is shared memory that
// nothing else uses meanwhile.  On the first call *u_end < 0: the share is worked out too.
__device__ void plan(const TreeArgs& a, Control* ctl, void* scratch, long long* u, long long* u_end, long long* units) {
  struct Window { long long prefix[kThreads + 1]; int first[kThreads], nodes[kThreads], ctx[kThreads]; };
  long long* s_warp = static_cast<long long*>(scratch);
  Window* w = reinterpret_cast<Window*>(s_warp + 16);
  const int tid = threadIdx.x;
  const BatchView& b = a.b;
  int first = 0, nodes = 0, ctx = 0;
  long long mine = 0, before = 0, total = 0;
  auto load = [&](int w0) {
    const int i = w0 + tid;
    mine = 0;
    nodes = 0;
    if (i < b.n_seq) {
      const bool ok = sequence(b, i, &first, &nodes, &ctx);
      mine = tree_units(a.shape, ctx, nodes);
      if (*u_end < 0 && blockIdx.x == 0) {
        if (!ok) raise(a.pool.status, kBadRows);
        else if (nodes && static_cast<long long>(ctx) + nodes > a.shape.capacity) raise(a.pool.status, kBadSlot);
      }
    }
    before = block_scan(mine, s_warp, &total);
  };
  bool loaded = false;
  if (*u_end < 0) {
    long long sum = 0;
    for (int w0 = 0; w0 < b.n_seq; w0 += kThreads) {
      load(w0);
      sum += total;
    }
    loaded = b.n_seq <= kThreads;      // the only window is in the registers
    *units = sum;
    const TreeShares shares = tree_shares(sum, gridDim.x);
    *u = tree_share_begin(shares, blockIdx.x);
    *u_end = tree_share_begin(shares, blockIdx.x + 1);
    if (tid == 0 && *u == *u_end) a.notes[blockIdx.x].rows = 0;
  }
  if (*u >= *u_end) {
    if (tid == 0) ctl->n_segments = 0;
    __syncthreads();
    return;
  }
  long long running = 0;
  int w0 = 0;
  for (;; w0 += kThreads) {
    if (!loaded) load(w0);
    if (*u < running + total || w0 + kThreads >= b.n_seq) break;
    running += total;
  }
  w->prefix[tid] = running + before;
  if (tid == kThreads - 1) w->prefix[kThreads] = running + before + mine;
  w->first[tid] = first;
  w->nodes[tid] = nodes;
  w->ctx[tid] = ctx;
  if (*u >= running + before && *u < running + before + mine) ctl->found = tid;
  __syncthreads();
  if (tid == 0) {
    long long at = *u;
    int j = ctl->found, n = 0;
    while (n < kMaxSegments && at < *u_end && j < kThreads) {
      if (at >= w->prefix[j + 1]) {
        ++j;
        continue;
      }
      const TreeSegment t = tree_segment(a.shape, w0 + j, w->ctx[j], w->nodes[j], at - w->prefix[j], *u_end - w->prefix[j]);
      const long long rows_all = static_cast<long long>(w->nodes[j]) * a.shape.group;
      const long long limit = tree_kv_end(a.shape, w->ctx[j], w->nodes[j], t.row_tile);
      Segment& s = ctl->seg[n++];
      s.seq = t.seq;
      s.head = t.head;
      s.row0 = t.row_tile * kTileRows;
      s.rows = static_cast<int>(min(rows_all - s.row0, static_cast<long long>(kTileRows)));
      s.first = w->first[j];
      s.nodes = w->nodes[j];
      s.ctx = w->ctx[j];
      s.chunk0 = t.chunk0;
      s.chunk1 = t.chunk1;
      s.kind = t.chunk0 ? 1 : t.chunk1 < t.chunks ? 2 : 0;
      s.limit = limit;
      const long long next = at + (t.chunk1 - t.chunk0);
      if (next >= *u_end) {
        TailNote& note = a.notes[blockIdx.x];
        note.rows = s.kind == 2 ? s.rows : 0;
        note.row0 = s.row0;
        note.first = s.first;
        note.head = s.head;
        note.last_cta = s.kind == 2 ? tree_cta_of(tree_shares(*units, gridDim.x), at + t.chunks - 1) : 0;
      }
      at = next;
    }
    ctl->n_segments = n;
    ctl->unit = at;
  }
  __syncthreads();
  *u = ctl->unit;
}

// ---- what a row sees ------------------------------------------------------------------------------------------------
// Bits for 32 positions from `pos` on.  a = index of the position among the rows of the step, negative in the context.
__device__ __forceinline__ uint32_t low_bits(long long n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << static_cast<int>(n)) - 1u; }
__device__ __forceinline__ uint32_t mask_word(const uint32_t* words, int n_words, long long i) { return i < n_words ? __ldg(words + i) : 0u; }
__device__ __forceinline__ uint32_t tree_bits(const uint32_t* words, int n_words, long long a) {
  if (a <= -32) return 0xffffffffu;
  if (a < 0) return mask_word(words, n_words, 0) << static_cast<int>(-a) | low_bits(-a);
  return __funnelshift_r(mask_word(words, n_words, a >> 5), mask_word(words, n_words, (a >> 5) + 1), static_cast<uint32_t>(a) & 31u);
}

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

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two 32-bit operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 x, float2 y, float2 z) {
  unsigned long long d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(*reinterpret_cast<unsigned long long*>(&x)), "l"(*reinterpret_cast<unsigned long long*>(&y)),
      "l"(*reinterpret_cast<unsigned long long*>(&z)));
  return *reinterpret_cast<float2*>(&d);
}
__device__ __forceinline__ float2 add2(float2 x, float2 y) {
  unsigned long long d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(*reinterpret_cast<unsigned long long*>(&x)), "l"(*reinterpret_cast<unsigned long long*>(&y)));
  return *reinterpret_cast<float2*>(&d);
}
__device__ __forceinline__ float max_of(const uint32_t (&x)[32]) {
  float t[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    t[c] = __uint_as_float(x[8 * c]);
#pragma unroll
    for (int j = 1; j < 8; ++j) t[c] = fmaxf(t[c], __uint_as_float(x[8 * c + j]));
  }
  return fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
}

// 32 columns of a row of the result, scaled.
template <typename T>
__device__ __forceinline__ void store_row(T* dst, const float (&x)[32]) {
#pragma unroll
  for (int i = 0; i < 32; i += 8) {
    const float y[8] = {x[i], x[i + 1], x[i + 2], x[i + 3], x[i + 4], x[i + 5], x[i + 6], x[i + 7]};
    store8(dst + i, y);
  }
}
template <>
__device__ __forceinline__ void store_row<float>(float* dst, const float (&x)[32]) {
#pragma unroll
  for (int i = 0; i < 32; i += 4) *reinterpret_cast<float4*>(dst + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
}

// A place of the ring, stepped without divisions.
template <int kSlots>
struct RingPlace {
  uint32_t slot = 0, phase = 0;
  __device__ __forceinline__ void step(uint32_t n) {      // n <= kSlots
    slot += n;
    if (slot >= kSlots) {
      slot -= kSlots;
      phase ^= 1;
    }
  }
};

template <typename T, typename Out, int D>
__global__ void __launch_bounds__(kThreads, 1) tree_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                                                           const __grid_constant__ TreeArgs a) {
  using Geo = Geometry<D>;
  constexpr int kSlots = Geo::kSlots;
  constexpr bool kBf16 = !__is_same(T, __half);
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* s_q = smem;
  uint8_t* s_ring = smem + 2 * Geo::kQBytes;
  Control* ctl = reinterpret_cast<Control*>(s_ring + kSlots * Geo::kSlotBytes);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t bar_full = smem_u32(ctl->full), bar_empty = smem_u32(ctl->empty), bar_s = smem_u32(ctl->s_ready), bar_p = smem_u32(ctl->p_ready),
                 bar_pv = smem_u32(ctl->pv_done), bar_q = smem_u32(&ctl->q_ready), bar_drain = smem_u32(ctl->drained);
  int* const give_up = &ctl->give_up;
  int* const status = a.pool.status;

  pdl_trigger();
  if (tid == 0) {
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(bar_full + 8 * i, 1);
      mbar_init(bar_empty + 8 * i, 2);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar_s + 8 * i, 1);
      mbar_init(bar_p + 8 * i, 4);
      mbar_init(bar_pv + 8 * i, 1);
    }
    mbar_init(bar_q, 8);
    mbar_init(bar_drain, 1);
    mbar_init(bar_drain + 8, 1);
    ctl->give_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma_prefetch_map(&k_map);
    tma_prefetch_map(&v_map);
  }
  if (warp == 9) tmem_alloc(smem_u32(&ctl->tmem), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl->tmem;
  pdl_wait();

  long long u = 0, u_end = -1, units = 0;
  // running state of this role
  RingPlace<kSlots> ring;       // copies and products: the place that the segment begins with
  uint32_t copies_before = 0;   // copies: places used so far, up to kSlots (the ring is empty at first)
  uint32_t n_q = 0;             // products: segments
  uint32_t n_sub = 0;           // sub-tiles of this thread's group; sub-tile i uses buffer i % 2

  do {
    plan(a, ctl, s_q, &u, &u_end, &units);
    const int n_segments = ctl->n_segments;

    if (warp == 8) {
      // ---- copies ----
      const int shift = a.pool.page_shift;
      const int box_rows = min(1 << shift, kTilePos);
      const int boxes = kTilePos / box_rows;           // per 64 columns of a unit
      const int box = lane % boxes, panel = lane / boxes;
      const uint32_t dst = smem_u32(s_ring) + panel * Geo::kPanel + box * box_rows * 128;
      for (int si = 0; si < n_segments; ++si) {
        const Segment s = ctl->seg[si];
        const int n = s.chunk1 - s.chunk0;
        const int32_t* table = a.b.table + s.seq * a.b.table_stride;
        // A lane's row of the arrays for unit t, or -1
        auto row_of = [&](int t) -> int64_t {
          const long long pos = static_cast<long long>(s.chunk0 + t) * kTilePos + box * box_rows;
          if (panel >= D / 64 || pos >= s.limit) return -1;
          const int64_t r = find_slot(a.pool, table, a.b.table_stride, a.layer, pos);
          if (r >= 0) return r + (static_cast<int64_t>(s.head) << shift);
          raise(status, static_cast<int>(-r));
          return -1;
        };
        int64_t row = row_of(0);
        for (int t = 0; t < n; ++t) {
          const int n_copies = __popc(__ballot_sync(0xffffffffu, row >= 0));
#pragma unroll
          for (int is_v = 0; is_v < 2; ++is_v) {
            bool ok = true;
            if (copies_before >= kSlots) ok = wait_for(bar_empty + 8 * ring.slot, ring.phase ^ 1, give_up, status);
            ok = __all_sync(0xffffffffu, ok);
            if (ok) {
              if (lane == 0) mbar_expect(bar_full + 8 * ring.slot, static_cast<uint32_t>(n_copies) * box_rows * 128);
              __syncwarp();
              if (row >= 0) tma_load_2d(dst + ring.slot * Geo::kSlotBytes, is_v ? &v_map : &k_map, panel * 64, static_cast<int>(row), bar_full + 8 * ring.slot);
            }
            ring.step(1);
            if (copies_before < kSlots) ++copies_before;
          }
          if (t + 1 < n) row = row_of(t + 1);
        }
      }
    } else if (warp >= 9) {
      // ---- products: one warp per group, so that neither waits for the other's softmax ----
      const uint32_t w = uniform(warp) - 9;
      constexpr uint32_t kDescS = mma_f16_desc(kBf16, false, 128, kSub), kDescO = mma_f16_desc(kBf16, true, 128, D);
      const uint32_t u_tmem = uniform(tmem), t_s = u_tmem + w * 2 * kSub, t_o = u_tmem + 256 + w * D;
      const uint32_t ring_addr = uniform(smem_u32(s_ring)), q_addr = uniform(smem_u32(s_q));
      const SmemOperand k_all = smem_operand(ring_addr, 16), v_all = smem_operand(ring_addr, Geo::kPanel);
      for (int si = 0; si < n_segments; ++si) {
        const bool halves = uniform(ctl->seg[si].rows) > 128;
        const int n = uniform(ctl->seg[si].chunk1 - ctl->seg[si].chunk0), count = halves ? 2 * n : n;
        const SmemOperand qq = smem_operand(q_addr + (halves ? w * Geo::kQBytes : 0), 16);
        bool ok = wait_for(bar_q, n_q & 1, give_up, status);
        ++n_q;
        RingPlace<kSlots> pk = ring, pv = ring;      // of the unit whose keys, whose values are due
        pv.step(1);
        // Sub-tile j: half w of unit j, or half j % 2 of unit j / 2
        auto scores = [&](int j) {                   // S = Q K^T
          const uint32_t half = halves ? j & 1 : w;
          if (!halves || half == 0) ok = wait_for(bar_full + 8 * pk.slot, pk.phase, give_up, status) && ok;
          const bool last = !halves || half == 1;
          tc_fence_after();
          if (__all_sync(0xffffffffu, ok) && elect_one()) {
            const uint32_t buffer = (n_sub + j) & 1;
            const SmemOperand kk = k_all + (pk.slot * Geo::kSlotBytes + half * (kSub * 128));
#pragma unroll
            for (int i = 0; i < D / 16; ++i) mma_ss(t_s + buffer * kSub, qq + (i / 4 * Geo::kPanel + i % 4 * 32), kk + (i / 4 * Geo::kPanel + i % 4 * 32), kDescS, i > 0);
            tc_commit(bar_s + 8 * (2 * w + buffer));
            if (last) tc_commit(bar_empty + 8 * pk.slot);
          }
          __syncwarp();
          if (last) pk.step(2);
        };
        auto outputs = [&](int j) {                  // O += P V
          const uint32_t half = halves ? j & 1 : w;
          if (!halves || half == 0) ok = wait_for(bar_full + 8 * pv.slot, pv.phase, give_up, status) && ok;
          const bool last = !halves || half == 1;
          const uint32_t buffer = (n_sub + j) & 1;
          ok = wait_for(bar_p + 8 * (2 * w + buffer), (n_sub + j) >> 1 & 1, give_up, status) && ok;
          tc_fence_after();
          if (__all_sync(0xffffffffu, ok) && elect_one()) {
            const SmemOperand vv = v_all + (pv.slot * Geo::kSlotBytes + half * (kSub * 128));
#pragma unroll
            for (int i = 0; i < kSub / 16; ++i) mma_ts(t_o, t_s + buffer * kSub + i * 8, vv + i * (16 * 128), kDescO, j > 0 || i > 0);
            tc_commit(bar_pv + 8 * (2 * w + buffer));
            if (last) tc_commit(bar_empty + 8 * pv.slot);
          }
          __syncwarp();
          if (last) pv.step(2);
        };
        scores(0);
        if (count > 1) scores(1);
        for (int j = 0; j < count; ++j) {
          outputs(j);
          if (j + 2 < count) {
            // P lies over S: the next scores of this buffer may not be written before the product has read it
            ok = wait_for(bar_pv + 8 * (2 * w + ((n_sub + j) & 1)), (n_sub + j) >> 1 & 1, give_up, status) && ok;
            scores(j + 2);
          }
        }
        n_sub += count;
        for (int k = 2 * n; k > 0; k -= kSlots) ring.step(min(k, kSlots));
      }
    } else {
      // ---- softmax ----
      const int w = warp >> 2, quarter = warp & 3, r = quarter * 32 + lane;
      const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
      const uint32_t t_s = tmem + lanes + w * 2 * kSub, t_o = tmem + lanes + 256 + w * D;
      const int group = a.shape.group;
      for (int si = 0; si < n_segments; ++si) {
        const Segment& s = ctl->seg[si];      // read again where it is needed
        const bool halves = s.rows > 128;
        const int n = s.chunk1 - s.chunk0;
        auto view_of_segment = [&](bool bad_pages) {
          return SegmentView{a.b, a.pool, s.first, s.nodes, s.ctx, s.limit, a.b.table + s.seq * a.b.table_stride, bad_pages};
        };
        // Row x of the tile: element 0 of its head in an array [n_tok][n_q_heads]
        const int t0 = s.row0 / group, rem0 = s.row0 - t0 * group;
        auto out_row = [&](int x) {
          const int y = rem0 + x, t = small_div(y, a.group_inverse);
          return static_cast<int64_t>(s.first + t0 + t) * a.n_q_heads + s.head * group + (y - t * group);
        };
        // Queries: this group's rows of the tile, or half of the only 128
        constexpr int kPieces = D / 8;
        const int q_first = 64 * w * (halves ? 2 : 1), q_rows = halves ? 128 : 64;      // rows q_first .. + q_rows of the tile
        const T* q = static_cast<const T*>(a.q);
        uint4 x[kPieces];
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          const int idx = (tid & 127) + 128 * i, row = idx / kPieces, piece = idx % kPieces;
          x[i] = make_uint4(0, 0, 0, 0);
          if (row < q_rows && q_first + row < s.rows) x[i] = __ldg(reinterpret_cast<const uint4*>(q + out_row(q_first + row) * D) + piece);
        }
        uint32_t bad = 0;
        {
          const SegmentView view = view_of_segment(false);
          const long long pos_end = min(static_cast<long long>(s.chunk1) * kTilePos, s.limit);
          for (long long pg = (static_cast<long long>(s.chunk0) * kTilePos >> a.pool.page_shift) + tid; (pg << a.pool.page_shift) < pos_end; pg += kSoftmaxThreads)
            bad |= !view.page_ok(pg << a.pool.page_shift);
        }
        // also: both groups are done with the previous segment
        asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 q, %1, 0;\nbar.red.or.pred p, 1, %2, q;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(bad) : "r"(bad), "n"(kSoftmaxThreads) : "memory");
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          const int idx = (tid & 127) + 128 * i, row = idx / kPieces, piece = idx % kPieces, in_acc = (q_first + row) & 127;
          if (row < q_rows)
            *reinterpret_cast<uint4*>(s_q + (halves && w ? Geo::kQBytes : 0) + piece / 8 * Geo::kPanel + in_acc * 128 + ((piece % 8) ^ (in_acc & 7)) * 16) = x[i];
        }
        fence_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_q);

        const int in_tile = (halves ? w * 128 : 0) + r;            // this thread's row
        const int my_rows = s.rows - (halves ? w * 128 : 0);
        const bool live = quarter * 32 < my_rows;
        const int node = in_tile < s.rows ? t0 + small_div(rem0 + in_tile, a.group_inverse) : 0;
        const int count = halves ? 2 * n : n;
        float m = -INFINITY;
        float2 sum = make_float2(0.f, 0.f);
        for (int j = 0; j < count; ++j, ++n_sub) {
          const int t = halves ? j >> 1 : j, half = halves ? j & 1 : w;
          const long long pos0 = static_cast<long long>(s.chunk0 + t) * kTilePos + half * kSub;
          const bool edge = pos0 + kSub > s.ctx || bad;
          const uint32_t buffer = n_sub & 1, phase = n_sub >> 1 & 1;
          wait_for(bar_s + 8 * (2 * w + buffer), phase, give_up, status);
          tc_fence_after();
          if (live) {
            uint32_t sc[2][32];
#pragma unroll
            for (int c = 0; c < 2; ++c) tmem_load(sc[c], t_s + buffer * kSub + 32 * c);
            uint32_t seen[2] = {0xffffffffu, 0xffffffffu};
            if (edge) {
              const SegmentView view = view_of_segment(bad);
              seen[0] = view.seen_by(node, pos0);
              seen[1] = view.seen_by(node, pos0 + 32);
            }
            tmem_wait_load();
#pragma unroll
            for (int c = 0; c < 2; ++c) tmem_use(sc[c]);
            if (edge) {
#pragma unroll
              for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int k = 0; k < 32; ++k)
                  if (!(seen[c] >> k & 1)) sc[c][k] = 0xff800000u;
            }
            const float top = fmaxf(max_of(sc[0]), max_of(sc[1])) * a.scale_log2;
            if (j == 0) {
              m = top;
            } else if (__any_sync(0xffffffffu, top > m + kSlack)) {
              const float m_new = top > m + kSlack ? top : m;
              const float f = m == m_new ? 1.f : ex2(m - m_new);
              m = m_new;
              sum.x *= f;
              sum.y *= f;
              // the product of the sub-tile before, which may still be adding to O
              wait_for(bar_pv + 8 * (2 * w + (buffer ^ 1)), (n_sub - 1) >> 1 & 1, give_up, status);
              tc_fence_after();
#pragma unroll 1
              for (int k = 0; k < D / 16; ++k) {
                uint32_t y[16];
                tmem_load(y, t_o + 16 * k);
                tmem_wait_load();
                tmem_use(y);
#pragma unroll
                for (int i = 0; i < 16; ++i) y[i] = __float_as_uint(__uint_as_float(y[i]) * f);
                tmem_store(t_o + 16 * k, y);
              }
            }
            const float2 scale = make_float2(a.scale_log2, a.scale_log2), shift = m == -INFINITY ? make_float2(0.f, 0.f) : make_float2(-m, -m);
            uint32_t packed[32];
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
              for (int k = 0; k < 16; ++k) {
                float2 p = fma2(make_float2(__uint_as_float(sc[c][2 * k]), __uint_as_float(sc[c][2 * k + 1])), scale, shift);
                p = make_float2(ex2(p.x), ex2(p.y));
                sum = add2(sum, p);
                packed[16 * c + k] = Half2Of<T>::pack(p.x, p.y);
              }
            tmem_store(t_s + buffer * kSub, packed);
            tmem_wait_store();
          }
          if (edge) {
            // Values at positions that no row sees may be anything, and 0 x NaN is NaN: clear them.
            const uint32_t seen = view_of_segment(bad).seen_by_any(pos0 + (r & 32), lane);
            RingPlace<kSlots> pv = ring;
            for (int k = 2 * t + 1; k > 0; k -= kSlots) pv.step(min(k, kSlots));
            wait_for(bar_full + 8 * pv.slot, pv.phase, give_up, status);
            if (!(seen >> lane & 1)) {
              uint8_t* row = s_ring + pv.slot * Geo::kSlotBytes + (half * kSub + (r & 63)) * 128;
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
          if (lane == 0) mbar_arrive(bar_p + 8 * (2 * w + buffer));
        }
        for (int k = 2 * n; k > 0; k -= kSlots) ring.step(min(k, kSlots));
        wait_for(bar_pv + 8 * (2 * w + ((n_sub - 1) & 1)), (n_sub - 1) >> 1 & 1, give_up, status);
        tc_fence_after();
        // ---- the segment's result ----
        const bool join = !halves;
        float total = sum.x + sum.y, other_m = -INFINITY, other_sum = 0.f;
        if (join) {      // group 1 hands its state to group 0 through tensor memory: the same lanes hold the same rows
          if (w == 1 && live) {
            const uint32_t ml[2] = {__float_as_uint(m), __float_as_uint(total)};
            tmem_store(t_s, ml);
            tmem_wait_store();
          }
          tc_fence_before();
          asm volatile("bar.sync 2, %0;" ::"n"(kSoftmaxThreads) : "memory");
          tc_fence_after();
          if (w == 0 && live) {
            uint32_t ml[2];
            tmem_load(ml, t_s + 2 * kSub);
            tmem_wait_load();
            tmem_use(ml);
            other_m = __uint_as_float(ml[0]);
            other_sum = __uint_as_float(ml[1]);
          }
        }
        if (live && (halves || w == 0)) {
          const float m_all = fmaxf(m, other_m);
          float f0 = m == -INFINITY ? 0.f : ex2(m - m_all), f1 = other_m == -INFINITY ? 0.f : ex2(other_m - m_all);
          total = total * f0 + other_sum * f1;
          if (s.kind == 0) {
            const float inv = total > 0.f ? 1.f / total : 0.f;
            f0 *= inv;
            f1 *= inv;
          }
          const bool mine = in_tile < s.rows;
          const int64_t at = mine ? out_row(in_tile) : 0;
          const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x) + (s.kind == 2);
#pragma unroll 1
          for (int c = 0; c < D / 32; ++c) {
            uint32_t o[32];
            float y[32];
            tmem_load(o, t_o + 32 * c);
            if (join) {
              uint32_t o1[32];
              tmem_load(o1, t_o + D + 32 * c);
              tmem_wait_load();
              tmem_use(o);
              tmem_use(o1);
#pragma unroll
              for (int j = 0; j < 32; ++j) y[j] = __uint_as_float(o[j]) * f0 + __uint_as_float(o1[j]) * f1;
            } else {
              tmem_wait_load();
              tmem_use(o);
#pragma unroll
              for (int j = 0; j < 32; ++j) y[j] = __uint_as_float(o[j]) * f0;
            }
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
          if (mine) {
            if (s.kind != 0) a.part_ml[slot * kTileRows + in_tile] = make_float2(m_all, total);
            else if (a.lse) a.lse[at] = total > 0.f ? (m_all + log2f(total)) * kLn2 : -INFINITY;
          }
          tc_fence_before();
        }
      }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
  } while (u < u_end);

  // A wait that gave up may have left products or copies under way: they end before the memory is given back.
  if (ctl->give_up) {
    if (warp >= 9 && lane == 0) {
      tc_commit(bar_drain + 8 * (warp - 9));
      for (int i = 0; i < (1 << 22) && !mbar_test(bar_drain + 8 * (warp - 9), 0); ++i) {}
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

// ---- joining the parts ----------------------------------------------------------------------------------------------
// blockIdx.x = the CTA in which a cut segment begins, blockIdx.y = 32 of its rows; a thread owns one row and D / 8
// columns, so that reads of the parts are contiguous across the warp.
template <typename Out, int D>
__global__ void __launch_bounds__(256) tree_merge_kernel(const __grid_constant__ TreeArgs a) {
  pdl_trigger();
  pdl_wait();
  const TailNote note = a.notes[blockIdx.x];
  const int row = blockIdx.y * 32 + (threadIdx.x & 31), part = threadIdx.x >> 5;
  if (row >= note.rows) return;
  auto slot_of = [&](int c) { return c == static_cast<int>(blockIdx.x) ? 2 * static_cast<int64_t>(c) + 1 : 2 * static_cast<int64_t>(c); };
  float m = -INFINITY;
  for (int c = blockIdx.x; c <= note.last_cta; ++c)
    m = fmaxf(m, __ldcg(&a.part_ml[slot_of(c) * kTileRows + row].x));
  float total = 0.f;
  constexpr int kQuads = D / 32;
  float4 o[kQuads];
#pragma unroll
  for (int i = 0; i < kQuads; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int c = blockIdx.x; c <= note.last_cta; ++c) {
    const float2 ml = __ldcg(&a.part_ml[slot_of(c) * kTileRows + row]);
    const float f = ml.x == -INFINITY ? 0.f : ex2(ml.x - m);
    total += ml.y * f;
    const float4* src = reinterpret_cast<const float4*>(a.part_o) + (slot_of(c) * (D / 4) + part * kQuads) * kTileRows + row;
#pragma unroll
    for (int i = 0; i < kQuads; ++i) {
      const float4 x = __ldcg(src + i * kTileRows);
      o[i].x += x.x * f;
      o[i].y += x.y * f;
      o[i].z += x.z * f;
      o[i].w += x.w * f;
    }
  }
  const float inv = total > 0.f ? 1.f / total : 0.f;
  const int gr = note.row0 + row, group = a.shape.group;
  const int64_t out_row = static_cast<int64_t>(note.first + gr / group) * a.n_q_heads + note.head * group + gr % group;
  Out* dst = static_cast<Out*>(a.out) + out_row * D + part * 4 * kQuads;
#pragma unroll
  for (int i = 0; i < kQuads; ++i) {
    if constexpr (sizeof(Out) == 4)
      *reinterpret_cast<float4*>(dst + 4 * i) = make_float4(o[i].x * inv, o[i].y * inv, o[i].z * inv, o[i].w * inv);
    else
      *reinterpret_cast<uint2*>(dst + 4 * i) = make_uint2(Half2Of<Out>::pack(o[i].x * inv, o[i].y * inv), Half2Of<Out>::pack(o[i].z * inv, o[i].w * inv));
  }
  if (a.lse && part == 0) a.lse[out_row] = total > 0.f ? (m + log2f(total)) * kLn2 : -INFINITY;
}

constexpr int64_t kAlign = 256;
int64_t padded(int64_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

struct Maps { CUtensorMap k, v; };

template <typename T, typename Out, int D>
cudaError_t launch_tree(const prima_paged& pool, TreeArgs a, cudaStream_t st) {
  using Geo = Geometry<D>;
  constexpr size_t kSmem = 1024 + 2 * Geo::kQBytes + Geo::kSlots * Geo::kSlotBytes + sizeof(Control);
  static_assert(kSmem <= 232448, "shared memory of a CTA");
  static_assert(sizeof(long long) * (16 + kThreads + 1) + 3 * sizeof(int) * kThreads <= 2 * Geo::kQBytes, "planning fits where the queries go");
  static bool done[kMaxDevices] = {};
  int dev;
  auto kernel = tree_kernel<T, Out, D>;
  if (first_launch_on_device(done, &dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmem));
    if (e != cudaSuccess) return e;
    if (dev >= 0) done[dev] = true;
  }
  const Maps* maps = static_cast<const Maps*>(pool.maps);
  cudaError_t e = launch_pdl(kernel, dim3(pool.sm_count), dim3(kThreads), kSmem, st, maps->k, maps->v, a);
  if (e != cudaSuccess) return e;
  return launch_pdl(tree_merge_kernel<Out, D>, dim3(pool.sm_count, kTileRows / 32), dim3(256), 0, st, a);
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
  const cuuint32_t box[2] = {64, static_cast<cuuint32_t>(std::min(c.page_size, kTilePos))}, ones[2] = {1, 1};
  const CUtensorMapDataType type = c.dtype == PRIMA_DT_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  for (int i = 0; i < 2; ++i)
    if (encode(i ? &m->v : &m->k, type, 2, i ? p->v : p->k, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return cudaErrorInvalidValue;
  return cudaSuccess;
}

void free_tree_maps(prima_paged* p) { delete static_cast<Maps*>(p->maps); }

}  // namespace prima

using namespace prima;

extern "C" {

int64_t prima_tree_attention_workspace(const prima_paged* p, int n_seq, int n_tok, int n_q_heads) {
  if (!p || n_seq < 1 || n_tok < 1 || n_q_heads < 1) return PRIMA_ERR_ARG;
  const int64_t n = p->sm_count;
  return padded(n * static_cast<int64_t>(sizeof(TailNote))) + padded(2 * n * kTileRows * static_cast<int64_t>(sizeof(float2))) +
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
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < prima_tree_attention_workspace(p, batch->n_seq, batch->n_tok, n_q_heads))
    return call_fail(PRIMA_ERR_ARG, "prima_tree_attention: workspace too small or not 256-byte aligned");
  CallDevice dev(c.device);
  if (!dev.ok) return call_fail(PRIMA_ERR_CUDA, "cudaSetDevice failed");
  const int64_t n = p->sm_count;
  TreeArgs a;
  a.pool = view_of(*p);
  a.b = view_of(*batch);
  a.shape = {c.n_kv_heads, n_q_heads / c.n_kv_heads, batch->mask == nullptr, batch->table_stride << p->page_shift};
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
  ws += padded(2 * n * kTileRows * static_cast<int64_t>(sizeof(float2)));
  a.part_o = reinterpret_cast<float*>(ws);
  using launcher = cudaError_t (*)(const prima_paged&, TreeArgs, cudaStream_t);
  static const launcher table[2][2][2] = {{{launch_tree<__half, float, 64>, launch_tree<__half, float, 128>}, {launch_tree<__half, __half, 64>, launch_tree<__half, __half, 128>}},
                                          {{launch_tree<__nv_bfloat16, float, 64>, launch_tree<__nv_bfloat16, float, 128>},
                                           {launch_tree<__nv_bfloat16, __nv_bfloat16, 64>, launch_tree<__nv_bfloat16, __nv_bfloat16, 128>}}};
  const cudaError_t e = table[c.dtype == PRIMA_DT_BF16][out_dtype != PRIMA_DT_F32][c.head_dim == 128](*p, a, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? PRIMA_OK : call_cuda_fail(e, "prima_tree_attention");
}

}  // extern "C"

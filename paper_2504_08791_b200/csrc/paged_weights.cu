// The attention weight that cached positions receive in a step.
//
//   w[s][g][j] = decay * w_in[s][g][j] + sum over rows t of s and query heads h of g that see j of exp(scale q_th . k_jg - lse_th)
//
// With the log-sum-exp of the attention the probabilities need no pass of their own: one product, one exponential a pair, one
// sum.  Few rows are bound by the keys (48 single tokens over up to 8192 positions, 40 and 8 heads of 128: 26.4 us, floor 18.2 at the
// copy bandwidth), many by the exponentials, which the special-function units take at 16 a cycle and SM (64 rows of 64 heads
// over 32,704 positions: 62 us, 31 of them exponentials at the least, 20.5 products).  Polynomials on the ordinary units for a
// part of the exponentials gave 63 for 65 at that point and are not used.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <type_traits>

#include "paged_device.cuh"

namespace prima {
namespace {

struct WeightsArgs {
  PoolView pool;
  BatchView b;
  int layer, n_q_heads, group;
  float scale_log2, decay;
  const void* q;
  const float* lse;
  const float* weight_in;
  float* weight_out;
  int32_t* born;
  int64_t stride, slots;     // slots: positions that the arrays have an entry for
};

// ---- the work ---------------------------------------------------------------------------------------------------------
// Positions are independent of one another, so nothing is joined: the blocks of kBlock positions of all (sequence, KV head)
// form one line, and every worker takes an equal stretch of it.  What the first block of a (sequence, KV head) costs besides
// counts as kOverhead places in front of it (48 single tokens over up to 8192 positions: 37 us without, 26.5 with 2).
constexpr int kStreamOverhead = 2, kBlockOverhead = 1;
struct WeightsWork {
  int seq, first, nodes, ctx, head;
  int n;                     // positions that the sequence has an entry for
  int block0, block1;
};
template <int kBlock, int kOverhead>
struct WeightsCursor {
  const WeightsArgs& a;
  const int lane;
  int64_t total = 0, u = 0, u_end = 0, window = 0, before = 0, blocks = 0;
  int w0 = 0, first = 0, nodes = 0, ctx = 0;

  __device__ __forceinline__ int64_t positions(int64_t ctx_, int64_t nodes_) const { return min(ctx_ + nodes_, a.slots); }
  __device__ __forceinline__ int64_t per_head(int64_t n) const { return kOverhead + (n + kBlock - 1) / kBlock; }
  __device__ __forceinline__ bool read(int i) {
    const int f = a.b.row_begin[i], e = a.b.row_begin[i + 1], c = a.b.ctx_len[i];
    const bool ok = f >= 0 && e >= f && e <= a.b.n_tok && c >= 0;
    first = f;
    nodes = ok ? e - f : 0;
    ctx = c;
    blocks = nodes ? per_head(positions(c, nodes)) * a.pool.n_kv_heads : 0;
    return ok;
  }
  __device__ void load(int64_t in_front) {
    blocks = 0;
    if (w0 + lane < a.b.n_seq) read(w0 + lane);
    int64_t x = blocks;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    before = in_front + x - blocks;
    window = in_front + __shfl_sync(0xffffffffu, x, 31);
  }
  __device__ WeightsCursor(const WeightsArgs& args, int lane_, int worker, int n_workers) : a(args), lane(lane_) {
    if (a.b.n_seq <= 32) {      // one window holds them all
      load(0);
      total = window;
    } else {
      for (int i = lane; i < a.b.n_seq; i += 32) {
        read(i);
        total += blocks;
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    }
    if (worker == 0)
      for (int i = lane; i < a.b.n_seq; i += 32) {
        if (!read(i)) raise(a.pool.status, kBadRows);
        else if (nodes && static_cast<int64_t>(ctx) + nodes > a.slots) raise(a.pool.status, kBadSlot);
      }
    const TreeShares shares = tree_shares(total, n_workers);
    u = tree_share_begin(shares, worker);
    u_end = tree_share_begin(shares, worker + 1);
    if (u < u_end) load(0);
  }
  __device__ bool next(WeightsWork* s) {
    while (u < u_end) {
      unsigned hit;
      while (!(hit = __ballot_sync(0xffffffffu, u >= before && u < before + blocks))) {      // ends: u is below the total
        w0 += 32;
        load(window);
      }
      const int src = __ffs(hit) - 1;
      s->seq = w0 + src;
      s->first = __shfl_sync(0xffffffffu, first, src);
      s->nodes = __shfl_sync(0xffffffffu, nodes, src);
      s->ctx = __shfl_sync(0xffffffffu, ctx, src);
      s->n = static_cast<int>(positions(s->ctx, s->nodes));
      const int64_t at = u - __shfl_sync(0xffffffffu, before, src), length = per_head(s->n);
      s->head = static_cast<int>(div_small(at, length));
      const int64_t r = at - s->head * length, places = min(length - r, u_end - u);
      s->block0 = static_cast<int>(max(r - kOverhead, static_cast<int64_t>(0)));
      s->block1 = static_cast<int>(max(r - kOverhead + places, static_cast<int64_t>(0)));
      u += places;
      if (s->block1 > s->block0) return true;
    }
    return false;
  }
};

// Whether row `node` of a sequence sees its row `i` (the position behind the context).
__device__ __forceinline__ bool sees(const WeightsArgs& a, int first, int node, int i) {
  if (!a.b.mask) return i <= node;
  const uint32_t* words = reinterpret_cast<const uint32_t*>(a.b.mask + static_cast<int64_t>(first + node) * a.b.mask_words);
  return mask_word(words, 2 * a.b.mask_words, i >> 5) >> (i & 31) & 1;
}
// -lse in binary exponents; -infinity (its probabilities are 0) for a row that is none or sees nothing.
__device__ __forceinline__ float shift_of(const WeightsArgs& a, const WeightsWork& s, int row) {
  if (row >= s.nodes * a.group) return -INFINITY;
  const int node = row / a.group;
  const float lse = a.lse[(s.first + node) * a.n_q_heads + s.head * a.group + (row - node * a.group)];
  return lse == -INFINITY ? -INFINITY : -lse * kLog2e;
}
// What position j of the sequence has had, and where it is to be.
__device__ __forceinline__ int64_t entry_of(const WeightsArgs& a, const WeightsWork& s, int64_t j) {
  return (static_cast<int64_t>(s.seq) * a.pool.n_kv_heads + s.head) * a.stride + j;
}
__device__ __forceinline__ void put_entry(const WeightsArgs& a, const WeightsWork& s, int j, float had, float sum) {
  const int64_t at = entry_of(a, s, j);
  a.weight_out[at] = j < s.ctx && a.weight_in ? fmaf(a.decay, had, sum) : sum;
  if (a.born && j >= s.ctx) a.born[at] = a.b.pos ? a.b.pos[s.first + (j - s.ctx)] : j;
}

// ---- few rows -----------------------------------------------------------------------------------------------------------
// Scores with the positions as rows of m16n8k16 products and the query rows as columns, S^T = K Q^T: a lane then holds
// scores of two positions, and the sum over the rows is one over its own columns and the quad.  A worker is a warp: it copies
// 16 positions at a time through a ring of its own, some steps ahead and on into its next stretches, and keeps kTiles * 8
// rows of queries in registers; where a sequence has more, it reads its queries again for every 16 positions (all sums of a
// position before what it had is added, which may be larger than all of them).
template <int D> struct StreamGeometry {
  static constexpr int kWarps = 8, kStages = D == 128 ? 3 : 6;
  static constexpr int kPanel = kFewPos * 128;                 // 64 columns of the keys of a step
  static constexpr int kStage = kFewPos * D * 2;
  static constexpr int kWarpBytes = kStages * kStage;
};
struct StreamControl {
  unsigned long long full[8][6];
  WeightsWork fifo[8][8];              // stretches between a warp's copies (at most five steps ahead) and its products
  int give_up;
};
constexpr int kStreamCtas = 2;         // per SM: what the registers allow
template <typename T, int D, int kTiles>
__global__ void __launch_bounds__(256, kStreamCtas) weights_stream_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ WeightsArgs a) {
  using Geo = StreamGeometry<D>;
  constexpr bool kBf16 = !__is_same(T, __half);
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ StreamControl ctl;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
  int* const status = a.pool.status;
  uint8_t* const base = smem + (1024 - (smem_u32(smem) & 1023)) % 1024;
  const uint32_t ring_addr = smem_u32(base) + warp * Geo::kWarpBytes, bar_full = smem_u32(ctl.full[warp]);
  pdl_trigger();
  if (tid == 0) {
    ctl.give_up = 0;
    tma_prefetch_map(&k_map);
  }
  if (lane < 6) mbar_init(bar_full + 8 * lane, 1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  __syncthreads();
  pdl_wait();
  const int shift = a.pool.page_shift;
  // Copies of a step: lane i < boxes takes 64 columns of box_rows positions.
  const int box_rows = min(1 << shift, kFewPos), halves = kFewPos / box_rows, boxes = D / 64 * halves;
  const int panel = lane / halves, half = lane % halves;
  const uint32_t box_at = ring_addr + panel * Geo::kPanel + half * box_rows * 128;

  WeightsCursor<kFewPos, kStreamOverhead> cursor(a, lane, blockIdx.x * Geo::kWarps + warp, gridDim.x * Geo::kWarps);
  RingPlace<Geo::kStages> put, get;
  uint32_t bad_stages[2] = {0, 0}, planned = 0, begun = 0;      // stages whose positions 0..7, 8..15 have no keys
  // The stretch that is copied, its next block, the page that this lane's box of that block lies on
  WeightsWork from{};
  int next = 0, page = -1;
  bool more = false;
  auto read_page = [&]() {
    const int pos = next * kFewPos + half * box_rows, slot = pos >> shift;
    page = more && lane < boxes && pos < from.n && slot < a.b.table_stride ? a.b.table[from.seq * a.b.table_stride + slot] : -1;
  };
  auto plan = [&]() {
    more = cursor.next(&from);
    next = from.block0;
    if (more) {
      __syncwarp();
      if (lane == 0) ctl.fifo[warp][planned & 7] = from;
      __syncwarp();
      ++planned;
    }
  };
  auto copy = [&]() {
    if (!more) return;
    const int pos = next * kFewPos + half * box_rows;
    const bool wanted = lane < boxes && pos < from.n, good = static_cast<unsigned>(page) < static_cast<unsigned>(a.pool.n_pages);
    if (wanted && !good) raise(status, pos >> shift < a.b.table_stride ? kBadPage : kBadSlot);
    const uint32_t copies = __ballot_sync(0xffffffffu, wanted && good);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool bad = __any_sync(0xffffffffu, wanted && !good && (halves == 1 || half == h));
      bad_stages[h] = (bad_stages[h] & ~(1u << put.slot)) | (bad ? 1u << put.slot : 0u);
    }
    if (lane == 0) mbar_expect(bar_full + 8 * put.slot, static_cast<uint32_t>(__popc(copies)) * box_rows * 128);
    __syncwarp();
    // below 2^31 rows (prima_paged_create)
    const int row = (((a.layer * a.pool.n_pages + page) * a.pool.n_kv_heads + from.head) << shift) + (pos & ((1 << shift) - 1));
    if (wanted && good) tma_load_2d(box_at + put.slot * Geo::kStage, &k_map, panel * 64, row, bar_full + 8 * put.slot);
    put.step(1);
    if (++next == from.block1) plan();
    read_page();
  };
  plan();
  read_page();
#pragma unroll 1
  for (int i = 0; i < Geo::kStages - 1; ++i) copy();

  while (begun < planned) {
    const WeightsWork s = ctl.fifo[warp][begun & 7];
    ++begun;
    const int rows = s.nodes * a.group;      // n_tok * n_q_heads is below 2^31
    const float* const had_from = a.weight_in ? a.weight_in + entry_of(a, s, 0) : nullptr;
    // Fragments of the queries: column g of tile n, elements 2 t4, + 1 and + 8, + 9 of every 16
    uint32_t q[kTiles][D / 16][2];
    float down[kTiles][2];
    auto load_queries = [&](int row0) {
#pragma unroll
      for (int n = 0; n < kTiles; ++n) {
        const int row = row0 + 8 * n + g, node = row / a.group;
        const uint32_t* src = reinterpret_cast<const uint32_t*>(static_cast<const T*>(a.q) + static_cast<int64_t>((s.first + node) * a.n_q_heads + s.head * a.group + (row - node * a.group)) * D) + t4;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          q[n][k][0] = row < rows ? src[8 * k] : 0u;
          q[n][k][1] = row < rows ? src[8 * k + 4] : 0u;
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) down[n][e] = shift_of(a, s, row0 + 8 * n + 2 * t4 + e);
        // A row that adds nothing: its scores are 0, whatever its query holds (its shift makes them 0 as probabilities).
        const float even = __shfl_sync(0xffffffffu, down[n][0], g >> 1), odd = __shfl_sync(0xffffffffu, down[n][1], g >> 1);
        if ((g & 1 ? odd : even) == -INFINITY)
#pragma unroll
          for (int k = 0; k < D / 16; ++k) q[n][k][0] = q[n][k][1] = 0u;
      }
    };
    // What position g (lanes with t4 = 0) or g + 8 (t4 = 1) of a block has had, read a block ahead
    auto had_of = [&](int block) {
      const int j = block * kFewPos + 8 * t4 + g;
      return t4 < 2 && had_from && block < s.block1 && j < min(s.n, s.ctx) ? __ldcg(had_from + j) : 0.f;
    };
    const bool again = rows > 8 * kTiles;
    float had_next = had_of(s.block0);
    load_queries(0);
#pragma unroll 1
    for (int block = s.block0; block < s.block1; ++block) {
      __syncwarp();      // all have read the step whose place is filled again
      copy();
      const float had = had_next;
      had_next = had_of(block + 1);
      wait_for(bar_full + 8 * get.slot, get.phase, &ctl.give_up, status);
      const uint32_t kk = ring_addr + get.slot * Geo::kStage;
      const bool bad[2] = {(bad_stages[0] >> get.slot & 1) != 0, (bad_stages[1] >> get.slot & 1) != 0};
      const bool edge = bad[0] || bad[1] || block * kFewPos + kFewPos > s.ctx;
      float sum[2] = {0.f, 0.f};
#pragma unroll 1
      for (int row0 = 0; row0 < rows; row0 += 8 * kTiles) {
        if (again) load_queries(row0);
        float c[kTiles][4];
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) c[n][e] = 0.f;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          uint32_t x[4];
          const int row = lane & 15, chunk = 2 * k + (lane >> 4);
          ldsm4(x, kk + chunk / 8 * Geo::kPanel + row * 128 + (chunk % 8 ^ (row & 7)) * 16);
#pragma unroll
          for (int n = 0; n < kTiles; ++n) mma16816<kBf16>(c[n], x, q[n][k][0], q[n][k][1]);
        }
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float p = ex2(fmaf(c[n][e], a.scale_log2, down[n][e & 1]));
            if (edge) {
              const int row = row0 + 8 * n + 2 * t4 + (e & 1), i = block * kFewPos + 8 * (e >> 1) + g - s.ctx;
              if (bad[e >> 1] || down[n][e & 1] == -INFINITY || (i >= 0 && !sees(a, s.first, row / a.group, i))) p = 0.f;
            }
            sum[e >> 1] += p;
          }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 1);
        sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 2);
      }
      if (t4 < 2) {
        const int j = block * kFewPos + 8 * t4 + g;
        if (j < s.n) put_entry(a, s, j, had, t4 ? sum[1] : sum[0]);
      }
      get.step(1);
    }
  }
  // A wait that gave up may have left copies under way: they end before the memory is given back.
  if (*static_cast<volatile int*>(&ctl.give_up))
    for (uint32_t i = 0; i < Geo::kStages; ++i)
      for (int j = 0; j < (1 << 16) && !mbar_test(bar_full + 8 * i, i < put.slot ? put.phase : put.phase ^ 1); ++j) {}
}

// ---- many rows ----------------------------------------------------------------------------------------------------------
// The same product on the tensor core: 128 positions (the rows of an accumulator) by tiles of 128 query rows (its columns),
// so that a thread has one position and adds over its columns, without any exchange; neither maximum nor second product is
// needed.  One persistent CTA per SM: warp 8 copies keys page by page into a ring, warp 9 issues the products, warp 10 plans,
// and two groups of four warps take the exponentials, each from two accumulators of its own in turns.  The tiles of a block
// of positions alternate between the groups (a single tile: the blocks do); up to four tiles stay in shared memory for a
// whole stretch, more are read again for every block, the next one under the exponentials of this one.
constexpr int kBlockThreads = 384, kRowTile = 128;
template <int D> struct BlockGeometry {
  static constexpr int kTileBytes = kRowTile * D * 2;          // queries of a tile
  static constexpr int kSlotBytes = kTilePos * D * 2;          // keys of a block
  static constexpr int kPanel = kTilePos * 128;                // 64 columns of either
  static constexpr int kSlots = D == 128 ? 3 : 6;
  static constexpr int kBytes = 4 * kTileBytes + kSlots * kSlotBytes;
};
struct BlockControl {
  unsigned long long full[6], empty[6], s_ready[4], s_free[4], q_ready[4], part_full, part_free, drained;
  unsigned long long work_full[2], work_empty[2];
  WeightsWork work[2];                 // block0 = block1: no more
  uint32_t tmem;
  int give_up;
  int bad[16];                         // of the last blocks: some page is none (ring and accumulators hold at most ten)
  alignas(16) float shift[4][kRowTile];      // [2 * group + slot]
  float part[kTilePos];                // sums of the second group
};

template <typename T, int D>
__global__ void __launch_bounds__(kBlockThreads, 1) weights_block_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ WeightsArgs a) {
  using Geo = BlockGeometry<D>;
  constexpr bool kBf16 = !__is_same(T, __half);
  extern __shared__ __align__(1024) uint8_t smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  int* const status = a.pool.status;
  if (smem_u32(smem) & 1023) {      // never seen, as in tree attention
    pdl_wait();
    if (tid == 0) raise(status, kGaveUp);
    return;
  }
  uint8_t* const s_ring = smem + 4 * Geo::kTileBytes;
  BlockControl* const ctl = reinterpret_cast<BlockControl*>(smem + Geo::kBytes);
  int* const give_up = &ctl->give_up;
  const uint32_t bar_full = smem_u32(ctl->full), bar_empty = smem_u32(ctl->empty), bar_s = smem_u32(ctl->s_ready), bar_free = smem_u32(ctl->s_free), bar_q = smem_u32(ctl->q_ready),
                 bar_part = smem_u32(&ctl->part_full), bar_part_free = smem_u32(&ctl->part_free), bar_work = smem_u32(ctl->work_full), bar_work_empty = smem_u32(ctl->work_empty);
  pdl_trigger();
  if (tid == 0) {
    for (int i = 0; i < 6; ++i) {
      mbar_init(bar_full + 8 * i, 1);
      mbar_init(bar_empty + 8 * i, 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar_s + 8 * i, 1);
      mbar_init(bar_free + 8 * i, 4);
      mbar_init(bar_q + 8 * i, 4);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_work + 8 * i, 1);
      mbar_init(bar_work_empty + 8 * i, 10);
    }
    mbar_init(bar_part, 4);
    mbar_init(bar_part_free, 4);
    mbar_init(smem_u32(&ctl->drained), 1);
    ctl->give_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma_prefetch_map(&k_map);
  }
  if (warp == 9) tmem_alloc(smem_u32(&ctl->tmem), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl->tmem;      // accumulators: columns 128 * (2 * group + turn)
  pdl_wait();

  // Stretch i of this CTA, or nothing when there are no more; the caller's warp gives it back with done_with(i).
  auto work = [&](uint32_t i) -> const WeightsWork* {
    const WeightsWork* s = &ctl->work[i & 1];
    if (!wait_segment(bar_work + 8 * (i & 1), i >> 1 & 1)) {
      if (lane == 0) raise(status, kGaveUp);
      return nullptr;
    }
    return s->block1 > s->block0 ? s : nullptr;
  };
  auto done_with = [&](uint32_t i) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar_work_empty + 8 * (i & 1));
  };
  auto tiles_of = [&](const WeightsWork& s) { return (s.nodes * a.group + kRowTile - 1) / kRowTile; };
  RingPlace<Geo::kSlots> ring;
  uint32_t copies_before = 0;      // copies: places used so far, up to kSlots (the ring is empty at first)

  if (warp == 10) {
    // ---- the plan ----
    WeightsCursor<kTilePos, kBlockOverhead> cursor(a, lane, blockIdx.x, gridDim.x);
    WeightsWork s;
    for (uint32_t i = 0;; ++i) {
      const bool more = cursor.next(&s);
      if (i >= 2 && !__all_sync(0xffffffffu, wait_segment(bar_work_empty + 8 * (i & 1), (i / 2 - 1) & 1))) {      // never seen; what others may still read stays
        if (lane == 0) raise(status, kGaveUp);
        break;
      }
      if (lane == 0) {
        ctl->work[i & 1] = s;
        if (!more) ctl->work[i & 1].block0 = ctl->work[i & 1].block1 = 0;
        mbar_arrive(bar_work + 8 * (i & 1));
      }
      __syncwarp();
      if (!more) break;
    }
  } else if (warp == 8) {
    // ---- copies ----
    const int shift = a.pool.page_shift, box_rows = min(1 << shift, kTilePos), boxes = kTilePos / box_rows;
    const int box = lane % boxes, panel = lane / boxes;
    const uint32_t dst = smem_u32(s_ring) + panel * Geo::kPanel + box * box_rows * 128;
    uint32_t n_read = 0;
    const WeightsWork* w;
    for (uint32_t i = 0; (w = work(i)); ++i) {
      const WeightsWork s = *w;
      done_with(i);
      const int32_t* table = a.b.table + s.seq * a.b.table_stride;
      // The page that this lane's box of a block lies on, read a block ahead
      auto page_of = [&](int block) {
        const int pos = block * kTilePos + box * box_rows, slot = pos >> shift;
        return panel < D / 64 && block < s.block1 && pos < s.n && slot < a.b.table_stride ? table[slot] : -1;
      };
      int next_page = page_of(s.block0);
      for (int block = s.block0; block < s.block1; ++block) {
        const int pos = block * kTilePos + box * box_rows, page = next_page;
        next_page = page_of(block + 1);
        const bool wanted = panel < D / 64 && pos < s.n, bad = wanted && static_cast<unsigned>(page) >= static_cast<unsigned>(a.pool.n_pages);
        int row = -1;      // below 2^31 (prima_paged_create)
        if (bad) raise(status, pos >> shift < a.b.table_stride ? kBadPage : kBadSlot);
        else if (wanted) row = (((a.layer * a.pool.n_pages + page) * a.pool.n_kv_heads + s.head) << shift) + (pos & ((1 << shift) - 1));
        const int n_copies = __popc(__ballot_sync(0xffffffffu, row >= 0));
        const bool any_bad = __any_sync(0xffffffffu, bad);
        bool ok = true;
        if (copies_before >= Geo::kSlots) ok = wait_for(bar_empty + 8 * ring.slot, ring.phase ^ 1, give_up, status);
        if (__all_sync(0xffffffffu, ok)) {
          if (lane == 0) {
            ctl->bad[n_read % 16] = any_bad;
            mbar_expect(bar_full + 8 * ring.slot, static_cast<uint32_t>(n_copies) * box_rows * 128);
          }
          __syncwarp();
          if (row >= 0) tma_load_2d(dst + ring.slot * Geo::kSlotBytes, &k_map, panel * 64, row, bar_full + 8 * ring.slot);
        }
        ring.step(1);
        if (copies_before < Geo::kSlots) ++copies_before;
        ++n_read;
      }
    }
  } else if (warp == 9) {
    // ---- products ----
    constexpr uint32_t kDesc = mma_f16_desc(kBf16, false, kTilePos, kRowTile);
    const uint32_t u_tmem = uniform(tmem), ring_addr = uniform(smem_u32(s_ring)), q_addr = uniform(smem_u32(smem));
    const SmemOperand k_all = smem_operand(ring_addr, 16);
    uint32_t turn[2] = {0, 0}, loads[4] = {0, 0, 0, 0};      // of the groups; of the tiles' places
    const WeightsWork* w;
    for (uint32_t i = 0; (w = work(i)); ++i) {
      const int tiles = uniform(tiles_of(*w)), blocks = uniform(w->block1 - w->block0);
      done_with(i);
      const bool again = tiles > 4;
      uint32_t in_stretch[2] = {0, 0};      // tiles of the groups
      bool ok = true;
      for (int block = 0; block < blocks; ++block) {
        ok = wait_for(bar_full + 8 * ring.slot, ring.phase, give_up, status) && ok;
        for (int t = 0; t < tiles; ++t) {
          const uint32_t h = tiles == 1 ? block & 1 : t & 1, n = h ? turn[1]++ : turn[0]++, nth = h ? in_stretch[1]++ : in_stretch[0]++;
          const uint32_t q = 2 * h + (again ? nth & 1 : tiles == 1 ? 0 : t >> 1);      // place of the tile
          if (again || block < (tiles == 1 ? 2 : 1)) {
            uint32_t phase = 0;      // no indexed registers
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j)
              if (j == q) phase = loads[j]++ & 1;
            ok = wait_for(bar_q + 8 * q, phase, give_up, status) && ok;
          }
          const uint32_t d = 2 * h + (n & 1);
          if (n >= 2) ok = wait_for(bar_free + 8 * d, (n / 2 - 1) & 1, give_up, status) && ok;
          tc_fence_after();
          if (__all_sync(0xffffffffu, ok) && elect_one()) {
            const SmemOperand qq = smem_operand(q_addr + q * Geo::kTileBytes, 16), kk = k_all + ring.slot * Geo::kSlotBytes;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) mma_ss(u_tmem + kRowTile * d, kk + (k / 4 * Geo::kPanel + k % 4 * 32), qq + (k / 4 * Geo::kPanel + k % 4 * 32), kDesc, k > 0);
            tc_commit(bar_s + 8 * d);
            if (t == tiles - 1) tc_commit(bar_empty + 8 * ring.slot);
          }
          __syncwarp();
        }
        ring.step(1);
      }
    }
  } else if (warp < 8) {
    // ---- exponentials and sums ----
    const int h = warp >> 2, quarter = warp & 3, r = quarter * 32 + lane;
    const uint32_t t_s = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + 2 * h * kRowTile;
    uint32_t turn = 0, n_part = 0, unit_base = 0;
    // Tile t of a stretch into place p of this group, in the background, and its rows' shifts.  `empty`, a bit for each place: this
    // thread's row adds nothing.
    uint32_t empty = 0;
    auto load_tile = [&](const WeightsWork& s, int t, int p) {
      const int row0 = t * kRowTile, token0 = row0 / a.group;
      load_query_tile<T, D>(smem_u32(smem) + (2 * h + p) * Geo::kTileBytes, Geo::kPanel,
                            static_cast<const T*>(a.q) + (static_cast<int64_t>(s.first + token0) * a.n_q_heads + s.head * a.group) * D, row0 - token0 * a.group, a.group,
                            static_cast<int64_t>(a.n_q_heads) * D, s.nodes * a.group - row0, r);
      const float shift = shift_of(a, s, t * kRowTile + r);
      ctl->shift[2 * h + p][r] = shift;
      const bool none = shift == -INFINITY && t * kRowTile + r < s.nodes * a.group;      // rows behind the last one are zeros already
      empty = (empty & ~(1u << p)) | (none ? 1u << p : 0u);
    };
    auto group_sync = [&]() { asm volatile("bar.sync %0, 128;" ::"r"(1 + h) : "memory"); };
    auto tile_ready = [&](int p) {
      asm volatile("cp.async.wait_all;" ::: "memory");
      fence_async_smem();
      group_sync();      // the group reads all shifts
      if (empty >> p & 1) {      // scores of 0, whatever the query holds
#pragma unroll
        for (int c = 0; c < D / 8; ++c) *reinterpret_cast<uint4*>(smem + (2 * h + p) * Geo::kTileBytes + c / 8 * Geo::kPanel + r * 128 + c % 8 * 16) = make_uint4(0, 0, 0, 0);
        fence_async_smem();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_q + 8 * (2 * h + p));
    };
    const float2 scale = make_float2(a.scale_log2, a.scale_log2);
    const WeightsWork* w;
    for (uint32_t i = 0; (w = work(i)); ++i) {
      const WeightsWork& s = *w;
      const int tiles = tiles_of(s), blocks = s.block1 - s.block0;
      const bool single = tiles == 1, again = tiles > 4;
      const int mine = single ? 1 : (tiles - h + 1) >> 1;      // tiles of this group
      const int32_t* const table = a.b.table + s.seq * a.b.table_stride;
      // The places are free: all of this group have seen the last scores of the stretch before and read its shifts.
      group_sync();
      if (!single || h < blocks) {
        for (int p = 0; p < min(mine, 2); ++p) load_tile(s, single ? 0 : 2 * p + h, p);
        for (int p = 0; p < min(mine, 2); ++p) tile_ready(p);
      }
      uint32_t nth = 0;      // tile of this group
#pragma unroll 1
      for (int block = single ? h : 0; block < blocks; block += single ? 2 : 1) {
        const int pos0 = (s.block0 + block) * kTilePos, j = pos0 + r;
        float had = 0.f;
        if ((single || h == 0) && a.weight_in && j < min(s.n, s.ctx)) had = a.weight_in[entry_of(a, s, j)];      // may be weight_out
        float2 sum = make_float2(0.f, 0.f);
        bool hidden = false;
#pragma unroll 1
        for (int m = 0; m < mine; ++m, ++turn, ++nth) {
          const int t = single ? 0 : 2 * m + h, p = again ? nth & 1 : m;
          const uint32_t d = turn & 1;
          wait_for(bar_s + 8 * (2 * h + d), turn >> 1 & 1, give_up, status);
          tc_fence_after();
          if (m == 0) hidden = *static_cast<volatile int*>(&ctl->bad[(unit_base + block) % 16]) != 0 && (j >= s.n || find_slot(a.pool, table, a.b.table_stride, a.layer, j) < 0);
          const bool edge = pos0 + kTilePos > s.ctx;
          const int behind = j - s.ctx;      // index of the position among the rows of the step
          const float* const shift = ctl->shift[2 * h + p];
          const int chunks = min(kRowTile / 32, (s.nodes * a.group - t * kRowTile + 31) >> 5);      // 32 columns each that hold rows
          // Full tiles, whose columns are known when this is compiled, and others.  64 rows of 64 heads over 32,704 positions 61 us,
          // with one body for both 64, with full tiles alone 60; but then 16 sequences of 4096 with 24 rows 36 us, so 32.
          auto take = [&](auto full) {
            constexpr bool kFull = decltype(full)::value;
            uint32_t x[2][32];
            tmem_load(x[0], t_s + kRowTile * d);
  #pragma unroll
            for (int c = 0; c < kRowTile / 32; ++c) {
              if (!kFull && c == chunks) break;
              tmem_wait_load();
              tmem_use(x[c & 1]);
              if (kFull ? c + 1 < kRowTile / 32 : c + 1 < chunks) {
                tmem_load(x[(c + 1) & 1], t_s + kRowTile * d + 32 * (c + 1));
              } else {      // all are read: the next product may have the accumulator
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_free + 8 * (2 * h + d));
              }
              uint32_t seen = 0xffffffffu;
              if (edge && behind >= 0) {
                const int row = t * kRowTile + 32 * c;
                if (!a.b.mask) {      // rows from the position's own node on
                  const long long skip = static_cast<long long>(behind) * a.group - row;
                  seen = skip >= 32 ? 0u : skip <= 0 ? 0xffffffffu : 0xffffffffu << static_cast<int>(skip);
                } else {
                  seen = 0;
  #pragma unroll 1
                  for (int e = 0; e < 32; ++e) {
                    const int node = (row + e) / a.group;
                    if (node < s.nodes && sees(a, s.first, node, behind)) seen |= 1u << e;
                  }
                }
              }
  #pragma unroll
              for (int e = 0; e < 32; e += 4) {
                const float4 z = *reinterpret_cast<const float4*>(shift + 32 * c + e);
                float2 u = fma2(make_float2(__uint_as_float(x[c & 1][e]), __uint_as_float(x[c & 1][e + 1])), scale, make_float2(z.x, z.y));
                float2 v = fma2(make_float2(__uint_as_float(x[c & 1][e + 2]), __uint_as_float(x[c & 1][e + 3])), scale, make_float2(z.z, z.w));
                u = make_float2(ex2(u.x), ex2(u.y));
                v = make_float2(ex2(v.x), ex2(v.y));
                if (edge) {
                  u.x = seen >> e & 1 ? u.x : 0.f;
                  u.y = seen >> (e + 1) & 1 ? u.y : 0.f;
                  v.x = seen >> (e + 2) & 1 ? v.x : 0.f;
                  v.y = seen >> (e + 3) & 1 ? v.y : 0.f;
                }
                sum = add2(sum, add2(u, v));
              }
            }
          };
          if (chunks == kRowTile / 32) take(std::true_type());
          else take(std::false_type());
          // Many tiles: the one after the next into this place, whose scores are there (for the next block, from the first on).
          if (again && !(block == blocks - 1 && m + 2 >= mine)) {
            group_sync();      // all have read the shifts
            load_tile(s, 2 * (m + 2 < mine ? m + 2 : m + 2 - mine) + h, p);
            tile_ready(p);
          }
        }
        float total = sum.x + sum.y;
        if (!single) {
          const uint32_t phase = n_part++ & 1;
          if (h == 1) {
            if (n_part > 1) wait_for(bar_part_free, phase ^ 1, give_up, status);
            ctl->part[r] = total;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_part);
          } else {
            wait_for(bar_part, phase, give_up, status);
            total += ctl->part[r];
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_part_free);
          }
        }
        if ((single || h == 0) && j < s.n) put_entry(a, s, j, had, hidden ? 0.f : total);
      }
      unit_base += blocks;
      done_with(i);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // A wait that gave up may have left products or copies under way: they end before the memory is given back.
  if (ctl->give_up) {
    if (tid == 9 * 32) {
      tc_commit(smem_u32(&ctl->drained));
      for (int i = 0; i < (1 << 22) && !mbar_test(smem_u32(&ctl->drained), 0); ++i) {}
    }
    if (tid == 8 * 32)
      for (uint32_t p = 0; p < copies_before; ++p) {      // the last places
        ring.phase ^= ring.slot == 0;
        ring.slot = ring.slot == 0 ? Geo::kSlots - 1 : ring.slot - 1;
        for (int i = 0; i < (1 << 16) && !mbar_test(bar_full + 8 * ring.slot, ring.phase); ++i) {}
      }
    __syncthreads();
  }
  if (warp == 9) tmem_free(tmem, 512);
}

constexpr int64_t kLongest = 2147483647 - 255;      // positions that the arrays may have entries for: numbers of blocks' ends fit 32 bits

template <typename T, int D, int kTiles>
cudaError_t launch_stream(const prima_paged& pool, const WeightsArgs& a, cudaStream_t st) {
  constexpr size_t kSmem = 1024 + StreamGeometry<D>::kWarps * StreamGeometry<D>::kWarpBytes;
  static bool done[kMaxDevices] = {};
  auto kernel = weights_stream_kernel<T, D, kTiles>;
  const cudaError_t e = allow_smem(kernel, kSmem, done);
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3(kStreamCtas * pool.sm_count), dim3(256), kSmem, st, static_cast<const Maps*>(pool.maps)->k_few, a);
}
template <typename T, int D>
cudaError_t launch_block(const prima_paged& pool, const WeightsArgs& a, cudaStream_t st) {
  constexpr size_t kSmem = BlockGeometry<D>::kBytes + sizeof(BlockControl);
  static_assert(kSmem <= 232448, "shared memory of a CTA");
  static bool done[kMaxDevices] = {};
  auto kernel = weights_block_kernel<T, D>;
  const cudaError_t e = allow_smem(kernel, kSmem, done);
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3(pool.sm_count), dim3(kBlockThreads), kSmem, st, static_cast<const Maps*>(pool.maps)->k, a);
}
template <typename T, int D>
cudaError_t launch_weights(const prima_paged& pool, const WeightsArgs& a, cudaStream_t st) {
  // Rows that a KV head has of a sequence on average; each variant is right for any.  Streaming against tensor memory, 8 KV
  // heads, B200: of 128, 16 sequences of 4096 positions, 4 rows 27 and 33 us, 16 rows 29 and 33; 64 of 600, 15 and 26, 19 and 26;
  // one of 8192, 6.7 and 8.8, 9.3 and 8.8.  Of 64, 17 and 24, 23 and 24; 13 and 22, 16 and 22; 6.1 and 7.7, 8.0 and 7.7.  32 rows
  // in registers: heads of 128 53 and 33, 35 and 26, 14 and 8.7; of 64 31 and 24, 22 and 21, 12 and 7.7.
  const int64_t rows = (static_cast<int64_t>(a.b.n_tok) + a.b.n_seq - 1) / a.b.n_seq * a.group;
  if (rows > 16) return launch_block<T, D>(pool, a, st);
  return (rows <= 8 ? launch_stream<T, D, 1> : launch_stream<T, D, 2>)(pool, a, st);
}

}  // namespace
}  // namespace prima

using namespace prima;

extern "C" {

int prima_paged_weights(prima_paged* p, int layer, const prima_paged_batch* batch, const void* q, int n_q_heads, float scale, const float* lse,
                        const float* weight_in, float* weight_out, int32_t* born, int64_t stride, float decay, void* stream) {
  const int rc = check_batch(p, batch, "prima_paged_weights");
  if (rc != PRIMA_OK) return rc;
  auto refuse = [](const char* what) {
    char msg[160];
    snprintf(msg, sizeof msg, "prima_paged_weights: %s", what);
    return call_fail(PRIMA_ERR_ARG, msg);
  };
  const prima_paged_config& c = p->cfg;
  if (layer < 0 || layer >= c.n_layers) return refuse("layer out of range");
  if (!q || !lse || !weight_out) return refuse("null q, lse or weight_out");
  if (n_q_heads < 1 || n_q_heads % c.n_kv_heads || n_q_heads / c.n_kv_heads > 64) return refuse("n_q_heads must be a multiple of n_kv_heads, at most 64 times it");
  if (!(scale > 0.f) || std::isinf(scale)) return refuse("scale must be positive and finite");
  if (!(decay >= 0.f && decay <= 1.f)) return refuse("decay outside 0..1");
  if (stride < 1 || stride > kLongest) return refuse("stride outside 1..2^31 - 256");
  if (!aligned_to(q, 16)) return refuse("q must be 16-byte aligned");
  if (!aligned_to(lse, 4) || !aligned_to(weight_in, 4) || !aligned_to(weight_out, 4) || !aligned_to(born, 4)) return refuse("an array is not 4-byte aligned");
  if (static_cast<int64_t>(batch->n_tok) * n_q_heads > 2147483647) return refuse("n_tok * n_q_heads reaches 2^31");
  const int64_t bytes = 4 * static_cast<int64_t>(batch->n_seq) * c.n_kv_heads * stride;
  const char *in = reinterpret_cast<const char*>(weight_in), *to = reinterpret_cast<const char*>(weight_out);
  if (in && in != to && in < to + bytes && to < in + bytes) return refuse("weight_in overlaps weight_out without being it");
  CallDevice dev(c.device);
  if (!dev.ok) return call_fail(PRIMA_ERR_CUDA, "cudaSetDevice failed");
  WeightsArgs a;
  a.pool = view_of(*p);
  a.b = view_of(*batch);
  a.layer = layer;
  a.n_q_heads = n_q_heads;
  a.group = n_q_heads / c.n_kv_heads;
  a.scale_log2 = scale * kLog2e;
  a.decay = decay;
  a.q = q;
  a.lse = lse;
  a.weight_in = weight_in;
  a.weight_out = weight_out;
  a.born = born;
  a.stride = a.slots = stride;
  using launcher = cudaError_t (*)(const prima_paged&, const WeightsArgs&, cudaStream_t);
  static const launcher table[2][2] = {{launch_weights<__half, 64>, launch_weights<__half, 128>}, {launch_weights<__nv_bfloat16, 64>, launch_weights<__nv_bfloat16, 128>}};
  const cudaError_t e = table[c.dtype == PRIMA_DT_BF16][c.head_dim == 128](*p, a, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? PRIMA_OK : call_cuda_fail(e, "prima_paged_weights");
}

}  // extern "C"

// Index arithmetic of the paged cache, in plain C++: the kernels use it, and the tests run it on the host.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define PRIMA_HD __host__ __device__ __forceinline__
#else
#define PRIMA_HD inline
#endif

namespace prima {

// Bits of the pool's status word.
constexpr int kBadPage = 1;      // a page id outside 0 .. n_pages - 1
constexpr int kBadSlot = 2;      // a slot beyond the page table
constexpr int kBadRows = 4;      // row_begin decreases or ends beyond n_tok, or a negative length
constexpr int kBadPath = 8;      // a path entry outside the step, a parent outside the beams
constexpr int kGaveUp = 16;      // a bounded wait inside a kernel gave up

struct PageShape {
  int n_layers, n_pages, page_shift, n_kv_heads;
};

// Row of the arrays [n_layers * n_pages * n_kv_heads * page_size][head_dim] that holds slot `slot` of KV head 0 of a
// sequence in `layer` (rows of KV head g follow at g << page_shift), or minus the bit to raise.
PRIMA_HD int64_t find_slot(const PageShape& p, const int32_t* table_row, int64_t table_stride, int layer, int64_t slot) {
  if (slot < 0 || (slot >> p.page_shift) >= table_stride) return -kBadSlot;
  const int page = table_row[slot >> p.page_shift];
  if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.n_pages)) return -kBadPage;
  return (((static_cast<int64_t>(layer) * p.n_pages + page) * p.n_kv_heads) << p.page_shift) + (slot & ((1 << p.page_shift) - 1));
}

// ---- how the work of tree attention is dealt out -------------------------------------------------------------------
// The rows of a sequence that read one KV head (node-major: row = node * group + query head in the group) are cut into
// tiles of tile_rows, the positions that a tile may see into units of kTilePos.  The units of all sequences, KV heads
// and row tiles, in this order, form one line that is cut into equal shares, one per CTA, so that long and short
// sequences balance.  A stretch of units of one (sequence, KV head, row tile) inside a share is a segment.  Queries, the
// first scores and the output cost a segment as much as some units, so each (sequence, KV head, row tile) has `overhead`
// places at its head in the line that stand for no unit.
constexpr int kTilePos = 128;

struct TreeShape {
  int n_kv_heads, group;     // query heads that share a KV head
  int causal;                // no mask: row i of a sequence sees rows 0 .. i
  int64_t capacity;          // positions that a page table row can name
  int overhead;              // what a segment costs besides its units, in units
  int tile_rows;
};

PRIMA_HD int tree_row_tiles(const TreeShape& t, int nodes) {
  return static_cast<int>((static_cast<int64_t>(nodes) * t.group + t.tile_rows - 1) / t.tile_rows);
}
// Positions 0 .. result-1 are all that the rows of tile rt may see.
PRIMA_HD int64_t tree_kv_end(const TreeShape& t, int ctx, int nodes, int rt) {
  int64_t seen = nodes;
  if (t.causal) {
    const int64_t last = (static_cast<int64_t>(rt + 1) * t.tile_rows + t.group - 1) / t.group;
    if (last < seen) seen = last;
  }
  const int64_t end = ctx + seen;
  return end < t.capacity ? end : t.capacity;
}
PRIMA_HD int64_t tree_chunks(const TreeShape& t, int ctx, int nodes, int rt) { return (tree_kv_end(t, ctx, nodes, rt) + kTilePos - 1) / kTilePos; }
// Places in the line of one (sequence, KV head, row tile).
PRIMA_HD int64_t tree_length(const TreeShape& t, int ctx, int nodes, int rt) { return t.overhead + tree_chunks(t, ctx, nodes, rt); }
PRIMA_HD int64_t tree_units(const TreeShape& t, int ctx, int nodes) {      // of one KV head of a sequence
  const int tiles = tree_row_tiles(t, nodes);
  if (!t.causal || tiles <= 1) return tiles ? tiles * tree_length(t, ctx, nodes, 0) : 0;
  int64_t n = 0;
  for (int rt = 0; rt < tiles; ++rt) n += tree_length(t, ctx, nodes, rt);
  return n;
}
// Division of non-negative numbers that are nearly always small: 64-bit division is a long subroutine on the GPU.
PRIMA_HD int64_t div_small(int64_t a, int64_t b) {
  return (a | b) >> 31 ? a / b : static_cast<int64_t>(static_cast<uint32_t>(a) / static_cast<uint32_t>(b));
}
// Shares: CTA c of n_cta has base units, the first `more` CTAs one more.
struct TreeShares {
  int64_t base;
  int more;
};
PRIMA_HD TreeShares tree_shares(int64_t units, int n_cta) {
  const int64_t q = div_small(units, n_cta);
  return {q, static_cast<int>(units - q * n_cta)};
}
PRIMA_HD int64_t tree_share_begin(const TreeShares& s, int c) { return s.base * c + (c < s.more ? c : s.more); }
// The CTA whose share holds unit u.
PRIMA_HD int tree_cta_of(const TreeShares& s, int64_t u) {
  const int64_t long_ones = (s.base + 1) * s.more;
  return static_cast<int>(u < long_ones ? div_small(u, s.base + 1) : s.more + div_small(u - long_ones, s.base));
}

// x / d for 0 <= x < 256 + 64, 1 <= d <= 64, by a multiplication with m = small_inverse(d).
PRIMA_HD uint32_t small_inverse(int d) { return 65536u / static_cast<uint32_t>(d) + 1u; }
PRIMA_HD int small_div(int x, uint32_t m) { return static_cast<int>(static_cast<uint32_t>(x) * m >> 16); }

struct TreeSegment {
  int head, row_tile;        // head: KV head
  int chunk0, chunk1;        // units of this share; none where the share has only places at the head
  int chunks;                // units of the whole (sequence, KV head, row tile)
  int64_t places;            // of this share, and to the end of the whole
  int64_t to_end;
};
// The segment at place u of a sequence whose KV heads have `per_head` places each; it ends at or before place u_end.
PRIMA_HD TreeSegment tree_segment(const TreeShape& t, int ctx, int nodes, int64_t per_head, int64_t u, int64_t u_end) {
  TreeSegment s;
  const int tiles = tree_row_tiles(t, nodes);
  s.head = static_cast<int>(div_small(u, per_head));
  int64_t r = u - s.head * per_head;
  int64_t length = tree_length(t, ctx, nodes, 0);
  int rt = 0;
  if (!t.causal) {
    rt = static_cast<int>(div_small(r, length));
    r -= rt * length;
  } else {
    while (rt + 1 < tiles && r >= length) {
      r -= length;
      length = tree_length(t, ctx, nodes, ++rt);
    }
  }
  s.row_tile = rt;
  s.chunks = static_cast<int>(length - t.overhead);
  s.to_end = length - r;
  s.places = s.to_end < u_end - u ? s.to_end : u_end - u;
  const int64_t c0 = r - t.overhead, c1 = c0 + s.places;
  s.chunk0 = static_cast<int>(c0 > 0 ? c0 : 0);
  s.chunk1 = static_cast<int>(c1 > 0 ? c1 : 0);
  return s;
}

}  // namespace prima

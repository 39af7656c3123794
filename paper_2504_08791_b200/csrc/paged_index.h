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

}  // namespace prima

// What the attention kernels over the paged cache share on the device: bounded waits, masks, the softmax's arithmetic,
// copies and fragments.
#pragma once

#include <cuda.h>

#include "paged.cuh"
#include "tcgen05.cuh"

namespace prima {

// ---- constants -------------------------------------------------------------------------------------------------------
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;
// Binary exponents: a reference is set kHeadroom below the row's maximum and stays until a score exceeds it by kSlack.  A
// row's largest probability is held as 2^7 to 2^15 (binary16 ends at 65504), not as 1: what binary16 rounds below its normal
// numbers, by up to 2^-25, is then 2^-32 of the largest, and thousands of positions that have 2^-25 of its weight
// each are not rounded away one by one.
constexpr float kHeadroom = 7.f, kSlack = 15.f;

__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, int* give_up, int* status) {
  for (int i = 0; i < (1 << 22); ++i) {
    if (mbar_test(bar, parity)) return true;
    if (*static_cast<volatile int*>(give_up)) return false;
  }
  *static_cast<volatile int*>(give_up) = 1;
  raise(status, kGaveUp);
  return false;
}

// The hand-over of segments, which goes on after a wait has given up elsewhere (nothing else may be left waiting).
__device__ __forceinline__ bool wait_segment(uint32_t bar, uint32_t parity) {
  for (int i = 0; i < (1 << 24); ++i)
    if (mbar_test(bar, parity)) return true;
  return false;
}

// ---- what a row sees ------------------------------------------------------------------------------------------------
// Bits for 32 positions from `pos` on.  a = index of the position among the rows of the step, negative in the context.
__device__ __forceinline__ uint32_t low_bits(long long n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << static_cast<int>(n)) - 1u; }
__device__ __forceinline__ uint32_t mask_word(const uint32_t* words, int n_words, long long i) { return i < n_words ? words[i] : 0u; }
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
    return static_cast<unsigned>(table[pos >> pool.page_shift]) < static_cast<unsigned>(pool.n_pages);
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

// ---- arithmetic ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A row that sees nothing has a sum of 0: its output is 0, its log-sum-exp -infinity.  A NaN stays one.
__device__ __forceinline__ float inverse_of(float total) { return total == 0.f ? 0.f : 1.f / total; }
__device__ __forceinline__ float log_sum(float reference, float total) {
  constexpr float kDown = 1.f / 128.f;      // 2^-kHeadroom
  return total == 0.f ? -INFINITY : (reference + kHeadroom + log2f(total * kDown)) * kLn2;
}

__device__ __forceinline__ float max3(float x, float y, float z) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(x), "f"(y), "f"(z));
  return d;
}
__device__ __forceinline__ float max_of(const uint32_t (&x)[32], float top) {
  float t[4] = {top, __uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(x[2])};
#pragma unroll
  for (int j = 3; j + 1 < 32; j += 2) t[j / 2 & 3] = max3(t[j / 2 & 3], __uint_as_float(x[j]), __uint_as_float(x[j + 1]));
  return fmaxf(max3(t[0], t[1], t[2]), fmaxf(t[3], __uint_as_float(x[31])));
}

template <typename T>
__device__ __forceinline__ void store4(T* dst, float4 x) {
  *reinterpret_cast<uint2*>(dst) = make_uint2(Half2Of<T>::pack(x.x, x.y), Half2Of<T>::pack(x.z, x.w));
}
template <>
__device__ __forceinline__ void store4<float>(float* dst, float4 x) { *reinterpret_cast<float4*>(dst) = x; }

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
  __device__ __forceinline__ void skip(int n) {
    for (; n > 0; n -= kSlots) step(min(n, kSlots));
  }
};

// 16 bytes to shared memory in the background; zeros where there is nothing to copy.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}

// A tile of up to 128 rows of queries into shared memory in the background, by 128 threads (r: this one): rows of 128 bytes in
// the 128-byte swizzle, 64 columns a panel; rows behind the last one are zeros.  Row x is query head (in0 + x) % group of a KV
// head, (in0 + x) / group tokens behind the one that `from` (that token's first query head of the KV head) belongs to.  A
// thread takes one 16-byte piece of every 128 / (D / 8)-th row and steps its place without divisions.
template <typename T, int D>
__device__ __forceinline__ void load_query_tile(uint32_t tile, int panel_bytes, const T* from, int in0, int group, int64_t token_stride, int rows, int r) {
  constexpr int kPieces = D / 8, kStep = 128 / kPieces;
  const int piece = r % kPieces, row0 = r / kPieces, tokens = kStep / group, heads = kStep - tokens * group;
  int token = (in0 + row0) / group, in_group = in0 + row0 - token * group;
  const uint32_t dst = tile + piece / 8 * panel_bytes;
#pragma unroll 4
  for (int row = row0; row < 128; row += kStep) {
    const bool there = row < rows;
    copy16(dst + row * 128 + ((piece % 8) ^ (row & 7)) * 16, from + (there ? token * token_stride + in_group * D : 0) + piece * 8, there);
    token += tokens;
    in_group += heads;
    if (in_group >= group) {
      in_group -= group;
      ++token;
    }
  }
  asm volatile("cp.async.commit_group;" ::: "memory");
}

// ---- fragments of m16n8k16 -------------------------------------------------------------------------------------------
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <bool kBf16>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (kBf16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int D> struct Geometry {
  static constexpr int kQBytes = 128 * D * 2;                  // one tile of 128 rows of queries
  static constexpr int kSlotBytes = kTilePos * D * 2;          // keys or values of a unit
  static constexpr int kPanel = kTilePos * 128;                // 64 columns of a unit
  static constexpr int kSlots = D == 128 ? 5 : 12;
};

// ---- host ------------------------------------------------------------------------------------------------------------
struct Maps {      // of a pool's two arrays: pages, or their rows 16 at a time
  CUtensorMap k, v, k_few, v_few;
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
template <typename Kernel>
inline cudaError_t allow_smem(Kernel kernel, size_t bytes, bool (&done)[kMaxDevices]) {
  int dev;
  if (!first_launch_on_device(done, &dev)) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
  if (e == cudaSuccess && dev >= 0) done[dev] = true;
  return e;
}

}  // namespace prima

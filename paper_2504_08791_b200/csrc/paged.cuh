// What the operators over a paged cache share: the pool, the batch as the kernels see it, type helpers.
#pragma once

#include <cuda_bf16.h>

#include "../../include/prima.h"
#include "common.cuh"
#include "paged_index.h"

struct prima_paged {
  prima_paged_config cfg{};
  void* k = nullptr;             // caller's arrays
  void* v = nullptr;
  double* freq = nullptr;        // device, [head_dim/2]: turns per position of every pair, theta^(-2i/head_dim) / (2 pi)
  int* status = nullptr;         // device word, see kBad*
  int sm_count = 0;
  int page_shift = 0;
  void* maps = nullptr;          // host, tensor maps of the two arrays (tree_attention.cu)
};

namespace prima {

// Records the text of a context-free call's error for prima_last_error(NULL); returns `code`.
int call_fail(int code, const char* what);
int call_cuda_fail(cudaError_t e, const char* what);

struct CallDevice {              // makes a device current for the duration of a call
  int prev = -1;
  bool ok = true;
  explicit CallDevice(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) prev = -1;
    ok = prev == dev || cudaSetDevice(dev) == cudaSuccess;
    if (prev == dev) prev = -1;
  }
  ~CallDevice() {
    if (prev >= 0) cudaSetDevice(prev);
  }
};

// Whether an address is a multiple of n, a power of two (device code faults on others).
inline bool aligned_to(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// The checks of a batch that need no device memory; PRIMA_OK or an error that is already recorded.
int check_batch(const prima_paged* pool, const prima_paged_batch* b, const char* who);

// The tensor maps that the attention kernel's copies use (tree_attention.cu).
cudaError_t make_tree_maps(prima_paged* pool);
void free_tree_maps(prima_paged* pool);

struct BatchView {
  int n_seq, n_tok;
  const int32_t* row_begin;
  const int32_t* ctx_len;
  const int32_t* table;
  int64_t table_stride;
  const int32_t* pos;
  const uint64_t* mask;
  int mask_words;
};
struct PoolView : PageShape {
  void* k;
  void* v;
  int* status;
};
inline BatchView view_of(const prima_paged_batch& b) {
  return {b.n_seq, b.n_tok, b.row_begin, b.ctx_len, b.table, b.table_stride, b.pos, b.mask, b.mask ? b.mask_words : 0};
}
inline PoolView view_of(const prima_paged& p) { return {{p.cfg.n_layers, p.cfg.n_pages, p.page_shift, p.cfg.n_kv_heads}, p.k, p.v, p.status}; }

#ifdef __CUDACC__
__device__ __forceinline__ void raise(int* status, int bit) { atomicOr(status, bit); }

// Sequence of row t: the number of sequences that end at or before it.  Called by a whole warp; the bounds are read
// side by side (a binary search would be a chain of dependent reads, 0.5 us each).
__device__ __forceinline__ int seq_of_row(const BatchView& b, int t, int lane) {
  int n = 0;
  for (int i = lane; i < b.n_seq; i += 32) n += __ldg(b.row_begin + i + 1) <= t ? 1 : 0;
  return __reduce_add_sync(0xffffffffu, n);
}

// find_slot, with the status word raised for a bad entry (-1).
__device__ __forceinline__ int64_t slot_row(const PoolView& p, const int32_t* table_row, int64_t table_stride, int layer, int64_t slot) {
  const int64_t row = find_slot(p, table_row, table_stride, layer, slot);
  if (row >= 0) return row;
  raise(p.status, static_cast<int>(-row));
  return -1;
}

template <typename T> struct Half2Of;
template <> struct Half2Of<__half> {
  __device__ static uint32_t pack(float a, float b) { const __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<const uint32_t*>(&h); }
  __device__ static float2 unpack(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }
};
template <> struct Half2Of<__nv_bfloat16> {
  __device__ static uint32_t pack(float a, float b) { const __nv_bfloat162 h = __floats2bfloat162_rn(a, b); return *reinterpret_cast<const uint32_t*>(&h); }
  __device__ static float2 unpack(uint32_t u) { return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u)); }
};

// Eight consecutive elements as they lie in memory (half the registers of fp32 where they wait for something), and
// as fp32.  `wide`: the address is 16-byte aligned.
template <typename T> struct Raw8 { uint32_t w[8 * sizeof(T) / 4]; };
template <typename T>
__device__ __forceinline__ void load8(const T* p, bool wide, Raw8<T>& x) {
  if (wide) {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(x.w) / 16); ++i) *(reinterpret_cast<uint4*>(x.w) + i) = __ldg(reinterpret_cast<const uint4*>(p) + i);
  } else {
    T* e = reinterpret_cast<T*>(x.w);
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = p[i];
  }
}
template <typename T>
__device__ __forceinline__ void to_f(const Raw8<T>& x, float (&y)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      y[2 * i] = __uint_as_float(x.w[2 * i]);
      y[2 * i + 1] = __uint_as_float(x.w[2 * i + 1]);
    } else {
      const float2 f = Half2Of<T>::unpack(x.w[i]);
      y[2 * i] = f.x;
      y[2 * i + 1] = f.y;
    }
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {      // 16-byte aligned
  *reinterpret_cast<uint4*>(p) = make_uint4(Half2Of<T>::pack(x[0], x[1]), Half2Of<T>::pack(x[2], x[3]), Half2Of<T>::pack(x[4], x[5]),
                                            Half2Of<T>::pack(x[6], x[7]));
}
#endif

}  // namespace prima

// Beam selection: the best continuations of a request's beams over the vocabulary.
//
//   score(b, w) = cum[b] + (x[b][w] - m_b - log sum_v exp(x[b][v] - m_b)),   m_b = max_v x[b][v]
//
// The logits are read once.  A CTA holds a slice of one row in registers and leaves the slice's maximum, its sum of
// exponentials and its `keep` best logits; a second kernel joins the slices of a request.  Within a row the order of
// the scores is the order of the logits, so the slices can be cut down before the row's sum is known.
// Which of two near candidates of DIFFERENT beams is ahead depends on the last bits of the two sums, so everything
// behind a thread's own partial sum is in 64 bits.  Every sum has a fixed order that follows the index in the row, not
// the address: equal rows get equal bits, and their candidates tie exactly (the lower index wins).
// Rows that cannot contribute (finished beams, cum = -infinity) are not read.
#include <cfloat>
#include <cstdio>

#include "paged.cuh"

namespace prima {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxKeep = 64;

struct Best { float x; int32_t w; };                   // a logit and its word
struct SliceStat { double sum; float top; int32_t n; };

// (value, index) as one integer that orders by value, then by the lower index.  0 is below everything that is stored.
__device__ __forceinline__ unsigned long long key_of(float x, unsigned idx) {
  const unsigned u = __float_as_uint(x);
  const unsigned o = u & 0x80000000u ? ~u : u | 0x80000000u;
  return static_cast<unsigned long long>(o) << 32 | (0xffffffffu - idx);
}
__device__ __forceinline__ unsigned long long key_of(double x) {
  const unsigned long long u = __double_as_longlong(x);
  return u >> 63 ? ~u : u | 0x8000000000000000ull;
}

template <typename T> __device__ __forceinline__ float as_float(T x);
template <> __device__ __forceinline__ float as_float<float>(float x) { return x; }
template <> __device__ __forceinline__ float as_float<__half>(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float as_float<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }

// NaN and -infinity: no candidate; +infinity: the largest finite value.
__device__ __forceinline__ float usable(float x) { return fminf(fmaxf(x, -INFINITY), FLT_MAX); }

// The kth largest (k = 1..) of the threads' keys: every thread sorts with its warp, then thread (w, l) counts how many
// keys of the other warps are above its own by a binary search in their sorted lists.
__device__ __forceinline__ unsigned long long kth_of_block(unsigned long long key, int k, unsigned long long* s_keys, unsigned long long* s_kth) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
    for (int step = size >> 1; step > 0; step >>= 1) {
      const unsigned long long o = __shfl_xor_sync(0xffffffffu, key, step);
      const bool keep_large = ((lane & step) == 0) == ((lane & size) == 0);      // descending overall
      key = keep_large == (key > o) ? key : o;
    }
  s_keys[threadIdx.x] = key;
  if (threadIdx.x == 0) *s_kth = 0;
  __syncthreads();
  if (key != 0) {
    int rank = lane;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
      if (w == warp) continue;
      int above = 0;
#pragma unroll
      for (int step = 16; step > 0; step >>= 1)
        if (s_keys[32 * w + above + step - 1] > key) above += step;
      if (above == 31 && s_keys[32 * w + 31] > key) above = 32;
      rank += above;
    }
    if (rank == k - 1) *s_kth = key;      // keys that are not 0 are all different
  }
  __syncthreads();
  return *s_kth;                          // 0: fewer than k keys
}

// E logits per thread: a slice of kThreads * E words of one row.
template <typename T, int E>
__global__ void __launch_bounds__(kThreads) beam_slice_kernel(const T* __restrict__ logits, int64_t row_stride, int vocab, const float* __restrict__ cum,
                                                              const uint8_t* __restrict__ finished, int keep, int n_slices, bool wide,
                                                              SliceStat* __restrict__ stat, Best* __restrict__ best) {
  constexpr int kVec = 16 / sizeof(T);
  __shared__ unsigned long long s_keys[kThreads], s_kth;
  __shared__ float s_top[kThreads / 32];
  __shared__ double s_sum[kThreads / 32];
  __shared__ int s_n;
  extern __shared__ unsigned long long s_found[];      // keep * E
  pdl_trigger();
  pdl_wait();
  const int row = blockIdx.y, slice = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const float c = __ldg(cum + row);
  if ((finished && finished[row]) || !(c > -INFINITY)) return;
  const T* x0 = logits + row * row_stride;
  const int first = slice * kThreads * E;
  float x[E];
  // element i of a thread is word first + (i / kVec) * kThreads * kVec + tid * kVec + i % kVec
#pragma unroll
  for (int i = 0; i < E; i += kVec) {
    const int w = first + i * kThreads + tid * kVec;
    if (wide && w + kVec <= vocab) {
      const uint4 u = __ldcs(reinterpret_cast<const uint4*>(x0 + w));
      const T* e = reinterpret_cast<const T*>(&u);
#pragma unroll
      for (int j = 0; j < kVec; ++j) x[i + j] = usable(as_float<T>(e[j]));
    } else {
#pragma unroll
      for (int j = 0; j < kVec; ++j) x[i + j] = w + j < vocab ? usable(as_float<T>(x0[w + j])) : -INFINITY;
    }
  }
  float top = x[0];
  int at = 0;
#pragma unroll
  for (int i = 1; i < E; ++i)
    if (x[i] > top) {
      top = x[i];
      at = i;
    }
  auto word = [&](int i) { return first + (i / kVec) * kThreads * kVec + tid * kVec + i % kVec; };
  const unsigned long long mine = top > -INFINITY ? key_of(top, word(at)) : 0ull;
  float m = top;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lane == 0) s_top[warp] = m;
  if (tid == 0) s_n = 0;
  const unsigned long long kth = kth_of_block(mine, keep, s_keys, &s_kth);
  m = s_top[0];
#pragma unroll
  for (int w = 1; w < kThreads / 32; ++w) m = fmaxf(m, s_top[w]);
  // Sum of exp(x - m): the difference first (exact for the large terms), then one ex2 (relative error 2^-22).
  float part = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const float d = x[i] - m;
    part += d > -INFINITY ? exp2f(d * 1.4426950408889634f) : 0.f;
  }
  double sum = part;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) s_sum[warp] = sum;
  // At most `keep` threads have a best key that reaches the kth, so at most keep * E elements do.
  if (mine >= kth && mine != 0) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const unsigned long long k = key_of(x[i], word(i));
      if (x[i] > -INFINITY && k >= kth) s_found[atomicAdd(&s_n, 1)] = k;
    }
  }
  __syncthreads();
  const int n = s_n;
  const int64_t out = static_cast<int64_t>(row) * n_slices + slice;
  for (int i = tid; i < n; i += kThreads) {
    const unsigned long long k = s_found[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += s_found[j] > k;
    if (rank < keep) {
      const unsigned o = static_cast<unsigned>(k >> 32);
      best[out * keep + rank] = {__uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o), static_cast<int32_t>(0xffffffffu - static_cast<unsigned>(k))};
    }
  }
  if (tid == 0) {
    double total = 0;
    for (int w = 0; w < kThreads / 32; ++w) total += s_sum[w];
    stat[out] = {total, m, min(n, keep)};
  }
}

// One CTA per request joins the slices of its beams.
constexpr int kFound = 2048;
__global__ void __launch_bounds__(kThreads) beam_join_kernel(int n_beams, int vocab, const float* __restrict__ cum, const uint8_t* __restrict__ finished,
                                                             int end_token, int keep, int n_slices, const SliceStat* __restrict__ stat,
                                                             const Best* __restrict__ best, float* __restrict__ score, int32_t* __restrict__ parent,
                                                             int32_t* __restrict__ token) {
  __shared__ double s_top[kMaxKeep], s_log[kMaxKeep];      // of every beam: maximum (+infinity: no row was read), log of the sum
  __shared__ unsigned long long s_keys[kThreads], s_kth, s_best[kThreads / 32];
  __shared__ double s_score[kFound];
  __shared__ int s_at[kFound], s_n;
  __shared__ int s_best_at[kThreads / 32];
  pdl_trigger();
  pdl_wait();
  const int req = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row0 = req * n_beams;
  for (int b = warp; b < n_beams; b += kThreads / 32) {
    const float c = __ldg(cum + row0 + b);
    double top = INFINITY, sum = 0;
    if (!(finished && finished[row0 + b]) && c > -INFINITY) {
      const SliceStat* st = stat + static_cast<int64_t>(row0 + b) * n_slices;
      float m = -INFINITY;
      for (int i = lane; i < n_slices; i += 32) m = fmaxf(m, st[i].top);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      for (int i = lane; i < n_slices; i += 32)
        if (st[i].top > -INFINITY) sum += st[i].sum * exp(static_cast<double>(st[i].top) - static_cast<double>(m));
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (m > -INFINITY) top = m;
    }
    if (lane == 0) {
      s_top[b] = top;
      s_log[b] = log(sum);
    }
  }
  if (tid == 0) s_n = 0;
  __syncthreads();

  const int per_beam = n_slices * keep;
  const int n = n_beams * per_beam;
  // Candidate i: place i % keep of slice i / keep % n_slices of beam i / per_beam; a finished beam has its end token as
  // the candidate of place 0 of slice 0.  Returns whether there is one.
  auto candidate = [&](int i, double* sc, int* at) {
    const int b = i / per_beam, r = i - b * per_beam, sl = r / keep, place = r - sl * keep;
    const float c = __ldg(cum + row0 + b);
    if (!(c > -INFINITY)) return false;
    if (finished && finished[row0 + b]) {
      *sc = c;
      *at = b * vocab + end_token;
      return r == 0;
    }
    if (isinf(s_top[b])) return false;
    const int64_t s = static_cast<int64_t>(row0 + b) * n_slices + sl;
    if (place >= stat[s].n) return false;
    const Best e = best[s * keep + place];
    *sc = c + ((static_cast<double>(e.x) - s_top[b]) - s_log[b]);
    *at = b * vocab + e.w;
    return true;
  };
  // ordered by (score, lower index)
  auto ahead = [](double s, int a, double s2, int a2) { return s > s2 || (s == s2 && a < a2); };

  double my = -INFINITY;
  int my_at = 0x7fffffff;
  bool any = false;
  for (int i = tid; i < n; i += kThreads) {
    double sc;
    int at;
    if (candidate(i, &sc, &at) && (!any || ahead(sc, at, my, my_at))) {
      my = sc;
      my_at = at;
      any = true;
    }
  }
  // A bound that at least `keep` threads reach (the scores alone: ties may let a few more through).
  const unsigned long long mine = any ? key_of(my) : 0ull;
  const unsigned long long uniq = mine == 0 ? 0 : (mine & ~255ull) | (255 - tid);      // all different; 2^-44 coarser
  const unsigned long long kth = kth_of_block(uniq, keep, s_keys, &s_kth) & ~255ull;
  if (mine >= kth && any)
    for (int i = tid; i < n; i += kThreads) {
      double sc;
      int at;
      if (candidate(i, &sc, &at) && key_of(sc) >= kth) {
        const int place = atomicAdd(&s_n, 1);
        if (place < kFound) {
          s_score[place] = sc;
          s_at[place] = at;
        }
      }
    }
  __syncthreads();
  const int found = s_n;
  float* o_score = score + static_cast<int64_t>(req) * keep;
  int32_t* o_parent = parent + static_cast<int64_t>(req) * keep;
  int32_t* o_token = token + static_cast<int64_t>(req) * keep;
  auto put = [&](int place, double sc, int at) {
    const bool none = sc == -INFINITY;
    o_score[place] = static_cast<float>(sc);
    o_parent[place] = none ? 0 : at / vocab;
    o_token[place] = none ? -1 : at % vocab;
  };
  for (int i = found + tid; i < keep; i += kThreads) put(i, -INFINITY, 0);
  if (found <= kFound) {
    for (int i = tid; i < found; i += kThreads) {
      const double sc = s_score[i];
      const int at = s_at[i];
      int rank = 0;
      for (int j = 0; j < found; ++j) rank += ahead(s_score[j], s_at[j], sc, at);
      if (rank < keep) put(rank, sc, at);
    }
    return;
  }
  // More candidates near the bound than fit (thousands of equal scores): one after the other.
  double last = INFINITY;
  int last_at = -1;
  for (int place = 0; place < keep; ++place) {
    double bs = -INFINITY;
    int ba = 0x7fffffff;
    for (int i = tid; i < n; i += kThreads) {
      double sc;
      int at;
      if (candidate(i, &sc, &at) && (place == 0 || ahead(last, last_at, sc, at)) && ahead(sc, at, bs, ba)) {
        bs = sc;
        ba = at;
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const double s2 = __shfl_xor_sync(0xffffffffu, bs, o);
      const int a2 = __shfl_xor_sync(0xffffffffu, ba, o);
      if (ahead(s2, a2, bs, ba)) {
        bs = s2;
        ba = a2;
      }
    }
    __syncthreads();
    if (lane == 0) {
      s_best[warp] = __double_as_longlong(bs);
      s_best_at[warp] = ba;
    }
    __syncthreads();
    for (int w = 0; w < kThreads / 32; ++w) {
      const double s2 = __longlong_as_double(s_best[w]);
      if (ahead(s2, s_best_at[w], bs, ba)) {
        bs = s2;
        ba = s_best_at[w];
      }
    }
    if (tid == 0) put(place, bs, ba);
    last = bs;
    last_at = ba;
  }
}

// Words per thread: 32 where that still gives every SM a few CTAs, else 8, for the latency of small calls.
int words_per_thread(int64_t rows, int vocab) { return rows * ((vocab + 32 * kThreads - 1) / (32 * kThreads)) >= 4 * 148 ? 32 : 8; }
int slices_of(int64_t rows, int vocab) {
  const int w = words_per_thread(rows, vocab) * kThreads;
  return (vocab + w - 1) / w;
}

template <typename T>
cudaError_t launch_select(const void* logits, int n_req, int n_beams, int vocab, int64_t row_stride, const float* cum, const uint8_t* finished,
                          int end_token, int keep, float* score, int32_t* parent, int32_t* token, void* workspace, cudaStream_t st) {
  const int64_t rows = static_cast<int64_t>(n_req) * n_beams;
  const int n_slices = slices_of(rows, vocab), e = words_per_thread(rows, vocab);
  SliceStat* stat = static_cast<SliceStat*>(workspace);
  Best* best = reinterpret_cast<Best*>(stat + rows * n_slices);
  const bool wide = (reinterpret_cast<uintptr_t>(logits) & 15) == 0 && row_stride % (16 / static_cast<int64_t>(sizeof(T))) == 0;
  const dim3 grid(static_cast<unsigned>(n_slices), static_cast<unsigned>(rows));
  auto kernel = e == 32 ? beam_slice_kernel<T, 32> : beam_slice_kernel<T, 8>;
  cudaError_t err = launch_pdl(kernel, grid, dim3(kThreads), static_cast<size_t>(keep) * e * 8, st, static_cast<const T*>(logits), row_stride, vocab, cum, finished, keep,
                               n_slices, wide, stat, best);
  if (err != cudaSuccess) return err;
  return launch_pdl(beam_join_kernel, dim3(static_cast<unsigned>(n_req)), dim3(kThreads), 0, st, n_beams, vocab, cum, finished, end_token, keep, n_slices,
                    static_cast<const SliceStat*>(stat), static_cast<const Best*>(best), score, parent, token);
}

const char* select_error(int n_req, int n_beams, int vocab, int keep) {
  if (n_req < 1 || vocab < 1) return "n_req and vocab must be positive";
  if (n_beams < 1 || n_beams > kMaxKeep || keep < 1 || keep > kMaxKeep) return "n_beams and keep are 1..64";
  if (static_cast<int64_t>(n_beams) * vocab > 2147483647) return "n_beams * vocab reaches 2^31";
  if (static_cast<int64_t>(n_req) * n_beams > 65535) return "more than 65535 beams";
  return nullptr;
}

}  // namespace
}  // namespace prima

using namespace prima;

extern "C" {

int64_t prima_beam_select_workspace(int n_req, int n_beams, int vocab, int keep) {
  if (select_error(n_req, n_beams, vocab, keep)) return PRIMA_ERR_ARG;
  const int64_t rows = static_cast<int64_t>(n_req) * n_beams;
  const int64_t n = rows * slices_of(rows, vocab);
  return n * static_cast<int64_t>(sizeof(SliceStat)) + n * keep * static_cast<int64_t>(sizeof(Best));
}

int prima_beam_select(const void* logits, int dtype, int n_req, int n_beams, int vocab, int64_t row_stride, const float* cum,
                      const uint8_t* finished, int end_token, int keep, float* score, int32_t* parent, int32_t* token, void* workspace,
                      int64_t workspace_bytes, void* stream) {
  if (const char* bad = select_error(n_req, n_beams, vocab, keep)) {
    char msg[120];
    snprintf(msg, sizeof msg, "prima_beam_select: %s", bad);
    return call_fail(PRIMA_ERR_ARG, msg);
  }
  if (!logits || !cum || !score || !parent || !token || !workspace) return call_fail(PRIMA_ERR_ARG, "prima_beam_select: null argument");
  if (dtype != PRIMA_DT_F32 && dtype != PRIMA_DT_F16 && dtype != PRIMA_DT_BF16) return call_fail(PRIMA_ERR_ARG, "prima_beam_select: unknown dtype");
  if (row_stride < vocab) return call_fail(PRIMA_ERR_ARG, "prima_beam_select: row_stride is shorter than a row");
  if (finished && (end_token < 0 || end_token >= vocab)) return call_fail(PRIMA_ERR_ARG, "prima_beam_select: end_token outside the vocabulary");
  if ((reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < prima_beam_select_workspace(n_req, n_beams, vocab, keep))
    return call_fail(PRIMA_ERR_ARG, "prima_beam_select: workspace too small or not 256-byte aligned");
  auto run = dtype == PRIMA_DT_F32 ? launch_select<float> : dtype == PRIMA_DT_F16 ? launch_select<__half> : launch_select<__nv_bfloat16>;
  const cudaError_t e = run(logits, n_req, n_beams, vocab, row_stride, cum, finished, end_token, keep, score, parent, token, workspace,
                            static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? PRIMA_OK : call_cuda_fail(e, "prima_beam_select");
}

}  // extern "C"
